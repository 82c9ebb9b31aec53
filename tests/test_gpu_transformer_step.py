"""The operators in a run, as a program uses them: one training step of a factorized Transformer block with experts, from its inputs
to the updated factors, against the same block in 64 bits."""
import pytest
import torch

import _ops
import paper_2103_03936_b200 as pf

pytestmark = pytest.mark.gpu
T, WIDTH, HEADS, DIM, RANK, EXPERTS, CHOICES, HIDDEN, CAPACITY = 160, 128, 4, 32, 32, 4, 2, 192, 72
BF16 = torch.bfloat16
# Relative errors of whole tensors.  fp32: the library's bound for a factorized layer, 1e-4 (layers add up 1e-6 each, and a
# softmax's gradient is a difference of terms a few times its size).  bf16: a value passes a dozen roundings of 2^-9 in the root mean
# square, 0.7 %, but max(0, .) passes or stops a gradient by the sign of such a value: of normal values those within
# 0.7 % of zero, 0.56 % of all, are in doubt and half of them take the wrong side, and a gradient that is whole or nothing in 0.28 % of its elements is
# off by the root of that, 5.3 %, before what does not pass the experts dilutes it.
TOLERANCE = {torch.float32: 1e-4, BF16: 6e-2}


def normal(shape, seed, scale=1.0):
    """bf16 values, for either type."""
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(BF16).cuda()


def close(got, want, what, tol):
    err = float((got.double() - want).norm() / want.norm())
    assert err <= tol, f"{what}: relative error {err:.3g}"


def parameters():
    s = lambda n: n ** -0.5  # noqa: E731
    return {"Uqkv": normal((3, WIDTH, RANK), 1, s(WIDTH)), "Vqkv": normal((3, WIDTH, RANK), 2, s(RANK)),
            "wq": (1 + normal((DIM,), 3, 0.2).float()).to(BF16), "wk": (1 + normal((DIM,), 4, 0.2).float()).to(BF16),
            "U1": normal((EXPERTS, WIDTH, RANK), 5, s(WIDTH)), "V1": normal((EXPERTS, HIDDEN, RANK), 6, s(RANK)),
            "U2": normal((EXPERTS, HIDDEN, RANK), 7, s(HIDDEN)), "V2": normal((EXPERTS, WIDTH, RANK), 8, s(RANK))}


def attention(q, k, v):
    """Causal attention, elementary operations only: [T, heads, dim] each."""
    logits = torch.einsum("thd,shd->hts", q, k) * DIM ** -0.5
    logits = logits.masked_fill(torch.ones(T, T, dtype=torch.bool, device=q.device).triu(1), float("-inf"))
    return torch.einsum("hts,shd->thd", logits.softmax(-1), v).reshape(T, WIDTH)


def reference(x, ids, weights, angle, p):
    """The block's output in 64 bits, differentiable."""
    qkv = torch.einsum("tk,gkr,gnr->gtn", x, p["Uqkv"], p["Vqkv"]).view(3, T, HEADS, DIM)
    q, k = (_ops.turn(z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-6) * p[w], angle, False) for z, w in ((qkv[0], "wq"), (qkv[1], "wk")))
    h = x + attention(q, k, qkv[2])
    slots = torch.tensor(_ops.sort(ids.tolist(), EXPERTS, CAPACITY)[0], device="cuda").view(T, CHOICES)
    out = torch.zeros_like(h)
    for e in range(EXPERTS):
        for j in range(CHOICES):
            t = ((ids[:, j] == e) & (slots[:, j] >= 0)).nonzero().flatten()
            z = torch.relu(h[t] @ p["U1"][e] @ p["V1"][e].T) @ p["U2"][e] @ p["V2"][e].T
            out = out.index_add(0, t, z * weights[t, j:j + 1])
    return h + out


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_a_training_step_of_a_block_with_experts(dtype):
    p = {n: t.to(dtype) for n, t in parameters().items()}
    x, dy = normal((T, WIDTH), 10).to(dtype), normal((T, WIDTH), 11).to(dtype)
    ids = torch.randint(0, EXPERTS, (T, CHOICES), generator=torch.Generator().manual_seed(12)).to(torch.int32).cuda()
    weights = torch.rand((T, CHOICES), generator=torch.Generator().manual_seed(13)).cuda()
    freq = (10000.0 ** (-torch.arange(DIM // 2, dtype=torch.float64) / (DIM // 2))).float().cuda()
    positions = (torch.arange(T) % 40 + 100000).cuda()

    # forward: projections, norm and rotation, attention, experts
    qkv, Tqkv = pf.pf_lowrank_linear_grouped_fwd(x, p["Uqkv"], p["Vqkv"], want_stash=True)
    q, k, v = (qkv[g].view(T, HEADS, DIM) for g in range(3))
    qr, kr = pf.pf_qk_norm_rope_fwd(q, k, p["wq"], p["wk"], freq, positions=positions)
    a_in = [t.detach().float().requires_grad_() for t in (qr, kr, v)]
    a = attention(*a_in)
    h = (x.float() + a).to(dtype).detach()
    slots, sources, counts, offsets = pf.pf_expert_sort(ids, EXPERTS, capacity=CAPACITY)
    xs = pf.pf_expert_dispatch_fwd(h, slots, sources).view(EXPERTS, CAPACITY, WIDTH)
    z, T1 = pf.pf_lowrank_linear_grouped_fwd(xs, p["U1"], p["V1"], want_stash=True)
    act = torch.relu(z)
    ys, T2 = pf.pf_lowrank_linear_grouped_fwd(act, p["U2"], p["V2"], want_stash=True)
    ys = ys.view(EXPERTS * CAPACITY, WIDTH)
    y = h + pf.pf_expert_combine_fwd(ys, slots, weights)

    # backward
    grads = {}
    dys, dweights = pf.pf_expert_combine_bwd(ys, slots, sources, weights, dy)
    dact, grads["U2"], grads["V2"] = pf.pf_lowrank_linear_grouped_bwd(act, p["U2"], p["V2"], dys.view(EXPERTS, CAPACITY, WIDTH), T_stash=T2)
    dz = dact.view(EXPERTS * CAPACITY, HIDDEN)
    pf.pf_bias_act_bwd(act.view(EXPERTS * CAPACITY, HIDDEN), dz, want_dbias=False)
    dxs, grads["U1"], grads["V1"] = pf.pf_lowrank_linear_grouped_bwd(xs, p["U1"], p["V1"], dz.view(EXPERTS, CAPACITY, HIDDEN), T_stash=T1)
    dh = dy + pf.pf_expert_dispatch_bwd(dxs.view(EXPERTS * CAPACITY, WIDTH), slots)
    dqr, dkr, dv = torch.autograd.grad(a, a_in, dh.float())
    dq, dk, grads["wq"], grads["wk"] = pf.pf_qk_norm_rope_bwd(q, k, p["wq"], p["wk"], freq, dqr.to(dtype).contiguous(), dkr.to(dtype).contiguous(),
                                                             positions=positions)
    dqkv = torch.stack([dq.view(T, WIDTH), dk.view(T, WIDTH), dv.to(dtype).reshape(T, WIDTH)])
    dx, grads["Uqkv"], grads["Vqkv"] = pf.pf_lowrank_linear_grouped_bwd(x, p["Uqkv"], p["Vqkv"], dqkv, T_stash=Tqkv)
    dx = dx + dh

    # the same in 64 bits
    assert int((slots < 0).sum()) > 0      # some assignments were dropped
    d = {n: t.double().requires_grad_() for n, t in (p | {"x": x, "weights": weights}).items()}
    out = reference(d["x"], ids, d["weights"], _ops.angles(positions, freq), d)
    close(y, out.detach(), "y", TOLERANCE[dtype])
    wanted = torch.autograd.grad(out, list(d.values()), dy.double())
    for (name, want) in zip(d, wanted):
        close({"x": dx, "weights": dweights}[name] if name in ("x", "weights") else grads[name], want, "gradient of " + name, TOLERANCE[dtype])

    # the update, from the flat buffer that was exchanged
    names = list(p)
    flat, offs = pf.pf_pack_factor_grads([grads[n] for n in names])
    views = [flat[offs[i]:offs[i + 1]].view(p[n].shape) for i, n in enumerate(names)]
    hyper = dict(lr=1e-3, betas=(0.9, 0.98), eps=1e-8, weight_decay=0.01, step=1, grad_scale=0.25)
    zeros = lambda dt: [torch.zeros(p[n].shape, dtype=dt, device="cuda") for n in names]  # noqa: E731
    masters = [p[n].float() for n in names]
    before = [t.clone() for t in masters]
    state, params = {"m": zeros(torch.float32), "v": zeros(torch.float32)}, [p[n].clone() for n in names]
    pf.pf_adamw_step(params, views, **state, masters=masters if dtype == BF16 else None, **hyper)
    eight = {"m": zeros(torch.float8_e4m3fn), "v": zeros(torch.float8_e5m2)}
    eight |= {s: [torch.zeros(-(-t.numel() // 256), device="cuda") for t in params] for s in ("m_scales", "v_scales")}
    other = [p[n].clone() for n in names]
    pf.pf_adamw_step(other, views, **eight, **hyper, seed=3)
    for i, n in enumerate(names):
        want, slack = _ops.adamw(before[i], grads[n], torch.zeros_like(before[i]), torch.zeros_like(before[i]), **hyper)[:2]
        _ops.close(params[i], want, slack, n)
        if dtype == BF16:
            _ops.close(masters[i], want, slack, "master of " + n)
        _ops.close(other[i], want, slack, n + " with states in 8 bits")
    assert pf.pf_last_device_status() == 0
