"""GPU parity of the AdamW step: fp32 states against a plain form in 64 bits, 8-bit states bit for bit against their definition."""
import pytest
import torch

import _ops
import paper_2103_03936_b200 as pf

pytestmark = pytest.mark.gpu
H = dict(lr=1e-2, betas=(0.9, 0.98), eps=1e-8, weight_decay=0.1, step=5, grad_scale=0.5)
SIZES = [1, 7, 255, 256, 257, 0, 4096, 4103, 10001, 2, 512 * 128]
KINDS = [(torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, False), (torch.bfloat16, torch.bfloat16, False),
         (torch.bfloat16, torch.float32, False), (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, True)]


def views(sizes, dtype, gap, shift=0):
    """Tensors of their own (gap "own"), or inside one sentinel-filled buffer, the first `shift` elements from its start, `gap` elements
    between them: (tensors, check that nothing else was written)."""
    if gap == "own":
        return [torch.empty(n, dtype=dtype, device="cuda") for n in sizes], lambda: None
    buf = torch.full((sum(sizes) + len(sizes) * gap + shift + 64,), 3.0, device="cuda").to(dtype)
    before, out, at, used = buf.view(torch.uint8).clone(), [], shift, torch.zeros(buf.numel(), dtype=torch.bool, device="cuda")
    for n in sizes:
        out.append(buf[at:at + n])
        used[at:at + n] = True
        at += n + gap

    def check():
        now = buf.view(torch.uint8).view(buf.numel(), -1)
        assert (now == before.view(buf.numel(), -1))[~used].all(), "written outside the tensors"
    return out, check


def lists(sizes, pdt, gdt, masters, gap, shift, seed):
    g = torch.Generator().manual_seed(seed)
    data = [(torch.randn(n, generator=g) * 0.05, torch.randn(n, generator=g) * 1e-3, torch.randn(n, generator=g) * 1e-3,
             torch.rand(n, generator=g) * 1e-6) for n in sizes]
    t, checks = {}, []
    for name, dt, of in (("params", pdt, 0), ("grads", gdt, 1), ("m", torch.float32, 2), ("v", torch.float32, 3)) + ((("masters", torch.float32, 0),) if masters else ()):
        t[name], check = views(sizes, dt, gap, shift)
        checks.append(check)
        for x, d in zip(t[name], data):
            x.copy_(d[of])
    return t, checks


def clones(t):
    return {n: [x.clone() for x in l] for n, l in t.items()}


@pytest.mark.parametrize("pdt,gdt,masters", KINDS)
@pytest.mark.parametrize("gap,shift", [("own", 0), (0, 0), (1, 3), (8, 8)])
def test_fp32_states(pdt, gdt, masters, gap, shift):
    t, checks = lists(SIZES, pdt, gdt, masters, gap, shift, 1)
    old = clones(t)
    assert pf.pf_adamw_step(**t, **H) is None
    for check in checks:
        check()
    for i in range(len(SIZES)):
        p0 = old["masters" if masters else "params"][i]
        p, p_slack, m, m_slack, v, v_slack = _ops.adamw(p0, old["grads"][i], old["m"][i], old["v"][i], **H)
        _ops.close(t["params"][i], p, p_slack, f"params {i}")
        if masters:
            _ops.close(t["masters"][i], p, p_slack, f"masters {i}")
            assert torch.equal(t["params"][i], t["masters"][i].bfloat16())
        _ops.close(t["m"][i], m, m_slack, f"m {i}")
        _ops.close(t["v"][i], v, v_slack, f"v {i}")
        assert torch.equal(t["grads"][i], old["grads"][i])


def test_arrays_of_different_alignment():
    """Arrays that never come to 16-byte boundaries together."""
    t, checks = lists(SIZES, torch.float32, torch.float32, False, 0, 0, 3)
    moved, check = views(SIZES, torch.float32, 0, 1)
    for a, b in zip(moved, t["m"]):
        a.copy_(b)
    t["m"] = moved
    old = clones(t)
    pf.pf_adamw_step(**t, **H)
    for c in checks + [check]:
        c()
    for i in range(len(SIZES)):
        p, p_slack, m, m_slack, v, v_slack = _ops.adamw(old["params"][i], old["grads"][i], old["m"][i], old["v"][i], **H)
        _ops.close(t["params"][i], p, p_slack, f"params {i}")
        _ops.close(t["m"][i], m, m_slack, f"m {i}")
        _ops.close(t["v"][i], v, v_slack, f"v {i}")


def test_many_tensors_span_several_launches():
    sizes = [int(n) for n in torch.randint(0, 700, (700,), generator=torch.Generator().manual_seed(0))]
    t, checks = lists(sizes, torch.float32, torch.float32, False, 0, 0, 2)
    old, before = clones(t), pf.pf_launch_count()
    pf.pf_adamw_step(**t, **H)
    assert pf.pf_launch_count() - before == 2
    checks[0]()
    for name in ("params", "m", "v"):
        got = torch.cat(t[name])
        want = _ops.adamw(*(torch.cat(old[n]) for n in ("params", "grads", "m", "v")), **H)
        at = {"params": 0, "m": 2, "v": 4}[name]
        _ops.close(got, want[at], want[at + 1], name)


def state8(sizes, pdt, gdt, masters, gap, shift, seed):
    t, checks = lists(sizes, pdt, gdt, masters, gap, shift, seed)
    for name, dt in (("m", torch.float8_e4m3fn), ("v", torch.float8_e5m2)):
        values = t[name]
        t[name], check = views(sizes, dt, gap, shift)
        checks.append(check)
        t[name + "_scales"], check = views([-(-n // 256) for n in sizes], torch.float32, 1)
        checks.append(check)
        for i, x in enumerate(values):
            codes, scales = _ops.encode(x.cpu(), torch.zeros(x.numel(), dtype=torch.long), name == "m")
            t[name][i].copy_(codes)
            t[name + "_scales"][i].copy_(scales)
    return t, checks


def check8(t, old, sizes, masters, h, seed):
    raw = lambda x: x.cpu().view(torch.uint8)  # noqa: E731
    for i, n in enumerate(sizes):
        m0, v0 = (_ops.decode(old[s][i].cpu(), old[s + "_scales"][i].cpu()) for s in "mv")
        g = old["grads"][i].cpu()
        m, v = _ops.moments32(g, m0, v0, h["betas"], h["grad_scale"])
        bits = _ops.noise(n, seed, i)
        for s, value, half in (("m", m, bits & 0xFFFF), ("v", v, bits >> 16)):
            codes, scales = _ops.encode(value, half, s == "m")
            assert torch.equal(raw(t[s][i]), raw(codes)), f"codes of {s} {i}"
            assert torch.equal(t[s + "_scales"][i].cpu(), scales), f"scales of {s} {i}"
        p0 = old["masters" if masters else "params"][i].cpu()
        p, slack = _ops.adamw(p0, g, m0, v0, **h)[:2]
        _ops.close(t["params"][i].cpu(), p, slack, f"params {i}")
        if masters:
            _ops.close(t["masters"][i].cpu(), p, slack, f"masters {i}")


@pytest.mark.parametrize("pdt,gdt,masters", KINDS)
@pytest.mark.parametrize("gap,shift", [("own", 0), (0, 0), (3, 5)])
def test_8bit_states(pdt, gdt, masters, gap, shift):
    t, checks = state8(SIZES, pdt, gdt, masters, gap, shift, 1)
    for step, seed in ((5, 0), (6, 0xFFFFFFFF)):
        old, h = clones(t), H | {"step": step}
        pf.pf_adamw_step(**t, **h, seed=seed)
        for check in checks:
            check()
        check8(t, old, SIZES, masters, h, seed)


def test_8bit_states_from_zero():
    """The first step from zeroed codes and scales, in a list that spans several launches (a tensor's place counts in the whole list)."""
    sizes = [300 + i % 7 for i in range(500)]
    t, _ = state8(sizes, torch.float32, torch.float32, False, "own", 0, 3)
    for name in ("m", "v", "m_scales", "v_scales"):
        for s in t[name]:
            s.view(torch.uint8).zero_()
    old = clones(t)
    pf.pf_adamw_step(**t, **(H | {"step": 1}), seed=9)
    check8(t, old, sizes, False, H | {"step": 1}, 9)


def test_8bit_states_of_odd_gradients():
    """Blocks of zeros, of one value among zeros, of a wide range, of subnormal and huge numbers."""
    sizes = [256 * 8]
    t, _ = state8(sizes, torch.float32, torch.float32, False, "own", 0, 3)
    for name in ("m", "v", "m_scales", "v_scales"):
        t[name][0].view(torch.uint8).zero_()
    g = t["grads"][0].view(8, 256)
    g[0] = 0
    g[1] = 0
    g[1, 77] = 1e-3
    g[2] = torch.logspace(-30, 3, 256, device="cuda")
    g[3] = 1e-41
    g[4] = -1e18
    g[5, ::2] = 0
    g[6] = 1e-22
    old = clones(t)
    pf.pf_adamw_step(**t, **H, seed=5)
    check8(t, old, sizes, False, H, 5)


def test_8bit_states_at_the_top_of_fp32():
    """Values of the highest binade are rounded up to the code of 2^128, and are not infinite; what follows from the codes is finite.

    beta = 0 makes m the gradient and v its square: the first four blocks overflow v in fp32, the others have v near its end."""
    sizes = [256 * 8 + 100]
    t, _ = state8(sizes, torch.float32, torch.float32, False, "own", 0, 3)
    for name in ("m", "v", "m_scales", "v_scales"):
        t[name][0].view(torch.uint8).zero_()
    g = t["grads"][0]
    g[:1024] = 3.38e38
    g[256:512:3] *= -1
    g[512:1024:5] = -1e30
    g[1024:] = 1.842e19
    g[1100::7] = -1.7e19
    g[2048:2060] = 1e10
    h = H | {"betas": (0.0, 0.0), "step": 1, "grad_scale": 1.0}
    old = t["grads"][0].cpu()
    pf.pf_adamw_step(**t, **h, seed=5)
    m, v = _ops.moments32(old, torch.zeros(sizes[0]), torch.zeros(sizes[0]), h["betas"])
    bits = _ops.noise(sizes[0], 5, 0)
    for s, value, half in (("m", m, bits & 0xFFFF), ("v", v, bits >> 16)):
        codes, scales = _ops.encode(value, half, s == "m")
        assert torch.equal(t[s][0].cpu().view(torch.uint8), codes.view(torch.uint8)), s
        assert torch.equal(t[s + "_scales"][0].cpu(), scales), s
    assert (t["m"][0][:256].float() == 256).sum() > 100 and (t["v"][0][1024:].float() == 2.0 ** 15).sum() > 100
    t["grads"][0].zero_()
    pf.pf_adamw_step(**t, **H, seed=6)
    assert torch.isfinite(t["m"][0].float()).all() and torch.isfinite(t["v"][0][1024:].float()).all()


def test_what_is_not_finite_stays_where_it_is():
    for eight in (False, True):
        make = state8 if eight else lists
        t, _ = make([1000], torch.float32, torch.float32, False, "own", 0, 4)
        same, _ = make([1000], torch.float32, torch.float32, False, "own", 0, 4)
        where = torch.tensor([3, 300, 301, 999], device="cuda")
        t["grads"][0][where] = torch.tensor([float("nan"), float("inf"), -float("inf"), float("nan")], device="cuda")
        same["grads"][0][where] = 0
        if eight:
            for u in (t, same):         # not the largest of their blocks, so the scales agree
                u["m"][0].view(torch.uint8)[where] = 0
                u["v"][0].view(torch.uint8)[where] = 0
        for u in (t, same):
            pf.pf_adamw_step(**u, **H, seed=1)
        fine = torch.ones(1000, dtype=torch.bool, device="cuda")
        fine[where] = False
        for name in ("params", "m", "v"):
            a, b = t[name][0].float(), same[name][0].float()
            assert torch.equal(a[fine], b[fine]), name
            assert not torch.isfinite(a[~fine]).any(), name


def test_captured_and_replayed():
    """A step in a CUDA graph whose learning rate, corrections, scale and seed come from a device tensor."""
    for eight in (False, True):
        make = state8 if eight else lists
        t, _ = make([5000, 77], torch.bfloat16, torch.bfloat16, True, "own", 0, 5)
        u = clones(t)
        scalars = torch.empty(5, device="cuda")
        fixed = dict(betas=(0.9, 0.98), eps=1e-8, weight_decay=0.1)
        first = dict(lr=1e-2, step=3, grad_scale=0.5, seed=4)
        scalars.copy_(pf.pf_adamw_scalars(betas=(0.9, 0.98), **first))
        side = clones(t)
        pf.pf_adamw_step(**side, **fixed, scalars=scalars)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pf.pf_adamw_step(**t, **fixed, scalars=scalars)
        for step in (3, 4):
            change = first | {"step": step, "lr": 1e-2 / step, "seed": 4 + step}
            scalars.copy_(pf.pf_adamw_scalars(betas=(0.9, 0.98), **change))
            graph.replay()
            pf.pf_adamw_step(**u, **fixed, **change)
            for name in u:
                for a, b in zip(t[name], u[name]):
                    if name == "masters":       # corrections rounded to fp32 and again as reciprocals: 2^-22 of an update of at most ~ 10 lr
                        assert ((a - b).abs() <= 2.0 ** -22 * (b.abs() + change["lr"] * 10)).all()
                        b.copy_(a)
                    elif name == "params":      # one step of bf16 where the masters straddle a border
                        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs()).all()
                    else:
                        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name


def test_prepared_and_on_another_stream():
    t, _ = lists([3000, 5], torch.float32, torch.float32, False, "own", 0, 6)
    u = clones(t)
    call, none = pf.pf_adamw_step(**t, **H, prepare=True)
    assert none is None
    call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pf.pf_adamw_step(**u, **H, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for name in t:
        assert all(torch.equal(a, b) for a, b in zip(t[name], u[name]))


def test_a_tensor_beyond_32_bits():
    """The last elements of a tensor of more than 2^31 take the same step as by themselves."""
    n, tail = (1 << 31) + 77, 5000
    t = {"params": torch.zeros(n, dtype=torch.bfloat16, device="cuda"), "grads": torch.zeros(n, dtype=torch.bfloat16, device="cuda"),
         "m": torch.zeros(n, device="cuda"), "v": torch.zeros(n, device="cuda")}
    small, _ = lists([tail], torch.bfloat16, torch.bfloat16, False, "own", 0, 7)
    for name in t:
        t[name][-tail:] = small[name][0]
    pf.pf_adamw_step(**{k: [x] for k, x in t.items()}, **H)
    pf.pf_adamw_step(**small, **H)
    for name in t:
        assert torch.equal(t[name][-tail:], small[name][0]), name
        assert (t[name][:-tail] == 0).all()


def test_two_lists_at_once():
    """Steps of two lists on two streams: nothing is shared."""
    a, _ = lists([50000, 333], torch.float32, torch.float32, False, "own", 0, 8)
    b, _ = lists([40000, 222], torch.float32, torch.float32, False, "own", 0, 9)
    want_a, want_b = clones(a), clones(b)
    for _ in range(3):
        pf.pf_adamw_step(**want_a, **H)
        pf.pf_adamw_step(**want_b, **H)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        pf.pf_adamw_step(**a, **H)
        pf.pf_adamw_step(**b, **H, stream=side)
    torch.cuda.synchronize()
    for t, w in ((a, want_a), (b, want_b)):
        for name in t:
            assert all(torch.equal(x, y) for x, y in zip(t[name], w[name]))


def test_refusals():
    p = [torch.zeros(10, device="cuda"), torch.zeros(300, device="cuda")]
    z = lambda dt=torch.float32: [torch.zeros(10, dtype=dt, device="cuda"), torch.zeros(300, dtype=dt, device="cuda")]  # noqa: E731
    s = lambda a, b: [torch.zeros(a, device="cuda"), torch.zeros(b, device="cuda")]  # noqa: E731
    e4, e5 = z(torch.float8_e4m3fn), z(torch.float8_e5m2)
    for args, more in (((p, z()[:1], z(), z()), {}), ((p, z(), [z()[0]] * 2, z()), {}), ((p, z(), z(), z(torch.bfloat16)), {}),
                       ((p, [z()[0], z(torch.bfloat16)[1]], z(), z()), {}), ((p, z(), z(), z()), {"masters": z()}),
                       ((p, z(), e4, e5), {}), ((p, z(), e4, e5), {"m_scales": s(1, 2)}), ((p, z(), e4, e4), {"m_scales": s(1, 2), "v_scales": s(1, 2)}),
                       ((p, z(), e4, e5), {"m_scales": s(1, 1), "v_scales": s(1, 2)}), ((p, z(), z(), z()), {"m_scales": s(1, 2), "v_scales": s(1, 2)}),
                       (([p[0], p[1][::3]], [z()[0], z()[1][:100]], [z()[0], z()[1][:100]], [z()[0], z()[1][:100]]), {}),
                       ((p, [t.cpu() for t in z()], z(), z()), {}), ((p, z(), z(), z()), {"seed": -1}), ((p, z(), z(), z()), {"seed": 1 << 32}),
                       ((p, z(), z(), z()), {"scalars": torch.zeros(4, device="cuda")}), ((p, z(), z(), z()), {"scalars": torch.zeros(5)}),
                       ((p, z(), z(), None), {})):
        with pytest.raises(ValueError):
            pf.pf_adamw_step(*args, **more)
    with pytest.raises(TypeError):
        pf.pf_adamw_step([t.half() for t in p], z(), z(), z())
    with pytest.raises(TypeError):
        pf.pf_adamw_step(p, [t.half() for t in z()], z(), z())
    for more in ({"step": 0}, {"betas": (1.0, 0.9)}, {"eps": -1.0}, {"lr": float("nan")}):
        with pytest.raises(pf.PfError) as e:
            pf.pf_adamw_step(p, z(), z(), z(), **more)
        assert e.value.status == 1
    assert all((t == 0).all() for t in p)


@pytest.mark.parametrize("gdt,masters", [(torch.bfloat16, False), (torch.float32, False), (torch.bfloat16, True)])
def test_8bit_states_of_a_network(gdt, masters):
    """Lists of more than 16 blocks for each SM, whose blocks of bf16 parameters take two pieces a thread: whole ones, ragged ones and odd tensors."""
    sizes = [3_000_064, 2049, 0, 1_900_001, 256 * 16, 300, 200_000]
    t, checks = state8(sizes, torch.bfloat16, gdt, masters, "own", 0, 11)
    old = clones(t)
    pf.pf_adamw_step(**t, **H, seed=21)
    for check in checks:
        check()
    check8(t, old, sizes, masters, H, 21)


def test_8bit_states_step_after_step():
    """Sixty steps from zero, each from what the last one left, bit for bit; gradients of a block from 1 down to 2^-20."""
    sizes = [256 * 6, 511]
    t, _ = state8(sizes, torch.float32, torch.float32, False, "own", 0, 12)
    for name in ("m", "v", "m_scales", "v_scales"):
        for s in t[name]:
            s.view(torch.uint8).zero_()
    g = torch.Generator().manual_seed(12)
    sizes_of = [2.0 ** (-20 * torch.rand(n, generator=g)) for n in sizes]
    for step in range(1, 61):
        for x, s in zip(t["grads"], sizes_of):
            x.copy_(s * (0.5 + torch.rand(s.shape, generator=g)))
        old, h = clones(t), H | {"step": step}
        pf.pf_adamw_step(**t, **h, seed=step)
        check8(t, old, sizes, False, h, step)


def test_8bit_states_of_a_tensor_beyond_32_bits():
    """The last elements of a tensor of more than 2^32, on either side of that place: codes, scales and random bits by their definition."""
    border, tail, n = 1 << 32, 512, (1 << 32) + 3000
    first = border - tail
    t = {"params": torch.zeros(n, dtype=torch.bfloat16, device="cuda"), "grads": torch.zeros(n, dtype=torch.bfloat16, device="cuda"),
         "m": torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn), "v": torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e5m2),
         "m_scales": torch.zeros(-(-n // 256), device="cuda"), "v_scales": torch.zeros(-(-n // 256), device="cuda")}
    small, _ = state8([n - first], torch.bfloat16, torch.bfloat16, False, "own", 0, 13)
    for name in t:
        (t[name][first // 256:] if "scales" in name else t[name][first:]).copy_(small[name][0])
    pf.pf_adamw_step(**{k: [x] for k, x in t.items()}, **H, seed=31)
    m0, v0 = (_ops.decode(small[s][0].cpu(), small[s + "_scales"][0].cpu()) for s in "mv")
    m, v = _ops.moments32(small["grads"][0].cpu(), m0, v0, H["betas"], H["grad_scale"])
    bits = torch.cat([_ops.noise(tail, 31, 0, first), _ops.noise(n - border, 31, 0, border)])
    for s, value, half in (("m", m, bits & 0xFFFF), ("v", v, bits >> 16)):
        codes, scales = _ops.encode(value, half, s == "m")
        assert torch.equal(t[s][first:].cpu().view(torch.uint8), codes.view(torch.uint8)), s
        assert torch.equal(t[s + "_scales"][first // 256:].cpu(), scales), s
    p, slack = _ops.adamw(small["params"][0].cpu(), small["grads"][0].cpu(), m0, v0, **H)[:2]
    _ops.close(t["params"][first:].cpu(), p, slack, "params")
    assert (t["params"][:first] == 0).all()
