"""GPU parity of gated factorized layers and their gradients against a plain form in 64 bits."""
import pytest
import torch

import _more_ops as ref
import paper_2103_03936_b200 as pf
from _gpu import Scratch
from _more_ops import Rows, normal
from _ops import close

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
DT = [BF16, F32]
ACTS = {"silu": pf.PF_GATE_SILU, "gelu": pf.PF_GATE_GELU, "sigmoid": pf.PF_GATE_SIGMOID, "relu": pf.PF_GATE_RELU}
# Relative errors of whole gradients.  bf16: dZ and dZ V are rounded on the way and the result once more, each 2^-9 in the root mean square or less: 2^-8.2 together,
# and a third for what their sums may cancel.  fp32: the library's bound for a layer.
GRAD = {BF16: 1e-2, F32: 1e-4}


def pairs(rows, cols, dtype, seed, scale, layout="plain"):
    """[2, rows, cols], with gaps or at odd places."""
    t = normal((2, rows, cols), dtype, seed, scale)
    if layout == "plain":
        return t
    ld, shift = (cols + 24, 0) if layout == "padded" else (cols + 3, 1)
    gs = rows * ld + (40 if layout == "padded" else 5)
    out = torch.full((2 * gs + 64,), -7.0, dtype=dtype, device="cuda").as_strided((2, rows, cols), (gs, ld, 1), shift)
    out.copy_(t)
    return out


def near(got, want, tol, what):
    norm = float(want.norm())
    err = float((got.double() - want).norm()) / (norm or 1.0)
    assert err <= tol, f"{what}: relative error {err:.3g}"


def check(m, k, n, r, dtype, act="silu", *, bias=False, stash=True, layout="plain", need_dX=True, seed=1):
    how = {"plain": lambda c: {}, "padded": lambda c: {"ld": c + 24}, "odd": lambda c: {"ld": c + 3, "shift": 1}}[layout]
    x = Rows(m, k, dtype, **how(k)).fill(normal((m, k), dtype, seed))
    U, V = pairs(k, r, dtype, seed + 1, k ** -0.5, layout), pairs(n, r, dtype, seed + 2, 1.5 * r ** -0.5, layout)
    b = normal((2, n), dtype, seed + 3, 0.5) if bias else None
    y, dt = Rows(m, n, dtype, **how(n)), pf.PF_BF16 if dtype == BF16 else pf.PF_F32
    T = pairs(m, r, dtype, 0, 0.0, layout) if stash else None
    ws = Scratch(pf.pf_lowrank_linear_gated_workspace(m, k, n, r, dt, False))
    pf.pf_lowrank_linear_gated_fwd(x.t, U, V, bias=b, act=ACTS[act], y=y.t, T_stash=T, workspace=ws.t)
    ws.check()
    y.check()
    exact_T = x.t.double() @ U.double()
    if stash:
        close(T, exact_T, 2.0 ** -18 * (x.t.double().abs() @ U.double().abs()), "T")
    T_used = T if stash else pf.pf_lowrank_linear_gated_fwd(x.t, U, V, bias=b, act=ACTS[act], want_stash=True)[1]
    want, slack = ref.gated(T_used, V, b, act)
    tight = dtype == F32 or not (layout == "odd" and n % 8 == 0) and not (layout == "odd" and (k % 8 == 0 or r % 8 == 0))
    if tight:
        close(y.t, want, slack, "y")
    else:      # (g and u were rounded as well)
        near(y.t, want, 1e-2, "y")
    # backward
    dy, dX = Rows(m, n, dtype, **how(n)).fill(normal((m, n), dtype, seed + 4)), Rows(m, k, dtype, **how(k))
    dU, dV = pairs(k, r, dtype, 0, 0.0, layout), pairs(n, r, dtype, 0, 0.0, layout)
    ws = Scratch(pf.pf_lowrank_linear_gated_workspace(m, k, n, r, dt, True))
    got = pf.pf_lowrank_linear_gated_bwd(x.t, U, V, dy.t, bias=b, act=ACTS[act], T_stash=T, need_dX=need_dX, dX=dX.t if need_dX else None, dU=dU, dV=dV,
                                         workspace=ws.t)
    ws.check()
    # (from T as it was rounded, which decides on which side of zero a gate's argument lies)
    z = (T_used.double() @ V.double().transpose(1, 2) + (b.double()[:, None] if bias else 0.0)).requires_grad_()
    dZ = torch.autograd.grad(ref.act(z[0], act) * z[1], z, dy.t.double())[0]
    G = dZ @ V.double()
    wanted = [(G @ U.double().transpose(1, 2)).sum(0), x.t.double().T @ G, dZ.transpose(1, 2) @ T_used.double(), dZ.sum(1)]
    if need_dX:
        dX.check()
        near(dX.t, wanted[0], GRAD[dtype], "dX")
    else:
        assert got[0] is None
    near(dU, wanted[1], GRAD[dtype], "dU")
    near(dV, wanted[2], GRAD[dtype], "dV")
    if bias:
        near(got[3], wanted[3], GRAD[dtype], "dbias")
    else:
        assert got[3] is None
    assert pf.pf_last_device_status() == 0


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("act", list(ACTS))
def test_gates(dtype, act):
    check(300, 128, 264, 64, dtype, act)
    check(77, 72, 130, 20, dtype, act, bias=True)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("m,k,n,r", [(1, 512, 2048, 128), (1, 8, 8, 1), (2, 33, 65, 7), (20, 512, 2048, 128), (128, 64, 128, 64), (129, 64, 136, 72), (257, 100, 1000, 200),
                                     (700, 256, 392, 256), (300, 512, 520, 320), (2050, 128, 384, 40), (1000, 1364, 500, 100), (64, 2000, 300, 511)])
def test_sizes(dtype, m, k, n, r):
    check(m, k, n, r, dtype)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("layout", ["padded", "odd"])
@pytest.mark.parametrize("m,k,n,r", [(130, 64, 128, 64), (75, 100, 130, 33), (300, 136, 257, 65)])
def test_layouts(dtype, layout, m, k, n, r):
    check(m, k, n, r, dtype, "gelu", layout=layout, bias=True)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("m,k,n,r", [(200, 128, 256, 64), (90, 60, 70, 13)])
def test_without_stash_and_without_dx(dtype, m, k, n, r):
    check(m, k, n, r, dtype, stash=False)
    check(m, k, n, r, dtype, need_dX=False, bias=True)


def test_many_tiles():
    """More tiles than SMs, runs that end within a row of tiles, and a contraction that does not stay in shared memory."""
    check(2500, 96, 1500, 128, BF16)
    check(2500, 96, 1500, 300, BF16, "gelu")
    check(5000, 64, 72, 16, BF16, "relu")


@pytest.mark.parametrize("m,k,n,r,dtype,layout", [(9000, 40, 1001, 33, F32, "plain"), (8500, 36, 1000, 30, F32, "padded"), (9000, 33, 1003, 9, F32, "odd"),
                                                  (9000, 40, 1001, 33, BF16, "odd"), (900, 130, 10000, 66, F32, "plain")])
def test_rows_in_turns(m, k, n, r, dtype, layout):
    """Results of more than 2^23 elements, which are made some rows at a time where the gate is a kernel of its own."""
    check(m, k, n, r, dtype, layout=layout, bias=True)
    check(m, k, n, r, dtype, "gelu", layout=layout, stash=False)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", DT)
def test_far_arguments(dtype, act):
    """Gates far out on both sides, where exponentials overflow: finite, and their limits."""
    U = torch.zeros(2, 8, 8, dtype=dtype, device="cuda")
    V = torch.zeros(2, 16, 8, dtype=dtype, device="cuda")
    bias = torch.zeros(2, 16, dtype=dtype, device="cuda")
    bias[0] = torch.tensor([0.0, 1.0, -1.0, 30.0, -30.0, 90.0, -90.0, 200.0, -200.0, 1e4, -1e4, 1e10, -1e10, 1e25, -1e25, 0.5])
    bias[1] = 2.0
    x = normal((3, 8), dtype, 1)
    y = pf.pf_lowrank_linear_gated_fwd(x, U, V, bias=bias, act=ACTS[act])
    z = bias[0].double()
    want = 2 * (z * torch.sigmoid(1.5957691216057308 * (z + 0.044715 * z ** 3)) if act == "gelu" else ref.act(z, act))
    # (the exponent of the tanh form, up to 90 before the result is below 1e-36: off by 2^-22 of it)
    close(y, want.expand(3, 16), 2.0 ** -15 * want.abs() + 1e-36, "y")
    dx, dU, dV, db = pf.pf_lowrank_linear_gated_bwd(x, U, V, torch.ones_like(y), bias=bias, act=ACTS[act])
    assert all(torch.isfinite(t).all() for t in (dx, dU, dV, db))
    w = z.clone().requires_grad_()
    out = w * torch.sigmoid(1.5957691216057308 * (w + 0.044715 * w ** 3)) if act == "gelu" else ref.act(w, act)
    slope = torch.autograd.grad(out.sum(), w)[0].nan_to_num(nan=0.0)
    if act == "sigmoid":      # (1 - sigmoid without its cancellation)
        slope = torch.sigmoid(z) * torch.sigmoid(-z)
    slope = torch.where(z >= 90, 0.0 if act == "sigmoid" else 1.0, torch.where(z <= -90, 0.0, slope))
    got = db[0].double()
    # rows are rounded before the three are added up: a half step each
    allowed = (2.0 ** -7 if dtype == BF16 else 2.0 ** -15) * 6 * slope.abs() + 1e-30
    assert ((got - 6 * slope).abs() <= allowed).all(), (got, 6 * slope)


def test_no_rows():
    U, V = normal((2, 64, 16), BF16, 1), normal((2, 32, 16), BF16, 2)
    x, b = torch.empty(0, 64, dtype=BF16, device="cuda"), normal((2, 32), BF16, 3)
    y, T = pf.pf_lowrank_linear_gated_fwd(x, U, V, want_stash=True)
    assert y.shape == (0, 32) and T.shape == (2, 0, 16)
    dX, dU, dV, db = pf.pf_lowrank_linear_gated_bwd(x, U, V, y, bias=b)
    assert dX.shape == (0, 64) and all((t == 0).all() for t in (dU, dV, db))


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gradient_against_differences(act):
    x, U, V, b, g = (normal(s, F32, i, 0.7) for i, s in enumerate(((5, 6), (2, 6, 3), (2, 7, 3), (2, 7), (5, 7))))
    got = pf.pf_lowrank_linear_gated_bwd(x, U, V, g, bias=b, act=ACTS[act])

    def f(x, U, V, b):
        z = (x @ U) @ V.transpose(1, 2) + b[:, None]
        return (ref.act(z[0], act) * z[1] * g.double()).sum()
    args = [t.double() for t in (x, U, V, b)]
    for i, t in enumerate(got):
        at = range(0, t.numel(), 3)
        want = ref.differences(lambda v: f(*args[:i], v, *args[i + 1:]), args[i], at)
        assert torch.allclose(t.double().view(-1)[list(at)].cpu(), want, rtol=1e-4, atol=1e-4), i


def test_repeats_replays_and_streams():
    m, k, n, r = 700, 256, 520, 96
    x, U, V, g = normal((m, k), BF16, 1), normal((2, k, r), BF16, 2, 0.06), normal((2, n, r), BF16, 3, 0.1), normal((m, n), BF16, 4)
    y, T = pf.pf_lowrank_linear_gated_fwd(x, U, V, want_stash=True)
    first = pf.pf_lowrank_linear_gated_bwd(x, U, V, g, T_stash=T)[:3]
    assert all(torch.equal(a, b) for a, b in zip(first, pf.pf_lowrank_linear_gated_bwd(x, U, V, g, T_stash=T)))
    torch.cuda.synchronize()
    # (shared SMs may delay the layers' split sums: one stream at a time)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, T2 = pf.pf_lowrank_linear_gated_fwd(x, U, V, want_stash=True)
        second = pf.pf_lowrank_linear_gated_bwd(x, U, V, g, T_stash=T2)[:3]
    for t in (y2, T2) + second:
        t.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(T, T2) and all(torch.equal(a, b) for a, b in zip(first, second))
    side = torch.cuda.Stream()
    y3 = pf.pf_lowrank_linear_gated_fwd(x, U, V, stream=side)
    side.synchronize()
    assert torch.equal(y, y3)
    call, out = pf.pf_lowrank_linear_gated_fwd(x, U, V, prepare=True)
    call()
    assert torch.equal(out, y) and pf.pf_last_device_status() == 0


def test_arguments_are_checked():
    x, U, V = normal((4, 16), BF16, 1), normal((2, 16, 8), BF16, 2), normal((2, 24, 8), BF16, 3)
    for bad in (dict(U=U[:1]), dict(V=V[:, :, :7]), dict(U=U.float()), dict(bias=normal((2, 23), BF16, 1)), dict(bias=normal((24,), BF16, 1)),
                dict(y=torch.empty(4, 23, dtype=BF16, device="cuda")), dict(T_stash=torch.empty(2, 3, 8, dtype=BF16, device="cuda")), dict(V=V[:, :20].mT)):
        with pytest.raises(ValueError):
            pf.pf_lowrank_linear_gated_fwd(**(dict(x=x, U=U, V=V) | bad))
    with pytest.raises(pf.PfError):
        pf.pf_lowrank_linear_gated_fwd(x, U, V, act=4)
    with pytest.raises(pf.PfError):
        pf.pf_lowrank_linear_gated_fwd(x, U[:1].expand(2, 16, 8), V)
    with pytest.raises(pf.PfError):
        pf.pf_lowrank_linear_gated_fwd(x, U, V, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("n", [16, 130, 1024])
def test_far_products(dtype, act, n):
    """Both operands of the product far out: what a gate closes is 0 however large the other side is, also where the two alone would overflow."""
    g = torch.tensor([-1e20, -1e10, -100.0, -1e25, 1e10, 1e18, 0.0, 2.0]).repeat(-(-n // 8))[:n]
    u = torch.tensor([1e20, 1e30, 1e38, -1e15, -1e20, 1e20, 1e38, 3e37]).repeat(-(-n // 8))[:n]
    U, V = torch.zeros(2, 8, 8, dtype=dtype, device="cuda"), torch.zeros(2, n, 8, dtype=dtype, device="cuda")
    bias = torch.stack((g, u)).to(dtype).cuda()
    x = normal((3, 8), dtype, 1)
    y = pf.pf_lowrank_linear_gated_fwd(x, U, V, bias=bias, act=ACTS[act])
    z, v = bias.double()
    a = z * torch.sigmoid(1.5957691216057308 * (z + 0.044715 * z ** 3)) if act == "gelu" else ref.act(z, act)
    want = (a * v).expand(3, n)
    # (what a gate leaves below 2^-126 may be taken as nothing)
    close(y, want, 2.0 ** -15 * want.abs() + (2.0 ** -126 * v.abs() * torch.clamp(z.abs(), min=1.0)), "y")
    got = pf.pf_lowrank_linear_gated_bwd(x, U, V, torch.full_like(y, 1e-30), bias=bias, act=ACTS[act])
    assert all(torch.isfinite(t).all() for t in got)
    # gradients that overflow beside u, but not beside a gate that is closed
    db = pf.pf_lowrank_linear_gated_bwd(x, U, V, torch.full_like(y, 30.0), bias=bias, act=ACTS[act])[3]
    closed = g <= -100
    assert torch.isfinite(db[0, closed]).all() and (db[1, closed].abs() <= 1e-30).all()


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("odd", ["x", "U", "V", "T", "y", "x U V T y"])
@pytest.mark.parametrize("m,k,n,r", [(158, 728, 224, 112), (97, 8, 288, 8), (2000, 16, 1736, 40), (9000, 1000, 72, 16)])
def test_bf16_matrices_at_odd_places(act, odd, m, k, n, r):
    """Matrices of whole 16-byte rows that do not lie on 16 bytes: what g and u are is rounded no more than where they do, so that the results are the same, and
    gradients are as near (g of max(0, .) on the right side of zero)."""
    def place(t, name, pair=False):
        if name not in odd.split():
            return t
        rows, cols = t.shape[-2:]
        gs, ld = rows * (cols + 3) + 5, cols + 3
        out = torch.zeros((2 if pair else 1) * gs + 64, dtype=BF16, device="cuda")
        return (out.as_strided((2, rows, cols), (gs, ld, 1), 1) if pair else out.as_strided((rows, cols), (ld, 1), 1)).copy_(t)
    x, U, V = normal((m, k), BF16, 1), normal((2, k, r), BF16, 2, k ** -0.5), normal((2, n, r), BF16, 3, 1.5 * r ** -0.5)
    b, dY = normal((2, n), BF16, 4, 0.5), normal((m, n), BF16, 5)
    y, T = pf.pf_lowrank_linear_gated_fwd(x, U, V, bias=b, act=ACTS[act], want_stash=True)
    x_, U_, V_, dY_ = place(x, "x"), place(U, "U", True), place(V, "V", True), place(dY, "y")
    T_, y_ = place(torch.zeros_like(T), "T", True), place(torch.zeros_like(y), "y")
    ws = Scratch(pf.pf_lowrank_linear_gated_workspace(m, k, n, r, pf.PF_BF16, False))
    pf.pf_lowrank_linear_gated_fwd(x_, U_, V_, bias=b, act=ACTS[act], y=y_, T_stash=T_, workspace=ws.t)
    ws.check()
    exact_T = x.double() @ U.double()
    for t in (T, T_):
        close(t, exact_T, 2.0 ** -18 * (x.double().abs() @ U.double().abs()), "T")
    want, slack = ref.gated(T_, V, b, act)
    close(y_, want, slack, "y")
    for stash in (T_, None):
        ws = Scratch(pf.pf_lowrank_linear_gated_workspace(m, k, n, r, pf.PF_BF16, True))
        dX, dU, dV, db = pf.pf_lowrank_linear_gated_bwd(x_, U_, V_, dY_, bias=b, act=ACTS[act], T_stash=stash, workspace=ws.t)
        ws.check()
        z = (T_.double() @ V.double().transpose(1, 2) + b.double()[:, None]).requires_grad_()
        dZ = torch.autograd.grad(ref.act(z[0], act) * z[1], z, dY.double())[0]
        G = dZ @ V.double()
        near(dX, (G @ U.double().transpose(1, 2)).sum(0), GRAD[BF16], "dX")
        near(dU, x.double().T @ G, GRAD[BF16], "dU")
        near(dV, dZ.transpose(1, 2) @ T_.double(), GRAD[BF16], "dV")
        near(db, dZ.sum(1), GRAD[BF16], "dbias")
