"""GPU parity of the norm and rotation of queries and keys against a plain form in 64 bits."""
import pytest
import torch

import _ops
import paper_2103_03936_b200 as pf
from _gpu import Scratch

pytestmark = pytest.mark.gpu
DT = [torch.bfloat16, torch.float32]


def normal(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def frequencies(half):
    return (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float().cuda()


class Rows:
    """[tokens, heads, dim] inside a sentinel-filled buffer with chosen strides of tokens and heads."""

    def __init__(self, tokens, heads, dim, dtype, ld=None, s=None, shift=0):
        s = dim if s is None else s
        ld = heads * s if ld is None else ld
        n = max(0, (tokens - 1) * ld + (heads - 1) * s + dim) if tokens and heads else 0
        self.buf = torch.full((n + 128,), -7.0, dtype=dtype, device="cuda")
        self.t = self.buf.as_strided((tokens, heads, dim), (ld, s, 1), 64 + shift)

    def fill(self, values):
        self.t.copy_(values)
        return self.t

    def check(self):
        seen = torch.zeros_like(self.buf, dtype=torch.bool)
        seen.as_strided(self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(True)
        assert (self.buf[~seen] == -7).all(), "written outside the rows"


def check(tokens, hq, hk, dim, rot, dtype, *, pairs=False, weights=True, positions="far", layout="plain", eps=1e-6, f32=False, seed=1):
    style = pf.PF_ROPE_PAIRS if pairs else pf.PF_ROPE_HALVES
    how = {"plain": lambda h: {}, "padded": lambda h: {"s": dim + 24, "ld": h * (dim + 24) + 40}, "heads first": lambda h: {"ld": dim, "s": tokens * dim},
           "odd": lambda h: {"s": dim + 1, "ld": h * (dim + 1) + 3, "shift": 1}}[layout]
    make = lambda h: Rows(tokens, h, dim, dtype, **how(h))  # noqa: E731
    x = [make(h).fill(normal((tokens, h, dim), dtype, seed + i, 1.7 - i)) if h else None for i, h in enumerate((hq, hk))]
    g = [make(h).fill(normal((tokens, h, dim), dtype, seed + 2 + i)) if h else None for i, h in enumerate((hq, hk))]
    w = [(1 + normal((dim,), torch.float32, seed + 4 + i, 0.3)).to(dtype) if weights and h else None for i, h in enumerate((hq, hk))]
    out, dx = ([make(h) if h else None for h in (hq, hk)] for _ in range(2))
    t_of = lambda rows: [r.t if r else None for r in rows]  # noqa: E731
    pos = {"far": torch.randint(0, 1 << 20, (tokens,), generator=torch.Generator().manual_seed(seed)).cuda(), "none": None,
           "ends": (torch.arange(tokens) * ((1 << 33) + 12345) - 17).cuda()}[positions]
    freq = frequencies(rot // 2)
    rest = dict(positions=pos, style=style, eps=eps)
    pf.pf_qk_norm_rope_fwd(*x, *w, freq, q_out=t_of(out)[0], k_out=t_of(out)[1], **rest)
    grads = pf.pf_qk_norm_rope_bwd(*x, *w, freq, *g, dq=t_of(dx)[0], dk=t_of(dx)[1], grads_f32=f32, **rest)
    angle = _ops.angles(torch.arange(tokens, device="cuda") if pos is None else pos, freq)
    for i, name in enumerate("qk"):
        if x[i] is None:
            continue
        out[i].check()
        dx[i].check()
        want, slack = _ops.norm_rope(x[i], w[i], angle, pairs, eps)
        _ops.close(out[i].t, want, slack, name + "_out")
        want, slack, dw, dw_slack = _ops.norm_rope_bwd(x[i], w[i], angle, pairs, eps, g[i])
        _ops.close(dx[i].t, want, slack, "d" + name)
        if w[i] is None:
            assert grads[2 + i] is None
        else:
            assert grads[2 + i].dtype == (torch.float32 if f32 else dtype)
            _ops.close(grads[2 + i], dw, dw_slack, "dw" + name)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 128), (128, 64), (80, 80), (96, 32), (192, 192), (256, 256), (512, 512), (32, 32), (16, 16), (64, 0),
                                     (128, 96), (1, 0), (2, 2), (7, 4), (18, 18), (66, 66), (100, 60), (333, 100), (1024, 1024), (1023, 14), (48, 8)])
def test_dims(dtype, pairs, dim, rot):
    check(9, 4, 2, dim, rot, dtype, pairs=pairs)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("layout", ["plain", "padded", "heads first", "odd"])
@pytest.mark.parametrize("tokens,hq,hk", [(1, 1, 1), (1, 32, 8), (2, 5, 1), (37, 3, 3), (700, 8, 8), (33, 28, 4), (5, 0, 3), (6, 7, 0), (3000, 2, 1), (1001, 1, 1), (777, 16, 1)])
def test_layouts(dtype, layout, tokens, hq, hk):
    check(tokens, hq, hk, 64, 64, dtype, layout=layout)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,rot", [(32, 32), (64, 32), (128, 128), (66, 66), (100, 40), (20, 14)])
def test_one_and_two_heads(dim, rot, pairs):
    """Sides whose heads leave most of a warp's rows to other tokens."""
    for dtype in DT:
        check(203, 2, 1, dim, rot, dtype, pairs=pairs, positions="ends")
        check(5, 9, 1, dim, rot, dtype, pairs=pairs, f32=True, eps=0.0)


def test_many_tokens():
    """More units than warps of the grid, on the vector kernels and on the others."""
    check(5000, 6, 3, 128, 128, torch.bfloat16)
    check(5000, 6, 3, 50, 50, torch.bfloat16, pairs=True)


@pytest.mark.parametrize("positions", ["none", "ends"])
def test_positions(positions):
    check(60, 4, 2, 64, 64, torch.float32, positions=positions)
    check(60, 4, 2, 30, 20, torch.float32, positions=positions, pairs=True)


def test_no_weights_and_fp32_gradients():
    check(40, 4, 2, 64, 32, torch.bfloat16, weights=False)
    check(40, 4, 2, 64, 32, torch.bfloat16, f32=True)
    check(40, 4, 2, 34, 34, torch.bfloat16, f32=True, eps=0.0)
    check(41, 5, 3, 64, 64, torch.float32, eps=0.0)      # heads that do not fill a warp: nothing of the empty places reaches dw


def test_rows_of_zeros_and_infinities():
    """A row of zeros gives zeros and r = 1 / sqrt(eps); what is not finite stays in its row, but for dw."""
    for dim in (64, 50):
        q = normal((4, 3, dim), torch.float32, 1)
        q[1, 2] = 0
        q[2, 0, 5] = float("inf")
        w, f = torch.ones(dim, device="cuda"), frequencies(dim // 2)
        out, _ = pf.pf_qk_norm_rope_fwd(q, None, w, None, f)
        assert (out[1, 2] == 0).all() and torch.isnan(out[2, 0]).any()
        out[2, 0] = 0
        assert torch.isfinite(out).all()
        g = normal((4, 3, dim), torch.float32, 2)
        dq = pf.pf_qk_norm_rope_bwd(q, None, w, None, f, g, None)[0]
        dq[2, 0] = 0
        assert torch.isfinite(dq).all()
        turned_back = _ops.turn(g.double(), -_ops.angles(torch.arange(4, device="cuda"), f), False)[1, 2]
        _ops.close(dq[1, 2], 1000 * turned_back, 1000 * 2.0 ** -18 * _ops.other(g.double(), dim // 2, False)[1, 2], "dq of a row of zeros")


def test_gradients_accumulate():
    q, k, g = normal((30, 4, 64), torch.bfloat16, 1), normal((30, 2, 64), torch.bfloat16, 2), normal((30, 6, 64), torch.bfloat16, 3)
    gq, gk = g[:, :4].contiguous(), g[:, 4:].contiguous()
    w, f = torch.ones(64, dtype=torch.bfloat16, device="cuda"), frequencies(32)
    _, _, a, b = pf.pf_qk_norm_rope_bwd(q, k, w, w, f, gq, gk, grads_f32=True)
    start = torch.arange(64, device="cuda").float()
    dwq, dwk = start.clone(), -start
    pf.pf_qk_norm_rope_bwd(q, k, w, w, f, gq, gk, dwq=dwq, dwk=dwk, accumulate=True, grads_f32=True)
    assert torch.equal(dwq, start + a) and torch.equal(dwk, b - start)
    with pytest.raises(ValueError):
        pf.pf_qk_norm_rope_bwd(q, k, w, w, f, gq, gk, accumulate=True)
    assert pf.pf_qk_norm_rope_bwd(q, k, w, w, f, gq, gk, need_dw=False)[2:] == (None, None)


def test_no_tokens():
    q, w, f = torch.empty((0, 4, 64), device="cuda"), torch.ones(64, device="cuda"), frequencies(32)
    assert pf.pf_qk_norm_rope_fwd(q, q, w, w, f)[0].shape == (0, 4, 64)
    dq, dk, dwq, dwk = pf.pf_qk_norm_rope_bwd(q, q, w, w, f, q, q)
    assert (dwq == 0).all() and (dwk == 0).all() and dq.shape == (0, 4, 64)
    keep, also = torch.full((64,), 5.0, device="cuda"), torch.full((64,), 6.0, device="cuda")
    pf.pf_qk_norm_rope_bwd(q, q, w, w, f, q, q, dwq=keep, dwk=also, accumulate=True)
    assert (keep == 5).all() and (also == 6).all()


@pytest.mark.parametrize("tokens,hq,hk,dim", [(3, 1, 1, 64), (5000, 8, 1, 64), (9000, 32, 8, 128), (4000, 3, 3, 66), (3000, 2, 2, 600)])
def test_a_workspace_of_the_queried_size(tokens, hq, hk, dim):
    q, k, w, f = normal((tokens, hq, dim), torch.bfloat16, 1), normal((tokens, hk, dim), torch.bfloat16, 2), normal((dim,), torch.bfloat16, 3), frequencies(dim // 2)
    scratch = Scratch(pf.pf_qk_norm_rope_bwd_workspace(tokens, hq, hk, dim))
    got = pf.pf_qk_norm_rope_bwd(q, k, w, w, f, q, k, workspace=scratch.t)
    scratch.check()
    for a, b in zip(got, pf.pf_qk_norm_rope_bwd(q, k, w, w, f, q, k)):
        assert torch.equal(a, b)


def test_a_side_without_heads():
    q, none, w, f = normal((9, 4, 64), torch.bfloat16, 1), torch.empty((9, 0, 64), dtype=torch.bfloat16, device="cuda"), normal((64,), torch.bfloat16, 2), frequencies(32)
    a, b = pf.pf_qk_norm_rope_fwd(q, none, w, w, f)
    assert b.shape == (9, 0, 64) and torch.equal(a, pf.pf_qk_norm_rope_fwd(q, None, w, None, f)[0])
    dq, dk, dwq, dwk = pf.pf_qk_norm_rope_bwd(q, none, w, w, f, q, none)
    assert dwk is None and dk.shape == (9, 0, 64)
    want = pf.pf_qk_norm_rope_bwd(q, None, w, None, f, q, None)
    assert torch.equal(dq, want[0]) and torch.equal(dwq, want[2])


@pytest.mark.parametrize("dim,pairs", [(64, False), (64, True), (54, False)])
def test_gradient_against_differences(dim, pairs):
    """<gradient, direction> of a weighted sum of the outputs against its central difference in 64 bits: the difference is off by
    the step's square (1e-8 of a third derivative), the gradient by 2^-16 of its terms."""
    style = pf.PF_ROPE_PAIRS if pairs else pf.PF_ROPE_HALVES
    q, g = normal((6, 3, dim), torch.float32, 1), normal((6, 3, dim), torch.float32, 2)
    w, f = 1 + normal((dim,), torch.float32, 3, 0.2), frequencies(dim // 2)
    dq, _, dw, _ = pf.pf_qk_norm_rope_bwd(q, None, w, None, f, g, None, style=style)
    angle = _ops.angles(torch.arange(6, device="cuda"), f)
    loss = lambda x, v: float((_ops.norm_rope(x, v, angle, pairs, 1e-6)[0] * g.double()).sum())  # noqa: E731
    for seed in range(4):
        a, b, h = normal((6, 3, dim), torch.float64, 10 + seed), normal((dim,), torch.float64, 20 + seed), 1e-4
        for got, step in ((float((dq.double() * a).sum()), (a, 0)), (float((dw.double() * b).sum()), (0, b))):
            want = (loss(q.double() + h * step[0], w.double() + h * step[1]) - loss(q.double() - h * step[0], w.double() - h * step[1])) / (2 * h)
            assert abs(got - want) <= 2.0 ** -16 * float(g.abs().sum()) * 4 + 1e-5


def test_rows_beyond_32_bits():
    """Rows more than 2^31 elements behind the first."""
    tokens, dim = 3, 128
    x = normal((tokens, 2, dim), torch.bfloat16, 1)
    pitch = (1 << 30) + 64
    strided = lambda: torch.empty(((tokens - 1) * pitch + 2 * dim,), dtype=torch.bfloat16, device="cuda").as_strided((tokens, 2, dim), (pitch, dim, 1))  # noqa: E731
    big, out = strided(), strided()
    big.copy_(x)
    f, w = frequencies(64), torch.ones(dim, dtype=torch.bfloat16, device="cuda")
    want = pf.pf_qk_norm_rope_fwd(x, None, w, None, f)[0]
    pf.pf_qk_norm_rope_fwd(big, None, w, None, f, q_out=out)
    assert torch.equal(out, want)
    a, b = pf.pf_qk_norm_rope_bwd(big, None, w, None, f, out, None), pf.pf_qk_norm_rope_bwd(x, None, w, None, f, want, None)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_captured_and_replayed_and_prepared():
    q, k, w, f = normal((70, 8, 64), torch.bfloat16, 1), normal((70, 2, 64), torch.bfloat16, 2), normal((64,), torch.bfloat16, 3), frequencies(32)
    pos = torch.arange(70, device="cuda")

    def whole():
        a, b = pf.pf_qk_norm_rope_fwd(q, k, w, w, f, positions=pos)
        return (a, b) + pf.pf_qk_norm_rope_bwd(q, k, w, w, f, a, b, positions=pos)
    whole()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = whole()
    q.copy_(normal((70, 8, 64), torch.bfloat16, 7))
    pos.add_(1000)
    graph.replay()
    for a, b in zip(out, whole()):
        assert torch.equal(a, b)
    call, (a, b) = pf.pf_qk_norm_rope_fwd(q, k, w, w, f, positions=pos, prepare=True)
    call()
    assert torch.equal(a, out[0]) and torch.equal(b, out[1])
    call, got = pf.pf_qk_norm_rope_bwd(q, k, w, w, f, a, b, positions=pos, prepare=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        others = pf.pf_qk_norm_rope_bwd(q, k, w, w, f, a, b, positions=pos)
    call()
    torch.cuda.synchronize()
    for x, y in zip(got, others):
        assert torch.equal(x, y)


def test_refusals():
    q, w, f = normal((4, 3, 64), torch.float32, 1), torch.ones(64, device="cuda"), frequencies(32)
    for call in (lambda: pf.pf_qk_norm_rope_fwd(q[0], None, w, None, f), lambda: pf.pf_qk_norm_rope_fwd(q, q[:3], w, w, f),
                 lambda: pf.pf_qk_norm_rope_fwd(q, q[..., :32], w, w, f), lambda: pf.pf_qk_norm_rope_fwd(q, None, w[:63], None, f),
                 lambda: pf.pf_qk_norm_rope_fwd(q, None, w.bfloat16(), None, f), lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f.double()),
                 lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f, positions=torch.arange(3, device="cuda")),
                 lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f, positions=torch.arange(4, device="cuda").int()),
                 lambda: pf.pf_qk_norm_rope_fwd(q.permute(0, 2, 1), None, None, None, f[:1]), lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f.cpu()),
                 lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f, q_out=q.bfloat16()), lambda: pf.pf_qk_norm_rope_bwd(q, None, w, None, f, None, None),
                 lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f, k_out=torch.empty_like(q)),
                 lambda: pf.pf_qk_norm_rope_bwd(q, None, w, None, f, q, None, dwq=torch.ones(63, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pf.pf_qk_norm_rope_fwd(q.half(), None, None, None, f)
    for call in (lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, frequencies(33)), lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f, style=3),
                 lambda: pf.pf_qk_norm_rope_fwd(q, None, w, None, f, eps=-1.0),
                 lambda: pf.pf_qk_norm_rope_fwd(q[:, :1].expand(4, 3, 64), None, w, None, f)):
        with pytest.raises(pf.PfError) as e:
            call()
        assert e.value.status == 1


def test_a_workspace_that_is_no_whole_buffer_on_the_device_is_refused():
    q, w, f = normal((50, 4, 64), torch.bfloat16, 1), normal((64,), torch.bfloat16, 3), frequencies(32)
    need = pf.pf_qk_norm_rope_bwd_workspace(50, 4, 0, 64)
    for room in (torch.empty(need, dtype=torch.uint8), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2],
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(need)):
        with pytest.raises(ValueError, match="workspace"):
            pf.pf_qk_norm_rope_bwd(q, None, w, None, f, q, None, workspace=room)


@pytest.mark.parametrize("dim,heads", [(64, 4), (64, 1), (66, 3), (1024, 2)])
def test_angles_near_quarter_turns(dim, heads):
    """In fp32 a cosine or sine near zero keeps its digits, as far as an angle in 2^-32 of a turn has them.

    Rows of ones and zeros have r = sqrt(2), to 2^-22 (two units of rsqrt, roundings of 1 / dim and of the mean); sine and cosine to two
    units and the angle's rounding, the product one more: below 2^-20 of the result.  Of the angle, what is cut off is below 2^-32 of a turn."""
    half = dim // 2
    i = torch.arange(half, dtype=torch.float64)
    f = (torch.pi / 2 * (1 + i % 4) + (i - half / 2) * 1e-6).float().cuda()
    positions = torch.tensor([0, 1, 3, -5, 1001], device="cuda")
    x = torch.zeros((5, heads, dim), device="cuda")
    x[..., :half] = 1
    out = pf.pf_qk_norm_rope_fwd(x, None, None, None, f, positions=positions, eps=0.0)[0]
    angle = _ops.angles(positions, f)[:, None]
    want = 2 ** 0.5 * torch.cat([angle.cos(), angle.sin()], -1).expand_as(out)
    _ops.close(out, want, 2.0 ** -20 * want.abs() + 2 ** 0.5 * 2 * torch.pi * 2.0 ** -32 * 1.01, "turned")


@pytest.mark.parametrize("position", [(1 << 40) - 3, 1 << 40, -(1 << 40) + 12345, 987654321987])
def test_far_angles_near_quarter_turns(position):
    """As above at far positions, for frequencies whose angle there is near a quarter turn: a position's part of a turn is rounded to nearest, off by 2^-65."""
    g = torch.Generator().manual_seed(3)
    f = torch.cat([torch.rand(200000, generator=g), torch.logspace(-6, 2, 200000)])
    near = _ops.angles(torch.tensor([position]), f)[0] / (torch.pi / 2)
    f = f[(near - near.round()).abs().argsort()[:32]].cuda()
    positions = torch.tensor([position], device="cuda")
    x = torch.zeros((1, 2, 64), device="cuda")
    x[..., :32] = 1
    out = pf.pf_qk_norm_rope_fwd(x, None, None, None, f, positions=positions, eps=0.0)[0]
    angle = _ops.angles(positions, f)[:, None]
    want = 2 ** 0.5 * torch.cat([angle.cos(), angle.sin()], -1).expand_as(out)
    off = 2 ** 0.5 * 2 * torch.pi * (2.0 ** -32 + abs(position) * 2.0 ** -65) * 1.01
    _ops.close(out, want, 2.0 ** -20 * want.abs() + off, "turned")


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,heads", [(64, 4), (64, 1), (66, 3), (1024, 2), (256, 2)])
def test_a_frequency_that_is_not_finite_makes_its_pair_nan(dtype, pairs, dim, heads):
    """At every position (0 times infinity too), and nothing else of the row."""
    half = dim // 2
    x, f = normal((37, heads, dim), dtype, 1), frequencies(half)
    style = pf.PF_ROPE_PAIRS if pairs else pf.PF_ROPE_HALVES
    want = pf.pf_qk_norm_rope_fwd(x, None, None, None, f, style=style)[0]
    bad = [1, half // 2, half - 1]
    f[bad] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda")
    got = pf.pf_qk_norm_rope_fwd(x, None, None, None, f, style=style)[0]
    where = torch.zeros(dim, dtype=torch.bool, device="cuda")
    for i in bad:
        where[[2 * i, 2 * i + 1] if pairs else [i, half + i]] = True
    assert torch.isnan(got[..., where]).all() and torch.equal(got[..., ~where], want[..., ~where])
