"""GPU parity of the residual's addition with its norm, in the inputs' type and in 8 bits, and of the gradients, against a plain form in 64 bits."""
import pytest
import torch

import _more_ops as ref
import paper_2103_03936_b200 as pf
from _gpu import Scratch
from _more_ops import Rows, normal
from _ops import close

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
DT = [BF16, F32]


def layout_of(layout, width):
    return {"plain": {}, "padded": {"ld": width + 40}, "odd": {"ld": width + 3, "shift": 1}}[layout]


def check_codes(y8, scales, y, slack, block):
    """Codes are y / scale to half a step of the format (2^-4 of the value, 2^-10 below its normal numbers), scales 1 / 448 of a block's largest."""
    tokens, width = y.shape
    b = block or width
    blocks = -(-width // b)
    padded = lambda t: torch.nn.functional.pad(t, (0, blocks * b - width)).view(tokens, blocks, b)  # noqa: E731
    most = padded(y.abs()).amax(2)
    close(scales, most / 448, (2.0 ** -22 * most + padded(slack).amax(2)) / 448, "scales")
    s = scales.double().repeat_interleave(b, 1)[:, :width]
    v = torch.where(s > 0, y / s, 0.0)
    allowed = torch.maximum(2.0 ** -4 * v.abs(), torch.tensor(2.0 ** -10, device=v.device, dtype=v.dtype))
    allowed = allowed * (1 + 2.0 ** -16) + torch.where(s > 0, slack / s, 0.0) + 2.0 ** -20 * v.abs()
    bad = ~((y8.double() - v).abs() <= allowed)
    assert not bad.any(), f"codes: {int(bad.sum())} off"
    assert (y8.double()[s == 0] == 0).all()


def check(tokens, width, dtype, *, layout="plain", residual=True, weight=True, block=None, want_y=True, dh=True, f32=False, eps=1e-6, seed=1):
    make = lambda i, scale=1.0: Rows(tokens, width, dtype, **layout_of(layout, width)).fill(normal((tokens, width), dtype, seed + i, scale))  # noqa: E731
    x, res = make(0), make(1, 3.0).t if residual else None
    w = (1 + normal((width,), F32, seed + 2, 0.3)).to(dtype) if weight else None
    h, y = Rows(tokens, width, dtype, **layout_of(layout, width)), Rows(tokens, width, dtype, **layout_of(layout, width))
    more = {}
    if block is not None:
        codes = Rows(tokens, width, E4M3, **layout_of(layout, width))
        more = {"block": block, "y8": codes.t}
    got = pf.pf_add_rms_norm_fwd(x.t, res, w, eps=eps, want_y=want_y, h=h.t if residual else None, y=y.t if want_y else None, **more)
    want_h, h_slack, want, slack = ref.norm(x.t, res, w, eps)
    if residual:
        h.check()
        close(h.t, want_h, h_slack, "h")
    else:
        assert got[0] is None
    if want_y:
        y.check()
        close(y.t, want, slack, "y")
    if block is not None:
        codes.check()
        check_codes(codes.t, got[3], want, slack, block)
    # backward
    g, d, dx = make(3), make(4).t if dh else None, Rows(tokens, width, dtype, **layout_of(layout, width))
    hh = make(5, 2.0)
    need = pf.pf_add_rms_norm_bwd_workspace(tokens, width)
    ws = Scratch(need)
    _, dw = pf.pf_add_rms_norm_bwd(hh.t, w, g.t, dh=d, eps=eps, dx=dx.t, grads_f32=f32, workspace=ws.t)
    ws.check()
    dx.check()
    want, slack, want_dw, dw_slack = ref.norm_bwd(hh.t, w, g.t, d, eps)
    close(dx.t, want, slack, "dx")
    if weight:
        assert dw.dtype == (F32 if f32 else dtype)
        close(dw, want_dw, dw_slack, "dw")
    else:
        assert dw is None


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("width", [1, 2, 7, 8, 31, 64, 100, 128, 500, 512, 513, 1000, 1024, 1500, 2048, 4096, 4097, 5000, 8192, 12296, 16384, 16383])
def test_widths(dtype, width):
    check(5, width, dtype, block=128)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("layout", ["plain", "padded", "odd"])
@pytest.mark.parametrize("tokens,width", [(1, 512), (2, 96), (700, 256), (33, 1504), (9, 33), (5000, 64), (1300, 2048)])
def test_layouts(dtype, layout, tokens, width):
    check(tokens, width, dtype, layout=layout, block=32)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("width", [64, 200, 512, 1000, 1030, 1500, 2000, 2300, 2600, 2968, 3400, 4096, 4500, 9000, 16384])
def test_workspace_holds_the_sums_of_all_blocks(dtype, width):
    """As many rows as keep every SM full, whatever the number of warps that a row takes: nothing is written behind the workspace."""
    tokens = 148 * 4 * 66 if width <= 256 else 148 * 4 * 8 if width <= 512 else 148 * 8
    h, dy = normal((tokens, width), dtype, 1), normal((tokens, width), dtype, 2)
    ws = Scratch(pf.pf_add_rms_norm_bwd_workspace(tokens, width))
    dx, dw = pf.pf_add_rms_norm_bwd(h, torch.ones(width, dtype=dtype, device="cuda"), dy, workspace=ws.t)
    ws.check()
    _, _, want, slack = ref.norm_bwd(h, None, dy, None, 1e-6)
    close(dw, want, slack, "dw")


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("tokens", [1, 63, 3001])
@pytest.mark.parametrize("width", [3, 16, 60, 64, 65, 127, 192, 256, 260])
def test_narrow_rows(dtype, tokens, width):
    """Rows that share a warp."""
    for block in (None, 0, 32, 128) if tokens == 63 else (32,):
        check(tokens, width, dtype, block=block, seed=width)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("block", [0, 32, 128])
@pytest.mark.parametrize("width", [20, 256, 500, 777, 1536, 9000])
def test_codes_alone(dtype, block, width):
    check(37, width, dtype, block=block, want_y=False)
    check(3, width, dtype, block=block, residual=False, layout="odd")


@pytest.mark.parametrize("dtype", DT)
def test_what_may_be_left_out(dtype):
    check(40, 512, dtype, residual=False)
    check(40, 512, dtype, weight=False, dh=False)
    check(40, 300, dtype, weight=False, residual=False, eps=0.0)
    check(41, 600, dtype, f32=True, dh=False, eps=0.0)
    x = normal((4, 64), dtype, 1)
    assert pf.pf_add_rms_norm_bwd(x, x[0].contiguous(), x, need_dw=False)[1] is None


@pytest.mark.parametrize("block", [0, 32, 128])
def test_codes_at_the_ends_of_the_format(block):
    """Blocks of zeros, tiny blocks, and what is not finite."""
    x = torch.zeros(5, 256, device="cuda")
    x[0, 200:] = 1.0                      # blocks of zeros before it
    x[1] = normal((256,), F32, 1, 1e-38)  # eps makes y of the size of 1e-35: a scale below the normal numbers
    x[2] = normal((256,), F32, 2, 1e-30)
    x[3] = normal((256,), F32, 3)
    x[3, 7] = float("inf")
    x[4, 9] = float("nan")
    _, y, y8, scales = pf.pf_add_rms_norm_fwd(x, block=block)
    _, _, want, slack = ref.norm(x[:3], None, None, 1e-6)
    close(y[:3], want, slack + 1e-45, "y")
    s = scales.double().repeat_interleave(block or 256, 1)
    value = y8.double() * s
    # what is held is y to half a step, or to half of the smallest code's where that is more; a scale is 2^-126 at least
    off = (value[:3] - want).abs()
    assert (off <= torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * s[:3]) * 1.001 + slack).all()
    assert (scales[:3][scales[:3] > 0] >= 2.0 ** -126).all()
    if block:
        assert scales[0, 0] == 0 and (y8[0, :128].float() == 0).all()
    assert torch.isnan(y[3:]).any(1).all() and torch.isnan(scales[4]).any() and torch.isnan(y8[4].float()).any()
    assert torch.isfinite(y[:3]).all() and torch.isfinite(y8[:3].float()).all()


def test_rows_that_are_not_finite_stay_in_their_rows():
    for dtype in DT:
        h, g = normal((6, 512), dtype, 1), normal((6, 512), dtype, 2)
        h[2, 5], h[4, 300] = float("inf"), float("nan")
        w = torch.ones(512, dtype=dtype, device="cuda")
        _, y, _, _ = pf.pf_add_rms_norm_fwd(h, torch.zeros_like(h), w)
        dx, _ = pf.pf_add_rms_norm_bwd(h, w, g, need_dw=False)
        for t in (y, dx):
            assert torch.isnan(t[2]).any() and torch.isnan(t[4]).all() and torch.isfinite(t[[0, 1, 3, 5]]).all()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("width", [512, 333])
def test_in_place(dtype, width):
    x, r, w = normal((70, width), dtype, 1), normal((70, width), dtype, 2), normal((width,), dtype, 3)
    h, y, _, _ = pf.pf_add_rms_norm_fwd(x, r, w)
    for own in (0, 1):
        t = [x.clone(), r.clone()]
        h2, y2, _, _ = pf.pf_add_rms_norm_fwd(t[0], t[1], w, h=t[own])
        assert torch.equal(h2, h) and torch.equal(y2, y) and h2.data_ptr() == t[own].data_ptr()
    g, d = normal((70, width), dtype, 4), normal((70, width), dtype, 5)
    dx, dw = pf.pf_add_rms_norm_bwd(h, w, g, dh=d)
    for own in range(3):
        t = [h.clone(), g.clone(), d.clone()]
        dx2, dw2 = pf.pf_add_rms_norm_bwd(t[0], w, t[1], dh=t[2], dx=t[own])
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw)


def test_gradients_accumulate():
    h, g, w = normal((3000, 512), BF16, 1), normal((3000, 512), BF16, 2), normal((512,), BF16, 3)
    _, dw = pf.pf_add_rms_norm_bwd(h, w, g, grads_f32=True)
    start = torch.arange(512, device="cuda").float()
    total = start.clone()
    pf.pf_add_rms_norm_bwd(h, w, g, dw=total, accumulate=True, grads_f32=True)
    assert torch.equal(total, start + dw)
    with pytest.raises(ValueError):
        pf.pf_add_rms_norm_bwd(h, w, g, accumulate=True)
    rounded = pf.pf_add_rms_norm_bwd(h, w, g)[1]
    assert torch.equal(rounded, dw.to(BF16))


def test_no_tokens():
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    h, y, y8, scales = pf.pf_add_rms_norm_fwd(x, x, w, block=32)
    assert h.shape == y.shape == (0, 64) and y8.shape == (0, 64) and scales.shape == (0, 2)
    dw = torch.full((64,), 5.0, device="cuda")
    dx, _ = pf.pf_add_rms_norm_bwd(x, w, x, dw=dw, accumulate=True)
    assert dx.shape == (0, 64) and (dw == 5).all()
    assert (pf.pf_add_rms_norm_bwd(x, w, x, dw=dw)[1] == 0).all()


def test_gradient_against_differences():
    h, w, g = (normal(s, F32, i) for i, s in enumerate(((2, 24), (24,), (2, 24))))
    dx, dw = pf.pf_add_rms_norm_bwd(h, w, g)
    f = lambda a, b: float((ref.norm(a, None, b, 1e-6)[2] * g.double()).sum())  # noqa: E731
    at = range(0, 48, 7)
    want = ref.differences(lambda v: f(v, w), h.double(), at)
    assert torch.allclose(dx.double().view(-1)[list(at)].cpu(), want, rtol=1e-4, atol=1e-5)
    want = ref.differences(lambda v: f(h, v), w.double(), range(24))
    assert torch.allclose(dw.double().cpu(), want, rtol=1e-4, atol=1e-5)


def test_repeats_are_bit_identical_and_replays_too():
    h, w, g = normal((5000, 512), BF16, 1), normal((512,), BF16, 2), normal((5000, 512), BF16, 3)
    first = pf.pf_add_rms_norm_bwd(h, w, g, dh=g)
    again = pf.pf_add_rms_norm_bwd(h, w, g, dh=g)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    call, out = pf.pf_add_rms_norm_bwd(h, w, g, dh=g, prepare=True)
    fcall, fout = pf.pf_add_rms_norm_fwd(h, g, w, block=128, prepare=True)
    want = pf.pf_add_rms_norm_fwd(h, g, w, block=128)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a = pf.pf_add_rms_norm_bwd(h, w, g, dh=g)
        b = pf.pf_add_rms_norm_fwd(h, g, w, block=128)
    for t in a + b:
        t.fill_(0)
    graph.replay()
    call()
    fcall()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, first)) and all(torch.equal(x.float(), y.float()) for x, y in zip(b, want))
    assert all(torch.equal(x, y) for x, y in zip(out, first)) and all(torch.equal(x.float(), y.float()) for x, y in zip(fout, want))


def test_another_stream():
    side = torch.cuda.Stream()
    x, w = normal((400, 512), BF16, 1), normal((512,), BF16, 2)
    want = pf.pf_add_rms_norm_fwd(x, x, w)
    torch.cuda.synchronize()
    got = pf.pf_add_rms_norm_fwd(x, x, w, stream=side)
    dx, dw = pf.pf_add_rms_norm_bwd(x, w, x, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ref_dx, ref_dw = pf.pf_add_rms_norm_bwd(x, w, x)
    assert torch.equal(dx, ref_dx) and torch.equal(dw, ref_dw)


def test_arguments_are_checked():
    x, w = normal((4, 64), BF16, 1), normal((64,), BF16, 2)
    for bad in (dict(residual=x[:3]), dict(w=w[:60].contiguous()), dict(w=w.float()), dict(block=64), dict(y8=torch.empty(4, 64, device="cuda", dtype=E4M3)),
                dict(block=32, scales=torch.empty(4, 1, device="cuda")), dict(residual=x.float()), dict(residual=x.T)):
        with pytest.raises(ValueError):
            pf.pf_add_rms_norm_fwd(x, **bad)
    with pytest.raises(TypeError):
        pf.pf_add_rms_norm_fwd(x.half())
    with pytest.raises(pf.PfError):
        pf.pf_add_rms_norm_fwd(x[:1].expand(4, 64), x)
    with pytest.raises(pf.PfError):
        pf.pf_add_rms_norm_fwd(normal((1, 16392), BF16, 1))
    with pytest.raises(pf.PfError):
        pf.pf_add_rms_norm_bwd(x, w, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("block", [0, 32, 128])
@pytest.mark.parametrize("width", [256, 333])
def test_codes_of_the_largest_numbers(dtype, block, width):
    """Weights up to 3e38: blocks whose largest number is above 2^126 have codes up to 448 as any other."""
    x = normal((6, width), F32, 1).sign().to(dtype)      # (n is 1 or -1)
    w = torch.tensor([1.0, 1e30, 8e37, 9e37, 1.8e38, 3e38])[torch.arange(width) // 32 % 6].to(dtype).cuda()
    _, y, y8, scales = pf.pf_add_rms_norm_fwd(x, None, w, block=block)
    _, _, want, slack = ref.norm(x, None, w, 1e-6)
    close(y, want, slack, "y")
    check_codes(y8, scales, want, slack, block)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("width", [40, 64, 200, 512, 777, 1200, 2500, 4096, 9000, 16384])
def test_rows_with_an_infinity_are_nan_throughout(dtype, width):
    """Rows with an infinity or a NaN, given or from the sum: NaN in every element, code and scale, and in every element of their gradient; others are as without them."""
    x, r, g, w = (normal((7, width), dtype, i) for i in range(4))
    want = pf.pf_add_rms_norm_fwd(x, r, w[0], block=32)
    want_dx = pf.pf_add_rms_norm_bwd(want[0], w[0], g, dh=r, need_dw=False)[0]
    x[1, width // 2], x[3, 0], r[5, width - 1] = float("inf"), float("nan"), float("-inf")
    x[6, 3] = r[6, 3] = torch.finfo(dtype).max      # (their sum is infinite)
    bad, good = [1, 3, 5, 6], [0, 2, 4]
    h, y, y8, scales = pf.pf_add_rms_norm_fwd(x, r, w[0], block=32)
    y80, scales0 = pf.pf_add_rms_norm_fwd(x, r, w[0], block=0, want_y=False)[2:]
    dx = pf.pf_add_rms_norm_bwd(h, w[0], g, dh=r, need_dw=False)[0]
    for t, plain in ((y, want[1]), (y8.float(), want[2].float()), (scales, want[3]), (dx, want_dx)):
        assert torch.isnan(t[bad]).all() and torch.equal(t[good], plain[good])
    for t in (y80.float(), scales0):
        assert torch.isnan(t[bad]).all() and torch.isfinite(t[good]).all()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-30])
@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("width", [5, 64, 200, 512, 1200, 2500, 4096, 9000, 16384])
def test_rows_whose_squares_leave_the_range(dtype, eps, layout, width):
    """Rows of every size that the types hold, beside one another in a block: h^2 is beyond fp32 from 10^19 on and nothing (where eps is, too) from 10^-23 down."""
    sizes = [1.0, 1e15, 1e19, 1e25, 1e38, 1e-10, 3e17, 1e36] + ([1e-18, 1e-20, 1e-25, 1e-30] if eps < 1e-20 else [])
    tokens = 2 * len(sizes) + 1
    size = torch.tensor(sizes + [1.0] + sizes)[:, None].cuda()
    how = layout_of(layout, width)
    # (three values of either sign, none of them near nothing: sums are as relatively exact as those of normal rows)
    pick = lambda seed: torch.tensor([0.5, 1.0, 2.5])[torch.randint(0, 3, (tokens, width), generator=torch.Generator().manual_seed(seed))].cuda()  # noqa: E731
    x = Rows(tokens, width, dtype, **how).fill((pick(1) * normal((tokens, width), F32, 2).sign() * size).to(dtype))
    w = (1 + normal((width,), F32, 3, 0.3)).to(dtype)
    _, y, y8, scales = pf.pf_add_rms_norm_fwd(x.t, None, w, eps=eps, block=128)
    _, _, want, slack = ref.norm(x.t, None, w, eps)
    close(y, want, slack, "y")
    check_codes(y8, scales, want, slack, 128)
    g = normal((tokens, width), dtype, 4)
    g = torch.where(size < 1e-4, (g.double() * size).to(dtype), g)      # (gradients of tiny rows are as large as those are small)
    dx, dw = pf.pf_add_rms_norm_bwd(x.t, w, g, eps=eps, grads_f32=True)
    want, slack, want_dw, dw_slack = ref.norm_bwd(x.t, w, g, None, eps)
    # (r below the normal numbers has fewer bits: 2^-149, of what stands beside it; and below 2^-126 bf16's numbers are 2^-133 apart: half a step is 2^-134, not 2^-8 of the value)
    close(dx, want, slack + 2.0 ** -146 * (1 + g.double().abs()) + (2.0 ** -134 if dtype == BF16 else 0.0), "dx")
    close(dw, want_dw, dw_slack, "dw")
