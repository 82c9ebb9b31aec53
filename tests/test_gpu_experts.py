"""GPU parity of the experts' sort, dispatch and combine against plain forms in 64 bits."""
import os
import subprocess
import sys

import pytest
import torch

import _ops
import paper_2103_03936_b200 as pf
from _gpu import Scratch

pytestmark = pytest.mark.gpu
DT = [torch.bfloat16, torch.float32]


def choose(tokens, k, experts, seed, bad=0.0):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, experts, (tokens, k), generator=g)
    if bad:
        out = torch.rand((tokens, k), generator=g) < bad
        ids = torch.where(out, torch.randint(0, 2, (tokens, k), generator=g) * (experts + 70000) - 1, ids)      # -1 and beyond the last
    return ids.to(torch.int32)


def guarded(shape, dtype, pitch=None, fill=-7):
    """An output inside a larger buffer: (tensor, check that nothing around it was written)."""
    rows, cols = (1, shape[0]) if len(shape) == 1 else shape
    pitch = pitch or cols
    buf = torch.full((rows * pitch + 128,), fill, dtype=dtype, device="cuda")
    t = buf[64:64 + rows * pitch].view(rows, pitch)[:, :cols]

    def check():
        assert (buf[:64] == fill).all() and (buf[64 + rows * pitch:] == fill).all(), "written outside"
        assert (buf[64:64 + rows * pitch].view(rows, pitch)[:, cols:] == fill).all(), "written between rows"
    return (t if len(shape) == 2 else t.view(-1)), check


def sorted_rows(ids, experts, capacity):
    rows = pf.pf_expert_rows(*ids.shape, experts, capacity)
    outs = [guarded(s, torch.int32) for s in (tuple(ids.shape), (rows,), (experts,), (experts + 1,))]
    got = pf.pf_expert_sort(ids.cuda(), experts, capacity=capacity, **{n: o[0] for n, o in zip(("slots", "sources", "counts", "offsets"), outs)})
    for o in outs:
        o[1]()
    return got


@pytest.mark.parametrize("tokens,k,experts,capacity", [
    (1, 1, 1, 0), (1, 2, 8, 0), (3, 1, 2, 1), (20, 2, 8, 0), (31, 1, 5, 4), (33, 3, 7, 9), (512, 1, 3, 0), (511, 2, 64, 20), (1111, 3, 61, 0),
    (2000, 8, 256, 70), (4097, 1, 1, 5000), (5000, 4, 2048, 12), (777, 5, 513, 0), (16384, 2, 64, 640), (40000, 8, 1000, 0), (9000, 7, 2, 31000),
    (16385, 2, 64, 0), (33000, 1, 3, 12000), (50001, 3, 2048, 70), (100000, 2, 7, 0)])
def test_sort(tokens, k, experts, capacity):
    for seed, bad in ((1, 0.0), (2, 0.3)):
        ids = choose(tokens, k, experts, seed, bad)
        got = sorted_rows(ids, experts, capacity)
        for g, w, name in zip(got, _ops.sort(ids.tolist(), experts, capacity), ("slots", "sources", "counts", "offsets")):
            assert g.reshape(-1).tolist() == w, name


@pytest.mark.parametrize("tokens,k,experts", [(32769, 1, 2048), (200001, 1, 5), (60000, 8, 256)])
def test_a_workspace_of_the_queried_size(tokens, k, experts):
    ids = choose(tokens, k, experts, 4).cuda()
    scratch = Scratch(pf.pf_expert_sort_workspace(tokens, k, experts))
    got = pf.pf_expert_sort(ids, experts, workspace=scratch.t)
    scratch.check()
    order = torch.sort(ids.flatten(), stable=True).indices
    assert torch.equal(got[1].long(), order) and torch.equal(got[0].flatten().long()[order], torch.arange(tokens * k, device="cuda"))
    for a, b in zip(got, pf.pf_expert_sort(ids, experts)):
        assert torch.equal(a, b)


def test_sort_where_shared_memory_reaches_48_kb():
    """Numbers of experts around those at which a block needs more than 48 KB, in a process that has not sorted for more of them."""
    code = """
import torch, paper_2103_03936_b200 as pf
for tokens in (500, 20000):
    for experts in (640, *range(643, 650)):
        ids = torch.randint(experts, (tokens, 2), dtype=torch.int32, device="cuda")
        order = pf.pf_expert_sort(ids, experts)[1]
        assert torch.equal(order.long(), torch.sort(ids.flatten(), stable=True).indices), (tokens, experts)
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0, done.stderr


def test_sort_of_one_expert_and_of_none():
    """All tokens at the last expert, beyond its capacity; no valid id at all; no tokens."""
    ids = torch.full((3000, 2), 6, dtype=torch.int32)
    for capacity in (0, 100):
        for g, w in zip(sorted_rows(ids, 7, capacity), _ops.sort(ids.tolist(), 7, capacity)):
            assert g.reshape(-1).tolist() == w
    slots, sources, counts, offsets = sorted_rows(torch.full((50, 3), -1, dtype=torch.int32), 4, 10)
    assert (slots == -1).all() and (sources == -1).all() and (counts == 0).all() and offsets.tolist() == [0, 10, 20, 30, 40]
    for capacity in (0, 3):
        slots, sources, counts, offsets = sorted_rows(torch.empty((0, 3), dtype=torch.int32), 4, capacity)
        assert slots.shape == (0, 3) and (sources == -1).all() and (counts == 0).all() and offsets.tolist() == [i * capacity for i in range(5)]


def normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def padded(t, pitch, shift):
    """The same matrix at another pitch, `shift` elements behind a 256-byte boundary."""
    buf = torch.full((t.shape[0] * pitch + shift + 8,), float("nan"), dtype=t.dtype, device="cuda")
    out = buf[shift:shift + t.shape[0] * pitch].view(t.shape[0], pitch)[:, :t.shape[1]]
    out.copy_(t)
    return out


WIDTHS = [(1, 1, 0), (7, 7, 0), (64, 64, 0), (512, 512, 0), (1500, 1500, 0), (255, 257, 1), (1030, 1032, 2), (1030, 1036, 4), (2056, 2056, 8), (4096, 4096, 0)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("width,pitch,shift", WIDTHS)
@pytest.mark.parametrize("tokens,k,experts,capacity", [(1, 1, 1, 0), (20, 2, 8, 0), (133, 3, 7, 40), (300, 6, 5, 500)])
def test_rows_there_and_back(dtype, width, pitch, shift, tokens, k, experts, capacity):
    ids = choose(tokens, k, experts, 3, 0.1)
    slots, sources, counts, offsets = pf.pf_expert_sort(ids.cuda(), experts, capacity=capacity)
    rows = sources.shape[0]
    keep = slots >= 0
    x, ys, dy, dxs = (normal((n, width), dtype, s) for n, s in ((tokens, 4), (rows, 5), (tokens, 6), (rows, 7)))
    ys[sources < 0] = float("nan")                      # what no token reads may hold anything
    dxs[sources < 0] = float("inf")
    w = torch.randn((tokens, k), generator=torch.Generator().manual_seed(8)).cuda()
    w[~keep] = float("nan")
    x, ys, dy, dxs = (padded(t, pitch, shift) for t in (x, ys, dy, dxs))
    out = {n: guarded((r, width), dtype, pitch) for n, r in (("xs", rows), ("y", tokens), ("dys", rows), ("dx", tokens))}
    dw, dw_check = guarded((tokens, k), torch.float32)
    pf.pf_expert_dispatch_fwd(x, slots, sources, xs=out["xs"][0])
    pf.pf_expert_combine_fwd(ys, slots, w, y=out["y"][0])
    pf.pf_expert_combine_bwd(ys, slots, sources, w, dy, dys=out["dys"][0], dweights=dw)
    pf.pf_expert_dispatch_bwd(dxs, slots, dx=out["dx"][0])
    dw_check()
    for _, check in out.values():
        check()
    token = sources.clamp(min=0).long() // k
    used = (sources >= 0)[:, None]
    assert torch.equal(out["xs"][0], torch.where(used, x[token], torch.zeros((), dtype=dtype, device="cuda")))
    # sums of k products, each rounded: k + 1 times 2^-24 of the magnitudes
    wk = torch.where(keep, w, 0.0).double()
    parts = _ops.rows_of(torch.nan_to_num(ys), slots) * wk.unsqueeze(-1)
    _ops.close(out["y"][0], parts.sum(1), (k + 1) * 2.0 ** -24 * parts.abs().sum(1), "y")
    parts = _ops.rows_of(torch.nan_to_num(dxs), slots)
    _ops.close(out["dx"][0], parts.sum(1), (k + 1) * 2.0 ** -24 * parts.abs().sum(1), "dx")
    flat = torch.where(keep, w, 0.0).reshape(-1).double()[sources.clamp(min=0).long()]
    want = torch.where(used, dy.double()[token] * flat[:, None], 0.0)
    _ops.close(out["dys"][0], want, 2.0 ** -23 * want.abs(), "dys")
    # a lane adds up to width / 32 products, then five sums of lanes and eight of warps
    parts = _ops.rows_of(torch.nan_to_num(ys), slots) * dy.double().unsqueeze(1)
    _ops.close(dw, parts.sum(-1), (width / 32 + 40) * 2.0 ** -24 * parts.abs().sum(-1), "dweights")
    assert (dw[~keep] == 0).all()


def test_a_part_of_the_backward_and_no_weights():
    slots, sources, _, _ = pf.pf_expert_sort(choose(90, 3, 4, 1).cuda(), 4, capacity=80)
    ys, dy, w = normal((320, 136), torch.bfloat16, 1), normal((90, 136), torch.bfloat16, 2), torch.rand(90, 3, device="cuda")
    dys, dw = pf.pf_expert_combine_bwd(ys, slots, sources, w, dy)
    assert torch.equal(pf.pf_expert_combine_bwd(ys, slots, sources, w, dy, need_dys=False)[1], dw)
    only, none = pf.pf_expert_combine_bwd(ys, slots, sources, w, dy, need_dweights=False)
    assert none is None and torch.equal(only, dys)
    assert torch.equal(pf.pf_expert_combine_fwd(ys, slots), pf.pf_expert_combine_fwd(ys, slots, torch.ones_like(w)))
    assert torch.equal(pf.pf_expert_combine_fwd(ys, slots), pf.pf_expert_dispatch_bwd(ys, slots))


def test_no_tokens_and_no_rows():
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    slots, sources, _, _ = pf.pf_expert_sort(none, 3, capacity=4)
    x = torch.empty((0, 40), dtype=torch.bfloat16, device="cuda")
    xs = pf.pf_expert_dispatch_fwd(x, slots, sources, xs=torch.full((12, 40), 3.0, dtype=torch.bfloat16, device="cuda"))
    assert (xs == 0).all()
    dys, dw = pf.pf_expert_combine_bwd(xs, slots, sources, torch.empty((0, 2), device="cuda"), x)
    assert (dys == 0).all() and dw.shape == (0, 2) and pf.pf_expert_combine_fwd(xs, slots).shape == (0, 40)
    slots, sources, _, _ = pf.pf_expert_sort(none, 3)
    assert sources.shape == (0,) and pf.pf_expert_dispatch_fwd(x, slots, sources).shape == (0, 40)


def test_indexes_outside_the_rows_count_as_none():
    slots = torch.tensor([[0, 5], [1 << 30, -9], [2, 1]], dtype=torch.int32, device="cuda")
    ys, dy = normal((3, 24), torch.float32, 1), normal((3, 24), torch.float32, 2)
    sources = torch.tensor([0, 5, 4], dtype=torch.int32, device="cuda")
    y = pf.pf_expert_combine_fwd(ys, slots)
    assert torch.equal(y, torch.stack([ys[0], torch.zeros_like(ys[0]), ys[2] + ys[1]]))
    dys, dw = pf.pf_expert_combine_bwd(ys, slots, sources, torch.ones(3, 2, device="cuda"), dy)
    assert torch.equal(dys, dy[[0, 2, 2]]) and dw[0, 1] == 0 and (dw[1] == 0).all()
    assert torch.equal(pf.pf_expert_dispatch_fwd(dy, slots, sources), dy[[0, 2, 2]])


def test_infinities_stay_with_their_tokens():
    slots, sources, _, _ = pf.pf_expert_sort(choose(64, 2, 4, 5).cuda(), 4)
    ys = normal((128, 96), torch.bfloat16, 3)
    bad = 17
    ys[bad, 5] = float("inf")
    ys[bad, 6] = float("nan")
    y = pf.pf_expert_combine_fwd(ys, slots, torch.ones(64, 2, device="cuda"))
    owner = int(sources[bad]) // 2
    wrong = ~torch.isfinite(y.float())
    assert wrong.nonzero().tolist() == [[owner, 5], [owner, 6]] and torch.isinf(y[owner, 5]) and torch.isnan(y[owner, 6])


def test_rows_beyond_32_bits():
    """Rows whose place in their buffer passes 2^31 elements."""
    width, rows = 1 << 18, 8500
    ids = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    slots, sources, _, _ = pf.pf_expert_sort(ids, 1)
    x = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    last = normal((3, width), torch.bfloat16, 1)
    x[-3:] = last
    x[:, 0] = torch.arange(rows, device="cuda") % 64
    xs = pf.pf_expert_dispatch_fwd(x, slots, sources)
    assert torch.equal(xs[-3:], x[-3:]) and torch.equal(xs[:, 0], x[:, 0])
    del xs
    y = pf.pf_expert_combine_fwd(x, slots)
    assert torch.equal(y[-3:], x[-3:]) and torch.equal(y[:, 0], x[:, 0])
    del y
    w = torch.full((rows, 1), 2.0, device="cuda")
    dys, dw = pf.pf_expert_combine_bwd(x, slots, sources, w, x)
    assert torch.equal(dys[-3:], 2 * x[-3:]) and torch.equal(dys[:, 0], 2 * x[:, 0])
    want = x[-3:].double().square().sum(1)
    assert ((dw[-3:, 0].double() - want).abs() <= (width / 32 + 40) * 2.0 ** -24 * want).all()


def test_captured_and_replayed():
    """A whole pass in a CUDA graph, replayed with other choices."""
    ids = choose(257, 2, 6, 1).cuda()
    x, w = normal((257, 128), torch.bfloat16, 1), torch.rand(257, 2, device="cuda")

    def whole():
        slots, sources, _, _ = pf.pf_expert_sort(ids, 6, capacity=70)
        xs = pf.pf_expert_dispatch_fwd(x, slots, sources)
        y = pf.pf_expert_combine_fwd(xs, slots, w)
        return (slots, sources, xs, y) + pf.pf_expert_combine_bwd(xs, slots, sources, w, x)
    whole()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = whole()
    for seed in (2, 3):
        ids.copy_(choose(257, 2, 6, seed))
        x.copy_(normal((257, 128), torch.bfloat16, seed))
        graph.replay()
        for a, b in zip(out, whole()):
            assert torch.equal(a, b)


def test_on_another_stream():
    ids, x = choose(500, 2, 5, 1).cuda(), normal((500, 72), torch.float32, 1)
    want = pf.pf_expert_dispatch_fwd(x, *pf.pf_expert_sort(ids, 5)[:2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    slots, sources, counts, offsets = pf.pf_expert_sort(ids, 5, stream=side)
    got = pf.pf_expert_dispatch_fwd(x, slots, sources, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    call, xs = pf.pf_expert_dispatch_fwd(x, slots, sources, prepare=True)
    xs.zero_()
    call()
    assert torch.equal(xs, want)


def test_a_capacity_that_is_refused_takes_no_memory():
    ids = choose(10, 2, 4, 1).cuda()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    with pytest.raises(pf.PfError) as e:
        pf.pf_expert_sort(ids, 4, capacity=1 << 29)
    assert e.value.status == 2 and torch.cuda.max_memory_allocated() - before < 1 << 20


def test_refusals():
    ids = choose(10, 2, 3, 1).cuda()
    slots, sources, _, _ = pf.pf_expert_sort(ids, 3)
    x, ys, w = normal((10, 16), torch.float32, 1), normal((20, 16), torch.float32, 1), torch.rand(10, 2, device="cuda")
    for call in (lambda: pf.pf_expert_sort(ids.long(), 3), lambda: pf.pf_expert_sort(ids.t(), 3), lambda: pf.pf_expert_sort(ids, 0),
                 lambda: pf.pf_expert_sort(ids, 3, capacity=-1), lambda: pf.pf_expert_sort(ids, 3, slots=slots[:5]),
                 lambda: pf.pf_expert_sort(ids, 3, sources=sources[:7]), lambda: pf.pf_expert_dispatch_fwd(x[:9], slots, sources),
                 lambda: pf.pf_expert_dispatch_fwd(x, slots, sources, xs=ys[:, :8]), lambda: pf.pf_expert_dispatch_fwd(x, slots, sources, xs=ys.bfloat16()),
                 lambda: pf.pf_expert_dispatch_fwd(x.t(), slots, sources), lambda: pf.pf_expert_dispatch_fwd(x, slots.long(), sources),
                 lambda: pf.pf_expert_combine_fwd(ys, slots, w.bfloat16()), lambda: pf.pf_expert_combine_fwd(ys, slots, w[:, :1].contiguous()),
                 lambda: pf.pf_expert_combine_bwd(ys, slots, sources[:19], w, x), lambda: pf.pf_expert_combine_bwd(ys, slots, sources, w, x.bfloat16()),
                 lambda: pf.pf_expert_dispatch_fwd(x.cpu(), slots, sources), lambda: pf.pf_expert_dispatch_fwd(x, slots.cpu(), sources)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pf.pf_expert_dispatch_fwd(x.half(), slots, sources)
    with pytest.raises(pf.PfError) as e:
        pf.pf_expert_sort(ids, 4000)
    assert e.value.status == 2
    with pytest.raises(pf.PfError):
        pf.pf_expert_combine_bwd(ys, slots, sources, w, x, need_dys=False, need_dweights=False)


@pytest.mark.parametrize("tokens,k,experts,capacity", [
    (3, 1, 2, 0), (40, 1, 2, 0), (20, 2, 8, 0), (511, 2, 64, 20), (1111, 3, 61, 0), (2000, 8, 256, 70), (777, 5, 513, 0), (5000, 4, 2048, 12), (1, 2, 1, 1),
    (40000, 1, 7, 0), (33000, 2, 64, 900), (50001, 3, 2048, 70), (32769, 1, 1, 0)])
def test_any_id_outside_the_experts_gets_no_row(tokens, k, experts, capacity):
    """Negative ids of every kind (those whose low bits are an expert's among them) and those beyond the last, alone and in front of all of 32."""
    g = torch.Generator().manual_seed(11)
    bits, low = experts.bit_length(), -(1 << 31)
    pool = [-1, -2, -8, -29, -100, low, low + 1, low + experts - 1, experts, experts + 1, (1 << 31) - 1]
    pool += [-(1 << b) + e for b in (bits, bits + 1, bits + 4, 20, 30) for e in (0, experts // 2, experts - 1)]
    pool = torch.tensor(sorted({i for i in pool if not 0 <= i < experts}))
    for share in (0.1, 0.6):
        ids = torch.randint(0, experts, (tokens * k,), generator=g)
        out = torch.rand(tokens * k, generator=g) < share
        out[::32] = True
        ids = torch.where(out, pool[torch.randint(0, len(pool), (tokens * k,), generator=g)], ids).to(torch.int32).view(tokens, k)
        got = sorted_rows(ids, experts, capacity)
        for a, w, name in zip(got, _ops.sort(ids.tolist(), experts, capacity), ("slots", "sources", "counts", "offsets")):
            assert a.reshape(-1).tolist() == w, name


def test_a_workspace_that_is_no_whole_buffer_on_the_device_is_refused():
    ids = choose(40000, 1, 64, 1).cuda()
    need = pf.pf_expert_sort_workspace(40000, 1, 64)
    for room in (torch.empty(need, dtype=torch.uint8), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2],
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(need)):
        with pytest.raises(ValueError, match="workspace"):
            pf.pf_expert_sort(ids, 64, workspace=room)
        x = torch.zeros(8, 8, device="cuda")
        with pytest.raises(ValueError, match="workspace"):
            pf.pf_lowrank_linear_fwd(x, x, x, workspace=room)
    with pytest.raises(TypeError):
        pf.pf_expert_sort(ids, 64, workspace=need)
    with pytest.raises(pf.PfError) as e:
        pf.pf_expert_sort(ids, 64, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


def test_outputs_dropped_at_once_on_another_stream_are_not_handed_out_again():
    """While the other stream still has to write them: an allocation of the same size on the current stream gets other memory."""
    ids, x, q, f = choose(3000, 2, 5, 1).cuda(), normal((3000, 64), torch.bfloat16, 1), normal((3000, 4, 64), torch.bfloat16, 2), torch.ones(32, device="cuda")
    slots, sources, _, _ = pf.pf_expert_sort(ids, 5, capacity=2000)
    w, side = torch.rand(3000, 2, device="cuda"), torch.cuda.Stream()
    xs = pf.pf_expert_dispatch_fwd(x, slots, sources)
    calls = {"sort": lambda: pf.pf_expert_sort(ids, 5, capacity=2000, stream=side), "dispatch": lambda: pf.pf_expert_dispatch_fwd(x, slots, sources, stream=side),
             "combine": lambda: pf.pf_expert_combine_fwd(xs, slots, w, stream=side),
             "backward": lambda: pf.pf_expert_combine_bwd(xs, slots, sources, w, x, stream=side), "linear": lambda: pf.pf_lowrank_linear_fwd(x, x[:64], x[:64], stream=side),
             "norm": lambda: pf.pf_qk_norm_rope_fwd(q, None, None, None, f, stream=side),
             "norm backward": lambda: pf.pf_qk_norm_rope_bwd(q, None, x[0], None, f, q, None, stream=side)}
    for name, call in calls.items():
        call()                                      # (a first launch loads its kernels, which may wait for the device)
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        with torch.cuda.stream(side):
            torch.cuda._sleep(400_000_000)      # 0.2 s
        out = call()
        out = [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]
        shapes, places = [(t.shape, t.dtype) for t in out], {t.data_ptr() for t in out}
        del out
        again = [torch.empty(s, dtype=d, device="cuda") for s, d in shapes]
        waiting = not side.query()
        assert waiting and not places & {t.data_ptr() for t in again}, name
    torch.cuda.synchronize()


def test_experts_that_are_refused_take_no_memory():
    ids = choose(10, 2, 4, 1).cuda()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    for experts in (2049, 1 << 28):
        with pytest.raises(pf.PfError) as e:
            pf.pf_expert_sort(ids, experts)
        assert e.value.status == 2 and torch.cuda.max_memory_allocated() - before < 1 << 20


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("width,pitch,shift", [(528, 528, 0), (266, 268, 2), (523, 525, 1)])
@pytest.mark.parametrize("k,experts,capacity", [(1, 3, 0), (2, 8, 700), (3, 7, 0), (8, 16, 1400)])
def test_long_rows_of_many_tokens(dtype, width, pitch, shift, k, experts, capacity):
    """Rows longer than a warp of tokens enough for every warp: the backward of combine by a warp to a token."""
    test_rows_there_and_back(dtype, width, pitch, shift, 2500, k, experts, capacity)


def test_captured_on_a_stream_that_joins_the_capture():
    """Calls on another stream inside a capture, their lists dropped at once: the replay has other choices and the same results as eager calls."""
    ids, x = choose(40000, 1, 6, 1).cuda(), normal((40000, 64), torch.bfloat16, 1)
    side = torch.cuda.Stream()

    def whole(stream):
        slots, sources, _, _ = pf.pf_expert_sort(ids, 6, capacity=8000, stream=stream)
        return pf.pf_expert_combine_fwd(pf.pf_expert_dispatch_fwd(x, slots, sources, stream=stream), slots, stream=stream)
    whole(None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        out = whole(side)
        torch.cuda.current_stream().wait_stream(side)
    for seed in (2, 3):
        ids.copy_(choose(40000, 1, 6, seed, 0.1))
        graph.replay()
        assert torch.equal(out, whole(None))
