"""Without a GPU: what the operators around the layers refuse, and properties of the 8-bit states' format."""
import ctypes

import pytest
import torch

import _ops
import paper_2103_03936_b200 as pf
from paper_2103_03936_b200 import build as pf_build

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 0x7F0000001000  # fake, aligned "device pointer"; never dereferenced


@pytest.fixture(scope="module")
def L():
    pf_build.build()
    return pf.lib()


# ---------------------------------------------------------------------------- experts
def test_rows():
    assert pf.pf_expert_rows(10, 2, 4) == 20 and pf.pf_expert_rows(10, 2, 4, 7) == 28
    assert pf.pf_expert_rows(-1, 2, 4) == 0 and pf.pf_expert_rows(10, 0, 4) == 0 and pf.pf_expert_rows(10, 2, 4, -1) == 0


def test_rows_of_refused_sizes():
    """None, so that a caller who sizes `sources` by them asks for no memory (or for a product that wrapped)."""
    for sizes in ((10, 2, 4, 1 << 29), (10, 2, 2048, 1 << 62), (1 << 30, 2, 4, 0), (1 << 62, 4, 4, 0), (10, 2, 2049, 0), (10, (1 << 16) + 1, 4, 0)):
        assert pf.pf_expert_rows(*sizes) == 0, sizes
    assert pf.pf_expert_rows(1 << 29, 2, 4) == 1 << 30 and pf.pf_expert_rows(1, 1, 4, 1 << 28) == 1 << 30


def test_queries_of_numbers_beyond_the_c_types():
    """4 more than 2^32 experts are not 4."""
    for sizes in ((10, 2, (1 << 32) + 4, 7), (10, (1 << 32) + 2, 4, 7), ((1 << 64) + 10, 2, 4, 0), (10, 2, 4, (1 << 64) + 7)):
        assert pf.pf_expert_rows(*sizes) == 0, sizes
    assert pf.pf_expert_sort_workspace(100000, 2, (1 << 32) + 64) == 0 and pf.pf_expert_sort_workspace((1 << 64) + 100000, 2, 64) == 0
    for sizes in (((1 << 64) + 5, 4, 2, 16), (5, (1 << 32) + 4, 2, 16), (5, 4, 1 << 32, 16), (5, 4, 2, (1 << 32) + 16)):
        assert pf.pf_qk_norm_rope_bwd_workspace(*sizes) == 0, sizes


def test_sort_refuses(L):
    def call(**kw):
        a = dict(ids=P, tokens=10, k=2, experts=4, capacity=0, slots=P, sources=P, counts=P, offsets=P, ws=0, wsb=0, stream=0) | kw
        return L.pf_expert_sort(*a.values())
    for name in ("ids", "slots", "sources", "counts", "offsets"):
        assert call(**{name: 0}) == INVALID and call(**{name: P + 2}) == INVALID
    assert call(tokens=-1) == INVALID and call(k=0) == INVALID and call(experts=0) == INVALID and call(capacity=-1) == INVALID
    assert call(experts=2049) == UNSUPPORTED and call(tokens=1 << 30) == UNSUPPORTED and call(capacity=1 << 29) == UNSUPPORTED
    need = pf.pf_expert_sort_workspace(100000, 2, 64)
    assert need > 0 and need % 256 == 0 and pf.pf_expert_sort_workspace(100, 2, 64) == 0 and pf.pf_expert_sort_workspace(100000, 2, 4000) == 0
    for ws, room in ((0, need), (P + 16, need), (P, need - 1)):
        assert call(tokens=100000, experts=64, ws=ws, wsb=room) == WORKSPACE


def test_rows_are_refused(L):
    base = dict(tokens=10, k=2, rows=20, width=8, dtype=1, stream=0)
    calls = {
        "pf_expert_dispatch_fwd": dict(x=P, ldx=8, slots=P, sources=P, xs=P, ldxs=8),
        "pf_expert_dispatch_bwd": dict(dxs=P, lddxs=8, slots=P, dx=P, lddx=8),
        "pf_expert_combine_fwd": dict(ys=P, ldys=8, slots=P, weights=P, y=P, ldy=8),
        "pf_expert_combine_bwd": dict(ys=P, ldys=8, slots=P, sources=P, weights=P, dy=P, lddy=8, dys=P, lddys=8, dweights=P)}
    for entry, own in calls.items():
        call = lambda **kw: getattr(L, entry)(*(own | base | kw).values())  # noqa: E731
        for name in own:
            if name.startswith("ld"):
                assert call(**{name: 7}) == INVALID, (entry, name)
            else:
                assert call(**{name: P + 1}) == INVALID, (entry, name)
                if name not in ("dys", "dweights") and (entry, name) != ("pf_expert_combine_fwd", "weights"):
                    assert call(**{name: 0}) == INVALID, (entry, name)
        assert call(tokens=-1) == INVALID and call(k=0) == INVALID and call(rows=-1) == INVALID and call(width=0) == INVALID and call(dtype=5) == INVALID
        assert call(tokens=1 << 30) == UNSUPPORTED and call(rows=(1 << 30) + 1) == UNSUPPORTED
        assert call(width=(1 << 28) + 1, **{n: 1 << 29 for n in own if n.startswith("ld")}) == UNSUPPORTED
    assert L.pf_expert_combine_bwd(*(calls["pf_expert_combine_bwd"] | dict(dys=0, dweights=0) | base).values()) == INVALID
    # nothing to write
    assert L.pf_expert_dispatch_fwd(0, 8, 0, 0, 0, 8, 0, 2, 0, 8, 1, 0) == OK
    assert L.pf_expert_combine_fwd(P, 8, 0, P, 0, 8, 0, 2, 20, 8, 1, 0) == OK
    assert L.pf_expert_combine_bwd(0, 8, 0, 0, 0, 0, 8, 0, 8, 0, 0, 2, 0, 8, 1, 0) == OK


# ---------------------------------------------------------------------------- norm and rotation
FWD = dict(q=P, ldq=64, sq=16, k=P, ldk=32, sk=16, wq=P, wk=P, positions=P, inv_freq=P, qo=P, ldqo=64, sqo=16, ko=P, ldko=32, sko=16)
SIZES = dict(tokens=5, q_heads=4, k_heads=2, dim=16, rot=16, style=0, eps=1e-6, dtype=1)
BWD = dict(list(FWD.items())[:10]) | dict(gq=P, ldgq=64, sgq=16, gk=P, ldgk=32, sgk=16, dq=P, lddq=64, sdq=16, dk=P, lddk=32, sdk=16, dwq=P, dwk=P)


def test_norm_rope_refuses(L):
    def fwd(**kw):
        return L.pf_qk_norm_rope_fwd(*(FWD | SIZES | dict(stream=0) | kw).values())

    def bwd(**kw):
        return L.pf_qk_norm_rope_bwd(*(BWD | SIZES | dict(flags=0, ws=P, wsb=1 << 24, stream=0) | kw).values())
    for call, names in ((fwd, ("q", "k", "qo", "ko")), (bwd, ("q", "k", "gq", "gk", "dq", "dk"))):
        for name in names:
            assert call(**{name: 0}) == INVALID and call(**{name: P + 1}) == INVALID, name
            assert call(**{"s" + name: 15}) == INVALID and call(**{"ld" + name: 31}) == INVALID and call(**{"ld" + name: -64}) == INVALID, name
        assert call(wq=P + 1) == INVALID and call(inv_freq=0) == INVALID and call(inv_freq=P + 2) == INVALID and call(positions=P + 4) == INVALID
        assert call(tokens=-1) == INVALID and call(q_heads=-1) == INVALID and call(q_heads=0, k_heads=0) == INVALID and call(dim=0) == INVALID
        assert call(rot=18) == INVALID and call(rot=7) == INVALID and call(rot=-2) == INVALID and call(style=2) == INVALID and call(dtype=3) == INVALID
        assert call(eps=-1.0) == INVALID and call(eps=float("nan")) == INVALID and call(eps=float("inf")) == INVALID
        wide = {n: 1 << 20 for n in FWD | BWD if n.startswith("ld")} | {n: 1100 for n in ("sq", "sk", "sqo", "sko", "sgq", "sgk", "sdq", "sdk")}
        assert call(dim=1025, rot=1024, **{n: v for n, v in wide.items() if n in (FWD if call is fwd else BWD)}) == UNSUPPORTED
    assert fwd(tokens=0) == OK and fwd(tokens=0, q=0, qo=0) == OK
    assert bwd(tokens=0, dwq=0, dwk=0) == OK
    assert bwd(dwq=P + 1) == INVALID and bwd(flags=4) == INVALID and bwd(flags=2, dwk=P + 2) == INVALID
    assert bwd(k_heads=0) == INVALID                                    # dwk without keys
    assert bwd(ws=0) == WORKSPACE and bwd(ws=P + 16) == WORKSPACE and bwd(wsb=64) == WORKSPACE
    assert pf.pf_qk_norm_rope_bwd_workspace(0, 4, 2, 16) == 0 and pf.pf_qk_norm_rope_bwd_workspace(5, 4, 2, 16) >= 4 * 2 * 16


# ---------------------------------------------------------------------------- AdamW
class Hyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("step", ctypes.c_int64), ("grad_scale", ctypes.c_float),
                                                                                                 ("seed", ctypes.c_uint32)]


def test_adamw_refuses(L):
    def call(numels=(8, 0, 5), masters=False, state8=False, pdt=0, gdt=0, state=None, scalars=0, hyper=True, count=None, **kw):
        n = len(numels)
        lists = {name: (ctypes.c_void_p * n)(*[P + 4096 * i for i in range(n)]) for name in ("params", "masters", "grads", "m", "v", "ms", "vs")}
        if not masters:
            lists["masters"] = None
        elif masters is not True:
            lists["masters"][2] = masters
        if not state8:
            lists["ms"] = lists["vs"] = None
        h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, grad_scale=1.0, seed=0)
        for name, value in kw.items():
            if name in h:
                h[name] = value
            elif value is None:
                lists[name] = None
            else:
                lists[name][2] = value      # the last tensor's
        return L.pf_adamw_step(*lists.values(), (ctypes.c_int64 * n)(*numels), n if count is None else count, pdt, gdt,
                               int(state8) if state is None else state, ctypes.byref(Hyper(**h)) if hyper else None, scalars, None)
    for name in ("params", "grads", "m", "v"):
        assert call(**{name: None}) == INVALID and call(**{name: 0}) == INVALID and call(**{name: P + 2}) == INVALID, name
        assert call(state8=True, **{name: 0}) == INVALID, name
    for name in ("ms", "vs"):
        assert call(state8=True, **{name: None}) == INVALID and call(state8=True, **{name: P + 2}) == INVALID and call(state8=True, **{name: 0}) == INVALID
    assert call(pdt=1, params=P + 1) == INVALID and call(gdt=1, grads=P + 1) == INVALID and call(pdt=1, masters=P + 2) == INVALID
    assert call(masters=True) == INVALID                                # masters of fp32 parameters
    for name, bad in (("beta1", 1.0), ("beta1", -0.1), ("beta2", 1.0), ("beta2", float("nan")), ("eps", -1.0), ("eps", float("inf")),
                      ("weight_decay", float("nan")), ("lr", float("inf")), ("step", 0), ("step", -3), ("grad_scale", float("nan"))):
        assert call(**{name: bad}) == INVALID, (name, bad)
    assert call(pdt=2) == INVALID and call(gdt=-1) == INVALID and call(state=2) == INVALID and call(hyper=False) == INVALID and call(count=-1) == INVALID
    assert call(numels=(8, -1, 5)) == INVALID and call(numels=(8, 1, (1 << 42) + 1)) == UNSUPPORTED and call(scalars=P + 2) == INVALID
    assert call(numels=()) == OK and call(numels=(0, 0, 0), params=0, m=0) == OK


def test_tensors_on_the_host_are_refused():
    t = torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA"):
        pf.pf_adamw_step([t], [t], [t], [t])
    with pytest.raises(ValueError, match="CUDA"):
        pf.pf_expert_sort(torch.zeros(4, 2, dtype=torch.int32), 3)
    with pytest.raises(ValueError, match="CUDA"):
        pf.pf_qk_norm_rope_fwd(torch.zeros(2, 3, 8), None, None, None, torch.zeros(4))
    with pytest.raises(TypeError, match="q or k"):
        pf.pf_qk_norm_rope_fwd(None, None, None, None, torch.zeros(4))
    assert pf.pf_adamw_step([], [], [], []) is None


def test_scalars_of_a_replayed_step():
    t = pf.pf_adamw_scalars(lr=1e-3, betas=(0.9, 0.98), step=7, grad_scale=0.5, seed=0xFFFFFFFE)
    assert t.dtype == torch.float32 and t[:4].tolist() == torch.tensor([1e-3, 1 - 0.9 ** 7, 1 - 0.98 ** 7, 0.5]).tolist()
    assert int(t.view(torch.int32)[4]) == -2 and int(pf.pf_adamw_scalars(lr=1.0, step=1, seed=5).view(torch.int32)[4]) == 5


def test_scalars_refuse_what_the_step_refuses():
    """Step 0 has corrections of zero, which would make every parameter infinite."""
    for bad in (dict(step=0), dict(step=-1), dict(step=1, seed=-1), dict(step=1, seed=1 << 32)):
        with pytest.raises(ValueError):
            pf.pf_adamw_scalars(lr=1e-3, **bad)


def test_scalars_refuse_what_would_make_every_parameter_infinite_or_nan():
    """beta = 1 has a correction of zero; lr and grad_scale as the step refuses them."""
    for bad in (dict(betas=(1.0, 0.98)), dict(betas=(0.9, 1.0)), dict(betas=(-0.1, 0.9)), dict(betas=(0.9, float("nan"))), dict(lr=float("inf")),
                dict(lr=float("nan")), dict(grad_scale=float("nan")), dict(grad_scale=-float("inf"))):
        with pytest.raises(ValueError):
            pf.pf_adamw_scalars(**(dict(lr=1e-3, step=1) | bad))
    assert pf.pf_adamw_scalars(lr=0.0, betas=(0.0, 0.0), step=3)[:4].tolist() == [0.0, 1.0, 1.0, 1.0]


@pytest.mark.parametrize("e4m3", [True, False])
def test_rounding_of_states_is_fair(e4m3):
    """Mean of what a value is rounded to over the random bits of many places and seeds: the value itself, to the spread of the mean
    (half a step at most, over the root of the count; five of those) and the 2^-16 steps of the bits."""
    step = 2.0 ** -3 if e4m3 else 2.0 ** -2
    x = torch.full((1 << 16,), 1.30859375)
    bits = torch.cat([_ops.noise(1 << 13, seed, tensor) for seed in (0, 1, 2, 77) for tensor in (0, 5)])
    half = bits & 0xFFFF if e4m3 else bits >> 16
    values = _ops.decode(*_ops.encode(x, half, e4m3))
    assert set(values.tolist()) <= {1.25, 1.375} if e4m3 else set(values.tolist()) <= {1.25, 1.5}
    assert abs(float(values.double().mean()) - 1.30859375) < 5 * step / 2 / 256 + step * 2.0 ** -16
    # the two halves of the bits do not go together, nor do neighbours
    a, b = (bits & 0xFFFF).double() / 65536 - 0.5, (bits >> 16).double() / 65536 - 0.5
    for u, v in ((a, b), (a[1:], a[:-1]), (b[1:], b[:-1]), (a[256:], a[:-256])):
        assert abs(float((u * v).mean()) * 12) < 5 / 256                # correlation of 65536 independent pairs: 1 / 256


def test_states_at_the_ends_of_the_format():
    big = torch.tensor([3.0e38, -3.0e38, 1e30, 0.0, 1e-45, -1e-40])
    m, s = _ops.encode(big, torch.full((6,), 0xFFFF), True)
    assert torch.isfinite(_ops.decode(m, s)).all() and _ops.decode(m, s)[3:].tolist() == [0, 0, 0]
    v, s = _ops.encode(big.abs(), torch.full((6,), 0xFFFF), False)
    assert torch.isfinite(v.float()).all() and v.float()[3] == 0 and (v.float()[4:] == 2.0 ** -14).all()
    # the least scale of m is 2^-119: what is below 2^-6 of it, that is below 2^-125 = 2.4e-38, is zero
    tiny, s = _ops.encode(torch.tensor([1e-38, 2e-38, 2.0 ** -125]), torch.zeros(3, dtype=torch.long), True)
    assert s[0] == 2.0 ** -119 and tiny.float().tolist() == [0, 0, 2.0 ** -6]
