"""A wait that runs out ends its kernel with a status: no thread is left behind at a barrier, other blocks' rows are whole, and the device goes on.  (Kernels compiled
with barriers of some blocks that expect more than is copied: tests/device.)"""
import ctypes
import os
import subprocess
import time

import pytest
import torch

import paper_2103_03936_b200 as pf
from paper_2103_03936_b200 import build as pf_build

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
TIMEOUT = 5      # of the status word
SECONDS = 20     # two limits of two seconds each, and room


def built(tmp_path_factory, name):
    path = str(tmp_path_factory.mktemp("waits") / f"lib{name}.so")
    include = ["-I", os.path.join(pf_build.ROOT, "include"), "-I", pf_build.CSRC]
    subprocess.check_call([pf_build.nvcc()] + pf_build.NVCC_FLAGS + include + ["-shared", "-o", path, os.path.join(HERE, "device", name + ".cu")])
    return ctypes.CDLL(path)


@pytest.fixture(scope="module")
def waits(tmp_path_factory):
    lib = built(tmp_path_factory, "vocab_waits")
    for name in ("pf_logprobs_fwd", "pf_logprobs_bwd", "pf_distill_fwd", "pf_distill_bwd"):
        getattr(lib, name).argtypes = getattr(pf.lib(), name).argtypes
    torch.zeros(1, device="cuda")
    assert lib.waits_status() == 0
    return lib


@pytest.fixture
def rows(request):
    tokens, vocab = request.param
    g = torch.Generator().manual_seed(1)
    z = (torch.randn((tokens, vocab), generator=g) * 2).to(torch.bfloat16).cuda()
    return z, torch.randint(0, vocab, (tokens,), generator=g).cuda()


def whole(tokens, vocab, blocks, parts):
    """Rows that no block with such a barrier has worked on, nor would have after it."""
    return [r for r in range(tokens) if all((r * parts + i if parts > 1 else r % blocks) % 64 != 5 for i in range(parts))]


def gives_up(lib, call):
    start = time.time()
    assert call() == 0
    assert lib.waits_status() == TIMEOUT and time.time() - start < SECONDS


LONG, PARTS = (900, 40001), (9, 70000)      # through a ring, 444 blocks; in 8 parts
KEEP = {LONG: whole(*LONG, 444, 1), PARTS: whole(*PARTS, 0, 8)}


@pytest.mark.parametrize("top", [0, 8])
@pytest.mark.parametrize("rows", [LONG, PARTS], indirect=True)
def test_log_probabilities(waits, rows, top):
    z, ids = rows
    tokens, vocab = z.shape
    want = pf.pf_logprobs_fwd(z, ids, top=top, want_entropy=True, want_lse=True)
    got = [None if t is None else torch.zeros_like(t) for t in want]
    p = [None if t is None else t.data_ptr() for t in got]
    torch.cuda.synchronize()
    gives_up(waits, lambda: waits.pf_logprobs_fwd(z.data_ptr(), vocab, ids.data_ptr(), 1.0, p[0], p[1], p[2], top, p[3], p[4], tokens, vocab, pf.PF_BF16, None))
    keep = KEEP[tokens, vocab]
    assert len(keep) > tokens // 2
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, want) if a is not None)
    # the device, and the same rows, go on
    again = pf.pf_logprobs_fwd(z, ids, top=top, want_entropy=True, want_lse=True)
    assert all(torch.equal(a, b) for a, b in zip(again, want) if a is not None) and pf.pf_last_device_status() == 0


@pytest.mark.parametrize("rows", [LONG, PARTS], indirect=True)
def test_gradients_and_divergences(waits, rows):
    z, ids = rows
    tokens, vocab = z.shape
    t_ids, teacher = torch.stack((ids, (ids + 5) % vocab), 1), torch.zeros(tokens, 2, device="cuda")
    ones = torch.ones(tokens, device="cuda")
    keep = KEEP[tokens, vocab]
    want, got = pf.pf_distill_fwd(z, t_ids, teacher), torch.zeros(tokens, device="cuda")
    torch.cuda.synchronize()
    gives_up(waits, lambda: waits.pf_distill_fwd(z.data_ptr(), vocab, t_ids.data_ptr(), teacher.data_ptr(), None, 2, 1.0, got.data_ptr(), tokens, vocab, pf.PF_BF16, None))
    assert torch.equal(got[keep], want[keep])
    if (tokens, vocab) == LONG:
        return
    want, dz = pf.pf_logprobs_bwd(z, ids, ones, ones)[0], torch.zeros_like(z)
    torch.cuda.synchronize()
    gives_up(waits, lambda: waits.pf_logprobs_bwd(z.data_ptr(), vocab, ids.data_ptr(), 1.0, ones.data_ptr(), ones.data_ptr(), dz.data_ptr(), vocab, None, None, tokens, vocab,
                                                  pf.PF_BF16, None))
    assert torch.equal(dz[keep], want[keep])


@pytest.fixture(scope="module")
def gates(tmp_path_factory):
    lib = built(tmp_path_factory, "gated_waits")
    lib.waits_gated.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_longlong] * 3
    return lib


@pytest.mark.parametrize("r,backward", [(64, False), (256, False), (320, False), (64, True)])
def test_gates(gates, r, backward):
    """Pairs of blocks, of which one's barriers count the copies of both."""
    lib, m, n = gates, 4096, 2048
    g = torch.Generator().manual_seed(r)
    T, V = (torch.randn(s, generator=g).mul_(r ** -0.25).to(torch.bfloat16).cuda() for s in ((2, m, r), (2, n, r)))
    dY = torch.randn((m, n), generator=g).to(torch.bfloat16).cuda()
    z = T.double() @ V.double().transpose(1, 2)
    s = torch.sigmoid(z[0])
    want = torch.stack((dY.double() * z[1] * (s + z[0] * s * (1 - s)), dY.double() * z[0] * s)) if backward else (z[0] * s * z[1])[None]
    out = torch.zeros((2 if backward else 1, m, n), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    gives_up(lib, lambda: lib.waits_gated(T.data_ptr(), V.data_ptr(), dY.data_ptr() if backward else None, out.data_ptr(), m, n, r))
    # tiles of 256 x 128: a run of neighbouring ones to a pair, or every pairs-th
    pairs, tiles = 74, [(i // 16, i % 16) for i in range(256)]
    of = [next(p for p in range(pairs) if 256 * p // pairs <= i < 256 * (p + 1) // pairs) if not backward and r <= 256 else i % pairs for i in range(256)]
    kept = [t for t, p in zip(tiles, of) if 2 * p % 64 != 4]
    assert len(kept) > 200
    for a, b in kept:
        at = (slice(None), slice(256 * a, 256 * a + 256), slice(128 * b, 128 * b + 128))
        assert float((out[at].double() - want[at]).norm()) <= 1e-2 * float(want[at].norm())
    x, U = torch.ones((8, 16), dtype=torch.bfloat16, device="cuda"), torch.ones((2, 16, 8), dtype=torch.bfloat16, device="cuda")
    y = pf.pf_lowrank_linear_gated_fwd(x, U, U)      # (the device goes on: g = u = 128 throughout)
    assert torch.equal(y, torch.full_like(y, 16384.0)) and pf.pf_last_device_status() == 0
