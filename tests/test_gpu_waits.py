"""A wait that runs out ends its kernel with a status: no thread is left behind at a barrier, other blocks' rows are whole, and the device goes on.  (The kernels over
a vocabulary's rows, compiled with barriers of some blocks that expect more than is copied: tests/device/vocab_waits.cu.)"""
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


@pytest.fixture(scope="module")
def waits(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("waits") / "libwaits.so")
    include = ["-I", os.path.join(pf_build.ROOT, "include"), "-I", pf_build.CSRC]
    subprocess.check_call([pf_build.nvcc()] + pf_build.NVCC_FLAGS + include + ["-shared", "-o", path, os.path.join(HERE, "device", "vocab_waits.cu")])
    lib = ctypes.CDLL(path)
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
