"""Token probabilities with cuts where a CTA of a row's cluster does not send what the others wait for, or sends it after
they have given up waiting: the call ends, the whole row is 0 and flagged, other rows are what they should be.

The kernel is built here with a hook at its sends, which withholds some of them; nothing faults, every wait has its limit
of a second.  Exchanges: 0 the maxima, 1 sums of groups of bins, 2 sums of bins, 3 exact sums, 4 the bin's tokens, 5 the
sum of what is kept."""
import ctypes
import subprocess

import pytest
import torch

from paper_2510_05421_gb300 import build as build_mod
from paper_2510_05421_gb300 import token_probs

pytestmark = pytest.mark.gpu

SOURCE = """
#include "token_probs.cuh"
namespace dvi {
struct Hold { int exchange, from, to, after, late_ms; };
__device__ Hold g_hold;
__device__ unsigned g_seen[8 * 8 * 512];
// Of row 0: whether this thread's message to CTA r goes.
__device__ __forceinline__ bool sends(int k, int r) {
  const Hold h = g_hold;
  const int rank = cg::this_cluster().block_rank();
  if (k != h.exchange || blockIdx.x / cg::this_cluster().num_blocks()) return true;
  if ((h.from >= 0 && rank != h.from) || (h.to >= 0 && r != h.to)) return true;
  if (atomicAdd(&g_seen[(rank * 8 + r) * 512 + threadIdx.x], 1u) < h.after) return true;
  if (!h.late_ms) return false;
  for (const uint64_t t0 = global_ns(); global_ns() - t0 < h.late_ms * 1000000ull;) {
  }
  return true;
}
}  // namespace dvi
#define DVI_SENDS(k, r) sends(k, r)
#include "token_probs_cut.cu"
extern "C" int hold(const dvi::Hold* h) {
  static unsigned none[8 * 8 * 512];
  cudaError_t e = cudaMemcpyToSymbol(dvi::g_hold, h, sizeof *h);
  return e ? e : cudaMemcpyToSymbol(dvi::g_seen, none, sizeof none);
}
extern "C" int probs(const float* x, float* out, int rows, int vocab, float temperature, int top_k, float top_p, int* status,
                     cudaStream_t stream) {
  dvi::TokenProbsArgs a{};
  a.x = x, a.ld = vocab, a.out = out, a.ld_out = vocab, a.n_rows = rows, a.vocab = vocab;
  a.temperature_all = temperature, a.top_k_all = top_k, a.top_p_all = top_p, a.status = status;
  return dvi::launch_probs_cut(a, DVI_F32, stream);
}
"""


class Hold(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("exchange", "from_", "to", "after", "late_ms")]


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    d = tmp_path_factory.mktemp("held")
    (d / "held.cu").write_text(SOURCE)
    cmd = [build_mod.nvcc(), *build_mod.ARCH, *build_mod.FLAGS, "-I" + build_mod.CSRC, "-shared", "-o", str(d / "held.so"),
           str(d / "held.cu")]
    subprocess.run(cmd, check=True)
    lib = ctypes.CDLL(str(d / "held.so"))
    vp, i, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.probs.argtypes = [vp, vp, i, i, f, i, f, vp, vp]
    return lib


def run(L, x, hold, temperature, top_k, top_p):
    """(probabilities over what was there before, status)"""
    assert L.hold(ctypes.byref(Hold(*hold))) == 0
    out, status = torch.full_like(x, 7.0), torch.zeros(1, dtype=torch.int32, device="cuda")
    assert L.probs(x.data_ptr(), out.data_ptr(), *x.shape, temperature, top_k, top_p, status.data_ptr(),
                   torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    return out, int(status)


def logits(kind, vocab):
    g = torch.Generator().manual_seed(vocab)
    x = torch.randn(2, vocab, generator=g) * 2
    if kind == "flat":       # (more tokens in a bin than are listed: parts of it are tried, then 10 bits at a time)
        x = 5 + x * 1e-4
    return x.cuda()


NUCLEUS, LIKELIEST, GREEDY, ALL, BOTH = (0.8, 0, 0.9), (0.8, 50, 1.0), (0.0, 0, 0.9), (0.8, 0, 1.0), (0.8, 5000, 0.9)


@pytest.mark.parametrize("kind,vocab,hold,settings", [
    ("normal", 32000, (0, 1, -1, 0, 0), NUCLEUS), ("normal", 32000, (0, 3, 0, 0, 0), GREEDY),
    ("normal", 8000, (0, 0, 1, 0, 1300), NUCLEUS), ("normal", 32000, (1, 2, -1, 0, 0), NUCLEUS),
    ("normal", 16000, (1, 0, 3, 0, 1300), LIKELIEST), ("normal", 32000, (2, 7, 0, 0, 0), NUCLEUS),
    ("normal", 32000, (3, 1, 1, 0, 0), NUCLEUS), ("normal", 32000, (3, 5, -1, 0, 1300), LIKELIEST),
    ("normal", 32000, (4, 1, 2, 0, 0), LIKELIEST), ("normal", 32000, (5, 1, 0, 0, 0), ALL),
    ("normal", 32000, (5, 4, -1, 0, 1300), ALL), ("normal", 32000, (1, 2, 1, 1, 0), BOTH),
    ("flat", 32000, (3, 1, 6, 1, 0), NUCLEUS), ("flat", 32000, (1, 3, -1, 1, 0), BOTH)])
def test_a_message_that_does_not_come(L, kind, vocab, hold, settings):
    x = logits(kind, vocab)
    want, flags = run(L, x, (-1, 0, 0, 0, 0), *settings)
    # (without cuts token_probs has a kernel of its own; |x - max| / T is below 30 here, and each side is off by
    # 2 units of 2^-24 for each unit of it and a few: 140 2^-24 < 1e-5)
    assert flags == 0 and torch.allclose(want, token_probs(x, *settings), rtol=1e-5, atol=0)
    got, flags = run(L, x, hold, *settings)
    assert flags == 2 and bool((got[0] == 0).all())
    assert torch.equal(got[1], want[1])
    got, flags = run(L, x, (-1, 0, 0, 0, 0), *settings)
    assert flags == 0 and torch.equal(got, want)
