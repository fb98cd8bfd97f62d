"""Every tile of the 4-bit product over many steps of K: which kernel a size launches, how many steps run with fetches beside the instructions, and the result.

A tile of the table below walks K in steps of 256 with a ring of S stages; all but the last S whole steps and a ragged one are of the steady form.  The
cases have odd and even numbers of steps (exponents are fetched for two at a time), whole and ragged ends, and tiles that the rows and columns do not fill."""
import pytest
import torch

import paper_2510_24061_amd as fq
from test_gpu_mx import check_linear, linear

pytestmark = pytest.mark.gpu
# (rows / 64, columns / 64, stages) of the tile, tokens, inputs, outputs, steady steps
CASES = [((1, 1, 4), 100, 4128, 1040, 12), ((1, 1, 4), 100, 2304, 1024, 5), ((1, 1, 4), 253, 5504, 288, 17),
         ((2, 1, 4), 300, 4128, 4112, 12), ((2, 1, 4), 300, 2304, 4096, 5), ((2, 1, 4), 257, 2048, 4112, 4),
         ((2, 2, 4), 777, 4128, 4112, 12), ((2, 2, 4), 777, 2304, 4096, 5),
         ((2, 2, 2), 1500, 2080, 4112, 6), ((2, 2, 2), 1500, 2304, 4112, 7),
         ((4, 4, 2), 2100, 2080, 8208, 6), ((4, 4, 2), 2100, 2304, 4112, 7), ((4, 4, 2), 4100, 1056, 4112, 2), ((4, 4, 2), 2049, 4096, 4112, 14)]


def kernels(f):
    """Names of the kernels that f launches."""
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as p:
        f()
        torch.cuda.synchronize()
    return [e.name for e in p.events()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tile,T,n,m,steady", CASES)
def test_many_steps(tile, T, n, m, steady, dtype):
    assert n // 256 - tile[2] == steady >= 2
    x, w = torch.randn(T, n, device="cuda").bfloat16(), torch.randn(m, n, device="cuda")
    linear(x, w)                                                               # what torch launches once is launched
    names = kernels(lambda: linear(x, w, dtype))
    assert sum("mx4_gemm_kernel<%d, %d, %d>" % tile in k for k in names) == 1 and not any("mx4_thin" in k for k in names), names
    check_linear(T, n, m, dtype)


def test_rings_hold_their_place():
    """Codes of one block of 256 inputs at a time, all others zeros: a step that read another's codes or exponents would show."""
    for tile, T, n, m, _ in (CASES[0], CASES[3], CASES[6], CASES[8], CASES[11]):
        x, w = torch.randn(T, n, device="cuda").bfloat16(), torch.randn(m, n, device="cuda")
        for k in range(0, n, 256):
            part = torch.zeros_like(x)
            part[:, k:k + 256] = x[:, k:k + 256] * 2.0 ** (k // 256 % 5)       # exponents differ from step to step
            y, wq, we, xq, xe = linear(part, w)
            a, b = (torch.empty(r, n, device="cuda") for r in (T, m))
            fq.mx_dequantize(xq, xe, fq.MX_E2M1, a)
            fq.mx_dequantize(wq, we, fq.MX_E2M1, b)
            # at most 256 products of codes, exact; their sum in any order
            terms = a.abs().double()[:, k:k + 256] @ b.abs().double()[:, k:k + 256].t()
            want = a.double()[:, k:k + 256] @ b.double()[:, k:k + 256].t()
            assert bool(((y.double() - want).abs() <= 256 * 2.0 ** -24 * terms).all()), (tile, k)
