"""Which kernels of the operators around the melded layer spill registers: those that the norms' source names, and no others."""
import os
import re

import pytest

import paper_2510_24061_amd as fq
from test_register_spills import _kernels

# norm_bwd_kernel<type, pieces, codes, mode>: two pieces of bf16 from checkpoints with a plain branch; four pieces of fp32 with a branch
NAMED = (r"norm_bwd_kernelItLi2ELb1ELi1E", r"norm_bwd_kernelIfLi4ELb[01]ELi[123]E")
OPERATORS = (r"norm_fwd_kernel", r"norm_bwd_kernel", r"norm_sum_kernel", r"swiglu_(fwd|bwd)_kernel", r"mx_(quantize|values)_kernel", r"mx4_(gemm|thin)_kernel",
             r"token_(logprob|join|logprob_bwd)_kernel", r"preference_(one|pair|mean)_kernel")


def test_only_the_named_ones(tmp_path):
    if not os.path.exists(fq.lib_path()):
        pytest.skip("library not built")
    kernels = _kernels(fq.lib_path(), tmp_path)
    for pattern in OPERATORS:
        assert any(re.search(r"\d" + pattern, n) for n in kernels), pattern
    spill = [n for n, k in kernels.items() if k != (0, 0) and any(re.search(r"\d" + p, n) for p in OPERATORS)]
    assert not [n for n in spill if not any(re.search(p, n) for p in NAMED)], spill
    assert all(kernels[n][0] <= 5 for n in spill if "kernelIt" in n)
