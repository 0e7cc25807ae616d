"""A scale that is finite, but not in the log2 units the kernels work in, is
refused (no GPU: a call that passes its checks fails at its launch)."""
import ctypes

import pytest
import torch

INVALID, HIP = 1, 4


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would be launched")
@pytest.mark.parametrize("scale,code", [(3e38, INVALID), (-3e38, INVALID), (2.3e38, HIP),
                                        (-2.3e38, HIP), (1e-40, HIP)])
def test_scale(scale, code):
    import paper_2606_00724_amd as wf
    p = wf.make_prefix_params(share=2, heads=2, q_len=4, head_dim=64, prefix_cap=16, scale=scale)
    f = ctypes.c_void_p(1 << 20)  # aligned, never read
    assert wf.library().wf_prefix_attn(ctypes.byref(p), f, f, None, f, None, None, None, None,
                                       None, None, f, None, None, 0, None) == code
