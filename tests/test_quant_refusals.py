"""What the entry points of normalised heads and of the 8-bit cache refuse.  The library looks at its arguments before anything is launched, so
no GPU is needed: contexts and tensors are made up of addresses that nothing reads."""
import ctypes as C
import os

import pytest
import torch

from paper_2603_08026_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2603_08026_amd import build
        build.build(verbose=False)
    return B.load_library()


def test_without_a_context(lib):
    z = C.c_void_p(4096)
    assert lib.dyllm_head_norm_rope(None, z, 768, None, None, None, 1, 1, None, z, None) == -1
    assert lib.dyllm_head_norm_rope_quant(None, z, 768, None, None, None, 1, 1, None, z, None) == -1
    assert lib.dyllm_quant_write(None, z, z, None, 1, 1, None, None) == -1
    assert lib.dyllm_quant_read(None, None, None, 1, 1, z, z, None) == -1
    assert lib.dyllm_partial_attention_quant(None, z, None, None, None, 1, 1, z, None) == -1
    assert lib.dyllm_qkv_refresh_normed(None, None, None, None, z, None, 1, 1, None, None, z, None) == -1
    assert lib.dyllm_layer_step_quant(None, None, None, None, None, None, None, z, None, 1, 1, 0.5, None, None, None) == -1


def test_caches_that_are_none():
    k = torch.zeros(2, 5, 1, 64, dtype=torch.int8)
    s = torch.zeros(2, 1, 5)
    B.QuantCache(k, k.clone(), s, s.clone())
    for bad in ((k.float(), k.float(), s, s), (k, k.view(torch.float8_e4m3fn), s, s), (k, k[:1], s, s), (k[0], k[0], s, s),
                (k, k, s.half(), s), (k, k, s, s.transpose(1, 2)), (k.transpose(0, 1), k.transpose(0, 1), s.permute(2, 1, 0), s.permute(2, 1, 0))):
        with pytest.raises(ValueError):
            B.QuantCache(*bad)
