"""Head norms and rotation into pages: the axes of the pairs in every form that a caller may have them in."""
import numpy as np
import pytest
import torch

from paper_2603_08026_amd import binding as Bd
from synth import workload as W
from tests.test_gpu_pages import context, dev, ints, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,dh", [("bf16", 128), ("f32", 64)])
def test_axes_in_every_form(t, dh):
    """Bytes, lists, arrays and tensors of whole numbers of any width say the same; what is no axis is refused."""
    say("head_norm_rope_paged, axes", t, dh)
    g, H, Hkv, n = W.philox(71, t), 4, 2, 9
    ctx = context(t, H, Hkv, dh, 16)
    axis = [int(x) for x in g.integers(0, 3, dh // 2)]
    qkv = dev(g.standard_normal((n, (H + 2 * Hkv) * dh)), t)
    rows = Bd.PageRows(ints([0, n]), ints(np.arange(n)), ints(np.arange(n)))
    pos = ints(g.integers(0, 1000, (3, n)))

    def call(form):
        pages = Bd.Pages.empty(2, Hkv, 16, dh, 1, 1, qkv.dtype)
        q = torch.zeros(n, H, dh, dtype=qkv.dtype, device="cuda")
        ctx.head_norm_rope_paged(qkv, None, None, rows, pages, q, pos, form)
        return torch.cat([q.flatten(), pages.k.flatten()])
    want = call(bytes(axis))
    assert not torch.equal(want, call(bytes(dh // 2)))
    forms = [axis, tuple(axis), bytearray(axis), torch.tensor(axis), torch.tensor(axis, dtype=torch.uint8)]
    forms += [np.array(axis, dtype=d) for d in ("uint8", "int8", "int32", "int64")] + [np.array(axis * 2, dtype="int32").reshape(2, -1).T.copy()[:, 0]]
    for form in forms:
        assert torch.equal(call(form), want), type(form)
    for bad in (axis[:-1] + [256], axis[:-1] + [-1], np.array(axis[:-1] + [256]), axis[:-1] + [0.5]):
        with pytest.raises((ValueError, TypeError)):
            call(bad)
    with pytest.raises(Bd.DyllmError):
        call(np.array(axis[:-1] + [3]))
    ctx.close()
