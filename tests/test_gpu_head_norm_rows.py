"""Gradients of the head norms without eps: lanes that have no row add nothing to the weights' gradients."""
import pytest
import torch

from paper_2601_22379_b200 import binding
from tests import paged_reference as ref
from tests.test_gpu_head_norm import DEV, TYPES, backward, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1], ids=["wide", "unaligned"])
@pytest.mark.parametrize("d,rot,tokens,hq,hkv", [(128, 0, 1, 2, 1), (128, 64, 17, 3, 2), (64, 0, 33, 5, 1), (64, 6, 9, 7, 3), (48, 16, 11, 3, 1), (256, 0, 3, 1, 1)])
def test_no_eps(dtype, offset, d, rot, tokens, hq, hkv):
    """eps = 0 and no row of zeros: r is finite everywhere, and so are the gradients, however many rows a block's last round has."""
    t = TYPES[dtype]

    def some(heads, seed, size):
        flat = torch.zeros(tokens * heads * d + 8, dtype=t, device=DEV)
        x = flat[offset:offset + tokens * heads * d].view(tokens, heads, d)
        return x.copy_(rand(tokens, heads, d, dtype=t, seed=seed, size=size))

    q, k, gq, gk = some(hq, 1, 1.7), some(hkv, 2, 0.3), some(hq, 3, 1.0), some(hkv, 4, 1.0)
    wq, wk = 1 + 0.3 * rand(d, seed=5), 1 + 0.3 * rand(d, seed=6)
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV) * 131
    r = binding.Rope(d, rot_dim=rot)
    a = (0.0, pos, rot or d, False, ref.frequencies(rot or d), 1.0)
    dq, dwq, dk, dwk = r.norm_backward(pos, gq, q, wq, gk, k, wk, eps=0.0)
    for dx, dw, x, w, g in ((dq, dwq, q, wq, gq), (dk, dwk, k, wk, gk)):
        want, err, want_w, err_w = backward(g, x, w, *a)
        ref.check(dx, want, err, t, "dx")
        ref.check(dw, want_w, err_w, torch.float32, "dw")
