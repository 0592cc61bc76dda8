"""Single tokens on the GPU: broadcast rows at the C ABI and in the binding."""
import ctypes

import pytest

from helpers import to_dev
from test_gpu_decay import _inputs

pytestmark = pytest.mark.gpu


def _fv():
    import paper_2006_03555_amd as fv
    return fv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_for_every_head(dtype):
    """One query row for all sequences and heads, as a descriptor (batch = head = 0 and a token
    stride) and as an expanded tensor, gives what its copies give."""
    import torch
    fv = _fv()
    B, H, dk, dv = 3, 4, 64, 40
    x = _inputs(B, H, 1, dk, dv, dtype, 2)
    q, k, v = (to_dev(x[n][:, :, 0], dtype) for n in "qkv")
    g, S = to_dev(x["g"]), to_dev(x["S"])
    row = q[:1, :1].clone()
    whole = row.expand(B, H, dk).contiguous()
    want_state = S.clone()
    want = fv.attn_decay_step(whole, k, v, g, want_state)
    s = S.clone()
    assert torch.equal(fv.attn_decay_step(row.expand(B, H, dk), k, v, g, s), want)
    assert torch.equal(s, want_state)
    for token in (1, dk):
        d = fv.make_decay_desc(B, H, 1, dk, dv, fv.BF16 if dtype == "bf16" else fv.F32,
                               q=(0, 0, token))
        s, out = S.clone(), torch.empty_like(v)
        stream = torch.cuda.current_stream().cuda_stream
        assert fv.lib().favor_attn_decay_step(
            ctypes.byref(d), row.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), None, B,
            s.data_ptr(), out.data_ptr(), stream) == 0
        assert torch.equal(out, want) and torch.equal(s, want_state)
