"""Single tokens on the GPU: broadcast rows at the C ABI and in the binding; long runs."""
import ctypes

import numpy as np
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


@pytest.mark.parametrize("heads", [1, 32])
def test_many_tokens_do_not_drift(heads):
    """8192 tokens one by one, with decays so close to 1 that a rounded factor's error (up to
    2^-24 of the state per token, always the same) would add up to 8192 of them. What may
    remain are the roundings of single tokens, of either sign: two of at most 2^-24 each, whose
    sum over n tokens stays below 4 sqrt(n) 2^-24 (six standard deviations of uniform ones are
    6 sqrt(2 n / 3) / 2 = 2.4 sqrt(n))."""
    import torch
    fv = _fv()
    n, d = 8192, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.rand((n, 1, 1, d), generator=gen, device="cuda") for _ in range(2))
    e = np.linspace(2e-6, 2e-4, heads).astype(np.float32) if heads > 1 else np.float32([3.3e-5])
    g = to_dev(-e)
    s = torch.zeros((1, heads, d, d), device="cuda")
    out = torch.empty((1, heads, d), device="cuda")
    for t in range(n):
        kt, vt = k[t].expand(1, heads, d), v[t].expand(1, heads, d)
        fv.attn_decay_step(kt, kt, vt, g, s, out=out)
    w = torch.exp(g.double()[:, None] * torch.arange(n - 1, -1, -1, device="cuda"))
    ref = (k[:, 0, 0].double()[None] * w[:, :, None]).transpose(-1, -2).contiguous() \
        @ v[:, 0, 0].double()
    rel = ((s[0].double() - ref).norm(dim=(-1, -2)) / ref.norm(dim=(-1, -2))).cpu().numpy()
    assert (rel < 4 * n ** 0.5 * 2.0 ** -24).all(), rel * 2.0 ** 24
    _, whole = fv.attn_decay(*(x.permute(1, 2, 0, 3).expand(1, heads, n, d) for x in (k, k, v)), g,
                             return_state=True)
    assert ((s - whole).norm() / whole.norm()).item() < 5 * n ** 0.5 * 2.0 ** -24
