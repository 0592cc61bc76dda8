"""Positive log_decay: states and sums that grow, as the formula says, as long as a^64 and the
results are in fp32's range. Bounds as in test_gpu_decay (they are relative to the same formula
on absolute values, which grows alike)."""
import numpy as np
import pytest

from helpers import to_dev
from oracle import decay
from test_gpu_decay import _abs, _inputs, _near

pytestmark = pytest.mark.gpu


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def _segments(B, H, L, dk, dv, dtype):
    fv = _fv()
    g = fv.make_decay_desc(B, H, L, dk, dv, fv.BF16 if dtype == "bf16" else fv.F32)
    return fv.decay_workspace_size(g) // (4 * B * H * dk * dv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,H,L", [(0.05, 2, 1500), (0.5, 2, 150), (0.5, 300, 150), (1.25, 2, 64),
                                   (1.38, 2, 60), (1e-4, 2, 700)])
def test_growth_over_chunks_and_segments(g, H, L, dtype):
    fv = _fv()
    x = _inputs(1, H, L, 64, 40, dtype, 5)
    x["g"][:] = np.float32(g)
    y = _abs(x)
    q, k, v, do = (to_dev(x[n], dtype) for n in ("q", "k", "v", "do"))
    gd, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"], 0.5, state=x["S"])
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"], 0.5, state=y["S"])
    out, st = fv.attn_decay(q, k, v, gd, 0.5, state_in=S, return_state=True)
    _scaled(out, ref, mag, 64, L, dtype, "out")
    _scaled(st, end, mend, 64, L, "f32", "state")
    ref = decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"], 0.5, None, x["S"], x["G"])
    mag = decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"], 0.5, None, y["S"], y["G"])
    got = fv.attn_decay_backward(q, k, v, gd, do, 0.5, state_in=S, dstate_out=G,
                                 return_state_grad=True)
    for t, r, m, n in zip(got, ref, mag, ("dQ", "dK", "dV")):
        _scaled(t, r, m, 64, L, dtype, n)
    _scaled(got[3], ref[3], mag[3], 64, L, "f32", "dstate_in")


def _scaled(got, ref, mag, *more):
    """_near, whose norms would overflow, on numbers of ordinary size."""
    s = 1.0 / np.abs(mag).max()
    _near(got.double().cpu().numpy() * s, ref * s, mag * s, *more)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_zero_state_stays_zero(dtype):
    """Segments of zero keys in front, over which a^n passes fp32's range: nothing grows."""
    fv = _fv()
    B, H, L, d = 1, 64, 2048, 8
    per = L // _segments(B, H, L, d, d, dtype)
    assert per * 0.5 > 89   # a^per is Inf in fp32
    x = _inputs(B, H, L, d, d, dtype, 1)
    x["g"][:] = np.float32(0.5)
    for n in ("q", "k", "v"):
        x[n][:, :, :L - 100] = 0
    y = _abs(x)
    q, k, v = (to_dev(x[n], dtype) for n in "qkv")
    out, st = fv.attn_decay(q, k, v, to_dev(x["g"]), return_state=True)
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"])
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"])
    _scaled(out, ref, mag, d, L, dtype, "out")
    _scaled(st, end, mend, d, L, "f32", "state")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_small_state_grows_past_one_factors_range(dtype):
    """a^n of a segment is past fp32's range, its product with the state is not."""
    fv = _fv()
    B, H, L, d = 1, 128, 300, 8
    per = -(-L // 64 // _segments(B, H, L, d, d, dtype)) * 64
    assert per * 0.5 > 89
    x = _inputs(B, H, L, d, d, dtype, 2)
    x["g"][:] = np.float32(0.5)
    for n in ("k", "v"):
        x[n][:] = 0
    x["S"] *= np.float32(1e-31)
    y = _abs(x)
    q, k, v = (to_dev(x[n], dtype) for n in "qkv")
    out, st = fv.attn_decay(q, k, v, to_dev(x["g"]), state_in=to_dev(x["S"]), return_state=True)
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"], state=x["S"])
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"], state=y["S"])
    _scaled(out, ref, mag, d, L, dtype, "out")
    _scaled(st, end, mend, d, L, "f32", "state")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g,state", [(1.38, False), (1.38, True), (1.5, True)])
def test_past_the_range_rows_are_infinite_not_nan(g, state, dtype):
    """One chunk of positive terms: the first rows are finite and right, what lies past the
    range is Inf. (At 1.5 the weights themselves pass it, and meet no zeros here.)"""
    fv = _fv()
    L, d = 64, 64
    x = _inputs(1, 1, L, d, d, dtype, 3)
    x["g"][:] = np.float32(g)
    x["v"] *= 64
    x = {n: np.abs(t) if n != "g" else t for n, t in x.items()}
    q, k, v = (to_dev(x[n], dtype) for n in "qkv")
    out = fv.attn_decay(q, k, v, to_dev(x["g"]), state_in=to_dev(x["S"]) if state else None)
    ref, _ = decay.attn(x["q"], x["k"], x["v"], x["g"], state=x["S"] if state else None)
    got = out.double().cpu().numpy()
    assert not np.isnan(got).any()
    top = float(np.finfo(np.float32).max)
    assert (ref < top / 4).any() and (ref > top * 4).any()
    small = ref < top / 4
    assert np.isinf(got[ref > top * 4]).all() and np.isfinite(got[small]).all()
    rel = np.abs(got[small] - ref[small]) / ref[small]   # one rounding, as in test_gpu_decay
    assert rel.max() < (2.0 ** -8 * (1 + 2.0 ** -6) if dtype == "bf16" else 0) + 400 * 2.0 ** -24
