"""Beam search's selection and the reordering of pooled states on the GPU against the oracle."""
import numpy as np
import pytest

from helpers import to_dev, to_host, torch_dtype
from oracle import recurrent as rec
from test_gpu_conv import _round

pytestmark = pytest.mark.gpu


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def select(x, scores, n, dtype="f32", ended=None, end_token=-1, **kw):
    import torch
    e = None if ended is None else torch.tensor(ended, dtype=torch.bool, device="cuda")
    return _fv().beam_select(to_dev(x, dtype) if isinstance(x, np.ndarray) else x, to_dev(scores), n,
                             e, end_token, **kw)


def same(got, ref, V, scale=0.0):
    s, parent, token = got
    assert np.array_equal(parent.cpu().numpy(), ref[1])
    assert np.array_equal(token.cpu().numpy(), ref[2])
    s, r = s.double().cpu().numpy(), ref[0]
    assert np.array_equal(np.isinf(s), np.isinf(r))
    f = np.isfinite(r)
    # the score's rounding; the sum's: an exponential 8 + |x| and as many additions as a lane
    # makes, relative to itself, so absolute in its logarithm
    tol = 2.0 ** -24 * (np.abs(r[f]) + 16 + scale + V / 64)
    assert (np.abs(s[f] - r[f]) <= tol).all()


def data(B, K, V, dtype, seed, scale=3.0):
    r = np.random.default_rng(seed)
    return (_round(scale * r.standard_normal((B, K, V)), dtype),
            (-4 * r.random((B, K))).astype(np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,K,V,n", [
    (1, 1, 1, 1), (2, 3, 2, 5), (1, 4, 7, 4), (3, 5, 511, 8), (2, 2, 512, 64), (1, 3, 513, 3),
    (2, 8, 2049, 8), (1, 64, 300, 64), (1, 4, 50001, 4), (5, 1, 4100, 17), (64, 8, 9001, 6),
    (300, 16, 2100, 3)])
def test_selection(B, K, V, n, dtype):
    x, s = data(B, K, V, dtype, V + n)
    same(select(x, s, n, dtype), rec.beam_select(x, s, n), V, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 33, 64])
def test_rows_that_order_badly(n, dtype):
    """Equal logits, rising and falling ones, few values, the best at the row's ends."""
    V = 5000
    r = np.random.default_rng(3)
    x = np.zeros((1, 7, V), np.float32)
    x[0, 1] = np.arange(V) / 512.0
    x[0, 2] = -np.arange(V) / 512.0
    x[0, 3] = r.integers(0, 3, V)
    x[0, 4, [0, V - 1]] = 5
    x[0, 5] = -np.arange(V)[::-1] // 100
    x[0, 6, ::8] = 1
    x = _round(x, dtype)
    s = np.arange(7, dtype=np.float32)[None] * 0.37
    same(select(x, s, n, dtype), rec.beam_select(x, s, n), V, 20)
    for k in range(7):
        same(select(x[:, k:k + 1], s[:, k:k + 1], n, dtype),
             rec.beam_select(x[:, k:k + 1], s[:, k:k + 1], n), V, 20)


def test_equal_beams_and_alignment():
    """Equal rows have equal scores wherever they lie: the lower beam goes first."""
    import torch
    for dtype in ("bf16", "f32"):
        x, _ = data(1, 1, 3001, dtype, 4)
        rows = to_dev(np.repeat(x, 6, 1), dtype)   # rows of 3001: each at another alignment
        s, parent, token = select(rows, np.full((1, 6), -1.0, np.float32), 12, dtype)
        assert parent.tolist() == [[0, 1, 2, 3, 4, 5] * 2]
        assert (s[0, :6] == s[0, 0]).all() and (s[0, 6:] == s[0, 6]).all()
        assert token[0, :6].unique().numel() == 1
        wide = torch.full((1, 6, 3100), 50.0, device="cuda", dtype=torch_dtype(dtype))
        wide[:, :, 13:3014] = rows
        got = select(wide[:, :, 13:3014], np.full((1, 6), -1.0, np.float32), 12, dtype)
        for a, b in zip(got, (s, parent, token)):
            assert torch.equal(a, b)
        turned = rows.expand(3, 6, 3001).transpose(0, 1).contiguous().transpose(0, 1)
        got = select(turned, np.full((3, 6), -1.0, np.float32), 12, dtype)
        for a, b in zip(got, (s, parent, token)):
            assert torch.equal(a, b.expand(3, 12))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_and_what_is_no_number(dtype):
    V, inf = 1500, np.inf
    x, s = data(9, 3, V, dtype, 6)
    x[0, 1] = -inf                       # a beam with nothing left
    x[1, :, 2:] = -inf                   # two tokens each
    x[2, 0, 700] = np.nan                # a beam without a sum
    x[3, 2, 3] = inf
    s[4, 1] = -inf                       # a dead beam
    s[5, 1] = np.nan
    x[6] = -inf                          # nothing at all
    x[7, :, :] = -3.0e38                 # the type's lowest values
    x[7, 0, 9] = -1.0
    s[8] = [-inf, -inf, 0.5]             # a first step: one beam alive
    x[7] = _round(x[7], dtype)
    same(select(x, s, 10, dtype), rec.beam_select(x, s, 10), V, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [2.0 ** 24, 1e9, 1.07e9, 1.08e9, 1e10, 1e12, 1e20, 1e30, 9e37, 2e38])
def test_masks_of_any_size(value, dtype):
    """Masks and logits whose product with log2 e has few or no digits left for an exponential:
    they count as nothing beside others, and as they are where there are no others."""
    V = 6000
    x, s = data(6, 2, V, dtype, 9)
    r = np.random.default_rng(10)
    x[0, :, 3:] = -value                       # whole pieces and all lanes but one masked
    x[1, :, 1:V - 1] = -value
    x[2][r.random((2, V)) < 0.9] = -value
    x[3] = -value                              # nothing else
    x[4, 0] += value                           # logits as large themselves
    x[5, 0] = value
    x[5, 0, ::7] = -value
    x = _round(x, dtype)
    for n in (1, 4, 30):
        same(select(x, s, n, dtype), rec.beam_select(x, s, n), V, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [-np.inf, -3.38e38, -1e4, 0.0])
def test_masked_vocabulary(value, dtype):
    """Few tokens of many are left, more and fewer than are chosen; the masked ones are equal."""
    V = 30011
    x, s = data(4, 3, V, dtype, 12)
    r = np.random.default_rng(13)
    for b, few in enumerate((1, 6, 40, 300)):
        for k in range(3):
            keep = r.choice(V, few, replace=False)
            row = np.full(V, value, np.float32)
            row[keep] = x[b, k, keep]
            x[b, k] = row
    x = _round(x, dtype)
    for n in (1, 8, 64):
        same(select(x, s, n, dtype), rec.beam_select(x, s, n), V, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_past_fp32(dtype):
    """A second masked token in a row leaves fp32's range: its score would be -Inf, so it is not
    offered, and what is left over has parent 0 and the end's token."""
    low = -3.3e38
    x = _round(np.array([[[1, low, low], [low, 2, low]]], np.float32), dtype)
    s = np.array([[-3.2e38, -1]], np.float32)
    got = select(x, s, 6, dtype, end_token=2)
    same(got, rec.beam_select(x, s, 6, None, 2), 3, 20)
    assert got[1].tolist() == [[1, 0, 1, 1, 0, 0]] and got[2].tolist() == [[1, 0, 0, 2, 2, 2]]
    assert got[0].isinf().tolist() == [[False] * 4 + [True] * 2]


def test_ended_beams():
    x, s = data(4, 5, 900, "f32", 8)
    ended = np.zeros((4, 5), bool)
    ended[0, 2] = ended[1] = ended[2, [0, 4]] = True
    x[ended] = np.nan                    # not read
    s[0, 2] = 50.0
    s[2, 0] = -np.inf
    for n in (1, 5, 12):
        same(select(x, s, n, ended=ended, end_token=17), rec.beam_select(x, s, n, ended, 17), 900, 20)


def test_offsets_past_32_bits():
    """A row that starts behind 2^32 elements."""
    import torch
    big = torch.zeros(((1 << 32) + 4096,), dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((2, 1, 1000), (1 << 32, 1, 1))
    x[0, 0, 7] = 3
    x[1, 0, 999] = 2
    s, parent, token = select(x, np.zeros((2, 1), np.float32), 1, "bf16")
    assert token.tolist() == [[7], [999]] and parent.tolist() == [[0], [0]]


# ------------------------------------------------------------------ reordering
def _pools(n, seed, shapes):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((n,) + s, generator=g, device="cuda").to(t) for s, t in shapes]


def _reordered(parent, slots, pools):
    import torch
    fv = _fv()
    ref, want = rec.beam_reorder(parent, slots, [p.float().cpu().numpy() for p in pools])
    new = fv.beam_reorder(torch.tensor(parent, dtype=torch.int32, device="cuda"),
                          torch.tensor(slots, dtype=torch.int32, device="cuda"), pools)
    assert np.array_equal(new.cpu().numpy(), ref)
    for p, w in zip(pools, want):
        assert np.array_equal(p.float().cpu().numpy(), w)


@pytest.mark.parametrize("B,K", [(1, 1), (1, 2), (3, 5), (2, 64), (40, 8)])
def test_reorder(B, K):
    import torch
    r = np.random.default_rng(K)
    n = B * K + 5
    shapes = [((24, 3), torch.float32), ((3, 8), torch.bfloat16), ((2, 128, 130), torch.float32)]
    pools = _pools(n, 1, shapes if B * K < 200 else shapes[:2])
    for kind in range(3):
        parent = (r.integers(0, K, (B, K)) if kind == 0 else np.zeros((B, K), int) + K - 1
                  if kind == 1 else np.tile(np.arange(K)[::-1], (B, 1)))
        _reordered(parent, r.permutation(n)[:B * K].reshape(B, K), pools)


def test_reorder_absent_places_and_parents():
    """Padding among the places, parents outside the beams, pools of other lengths."""
    import torch
    pools = _pools(7, 2, [((16,), torch.float32)]) + _pools(3, 3, [((2, 4), torch.float32)])
    parent = [[1, 1, 9, 3], [0, -1, 0, 0], [2, 2, 2, 2]]
    slots = [[0, 1, 2, 6], [-1, 5, 4, 3], [-1, 9, -1, -1]]
    _reordered(parent, slots, pools)


def test_reorder_many_pools():
    """More pools than one launch takes, the last of them not of 64."""
    import torch
    pools = _pools(9, 4, [((4 * (i % 5 + 1),), torch.float32) for i in range(131)])
    _reordered([[0, 0, 2], [1, 1, 1]], [[4, 8, 0], [2, 1, 7]], pools)
    fv = _fv()
    none = fv.beam_reorder(torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), None, [])
    assert none.tolist() == [[1, 0]]


def test_reorder_states_past_32_bits():
    import torch
    fv = _fv()
    pool = torch.empty((5, 1 << 28), device="cuda")   # 1 GiB a place
    for k in range(5):
        pool[k] = k
    new = fv.beam_reorder(torch.tensor([[1, 1]], dtype=torch.int32, device="cuda"),
                          torch.tensor([[0, 4]], dtype=torch.int32, device="cuda"), [pool])
    assert new.tolist() == [[4, 0]]
    assert (pool[0] == 4).all() and (pool[1] == 1).all() and (pool[4] == 4).all()
