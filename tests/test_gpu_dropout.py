"""Counter-based dropout on the GPU: the mask bit for bit, values to one rounding."""
import numpy as np
import pytest

from helpers import to_dev
from oracle import decay
from workloads import bf16_round

pytestmark = pytest.mark.gpu


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def _x(n, dtype, seed=0):
    x = np.random.default_rng(seed).standard_normal(n).astype(np.float32)
    return bf16_round(x) if dtype == "bf16" else x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2049, 100003])
@pytest.mark.parametrize("p,residual", [(0.1, False), (0.5, True), (0.9999, False)])
def test_values(n, dtype, p, residual):
    fv = _fv()
    seed, offset = (1 << 63) + 12345, (1 << 40) + 7
    x, r = _x(n, dtype), _x(n, dtype, 1) if residual else None
    ref = decay.dropout(x, p, seed, offset, r)
    y = fv.dropout(to_dev(x, dtype), p, seed, offset,
                   residual=to_dev(r, dtype) if residual else None)
    got = y.double().cpu().numpy()
    if not residual:
        assert np.array_equal(got == 0, ref == 0)
    # fp32: the scale's, the product's and the sum's rounding; then the output's
    scaled = np.abs(ref - r) if residual else np.abs(ref)
    tol = 2 * 2.0 ** -24 * scaled * 1.01 + 2.0 ** -24 * np.abs(ref) * 1.01
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(ref) * 1.01
    assert (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_borders_of_p(dtype):
    import torch
    fv = _fv()
    x = to_dev(_x(1003, dtype), dtype)
    x[3], x[4] = float("nan"), float("inf")
    r = to_dev(_x(1003, dtype, 1), dtype)
    assert torch.equal(fv.dropout(x, 0.0, 1).nan_to_num(), x.nan_to_num())
    assert not fv.dropout(x, 1.0, 1).any()
    assert torch.equal(fv.dropout(x, 1.0, 1, residual=r), r)
    assert torch.equal(fv.dropout(x, 2.0 ** -18, 1).nan_to_num(), x.nan_to_num())
    assert torch.equal(fv.dropout(x[:0], 0.5, 1), x[:0])


def test_gradient_has_the_same_mask_and_other_counters_another():
    import torch
    fv = _fv()
    x = torch.ones(50000, device="cuda")
    y = fv.dropout(x, 0.3, 5, 6, residual=x) - 1
    assert torch.equal((y != 0).float() / (1 - decay.threshold(0.3) / 65536.0),
                       fv.dropout_backward(x, 0.3, 5, 6))
    for seed, offset in ((5, 7), (6, 6), (5 + (1 << 32), 6), (5, 6 + (1 << 32))):
        z = fv.dropout(x, 0.3, seed, offset)
        # two masks of share 0.3 agree on 0.58 of 50000 elements: six standard deviations
        same = ((z != 0) == (y != 0)).float().mean().item()
        assert abs(same - 0.58) < 6 * (0.58 * 0.42 / 50000) ** 0.5


def test_in_place_and_shapes():
    import torch
    fv = _fv()
    x = to_dev(_x(3 * 5 * 7, "f32").reshape(3, 5, 7))
    r = to_dev(_x(3 * 5 * 7, "f32", 1).reshape(3, 5, 7))
    want = fv.dropout(x, 0.4, 8, residual=r)
    assert want.shape == x.shape
    a = x.clone()
    assert fv.dropout(a, 0.4, 8, residual=r, out=a) is a and torch.equal(a, want)
    b = r.clone()
    fv.dropout(x, 0.4, 8, residual=b, out=b)
    assert torch.equal(b, want)


def test_elements_past_32_bits():
    """The counter of an element behind 2^32, and of the last odd ones."""
    import torch
    fv = _fv()
    n = (1 << 32) + 13
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    fv.dropout(x, 0.5, 3, 4, out=x)
    for first, m in ((0, 64), ((1 << 32) - 32, 45), (1 << 31, 64)):
        want = decay.dropout_bits(3, 4, first, m) >= decay.threshold(0.5)
        assert np.array_equal(x[first:first + m].float().cpu().numpy() != 0, want)


def test_nothing_behind_the_elements_is_written():
    import torch
    fv = _fv()
    for n in (1, 5, 8, 1003):
        y = torch.full((n + 16,), 7.0, device="cuda")
        fv.dropout(torch.ones(n, device="cuda"), 0.5, 1, out=y[:n])
        assert (y[n:] == 7).all()


def test_words_in_device_memory():
    """rng replaces seed and offset, and a captured call reads it at each replay."""
    import torch
    fv = _fv()
    x = to_dev(_x(5000, "bf16"), "bf16")
    rng = torch.tensor([11, 22], dtype=torch.int64, device="cuda")
    y = torch.empty_like(x)
    fv.dropout(x, 0.25, rng=rng, out=y)
    assert torch.equal(y, fv.dropout(x, 0.25, 11, 22))
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fv.dropout(x, 0.25, rng=rng, out=y)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        fv.dropout(x, 0.25, rng=rng, out=y)
    for i in range(3):
        rng[1] = 100 + i
        y.zero_()
        want = fv.dropout(x, 0.25, 11, 100 + i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
