"""The short causal convolution on the GPU against the fp64 oracle, element by element."""
import numpy as np
import pytest

from helpers import to_dev, to_host, torch_dtype
from oracle import recurrent as rec
from workloads import bf16_round

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def _round(x, dtype):
    return bf16_round(x.astype(np.float32)) if dtype == "bf16" else x.astype(np.float32)


def inputs(B, L, D, W, dtype, seed, bias=True, state=True):
    r = np.random.default_rng(seed)
    draw = lambda *s: _round(r.standard_normal(s), dtype)
    return dict(x=draw(B, L, D), w=r.uniform(-1, 1, (D, W)).astype(np.float32),
                bias=r.standard_normal(D).astype(np.float32) if bias else None,
                state=draw(B, W - 1, D) if state else None, dy=draw(B, L, D),
                dstate=draw(B, W - 1, D) if state else None)


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def near(got, ref, units, dtype, name):
    """units: the bound in 2^-24 before the output's rounding; 1.05 for higher orders."""
    got, ref = to_host(got), np.asarray(ref)
    tol = 1.05 * U * np.asarray(units) + half_step(dtype) * np.abs(ref) * 1.01 + 1e-37
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.abs(got - ref)[bad].max(), tol[bad].max(),
                           np.argwhere(bad)[:4].tolist())


def conv_units(i, silu, lengths=None):
    """Of y: W + 1 roundings of the sum's magnitude through the slope (at most 1.1), then
    sigmoid (the exponential's argument and value, the sum, the reciprocal) and the product."""
    W = i["w"].shape[1]
    m, _ = rec.conv(np.abs(i["x"]), np.abs(i["w"]), None if i["bias"] is None else np.abs(i["bias"]),
                    False, lengths, None if i["state"] is None else np.abs(i["state"]))
    u, _ = rec.conv(i["x"], i["w"], i["bias"], False, lengths, i["state"])
    if not silu:
        return (W + 1) * m
    return 1.1 * (W + 1) * m + np.abs(u) * rec.sigmoid(u) * (2 * np.abs(u) + 6)


def grad_units(i, silu, lengths=None):
    """Of (dx, dw, dbias, dstate)."""
    W, (B, L, D) = i["w"].shape[1], i["x"].shape
    absol = {k: None if v is None else np.abs(v) for k, v in i.items()}
    eg = np.zeros((B, L, D))   # error of g = dy silu'(u), in units
    g = absol["dy"] * (1.1 if silu else 1.0)
    if silu:
        m, _ = rec.conv(absol["x"], absol["w"], absol["bias"], False, lengths, absol["state"])
        u, _ = rec.conv(i["x"], i["w"], i["bias"], False, lengths, i["state"])
        # |silu''| <= 0.5; s (1 + u (1 - s)): its factors' errors and three products
        s = rec.sigmoid(u)
        slope = s * (1 + np.abs(u) * (1 - s))
        eg = absol["dy"] * (0.5 * (W + 1) * m + slope * (4 * np.abs(u) + 16))
    zero = lambda v: None if v is None else np.zeros_like(v)
    first = rec.conv_backward(absol["x"], absol["w"], eg, absol["bias"], False, lengths,
                              absol["state"], zero(absol["dstate"]))
    mag = rec.conv_backward(absol["x"], absol["w"], g, absol["bias"], False, lengths,
                            absol["state"], absol["dstate"])
    adds = (W + 2, 48 + L // 32, 48 + L // 32, W + 2)   # a run, its workgroup, the workgroups
    return [e + k * m for e, k, m in zip(first, adds, mag)]


def _dev(i, dtype):
    p = lambda v: None if v is None else to_dev(v)
    d = lambda v: None if v is None else to_dev(v, dtype)
    return dict(x=d(i["x"]), w=p(i["w"]), bias=p(i["bias"]), state=d(i["state"]), dy=d(i["dy"]),
                dstate=d(i["dstate"]))


SHAPES = [  # B, L, D, W
    (1, 1, 8, 2), (2, 3, 16, 8), (1, 7, 24, 5), (3, 33, 40, 3), (2, 129, 72, 4), (1, 300, 8, 6),
    (1, 65, 264, 7), (2, 1030, 136, 4),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,L,D,W", SHAPES)
@pytest.mark.parametrize("silu,bias,state", [(1, 1, 1), (0, 0, 0)])
def test_forward_and_backward(B, L, D, W, dtype, silu, bias, state):
    fv = _fv()
    i = inputs(B, L, D, W, dtype, 7 * L + W, bias, state)
    t = _dev(i, dtype)
    y, s = fv.causal_conv(t["x"], t["w"], t["bias"], silu, state_in=t["state"], return_state=True)
    ref, sref = rec.conv(i["x"], i["w"], i["bias"], silu, None, i["state"])
    near(y, ref, conv_units(i, silu), dtype, "y")
    assert np.array_equal(to_host(s), sref)
    g = fv.causal_conv_backward(t["x"], t["w"], t["dy"], t["bias"], silu, state_in=t["state"],
                                dstate_out=t["dstate"], return_state_grad=True)
    refs = rec.conv_backward(i["x"], i["w"], i["dy"], i["bias"], silu, None, i["state"], i["dstate"])
    units = grad_units(i, silu)
    assert (g[2] is None) == (not bias)
    for got, r, u, name in zip(g, refs, units, ("dx", "dw", "dbias", "dstate")):
        if got is not None:
            near(got, r, u, "f32" if name in ("dw", "dbias") else dtype, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch(dtype):
    """Lengths of 0, of less than the taps and out of range; padding that is NaN."""
    import torch
    fv = _fv()
    B, L, D, W = 6, 70, 24, 4
    lengths = [70, 0, 2, 41, -3, 99]
    i = inputs(B, L, D, W, dtype, 5)
    t = _dev(i, dtype)
    n = np.clip(lengths, 0, L)
    for b in range(B):
        t["x"][b, n[b]:] = float("nan")
        t["dy"][b, n[b]:] = float("inf")
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, s = fv.causal_conv(t["x"], t["w"], t["bias"], True, lens, t["state"], True)
    ref, sref = rec.conv(i["x"], i["w"], i["bias"], True, lengths, i["state"])
    near(y, ref, conv_units(i, True, lengths), dtype, "y")
    assert np.array_equal(to_host(s), sref)
    assert all(not y[b, n[b]:].any() for b in range(B))
    g = fv.causal_conv_backward(t["x"], t["w"], t["dy"], t["bias"], True, lens, t["state"],
                                t["dstate"], True)
    refs = rec.conv_backward(i["x"], i["w"], i["dy"], i["bias"], True, lengths, i["state"], i["dstate"])
    for got, r, u, name in zip(g, refs, grad_units(i, True, lengths), ("dx", "dw", "dbias", "dstate")):
        near(got, r, u, "f32" if name in ("dw", "dbias") else dtype, name)
    assert all(not g[0][b, n[b]:].any() for b in range(B))


def test_strides_and_untouched_neighbours():
    """Halves of a projection in and out, a transposed batch, a broadcast sequence."""
    import torch
    fv = _fv()
    B, L, D = 2, 50, 16
    i = inputs(B, L, D, 3, "f32", 9, state=False)
    t = _dev(i, "f32")
    want = fv.causal_conv(t["x"], t["w"], t["bias"], True)
    dwant = fv.causal_conv_backward(t["x"], t["w"], t["dy"], t["bias"], True)
    wide = torch.full((B, L, 3 * D), 5.0, device="cuda")
    wide[..., D:2 * D] = t["x"]
    out = torch.full((B, L, 3 * D), 7.0, device="cuda")
    fv.causal_conv(wide[..., D:2 * D], t["w"], t["bias"], True, out=out[..., D:2 * D])
    assert torch.equal(out[..., D:2 * D], want)
    assert (out[..., :D] == 7).all() and (out[..., 2 * D:] == 7).all()
    fv.causal_conv_backward(wide[..., D:2 * D], t["w"], t["dy"], t["bias"], True,
                            dx=out[..., :D])
    assert torch.equal(out[..., :D], dwant[0]) and (out[..., 2 * D:] == 7).all()
    swapped = t["x"].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(fv.causal_conv(swapped, t["w"], t["bias"], True), want)
    one = t["x"][:1].expand(3, L, D)
    assert torch.equal(fv.causal_conv(one, t["w"], t["bias"], True), want[:1].expand(3, L, D))
    still = t["x"][:, :1].expand(B, L, D)
    assert torch.equal(fv.causal_conv(still, t["w"], t["bias"], True),
                       fv.causal_conv(still.contiguous(), t["w"], t["bias"], True))


@pytest.mark.parametrize("L1", [1, 2, 37])
def test_pieces_and_state_in_place(L1):
    """Two pieces that hand the state on in place are the whole."""
    import torch
    fv = _fv()
    i = inputs(2, 60, 32, 4, "bf16", 3)
    t = _dev(i, "bf16")
    want, end = fv.causal_conv(t["x"], t["w"], t["bias"], True, state_in=t["state"], return_state=True)
    s = t["state"].clone()
    a = fv.causal_conv(t["x"][:, :L1], t["w"], t["bias"], True, state_in=s, state_out=s)
    b = fv.causal_conv(t["x"][:, L1:], t["w"], t["bias"], True, state_in=s, state_out=s)
    assert torch.equal(torch.cat((a, b), 1), want) and torch.equal(s, end)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,W", [(8, 2), (40, 4), (1032, 8)])
def test_single_tokens(D, W, dtype):
    """Tokens one by one on a pool: the same as the stretch; a place of its own for each, two
    absent sequences, two that share a place."""
    import torch
    fv = _fv()
    i = inputs(4, 12, D, W, dtype, 11)
    t = _dev(i, dtype)
    ref, end = rec.conv(i["x"], i["w"], i["bias"], True, None, i["state"])
    pool = torch.full((6, W - 1, D), 9.0, device="cuda", dtype=torch_dtype(dtype))
    places = [4, 0, 5, 2]
    pool[places] = t["state"]
    slots = torch.tensor(places[:1] + [-1] + places[1:] + [6], dtype=torch.int32, device="cuda")
    live = [0, 2, 3, 4]
    units = conv_units(i, True)
    for k in range(12):
        x = torch.zeros((6, D), device="cuda", dtype=torch_dtype(dtype))
        x[live] = t["x"][:, k]
        y = fv.causal_conv_step(x, t["w"], pool, t["bias"], True, slots)
        near(y[live], ref[:, k], units[:, k], dtype, f"token {k}")
        assert not y[1].any() and not y[5].any()
    assert np.array_equal(to_host(pool[places]), end)
    assert (pool[[1, 3]] == 9).all()
    # the same place three times: three tokens of one sequence
    pool[3] = t["state"][0]
    slots = torch.tensor([3, 1, 3, 3], dtype=torch.int32, device="cuda")
    x = torch.stack((t["x"][0, 0], t["x"][1, 0], t["x"][0, 1], t["x"][0, 2]))
    y = fv.causal_conv_step(x, t["w"], pool, t["bias"], True, slots)
    near(y[[0, 2, 3]], ref[0, :3], units[0, :3], dtype, "turns")


def test_empty_calls():
    import torch
    fv = _fv()
    w = torch.ones((8, 4), device="cuda")
    x = torch.zeros((2, 0, 8), device="cuda")
    s = torch.arange(48, dtype=torch.float32, device="cuda").reshape(2, 3, 8)
    y, out = fv.causal_conv(x, w, state_in=s, return_state=True)
    assert y.shape == x.shape and torch.equal(out, s)
    dx, dw, _, ds = fv.causal_conv_backward(x, w, x, state_in=s, dstate_out=s, return_state_grad=True)
    assert not dw.any() and torch.equal(ds, s)
    assert fv.causal_conv(torch.zeros((0, 5, 8), device="cuda"), w).shape == (0, 5, 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_no_sequence(dtype):
    """The filters' gradients of an empty batch are sums of nothing, whatever their memory held."""
    import torch
    fv = _fv()
    x = torch.zeros((0, 5, 72), device="cuda", dtype=torch_dtype(dtype))
    w, b = torch.ones((72, 4), device="cuda"), torch.ones(72, device="cuda")
    dw, db = torch.full_like(w, 7.0), torch.full_like(b, 7.0)
    dx, *got, ds = fv.causal_conv_backward(x, w, x, b, True, return_state_grad=True, dweight=dw, dbias=db)
    assert got[0] is dw and got[1] is db and not dw.any() and not db.any()
    assert dx.shape == x.shape and ds.shape == (0, 3, 72)
    fv.causal_conv_backward(x, w, x, dweight=dw.fill_(7))
    assert not dw.any()


def test_gradients_against_differences():
    """The kernels' own loss moves as their gradients say (fp32; central differences)."""
    import torch
    fv = _fv()
    i = inputs(2, 40, 16, 4, "f32", 13)
    t = _dev(i, "f32")
    dx, dw, db, ds = fv.causal_conv_backward(t["x"], t["w"], t["dy"], t["bias"], True,
                                             state_in=t["state"], dstate_out=t["dstate"],
                                             return_state_grad=True)
    r = np.random.default_rng(1)
    args = [i["x"], i["w"], i["bias"], i["state"]]
    for k, d in enumerate((dx, dw, db, ds)):
        step = r.standard_normal(d.shape)
        h = 1e-5

        def loss(s):
            a = [v + s * step if j == k else v.astype(np.float64) for j, v in enumerate(args)]
            y, end = rec.conv(a[0], a[1], a[2], True, None, a[3])
            return (y * i["dy"]).sum() + (end * i["dstate"]).sum()

        want = (loss(h) - loss(-h)) / (2 * h)
        # the gradients' own roundings, and the differences' curvature (h^2) and rounding
        assert abs((to_host(d) * step).sum() - want) < 1e-5 * np.abs(to_host(d) * step).sum()
