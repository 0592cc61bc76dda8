"""The short convolution, the selective scan and the beam search's step without a GPU: the
oracle's own pins (library convolution, closed sums, differences, brute force), the C ABI's and
the binding's refusals."""
import ctypes
import itertools
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2006_03555_amd as fv
from oracle import recurrent as rec

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
P = ctypes.c_void_p
A, NUL = P(1 << 20), P(0)   # an aligned address, never dereferenced


def at(n):
    """Distinct aligned addresses, 2^40 apart."""
    return P((n + 1) << 40)


# ------------------------------------------------------------------ oracle
def test_oracle_convolution_is_the_librarys():
    import torch
    r = np.random.default_rng(1)
    x, w, b, s = (r.standard_normal(v) for v in ((2, 9, 5), (5, 4), (5,), (2, 3, 5)))
    y, end = rec.conv(x, w, b, False, None, s)
    xp = torch.from_numpy(np.concatenate([s, x], 1)).transpose(1, 2)
    ref = torch.nn.functional.conv1d(xp, torch.from_numpy(w)[:, None], torch.from_numpy(b), groups=5)
    assert np.allclose(y, ref.transpose(1, 2).numpy(), rtol=1e-13, atol=1e-13)
    assert np.array_equal(end, x[:, -3:])
    z, _ = rec.conv(x, w, b, True, None, s)
    assert np.allclose(z, torch.nn.functional.silu(torch.from_numpy(y)).numpy(), rtol=1e-13, atol=1e-14)


def test_oracle_lengths_cut_sequences():
    r = np.random.default_rng(2)
    n = [4, 0, 1]
    x, w, s, dy, ds = (r.standard_normal(v) for v in ((3, 6, 2), (2, 4), (3, 3, 2), (3, 6, 2), (3, 3, 2)))
    y, end = rec.conv(x, w, None, True, n, s)
    grads = rec.conv_backward(x, w, dy, None, True, n, s, ds)
    for b, m in enumerate(n):
        o, e = rec.conv(x[b:b + 1, :m], w, None, True, None, s[b:b + 1])
        g = rec.conv_backward(x[b:b + 1, :m], w, dy[b:b + 1, :m], None, True, None, s[b:b + 1], ds[b:b + 1])
        assert np.array_equal(y[b, :m], o[0]) and not y[b, m:].any() and np.array_equal(end[b], e[0])
        assert np.allclose(grads[0][b, :m], g[0][0]) and not grads[0][b, m:].any()
        assert np.allclose(grads[3][b], g[3][0])


def _scan_data(seed=3, B=2, L=7, D=4, N=3, G=2):
    r = np.random.default_rng(seed)
    n = r.standard_normal
    return dict(x=n((B, L, D)), dt=n((B, L, D)), A=-np.exp(n((D, N))), Bm=n((B, L, G, N)),
                C=n((B, L, G, N)), skip=n(D), z=n((B, L, D)), bias=n(D), state=n((B, D, N)),
                dy=n((B, L, D)), dstate=n((B, D, N)))


def test_oracle_scan_is_the_closed_sum():
    i = _scan_data()
    y, end = rec.scan(i["x"], i["dt"], i["A"], i["Bm"], i["C"], i["skip"], i["z"], i["bias"],
                      state=i["state"])
    s = np.log1p(np.exp(i["dt"] + i["bias"]))
    total = np.cumsum(s, 1)
    B, L, D = y.shape
    for b, t, d in itertools.product(range(B), range(L), range(D)):
        h = np.exp(i["A"][d] * total[b, t, d]) * i["state"][b, d]
        for j in range(t + 1):
            h = h + (np.exp(i["A"][d] * (total[b, t, d] - total[b, j, d])) * s[b, j, d]
                     * i["x"][b, j, d] * i["Bm"][b, j, d // 2])
        z = i["z"][b, t, d]
        want = (h @ i["C"][b, t, d // 2] + i["skip"][d] * i["x"][b, t, d]) * z / (1 + np.exp(-z))
        assert np.isclose(y[b, t, d], want, rtol=1e-11, atol=1e-12)
        if t == L - 1:
            assert np.allclose(end[b, d], h, rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("lengths", [None, [5, 0]])
def test_oracle_gradients_against_differences(lengths):
    i = _scan_data(4)
    names = ("x", "dt", "A", "Bm", "C", "skip", "z", "bias", "state")

    def loss(j):
        y, end = rec.scan(*[j[k] for k in names[:8]], lengths=lengths, state=j["state"])
        return (y * i["dy"]).sum() + (end * i["dstate"]).sum()

    grads = rec.scan_backward(*[i[k] for k in names[:5]], i["dy"], i["skip"], i["z"], i["bias"], True,
                              lengths, i["state"], i["dstate"])
    r = np.random.default_rng(5)
    for k, g in zip(names, grads):
        step, h = r.standard_normal(g.shape), 1e-5
        up, down = (loss(dict(i, **{k: i[k] + s * h * step})) for s in (1, -1))
        assert np.isclose((up - down) / (2 * h), (g * step).sum(), rtol=1e-7, atol=1e-7), k
    x, w, b, s, dy, ds = (r.standard_normal(v) for v in ((2, 7, 4), (4, 3), (4,), (2, 2, 4), (2, 7, 4), (2, 2, 4)))
    args = [x, w, b, s]
    grads = rec.conv_backward(x, w, dy, b, True, lengths, s, ds)
    for k, g in enumerate(grads):
        step, h = r.standard_normal(g.shape), 1e-5

        def conv_loss(e):
            a = [v + e * step if j == k else v for j, v in enumerate(args)]
            y, end = rec.conv(a[0], a[1], a[2], True, lengths, a[3])
            return (y * dy).sum() + (end * ds).sum()

        assert np.isclose((conv_loss(h) - conv_loss(-h)) / (2 * h), (g * step).sum(), rtol=1e-7, atol=1e-7)


def test_bounds_hold_for_fp32_recurrences():
    """A plain fp32 recurrence stays inside scan_bounds, and a wrong state is outside."""
    i = _scan_data(6, B=1, L=200, D=4, N=3, G=1)
    i = {k: v.astype(np.float32) for k, v in i.items()}
    s = np.log1p(np.exp(i["dt"] + i["bias"]))
    h = i["state"].copy()
    y = np.zeros_like(i["x"])
    for t in range(200):
        h = np.exp(s[:, t, :, None] * i["A"]) * h + (s * i["x"])[:, t, :, None] * i["Bm"][:, t]
        y[:, t] = (h * i["C"][:, t]).sum(-1)
    y = (y + i["skip"] * i["x"]) * i["z"] / (1 + np.exp(-i["z"]))
    names = ("x", "dt", "A", "Bm", "C")
    ref, end = rec.scan(*[i[k] for k in names], i["skip"], i["z"], i["bias"], state=i["state"])
    units = rec.scan_bounds(*[i[k] for k in names], i["dy"], i["skip"], i["z"], i["bias"], True, None,
                            i["state"], i["dstate"])
    assert (np.abs(y - ref) <= 2.0 ** -24 * units[0]).all()
    assert (np.abs(h - end) <= 2.0 ** -24 * units[1]).all()
    wrong, _ = rec.scan(*[i[k] for k in names], i["skip"], i["z"], i["bias"], state=i["state"] * 1.001)
    assert (np.abs(wrong - ref) > 2.0 ** -24 * units[0])[:, :2].any()


def test_oracle_selection_is_brute_force():
    import torch
    r = np.random.default_rng(7)
    x, s = r.standard_normal((3, 4, 50)), r.standard_normal((3, 4))
    x[0] = np.round(x[0])
    x[1, 2] = -np.inf
    got = rec.beam_select(x, s, 9)
    p = (torch.from_numpy(x).log_softmax(-1) + torch.from_numpy(s)[..., None]).nan_to_num(nan=-np.inf)
    v, at_ = p.reshape(3, -1).sort(dim=-1, descending=True, stable=True)
    assert np.allclose(got[0], v[:, :9].numpy(), rtol=1e-12)
    assert np.array_equal(got[1][1:], at_[1:, :9].numpy() // 50)
    assert np.array_equal(got[2][1:], at_[1:, :9].numpy() % 50)


def test_oracle_reordering_continues_each_parent():
    r = np.random.default_rng(8)
    for _ in range(50):
        K = int(r.integers(1, 7))
        parent, slots = r.integers(0, K, (2, K)), r.permutation(2 * K + 2)[:2 * K].reshape(2, K)
        pool = r.standard_normal((2 * K + 2, 3))
        new, (after,) = rec.beam_reorder(parent, slots, [pool])
        for b in range(2):
            assert sorted(new[b]) == sorted(slots[b])
            for j in range(K):
                assert np.array_equal(after[new[b, j]], pool[slots[b, parent[b, j]]])


# ------------------------------------------------------------------ descriptors
def _conv(**kw):
    s = {k: kw.pop(k) for k in list(kw) if isinstance(kw[k], tuple)}
    base = dict(B=2, L=100, D=64, width=4, dtype=fv.BF16, silu=True)
    return fv.make_conv_desc(**{**base, **kw}, **s)


def _scan(**kw):
    s = {k: kw.pop(k) for k in list(kw) if isinstance(kw[k], tuple)}
    base = dict(B=2, L=100, D=64, N=16, dtype=fv.BF16, groups=2)
    return fv.make_scan_desc(**{**base, **kw}, **s)


@pytest.mark.parametrize("kw,status", [
    (dict(), 0), (dict(B=0), 0), (dict(L=0), 0), (dict(D=8), 0), (dict(width=2), 0), (dict(width=8), 0),
    (dict(B=-1), 1), (dict(L=-1), 1), (dict(D=0), 1), (dict(width=0), 1), (dict(dtype=2), 1),
    (dict(dtype=-1), 1), (dict(width=1), 2), (dict(width=9), 2), (dict(D=12), 2), (dict(B=65536), 2),
    (dict(D=65544), 2), (dict(L=(1 << 30) + 1), 2), (dict(L=1 << 30, D=65536), 2),
    (dict(x=(6400, 0, 64)), 0), (dict(x=(0, 0, 64)), 0), (dict(x=(6400, 0, 68)), 1),
    (dict(x=(-8, 0, 64)), 1), (dict(y=(6400, 0, 56)), 1), (dict(y=(0, 0, 64)), 1),
    (dict(y=(64, 0, 128)), 0), (dict(x=(1 << 46, 0, 64)), 2),
])
def test_conv_descriptor(kw, status):
    for op in (0, 2):
        if op == 2 and ("x" in kw or "y" in kw):
            continue
        assert fv.validate_conv_desc(_conv(**kw), op) == status, fv.last_error()
    assert fv.validate_conv_desc(_conv(), 3) == 1 and fv.validate_conv_desc(_conv(), -1) == 1
    if status:
        assert fv.conv_workspace_size(_conv(**kw)) == 0 or "y" in kw


@pytest.mark.parametrize("kw,status", [
    (dict(), 0), (dict(B=0), 0), (dict(L=0), 0), (dict(N=1), 0), (dict(N=256), 0), (dict(groups=8), 0),
    (dict(B=-1), 1), (dict(L=-1), 1), (dict(D=-8), 1), (dict(N=0), 1), (dict(groups=0), 1),
    (dict(groups=3), 1), (dict(dtype=5), 1), (dict(N=257), 2), (dict(groups=16), 2), (dict(D=4, groups=1), 2),
    (dict(B=70000), 2), (dict(D=131072), 2), (dict(L=1 << 30, D=65536), 2),
    (dict(b=(3501, 16, 35)), 0), (dict(b=(0, 0, 35)), 0), (dict(b=(-1, 16, 35)), 1),
    (dict(dt=(6400, 0, 4)), 1), (dict(z=(6400, 0, 0)), 0), (dict(y=(6400, 0, 0)), 1),
])
def test_scan_descriptor(kw, status):
    assert fv.validate_scan_desc(_scan(**kw), 0) == status, fv.last_error()
    assert fv.validate_scan_desc(_scan(), 3) == 1


def test_gradients_strides_are_read_by_the_backward_pass_only():
    bad = (6400, 0, 4)
    assert fv.validate_conv_desc(_conv(grad_x=bad), 0) == 0
    assert fv.validate_conv_desc(_conv(grad_x=bad), 1) == 1
    assert fv.validate_scan_desc(_scan(grad_dt=bad), 0) == 0
    assert fv.validate_scan_desc(_scan(grad_dt=bad), 1) == 1
    assert fv.validate_scan_desc(_scan(grad_b=(1600, 8, 32)), 1) == 1   # groups' rows overlap
    assert fv.validate_scan_desc(_scan(y=bad), 1) == 0


def test_workspaces():
    assert fv.scan_workspace_size(_scan(L=64)) == 0
    assert fv.scan_workspace_size(_scan(L=100000)) > 0
    assert fv.scan_workspace_size(_scan(L=0), True) == 0
    g = _scan(L=300)
    # three chunks' states, their gradients and dA's parts, three sums, dB's and dC's parts
    at_least = 4 * (2 * 3 * 64 * (3 * 16 + 3) + 2 * 2 * 300 * 2 * 16)
    assert at_least <= fv.scan_workspace_size(g, True) <= at_least + 8 * 256
    assert fv.conv_workspace_size(_conv()) == 2 * 5 * 64 * 4
    assert fv.beam_workspace_size(fv.make_beam_desc(2, 3, 100, 4, fv.F32)) == 256 + 256
    assert fv.beam_workspace_size(fv.make_beam_desc(0, 3, 100, 4, fv.F32)) == 0
    assert fv.beam_workspace_size(fv.make_beam_desc(2, 3, 100, 65, fv.F32)) == 0


# ------------------------------------------------------------------ calls
def _call_conv(g, **kw):
    a = dict(x=at(0), weight=A, bias=A, lengths=A, y=at(1), state_in=at(2), state_out=at(3))
    return fv.lib().favor_conv(ctypes.byref(g), *{**a, **kw}.values(), None)


def _call_conv_backward(g, **kw):
    a = dict(x=at(0), weight=at(8), bias=A, lengths=A, state_in=at(1), dy=at(2), dstate_out=at(3),
             dx=at(4), dweight=at(5), dbias=at(6), dstate_in=at(7), ws=A, n=1 << 40)
    return fv.lib().favor_conv_backward(ctypes.byref(g), *{**a, **kw}.values(), None)


def _call_conv_step(g, **kw):
    a = dict(x=at(0), weight=A, bias=A, slots=A, n_slots=4, state=at(1), y=at(2))
    return fv.lib().favor_conv_step(ctypes.byref(g), *{**a, **kw}.values(), None)


def _refused(call, g, name, word, **kw):
    assert call(g, **kw) == 1, (name, kw)
    assert word in fv.last_error(), fv.last_error()


def test_conv_refusals():
    g, odd = _conv(), P((1 << 20) + 2)
    for name in ("x", "weight", "y"):
        _refused(_call_conv, g, name, "NULL", **{name: NUL})
    for name in ("x", "weight", "bias", "lengths", "y", "state_in", "state_out"):
        _refused(_call_conv, g, name, "aligned", **{name: odd})
    _refused(_call_conv, g, "y", "must not be", y=at(0))
    size = 2 * 3 * 64 * 2
    _refused(_call_conv, g, "state", "overlaps", state_out=P((3 << 40) + size - 16))
    for name in ("x", "weight", "dy", "dx", "dweight"):
        _refused(_call_conv_backward, g, name, "NULL", **{name: NUL})
    for name in ("dbias", "dstate_in", "ws"):
        _refused(_call_conv_backward, g, name, "aligned", **{name: odd})
    _refused(_call_conv_backward, g, "ws", "NULL", ws=NUL)
    assert _call_conv_backward(g, n=10) == 3
    _refused(_call_conv_backward, g, "dx", "must not be", dx=at(2))
    _refused(_call_conv_backward, g, "dstate_in", "overlaps", dstate_in=at(3))
    _refused(_call_conv_backward, g, "dweight", "overlaps", dweight=at(8))
    for name in ("x", "weight", "y", "state"):
        _refused(_call_conv_step, g, name, "NULL", **{name: NUL})
    _refused(_call_conv_step, g, "n_slots", "negative", n_slots=-1)
    _refused(_call_conv_step, g, "slots", "states", slots=NUL, n_slots=1)
    _refused(_call_conv_step, g, "y", "must not be", y=at(0))
    assert _call_conv(_conv(B=0), x=NUL, y=NUL, weight=NUL) == 0
    assert _call_conv(_conv(L=0), x=NUL, y=NUL, state_out=NUL) == 0
    assert _call_conv_step(_conv(B=0), x=NUL, y=NUL, state=NUL) == 0


def _call_scan(g, **kw):
    a = dict(x=at(0), dt=at(1), A=A, Bm=at(2), C=at(3), skip=A, z=at(4), bias=A, lengths=A, y=at(5),
             state_in=at(6), state_out=at(7), ws=A, n=1 << 40)
    return fv.lib().favor_selective_scan(ctypes.byref(g), *{**a, **kw}.values(), None)


def _call_scan_backward(g, **kw):
    a = dict(x=at(0), dt=at(1), A=at(20), Bm=at(2), C=at(3), skip=A, z=at(4), bias=A, lengths=A,
             state_in=at(5), dy=at(6), dstate_out=at(7), dx=at(8), ddt=at(9), dA=at(10), dB=at(11),
             dC=at(12), dskip=at(13), dz=at(14), dbias=at(15), dstate_in=at(16), ws=A, n=1 << 40)
    return fv.lib().favor_selective_scan_backward(ctypes.byref(g), *{**a, **kw}.values(), None)


def _call_scan_step(g, **kw):
    a = dict(x=at(0), dt=at(1), A=A, Bm=at(2), C=at(3), skip=A, z=at(4), bias=A, slots=A, n_slots=4,
             state=at(5), y=at(6))
    return fv.lib().favor_selective_scan_step(ctypes.byref(g), *{**a, **kw}.values(), None)


def test_scan_refusals():
    g, odd = _scan(L=100000), P((1 << 20) + 1)
    for name in ("x", "dt", "A", "Bm", "C", "y", "ws"):
        _refused(_call_scan, g, name, "NULL", **{name: NUL})
    for name in ("x", "dt", "A", "Bm", "C", "skip", "z", "bias", "lengths", "y", "state_in", "state_out", "ws"):
        _refused(_call_scan, g, name, "aligned", **{name: odd})
    for k in (0, 1, 2, 3, 4):
        _refused(_call_scan, g, "y", "must not be", y=at(k))
    _refused(_call_scan, g, "state_out", "overlaps", state_out=P((7 << 40) + 64))
    assert _call_scan(g, n=10) == 3
    for name in ("x", "dt", "A", "Bm", "C", "dy", "dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "dbias", "ws"):
        _refused(_call_scan_backward, g, name, "NULL", **{name: NUL})
    for name in ("dx", "ddt", "dB", "dC", "dz"):
        for k in (0, 1, 2, 3, 4, 6):
            _refused(_call_scan_backward, g, name, "must not be", **{name: at(k)})
    _refused(_call_scan_backward, g, "dz", "must not be", dz=at(8))
    _refused(_call_scan_backward, g, "dA", "overlaps", dA=at(20))
    _refused(_call_scan_backward, g, "dstate_in", "overlaps", dstate_in=at(5))
    _refused(_call_scan_backward, g, "dstate_in", "overlaps", dstate_in=P((8 << 40) + 64))
    assert _call_scan_backward(g, n=10) == 3
    for name in ("x", "dt", "A", "Bm", "C", "y", "state"):
        _refused(_call_scan_step, g, name, "NULL", **{name: NUL})
    _refused(_call_scan_step, g, "slots", "states", slots=NUL, n_slots=1)
    _refused(_call_scan_step, g, "y", "must not be", y=at(4))
    assert _call_scan(_scan(B=0), x=NUL, y=NUL, A=NUL) == 0
    assert _call_scan_step(_scan(B=0), x=NUL, y=NUL, state=NUL) == 0


def _call_select(g, **kw):
    a = dict(logits=at(0), scores=at(1), ended=at(2), out=at(3), parent=at(4), token=at(5), ws=A, n=1 << 40)
    return fv.lib().favor_beam_select(ctypes.byref(g), *{**a, **kw}.values(), None)


def test_beam_select_refusals():
    mk = lambda **kw: fv.make_beam_desc(**{**dict(B=2, K=3, V=100, n=4, dtype=fv.F32, end_token=5), **kw})
    for kw, status in ((dict(B=-1), 1), (dict(K=0), 1), (dict(V=0), 1), (dict(n=0), 1), (dict(K=65), 2),
                       (dict(n=65), 2), (dict(V=(1 << 30) + 1), 2), (dict(B=30000), 2), (dict(dtype=3), 1),
                       (dict(end_token=100), 1), (dict(batch_stride=-1), 1), (dict(beam_stride=1 << 50), 2),
                       (dict(end_token=-1), 1)):
        assert _call_select(mk(**kw)) == status, kw
    for name in ("logits", "scores", "out", "parent", "token", "ws"):
        _refused(_call_select, mk(), name, "NULL", **{name: NUL})
    _refused(_call_select, mk(), "scores", "overlaps", out=at(1))
    assert _call_select(mk(), n=1) == 3
    assert _call_select(mk(B=0), logits=NUL) == 0


def test_beam_reorder_refusals():
    def call(B=2, K=3, parent=at(0), slots=at(1), new=at(2), pools=((at(3), 64, 6),)):
        table = (fv.FavorBeamPool * len(pools))(*pools)
        return fv.lib().favor_beam_reorder(B, K, parent, slots, new, table, len(pools), None)

    for kw, status, word in (
            (dict(B=-1), 1, "negative"), (dict(K=65), 2, "at most 64"), (dict(B=65536), 2, "65535"),
            (dict(parent=NUL), 1, "parent"), (dict(new=NUL), 1, "new_slots"), (dict(new=at(1)), 1, "overlaps"),
            (dict(new=P((1 << 40) + 8)), 1, "overlaps"), (dict(pools=((NUL, 64, 6),)), 1, "pool"),
            (dict(pools=((at(3), 40, 6),)), 2, "multiples of 16"), (dict(pools=((at(3), -16, 6),)), 1, "negative"),
            (dict(pools=((P(8), 64, 6),)), 1, "aligned"), (dict(pools=((at(3), 64, -1),)), 1, "negative"),
            (dict(pools=((at(3), 64, 6), (at(3), 64, 6))), 1, "are one"),
            (dict(pools=((at(3), 64, 6), (P(at(3).value + 64 * 6 - 16), 64, 6))), 1, "overlap"),
            (dict(pools=((P(at(3).value + 16), 64, 6), (at(3), 1 << 34, 1 << 30))), 1, "overlap")):
        assert call(**kw) == status and word in fv.last_error(), (kw, fv.last_error())
    assert call(B=0, parent=NUL, new=NUL) == 0
    # side by side: taken (with no entries, so that nothing is launched)
    for other in (at(3).value + 64 * 6, at(3).value - 64 * 6):
        assert call(B=0, pools=((at(3), 64, 6), (P(other), 64, 6))) == 0


def test_neighbouring_outputs_do_not_overlap():
    """Small tensors lie side by side: sizes of both sides count, not the larger one twice."""
    g = fv.make_beam_desc(2, 3, 100, 64, fv.F32, end_token=5)
    s = at(1).value   # scores: 24 bytes, out_scores: 512, ended: 6
    for lo, status, word in ((s + 24, 3, "workspace"), (s + 20, 1, "out_scores overlaps scores"),
                             (s - 512, 3, "workspace"), (s - 508, 1, "out_scores overlaps scores")):
        assert _call_select(g, out=P(lo), n=1) == status and word in fv.last_error(), lo - s
    e = at(2).value
    for lo, status in ((e + 8, 3), (e + 4, 1), (e - 512, 3), (e - 508, 1)):
        assert _call_select(g, token=P(lo), n=1) == status, lo - e


def test_sizes_past_what_offsets_hold():
    """Rows far apart, and more elements than 2^46, are refused before any size is formed."""
    far = (1 << 25) // 4 + 4
    for f in ("x", "dt", "z", "y"):
        g = _scan(dtype=fv.F32, L=4, **{f: (4 * far, far, far)})
        assert fv.validate_scan_desc(g, 0) == 2 and "2^25 bytes" in fv.last_error(), f
        assert fv.validate_scan_desc(_scan(dtype=fv.F32, L=4, **{f: (4 * far, far, far - 4)}), 0) == 0
    big = dict(B=65535, L=1 << 30)
    for op in (0, 1):
        assert fv.validate_conv_desc(_conv(D=8, **big), op) == 2 and "2^46" in fv.last_error()
        assert fv.validate_scan_desc(_scan(D=8, N=1, **big), op) == 2 and "2^46" in fv.last_error()
        assert fv.scan_workspace_size(_scan(D=8, N=1, **big), bool(op)) == 0
    # 2^30 rows of parts are held in 64 bits
    g = _conv(B=2048, L=1 << 30, D=8, width=2, dtype=fv.F32)
    assert fv.validate_conv_desc(g, 1) == 0 and fv.conv_workspace_size(g) > 1 << 30


def test_sizes_past_one_launch():
    """A launch takes less than 2^32 threads: what a card holds is taken, longer rows are refused
    before anything is launched."""
    for g in (_scan(B=1, L=1 << 26, D=8, N=64, groups=1), _scan(B=1, L=1 << 20, D=128, N=256, groups=16),
              _scan(B=1, L=1 << 30, D=8, N=1, groups=1), _scan(B=1, L=1 << 30, D=256, N=1, groups=32)):
        assert fv.validate_scan_desc(g, 1) == 0 and fv.scan_workspace_size(g, True) > 0
    for L, status in (((1 << 22), 0), ((1 << 22) + 1, 2)):
        for op in (0, 1):
            assert fv.validate_scan_desc(_scan(B=1, L=L, D=65536, N=1, groups=1), op) == status
            assert fv.validate_conv_desc(_conv(B=1, L=L, D=65536), op) == status
            assert status == 0 or "2^38" in fv.last_error()
        for g, check in ((_scan(B=1, L=L, D=65536, N=1, groups=1), fv.validate_scan_desc),
                         (_conv(B=1, L=L, D=65536), fv.validate_conv_desc)):
            assert check(g, 2) == 0   # a single token's L has no effect


def test_binding_refusals():
    import torch
    z = torch.zeros
    x, w, b = z(2, 5, 16), z(16, 4), z(16)
    s, A_, low = z(2, 3, 16), z(16, 8), z(2, 5, 2, 8)
    h, i32 = z(2, 16, 8), torch.int32
    bad = [
        (lambda: fv.causal_conv(x[0], w), "x must be"),
        (lambda: fv.causal_conv(x, w[0]), "weight must be"),
        (lambda: fv.causal_conv(x, w[:8]), "weight"),
        (lambda: fv.causal_conv(x, w.bfloat16()), "weight"),
        (lambda: fv.causal_conv(x, w, b[:8]), "bias"),
        (lambda: fv.causal_conv(x, z(16, 9)), "width=9"),
        (lambda: fv.causal_conv(x[..., ::2], w[:8]), "contiguous"),
        (lambda: fv.causal_conv(x, w, lengths=z(2)), "lengths"),
        (lambda: fv.causal_conv(x, w, state_in=s[:, :2]), "state_in"),
        (lambda: fv.causal_conv(x, w, state_in=s.bfloat16()), "state_in"),
        (lambda: fv.causal_conv(x, w, out=x[:, :4]), "out"),
        (lambda: fv.causal_conv(x.half(), w), "dtype"),
        (lambda: fv.causal_conv(x, w), "GPU tensors"),
        (lambda: fv.causal_conv_backward(x, w, x[:1]), "dout"),
        (lambda: fv.causal_conv_backward(x, w, x, dweight=z(16, 3)), "dweight"),
        (lambda: fv.causal_conv_step(x, w, s), "x must be"),
        (lambda: fv.causal_conv_step(x[:, 0], w, s[:, :2]), "state"),
        (lambda: fv.causal_conv_step(x[:, 0], w, s, slots=z(3, dtype=i32)), "slots"),
        (lambda: fv.selective_scan(x, x[:1], A_, low, low), "dt"),
        (lambda: fv.selective_scan(x, x, A_[0], low, low), "A must be"),
        (lambda: fv.selective_scan(x, x, A_[:8], low, low), "A"),
        (lambda: fv.selective_scan(x, x, A_, low[:, :, 0], low), "B must be"),
        (lambda: fv.selective_scan(x, x, A_, low, low[..., :4]), "C"),
        (lambda: fv.selective_scan(x, x, A_, low, low, z=x.bfloat16()), "z"),
        (lambda: fv.selective_scan(x, x, A_, low, low, D=b[:8]), "D"),
        (lambda: fv.selective_scan(x, x, A_, low, low, dt_bias=b.double()), "dt_bias"),
        (lambda: fv.selective_scan(x, x, A_, low, low, state_in=h[:, :8]), "state_in"),
        (lambda: fv.selective_scan(x, x, A_, z(2, 5, 4, 8), z(2, 5, 4, 8)), "multiple of 8"),
        (lambda: fv.selective_scan(x, x, A_, low, low), "GPU tensors"),
        (lambda: fv.selective_scan_backward(x, x, A_, low, low, x, dB=low[:, :, :1]), "dB"),
        (lambda: fv.selective_scan_backward(x, x, A_, low, low, x, dA=A_.t()), "dA"),
        (lambda: fv.selective_scan_step(x, x, A_, low, low, h), "x must be"),
        (lambda: fv.selective_scan_step(x[:, 0], x[:, 0], A_, low[:, 0], low[:, 0], h[0]), "state"),
        (lambda: fv.beam_select(x[0], z(2, 5)), "logits must be"),
        (lambda: fv.beam_select(x, z(2, 4)), "scores"),
        (lambda: fv.beam_select(x, z(2, 5), ended=z(2, 5)), "ended"),
        (lambda: fv.beam_select(x, z(2, 5), n=0), "n=0"),
        (lambda: fv.beam_select(x.transpose(1, 2), z(2, 16)), "contiguous"),
        (lambda: fv.beam_select(x, z(2, 5)), "GPU tensors"),
        (lambda: fv.beam_reorder(z(4, dtype=i32), None, []), "parent"),
        (lambda: fv.beam_reorder(z(2, 4), None, []), "parent"),
        (lambda: fv.beam_reorder(z(2, 4, dtype=i32), z(2, 3, dtype=i32), []), "slots"),
        (lambda: fv.beam_reorder(z(2, 4, dtype=i32), None, [z(8, 4)]), "GPU tensors"),
    ]
    for n, (call, text) in enumerate(bad):
        with pytest.raises(fv.FavorError) as e:
            call()
        assert text in str(e.value), (n, text, str(e.value))


# ------------------------------------------------------------------ under sanitizers
@pytest.fixture(scope="module")
def fuzzer(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(os.path.join(ROCM_INCLUDE, "hip")):
        pytest.skip("needs g++ and the HIP headers")
    csrc = "paper_2006_03555_amd/csrc"
    sources = ["tests/host/fuzz_recurrent.cpp", "tests/host/stubs.cpp",
               f"{csrc}/recurrent_api.cpp", f"{csrc}/favor_api.cpp", f"{csrc}/timing.cpp"]
    exe = str(tmp_path_factory.mktemp("host") / "fuzz_recurrent")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer",
                        "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", f"{ROOT}/include",
                        *[os.path.join(ROOT, x) for x in sources], "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_calls_fuzzed_under_sanitizers(fuzzer, seed):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([fuzzer, str(seed), "40000"], capture_output=True, text=True, env=env,
                       timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert " 0 failures" in r.stdout


def test_launches_of_many_and_huge_pools(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(os.path.join(ROCM_INCLUDE, "hip")):
        pytest.skip("needs g++ and the HIP headers")
    csrc = "paper_2006_03555_amd/csrc"
    sources = ["tests/host/reorder_launches.cpp", "tests/host/stubs.cpp",
               f"{csrc}/recurrent_api.cpp", f"{csrc}/favor_api.cpp", f"{csrc}/timing.cpp"]
    exe = str(tmp_path / "reorder_launches")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I",
                        f"{ROOT}/include", *[os.path.join(ROOT, x) for x in sources], "-o", exe,
                        "-Wl,--unresolved-symbols=ignore-all"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
