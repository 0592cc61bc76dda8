"""The selective scan on the GPU against the fp64 oracle, each element within the first-order
bound that the oracle carries through the same recurrences."""
import numpy as np
import pytest

from helpers import to_dev, to_host, torch_dtype
from oracle import recurrent as rec
from test_gpu_conv import _round, near

pytestmark = pytest.mark.gpu
GRADS = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "dstate")
PARAMS = ("dA", "dD", "ddt_bias", "dstate")


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def inputs(B, L, D, N, G, dtype, seed, skip=True, z=True, bias=True, state=True, soft=True):
    r = np.random.default_rng(seed)
    f32 = lambda v: v.astype(np.float32)
    draw = lambda *s: _round(r.standard_normal(s), dtype)
    dt = draw(B, L, D)
    if not soft:
        dt = _round(np.abs(dt) * 0.1, dtype)
    return dict(x=draw(B, L, D), dt=dt, A=f32(-np.exp(r.uniform(-3, 1.5, (D, N)))),
                Bm=draw(B, L, G, N), C=draw(B, L, G, N),
                skip=f32(r.standard_normal(D)) if skip else None, z=draw(B, L, D) if z else None,
                bias=f32(r.uniform(-4, 0, D) if soft else r.uniform(0, 0.1, D)) if bias else None,
                state=f32(r.standard_normal((B, D, N))) if state else None, dy=draw(B, L, D),
                dstate=f32(r.standard_normal((B, D, N))) if state else None)


def dev(i, dtype):
    own = ("x", "dt", "Bm", "C", "z", "dy")
    return {k: None if v is None else to_dev(v, dtype if k in own else "f32") for k, v in i.items()}


def forward(t, **kw):
    return _fv().selective_scan(t["x"], t["dt"], t["A"], t["Bm"], t["C"], t["skip"], t["z"], t["bias"],
                                state_in=t["state"], return_state=True, **kw)


def backward(t, **kw):
    return _fv().selective_scan_backward(
        t["x"], t["dt"], t["A"], t["Bm"], t["C"], t["dy"], t["skip"], t["z"], t["bias"],
        state_in=t["state"], dstate_out=t["dstate"], return_state_grad=True, **kw)


def _args(i):
    return [i[k] for k in ("x", "dt", "A", "Bm", "C")]


def _opts(i, soft, lengths):
    return dict(skip=i["skip"], z=i["z"], bias=i["bias"], soft=soft, lengths=lengths, state=i["state"])


def check(i, dtype, got, grads, soft=True, lengths=None):
    y, s = got
    ref, sref = rec.scan(*_args(i), **_opts(i, soft, lengths))
    refs = rec.scan_backward(*_args(i), i["dy"], dstate=i["dstate"], **_opts(i, soft, lengths))
    units = rec.scan_bounds(*_args(i), i["dy"], dstate=i["dstate"], **_opts(i, soft, lengths))
    near(y, ref, units[0], dtype, "y")
    near(s, sref, units[1], "f32", "state")
    for g, r, u, name in zip(grads, refs, units[2:], GRADS):
        assert (g is None) == (r is None), name
        if g is not None:
            near(g, r, u, "f32" if name in PARAMS else dtype, name)


SHAPES = [  # B, L, D, N, G
    (1, 1, 8, 1, 1), (2, 3, 16, 4, 2), (1, 8, 24, 16, 1), (1, 127, 8, 16, 1), (2, 128, 72, 5, 1),
    (1, 129, 40, 16, 1), (1, 385, 136, 16, 1), (3, 200, 48, 24, 3), (1, 150, 16, 64, 2),
    (1, 140, 8, 130, 1), (1, 131, 8, 256, 1), (1, 700, 64, 16, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,L,D,N,G", SHAPES)
def test_forward_and_backward(B, L, D, N, G, dtype):
    i = inputs(B, L, D, N, G, dtype, 3 * L + N)
    t = dev(i, dtype)
    check(i, dtype, forward(t), backward(t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("skip,z,bias,state,soft", [
    (0, 0, 0, 0, 1), (1, 0, 0, 1, 0), (0, 1, 1, 0, 0), (0, 0, 1, 1, 1), (1, 1, 0, 0, 1)])
def test_without_parts(skip, z, bias, state, soft, dtype):
    i = inputs(2, 133, 24, 7, 1, dtype, 17, skip, z, bias, state, soft)
    t = dev(i, dtype)
    check(i, dtype, forward(t, softplus=bool(soft)), backward(t, softplus=bool(soft)), bool(soft))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch(dtype):
    """Lengths of 0 and 1, at chunk borders and out of range; padding that is NaN or Inf."""
    import torch
    B, L = 7, 300
    lengths = [300, 0, 1, 128, 129, -3, 999]
    i = inputs(B, L, 16, 9, 2, dtype, 5)
    t = dev(i, dtype)
    n = np.clip(lengths, 0, L)
    for b in range(B):
        for k in ("x", "dt", "Bm", "C", "z", "dy"):
            t[k][b, n[b]:] = float("nan") if b % 2 else float("inf")
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got, grads = forward(t, lengths=lens), backward(t, lengths=lens)
    check(i, dtype, got, grads, True, lengths)
    for b in range(B):
        for v in (got[0], grads[0], grads[1], grads[3], grads[4], grads[6]):
            assert not v[b, n[b]:].any()
        if n[b] == 0:
            assert torch.equal(got[1][b], t["state"][b]) and torch.equal(grads[8][b], t["dstate"][b])


def test_strides_and_untouched_neighbours():
    """Slices of projections in and out, groups in another order, broadcast inputs."""
    import torch
    fv = _fv()
    B, L, D, N, G = 2, 140, 32, 8, 2
    i = inputs(B, L, D, N, G, "bf16", 23)
    t = dev(i, "bf16")
    want, wants = forward(t), backward(t)
    both = torch.full((B, L, 2 * D), 3.0, device="cuda", dtype=torch.bfloat16)
    both[..., :D], both[..., D:] = t["x"], t["z"]
    odd = 2 * G * N + 5   # B and C behind five others: not aligned
    low = torch.full((B, L, odd), 3.0, device="cuda", dtype=torch.bfloat16)
    bc = low[..., 5:].unflatten(-1, (2, N, G)).transpose(-1, -2)
    bc[:, :, 0], bc[:, :, 1] = t["Bm"], t["C"]
    # a group's states must be contiguous
    with pytest.raises(fv.FavorError, match="contiguous"):
        fv.selective_scan(t["x"], t["dt"], t["A"], bc[:, :, 0], bc[:, :, 1])
    bc = low[..., 5:].unflatten(-1, (2, G, N))
    bc[:, :, 0], bc[:, :, 1] = t["Bm"], t["C"]
    u = dict(t, x=both[..., :D], z=both[..., D:], Bm=bc[:, :, 0], C=bc[:, :, 1])
    out = torch.full((B, L, 3 * D), 7.0, device="cuda", dtype=torch.bfloat16)
    got = forward(u, out=out[..., D:2 * D])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (out[..., :D] == 7).all() and (out[..., 2 * D:] == 7).all()
    dboth = torch.full((B, L, 3 * D), 7.0, device="cuda", dtype=torch.bfloat16)
    dlow = torch.full((B, L, odd), 7.0, device="cuda", dtype=torch.bfloat16)
    dbc = dlow[..., 5:].unflatten(-1, (2, G, N))
    grads = backward(u, dx=dboth[..., :D], dz=dboth[..., D:2 * D], dB=dbc[:, :, 0], dC=dbc[:, :, 1])
    for a, b in zip(grads, wants):
        assert torch.equal(a, b)
    assert (dboth[..., 2 * D:] == 7).all() and (dlow[..., :5] == 7).all()
    still = dict(t, Bm=t["Bm"][:, :1].expand(B, L, G, N), x=t["x"][:1].expand(B, L, D))
    plain = {k: None if v is None else v.contiguous() for k, v in still.items()}
    for a, b in zip((*forward(still), *backward(still)), (*forward(plain), *backward(plain))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_and_states_in_place(dtype):
    """Two pieces whose state goes on in place, forward and back, against the whole's oracle."""
    B, L, L1 = 2, 300, 170
    i = inputs(B, L, 40, 16, 1, dtype, 31)
    t = dev(i, dtype)
    cut = lambda d, s: {k: v[:, s] if k in ("x", "dt", "Bm", "C", "z", "dy") else v for k, v in d.items()}
    a, b = cut(t, slice(0, L1)), cut(t, slice(L1, L))
    s = t["state"].clone()
    middle = None
    ya, _ = forward(dict(a, state=s), state_out=s)
    middle = s.clone()
    yb, end = forward(dict(b, state=s), state_out=s)
    q = t["dstate"].clone()
    gb = backward(dict(b, state=middle, dstate=q), dstate_in=q)
    ga = backward(dict(a, dstate=q), dstate_in=q)
    import torch
    grads = []
    for k, name in enumerate(GRADS):
        if name == "dstate":
            grads.append(q)
        elif name in PARAMS:
            grads.append(ga[k] + gb[k])
        else:
            grads.append(torch.cat((ga[k], gb[k]), 1))
    check(i, dtype, (torch.cat((ya, yb), 1), end), grads)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,N,G", [(8, 1, 1), (24, 5, 3), (72, 16, 1), (16, 64, 2), (8, 131, 1),
                                   (16, 256, 1)])
def test_single_tokens(D, N, G, dtype):
    """Tokens one by one on a pool against the stretch; absent sequences and shared places."""
    import torch
    fv = _fv()
    T = 6
    i = inputs(4, T, D, N, G, dtype, 41)
    t = dev(i, dtype)
    ref, end = rec.scan(*_args(i), **_opts(i, True, None))
    units = rec.scan_bounds(*_args(i), i["dy"], dstate=i["dstate"], **_opts(i, True, None))
    pool = torch.full((6, D, N), 9.0, device="cuda")
    places = [4, 0, 5, 2]
    pool[places] = t["state"]
    slots = torch.tensor(places[:1] + [-1] + places[1:] + [6], dtype=torch.int32, device="cuda")
    live = [0, 2, 3, 4]

    def spread(v, k):
        w = torch.zeros((6,) + v.shape[2:], device="cuda", dtype=torch_dtype(dtype))
        w[live] = v[:, k]
        return w

    for k in range(T):
        y = fv.selective_scan_step(spread(t["x"], k), spread(t["dt"], k), t["A"], spread(t["Bm"], k),
                                   spread(t["C"], k), pool, t["skip"], spread(t["z"], k), t["bias"],
                                   slots=slots)
        near(y[live], ref[:, k], units[0][:, k], dtype, f"token {k}")
        assert not y[1].any() and not y[5].any()
    near(pool[places], end, units[1], "f32", "states")
    assert (pool[[1, 3]] == 9).all()
    pool[3] = t["state"][0]
    order = [(0, 0), (1, 0), (0, 1), (0, 2)]
    row = lambda v: torch.stack([v[b, k] for b, k in order])
    y = fv.selective_scan_step(row(t["x"]), row(t["dt"]), t["A"], row(t["Bm"]), row(t["C"]), pool,
                               t["skip"], row(t["z"]), t["bias"],
                               slots=torch.tensor([3, 1, 3, 3], dtype=torch.int32, device="cuda"))
    near(y[[0, 2, 3]], ref[0, :3], units[0][0, :3], dtype, "turns")


def test_extreme_steps():
    """Steps of 0 and of many units, a decay of exp(-1e4), one of exp(-0)."""
    i = inputs(1, 260, 16, 4, 1, "f32", 51)
    i["dt"][0, :, 0] = -200.0      # softplus 0 in fp32: the state stays
    i["dt"][0, :, 1] = 60.0        # everything is forgotten at every token
    i["dt"][0, 100:110, 2] = 90.0
    i["A"][3] = -1e4
    i["A"][4] = -0.0
    t = dev(i, "f32")
    check(i, "f32", forward(t), backward(t))


def test_empty_calls():
    import torch
    fv = _fv()
    i = inputs(2, 4, 8, 3, 1, "f32", 1)
    t = dev(i, "f32")
    for k in ("x", "dt", "Bm", "C", "z", "dy"):
        t[k] = t[k][:, :0].contiguous()
    y, s = forward(t)
    assert y.shape == (2, 0, 8) and torch.equal(s, t["state"])
    g = backward(t)
    assert torch.equal(g[8], t["dstate"])
    for k in (2, 5, 7):
        assert not g[k].any()
    none = {k: v if v is None or k in ("A", "skip", "bias") else v[:0] for k, v in t.items()}
    assert forward(none)[0].shape == (0, 0, 8)
    _ = fv


def test_gradients_of_no_sequence():
    """The parameters' gradients of an empty batch are sums of nothing, whatever their memory held."""
    import torch
    fv = _fv()
    i = inputs(1, 150, 8, 3, 1, "f32", 2)
    t = {k: v if k in ("A", "skip", "bias") else v[:0] for k, v in dev(i, "f32").items()}
    into = {k: torch.full_like(t[n], 7.0) for k, n in (("dA", "A"), ("dD", "skip"), ("ddt_bias", "bias"))}
    g = dict(zip(GRADS, backward(t, **into)))
    for k, v in into.items():
        assert g[k] is v and not v.any(), k
    assert g["dx"].shape == (0, 150, 8) and g["dstate"].shape == (0, 8, 3)
    fv.selective_scan_backward(t["x"], t["dt"], t["A"], t["Bm"], t["C"], t["dy"], dA=into["dA"].fill_(7))
    assert not into["dA"].any()


def test_not_a_number_stays_in_its_channel():
    import torch
    i = inputs(2, 300, 24, 16, 1, "f32", 61)
    t = dev(i, "f32")
    want, grads = forward(t), backward(t)
    u = dict(t, x=t["x"].clone())
    u["x"][0, 150, 5] = float("nan")
    got = forward(u)
    hit = torch.zeros((2, 300, 24), dtype=torch.bool, device="cuda")
    hit[0, 150:, 5] = True
    assert torch.equal(got[0].isnan(), hit)
    assert torch.equal(got[0][~hit], want[0][~hit])
    dx = backward(u)[0]
    clean = torch.ones((2, 300, 24), dtype=torch.bool, device="cuda")
    clean[0, :, 5] = False
    assert torch.equal(dx[clean], grads[0][clean])


def test_gradients_against_differences():
    i = inputs(1, 40, 8, 6, 1, "f32", 71)
    grads = backward(dev(i, "f32"))
    r = np.random.default_rng(2)
    names = ("x", "dt", "A", "Bm", "C", "skip", "z", "bias", "state")
    for k, g in zip(names, grads):
        step = r.standard_normal(i[k].shape)
        h = 1e-5

        def loss(s):
            j = {n: None if v is None else v.astype(np.float64) for n, v in i.items()}
            j[k] = j[k] + s * step
            y, end = rec.scan(*_args(j), **_opts(j, True, None))
            return (y * j["dy"]).sum() + (end * j["dstate"]).sum()

        want = (loss(h) - loss(-h)) / (2 * h)
        assert abs((to_host(g) * step).sum() - want) < 2e-5 * np.abs(to_host(g) * step).sum(), k


@pytest.mark.parametrize("B,L,D,N", [(1, 4099, 64, 16), (2, 1999, 1000, 24), (1, 20000, 8, 8)])
def test_long_and_wide(B, L, D, N):
    """Sequences of many segments and chunks, by norm: fp32 against fp64 on sampled channels."""
    i = inputs(B, L, D, N, 1, "f32", 81)
    t = dev(i, "f32")
    got, grads = forward(t), backward(t)
    c = [0, D // 2, D - 1] if D > 8 else list(range(D))
    j = {k: None if v is None else
         v[..., c] if k in ("x", "dt", "skip", "z", "bias", "dy") else
         v[c] if k == "A" else v[:, c] if k in ("state", "dstate") else v for k, v in i.items()}
    ref = rec.scan(*_args(j), **_opts(j, True, None))
    refs = rec.scan_backward(*_args(j), j["dy"], dstate=j["dstate"], **_opts(j, True, None))
    pick = lambda v, name: to_host(v[c] if name in ("dA", "dD", "ddt_bias") else
                                   v[:, c] if name in ("dstate", "state") else v[..., c])
    for g, r, name in zip((*got, *grads), (*ref, *refs), ("y", "state") + GRADS):
        if name in ("dB", "dC") and len(c) < D:
            continue   # sums over all channels
        err = np.linalg.norm(pick(g, name) - r) / np.linalg.norm(r) if name not in ("dB", "dC") else (
            np.linalg.norm(to_host(g) - r) / np.linalg.norm(r))
        # a few dozen roundings of 2^-24 that do not conspire
        assert err < 40 * 2.0 ** -24, (name, err)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,L,D,N,G", [
    (16, 300, 2080, 16, 2), (20, 300, 2080, 5, 2), (20, 259, 2048, 16, 1), (17, 40, 2048, 128, 1)])
def test_many_workgroups(B, L, D, N, G, dtype):
    """Batches that fill the card: one segment forward, two and four tiles to a workgroup
    backward. The gradients that come in are zero but for three sequences, so the
    parameters' gradients are those of the three, with exact zeros of the others."""
    some = [0, B // 2 + 1, B - 1]
    i = inputs(B, L, D, N, G, dtype, 91)
    for k in ("dy", "dstate"):
        i[k][[b for b in range(B) if b not in some]] = 0
    t = dev(i, dtype)
    (y, s), grads = forward(t), backward(t)
    of = lambda k, v: v if v is None or k in ("A", "skip", "bias") else v[some]
    j = {k: of(k, v) for k, v in i.items()}
    cut = [g if name in ("dA", "dD", "ddt_bias") else g[some] for g, name in zip(grads, GRADS)]
    check(j, dtype, (y[some], s[some]), cut)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [300, 5])
def test_steps_of_nothing(L, dtype):
    """A dt of the type's lowest value or -Inf is a step of zero: the state stays bit by bit,
    x there has no gradient but through the skip, and dt none."""
    import torch
    i = inputs(2, L, 24, 16, 1, dtype, 17)
    t = dev(i, dtype)
    cut = L - 3
    low = float(torch.finfo(t["dt"].dtype).min)
    for value in (low, -np.inf):
        u = dict(t, dt=t["dt"].clone())
        u["dt"][:, cut:] = value
        y, s = forward(u)
        n = torch.full((2,), cut, dtype=torch.int32, device="cuda")
        y1, s1 = forward(t, lengths=n)
        assert torch.equal(s, s1) and torch.equal(y[:, :cut], y1[:, :cut])
        assert torch.isfinite(y.float()).all()
        g = dict(zip(GRADS, backward(u)))
        for name, v in g.items():
            assert torch.isfinite(v.float()).all(), name
        assert not g["ddt"][:, cut:].any() and not g["dB"][:, cut:].any()
        e = u["dy"].double() * torch.nn.functional.silu(u["z"].double())
        want = (e * u["skip"].double())[:, cut:].cpu().numpy()
        near(g["dx"][:, cut:], want, 16 * np.abs(want), dtype, "dx")


def test_growth_past_the_range_of_a_segment():
    """A positive A whose growth over 128 tokens is in fp32's range, but not over a segment of
    several chunks: a state of zero stays zero until inputs come, and decays elsewhere."""
    B, L, D, N = 1, 16640, 1024, 2
    i = inputs(B, L, D, N, 1, "f32", 5, z=False, bias=False, state=False, soft=False)
    i["dt"][:] = 0.5
    i["A"][:, 0], i["A"][:, 1] = 1.0, -1.0   # e^64 in 128 tokens, e^128 in 256
    i["x"][:, :L - 100] = 0
    t = dev(i, "f32")
    y, s = _fv().selective_scan(t["x"], t["dt"], t["A"], t["Bm"], t["C"], t["skip"],
                                softplus=False, return_state=True)
    tail = {k: v if v is None or k in ("A", "skip") else v[:, L - 100:] for k, v in i.items()}
    o = dict(skip=i["skip"], z=None, bias=None, soft=False, lengths=None, state=None)
    ref, sref = rec.scan(*_args(tail), **o)
    units = rec.scan_bounds(*_args(tail), tail["dy"], **o)
    near(y[:, L - 100:], ref, units[0], "f32", "y")
    near(s, sref, units[1], "f32", "state")
    assert not y[:, :L - 100].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [17, 40])
def test_padded_batch_of_many_states(N, dtype):
    """More than 16 states: the sums' workgroups take 16 each, also where a chunk has no token."""
    import torch
    B, L, D, lengths = 5, 270, 48, [0, 1, 128, 129, 270]
    i = inputs(B, L, D, N, 2, dtype, 23)
    t = dev(i, dtype)
    for k in ("x", "dt", "z", "dy", "Bm", "C"):
        for b, n in enumerate(lengths):
            t[k][b, n:] = float("nan")
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    (y, s), grads = forward(t, lengths=n), backward(t, lengths=n)
    check(i, dtype, (y, s), grads, lengths=np.array(lengths))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_workgroups_than_a_launch_takes(dtype):
    """More than 2^20 workgroups over chunks and 2^24 values of B and C in one backward pass: a
    long sequence that forgets everything every 1024 tokens has the gradients of the stretches as
    a batch, bit by bit."""
    import torch
    fv = _fv()
    P, T, G, N = 1024, 2051, 64, 1       # 64 groups of 8 channels, 8 chunks a stretch
    L, D = T * P, 8 * G
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch_dtype(dtype))
    x, dt, dy = draw(1, L, D), draw(1, L, D), draw(1, L, D)
    B, C = draw(1, L, G, N), draw(1, L, G, N)
    dt[:, ::P] = 300   # exp(-300) is 0 in fp32: nothing goes past a stretch's first token
    A = -1 - torch.rand((D, N), generator=gen, device="cuda")
    whole = fv.selective_scan_backward(x, dt, A, B, C, dy)
    rows = lambda v: v.view((T, P) + v.shape[2:])
    batch = fv.selective_scan_backward(rows(x), rows(dt), A, rows(B), rows(C), rows(dy))
    for w, b, name in zip(whole, batch, GRADS):
        if w is not None:
            assert torch.isfinite(w).all() and w.any(), name
            assert torch.equal(w.view(b.shape), b), name


# ------------------------------------------------------------------ forward calls in segments
def _segments(B, L, D, N, G):
    """(segments, chunks of one) of a forward call, by the size of its workspace: the states before
    each segment and their sums of steps."""
    fv = _fv()
    n = fv.scan_workspace_size(fv.make_scan_desc(B, L, D, N, fv.F32, G))
    per, chunks = 4 * B * D * (N + 1), -(-L // 128)
    nseg = round(n / per) if n else 1
    assert abs(n - nseg * per) <= 512 or nseg == 1
    return nseg, -(-chunks // nseg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,lengths", [(5, None), (20, None), (16, [6500, 2500])])
def test_carry_between_chunks_of_a_segment(N, lengths, dtype):
    """Segments of three chunks: the state goes on inside a segment, in the sums and in the rows,
    with ends in the middle of a segment and of a chunk."""
    import torch
    B, L, G = 1 if lengths is None else 2, 6875, 210 if lengths is None else 105
    D = 8 * G
    assert _segments(B, L, D, N, G) == (18, 3)
    i = inputs(B, L, D, N, G, dtype, 7 * N)
    i["A"] *= np.float32(0.02)   # what is 128 tokens old still counts
    i["bias"] -= 3
    t = dev(i, dtype)
    kw = {} if lengths is None else dict(lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    y, s = forward(t, **kw)
    groups = [0, G // 2, G - 1]
    c = np.concatenate([np.arange(8 * g, 8 * g + 8) for g in groups])
    j = {k: None if v is None else v[:, :, groups] if k in ("Bm", "C") else v[c] if k in ("A", "skip", "bias")
         else v[:, c] if k in ("state", "dstate") else v[..., c] for k, v in i.items()}
    o = _opts(j, True, lengths)
    ref, sref = rec.scan(*_args(j), **o)
    units = rec.scan_bounds(*_args(j), j["dy"], dstate=j["dstate"], **o)
    near(y[..., c], ref, units[0], dtype, "y")
    near(s[:, c], sref, units[1], "f32", "state")
    # a carry that is lost anywhere is outside these bounds
    cut = 384 * 3 + 128
    lost = {k: v[:, cut:cut + 100] if k in ("x", "dt", "Bm", "C", "z", "dy") else v for k, v in j.items()}
    wrong, _ = rec.scan(*_args(lost), **dict(_opts(lost, True, None), state=None))
    bad = np.abs(wrong - ref[:, cut:cut + 100]) > 1.05 * 2.0 ** -24 * units[0][:, cut:cut + 100] + (
        2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref[:, cut:cut + 100])
    assert bad[0].any(0).all()   # in every channel


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("skip,z,bias,state,soft", [
    (0, 0, 0, 0, 1), (1, 0, 0, 1, 0), (0, 1, 1, 1, 0), (0, 0, 1, 1, 1), (1, 1, 0, 0, 1)])
def test_segments_without_parts(skip, z, bias, state, soft, dtype):
    assert _segments(2, 700, 24, 7, 1) == (6, 1)
    i = inputs(2, 700, 24, 7, 1, dtype, 19, skip, z, bias, state, soft)
    t = dev(i, dtype)
    check(i, dtype, forward(t, softplus=bool(soft)), backward(t, softplus=bool(soft)), bool(soft))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch_in_segments(dtype):
    """As test_padded_batch, with segments before, around and behind each end."""
    import torch
    B, L = 6, 700
    lengths = [700, 0, 1, 256, 257, 640]
    assert _segments(B, L, 16, 9, 2) == (6, 1)
    i = inputs(B, L, 16, 9, 2, dtype, 6)
    t = dev(i, dtype)
    for b, n in enumerate(lengths):
        for k in ("x", "dt", "Bm", "C", "z", "dy"):
            t[k][b, n:] = float("nan") if b % 2 else float("inf")
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got, grads = forward(t, lengths=lens), backward(t, lengths=lens)
    check(i, dtype, got, grads, True, lengths)
    for b, n in enumerate(lengths):
        for v in (got[0], grads[0], grads[1], grads[3], grads[4], grads[6]):
            assert not v[b, n:].any()
    assert torch.equal(got[1][1], t["state"][1]) and torch.equal(grads[8][1], t["dstate"][1])


@pytest.mark.parametrize("state", [0, 1])
@pytest.mark.parametrize("name", ["x", "dt"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_not_a_number_stays_in_its_channel_in_segments(value, name, state):
    """One in a middle segment reaches its own channel alone, from its token on, and the gradients
    of no other channel's rows."""
    import torch
    B, L, D, at = 2, 700, 24, 330
    assert _segments(B, L, D, 16, 1) == (6, 1)
    i = inputs(B, L, D, 16, 1, "f32", 62, state=state)
    t = dev(i, "f32")
    want, grads = forward(t), backward(t)
    u = dict(t, **{name: t[name].clone()})
    u[name][0, at, 5] = value
    y, s = forward(u)
    hit = torch.zeros((B, L, D), dtype=torch.bool, device="cuda")
    hit[0, at:, 5] = True
    assert torch.equal(y[~hit], want[0][~hit])
    assert not torch.isfinite(y[0, at, 5])
    if value != value:
        assert y[hit].isnan().all() and s[0, 5].isnan().all()
    clean = torch.ones((B, D), dtype=torch.bool, device="cuda")
    clean[0, 5] = False
    assert torch.equal(s[clean], want[1][clean])
    after = backward(u)
    for k in (0, 1, 6):   # dx, ddt, dz
        assert torch.equal(after[k].transpose(1, 2)[clean], grads[k].transpose(1, 2)[clean])
