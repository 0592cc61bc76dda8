"""Linear attention with a decay per head on the GPU against the fp64 recurrence.

Bounds, per element, with A the same formula on absolute values (what the sums add up):
  fp32: products over dk, pairs over a chunk's 64 tokens and one carry per chunk, each sum
        off by at most its number of additions times 2^-24 A, and four roundings of
        weights: (dk + 64 + 4 chunks + 16) 2^-24 A.
  bf16: the output's rounding 2^-8 |o|, the pair weights' 2^-8 A or the state's (each
        enters as one bf16 term, and A is the sum of both parts), the state's products'
        2^-16 A (two terms, each off by at most 2^-8 of what it stands for) and the
        fp32 bound. A state that is returned is the fp32 sum of exact
        products.
A gradient is the same scan with the columns' roles exchanged, so the bound's width is
the larger of dk and dv."""
import numpy as np
import pytest

from helpers import to_dev, torch_dtype
from oracle import decay
from workloads import bf16_round

pytestmark = pytest.mark.gpu

DECAYS = [-1 / 32, 0.0, -0.7, -np.inf, -1e-3, -20.0]
DTYPES = ["bf16", "f32"]


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def _inputs(B, H, L, dk, dv, dtype, seed):
    rng = np.random.default_rng(seed)
    cast = bf16_round if dtype == "bf16" else (lambda x: x)
    q, k = (cast(rng.standard_normal((B, H, L, dk)).astype(np.float32)) for _ in range(2))
    v, do = (cast(rng.standard_normal((B, H, L, dv)).astype(np.float32)) for _ in range(2))
    S, G = (rng.standard_normal((B, H, dk, dv)).astype(np.float32) for _ in range(2))
    g = np.array([DECAYS[(seed + h) % len(DECAYS)] for h in range(H)], dtype=np.float32)
    return dict(q=q, k=k, v=v, do=do, S=S, G=G, g=g)


def _laid_out(x, dtype, layout):
    """A device tensor [B, H, L, d] of x's values in the given memory layout."""
    import torch
    t = to_dev(x, dtype)
    if layout == "bhld":
        return t
    if layout == "blhd":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    B, H, L, d = x.shape   # rows inside wider ones, heads further apart than they need
    big = torch.full((B, L + 3, H + 1, d + 16), float("nan"), dtype=t.dtype, device="cuda")
    view = big[:, 2:2 + L, 1:, 8:8 + d].transpose(1, 2)
    view.copy_(t)
    return view


def _host(t):
    return t.double().cpu().numpy()


def _near(got, ref, mag, width, L, dtype, what):
    """Every element within the bound (module comment)."""
    got = _host(got) if hasattr(got, "cpu") else got
    assert np.isfinite(got).all(), what
    tol = (width + 64 + 4 * (L // 64 + 1) + 16) * 2.0 ** -24 * mag
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + (2.0 ** -8 + 2.0 ** -16) * mag
    err = np.abs(got - ref)
    bad = err > tol
    assert not bad.any(), (what, float((err / np.maximum(tol, 1e-300)).max()), int(bad.sum()))
    # the roundings are independent: the norm is off by no more than two of them
    if dtype == "bf16" and np.linalg.norm(ref) > 0 and ref.size > 1000:
        rel = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert rel < 2 * 2.0 ** -8, (what, rel)


def _abs(x):
    return {n: np.abs(t) if n != "g" else t for n, t in x.items()}


SHAPES = [  # B, H, L, dk, dv
    (1, 1, 1, 64, 64), (1, 2, 63, 64, 64), (2, 3, 64, 64, 128), (1, 2, 65, 128, 128),
    (2, 2, 130, 8, 8), (1, 3, 200, 256, 64), (1, 2, 333, 256, 256), (1, 2, 700, 72, 40),
    (1, 1, 1300, 128, 248), (3, 1, 17, 16, 200), (1, 2, 2500, 64, 64), (2, 1, 1025, 200, 136),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    fv = _fv()
    B, H, L, dk, dv = shape
    x = _inputs(*shape, dtype, sum(shape))
    layout = ["bhld", "blhd", "wide"][sum(shape) % 3]
    q, k, v = (_laid_out(x[n], dtype, layout) for n in "qkv")
    g, S = to_dev(x["g"]), to_dev(x["S"])
    c = 0.3
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"], c, state=x["S"])
    y = _abs(x)
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"], c, state=y["S"])
    out, st = fv.attn_decay(q, k, v, g, c, state_in=S, return_state=True)
    _near(out, ref, mag, dk, L, dtype, "out")
    _near(st, end, mend, dk, L, "f32", "state")
    again, st2 = fv.attn_decay(q, k, v, g, c, state_in=S, return_state=True)
    assert np.array_equal(_host(out), _host(again)) and np.array_equal(_host(st), _host(st2))
    ref, _ = decay.attn(x["q"], x["k"], x["v"], x["g"], 1.0)
    mag, _ = decay.attn(y["q"], y["k"], y["v"], x["g"], 1.0)
    _near(fv.attn_decay(q, k, v, g), ref, mag, dk, L, dtype, "out without a state")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 2, 1, 64, 64), (2, 3, 130, 64, 128), (1, 2, 700, 72, 40),
                                   (1, 3, 500, 256, 64), (1, 2, 1999, 128, 128)])
def test_states_in_but_none_out(shape, dtype):
    """A state and a state's gradient come in, none is returned: the calls whose states only
    feed rows."""
    fv = _fv()
    B, H, L, dk, dv = shape
    x = _inputs(*shape, dtype, 3 * sum(shape))
    y = _abs(x)
    q, k, v, do = (_laid_out(x[n], dtype, "blhd") for n in ("q", "k", "v", "do"))
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    ref, _ = decay.attn(x["q"], x["k"], x["v"], x["g"], 0.3, state=x["S"])
    mag, _ = decay.attn(y["q"], y["k"], y["v"], x["g"], 0.3, state=y["S"])
    _near(fv.attn_decay(q, k, v, g, 0.3, state_in=S), ref, mag, dk, L, dtype, "out")
    ref = decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"], 0.3, state=x["S"],
                              dstate=x["G"])
    mag = decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"], 0.3, state=y["S"],
                              dstate=y["G"])
    got = fv.attn_decay_backward(q, k, v, g, do, 0.3, state_in=S, dstate_out=G)
    for t, r, m, n in zip(got, ref, mag, ("dQ", "dK", "dV")):
        _near(t, r, m, max(dk, dv), L, dtype, n)


@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("L,dk,dv", [(1, 128, 184), (4, 128, 248), (3, 256, 56), (64, 64, 64),
                                     (17, 16, 128)])
def test_few_rows_in_bf16(L, dk, dv, state):
    """Rows too few for the roundings of pair weights and states to average out: both come in
    two terms, so that an output's own rounding is what is left. Element by element: 2^-8 for
    that rounding; 2^-16 of A for the pair weights, the states and the products in a state;
    (dk + 64 + 4 + 16) 2^-24 A <= 340 2^-24 A for the fp32 sums."""
    fv = _fv()
    x = _inputs(3, 2, L, dk, dv, "bf16", L + dk)
    x["g"][:] = -1 / 32
    q, k, v, do = (to_dev(x[n], "bf16") for n in ("q", "k", "v", "do"))
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    kw = dict(state=x["S"]) if state else {}
    kd = dict(kw, dstate=x["G"]) if state else {}
    ref = [decay.attn(x["q"], x["k"], x["v"], x["g"], 0.5, **kw)[0],
           *decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"], 0.5, **kd)[:3]]
    got = [fv.attn_decay(q, k, v, g, 0.5, state_in=S if state else None),
           *fv.attn_decay_backward(q, k, v, g, do, 0.5, state_in=S if state else None,
                                   dstate_out=G if state else None)]
    y = _abs(x)
    ky = dict(state=y["S"]) if state else {}
    kyd = dict(ky, dstate=y["G"]) if state else {}
    mag = [decay.attn(y["q"], y["k"], y["v"], x["g"], 0.5, **ky)[0],
           *decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"], 0.5, **kyd)[:3]]
    for t, r, m, n in zip(got, ref, mag, ("out", "dQ", "dK", "dV")):
        tol = 2.0 ** -8 * np.abs(r) * (1 + 2.0 ** -8) + (3 * 2.0 ** -16 + 340 * 2.0 ** -24) * m
        assert (np.abs(_host(t) - r) <= tol).all(), (n, state)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dk,dv", [(128, 128), (88, 128), (256, 88), (64, 64)])
def test_many_heads(dk, dv, dtype):
    """Every compute unit busy with several workgroups: each element of each head against
    the same heads run a few at a time. (A wide store whose registers were written again
    too early went wrong here in some lanes, and only under load.)"""
    import torch
    fv = _fv()
    x = _inputs(5, 21, 174, dk, dv, dtype, 6)
    q, k, v, do = (to_dev(x[n], dtype) for n in ("q", "k", "v", "do"))
    g, S = to_dev(x["g"]), to_dev(x["S"])
    for _ in range(3):
        out = fv.attn_decay(q, k, v, g, state_in=S)
        grads = fv.attn_decay_backward(q, k, v, g, do, state_in=S)
        for b in range(5):
            s = slice(b, b + 1)
            few = [fv.attn_decay(q[s], k[s], v[s], g, state_in=S[s])]
            few += fv.attn_decay_backward(q[s], k[s], v[s], g, do[s], state_in=S[s])
            for t, r in zip((out, *grads), few):
                assert torch.equal(t[s], r)
    y = _abs(x)
    ref, _ = decay.attn(x["q"], x["k"], x["v"], x["g"], 1.0, state=x["S"])
    mag, _ = decay.attn(y["q"], y["k"], y["v"], x["g"], 1.0, state=y["S"])
    _near(out, ref, mag, dk, 174, dtype, "out")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype):
    fv = _fv()
    B, H, L, dk, dv = shape
    x = _inputs(*shape, dtype, sum(shape) + 1)
    layout = ["blhd", "wide", "bhld"][sum(shape) % 3]
    q, k, v, do = (_laid_out(x[n], dtype, layout) for n in ("q", "k", "v", "do"))
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    y = _abs(x)
    for state in (True, False):
        kw = dict(state=x["S"], dstate=x["G"]) if state else {}
        ky = dict(state=y["S"], dstate=y["G"]) if state else {}
        ref = decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"], 0.4, **kw)
        mag = decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"], 0.4, **ky)
        got = fv.attn_decay_backward(q, k, v, g, do, 0.4, return_state_grad=True,
                                     **(dict(state_in=S, dstate_out=G) if state else {}))
        for t, r, m, n in zip(got, ref, mag, ("dQ", "dK", "dV")):
            _near(t, r, m, max(dk, dv), L, dtype, (n, state))
        _near(got[3], ref[3], mag[3], max(dk, dv), L, "f32", ("dstate_in", state))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,H,L,dk,dv,lengths", [
    (4, 2, 130, 64, 64, [130, 0, 64, 1]),
    (3, 2, 1500, 128, 64, [1500, 256, 777]),
    (3, 1, 600, 40, 256, [-5, 10000, 255]),      # taken as 0 and as L
])
def test_padded_batch(B, H, L, dk, dv, lengths, dtype):
    """Padding is never read (it holds NaN), its rows come out as zeros, and the states and
    gradients are those of the sequences alone."""
    import torch
    fv = _fv()
    x = _inputs(B, H, L, dk, dv, dtype, L)
    n = np.clip(lengths, 0, L)
    y = _abs(x)
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"], 1.0, n, x["S"])
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"], 1.0, n, y["S"])
    back = decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"], 1.0, n, x["S"], x["G"])
    bmag = decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"], 1.0, n, y["S"], y["G"])
    dev = {m: _laid_out(x[m], dtype, "blhd") for m in ("q", "k", "v", "do")}
    for t in dev.values():
        for b in range(B):
            t[b, :, int(n[b]):] = float("nan")
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = torch.full_like(dev["v"], 7.0)
    out, st = fv.attn_decay(dev["q"], dev["k"], dev["v"], g, lengths=ln, state_in=S,
                            return_state=True, out=out)
    _near(out, ref, mag, dk, L, dtype, "out")
    _near(st, end, mend, dk, L, "f32", "state")
    grads = [torch.full_like(dev[m], 7.0) for m in ("q", "k", "v")]
    got = fv.attn_decay_backward(dev["q"], dev["k"], dev["v"], g, dev["do"], lengths=ln,
                                 state_in=S, dstate_out=G, return_state_grad=True,
                                 dQ=grads[0], dK=grads[1], dV=grads[2])
    for t, r, m, w in zip(got, back, bmag, ("dQ", "dK", "dV")):
        _near(t, r, m, max(dk, dv), L, dtype, w)
    _near(got[3], back[3], bmag[3], max(dk, dv), L, "f32", "dstate_in")
    for t in (out, *got[:3]):
        for b in range(B):
            assert not t[b, :, int(n[b]):].any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_nothing_around_the_rows_is_written(dtype):
    """Outputs inside wider tensors: what lies between and behind their rows stays."""
    import torch
    fv = _fv()
    B, H, L, dk, dv = 2, 2, 77, 72, 40
    x = _inputs(B, H, L, dk, dv, dtype, 5)
    q, k, v, do = (to_dev(x[n], dtype) for n in ("q", "k", "v", "do"))
    g = to_dev(x["g"])

    def inside(d):
        big = torch.full((B, L + 3, H + 1, d + 16), 9.0, dtype=q.dtype, device="cuda")
        return big, big[:, 2:2 + L, 1:, 8:8 + d].transpose(1, 2)

    pairs = [inside(d) for d in (dv, dk, dk, dv)]
    fv.attn_decay(q, k, v, g, out=pairs[0][1])
    fv.attn_decay_backward(q, k, v, g, do, dQ=pairs[1][1], dK=pairs[2][1], dV=pairs[3][1])
    for big, view in pairs:
        assert (view != 9).any()
        view.fill_(9.0)
        assert (big == 9).all()


def test_a_sequence_in_pieces():
    """Pieces that hand the state on, in place, give what the whole gives; the backward
    passes of the pieces from the last one hand its gradient back."""
    fv = _fv()
    x = _inputs(2, 3, 500, 64, 128, "f32", 8)
    q, k, v, do = (to_dev(x[n]) for n in ("q", "k", "v", "do"))
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    y = _abs(x)
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"], 1.0, None, x["S"])
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"], 1.0, None, y["S"])
    back = decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"], 1.0, None, x["S"], x["G"])
    bmag = decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"], 1.0, None, y["S"], y["G"])
    cuts = [(0, 1), (1, 130), (130, 130), (130, 500)]
    s, before = S.clone(), []
    for lo, hi in cuts:
        before.append(s.clone())
        o, _ = fv.attn_decay(q[:, :, lo:hi], k[:, :, lo:hi], v[:, :, lo:hi], g, state_in=s,
                             return_state=True, state_out=s)
        _near(o, ref[:, :, lo:hi], mag[:, :, lo:hi], 64, 500, "f32", (lo, hi))
    _near(s, end, mend, 64, 500, "f32", "state")
    d = G.clone()
    for (lo, hi), b in zip(reversed(cuts), reversed(before)):
        got = fv.attn_decay_backward(*(t[:, :, lo:hi] for t in (q, k, v)), g, do[:, :, lo:hi],
                                     state_in=b, dstate_out=d, return_state_grad=True,
                                     dstate_in=d)
        for t, r, m in zip(got[:3], back, bmag):
            _near(t, r[:, :, lo:hi], m[:, :, lo:hi], 128, 500, "f32", (lo, hi))
    _near(d, back[3], bmag[3], 128, 500, "f32", "dstate_in")


def test_broadcast_inputs():
    """One K for all heads and one V for all batch entries, as expanded tensors; the
    gradients come per head and batch entry."""
    fv = _fv()
    x = _inputs(2, 3, 150, 64, 64, "f32", 9)
    x["k"] = np.repeat(x["k"][:, :1], 3, 1)
    x["v"] = np.repeat(x["v"][:1], 2, 0)
    q, do, g = to_dev(x["q"]), to_dev(x["do"]), to_dev(x["g"])
    k = to_dev(x["k"][:, :1]).expand(2, 3, 150, 64)
    v = to_dev(x["v"][:1]).expand(2, 3, 150, 64)
    y = _abs(x)
    ref, _ = decay.attn(x["q"], x["k"], x["v"], x["g"])
    mag, _ = decay.attn(y["q"], y["k"], y["v"], x["g"])
    _near(fv.attn_decay(q, k, v, g), ref, mag, 64, 150, "f32", "out")
    back = decay.attn_backward(x["q"], x["k"], x["v"], x["g"], x["do"])
    bmag = decay.attn_backward(y["q"], y["k"], y["v"], x["g"], y["do"])
    for t, r, m in zip(fv.attn_decay_backward(q, k, v, g, do), back, bmag):
        _near(t, r, m, 64, 150, "f32", "gradient")


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_decay_over_many_chunks(dtype):
    """Decays so close to 1 that one float's rounding of a^64 would add up over the
    chunks of a single segment (512 heads: no segments are split)."""
    fv = _fv()
    import torch
    B, H, L = 16, 32, 8192
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.rand((B, 1, L, 8), generator=gen, device="cuda").to(torch_dtype(dtype))
            .expand(B, H, L, 8) for _ in range(2))
    e = np.linspace(2e-6, 2e-4, H).astype(np.float32)
    _, s = fv.attn_decay(k, k, v, to_dev(-e), return_state=True)
    w = torch.exp(to_dev(-e).double()[:, None] * torch.arange(L - 1, -1, -1, device="cuda"))
    ref = (k[:, :1].double() * w[None, :, :, None]).transpose(-1, -2).contiguous() \
        @ v[:, :1].double()
    # positive sums of L terms: random fp32 roundings of 128 carries and of the sums
    # within them, 2^-24 each; a systematic one would be 64 times 2^-25 at the average age
    rel = ((s.double() - ref).norm() / ref.norm()).item()
    assert rel < 16 * 2.0 ** -24, rel


def test_empty_sizes():
    import torch
    fv = _fv()
    S = to_dev(np.arange(2 * 3 * 64 * 8, dtype=np.float32).reshape(2, 3, 64, 8))
    g = to_dev(np.full(3, -0.5))
    z = lambda *s: torch.empty(s, device="cuda")
    out, st = fv.attn_decay(z(2, 3, 0, 64), z(2, 3, 0, 64), z(2, 3, 0, 8), g, state_in=S,
                            return_state=True)
    assert out.shape == (2, 3, 0, 8) and torch.equal(st, S)
    _, st = fv.attn_decay(z(2, 3, 0, 64), z(2, 3, 0, 64), z(2, 3, 0, 8), g, return_state=True)
    assert not st.any()
    got = fv.attn_decay_backward(z(2, 3, 0, 64), z(2, 3, 0, 64), z(2, 3, 0, 8), g, z(2, 3, 0, 8),
                                 dstate_out=S, return_state_grad=True)
    assert torch.equal(got[3], S)
    out = fv.attn_decay(z(0, 3, 9, 64), z(0, 3, 9, 64), z(0, 3, 9, 8), g)
    assert out.shape == (0, 3, 9, 8)
    assert fv.attn_decay_step(z(0, 3, 64), z(0, 3, 64), z(0, 3, 8), g, S).shape == (0, 3, 8)


def test_far_rows():
    """Element offsets past 32 bits (a batch of 2 with 2^33 bytes between its entries)."""
    import torch
    fv = _fv()
    x = _inputs(2, 1, 100, 64, 64, "bf16", 4)
    far = torch.empty((1 << 32) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    ts = []
    for i, n in enumerate("qkv"):
        t = far.as_strided((2, 1, 100, 64), (1 << 32, 64, 64, 1), 8192 * i)
        t.copy_(to_dev(x[n], "bf16"))
        ts.append(t)
    out = far.as_strided((2, 1, 100, 64), (1 << 32, 64, 64, 1), 8192 * 3)
    g = to_dev(x["g"])
    fv.attn_decay(*ts, g, out=out)
    assert torch.equal(out.contiguous(), fv.attn_decay(*(t.contiguous() for t in ts), g))


# ------------------------------------------------------------------ single tokens
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 64, 64), (1, 8, 128, 128), (5, 3, 8, 248),
                                       (3, 2, 256, 256), (40, 6, 64, 72), (2, 2, 136, 8)])
def test_steps(B, H, dk, dv, dtype):
    """Steps one after another against the recurrence; and the chunked form of the same
    tokens ends at the same state."""
    import torch
    fv = _fv()
    n = 5
    x = _inputs(B, H, n, dk, dv, dtype, B + H + dk)
    q, k, v = (_laid_out(x[m], dtype, "wide") for m in "qkv")
    g = to_dev(x["g"])
    y = _abs(x)
    ref, end = decay.attn(x["q"], x["k"], x["v"], x["g"], 0.5, state=x["S"])
    mag, mend = decay.attn(y["q"], y["k"], y["v"], x["g"], 0.5, state=y["S"])
    s = to_dev(x["S"])
    for t in range(n):
        o = fv.attn_decay_step(q[:, :, t], k[:, :, t], v[:, :, t], g, s, 0.5)
        # sums over dk and two roundings of the state per step; the output's own rounding
        tol = (dk + 4 * n) * 2.0 ** -24 * mag[:, :, t] + (
            2.0 ** -8 * np.abs(ref[:, :, t]) * (1 + 2.0 ** -8) if dtype == "bf16" else 0)
        assert (np.abs(_host(o) - ref[:, :, t]) <= tol).all(), t
    _near(s, end, mend, dk, n, "f32", "state")
    _, whole = fv.attn_decay(q, k, v, g, 0.5, state_in=to_dev(x["S"]), return_state=True)
    _near(whole, end, mend, dk, n, "f32", "state of the chunked form")


@pytest.mark.parametrize("slots", [
    [3, 0, 5], [6, -1, 2], [7, 1 << 30, -(1 << 31)],        # places outside: no state
    [4, 4, 4], [2, 5, 2], [5, 2, 2], [2, 2, 5],             # taken in order
])
def test_step_places(slots):
    import torch
    fv = _fv()
    H, dk, dv, pool = 2, 64, 40, 7
    x = _inputs(3, H, 1, dk, dv, "f32", 11)
    rng = np.random.default_rng(0)
    S = rng.standard_normal((pool, H, dk, dv)).astype(np.float32)
    s = to_dev(S)
    q, k, v = (to_dev(x[n][:, :, 0]) for n in "qkv")
    out = torch.full((3, H, dv), 9.0, device="cuda")
    fv.attn_decay_step(q, k, v, to_dev(x["g"]), s, slots=torch.tensor(slots, dtype=torch.int32,
                                                                      device="cuda"), out=out)
    want, state = np.zeros((3, H, dv)), S.astype(np.float64)
    for b, p in enumerate(slots):
        if 0 <= p < pool:
            o, e = decay.attn(*(x[n][b:b + 1] for n in "qkv"), x["g"], 1.0, None, state[p:p + 1])
            want[b], state[p] = o[0, :, 0], e[0]
    assert np.allclose(_host(out), want, rtol=0, atol=1e-4)   # sums of 64 products of N(0, 1):
    assert np.allclose(_host(s), state, rtol=0, atol=1e-5)    # 64 * 2^-24 * 25, and 2^-22 * 25
    for b, p in enumerate(slots):
        if not 0 <= p < pool:
            assert not out[b].any()
    for p in set(range(pool)) - set(slots):
        assert np.array_equal(_host(s[p]), S[p].astype(np.float64))


def test_step_of_a_large_batch_with_repeats():
    import torch
    fv = _fv()
    B, H, d = 600, 2, 8
    x = _inputs(B, H, 1, d, d, "f32", 12)
    rng = np.random.default_rng(1)
    slots = rng.integers(0, 300, B).astype(np.int32)
    S = rng.standard_normal((300, H, d, d)).astype(np.float32)
    s = to_dev(S)
    q, k, v = (to_dev(x[n][:, :, 0]) for n in "qkv")
    out = fv.attn_decay_step(q, k, v, to_dev(x["g"]), s,
                             slots=torch.from_numpy(slots).cuda())
    state = S.astype(np.float64)
    want = np.zeros((B, H, d))
    for b, p in enumerate(slots):
        o, e = decay.attn(*(x[n][b:b + 1] for n in "qkv"), x["g"], 1.0, None, state[p:p + 1])
        want[b], state[p] = o[0, :, 0], e[0]
    assert np.allclose(_host(out), want, rtol=0, atol=1e-4)
    assert np.allclose(_host(s), state, rtol=0, atol=1e-5)
