"""bf16 calls of the decayed linear attention: a row's result is off by its own rounding, whatever
batch it is in, how long its sequence is and whether a state is returned.

Bound, per element, with A the same formula on absolute values: the output's rounding
2^-8 |o|; what two bf16 terms leave, 2^-16 each: of the pair weights (their part of A), or of the
state and of the weighted values in it (its part of A), so 2 x 2^-16 A; and the fp32 sums,
(width + 64 + 4 chunks + 16) 2^-24 A.

The operands that make the pair weights (Q and K for the output and dV, V and dout for dQ and
dK) are not negative and the values have either sign. So A is not much above the sum's
own terms, many sums come out small, and a single bf16 term anywhere, off by 2^-8, shows: the
emulation says so for each of the three places."""
import functools

import numpy as np
import pytest

from oracle import decay
from workloads import bf16_round

DECAYS = [-1 / 32, -1e-3, -0.2, 0.0]


def _inputs(B, H, L, dk, dv, positive, seed):
    rng = np.random.default_rng(seed)
    draw = {True: lambda *s: rng.uniform(0, 1, s), False: lambda *s: rng.standard_normal(s)}
    x = {}
    for n, d in (("q", dk), ("k", dk), ("v", dv), ("do", dv)):
        some = positive == ("weights of out and dV" if n in "qk" else "weights of dQ and dK")
        x[n] = bf16_round(draw[some](B, H, L, d).astype(np.float32))
    x["S"], x["G"] = (rng.standard_normal((B, H, dk, dv)).astype(np.float32) for _ in range(2))
    x["g"] = np.array([DECAYS[(seed + h) % len(DECAYS)] for h in range(H)], dtype=np.float32)
    return x


def _off(got, ref, mag, width, L):
    """The largest error in units of the bound."""
    tol = (2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + 2 * 2.0 ** -16 * (1 + 2.0 ** -6) * mag
           + (width + 64 + 4 * (L // 64 + 1) + 16) * 2.0 ** -24 * mag)
    err = np.abs(got - ref)
    return float((err / np.where(tol > 0, tol, 1.0))[(tol > 0) | (err > 0)].max(initial=0.0))


# ------------------------------------------------------------------ the bound itself
def _terms(x, n):
    """x as the sum of n bf16 terms."""
    x = np.asarray(x, dtype=np.float32)
    total = np.zeros_like(x)
    for _ in range(n):
        total = total + bf16_round(x - total)
    return total.astype(np.float64)


def _emulated(q, k, v, g, terms):
    """The chunked form with its operands rounded to `terms` = (pair weights, state, weighted
    values) bf16 terms."""
    B, H, L = q.shape[:3]
    out = np.zeros(q.shape[:3] + v.shape[3:])
    i = np.arange(64)
    for h in range(H):
        a = np.exp(np.float64(g[h]))
        X = np.zeros((B, q.shape[3], v.shape[3]))
        for c in range(0, L, 64):
            n = min(64, L - c)
            qc, kc, vc = (t[:, h, c:c + n].astype(np.float64) for t in (q, k, v))
            lag = i[:n, None] - i[:n]
            P = qc @ kc.swapaxes(1, 2) * np.where(lag >= 0, a ** np.maximum(lag, 0), 0.0)
            o = a ** (i[:n, None] + 1) * (qc @ _terms(X, terms[1])) + _terms(P, terms[0]) @ vc
            out[:, h, c:c + n] = bf16_round(o.astype(np.float32))
            w = _terms(a ** (n - 1 - i[:n, None]) * vc, terms[2])
            X = a ** n * X + kc.swapaxes(1, 2) @ w
    return out


@pytest.mark.parametrize("B,H,L,dk,dv", [(4, 2, 300, 64, 64), (3, 3, 130, 16, 64)])
def test_the_bound_tells_one_term_from_two(B, H, L, dk, dv):
    """(A state's own roundings average out over dk, and weighted values are exact without a
    decay: few columns and heads that forget.)"""
    x = _inputs(B, H, L, dk, dv, "weights of out and dV", 3)
    x["g"] = np.array(DECAYS[:H], dtype=np.float32)
    ref, _ = decay.attn(x["q"], x["k"], x["v"], x["g"])
    mag, _ = decay.attn(x["q"], x["k"], np.abs(x["v"]), x["g"])
    off = {t: _off(_emulated(x["q"], x["k"], x["v"], x["g"], t), ref, mag, dk, L)
           for t in ((2, 2, 2), (1, 2, 2), (2, 1, 2), (2, 2, 1))}
    assert off[2, 2, 2] <= 1, off
    assert all(r > 1.5 for t, r in off.items() if t != (2, 2, 2)), off


# ------------------------------------------------------------------ on the GPU
CALLS = [  # B, H, L, dk, dv, lengths
    (16, 8, 8, 64, 64, None), (41, 5, 5, 64, 64, None),          # 1024 and 1025 rows
    (43, 8, 3, 128, 128, None), (300, 4, 1, 128, 128, None),     # tokens of many sequences
    (40, 8, 4, 256, 64, None), (20, 4, 64, 128, 96, None),
    (2, 2, 64, 64, 64, None), (2, 2, 65, 64, 64, None),
    (3, 2, 1500, 128, 64, (1, 5, 3)), (3, 2, 700, 64, 128, (2, 700, 64)),
    (1, 2, 333, 256, 256, None), (2, 1, 1025, 200, 136, None), (1, 2, 1999, 64, 64, None),
    (1, 1, 1300, 128, 248, None), (4, 21, 300, 128, 128, None), (6, 22, 200, 64, 128, None),
]


def _exact(x, state, lengths, c=0.5):
    """[out, dQ, dK, dV] as products over all pairs of tokens."""
    B, H, L = x["q"].shape[:3]
    n = np.full(B, L) if lengths is None else np.array(lengths)
    i = np.arange(L)
    live = (i < n[:, None])[:, None, :, None]
    q, k, v, do = (np.where(live, x[m].astype(np.float64), 0.0) for m in ("q", "k", "v", "do"))
    g = x["g"].astype(np.float64)
    lag = i[:, None] - i
    D = np.where(lag >= 0, np.exp(g[:, None, None] * np.maximum(lag, 0)), 0.0)
    t = lambda m: m.swapaxes(-1, -2)
    P, E = (a @ t(b) * D for a, b in ((q, k), (do, v)))
    got = [c * (P @ v), c * (E @ k), c * (t(E) @ q), c * (t(P) @ do)]
    if state:
        S, G = (x[m].astype(np.float64) for m in "SG")
        fade = np.exp(g[:, None] * (i + 1))[..., None]
        late = np.exp(g[:, None] * np.maximum(n[:, None] - 1 - i, 0)[:, None])[..., None]
        for y, add in zip(got, (c * fade * (q @ S), c * fade * (do @ t(S)), late * (v @ t(G)),
                                late * (k @ G))):
            y += np.where(live, add, 0.0)
    return got


@functools.lru_cache(maxsize=2)
def _case(call, positive, state):
    B, H, L, dk, dv, lengths = call
    x = _inputs(B, H, L, dk, dv, positive, B + H + L + dk + dv)
    y = {n: np.abs(t) if n != "g" else t for n, t in x.items()}
    return x, _exact(x, state, lengths), _exact(y, state, lengths)


def test_the_pairs_are_the_recurrence():
    x, ref, _ = _case((2, 3, 70, 8, 16, (70, 9)), "weights of out and dV", True)
    args = [x[n] for n in ("q", "k", "v", "g")]
    want = [decay.attn(*args, 0.5, (70, 9), x["S"])[0],
            *decay.attn_backward(*args, x["do"], 0.5, (70, 9), x["S"], x["G"])[:3]]
    for a, b in zip(ref, want):
        assert np.allclose(a, b, rtol=1e-11, atol=1e-11)


@pytest.mark.gpu
@pytest.mark.parametrize("state", ["none", "in", "in and out"])
@pytest.mark.parametrize("positive", ["weights of out and dV", "weights of dQ and dK"])
@pytest.mark.parametrize("call", CALLS)
def test_rows_are_off_by_their_own_rounding(call, positive, state):
    import torch
    import paper_2006_03555_amd as fv
    from helpers import to_dev
    L, dk, dv, lengths = call[2:]
    back, some = state == "in and out", state != "none"
    x, ref, mag = _case(call, positive, some)
    q, k, v, do = (to_dev(x[n], "bf16") for n in ("q", "k", "v", "do"))
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    kw = dict(lengths=ln, state_in=S) if some else dict(lengths=ln)
    out = fv.attn_decay(q, k, v, g, 0.5, return_state=back, **kw)
    back = fv.attn_decay_backward(q, k, v, g, do, 0.5, dstate_out=G if some else None,
                                  return_state_grad=back, **kw)
    got = (out[0] if isinstance(out, tuple) else out, *back[:3])
    off = {n: _off(t.double().cpu().numpy(), r, m, max(dk, dv), L)
           for n, t, r, m in zip(("out", "dQ", "dK", "dV"), got, ref, mag)}
    assert max(off.values()) <= 1, off
