"""Short causal convolution, selective state space scan and beam search's step, in fp64 on
the CPU.

Test infrastructure only (see ``oracle/__init__``). Convolution and scan are their defining
sums, token by token; their gradients the same in reverse. ``scan_bounds`` carries first-order
bounds of what fp32 arithmetic may be off by through the same recurrences, in units of 2^-24.
"""
import numpy as np


def _f64(*xs):
    return tuple(None if x is None else np.asarray(x, dtype=np.float64) for x in xs)


def _lengths(lengths, B, L):
    return np.full(B, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1 + e)


def softplus(x):
    return np.maximum(x, 0) + np.log1p(np.exp(-np.abs(x)))


# ---------------------------------------------------------------- convolution
def _padded(x, W, state):
    B, _, D = x.shape
    first = np.zeros((B, W - 1, D)) if state is None else state
    return np.concatenate([first, x], 1)


def conv(x, w, bias=None, silu=False, lengths=None, state=None):
    """(y [B, L, D], the last W - 1 inputs of each sequence [B, W - 1, D])."""
    x, w, bias, state = _f64(x, w, bias, state)
    (B, L, D), W = x.shape, w.shape[1]
    n = _lengths(lengths, B, L)
    xp = _padded(x, W, state)
    y = np.zeros((B, L, D))
    for b in range(B):
        for t in range(n[b]):
            y[b, t] = (xp[b, t:t + W] * w.T).sum(0) + (0 if bias is None else bias)
    if silu:
        y = y * sigmoid(y)
    return y, np.stack([xp[b, n[b]:n[b] + W - 1] for b in range(B)])


def conv_backward(x, w, dy, bias=None, silu=False, lengths=None, state=None, dstate=None):
    """(dx, dw, dbias, gradient of the incoming state)."""
    x, w, dy, bias, state, dstate = _f64(x, w, dy, bias, state, dstate)
    (B, L, D), W = x.shape, w.shape[1]
    n = _lengths(lengths, B, L)
    xp = _padded(x, W, state)
    dxp, dw, db = np.zeros_like(xp), np.zeros_like(w), np.zeros(D)
    for b in range(B):
        for t in range(n[b]):
            g = dy[b, t]
            if silu:
                u = (xp[b, t:t + W] * w.T).sum(0) + (0 if bias is None else bias)
                s = sigmoid(u)
                g = g * s * (1 + u * (1 - s))
            dxp[b, t:t + W] += g * w.T
            dw += (g * xp[b, t:t + W]).T
            db += g
        if dstate is not None:
            dxp[b, n[b]:n[b] + W - 1] += dstate[b]
    return dxp[:, W - 1:], dw, db, dxp[:, :W - 1]


# ---------------------------------------------------------------- selective scan
def _scan_terms(x, dt, bias, soft):
    raw = dt if bias is None else dt + bias
    return raw, softplus(raw) if soft else raw


def _spread(t, D):
    """[B, L, G, N] to [B, L, D, N]: each channel its group's."""
    return np.repeat(t, D // t.shape[2], axis=2)


def scan(x, dt, A, Bm, C, skip=None, z=None, bias=None, soft=True, lengths=None, state=None):
    """(y [B, L, D], the states after each sequence's last token [B, D, N])."""
    x, dt, A, Bm, C, skip, z, bias, state = _f64(x, dt, A, Bm, C, skip, z, bias, state)
    (B, L, D), N = x.shape, A.shape[1]
    n = _lengths(lengths, B, L)
    _, s = _scan_terms(x, dt, bias, soft)
    Bm, C = _spread(Bm, D), _spread(C, D)
    h = np.zeros((B, D, N)) if state is None else state.copy()
    y = np.zeros((B, L, D))
    for t in range(L):
        live = t < n
        h[live] = (np.exp(s[live, t, :, None] * A) * h[live]
                   + (s * x)[live, t, :, None] * Bm[live, t])
        y[live, t] = (C[live, t] * h[live]).sum(-1)
    if skip is not None:
        y = y + skip * x
    if z is not None:
        y = y * z * sigmoid(z)
    keep = np.arange(L)[:, None] < n[:, None, None]
    return np.where(keep, y, 0.0), h


def scan_backward(x, dt, A, Bm, C, dy, skip=None, z=None, bias=None, soft=True, lengths=None,
                  state=None, dstate=None):
    """(dx, ddt, dA, dB, dC, dskip, dz, dbias, gradient of the incoming state)."""
    x, dt, A, Bm, C, dy, skip, z, bias, state, dstate = _f64(
        x, dt, A, Bm, C, dy, skip, z, bias, state, dstate)
    (B, L, D), (G, N) = x.shape, Bm.shape[2:]
    n = _lengths(lengths, B, L)
    raw, s = _scan_terms(x, dt, bias, soft)
    Bs, Cs = _spread(Bm, D), _spread(C, D)
    keep = np.arange(L)[:, None] < n[:, None, None]
    silu = np.ones_like(x) if z is None else z * sigmoid(z)
    e = np.where(keep, dy * silu, 0.0)
    h = np.zeros((B, L + 1, D, N))
    if state is not None:
        h[:, 0] = state
    y = np.zeros((B, L, D))
    for t in range(L):
        live = t < n
        h[:, t + 1] = h[:, t]
        h[live, t + 1] = (np.exp(s[live, t, :, None] * A) * h[live, t]
                          + (s * x)[live, t, :, None] * Bs[live, t])
        y[:, t] = (Cs[:, t] * h[:, t + 1]).sum(-1)
    q = np.zeros((B, D, N)) if dstate is None else dstate.copy()
    dx, ds = np.zeros_like(x), np.zeros_like(x)
    dB, dC, dA = np.zeros_like(Bm), np.zeros_like(C), np.zeros_like(A)
    for t in reversed(range(L)):
        v = t < n
        g = Cs[v, t] * e[v, t, :, None] + q[v]
        dC[v, t] = (e[v, t, :, None] * h[v, t + 1]).reshape(-1, G, D // G, N).sum(2)
        dB[v, t] = (g * (s * x)[v, t, :, None]).reshape(-1, G, D // G, N).sum(2)
        q[v] = np.exp(s[v, t, :, None] * A) * g
        u = q[v] * h[v, t]
        dA += (u * s[v, t, :, None]).sum(0)
        into = (g * Bs[v, t]).sum(-1)
        ds[v, t] = (A * u).sum(-1) + x[v, t] * into
        dx[v, t] = s[v, t] * into
    if skip is not None:
        dx = dx + skip * e
        y = y + skip * x
    ddt = ds * sigmoid(raw) if soft else ds
    dz = None
    if z is not None:
        k = sigmoid(z)
        dz = np.where(keep, dy * y * k * (1 + z * (1 - k)), 0.0)
    x0 = np.where(keep, x, 0.0)
    return (np.where(keep, dx, 0.0), np.where(keep, ddt, 0.0), dA, dB, dC,
            None if skip is None else (e * x0).sum((0, 1)), dz,
            None if bias is None else np.where(keep, ddt, 0.0).sum((0, 1)), q)


def scan_bounds(x, dt, A, Bm, C, dy, skip=None, z=None, bias=None, soft=True, lengths=None,
                state=None, dstate=None):
    """First-order error bounds, in units of 2^-24, of (y, final state, and scan_backward's
    outputs) before their last rounding.

    H and Q are the recurrences on magnitudes, EH and EQ the errors they carry. Per token and
    state: exp(s A) has 3 |s A| + 6 of relative error (the product with A, the one with log2 e
    in it, the exponential; a lane's own step, its part in the powers of the joined lanes and
    their products), the input 4; sums of k terms add k. s = softplus(raw) is 6 off relatively,
    and by softplus' raw for raw's rounding.
    """
    x, dt, A, Bm, C, dy, skip, z, bias, state, dstate = _f64(
        x, dt, A, Bm, C, dy, skip, z, bias, state, dstate)
    (B, L, D), (G, N) = x.shape, Bm.shape[2:]
    n = _lengths(lengths, B, L)
    keep = np.arange(L)[:, None] < n[:, None, None]
    raw, s = _scan_terms(x, dt, bias, soft)
    s = np.where(keep, s, 0.0)
    sig = sigmoid(raw) if soft else np.ones_like(raw)
    raw_mag = np.abs(dt) + (0 if bias is None else np.abs(bias))
    Es = np.where(keep, (6 * s + sig * raw_mag) if soft else raw_mag, 0.0)
    s = np.abs(s)
    x, Bs, Cs, mA = np.abs(x), np.abs(_spread(Bm, D)), np.abs(_spread(C, D)), np.abs(A)
    sk = 0.0 if skip is None else np.abs(skip)
    if z is None:
        gate, Egate = np.ones_like(x), 0.0
    else:
        gate = np.abs(z * sigmoid(z))
        Egate = (2 * np.abs(z) + 6) * gate
    e = np.where(keep, np.abs(dy) * gate, 0.0)
    Ee = np.where(keep, np.abs(dy) * Egate + 2 * e, 0.0)
    tok = lambda v, t: v[:, t, :, None]
    H, EH = np.zeros((B, L + 1, D, N)), np.zeros((B, L + 1, D, N))
    if state is not None:
        H[:, 0] = np.abs(state)
    a, Ea = [], []
    Y, EY = np.zeros_like(x), np.zeros_like(x)
    for t in range(L):
        at = np.exp(np.where(keep[:, t, :, None], tok(np.where(keep, raw if not soft else s, 0.0), t) * A, 0.0))
        a.append(at)
        Ea.append(at * (3 * tok(s, t) * mA + 6 + mA * tok(Es, t)))
        b = tok(s * x, t) * Bs[:, t]
        Eb = 4 * b + tok(Es * x, t) * Bs[:, t]
        H[:, t + 1] = at * H[:, t] + b
        EH[:, t + 1] = at * EH[:, t] + Ea[t] * H[:, t] + Eb + H[:, t + 1]
        Y[:, t] = (Cs[:, t] * H[:, t + 1]).sum(-1)
        EY[:, t] = (Cs[:, t] * EH[:, t + 1]).sum(-1) + (N + 4) * Y[:, t]
    Y, EY = Y + sk * x, EY + 3 * sk * x
    Ey = EY * gate + Y * Egate + 2 * Y * gate
    Q = np.zeros((B, D, N)) if dstate is None else np.abs(dstate)
    EQ = np.zeros((B, D, N))
    add = 32 + D // G // 64
    rows = 64 + L // 8 + B * L // 128
    Edx, Eds, Mds = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    EdB, EdC, EdA = np.zeros_like(Bm), np.zeros_like(Bm), np.zeros_like(A)
    for t in reversed(range(L)):
        live = keep[:, t, :, None]
        ce = Cs[:, t] * tok(e, t)
        g = np.where(live, ce + Q, 0.0)
        Eg = np.where(live, EQ + Cs[:, t] * tok(Ee, t) + 2 * ce + g, 0.0)
        grp = lambda v: v.reshape(B, G, D // G, N).sum(2)
        EdC[:, t] = grp(tok(Ee, t) * H[:, t + 1] + tok(e, t) * (EH[:, t + 1] + add * H[:, t + 1]))
        sx, Esx = tok(s * x, t), tok(Es * x + 2 * s * x, t)
        EdB[:, t] = grp(Eg * sx + g * Esx + add * g * sx)
        Q = np.where(live, a[t] * g, Q)
        EQ = np.where(live, a[t] * Eg + Ea[t] * g + Q, EQ)
        u, Eu = Q * H[:, t], EQ * H[:, t] + Q * EH[:, t] + Q * H[:, t]
        u, Eu = np.where(live, u, 0.0), np.where(live, Eu, 0.0)
        EdA += (tok(s, t) * Eu + tok(Es, t) * u + rows * tok(s, t) * u).sum(0)
        into = (g * Bs[:, t]).sum(-1)
        Einto = (Eg * Bs[:, t]).sum(-1) + (N + 4) * into
        Edx[:, t] = Es[:, t] * into + s[:, t] * Einto + 4 * s[:, t] * into
        Mds[:, t] = (mA * u).sum(-1) + x[:, t] * into
        Eds[:, t] = (mA * Eu).sum(-1) + (N + 4) * (mA * u).sum(-1) + x[:, t] * (Einto + 2 * into)
    Edx = np.where(keep, Edx + sk * (Ee + 3 * e), 0.0)
    soft_units = (2 * raw_mag + 8) if soft else 1.0
    Eddt = np.where(keep, sig * (Eds + soft_units * Mds), 0.0)
    Mddt = np.where(keep, sig * Mds, 0.0)
    dz = None
    if z is not None:
        dz = np.abs(dy) * (1.1 * EY + Y * (4 * np.abs(z) + 12))
        dz = np.where(keep, dz, 0.0)
    x0 = np.where(keep, x, 0.0)
    return (np.where(keep, Ey, 0.0), EH[:, L], Edx, Eddt, EdA, EdB, EdC,
            None if skip is None else ((Ee + rows * e) * x0).sum((0, 1)), dz,
            None if bias is None else (Eddt + rows * Mddt).sum((0, 1)), EQ)


# ---------------------------------------------------------------- beams
def beam_select(logits, scores, n, ended=None, end_token=-1):
    """(scores [B, n], parent [B, n], token [B, n])."""
    x, scores = _f64(logits, scores)
    B, K, V = x.shape
    out = np.full((B, n), -np.inf)
    parent, token = np.zeros((B, n), np.int32), np.full((B, n), max(end_token, 0), np.int32)
    for b in range(B):
        found = []
        for k in range(K):
            if ended is not None and ended[b][k]:
                found.append((scores[b, k], k, 0.0, end_token))
                continue
            row = x[b, k]
            top = np.nanmax(row) if not np.isnan(row).all() else np.nan
            with np.errstate(all="ignore"):
                p = row - top - np.log(np.exp(row - top).sum()) + scores[b, k]
            found += [(p[v], k, row[v], v) for v in np.argsort(-row, kind="stable")[:n]]
        with np.errstate(over="ignore"):   # finite as they are returned, in fp32
            found = [f for f in found if np.isfinite(np.float32(f[0]))]
        found.sort(key=lambda f: (-f[0], f[1], -f[2], f[3]))
        for i, f in enumerate(found[:n]):
            out[b, i], parent[b, i], token[b, i] = f[0], f[1], f[3]
    return out, parent, token


def beam_reorder(parent, slots, pools):
    """(new slots, pools): a first child keeps its parent's place, the others, in order, take
    those of childless beams; a beam with no valid parent takes one with what it holds."""
    new, pools = np.array(slots), [np.array(p) for p in pools]
    K = new.shape[1]
    for p, s, o in zip(np.asarray(parent), np.asarray(slots), new):
        free = [s[k] for k in range(K) if k not in p]
        for j, k in enumerate(p):
            valid = 0 <= k < K
            o[j] = s[k] if valid and k not in p[:j] else free.pop(0)
            for pool in pools:
                if valid and o[j] != s[k] and 0 <= o[j] < len(pool) and 0 <= s[k] < len(pool):
                    pool[o[j]] = pool[s[k]]
    return new, pools
