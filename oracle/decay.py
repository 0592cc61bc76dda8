"""Linear attention with a decay per head and counter-based dropout, in fp64 on the CPU.

Test infrastructure only (see ``oracle/__init__``). The attention is the recurrence
itself, token by token: S_t = a S_{t-1} + k_t v_t^T, out_t = scale q_t^T S_t with
a = exp(log_decay[h]); its gradients are the recurrence in reverse. The dropout mask is
Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, SC'11) on Python-sized integers.
"""
import numpy as np


def _heads(q, log_decay, lengths):
    B, H, L = q.shape[:3]
    a = np.exp(np.asarray(log_decay, dtype=np.float64))[None, :, None, None]
    n = np.full(B, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)
    return B, H, L, a, n


def attn(q, k, v, log_decay, scale=1.0, lengths=None, state=None):
    """(out [B, H, L, dv], state after each sequence's last token [B, H, dk, dv])."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    B, H, L, a, n = _heads(q, log_decay, lengths)
    dk, dv = q.shape[-1], v.shape[-1]
    S = np.zeros((B, H, dk, dv)) if state is None else np.array(state, dtype=np.float64)
    out = np.zeros((B, H, L, dv))
    for t in range(L):
        live = t < n
        S[live] = a * S[live] + k[live, :, t, :, None] * v[live, :, t, None, :]
        out[live, :, t] = scale * np.einsum("bhk,bhkv->bhv", q[live, :, t], S[live])
    return out, S


def attn_backward(q, k, v, log_decay, dout, scale=1.0, lengths=None, state=None, dstate=None):
    """(dq, dk, dv, gradient of the incoming state)."""
    q, k, v, dout = (np.asarray(x, dtype=np.float64) for x in (q, k, v, dout))
    B, H, L, a, n = _heads(q, log_decay, lengths)
    S = (np.zeros((B, H, q.shape[-1], v.shape[-1])) if state is None
         else np.array(state, dtype=np.float64))
    G = np.zeros_like(S) if dstate is None else np.array(dstate, dtype=np.float64)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for t in range(L):
        live = t < n
        S[live] = a * S[live] + k[live, :, t, :, None] * v[live, :, t, None, :]
        dq[live, :, t] = scale * np.einsum("bhv,bhkv->bhk", dout[live, :, t], S[live])
    for t in reversed(range(L)):
        live = t < n
        G[live] += scale * q[live, :, t, :, None] * dout[live, :, t, None, :]
        dk[live, :, t] = np.einsum("bhkv,bhv->bhk", G[live], v[live, :, t])
        dv[live, :, t] = np.einsum("bhkv,bhk->bhv", G[live], k[live, :, t])
        G[live] = a * G[live]
    return dq, dk, dv, G


# ---------------------------------------------------------------- dropout
_M0, _M1, _W0, _W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
_LO = np.uint64(0xFFFFFFFF)
_S32 = np.uint64(32)


def philox4x32(counter, key):
    """Philox4x32-10: counter four arrays of 32-bit words, key two words -> four arrays."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k0, k1 = (int(x) for x in key)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(_M0), c[2] * np.uint64(_M1)
        c = [(p1 >> _S32) ^ c[1] ^ np.uint64(k0), p1 & _LO,
             (p0 >> _S32) ^ c[3] ^ np.uint64(k1), p0 & _LO]
        k0, k1 = (k0 + _W0) & 0xFFFFFFFF, (k1 + _W1) & 0xFFFFFFFF
    return c


def dropout_bits(seed, offset, first, n):
    """The 16 random bits of elements first .. first + n - 1."""
    e = np.arange(first, first + n, dtype=np.uint64)
    call, piece = e // np.uint64(8), (e % np.uint64(8)).astype(np.int64)
    zero = np.zeros_like(call)
    w = philox4x32((call & _LO, call >> _S32, zero + np.uint64(offset & 0xFFFFFFFF),
                    zero + np.uint64(offset >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    word = np.choose(piece // 2, w)
    return np.where(piece % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))


def threshold(p):
    return int(np.rint(p * 65536.0))


def dropout(x, p, seed, offset, residual=None):
    x = np.asarray(x, dtype=np.float64)
    t = threshold(p)
    kept = (dropout_bits(seed, offset, 0, x.size) >= t).reshape(x.shape)
    y = np.where(kept, x / (1.0 - t / 65536.0) if t < 65536 else 0.0, 0.0)
    return y if residual is None else y + np.asarray(residual, dtype=np.float64)
