"""The calls the decayed linear attention and the dropout are measured on.

Each case is a dict of plain values. Linear attention with a decay per head:
  kind      step    one token for each of B sequences, the carried states updated in place
            prompt  a stretch of L tokens, forward
            train   forward and backward over L tokens
  B, H, L   batch, heads and tokens
  dk, dv    width of a query or key, and of a value
  dtype     bf16 or f32: Q, K, V, the outputs and the gradients (states are always f32)
  layout    bhld: contiguous [B, H, L, d]; blhd: [B, L, H, d] in memory; packed: slices of
            one [B, L, 3, H, d] projection
  ragged    1: a right-padded batch, every sequence of its own length
  state     1: states carried in and out
  slots     step: 0: state b belongs to sequence b; n: sequences hold places in a pool of n
  feats     1: Q and K are ReLU random features (non-negative), 0: N(0, 1) / sqrt(dk)
Dropout from a counter-based generator (kind dropout):
  n         elements
  p         the share dropped
  residual  1: added to a residual
  grad      1: the gradient's pass too (the same mask again)
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_ATTN = dict(B=1, H=8, L=1, dk=64, dv=64, dtype="bf16", layout="bhld", ragged=0, state=0,
             slots=0, feats=0)


def _attn(name, kind, **kw):
    return dict(_ATTN, name=name, kind=kind, **kw)


def _drop(name, **kw):
    return dict(dict(kind="dropout", n=1, p=0.1, dtype="bf16", residual=0, grad=0), name=name,
                **kw)


def listed():
    return [
        # the next token of one sequence: only latency counts
        _attn("step_one", "step", H=8),
        # a decoding step of a full serving batch whose states live in a pool
        _attn("step_pool", "step", B=48, H=16, dk=128, dv=128, slots=64),
        # the next piece of a sequence that arrives in pieces
        _attn("prompt_piece", "prompt", L=128, state=1),
        # a padded batch of prompts of odd lengths, cut from one projection
        _attn("prompt_ragged", "prompt", B=6, H=16, L=1999, dk=128, dv=128, layout="packed",
              ragged=1, state=1),
        # one long document
        _attn("prompt_long", "prompt", H=16, L=65536, dk=128, dv=128, layout="blhd"),
        # a protein-length layer on materialised ReLU random features
        _attn("prompt_features", "prompt", B=4, H=8, L=8192, dk=256, feats=1),
        # a float32 prompt of odd length and a wide value
        _attn("prompt_f32", "prompt", B=2, L=1000, dv=128, dtype="f32", layout="blhd"),
        # a small float32 training step that carries a state through a piece
        _attn("train_f32", "train", B=2, L=777, dtype="f32", state=1),
        # a training step of a model's layer
        _attn("train_bf16", "train", B=4, H=16, L=4096, dk=128, dv=128, layout="blhd"),
        # the output of a piece of 128 tokens and 8 heads of 64
        _drop("dropout_piece", n=128 * 512),
        # a training step's residual stream: 16384 tokens of width 2048, and its gradient
        _drop("dropout_stream", n=16384 * 2048, residual=1, grad=1),
        # an odd number of float32 activations
        _drop("dropout_f32", n=4099 * 1023, dtype="f32", p=0.25, residual=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "prompt", "prompt", "train", "train", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "dropout":
        return dict(kind=kind, n=_log(rng, 1000, 1 << 25), p=round(rng.uniform(0.02, 0.5), 3),
                    dtype=dtype, residual=rng.randrange(2), grad=rng.randrange(2))
    dk, dv = (8 * rng.randint(2, 32) if rng.random() < 0.4 else rng.choice([64, 128, 256])
              for _ in range(2))
    H = rng.randint(1, 24)
    case = dict(_ATTN, kind=kind, H=H, dk=dk, dv=dv, dtype=dtype)
    if kind == "step":
        B = _log(rng, 1, 64)
        return dict(case, B=B, slots=rng.choice([0, B + rng.randint(0, 16)]))
    B = rng.randint(1, 6)
    most = (1 << (20 if kind == "prompt" else 18)) // (B * H) * 64 // max(dk, dv)
    layout = rng.choice(["bhld", "blhd", "packed"] if dk == dv else ["bhld", "blhd"])
    return dict(case, B=B, L=_log(rng, 1, max(2, min(40000, most))), layout=layout,
                ragged=rng.randrange(2) if kind == "prompt" else 0, state=rng.randrange(2),
                feats=rng.randrange(2))


# ------------------------------------------------------------------ inputs
def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _laid_out(case, gen, widths):
    """Tensors [B, H, L, width] in the case's memory layout."""
    B, H, L, dt = case["B"], case["H"], case["L"], _DTYPES[case["dtype"]]
    if case["layout"] == "packed":
        x = _rand(gen, B, L, len(widths), H, widths[0]).to(dt)
        ts = [x[:, :, i].transpose(1, 2) for i in range(len(widths))]
    elif case["layout"] == "blhd":
        ts = [_rand(gen, B, L, H, w).to(dt).transpose(1, 2) for w in widths]
    else:
        ts = [_rand(gen, B, H, L, w).to(dt) for w in widths]
    return ts


def _log_decay(H):
    """log(1 - 2^-e) with e spread over 5 .. 9: memories of 32 to 512 tokens."""
    rate = [2.0 ** -(5 + 4 * h / max(1, H - 1)) for h in range(H)]
    return torch.tensor([math.log1p(-r) for r in rate], dtype=torch.float32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["kind"] == "dropout":
        n, dt = case["n"], _DTYPES[case["dtype"]]
        return dict(case=case, seed=int(seed) * 0x9E3779B97F4A7C15 % (1 << 64), offset=int(seed) % 1000,
                    x=_rand(gen, n).to(dt), residual=_rand(gen, n).to(dt) if case["residual"] else None,
                    dout=_rand(gen, n).to(dt) if case["grad"] else None)
    B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
    st = dict(case=case, g=_log_decay(H), scale=1.0 if case["feats"] else dk ** -0.5,
              lengths=None, state=None, slots=None, dout=None, dstate=None)
    q, k, v = _laid_out(case, gen, (dk, dk, dv))
    if case["feats"]:
        q, k = (x.clamp_(min=0).mul_(dk ** -0.5).add_(1e-3) for x in (q, k))
    if case["kind"] == "step":
        st["q"], st["k"], st["v"] = q[:, :, 0], k[:, :, 0], v[:, :, 0]
        n = case["slots"] or B
        st["state"] = _rand(gen, n, H, dk, dv)
        if case["slots"]:
            st["slots"] = torch.randperm(n, generator=gen, device="cuda")[:B].to(torch.int32)
        return st
    st["q"], st["k"], st["v"] = q, k, v
    if case["ragged"]:
        st["lengths"] = torch.randint(min(L, 1 + L // 8), L + 1, (B,), generator=gen,
                                      device="cuda", dtype=torch.int32)
    if case["state"]:
        st["state"] = _rand(gen, B, H, dk, dv)
    if case["kind"] == "train":
        layout = "blhd" if case["layout"] == "packed" else case["layout"]
        st["dout"], = _laid_out(dict(case, layout=layout), gen, (dv,))
        if case["state"]:
            st["dstate"] = _rand(gen, B, H, dk, dv)
    return st


# ------------------------------------------------------------------ plain forms
def _powers(g, e):
    """decay^e [H, ...] in 64 bits for whole e >= 0 (decay^0 = 1)."""
    g = g.double().reshape((-1,) + (1,) * e.dim())
    return torch.where(e == 0, 1.0, torch.exp(g * e)).float()


def _rows(w):
    """[H, L] weights of rows, as [H, L, 1]."""
    return w.unsqueeze(-1)


def _scan(q, k, v, g, state):
    """out_i = sum_{j <= i} decay^(i - j) (q_i . k_j) v_j + decay^(i + 1) q_i state over
    [B, H, L, .] in float32, in chunks: products inside a chunk, and the states before
    every chunk from the chunks' own sums."""
    B, H, L, dk = q.shape
    dv = v.shape[-1]
    T = min(128 if L <= 8192 else 256, L)
    n = -(-L // T)

    def cut(x):
        x = torch.nn.functional.pad(x, (0, 0, 0, n * T - L))
        return x.reshape(B, H, n, T, x.shape[-1])

    q, k, v = cut(q), cut(k), cut(v)
    t = torch.arange(T, device=q.device)
    c = torch.arange(n, device=q.device)
    lag = t[:, None] - t
    D = _powers(g, lag.clamp(min=0)) * (lag >= 0)
    out = ((q @ k.transpose(-1, -2)) * D[:, None]) @ v
    kw = k * _rows(_powers(g, T - 1 - t))[:, None]
    sums = (kw.transpose(-1, -2) @ v).reshape(B, H, n, dk * dv)
    back = c[:, None] - 1 - c
    P = _powers(g, T * back.clamp(min=0)) * (back >= 0)
    before = P @ sums
    if state is not None:
        before = before + _rows(_powers(g, T * c)) * state.reshape(B, H, 1, dk * dv)
    qw = q * _rows(_powers(g, t + 1))[:, None]
    out = out + qw @ before.reshape(B, H, n, dk, dv)
    return out.reshape(B, H, n * T, dv)[:, :, :L]


def _final(k, v, g, lengths, state):
    """decay^len state + sum_j decay^(len - 1 - j) k_j v_j^T."""
    L = k.shape[2]
    lag = lengths[:, None] - 1 - torch.arange(L, device=k.device)
    w = _powers(g, lag.clamp(min=0)).transpose(0, 1) * (lag >= 0)[:, None]
    s = (k * w.unsqueeze(-1)).transpose(-1, -2) @ v
    if state is not None:
        s = s + _powers(g, lengths).transpose(0, 1)[..., None, None] * state
    return s


def _step(st):
    q, k, v = (st[n].float() for n in "qkv")
    idx = slice(None) if st["slots"] is None else st["slots"].long()
    s = st["state"][idx] * torch.exp(st["g"].double()).float()[:, None, None]
    s = s + k.unsqueeze(-1) * v.unsqueeze(-2)
    st["state"][idx] = s
    out = (q.unsqueeze(-2) @ s).squeeze(-2) * st["scale"]
    return out.to(st["q"].dtype), st["state"]


def _forward(st):
    q, k, v = (st[n].float() for n in "qkv")
    L, lengths = q.shape[2], st["lengths"]
    if lengths is None:
        lengths = torch.full((q.shape[0],), L, device=q.device)
    valid = (torch.arange(L, device=q.device) < lengths[:, None])[:, None, :, None]
    q, k, v = (torch.where(valid, x, 0.0) for x in (q, k, v))
    out = (_scan(q, k, v, st["g"], st["state"]) * st["scale"]).to(st["q"].dtype)
    if st["case"]["state"]:
        return out, _final(k, v, st["g"], lengths, st["state"])
    return (out,)


def _backward(st):
    """Gradients by the same scan: dQ with (dout, V, K) in its order, dK and dV with the
    tokens reversed; the incoming state's gradient decays from the last token back."""
    q, k, v, do = (st[n].float() for n in ("q", "k", "v", "dout"))
    g, s, ds, scale, dt = st["g"], st["state"], st["dstate"], st["scale"], st["q"].dtype
    dq = _scan(do, v, k, g, None if s is None else s.transpose(-1, -2)) * scale
    qr, kr, vr, dor = (x.flip(2) for x in (q, k, v, do))
    dv = _scan(kr, qr, dor, g, None).flip(2) * scale
    dk = _scan(vr, dor, qr, g, None).flip(2) * scale
    if ds is None:
        return dq.to(dt), dk.to(dt), dv.to(dt)
    L = q.shape[2]
    w = _rows(_powers(g, L - 1 - torch.arange(L, device=q.device)))
    dv = dv + (k * w) @ ds
    dk = dk + (v * w) @ ds.transpose(-1, -2)
    first = q * _rows(_powers(g, torch.arange(1, L + 1, device=q.device)))
    total = _powers(g, torch.tensor([L], device=q.device))[..., None]
    ds_in = first.transpose(-1, -2) @ do * scale + total * ds
    return dq.to(dt), dk.to(dt), dv.to(dt), ds_in


_M0, _M1, _W0, _W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
_LOW = 0xFFFFFFFF


def _philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 (Salmon et al., SC'11): 32-bit words held in int64."""
    for r in range(10):
        p0, p1 = c0 * _M0, c2 * _M1   # modulo 2^64: the low and high words are right
        c0, c1, c2, c3 = (((p1 >> 32) & _LOW) ^ c1 ^ ((k0 + r * _W0) & _LOW), p1 & _LOW,
                          ((p0 >> 32) & _LOW) ^ c3 ^ ((k1 + r * _W1) & _LOW), p0 & _LOW)
    return c0, c1, c2, c3


def _kept(st):
    """Whether each element stays: its 16 random bits are not below the threshold."""
    n, seed, offset = st["case"]["n"], st["seed"], st["offset"]
    i = torch.arange(-(-n // 8), device=st["x"].device)
    zero = torch.zeros_like(i)
    w = torch.stack(_philox(i & _LOW, i >> 32, zero + (offset & _LOW), zero + (offset >> 32),
                            seed & _LOW, seed >> 32), -1)
    bits = torch.stack((w & 0xFFFF, w >> 16), -1).reshape(-1)[:n]
    return bits >= round(st["case"]["p"] * 65536)


def _dropped(st, x, residual):
    t = round(st["case"]["p"] * 65536)
    y = torch.where(_kept(st), x.float() * (65536.0 / (65536 - t)), 0.0)
    return (y if residual is None else y + residual.float()).to(x.dtype)


def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own(st, kind)
    if kind == "dropout":
        y = _dropped(st, st["x"], st["residual"])
        return (y, _dropped(st, st["dout"], None)) if st["case"]["grad"] else (y,)
    if kind == "step":
        return _step(st)
    return _forward(st) + (_backward(st) if kind == "train" else ())


def _own(st, kind):
    import paper_2006_03555_amd as fv
    if kind == "dropout":
        p, seed, offset = st["case"]["p"], st["seed"], st["offset"]
        y = fv.dropout(st["x"], p, seed, offset, residual=st["residual"])
        if st["case"]["grad"]:
            return y, fv.dropout_backward(st["dout"], p, seed, offset)
        return (y,)
    q, k, v, g, scale = st["q"], st["k"], st["v"], st["g"], st["scale"]
    if kind == "step":
        return fv.attn_decay_step(q, k, v, g, st["state"], scale, slots=st["slots"]), st["state"]
    carried = bool(st["case"]["state"])
    got = fv.attn_decay(q, k, v, g, scale, lengths=st["lengths"], state_in=st["state"],
                        return_state=carried)
    got = got if carried else (got,)
    if kind == "train":
        got += fv.attn_decay_backward(q, k, v, g, st["dout"], scale, state_in=st["state"],
                                      dstate_out=st["dstate"], return_state_grad=carried)
    return got


# ------------------------------------------------------------------ work
def work(case):
    elt = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "dropout":
        n = case["n"]
        # x and y; the residual; the gradient in and out; ten rounds of eight operations
        # (two products of two words, four exclusive ors) for eight elements
        return {"bytes": n * elt * (2 + case["residual"] + 2 * case["grad"]),
                "flops": n * (1 + case["grad"]) * 12}
    B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
    rows, state = B * H * L, B * H * dk * dv
    by, fl = rows * elt * 2 * (dk + dv), 4 * rows * dk * dv
    if case["kind"] == "step" or case["state"]:
        by += 2 * 4 * state
    if case["kind"] == "train":
        # Q, K, V, dout again (the forward pass has long left the caches), three gradients
        by += rows * elt * (4 * dk + 3 * dv) + (3 * 4 * state if case["state"] else 0)
        fl += 10 * rows * dk * dv
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------ 64-bit results
def _bits16(seed, offset, n):
    """The elements' 16 random bits, in numpy."""
    calls = -(-n // 8)
    i = np.arange(calls, dtype=np.uint64)
    low, half = np.uint64(_LOW), np.uint64(32)
    c = [i & low, i >> half, np.full(calls, offset & _LOW, np.uint64),
         np.full(calls, offset >> 32, np.uint64)]
    key = [seed & _LOW, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(_M0), c[2] * np.uint64(_M1)
        c = [(b >> half) ^ c[1] ^ np.uint64(key[0]), b & low,
             (a >> half) ^ c[3] ^ np.uint64(key[1]), a & low]
        key = [(key[0] + _W0) & _LOW, (key[1] + _W1) & _LOW]
    words = np.stack(c, -1).astype("<u4")
    return words.view("<u2").reshape(-1)[:n]


def _pairs(case, st):
    """Row blocks (i, weights [H, rows, tokens]) of decay^(i - j), j <= i."""
    H, L = case["H"], case["L"]
    step = max(1, min(L, (1 << 27) // (case["B"] * H * L)))
    g = st["g"].double()[:, None, None]
    for i in range(0, L, step):
        r = torch.arange(i, min(L, i + step), device="cuda")
        lag = r[:, None] - torch.arange(int(r[-1]) + 1, device="cuda")
        w = torch.exp(g * lag.clamp(min=0))
        yield r, torch.where(lag >= 0, w, 0.0)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "dropout":
        kept = torch.from_numpy(_bits16(st["seed"], st["offset"], case["n"])
                                .astype(np.int32)).cuda() >= round(case["p"] * 65536)
        keep = 1.0 - round(case["p"] * 65536) / 65536
        y = torch.where(kept, st["x"].double() / keep, 0.0)
        if case["residual"]:
            y = y + st["residual"].double()
        return (y, torch.where(kept, st["dout"].double() / keep, 0.0)) if case["grad"] else (y,)
    B, H, L, dk, dv = (case[k] for k in ("B", "H", "L", "dk", "dv"))
    q, k, v = (st[n].double() for n in "qkv")
    g, scale = st["g"].double(), st["scale"]
    if case["kind"] == "step":
        pool = st["state"].double()
        at = torch.arange(B, device="cuda") if st["slots"] is None else st["slots"].long()
        s = pool[at] * g.exp()[:, None, None] + torch.einsum("bhk,bhv->bhkv", k, v)
        return (q[..., None] * s).sum(-2) * scale, pool.index_copy(0, at, s)
    q, k, v = (x.contiguous() for x in (q, k, v))
    state = st["state"].double() if case["state"] else None
    ages = torch.arange(1, L + 1, device="cuda")
    fade = torch.exp(g[:, None] * ages)   # of the carried state at each row
    n = st["lengths"].long() if case["ragged"] else torch.full((B,), L, device="cuda")
    train = case["kind"] == "train"
    do = st["dout"].double().contiguous() if train else None
    out = torch.zeros(B, H, L, dv, device="cuda", dtype=torch.float64)
    dq, dkey, dval = (torch.zeros_like(x) for x in (q, k, v)) if train else (None,) * 3
    for r, w in _pairs(case, st):
        lo, hi = int(r[0]), int(r[-1]) + 1
        kt, vt = (x[:, :, :hi].transpose(-1, -2).contiguous() for x in (k, v))
        a = q[:, :, lo:hi] @ kt * w
        out[:, :, lo:hi] = a @ v[:, :, :hi] * scale
        if train:
            e = do[:, :, lo:hi] @ vt * w
            dq[:, :, lo:hi] = e @ k[:, :, :hi] * scale
            dkey[:, :, :hi] += e.transpose(-1, -2).contiguous() @ q[:, :, lo:hi] * scale
            dval[:, :, :hi] += a.transpose(-1, -2).contiguous() @ do[:, :, lo:hi] * scale
    if state is not None:
        out += (q * fade[..., None]) @ state * scale
    out *= (ages <= n[:, None])[:, None, :, None]
    got = (out,)
    if state is not None:
        lag = n[:, None] - ages   # of token j at the sequence's end
        w = torch.where((lag >= 0)[:, None], torch.exp(g[:, None] * lag.clamp(min=0)[:, None]), 0.0)
        got += ((k * w[..., None]).transpose(-1, -2).contiguous() @ v
                + torch.exp(g * n[:, None])[..., None, None] * state,)
    if not train:
        return got
    ds_in = None
    if state is not None:
        ds = st["dstate"].double()
        dq += (do * fade[..., None]) @ state.transpose(-1, -2).contiguous() * scale
        late = torch.exp(g[:, None] * (L - ages))[..., None]
        dkey += (v * late) @ ds.transpose(-1, -2).contiguous()
        dval += (k * late) @ ds
        ds_in = ((q * fade[..., None]).transpose(-1, -2).contiguous() @ do * scale
                 + torch.exp(g * L)[:, None, None] * ds)
    return got + (dq, dkey, dval) + (() if ds_in is None else (ds_in,))
