"""The calls the selective scan, the short convolution and the beam search's step are measured on.

Each case is a dict of plain values. Short causal convolution, one filter per channel (op conv):
  kind      step    one token for each of B sequences, the last inputs kept in a pool
            prompt  a stretch of L tokens, forward
            train   forward and backward over L tokens
  B, L, D   batch, tokens and channels; width: taps of a filter
  dtype     bf16 or f32: inputs, outputs and their gradients (parameters are always f32)
  bias, silu  1: a bias, a SiLU behind the filter
  layout    bld: contiguous [B, L, D]; packed: one half of a [B, L, 2 D] projection
  ragged    1: a right-padded batch, every sequence of its own length
  state     1: the last inputs before the stretch come in, those after it go out
  slots     step: 0: state b belongs to sequence b; n: sequences hold places in a pool of n
Selective scan (op scan), the same keys and
  N, G      states per channel; groups of channels that share B and C
  z         1: the output is gated by silu(z)
  skip      1: the input skips the scan with a weight per channel
B and C are slices of one projection of the input, as a layer makes them.
Beam search's choice of the next tokens (op select):
  B, K, V   batch, beams, vocabulary; n: beams chosen
  dtype     of the logits
  ended     1: some beams have ended (they stay as they are, with the end token 2)
Moving pooled states behind the chosen beams (op reorder):
  B, K      batch and beams; dead: beams of each batch entry that no chosen one continues
  layers, D, N, width  the pools: a scan state and a convolution's inputs for every layer
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_CONV = dict(op="conv", kind="prompt", B=1, L=1, D=2048, width=4, dtype="bf16", bias=1, silu=1,
             layout="bld", ragged=0, state=0, slots=0)
_SCAN = dict(op="scan", kind="prompt", B=1, L=1, D=2048, N=16, G=1, dtype="bf16", layout="bld",
             z=1, skip=1, ragged=0, state=0, slots=0)


def _case(base, name, **kw):
    return dict(base, name=name, **kw)


def listed():
    return [
        # the next token of one sequence: only latency counts
        _case(_CONV, "conv_step", kind="step"),
        # a padded batch of float32 prompts of odd lengths, three taps, that carries its inputs
        _case(_CONV, "conv_ragged", B=6, L=1999, D=1000, width=3, dtype="f32", silu=0, ragged=1,
              state=1),
        # a training step of a layer on one half of its input projection
        _case(_CONV, "conv_train", kind="train", B=4, L=4096, D=4096, layout="packed"),
        # a decoding step of a full serving batch whose states live in a pool
        _case(_SCAN, "scan_step", kind="step", B=48, D=4096, slots=64),
        # a padded batch of float32 prompts of odd lengths that carries its states
        _case(_SCAN, "scan_ragged", B=6, L=1999, D=1000, N=24, G=1, dtype="f32", ragged=1, state=1),
        # one long document
        _case(_SCAN, "scan_long", L=65536, layout="packed"),
        # a small float32 training step that carries a state through a piece; shared B, C groups
        _case(_SCAN, "scan_train_f32", kind="train", B=2, L=777, D=512, N=64, G=2, dtype="f32", z=0,
              state=1),
        # a training step of a model's layer
        _case(_SCAN, "scan_train", kind="train", B=4, L=4096, layout="packed"),
        # one sentence, four beams, an odd vocabulary
        dict(name="select_one", op="select", B=1, K=4, V=50001, n=4, dtype="f32", ended=0),
        # a serving batch with eight beams each, some of them ended
        dict(name="select_batch", op="select", B=32, K=8, V=131072, n=8, dtype="bf16", ended=1),
        # one layer's states of one sentence
        dict(name="reorder_one", op="reorder", B=1, K=4, dead=2, layers=1, D=2048, N=16, width=4),
        # all layers' states of a serving batch
        dict(name="reorder_layers", op="reorder", B=8, K=8, dead=3, layers=24, D=2048, N=16, width=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv", "conv", "scan", "scan", "scan", "scan", "select", "reorder"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "select":
        B, K = _log(rng, 1, 32), rng.randint(1, 12)
        n = rng.randint(1, 16)
        return dict(op=op, B=B, K=K, V=_log(rng, 300, min(200000, (1 << 24) // (B * K))), n=n,
                    dtype=dtype, ended=rng.randrange(2))
    if op == "reorder":
        K = rng.randint(2, 12)
        return dict(op=op, B=_log(rng, 1, 8), K=K, dead=rng.randint(0, K - 1),
                    layers=_log(rng, 1, 16), D=8 * _log(rng, 8, 256), N=rng.choice([8, 16, 32]),
                    width=rng.randint(2, 5))
    kind = rng.choice(["step", "prompt", "prompt", "train", "train"])
    G = rng.choice([1, 1, 2, 4]) if op == "scan" else 1
    D = 8 * G * _log(rng, 8, 512 // G)
    extra = (dict(width=rng.randint(2, 5), bias=rng.randrange(2), silu=rng.randrange(2))
             if op == "conv" else
             dict(N=rng.choice([rng.randint(1, 64), 8, 16, 16, 16, 32, 64]), G=G,
                  z=rng.randrange(2), skip=rng.randrange(2)))
    case = dict(_CONV if op == "conv" else _SCAN, kind=kind, D=D, dtype=dtype, **extra)
    if kind == "step":
        B = _log(rng, 1, 64)
        return dict(case, B=B, slots=rng.choice([0, B + rng.randint(0, 16)]))
    B = rng.randint(1, 6)
    if op == "conv":
        most = (1 << 25) // (B * D)
    else:
        most = (1 << 28 if kind == "train" else 1 << 30) // (B * D * case["N"])
    return dict(case, B=B, L=_log(rng, 1, max(2, min(40000, most))),
                layout=rng.choice(["bld", "packed"]), state=rng.randrange(2),
                ragged=rng.randrange(2) if kind == "prompt" else 0)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _uniform(gen, lo, hi, *shape):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def _tokens(case, gen):
    """[B, L, D] inputs in the case's layout ([B, D] for single tokens)."""
    B, L, D, dt = case["B"], case["L"], case["D"], _DTYPES[case["dtype"]]
    if case["kind"] == "step":
        return _rand(gen, B, D).to(dt)
    if case["layout"] == "packed":
        return _rand(gen, B, L, 2 * D).to(dt)[..., :D]
    return _rand(gen, B, L, D).to(dt)


def _places(case, gen):
    n = case["slots"] or case["B"]
    if not case["slots"]:
        return n, None
    return n, torch.randperm(n, generator=gen, device="cuda")[:case["B"]].to(torch.int32)


def _lengths(case, gen):
    L = case["L"]
    if not case["ragged"]:
        return None
    return torch.randint(min(L, 1 + L // 8), L + 1, (case["B"],), generator=gen, device="cuda",
                         dtype=torch.int32)


def _prepare_conv(case, gen):
    B, L, D, W, dt = case["B"], case["L"], case["D"], case["width"], _DTYPES[case["dtype"]]
    st = dict(case=case, x=_tokens(case, gen), weight=_uniform(gen, -1, 1, D, W) * W ** -0.5,
              bias=_uniform(gen, -1, 1, D) * W ** -0.5 if case["bias"] else None, lengths=None,
              state=None, slots=None, dout=None, dstate=None)
    if case["kind"] == "step":
        n, st["slots"] = _places(case, gen)
        st["state"] = _rand(gen, n, W - 1, D).to(dt)
        return st
    st["lengths"] = _lengths(case, gen)
    if case["state"]:
        st["state"] = _rand(gen, B, W - 1, D).to(dt)
    if case["kind"] == "train":
        st["dout"] = _rand(gen, B, L, D).to(dt)
        if case["state"]:
            st["dstate"] = _rand(gen, B, W - 1, D).to(dt)
    return st


def _prepare_scan(case, gen):
    B, L, D, N, G, dt = (case[k] for k in ("B", "L", "D", "N", "G", "dtype"))
    dt = _DTYPES[dt]
    lead = (B,) if case["kind"] == "step" else (B, L)
    # decays of 1 .. N per unit of time, steps of 0.001 to 0.1 units
    step = torch.exp(_uniform(gen, math.log(1e-3), math.log(1e-1), D))
    low = _rand(gen, *lead, 2, G, N).to(dt)   # B and C side by side
    st = dict(case=case, x=_tokens(case, gen), dt=(0.5 * _rand(gen, *lead, D)).to(dt),
              A=-torch.arange(1, N + 1, device="cuda").float() * _uniform(gen, 0.8, 1.2, D, N),
              B=low.select(-3, 0), C=low.select(-3, 1),
              D=1 + 0.1 * _rand(gen, D) if case["skip"] else None,
              z=_tokens(case, gen) if case["z"] else None,
              dt_bias=step + torch.log(-torch.expm1(-step)),
              lengths=None, state=None, slots=None, dout=None, dstate=None)
    if case["kind"] == "step":
        n, st["slots"] = _places(case, gen)
        st["state"] = _rand(gen, n, D, N)
        return st
    st["lengths"] = _lengths(case, gen)
    if case["state"]:
        st["state"] = _rand(gen, B, D, N)
    if case["kind"] == "train":
        st["dout"] = _rand(gen, B, L, D).to(dt)
        if case["state"]:
            st["dstate"] = _rand(gen, B, D, N)
    return st


def _prepare_select(case, gen):
    B, K, V = case["B"], case["K"], case["V"]
    st = dict(case=case, logits=(3 * _rand(gen, B, K, V)).to(_DTYPES[case["dtype"]]),
              scores=-_uniform(gen, 0, 4, B, K), ended=None)
    if case["ended"]:
        st["ended"] = torch.rand((B, K), generator=gen, device="cuda") < 0.25
    return st


def _prepare_reorder(case, gen):
    B, K, dead = case["B"], case["K"], case["dead"]
    n = B * K + 3   # a pool with places to spare
    # K - dead beams that live on, each once, and some of them again
    alive = torch.rand((B, K), generator=gen, device="cuda").argsort(-1)[:, :K - dead]
    again = torch.randint(0, K - dead, (B, dead), generator=gen, device="cuda")
    parent = torch.cat((alive, alive.gather(1, again)), 1)
    mix = torch.rand((B, K), generator=gen, device="cuda").argsort(-1)
    slots = torch.randperm(n, generator=gen, device="cuda")[:B * K].reshape(B, K)
    pools = []
    for _ in range(case["layers"]):
        pools.append(_rand(gen, n, case["D"], case["N"]))
        pools.append(_rand(gen, n, case["width"] - 1, case["D"]).to(torch.bfloat16))
    return dict(case=case, parent=parent.gather(1, mix).to(torch.int32),
                slots=slots.to(torch.int32), pools=pools)


def prepare(case, seed):
    return {"conv": _prepare_conv, "scan": _prepare_scan, "select": _prepare_select,
            "reorder": _prepare_reorder}[case["op"]](case, _gen(seed))


# ------------------------------------------------------------------ plain forms
def _valid(st):
    """[B, L, 1]: the tokens that are there."""
    B, L = st["x"].shape[:2]
    n = st["lengths"]
    if n is None:
        n = torch.full((B,), L, device="cuda")
    return (torch.arange(L, device="cuda") < n[:, None]).unsqueeze(-1), n.long()


def _conv_step(st):
    idx = slice(None) if st["slots"] is None else st["slots"].long()
    x = torch.cat((st["state"][idx], st["x"].unsqueeze(1)), 1)
    u = (x.float() * st["weight"].t()).sum(1)
    if st["bias"] is not None:
        u = u + st["bias"]
    if st["case"]["silu"]:
        u = u * torch.sigmoid(u)
    st["state"][idx] = x[:, 1:]
    return u.to(st["x"].dtype), st["state"]


def _taps(st):
    """The inputs with the W - 1 before them, and the filters' sums."""
    W, (B, L, D) = st["case"]["width"], st["x"].shape
    ok, n = _valid(st)
    x = torch.where(ok, st["x"].float(), 0.0)
    first = torch.zeros(B, W - 1, D, device="cuda") if st["state"] is None else st["state"].float()
    x = torch.cat((first, x), 1)
    u = sum(x[:, j:j + L] * st["weight"][:, j] for j in range(W))
    if st["bias"] is not None:
        u = u + st["bias"]
    return x, u, ok, n


def _conv(st):
    case, dt = st["case"], st["x"].dtype
    W, (B, L, D) = case["width"], st["x"].shape
    x, u, ok, n = _taps(st)
    y = u * torch.sigmoid(u) if case["silu"] else u
    got = (torch.where(ok, y, 0.0).to(dt),)
    if case["state"]:
        at = n[:, None] + torch.arange(W - 1, device="cuda")
        got += (x.gather(1, at.unsqueeze(-1).expand(B, W - 1, D)).to(dt),)
    return got


def _conv_backward(st):
    case, dt = st["case"], st["x"].dtype
    W, (B, L, D) = case["width"], st["x"].shape
    x, u, _, _ = _taps(st)
    g = st["dout"].float()
    if case["silu"]:
        s = torch.sigmoid(u)
        g = g * (s * (1 + u * (1 - s)))
    dx = torch.zeros_like(x)
    for j in range(W):
        dx[:, j:j + L] += g * st["weight"][:, j]
    if st["dstate"] is not None:
        dx[:, L:] += st["dstate"].float()
    got = (dx[:, W - 1:].to(dt),
           torch.stack([(g * x[:, j:j + L]).sum((0, 1)) for j in range(W)], -1))
    if st["bias"] is not None:
        got += (g.sum((0, 1)),)
    return got + ((dx[:, :W - 1].to(dt),) if case["state"] else ())


def _channels(t, D):
    """[..., G, N] of groups as [..., D, N] of their channels."""
    return t.float().repeat_interleave(D // t.shape[-2], -2)


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def _gate(st, y):
    if st["z"] is None:
        return y
    z = st["z"].float()
    return y * (z * torch.sigmoid(z))


def _scan_step(st):
    idx = slice(None) if st["slots"] is None else st["slots"].long()
    x, D = st["x"].float(), st["x"].shape[-1]
    s = _softplus(st["dt"].float() + st["dt_bias"])
    h = st["state"][idx] * torch.exp(s.unsqueeze(-1) * st["A"])
    h = h + (s * x).unsqueeze(-1) * _channels(st["B"], D)
    st["state"][idx] = h
    y = (h * _channels(st["C"], D)).sum(-1)
    if st["D"] is not None:
        y = y + x * st["D"]
    return _gate(st, y).to(st["x"].dtype), st["state"]


def _recur(a, b, h):
    """h_t = a_t h_{t-1} + b_t along dimension 1, written over b: chunks side by side, their
    carried values, and what these add."""
    L = a.shape[1]
    T = max(1, int(L ** 0.5))
    n = -(-L // T)
    whole = [(i * T, min(L, (i + 1) * T)) for i in range(n)]
    full = L // T * T
    av, bv = (t[:, :full].unflatten(1, (L // T, T)) for t in (a, b))
    p = torch.empty_like(av)
    p[:, :, 0] = av[:, :, 0]
    for t in range(1, T):
        torch.mul(av[:, :, t], p[:, :, t - 1], out=p[:, :, t])
        bv[:, :, t].addcmul_(av[:, :, t], bv[:, :, t - 1])
    for i, (lo, hi) in enumerate(whole):
        if hi - lo == T:
            if h is not None:
                bv[:, i].addcmul_(p[:, i], h.unsqueeze(1))
        else:
            for t in range(lo, hi):
                if h is not None:
                    b[:, t].addcmul_(a[:, t], h)
                h = b[:, t]
        h = b[:, hi - 1]
    return b


def _terms(st):
    ok, n = _valid(st)
    x = torch.where(ok, st["x"].float(), 0.0)
    raw = torch.where(ok, st["dt"].float(), 0.0) + st["dt_bias"]
    s = torch.where(ok, _softplus(raw), 0.0)   # a step of no time leaves the state
    D = x.shape[-1]
    Bc, Cc = (_channels(torch.where(ok.unsqueeze(-1), st[k].float(), 0.0), D) for k in "BC")
    return ok, x, raw, s, Bc, Cc


def _scan(st, keep=False):
    ok, x, raw, s, Bc, Cc = _terms(st)
    a = torch.exp(s.unsqueeze(-1) * st["A"])
    h = _recur(a, (s * x).unsqueeze(-1) * Bc, st["state"])
    y = (h * Cc).sum(-1)
    if st["D"] is not None:
        y = y + x * st["D"]
    out = torch.where(ok, _gate(st, y), 0.0).to(st["x"].dtype)
    got = (out, h[:, -1].clone()) if st["case"]["state"] else (out,)
    return (got, (x, raw, s, Bc, Cc, a, h, y)) if keep else got


def _scan_train(st):
    case, dt = st["case"], st["x"].dtype
    G = case["G"]
    got, (x, raw, s, Bc, Cc, a, h, y) = _scan(st, keep=True)
    do = st["dout"].float()
    e = _gate(st, do)
    late = torch.cat((a[:, 1:], torch.ones_like(a[:, :1])), 1).flip(1)   # a_{t+1}
    g = _recur(late, (e.unsqueeze(-1) * Cc).flip(1), st["dstate"]).flip(1)
    before = torch.cat((torch.zeros_like(h[:, :1]) if st["state"] is None
                        else st["state"].unsqueeze(1), h[:, :-1]), 1)
    lost = g * a * before
    ds = (lost * st["A"]).sum(-1) + x * (g * Bc).sum(-1)
    dx = s * (g * Bc).sum(-1)
    if st["D"] is not None:
        dx = dx + e * st["D"]
    groups = (G, x.shape[-1] // G)
    dB, dC = (t.unflatten(2, groups).sum(3).to(dt)
              for t in (g * (s * x).unsqueeze(-1), h * e.unsqueeze(-1)))
    ddt = ds * torch.sigmoid(raw)
    got += (dx.to(dt), ddt.to(dt), (lost * s.unsqueeze(-1)).sum((0, 1)), dB, dC)
    if st["D"] is not None:
        got += ((e * x).sum((0, 1)),)
    if st["z"] is not None:
        z = st["z"].float()
        k = torch.sigmoid(z)
        got += ((do * y * (k * (1 + z * (1 - k)))).to(dt),)
    got += (ddt.sum((0, 1)),)
    return got + ((g[:, 0] * a[:, 0],) if case["state"] else ())


def _ordered(x):
    """Whole numbers of 32 bits in the order of the floats."""
    b = x.float().add(0.0).view(torch.int32).long()   # -0 and 0 are one value
    return torch.where(b >= 0, b, -(b & 0x7FFFFFFF))


def _select(st):
    """Each beam's best by logit (ties: the lower token), then the best of all."""
    x, n = st["logits"], st["case"]["n"]
    B, K, V = x.shape
    w = x.double()
    lse = torch.logsumexp(w, -1, keepdim=True)
    key = _ordered(x) * (1 << 32) - torch.arange(V, device="cuda")
    _, at = key.topk(min(n, V), -1)
    score = st["scores"].double().unsqueeze(-1) + (w.gather(-1, at) - lse)
    if st["ended"] is not None:
        over = st["ended"].unsqueeze(-1)
        only = torch.arange(score.shape[-1], device="cuda") == 0
        stay = torch.where(only, st["scores"].double().unsqueeze(-1), -math.inf)
        score = torch.where(over, stay, score)
        at = torch.where(over & only, 2, at)
    beam = torch.arange(K, device="cuda").view(1, K, 1).expand_as(at)
    score, at, beam = (t.reshape(B, -1) for t in (score, at, beam))
    score, best = score.sort(dim=-1, descending=True, stable=True)
    best, score = best[:, :n], score[:, :n]
    # too few to choose from: the rest is the first beam's, with the end token
    none = score == -math.inf
    parent, token = (torch.where(none, fill, t.gather(1, best)).to(torch.int32)
                     for t, fill in ((beam, 0), (at, 2)))
    short = n - score.shape[1]
    if short > 0:
        pad = torch.nn.functional.pad
        score, parent, token = (pad(t, (0, short), value=v) for t, v in
                                ((score, -math.inf), (parent, 0), (token, 2)))
    return score.float(), parent, token


def _reorder(st):
    """A beam's first child takes its place; the others, in order, those of childless beams."""
    parent, slots = st["parent"].long(), st["slots"]
    K = parent.shape[1]
    same = parent.unsqueeze(-1) == parent.unsqueeze(-2)
    more = (same & torch.ones(K, K, dtype=torch.bool, device="cuda").tril(-1)).any(-1)
    used = (parent.unsqueeze(-1) == torch.arange(K, device="cuda")).any(1)
    free = slots.gather(1, used.int().argsort(dim=-1, stable=True))
    rank = (more.long().cumsum(-1) - 1).clamp(min=0)
    source = slots.gather(1, parent)
    new = torch.where(more, free.gather(1, rank), source)
    at, to = source.flatten().long(), new.flatten().long()
    for p in st["pools"]:
        p[to] = p[at]
    return (new, *st["pools"])


def run(st):
    op, kind = st["case"]["op"], st["case"].get("kind")
    if own:
        return _own(st, op, kind)
    if op == "select":
        return _select(st)
    if op == "reorder":
        return _reorder(st)
    if kind == "step":
        return _conv_step(st) if op == "conv" else _scan_step(st)
    if op == "conv":
        return _conv(st) + (_conv_backward(st) if kind == "train" else ())
    return _scan_train(st) if kind == "train" else _scan(st)


def _own(st, op, kind):
    import paper_2006_03555_amd as fv
    if op == "select":
        return fv.beam_select(st["logits"], st["scores"], st["case"]["n"], ended=st["ended"],
                              end_token=2)
    if op == "reorder":
        return (fv.beam_reorder(st["parent"], st["slots"], st["pools"]), *st["pools"])
    carried = bool(st["case"]["state"])
    if op == "conv":
        x, w, bias, silu = st["x"], st["weight"], st["bias"], bool(st["case"]["silu"])
        if kind == "step":
            return fv.causal_conv_step(x, w, st["state"], bias, silu, slots=st["slots"]), st["state"]
        got = fv.causal_conv(x, w, bias, silu, lengths=st["lengths"], state_in=st["state"],
                             return_state=carried)
        got = got if carried else (got,)
        if kind == "train":
            dx, dw, db, *ds = fv.causal_conv_backward(
                x, w, st["dout"], bias, silu, state_in=st["state"], dstate_out=st["dstate"],
                return_state_grad=carried)
            got += (dx, dw) + (() if bias is None else (db,)) + tuple(ds)
        return got
    args = (st["x"], st["dt"], st["A"], st["B"], st["C"])
    opts = dict(D=st["D"], z=st["z"], dt_bias=st["dt_bias"])
    if kind == "step":
        return fv.selective_scan_step(*args, st["state"], slots=st["slots"], **opts), st["state"]
    got = fv.selective_scan(*args, lengths=st["lengths"], state_in=st["state"],
                            return_state=carried, **opts)
    got = got if carried else (got,)
    if kind == "train":
        g = fv.selective_scan_backward(*args, st["dout"], state_in=st["state"],
                                       dstate_out=st["dstate"], return_state_grad=carried, **opts)
        got += tuple(t for t in g if t is not None)
    return got


# ------------------------------------------------------------------ work
def work(case):
    elt = 2 if case.get("dtype") == "bf16" else 4
    B = case["B"]
    if case["op"] == "select":
        n = B * case["K"] * case["V"]
        # the logits; a difference, an exponential, a sum and a comparison for each
        return {"bytes": n * elt, "flops": 4 * n}
    if case["op"] == "reorder":
        state = case["layers"] * case["D"] * (4 * case["N"] + 2 * (case["width"] - 1))
        return {"bytes": 2 * B * case["dead"] * state + 12 * B * case["K"], "flops": B * case["K"]}
    rows, train, D = B * case["L"], case["kind"] == "train", case["D"]
    if case["op"] == "conv":
        W = case["width"]
        carried = (W - 1) * B * D * elt if case["kind"] == "step" or case["state"] else 0
        # x and y; backward: x, dy, dx; a multiply-add per tap (three backward), the SiLU
        return {"bytes": rows * D * elt * (5 if train else 2) + (4 if train else 2) * carried,
                "flops": rows * D * (2 * W * (4 if train else 1) + 6 * case["silu"])}
    N, low = case["N"], 2 * rows * case["G"] * case["N"] * elt
    carried = 4 * B * D * N if case["kind"] == "step" or case["state"] else 0
    by = rows * D * elt * (3 + case["z"]) + low + 2 * carried + 4 * D * N
    # the product with A, the exponential, the input, the state's and the output's sums
    fl = rows * D * (7 * N + 4)
    if train:
        # the inputs again and dy, four gradients; the gradient's own recurrence and five sums
        by += rows * D * elt * (3 + 2 * case["z"] + 2) + 2 * low + 3 * carried + 4 * D * N
        fl += rows * D * (20 * N + 8)
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------ 64-bit results
def _exact_conv(case, st):
    W, x, w = case["width"], st["x"].double(), st["weight"].double()
    step = case["kind"] == "step"
    if step:
        at = torch.arange(case["B"], device="cuda") if st["slots"] is None else st["slots"].long()
        x, first = x.unsqueeze(1), st["state"].double()[at]
    else:
        first = None if st["state"] is None else st["state"].double()
    B, L, D = x.shape
    if first is None:
        first = x.new_zeros(B, W - 1, D)
    x = torch.cat((first, x), 1)
    bias = 0 if st["bias"] is None else st["bias"].double()
    u = x.unfold(1, W, 1).mul(w).sum(-1) + bias if L * D < 1 << 22 else bias + torch.stack(
        [sum(x[b, j:j + L] * w[:, j] for j in range(W)) for b in range(B)])
    y = u / (1 + torch.exp(-u)) if case["silu"] else u
    if step:
        pool = st["state"].double()
        pool[at] = x[:, 1:]
        return y[:, 0], pool
    got = (y,)
    if case["ragged"]:
        y = torch.where(torch.arange(L, device="cuda")[:, None] < st["lengths"][:, None, None], y, 0.0)
        got = (y,)
    if case["state"]:
        n = [L] * B if st["lengths"] is None else st["lengths"].tolist()
        got += (torch.stack([x[b, m:m + W - 1] for b, m in enumerate(n)]),)
    if case["kind"] != "train":
        return got
    g = st["dout"].double()
    if case["silu"]:
        e = torch.exp(-u)
        g = g * (1 + e + u * e) / (1 + e) ** 2
    dx = torch.zeros_like(x)
    if st["dstate"] is not None:
        dx[:, L:] = st["dstate"].double()
    for j in range(W):
        dx[:, j:j + L] += g * w[:, j]
    got += (dx[:, W - 1:], torch.stack([(g * x[:, j:j + L]).sum(0).sum(0) for j in range(W)], 1))
    if st["bias"] is not None:
        got += (g.sum(0).sum(0),)
    return got + ((dx[:, :W - 1],) if case["state"] else ())


def _exact_scan(case, st):
    """Token by token, the states kept where a backward pass follows."""
    D, N, G, step = case["D"], case["N"], case["G"], case["kind"] == "step"
    x, dt, Bm, Cm = (st[k].double() for k in ("x", "dt", "B", "C"))
    z = None if st["z"] is None else st["z"].double()
    A, skip = st["A"].double(), 0 if st["D"] is None else st["D"].double()
    if step:
        x, dt, Bm, Cm = (t.unsqueeze(1) for t in (x, dt, Bm, Cm))
        z = None if z is None else z.unsqueeze(1)
        at = torch.arange(case["B"], device="cuda") if st["slots"] is None else st["slots"].long()
    B, L = x.shape[:2]
    raw = dt + st["dt_bias"].double()
    s = torch.logaddexp(raw, torch.zeros_like(raw))
    own_group = torch.arange(D, device="cuda") // (D // G)
    n = torch.full((B,), L, device="cuda") if st["lengths"] is None else st["lengths"].long()
    if step:
        h = st["state"].double()[at]
    else:
        h = x.new_zeros(B, D, N) if st["state"] is None else st["state"].double()
    train = case["kind"] == "train"
    y = torch.empty_like(x)
    kept = x.new_empty(L + 1 if train else 1, B, D, N)
    kept[0] = h
    for t in range(L):
        new = h * torch.exp(s[:, t, :, None] * A) + (s[:, t] * x[:, t])[..., None] * Bm[:, t, own_group]
        h = new if st["lengths"] is None else torch.where((t < n)[:, None, None], new, h)
        y[:, t] = (h * Cm[:, t, own_group]).sum(-1)
        if train:
            kept[t + 1] = h
    y = y + skip * x
    silu = 1 if z is None else z / (1 + torch.exp(-z))
    out = y * silu
    if st["lengths"] is not None:
        out = torch.where(torch.arange(L, device="cuda")[:, None] < n[:, None, None], out, 0.0)
    if step:
        pool = st["state"].double()
        pool[at] = h
        return out[:, 0], pool
    got = (out, h) if case["state"] else (out,)
    if not train:
        return got
    do = st["dout"].double()
    e = do * silu
    g = x.new_zeros(B, D, N) if st["dstate"] is None else st["dstate"].double()
    ds, dx, dA = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(A)
    dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
    for t in reversed(range(L)):
        a, now = torch.exp(s[:, t, :, None] * A), Bm[:, t, own_group]
        g = g + e[:, t, :, None] * Cm[:, t, own_group]
        dC[:, t] = (kept[t + 1] * e[:, t, :, None]).view(B, G, -1, N).sum(2)
        dB[:, t] = (g * (s[:, t] * x[:, t])[..., None]).view(B, G, -1, N).sum(2)
        in_ = (g * now).sum(-1)
        g = g * a
        through = g * kept[t]
        dA += (through * s[:, t, :, None]).sum(0)
        ds[:, t] = (through * A).sum(-1) + in_ * x[:, t]
        dx[:, t] = in_ * s[:, t]
    ddt = ds / (1 + torch.exp(-raw))
    got += (dx + skip * e, ddt, dA, dB, dC)
    if st["D"] is not None:
        got += ((e * x).sum(0).sum(0),)
    if z is not None:
        k = 1 / (1 + torch.exp(-z))
        got += (do * y * k * (1 + z * (1 - k)),)
    got += (ddt.sum(0).sum(0),)
    return got + ((g,) if case["state"] else ())


def _exact_select(case, st):
    B, K, V, n = case["B"], case["K"], case["V"], case["n"]
    got = ([], [], [])
    for b in range(B):
        p = torch.log_softmax(st["logits"][b].double(), -1) + st["scores"][b].double()[:, None]
        if st["ended"] is not None:
            for k in st["ended"][b].nonzero().flatten().tolist():
                p[k] = -math.inf
                p[k, 2] = st["scores"][b, k].double()
        s, i = p.flatten().sort(dim=0, descending=True, stable=True)
        s, i = s[:n], i[:n]
        i = torch.where(s == -math.inf, 2, i)
        for to, t in zip(got, (s, i // V, i % V)):
            to.append(t)
    s, parent, token = (torch.stack(t) for t in got)
    return s, parent.to(torch.int32), token.to(torch.int32)


def _exact_reorder(case, st):
    parent, slots = st["parent"].tolist(), st["slots"].tolist()
    new, moves = [], []
    for p, s in zip(parent, slots):
        free = [s[k] for k in range(case["K"]) if k not in p]
        row = []
        for j, k in enumerate(p):
            row.append(free.pop(0) if k in p[:j] else s[k])
            moves.append((s[k], row[-1]))
        new.append(row)
    pools = [t.clone() for t in st["pools"]]
    for a, b in moves:
        if a != b:
            for t in pools:
                t[b] = t[a]
    return (torch.tensor(new, dtype=torch.int32, device="cuda"), *pools)


def exact(case, seed):
    return {"conv": _exact_conv, "scan": _exact_scan, "select": _exact_select,
            "reorder": _exact_reorder}[case["op"]](case, prepare(case, seed))
