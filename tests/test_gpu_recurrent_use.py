"""The short convolution, the selective scan and the beam search's step as a program uses them:
prompts, single tokens and beams over pooled states, together with the decayed attention's;
captured into graphs; on other streams; workspaces that one call leaves to the next."""
import numpy as np
import pytest

from helpers import to_dev, to_host
from oracle import recurrent as rec
from test_gpu_beam import same

pytestmark = pytest.mark.gpu


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def close(got, ref, name):
    """Two fp32 computations of one value: chains of a few hundred roundings of 2^-24 each, of
    states that decay. What belongs to another beam is of the order of the norm."""
    got, ref = to_host(got), to_host(ref)
    assert np.isfinite(got).all(), name
    assert np.linalg.norm(got - ref) <= 1000 * 2.0 ** -24 * np.linalg.norm(ref), name


class Layer:
    """One layer over a vocabulary: convolution, scan, decayed attention, logits."""

    def __init__(self, V=301, D=64, N=16, W=4, H=2, d=32):
        import torch
        r = np.random.default_rng(5)
        m = lambda *s: to_dev((r.standard_normal(s) / np.sqrt(s[0])).astype(np.float32))
        self.D, self.N, self.W, self.H, self.d = D, N, W, H, d
        self.embed = to_dev(r.standard_normal((V, D)).astype(np.float32))
        self.taps, self.bias = m(W, D).t().contiguous(), m(D, 1)[:, 0].contiguous()
        self.in_dt, self.in_b, self.in_c, self.in_z = m(D, D), m(D, N), m(D, N), m(D, D)
        self.q, self.k, self.v = m(D, H * d), m(D, H * d), m(D, H * d)
        self.head = 3 * m(H * d, V)
        self.A = to_dev(-np.exp(r.uniform(-2, 1, (D, N))).astype(np.float32))
        self.skip, self.dt_bias = m(D, 1)[:, 0].contiguous(), to_dev(np.full(D, -2, np.float32))
        self.decay = torch.tensor([-0.05, -0.3], device="cuda")

    def _low(self, u):
        return (u @ self.in_dt, self.A, (u @ self.in_b).unsqueeze(-2), (u @ self.in_c).unsqueeze(-2))

    def prompt(self, tokens, lengths):
        """(logits of every token, the states after the last ones)."""
        fv, x = _fv(), self.embed[tokens]
        B, L = tokens.shape
        u, cs = fv.causal_conv(x, self.taps, self.bias, True, lengths, return_state=True)
        y, hs = fv.selective_scan(u, *self._low(u), self.skip, x @ self.in_z, self.dt_bias,
                                  lengths=lengths, return_state=True)
        heads = lambda m: (y @ m).view(B, L, self.H, self.d).transpose(1, 2)
        o, at = fv.attn_decay(heads(self.q), heads(self.k), heads(self.v), self.decay,
                              lengths=lengths, return_state=True)
        return o.transpose(1, 2).reshape(B, L, -1) @ self.head, (cs, hs, at)

    def token(self, tokens, pools, slots):
        fv, x = _fv(), self.embed[tokens]
        u = fv.causal_conv_step(x, self.taps, pools[0], self.bias, True, slots)
        y = fv.selective_scan_step(u, *self._low(u), pools[1], self.skip, x @ self.in_z,
                                   self.dt_bias, slots=slots)
        heads = lambda m: (y @ m).view(-1, self.H, self.d)
        o = fv.attn_decay_step(heads(self.q), heads(self.k), heads(self.v), self.decay, pools[2],
                               slots=slots)
        return o.reshape(len(tokens), -1) @ self.head

    def pools(self, n):
        import torch
        return [torch.full((n, *s), np.nan, device="cuda") for s in
                ((self.W - 1, self.D), (self.D, self.N), (self.H, self.d, self.d))]


def test_beam_search_over_pooled_states():
    """A padded batch of prompts, then beams: every choice is the oracle's on the logits it was
    made from, and the states and scores that the beams end with are those of running their
    tokens anew."""
    import torch
    fv, m = _fv(), Layer()
    B, K, T, V, end = 3, 4, 7, m.embed.shape[0], 11
    r = np.random.default_rng(1)
    lengths = [9, 1, 6]
    prompt = torch.tensor(r.integers(12, V, (B, 9)), device="cuda")
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    logits, states = m.prompt(prompt, lens)
    n_slots = B * K + 2
    slots = torch.tensor(r.permutation(n_slots)[:B * K].reshape(B, K), dtype=torch.int32,
                         device="cuda")
    pools = m.pools(n_slots)
    for pool, s in zip(pools, states):
        pool[slots[:, 0].long()] = s
    spare = [i for i in range(n_slots) if i not in slots.flatten().tolist()]
    last = logits[torch.arange(B), lens.long() - 1]
    logits = last[:, None].expand(B, K, V)   # all beams on one row of memory
    scores = torch.tensor([0.0] + [-np.inf] * (K - 1), device="cuda").repeat(B, 1)
    ended = torch.zeros(B, K, dtype=torch.bool, device="cuda")
    text = [[[] for _ in range(K)] for _ in range(B)]
    ends = 0
    for step in range(T):
        if step == 3:   # the best continuation of one entry's best beam ends it
            logits = logits.clone()
            logits[1, 0, end] = logits[1, 0].max() + 4
        got = fv.beam_select(logits, scores, K, ended, end)
        same(got, rec.beam_select(to_host(logits), scores.double().cpu().numpy(), K,
                                  ended.cpu().numpy(), end), V, 20)
        new_scores, parent, token = got
        new_slots = fv.beam_reorder(parent, slots, pools)
        assert [sorted(s) for s in new_slots.tolist()] == [sorted(s) for s in slots.tolist()]
        was = ended.gather(1, parent.long())
        text = [[text[b][p] + ([] if w else [t]) for p, t, w in zip(*row)] for b, row in
                enumerate(zip(parent.tolist(), token.tolist(), was.tolist()))]
        ended, scores, slots = was | (token == end), new_scores, new_slots
        ends += int(ended.sum())
        # ended beams run no more: they are absent
        run = torch.where(ended, -1, slots).flatten().contiguous()
        logits = m.token(token.flatten().long(), pools, run).view(B, K, V)
    assert ends   # some beam ended, and stayed
    # the same tokens, run anew (the end token is not run)
    rows = [prompt[b, :lengths[b]].tolist() + [t for t in text[b][k] if t != end]
            for b in range(B) for k in range(K)]
    n = torch.tensor([len(x) for x in rows], dtype=torch.int32, device="cuda")
    all_tokens = torch.zeros(B * K, int(n.max()), dtype=torch.long, device="cuda")
    for i, x in enumerate(rows):
        all_tokens[i, :len(x)] = torch.tensor(x)
    full, again = m.prompt(all_tokens, n)
    at = slots.flatten().long()
    for pool, s, name in zip(pools, again, ("inputs", "states", "sums")):
        close(pool[at], s, name)
        assert torch.isnan(pool[spare]).all()   # never written
    on = ~ended.flatten()
    close(logits.view(B * K, V)[on], full[torch.arange(B * K), n.long() - 1][on], "logits")
    logp = torch.log_softmax(full.double(), -1)
    for b in range(B):
        for k in range(K):
            if b == 1 or bool(ended[b, k]):
                continue   # logits that were made by hand; a token that was not run
            i, p = b * K + k, lengths[b]
            want = sum(float(logp[i, p - 1 + j, t]) for j, t in enumerate(text[b][k]))
            assert abs(float(scores[b, k]) - want) < 1000 * 2.0 ** -24 * (abs(want) + 10 * T)


def test_a_sequence_in_pieces_is_the_sequence():
    """Conv and scan over a sequence cut into pieces and single tokens, states in one buffer."""
    import torch
    fv, m = _fv(), Layer()
    r = np.random.default_rng(9)
    tokens = torch.tensor(r.integers(0, 301, (2, 400)), device="cuda")
    n = torch.tensor([400, 400], dtype=torch.int32, device="cuda")
    full, states = m.prompt(tokens, n)
    x = m.embed[tokens]
    cs, hs = torch.zeros_like(states[0]), torch.zeros_like(states[1])
    u = torch.empty_like(x)
    y = torch.empty_like(x)
    at = 0
    for piece in (1, 2, 130, 1, 1, 200, 65):
        s = slice(at, at + piece)
        if piece == 1:
            fv.causal_conv_step(x[:, at], m.taps, cs, m.bias, True, out=u[:, at])
            low = [v[:, 0] if v.dim() > 2 else v for v in m._low(u[:, s])]
            fv.selective_scan_step(u[:, at], *low, hs, m.skip, x[:, at] @ m.in_z, m.dt_bias,
                                   out=y[:, at])
        else:
            fv.causal_conv(x[:, s], m.taps, m.bias, True, None, cs, True, u[:, s], cs)
            fv.selective_scan(u[:, s], *m._low(u[:, s]), m.skip, x[:, s] @ m.in_z, m.dt_bias,
                              state_in=hs, return_state=True, out=y[:, s], state_out=hs)
        at += piece
    assert at == 400
    u1 = fv.causal_conv(x, m.taps, m.bias, True)
    y1 = fv.selective_scan(u1, *m._low(u1), m.skip, x @ m.in_z, m.dt_bias)
    for got, ref, name in ((u, u1, "u"), (y, y1, "y"), (cs, states[0], "cs"), (hs, states[1], "hs")):
        close(got, ref, name)


def _buffers(B, L, D, N, W, K, V, G=2, dtype="bf16"):
    """Inputs of a training step, of single tokens and of a beam step, and all that is written."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    new = lambda *s, dtype=t: torch.zeros(*s, dtype=dtype, device="cuda")
    f = lambda *s: new(*s, dtype=torch.float32)
    i32 = lambda *s: new(*s, dtype=torch.int32)
    i = dict(x=new(B, L, D), w=f(D, W), bias=f(D), dt=new(B, L, D), A=f(D, N), Bm=new(B, L, G, N),
             C=new(B, L, G, N), skip=f(D), z=new(B, L, D), dtb=f(D), dy=new(B, L, D),
             cs=new(B, W - 1, D), hs=f(B, D, N), lens=i32(B), slots=i32(B, K),
             logits=new(B, K, V), scores=f(B, K))
    o = dict(u=new(B, L, D), y=new(B, L, D), cs=new(B, W - 1, D), hs=f(B, D, N),
             dx=new(B, L, D), ddt=new(B, L, D), dA=f(D, N), dB=new(B, L, G, N), dC=new(B, L, G, N),
             dD=f(D), dz=new(B, L, D), dtb=f(D), dhs=f(B, D, N), dcx=new(B, L, D), dw=f(D, W),
             db=f(D), dcs=new(B, W - 1, D), ut=new(B * K, D), yt=new(B * K, D),
             cpool=new(B * K, W - 1, D), hpool=f(B * K, D, N), s=f(B, K), parent=i32(B, K),
             token=i32(B, K), slots=i32(B, K))
    return i, o


def _fill(i, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    for k, t in i.items():
        if k == "lens":
            t.copy_(torch.randint(0, i["x"].shape[1] + 1, t.shape, generator=g, device="cuda"))
        elif k == "slots":
            B, K = t.shape
            t.copy_(torch.randperm(B * K, generator=g, device="cuda").view(B, K))
        else:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    i["A"].copy_(-i["A"].abs() - 0.1)


def _step(i, o, ws):
    """Everything that has a buffer, one call after the other."""
    fv = _fv()
    fv.causal_conv(i["x"], i["w"], i["bias"], True, i["lens"], i["cs"], True, o["u"], o["cs"])
    fv.selective_scan(o["u"], i["dt"], i["A"], i["Bm"], i["C"], i["skip"], i["z"], i["dtb"], True,
                      i["lens"], i["hs"], True, o["y"], o["hs"], ws)
    fv.selective_scan_backward(
        o["u"], i["dt"], i["A"], i["Bm"], i["C"], i["dy"], i["skip"], i["z"], i["dtb"], True,
        i["lens"], i["hs"], i["hs"], True, o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"], o["dD"],
        o["dz"], o["dtb"], o["dhs"], ws)
    fv.causal_conv_backward(i["x"], i["w"], o["dx"], i["bias"], True, i["lens"], i["cs"], i["cs"],
                            True, o["dcx"], o["dw"], o["db"], o["dcs"], ws)
    B, K = i["slots"].shape
    at = i["slots"].view(-1)
    row = i["x"].view(-1, i["x"].shape[-1])[:B * K]
    low = lambda t: t.view(-1, *t.shape[2:])[:B * K]
    fv.causal_conv_step(row, i["w"], o["cpool"], i["bias"], True, at, o["ut"])
    fv.selective_scan_step(o["ut"], row, i["A"], low(i["Bm"]), low(i["C"]), o["hpool"], i["skip"],
                           row, i["dtb"], True, at, o["yt"])
    fv.beam_select(i["logits"], i["scores"], K, None, 0, o["s"], o["parent"], o["token"], ws)
    fv.beam_reorder(o["parent"], i["slots"], [o["cpool"], o["hpool"]], o["slots"])


def _workspace(i):
    import torch
    return torch.empty(64 << 20, dtype=torch.uint8, device="cuda")


def _equal(a, b, note):
    import torch
    for k in a:
        assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), (note, k)


@pytest.mark.parametrize("dtype,L", [("bf16", 500), ("f32", 300)])
def test_captured_step(dtype, L):
    """Two graphs that share a workspace, replayed on new inputs with eager work between, give
    what eager calls give, bit by bit."""
    import torch
    size = (3, L, 80, 16, 4, 4, 2000)
    i, ref = _buffers(*size, dtype=dtype)
    outs = [_buffers(*size, dtype=dtype)[1] for _ in range(2)]
    ws = _workspace(i)
    _fill(i, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(i, ref, ws)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for o in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _step(i, o, ws)
        graphs.append(graph)
    torch.cuda.synchronize()
    for rep in range(4):
        _fill(i, 10 + rep)
        pools = torch.randn_like(ref["hpool"]), torch.randn_like(ref["cpool"].float())
        for o in (ref, *outs):
            for k in o:
                o[k].zero_()
            o["hpool"].copy_(pools[0])
            o["cpool"].copy_(pools[1])
        _step(i, ref, torch.full_like(ws, 255))
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            _equal(o, ref, (dtype, rep))
        ws.fill_(0x7f)
    assert all(bool(torch.isfinite(ref[k].float()).all()) for k in ref if k != "s")


def test_two_streams_at_once():
    """Two steps at once on their own streams, buffers and workspaces; then the default
    workspaces of calls on another stream."""
    import torch
    size = (2, 900, 128, 16, 3, 4, 5000)
    runs = []
    for seed in (1, 2):
        i, ref = _buffers(*size)
        _fill(i, seed)
        ws = _workspace(i)
        _step(i, ref, ws)
        runs.append((i, ref, _buffers(*size)[1], ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for rep in range(3):
        for i, ref, o, ws, stream in runs:
            for k in o:
                o[k].zero_()
            stream.wait_stream(torch.cuda.current_stream())
        for i, ref, o, ws, stream in runs:
            with torch.cuda.stream(stream):
                _step(i, o, ws if rep else None)
        torch.cuda.synchronize()
        for i, ref, o, ws, stream in runs:
            _equal(o, ref, rep)


def test_calls_repeat_bit_by_bit():
    """Nothing depends on an order that may change: no atomics on sums."""
    import torch
    size = (4, 1500, 256, 16, 4, 3, 999)
    i, first = _buffers(*size)
    _fill(i, 3)
    _step(i, first, None)
    for rep in range(3):
        o = _buffers(*size)[1]
        _step(i, o, None)
        torch.cuda.synchronize()
        _equal(o, first, rep)


def test_rows_far_apart():
    """Tokens as far apart as the scan takes them (offsets past 32 bits): as contiguous rows."""
    import torch
    fv = _fv()
    i, o = _buffers(1, 300, 16, 8, 4, 1, 8)
    _fill(i, 4)
    i["lens"].fill_(300)
    far = torch.empty(1 + 299 * (1 << 24) + 64, dtype=torch.bfloat16, device="cuda")   # 10 GB
    rows = lambda at, n=16: far[at:].as_strided((1, 300, n), (0, 1 << 24, 1))
    names = dict(x=0, dt=16, z=32, dy=48)
    g = {k: rows(at) for k, at in names.items()}
    scan = lambda t: (*fv.selective_scan(t["x"], t["dt"], i["A"], i["Bm"], i["C"], i["skip"], t["z"],
                                         i["dtb"], state_in=i["hs"], return_state=True),
                      *fv.selective_scan_backward(t["x"], t["dt"], i["A"], i["Bm"], i["C"], t["dy"],
                                                  i["skip"], t["z"], i["dtb"], state_in=i["hs"]))
    conv = lambda t: (fv.causal_conv(t["x"], i["w"], i["bias"], True),
                      *fv.causal_conv_backward(t["x"], i["w"], t["dy"], i["bias"], True))
    want = [v.clone() for v in (*scan(i), *conv(i))]
    for k, v in g.items():
        v.copy_(i[k])
    assert g["dy"].stride(1) * 2 == 1 << 25
    for got, ref in zip((*scan(g), *conv(g)), want):
        assert torch.equal(got, ref)
    # and outputs: y and dx in rows of their own
    y, dx = rows(0), rows(16)
    fv.selective_scan(i["x"], i["dt"], i["A"], i["Bm"], i["C"], i["skip"], i["z"], i["dtb"],
                      state_in=i["hs"], out=y)
    fv.causal_conv_backward(i["x"], i["w"], i["dy"], i["bias"], True, dx=dx)
    assert torch.equal(y, want[0]) and torch.equal(dx, want[11])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_broadcast_inputs(dtype):
    """Inputs that are one row or one sequence for all, as views: as their copies."""
    import torch
    fv = _fv()
    B, L = 3, 140
    i, _ = _buffers(B, L, 48, 8, 3, 1, 8, dtype=dtype)
    _fill(i, 6)
    wide = dict(i, x=i["x"][:1].expand(B, L, 48), dt=i["dt"][:, :1].expand(B, L, 48),
                z=i["z"][:1, :1].expand(B, L, 48), dy=i["dy"][:1, :1].expand(B, L, 48),
                Bm=i["Bm"][:, :, :1].expand(B, L, 2, 8), C=i["C"][:1].expand(B, L, 2, 8))
    whole = {k: v.contiguous() for k, v in wide.items()}

    def run(t):
        a = [t[k] for k in ("x", "dt", "A", "Bm", "C")]
        return (fv.causal_conv(t["x"], t["w"], t["bias"], True),
                *fv.causal_conv_backward(t["x"], t["w"], t["dy"], t["bias"], True),
                fv.selective_scan(*a, t["skip"], t["z"], t["dtb"]),
                *fv.selective_scan_backward(*a, t["dy"], t["skip"], t["z"], t["dtb"]))

    for got, ref in zip(run(wide), run(whole)):
        assert torch.equal(got, ref)


def test_reorder_without_pools():
    """Only the places are worked out."""
    import torch
    slots = torch.tensor([[5, 2, 9], [1, 0, 7]], dtype=torch.int32, device="cuda")
    parent = torch.tensor([[1, 1, 0], [2, 2, 2]], dtype=torch.int32, device="cuda")
    ref, _ = rec.beam_reorder(parent.tolist(), slots.tolist(), [])
    assert np.array_equal(_fv().beam_reorder(parent, slots, []).cpu().numpy(), ref)
