"""The decayed linear attention and the dropout as a program uses them: on random features and
under dropout, forward and backward; prompts followed by single tokens; captured into graphs;
on other streams; with states handed on in place."""
import numpy as np
import pytest

import workloads as wl
from helpers import to_dev
from oracle import decay, favor
from test_gpu_decay import _abs, _host, _inputs, _near

pytestmark = pytest.mark.gpu


def _fv():
    import paper_2006_03555_amd as fv
    return fv


def test_features_attention_dropout_and_back():
    """A training step: materialised ReLU features of Q and K, decayed attention over them,
    dropout of its output onto a residual, and the gradients of features and values. Every
    step is compared with the oracle on the inputs the GPU gave it, so that each has only
    its own error; and the sum of gradient times step agrees with the oracle's loss."""
    import torch
    fv = _fv()
    B, H, L, d, M, p, seed = 2, 2, 300, 64, 128, 0.2, 77
    w = wl.Workload("t", "causal", B, H, L, d, M, "f32", 3)
    Q, K, V = wl.make_qkv(w)
    W, b = favor.orf_draw(5, H, M, d)
    g = np.array([-0.02, -0.4], dtype=np.float32)
    gen = np.random.default_rng(0)
    res, dy = (gen.standard_normal((B, H, L, d)).astype(np.float32) for _ in range(2))
    q, k, v = (to_dev(x) for x in (Q, K, V))
    Wd, bd, gd = to_dev(W), to_dev(b), to_dev(g)
    fq, fk = (fv.feature_map(x, Wd, bd, w.input_scale, kernel=fv.KERNEL_RELU) for x in (q, k))
    o = fv.attn_decay(fq, fk, v, gd)
    y = fv.dropout(o, p, seed, 1, residual=to_dev(res))
    do = fv.dropout_backward(to_dev(dy), p, seed, 1)
    dfq, dfk, dv = fv.attn_decay_backward(fq, fk, v, gd, do)
    hq, hk = _host(fq), _host(fk)
    ref, _ = decay.attn(hq, hk, V, g)
    mag, _ = decay.attn(np.abs(hq), np.abs(hk), np.abs(V), g)
    _near(o, ref, mag, M, L, "f32", "attention")
    yref = decay.dropout(_host(o), p, seed, 1, res)
    assert (np.abs(_host(y) - yref) <= 2.0 ** -21 * (np.abs(yref) + np.abs(res))).all()
    back = decay.attn_backward(hq, hk, V, g, _host(do))
    bmag = decay.attn_backward(*(np.abs(x) for x in (hq, hk, V)), g, np.abs(_host(do)))
    for t, r, m, n in zip((dfq, dfk, dv), back, bmag, ("dQ", "dK", "dV")):
        _near(t, r, m, M, L, "f32", n)
    # the loss sum(y dy) moves by the gradients' product with a step (it is linear in V)
    step = gen.standard_normal(V.shape)
    up = decay.dropout(decay.attn(hq, hk, V + step, g)[0], p, seed, 1, res)
    down = decay.dropout(decay.attn(hq, hk, V - step, g)[0], p, seed, 1, res)
    want = ((up - down) * dy).sum() / 2
    assert abs((_host(dv) * step).sum() - want) < 1e-5 * np.abs(_host(dv) * step).sum()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_tokens(dtype):
    """A padded batch of prompts leaves its states in a pool; then single tokens, the
    sequences in another order, one of them absent (place -1)."""
    import torch
    fv = _fv()
    B, H, L, dk, dv, T = 3, 2, 200, 64, 72, 4
    x = _inputs(B, H, L + T, dk, dv, dtype, 21)
    n = [200, 65, 131]
    q, k, v = (to_dev(x[m], dtype) for m in "qkv")
    g = to_dev(x["g"])
    pool = torch.zeros((5, H, dk, dv), device="cuda")
    lens = torch.tensor(n, dtype=torch.int32, device="cuda")
    fv.attn_decay(q[:, :, :L], k[:, :, :L], v[:, :, :L], g, lengths=lens, return_state=True,
                  state_out=pool[1:4])
    order = [2, 0, 1]
    y = _abs(x)
    rows = [[np.concatenate([z[m][b:b + 1, :, :n[b]], z[m][b:b + 1, :, L:]], 2) for m in "qkv"]
            for z in (x, y) for b in range(B)]
    ref = [decay.attn(*r, x["g"]) for r in rows[:B]]
    mag = [decay.attn(*r, x["g"]) for r in rows[B:]]
    for t in range(T):
        idx = torch.tensor(order, device="cuda")
        slots = torch.tensor([1 + b for b in order], dtype=torch.int32, device="cuda")
        if t == 2:   # the middle one (sequence 0) waits: its token comes behind the others'
            slots[1] = -1
        o = fv.attn_decay_step(q[idx, :, L + t], k[idx, :, L + t], v[idx, :, L + t], g, pool,
                               slots=slots)
        for i, b in enumerate(order):
            if t == 2 and b == 0:
                assert not o[i].any()
            elif b != 0 or t < 2:
                r = ref[b][0][0, :, n[b] + t]
                _near(o[i][None, :, None], r[None, :, None], mag[b][0][0, :, n[b] + t][None, :, None],
                      dk, L, dtype, (b, t))
    assert not pool[0].any() and not pool[4].any()
    for b in (1, 2):
        _near(pool[1 + b], ref[b][1][0], mag[b][1][0], dk, L, "f32", ("state", b))


@pytest.mark.parametrize("lengths", [None, [5000, 4097, 257, 0]])
def test_states_in_place(lengths):
    """state_out = state_in and dstate_in = dstate_out over many segments and one give what
    separate tensors give, bit for bit."""
    import torch
    fv = _fv()
    for L in (5000, 60):
        x = _inputs(4, 2, L, 64, 64, "bf16", 31)
        q, k, v, do = (to_dev(x[m], "bf16") for m in ("q", "k", "v", "do"))
        g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
        ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        o, st = fv.attn_decay(q, k, v, g, lengths=ln, state_in=S, return_state=True)
        want = fv.attn_decay_backward(q, k, v, g, do, lengths=ln, state_in=S, dstate_out=G,
                                      return_state_grad=True)
        for _ in range(3):
            s, d = S.clone(), G.clone()
            o2, s2 = fv.attn_decay(q, k, v, g, lengths=ln, state_in=s, return_state=True,
                                   state_out=s)
            assert s2 is s and torch.equal(o, o2) and torch.equal(st, s)
            got = fv.attn_decay_backward(q, k, v, g, do, lengths=ln, state_in=S, dstate_out=d,
                                         return_state_grad=True, dstate_in=d)
            assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_step_replays():
    """A training step and a decoding step captured once; every replay, with new contents in
    its buffers and the program's own work between, equals the eager calls."""
    import torch
    fv = _fv()
    B, H, L, dk, dv = 2, 3, 700, 128, 64
    x = _inputs(B, H, L, dk, dv, "bf16", 41)
    q, k, v, do = (to_dev(x[m], "bf16") for m in ("q", "k", "v", "do"))
    g, S, G = to_dev(x["g"]), to_dev(x["S"]), to_dev(x["G"])
    lens = torch.tensor([700, 300], dtype=torch.int32, device="cuda")
    rng = torch.tensor([3, 0], dtype=torch.int64, device="cuda")
    gd = fv.make_decay_desc(B, H, L, dk, dv, fv.BF16)
    n = fv.decay_workspace_size(gd), fv.decay_workspace_size(gd, True)

    def buffers():
        e = torch.empty_like
        return dict(out=e(v), so=e(S), y=e(v), dx=e(v), dQ=e(q), dK=e(k), dV=e(v), dS=e(S),
                    tok=torch.empty((B, H, dv), dtype=v.dtype, device="cuda"), pool=S.clone(),
                    ws=torch.empty(n[0], dtype=torch.uint8, device="cuda"),
                    wb=torch.empty(n[1], dtype=torch.uint8, device="cuda"))

    def step(b):
        fv.attn_decay(q, k, v, g, 0.5, lens, S, True, b["out"], b["so"], b["ws"])
        fv.dropout(b["out"], 0.3, rng=rng, residual=v, out=b["y"])
        fv.dropout(do, 0.3, rng=rng, out=b["dx"])
        fv.attn_decay_backward(q, k, v, g, b["dx"], 0.5, lens, S, G, True, b["dQ"], b["dK"],
                               b["dV"], b["dS"], b["wb"])
        fv.attn_decay_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], g, b["pool"], 0.5, out=b["tok"])

    cap, ref = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cap)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cap)
    torch.cuda.synchronize()
    for rep in range(4):
        new = _inputs(B, H, L, dk, dv, "bf16", 50 + rep)
        for t, m in ((q, "q"), (k, "k"), (v, "v"), (do, "do")):
            t.copy_(to_dev(new[m], "bf16"))
        for t, m in ((S, "S"), (G, "G"), (g, "g")):
            t.copy_(to_dev(new[m]))
        lens.copy_(torch.tensor([[700, 1], [0, 64], [513, 699], [700, 700]][rep],
                                dtype=torch.int32))
        rng[1] = rep
        for name in cap:
            if name not in ("pool", "ws", "wb"):
                cap[name].zero_()
                ref[name].zero_()
        cap["pool"].copy_(S)
        ref["pool"].copy_(S)
        step(ref)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in cap:
            if name not in ("ws", "wb"):
                assert torch.equal(cap[name], ref[name]), (rep, name)


def test_other_stream():
    """Calls on a stream of their own, behind work that stream still has to do."""
    import torch
    fv = _fv()
    x = _inputs(2, 4, 900, 64, 128, "bf16", 61)
    q, k, v, do = (to_dev(x[m], "bf16") for m in ("q", "k", "v", "do"))
    g, S = to_dev(x["g"]), to_dev(x["S"])
    want = [*fv.attn_decay(q, k, v, g, state_in=S, return_state=True),
            *fv.attn_decay_backward(q, k, v, g, do, state_in=S), fv.dropout(v, 0.5, 9)]
    s2 = S.clone()
    want += [fv.attn_decay_step(q[:, :, 1], k[:, :, 1], v[:, :, 1], g, s2), s2]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = [torch.zeros_like(t) for t in (q, k, v, do)]
    with torch.cuda.stream(side):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            big = big @ big * 1e-2
        for a, b in zip(late, (q, k, v, do)):
            a.copy_(b)
    ql, kl, vl, dl = late
    got = [*fv.attn_decay(ql, kl, vl, g, state_in=S, return_state=True, stream=side),
           *fv.attn_decay_backward(ql, kl, vl, g, dl, state_in=S, stream=side),
           fv.dropout(vl, 0.5, 9, stream=side)]
    s3 = S.clone()
    side.wait_stream(torch.cuda.current_stream())
    got += [fv.attn_decay_step(ql[:, :, 1], kl[:, :, 1], vl[:, :, 1], g, s3, stream=side), s3]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_most_heads():
    """65535 heads of one and of two tokens; one more is refused."""
    import torch
    fv = _fv()
    H = 65535
    q, k, v = (torch.randn(1, H, 2, 8, device="cuda") for _ in range(3))
    g = torch.full((H,), -0.5, device="cuda")
    out = fv.attn_decay(q, k, v, g)
    a = np.exp(np.float64(np.float32(-0.5)))
    w = (q @ k.transpose(-1, -2).contiguous()).double()
    want = torch.stack([w[:, :, 0, 0, None] * v[:, :, 0],
                        w[:, :, 1, 0, None] * a * v[:, :, 0] + w[:, :, 1, 1, None] * v[:, :, 1]], 2)
    assert (out.double() - want).abs().max() < 2e-4   # eight products of N(0, 1): < 64 * 2^-20
    grads = fv.attn_decay_backward(q, k, v, g, v)
    few = fv.attn_decay_backward(q[:, -64:], k[:, -64:], v[:, -64:], g[-64:], v[:, -64:])
    assert all(torch.equal(x[:, -64:], y) for x, y in zip(grads, few))
    with pytest.raises(fv.FavorError):
        z = torch.zeros(1, H + 1, 1, 8, device="cuda")
        fv.attn_decay(z, z, z, torch.zeros(H + 1, device="cuda"))
