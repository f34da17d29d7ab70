"""GPU parity of jf_token_logprobs and jf_token_logprobs_grad against
oracle/batch.py in 64 bits, and a run of the component calls together:
8-bit cache, attention, LM head, log probabilities.

Bounds.  With d = m - x and averages over the row's p: an exponential is off
by 2^-22 + d 2^-23 of itself (its argument's rounding and the function's two
units), a sum of n terms a thread and the joins by (n + 14) 2^-24, so log s is
off by e = 2^-22 + E[d] 2^-23 + (n + 14) 2^-24, plus its own rounding.
"""
import numpy as np
import pytest

from oracle import batch as ob

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tj():
    import torch
    from paper_2512_14681_amd import jf
    assert torch.cuda.is_available()
    return torch, jf


def stats(x):
    """(p, E[d], E[d^2]) of finite rows; zeros for the others."""
    with np.errstate(invalid="ignore"):
        m = x.max(1, keepdims=True)
        d = np.where(x > -np.inf, m - x, 0.0)
        w = np.where(x > -np.inf, np.exp(-d), 0.0)
        p = w / w.sum(1, keepdims=True)
        return p, (p * d).sum(1), (p * d * d).sum(1)


def device_rows(torch, x, dtype, pad, offset):
    R, V = x.shape
    buf = torch.full((R * (V + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:].view(R, V + pad)[:, :V]
    view.copy_(torch.tensor(x, dtype=torch.float64).to(dtype))
    return view


def run(tj, view, tokens, k, all_outputs=True):
    torch, jf = tj
    R, V = view.shape
    f = dict(dtype=torch.float32, device="cuda")
    lp, ent, norm, top = (torch.full(s, 9.0, **f) for s in ((R,), (R,), (R, 2), (R, k)))
    ids = torch.full((R, k), 9, dtype=torch.int32, device="cuda")
    ws = torch.full((jf.token_logprobs_ws_bytes(R, V, k),), 0xFF, dtype=torch.uint8, device="cuda")
    tok = torch.tensor(np.asarray(tokens, np.int32)).cuda()
    jf.token_logprobs(view, ws, d_tokens=tok, k=k, d_logprob=lp, d_entropy=ent, d_norm=norm, d_top_ids=ids,
                      d_top_logprob=top)
    return lp, ent, norm, ids, top, tok


def check(tj, x, tokens, k, dtype, pad=0, offset=0):
    torch, jf = tj
    view = device_rows(torch, x, dtype, pad, offset)
    x = view.double().cpu().numpy()
    R, V = x.shape
    got = [t.cpu().numpy() for t in run(tj, view, tokens, k)[:5]]
    with np.errstate(invalid="ignore"):
        want = ob.token_logprobs(x, tokens, k)
    assert np.array_equal(got[3], want[3])
    p, d1, d2 = stats(x)
    n = -(-V // 256)
    e = 2.0 ** -22 + d1 * 2.0 ** -23 + (n + 14) * 2.0 ** -24
    ls = np.nan_to_num(np.abs(want[2][:, 1]))
    tol_ls = e + ls * 2.0 ** -23
    # x - m and the difference round once each
    tol = lambda lp: tol_ls + 2 * np.nan_to_num(np.abs(lp), posinf=0, neginf=0) * 2.0 ** -24  # noqa: E731

    def close(a, b, t):
        same = np.isnan(b) == np.isnan(a)
        with np.errstate(invalid="ignore"):
            return same & (np.isnan(b) | (a == b) | (np.abs(a - b) <= t))
    assert close(got[0], want[0], tol(want[0])).all()
    # u / s: each term's d carries its own rounding, the sum's as above
    tol_u = d1 * (e + (n + 14) * 2.0 ** -24) + d2 * 2.0 ** -23 + d1 * 2.0 ** -22
    assert close(got[1], want[1], tol_ls + tol_u + np.nan_to_num(np.abs(want[1])) * 2.0 ** -23).all()
    assert close(got[2][:, 0], want[2][:, 0], 0).all()
    assert close(got[2][:, 1], want[2][:, 1], tol_ls).all()
    assert close(got[4], want[4], np.stack([tol(want[4][:, i]) for i in range(k)], 1) if k else 0).all()
    return view


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V,k", [(1, 1, 1), (3, 2, 5), (2, 17, 32), (5, 255, 8), (5, 256, 0), (4, 257, 1),
                                   (3, 4095, 20), (3, 4096, 20), (2, 4097, 32), (64, 1000, 5), (3, 50257, 20),
                                   (1, 152064, 32), (1100, 300, 3)])
def test_logprobs(tj, R, V, k, dtype):
    torch, jf = tj
    rng = np.random.default_rng([R, V])
    x = rng.normal(size=(R, V)) * 3
    tok = rng.integers(0, V, R)
    tok[rng.random(R) < 0.2] = -1
    for pad, offset in ((0, 0), (64 - V % 64, 0), (3, 1)):
        check(tj, x, tok, k, getattr(torch, dtype), pad, offset)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [40, 5000])
def test_masked_and_broken_rows(tj, V, dtype):
    torch, jf = tj
    rng = np.random.default_rng(V)
    x = rng.normal(size=(12, V))
    x[0] = -np.inf                                  # nothing left
    x[1, :] = -np.inf
    x[1, V - 3] = 2.0                               # one token left
    x[2, rng.random(V) < 0.9] = -np.inf
    x[3, 5] = np.nan
    x[4, V - 1] = np.inf
    x[5] = -np.inf
    x[5, 7] = np.nan
    x[6] = np.finfo(np.float32).min if dtype == "float32" else -3.3e38    # masks of the type's lowest value
    x[7, ::2] = -3.3e38
    x[8] += 10000.0                                 # a common offset
    x[9] = -1e30
    x[9, 3] = 0.0
    x[10] = 0.0
    tok = np.array([0, V - 3, 3, 5, 2, 7, 1, 1, 2, 3, V, -5])
    check(tj, x, tok, 8, getattr(torch, dtype))
    check(tj, x, tok, 32, getattr(torch, dtype), pad=1)


@pytest.mark.parametrize("order", ["equal", "rising", "falling", "few", "one lane"])
def test_ties_and_orders(tj, order):
    """Ties go to the lowest id; an ascending row replaces its alternatives all the time."""
    torch, jf = tj
    V = 9000
    x = {"equal": np.zeros(V), "rising": np.arange(V) / 16.0, "falling": -np.arange(V) / 16.0,
         "few": np.arange(V) % 3 * 1.0, "one lane": np.where(np.arange(V) % 256 == 5, 4.0, 0.0)}[order]
    x = np.stack([x, np.roll(x, 77)])
    check(tj, x, [1, V - 1], 32, torch.float32)
    check(tj, x, [1, V - 1], 7, torch.bfloat16, pad=3)


@pytest.mark.parametrize("k", [1, 8, 32])
def test_alternatives_over_many_steps(tj, k):
    """Rows that are not split: their best come from any step, from many, or are equal across steps."""
    rng = np.random.default_rng(k)
    R, V = 1024, 12388
    x = rng.integers(-8, 9, (R, V)) / 2.0  # many equal values
    x[::4] = rng.standard_normal((R // 4, V)) + np.arange(V) / 4096.0
    x[1::4] += 4.0 * (np.arange(V) // 4096 % 2)
    x[2::4, 4096:] -= 32.0
    x[3::8] = np.where(rng.random((R // 8, V)) < 0.001, x[3::8], -np.inf)
    check(tj, x, rng.integers(-1, V, R), k, tj[0].float32)


def test_outputs_are_optional(tj):
    torch, jf = tj
    x = torch.randn(5, 300, device="cuda")
    lp, ent, norm, ids, top, tok = run(tj, x, [1, 2, 3, 4, 5], 4)
    ws = torch.empty(jf.token_logprobs_ws_bytes(5, 300, 4), dtype=torch.uint8, device="cuda")
    for name, want in (("d_entropy", ent), ("d_norm", norm), ("d_top_ids", ids), ("d_top_logprob", top)):
        o = torch.zeros_like(want)
        jf.token_logprobs(x, ws, k=4, **{name: o})
        assert bool((o == want).all()), name
    o = torch.zeros_like(lp)
    jf.token_logprobs(x, ws, d_tokens=tok, d_logprob=o)
    assert bool((o == lp).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V,pad,offset", [(1, 1, 0, 0), (4, 257, 0, 0), (3, 4096, 0, 0), (3, 4099, 5, 1),
                                            (2, 50257, 47, 0), (70, 640, 0, 0)])
def test_gradient(tj, R, V, pad, offset, dtype):
    torch, jf = tj
    dt = getattr(torch, dtype)
    rng = np.random.default_rng([R, V, pad])
    x = rng.normal(size=(R, V)) * 3
    if V > 100:
        x[:, rng.random(V) < 0.2] = -np.inf
    tok = rng.integers(0, V, R)
    x[np.arange(R), tok] = 1.0
    g, h = rng.normal(size=R).astype(np.float32), rng.normal(size=R).astype(np.float32)
    if R > 2:
        tok[0] = -1
        g[1] = h[1] = 0.0
        h[2] = 0.0
    view = device_rows(torch, x, dt, pad, offset)
    x64 = view.double().cpu().numpy()
    lp, ent, norm, _, _, d_tok = run(tj, view, tok, 0)
    d_g, d_h = torch.tensor(g).cuda(), torch.tensor(h).cuda()
    out = device_rows(torch, np.full((R, V), 5.0), dt, pad, offset)
    jf.token_logprobs_grad(view, norm, out, d_tokens=d_tok, d_entropy=ent, d_g_logprob=d_g, d_g_entropy=d_h)
    got = out.double().cpu().numpy()
    want = ob.token_logprobs_grad(x64, tok, g.astype(np.float64), h.astype(np.float64))
    p, d1, d2 = stats(x64)
    n = -(-V // 256)
    e = 2.0 ** -22 + d1 * 2.0 ** -23 + (n + 14) * 2.0 ** -24
    ls = np.log(1 / p.max(1))
    tol_ls = (e + ls * 2.0 ** -23)[:, None]
    tol_h = tol_ls + (d1 * (e + (n + 14) * 2.0 ** -24) + d2 * 2.0 ** -23 + d1 * 2.0 ** -22)[:, None] + 2.0 ** -23 * (ls + d1)[:, None]
    a = np.where(p > 0, -np.log(np.where(p > 0, p, 1.0)), 0.0)           # -log p
    rel = tol_ls + a * 2.0 ** -22 + 2.0 ** -22                           # of p
    ga, ha = np.abs(g)[:, None], np.abs(h)[:, None]
    H = (p * a).sum(1, keepdims=True)
    bound = ga * p * (rel + 2.0 ** -22) + ha * p * (np.abs(H - a) * (rel + 2.0 ** -22) + tol_h + tol_ls + a * 2.0 ** -23)
    bound = bound + (np.finfo(np.float32).eps * 2 + (2.0 ** -8 if dtype == "bfloat16" else 0)) * np.abs(want) + 1e-37
    bound[np.arange(R), np.maximum(tok, 0)] += ga[:, 0] * 2.0 ** -23     # g - g p
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
    # in place, and without one of the two upstream gradients
    half = out.clone()
    jf.token_logprobs_grad(view, norm, half, d_tokens=d_tok, d_g_logprob=d_g)
    only_g = ob.token_logprobs_grad(x64, tok, g.astype(np.float64), np.zeros(R))
    assert (np.abs(half.double().cpu().numpy() - only_g) <= bound + (2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -22) * np.abs(only_g)).all()
    jf.token_logprobs_grad(view, norm, view, d_tokens=d_tok, d_entropy=ent, d_g_logprob=d_g, d_g_entropy=d_h)
    assert bool((view == out).all())


def test_gradient_of_special_rows(tj):
    """No upstream gradient: zeros, whatever the logits; a row that is no distribution: NaN; -inf: zero."""
    torch, jf = tj
    x = np.zeros((5, 100))
    x[0] = -np.inf
    x[1] = -np.inf
    x[2, 4] = np.nan
    x[3, ::2] = -np.inf
    tok = [1, 1, 1, 1, 200]
    view = device_rows(torch, x, torch.float32, 0, 0)
    lp, ent, norm, _, _, d_tok = run(tj, view, tok, 0)
    g = torch.tensor([0.0, 1.0, 1.0, 1.0, 1.0], device="cuda")
    h = torch.tensor([0.0, 1.0, 0.0, 1.0, 0.0], device="cuda")
    out = torch.full((5, 100), 5.0, device="cuda")
    jf.token_logprobs_grad(view, norm, out, d_tokens=d_tok, d_entropy=ent, d_g_logprob=g, d_g_entropy=h)
    o = out.cpu().numpy()
    assert (o[0] == 0).all() and np.isnan(o[1]).all() and np.isnan(o[2]).all() and np.isnan(o[4]).all()
    assert (o[3, ::2] == 0).all() and abs(o[3, 1] - (1 - 1 / 50)) < 2.0 ** -20 and abs(o[3, 3] + 1 / 50) < 2.0 ** -20


def test_rows_beyond_32_bit_offsets(tj):
    """Rows 2^31 + 8 elements apart, the gradient in place: what rows side by side give."""
    torch, jf = tj
    R, V, k, ld = 3, 5003, 5, (1 << 31) + 8
    x = torch.randn(R, V, device="cuda").to(torch.bfloat16)
    flat = torch.zeros((R - 1) * ld + V + 64, dtype=torch.bfloat16, device="cuda")
    far = flat.as_strided((R, V), (ld, 1))
    far.copy_(x)
    tok = torch.tensor([1, 5002, -1], dtype=torch.int32, device="cuda")
    g = torch.tensor([1.0, -2.0, 0.5], device="cuda")
    outs = []
    for t in (x, far):
        lp, ent, norm, ids, top, _ = run(tj, t, tok.cpu().numpy(), k)
        jf.token_logprobs_grad(t, norm, t, d_tokens=tok, d_entropy=ent, d_g_logprob=g, d_g_entropy=g)
        outs.append((lp, ent, norm, ids, top, t))
    for a, b in zip(*outs):
        assert bool((a == b).all())
    assert float(x.float().abs().sum()) > 0 and bool((flat[V:ld] == 0).all()) and bool((flat[-64:] == 0).all())


def test_captured(tj):
    """Both calls captured on a stream of their own, replayed with new logits between eager work."""
    torch, jf = tj
    R, V, k = 9, 20011, 6
    x, grad = torch.zeros(R, V, device="cuda"), torch.zeros(R, V, device="cuda")
    f = dict(dtype=torch.float32, device="cuda")
    lp, ent, norm, top = (torch.zeros(s, **f) for s in ((R,), (R,), (R, 2), (R, k)))
    ids = torch.zeros(R, k, dtype=torch.int32, device="cuda")
    tok = torch.arange(R, dtype=torch.int32, device="cuda") * 2000
    g = torch.ones(R, device="cuda")
    ws = torch.empty(jf.token_logprobs_ws_bytes(R, V, k), dtype=torch.uint8, device="cuda")

    def both():
        jf.token_logprobs(x, ws, d_tokens=tok, k=k, d_logprob=lp, d_entropy=ent, d_norm=norm, d_top_ids=ids,
                          d_top_logprob=top)
        jf.token_logprobs_grad(x, norm, grad, d_tokens=tok, d_entropy=ent, d_g_logprob=g, d_g_entropy=g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
        for i in range(4):
            x.copy_(torch.randn(R, V, device="cuda"))
            graph.replay()
            kept = [t.clone() for t in (lp, ent, norm, ids, top, grad)]
            both()
            torch.cuda.synchronize()
            assert all(bool((a == b).all()) for a, b in zip(kept, (lp, ent, norm, ids, top, grad)))


def test_run_together(tj):
    """Three sequences decode through an 8-bit cache: prompts appended, then steps of 1 to 4 rows, each
    attended, put through the LM head and scored, the last step's loss differentiated."""
    torch, jf = tj
    L = jf.lib()
    H, G, hd, V, B = 4, 2, 64, 512, 3
    d = H * hd
    rng = np.random.default_rng(77)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = np.array([[5, 0, 7], [2, 8, 4], [1, 6, 3]], np.int32)
    d_table = torch.tensor(table).cuda()
    raw = torch.zeros(9, jf.kv_page_bytes(G, hd, jf.JF_E4M3), dtype=torch.uint8, device="cuda")
    w = torch.tensor(rng.normal(size=(V, d)) * 0.05, dtype=torch.float32).to(torch.bfloat16).cuda()
    wp = torch.empty(L.jf_packed_matrix_bytes(V, d, jf.JF_BF16), dtype=torch.uint8, device="cuda")
    jf.check(L.jf_pack_matrix(V, d, jf.JF_BF16, jf._ptr(w), jf._ptr(wp), jf._stream()))
    ctx = np.zeros(B, np.int32)
    for step, rows in enumerate(([70, 3, 64], [1, 1, 1], [4, 1, 2], [1, 4, 1])):
        start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        R = int(start[-1])
        x = torch.tensor(rng.normal(size=(R, (H + 2 * G) * hd)), dtype=torch.float32).cuda()
        b = jf.Batch(torch.tensor(start).cuda(), torch.tensor(ctx).cuda(), d_table, R, max(rows), 192, 9)
        q = torch.empty(2, R, H, hd, dtype=torch.bfloat16, device="cuda")
        flags = torch.zeros(1, **i32)
        jf.kv_append(b, H, G, hd, jf.JF_E4M3, raw, x[:, d:d + G * hd], x[:, d + G * hd:], d_q=x[:, :d], d_q_out=q,
                     rope_base=1e4, d_flags=flags)
        out = torch.zeros(2, (R + 15) // 16 * 16 * d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(jf.attention_kv8_ws_bytes(b, H, G, hd), dtype=torch.uint8, device="cuda")
        jf.attention_kv8(b, H, G, hd, jf.JF_BF16, q, raw, out, ws, d_flags=flags)
        logits = torch.empty(R, V, device="cuda")
        am = torch.empty(R, **i32)
        lws = torch.empty(L.jf_lm_head_ws_bytes(R, V), dtype=torch.uint8, device="cuda")
        jf.check(L.jf_lm_head_accept(R, d, V, jf.JF_BF16, jf._ptr(out), jf._ptr(wp), None, jf._ptr(am), None,
                                     jf._ptr(logits), jf._ptr(lws), jf._stream()))
        tok = rng.integers(0, V, R)
        lp, ent, norm, ids, top, d_tok = run(tj, logits, tok, 4)
        assert int(flags) == 0 and bool((ids[:, 0] == am).all())
        # the oracle on what the cache holds (its rounding is pinned by the append's own tests)
        pool = ob.Pool8(raw.cpu().numpy(), G, hd)
        q64 = ob.rotate(x[:, :d].double().cpu().numpy().reshape(R, H, hd),
                        np.concatenate([c + np.arange(n) for c, n in zip(ctx, rows)]), 1e4)
        o = np.concatenate([ob.attention(q64[start[s]:start[s + 1]], ob.gather(pool, table[s], ctx[s] + rows[s], G, 0),
                                         ob.gather(pool, table[s], ctx[s] + rows[s], G, 1), ctx[s],
                                         np.tril(np.ones((rows[s],) * 2, bool))) for s in range(B)])
        z = o.reshape(R, d) @ w.double().cpu().numpy().T
        # 16-bit activations on values below 5: 2^-16 * 5 * sum |w| over d = 256 terms of 0.05
        assert np.abs(logits.double().cpu().numpy() - z).max() <= 2.0 ** -16 * 5 * 256 * 0.05 * 2
        wlp, went, *_ = ob.token_logprobs(logits.double().cpu().numpy(), tok, 4)
        assert np.abs(lp.cpu().numpy() - wlp).max() <= 2.0 ** -18 and np.abs(ent.cpu().numpy() - went).max() <= 2.0 ** -17
        ctx = ctx + np.array(rows, np.int32)
    g = torch.full((R,), -1.0 / R, device="cuda")
    jf.token_logprobs_grad(logits, norm, logits, d_tokens=d_tok, d_g_logprob=g)
    assert abs(float(logits.double().sum())) <= 2.0 ** -20 * R      # a softmax's gradient sums to nothing


def test_decoder_scores(tj):
    """Decoder.score against the oracle's decoder: greedy tokens are its best alternatives, and a forced
    continuation in several steps has the log probabilities of the oracle's logits."""
    torch, jf = tj
    import jf_inputs
    from oracle import jacobi as ojac
    from oracle.model import DecoderOracle
    from paper_2512_14681_amd import decode
    shape = jf_inputs.MODEL_SHAPES["tiny"]
    w = jf_inputs.model_weights(shape, seed=0)
    prompt = jf_inputs.prompt(1, 20, shape["vocab"])
    toks = jf_inputs.token_ids(9, 1, 21, shape["vocab"])
    dec = decode.Decoder(jf.Model(shape, w, max_rows=8, max_ctx=128))
    lp, ent, ids, top = dec.score(prompt, toks, k=3)
    assert dec.length() == len(prompt) + len(toks) - 1
    back = ojac.TransformerBackend(DecoderOracle(shape, w))
    back.prefill(list(prompt[:-1]))
    feed = [int(prompt[-1])] + [int(t) for t in toks[:-1]]
    back.step(feed, ojac.linear_segments(len(feed)))
    z = np.asarray(back.last[1], np.float64)
    wlp, went, _, wids, wtop = ob.token_logprobs(z, toks, 3)
    # fp32 logits of the tiny decoder are within 2^-12 of the oracle's
    assert np.abs(lp - wlp).max() <= 2.0 ** -11 and np.abs(ent - went).max() <= 2.0 ** -11
    assert np.abs(top - wtop).max() <= 2.0 ** -11
    with pytest.raises(ValueError):
        dec.score(prompt[:1], toks)
