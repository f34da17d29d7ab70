"""The component operators around the engine: a paged key/value cache that is appended to and read back, attention over
such a cache in 8 bits, and the log probabilities of tokens with their gradient.

Each case is one pass through one of them, as a program that serves or trains a model calls it.  Where ``own`` is false
``run`` computes the same in elementary torch operations.  All inputs are made on the GPU from the seed; how long each
sequence is belongs to the case.
"""
import math
import random

import torch

own = False

# Attention dimensions (query heads, KV heads, head_dim, RoPE base) of the repository's decoder shapes.
DIMS = {
    "7b": (28, 4, 128, 1e6),     # the benchmark's decoder shape
    "mid": (16, 4, 128, 1e6),    # the mid-size bf16 decoder of the tests
    "small": (16, 2, 64, 1e4),   # generic: head_dim 64
    "tiny": (4, 4, 32, 1e4),     # the tests' fp32 decoder: every query head has keys of its own
}
PAGE = 64            # tokens of a cache page
F8_MAX = 448.0       # largest e4m3 value
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # One token of one sequence into a bf16 cache: the smallest call, launch and host time.
        {"name": "append_rows1", "kind": "append", "dims": "7b", "kv": "bf16", "x": "f32", "act": "bf16", "seqs": 1,
         "ctx": 1000, "rows": 1, "tree": False},
        # One decoding step of 64 sequences of ragged lengths into an 8-bit cache.
        {"name": "append_e4m3_batch64", "kind": "append", "dims": "7b", "kv": "e4m3", "x": "bf16", "act": "f32",
         "seqs": 64, "ctx": 4000, "rows": 1, "tree": False},
        # The prompts of five sequences behind a shared-length history, ragged, into an 8-bit cache.
        {"name": "append_e4m3_prefill", "kind": "append", "dims": "mid", "kv": "e4m3", "x": "f32", "act": "f32",
         "seqs": 5, "ctx": 700, "rows": 4001, "tree": False},
        # One row over 1024 keys: greedy decoding of one sequence, where latency counts.
        {"name": "attention_rows1", "kind": "attention", "dims": "7b", "act": "bf16", "seqs": 1, "ctx": 1024,
         "rows": 1, "tree": False},
        # One decoding step of 64 sequences of up to 8192 tokens: the cache is the traffic.
        {"name": "attention_batch64", "kind": "attention", "dims": "7b", "act": "bf16", "seqs": 64, "ctx": 8191,
         "rows": 1, "tree": False},
        # A multi-block step: 192 rows under a tree mask after 2048 tokens.
        {"name": "attention_tree192", "kind": "attention", "dims": "7b", "act": "bf16", "seqs": 1, "ctx": 2048,
         "rows": 192, "tree": True},
        # A prefill chunk of 512 rows behind a long prompt: bound by the matrix cores.
        {"name": "attention_rows512", "kind": "attention", "dims": "7b", "act": "bf16", "seqs": 1, "ctx": 8000,
         "rows": 512, "tree": False},
        # Draft blocks of 13 rows in five sequences of a small decoder, activations in fp32, tree masks.
        {"name": "attention_small_f32", "kind": "attention", "dims": "small", "act": "f32", "seqs": 5, "ctx": 777,
         "rows": 13, "tree": True},
        # One row of logits at the full vocabulary, with the 20 best alternatives: a served token.
        {"name": "logprobs_rows1", "kind": "logprobs", "x": "f32", "rows": 1, "vocab": 152064, "k": 20,
         "masked": False},
        # The rows of a 64-token window in bf16, a part of the vocabulary masked out, 8 alternatives.
        {"name": "logprobs_rows64_bf16", "kind": "logprobs", "x": "bf16", "rows": 64, "vocab": 152064, "k": 8,
         "masked": True},
        # The logits of a packed training sequence: log probabilities, entropies and their gradient.
        {"name": "loss_rows512", "kind": "loss", "x": "f32", "rows": 512, "vocab": 152064, "masked": False},
        # A small training batch in bf16 over an odd vocabulary, with padded rows.
        {"name": "loss_rows48_odd", "kind": "loss", "x": "bf16", "rows": 48, "vocab": 50257, "masked": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attention", "attention", "attention", "logprobs", "logprobs", "loss"])
    if kind in ("logprobs", "loss"):
        c = {"kind": kind, "x": rng.choice(["f32", "bf16"]), "rows": _log_int(rng, 1, 400),
             "vocab": _log_int(rng, 1000, 152064), "masked": rng.random() < 0.4}
        if kind == "logprobs":
            c["k"] = rng.choice([0, 1, 5, 8, 20, 32])
        return c
    c = {"kind": kind, "dims": rng.choice(["7b", "7b", "mid", "small", "tiny"]), "seqs": _log_int(rng, 1, 64)}
    if kind == "append":
        c["kv"] = rng.choice(["f32", "bf16", "e4m3", "e4m3"])
        c["x"], c["act"] = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
        c["ctx"] = _log_int(rng, 1, 8000)
        c["rows"] = _log_int(rng, 1, max(1, min(4000, 12000 // c["seqs"])))
        c["tree"] = rng.random() < 0.3
        return c
    c["act"] = "f32" if rng.random() < 0.25 else "bf16"
    c["ctx"] = _log_int(rng, 1, min(131072, 262144 // c["seqs"]))
    most = min(512, (1 << 22) // (c["seqs"] * max(c["ctx"], 512)))
    c["rows"] = _log_int(rng, 1, max(1, most))
    c["tree"] = rng.random() < 0.4
    return c


# ---- lengths --------------------------------------------------------------------------
def _lengths(case):
    """(committed tokens, rows) of each sequence: the first has the case's, the others down to a quarter of them."""
    rng = random.Random(case["seqs"] * 1000003 + case["ctx"] * 1009 + case["rows"])
    n = case["seqs"]
    ctx = [case["ctx"]] + [rng.randint(case["ctx"] // 4, case["ctx"]) for _ in range(n - 1)]
    rows = [case["rows"]] + [rng.randint((case["rows"] + 3) // 4, case["rows"]) for _ in range(n - 1)]
    return ctx, rows


def _starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def _parents(n, tree):
    """A row's parent among its sequence's rows: a chain, or half a chain and branches of 8 under the first row."""
    half = (n + 1) // 2
    if not tree:
        return list(range(-1, n - 1))
    return [i - 1 if i < half or (i - half) % 8 else (0 if i else -1) for i in range(n)]


def _depths(n, tree):
    out = []
    for i, p in enumerate(_parents(n, tree)):
        out.append(0 if p < 0 else out[p] + 1)
    return out


def _visible(n, tree):
    """[n][n] bool: a row sees its ancestors and itself."""
    vis = torch.zeros(n, n, dtype=torch.bool)
    for i, p in enumerate(_parents(n, tree)):
        if p >= 0:
            vis[i] = vis[p]
        vis[i, i] = True
    return vis


# ---- inputs ---------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _page_table(case, seed):
    """(page table [seqs][stride] int32, physical pages): every sequence's pages, scattered over the pool."""
    ctx, rows = _lengths(case)
    need = [(c + r + PAGE - 1) // PAGE for c, r in zip(ctx, rows)]
    total = sum(need) + 3
    perm = torch.randperm(total, device="cuda", generator=_gen(seed, 1)).to(torch.int32)
    table = torch.zeros(len(need), max(need), dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n]
        at += n
    return table, total


def _page_bytes(G, hd):
    """An e4m3 page: codes of the keys, codes of the values, a scale of each for every head; a multiple of 128."""
    return (2 * G * PAGE * hd + 8 * G + 127) // 128 * 128


def _random_pool(case, seed, n_pages):
    """The cache before the call: what earlier calls left in it."""
    _, G, hd, _ = DIMS[case["dims"]]
    g = _gen(seed, 2)
    if case["kv"] != "e4m3":
        return _normal(g, n_pages, 2 * G * PAGE * hd, dtype=TYPES[case["kv"]])
    pool = torch.zeros(n_pages, _page_bytes(G, hd), dtype=torch.uint8, device="cuda")
    n = 2 * G * PAGE * hd
    codes = torch.randint(0, 256, (n_pages, n), dtype=torch.uint8, device="cuda", generator=g)
    pool[:, :n] = torch.where((codes & 0x7F) == 0x7F, codes - 64, codes)
    exps = torch.randint(-9, -4, (n_pages, 2 * G), device="cuda", generator=g)
    pool[:, n:n + 8 * G] = torch.exp2(exps.float()).view(torch.uint8)
    return pool


def _append_inputs(case, seed):
    """Rows of a fused projection, [R][(H + 2 G) hd]: queries, keys, values."""
    H, G, hd, _ = DIMS[case["dims"]]
    return _normal(_gen(seed, 3), _starts(_lengths(case)[1])[-1], (H + 2 * G) * hd, dtype=TYPES[case["x"]])


def _quantise(x):
    """[pages][64][G][hd] -> (e4m3 codes of x / scale, power-of-two scales [pages][G])."""
    amax = x.abs().amax((1, 3))
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(amax > 0, amax / F8_MAX, 1.0))))
    return (x / scale[:, None, :, None]).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn), scale


def _planes(x, act):
    """An fp32 tensor as activation planes: hi and lo bf16, or one fp32 plane."""
    if act == "f32":
        return x[None]
    hi = x.to(torch.bfloat16)
    return torch.stack([hi, (x - hi.float()).to(torch.bfloat16)])


def _attention_inputs(case, seed):
    """(q planes [P][R][H][hd], (K codes, K scales, V codes, V scales) by physical page, page table)."""
    H, G, hd, _ = DIMS[case["dims"]]
    table, n_pages = _page_table(case, seed)
    g = _gen(seed, 4)
    R = _starts(_lengths(case)[1])[-1]
    q = _planes(_normal(g, R, H, hd, std=2.0), case["act"]).contiguous()
    pages = []
    for _ in range(2):
        codes, scales = _quantise(_normal(g, n_pages, PAGE, G, hd))
        pages += [codes, scales]
    return q, pages, table


def _pack_keys(x):
    """[N][64][G][hd] one-byte keys in the page's order: [G][hd / 16][64 lanes][16], lane = t % 16 + 16 (dim / (hd / 4)),
    byte 16 n + e of a lane = (t / 16) (hd / 4) + dim % (hd / 4)."""
    N, _, G, hd = x.shape
    x = x.reshape(N, 4, 16, G, 4, hd // 4).permute(0, 3, 1, 5, 4, 2).reshape(N, G, hd // 16, 16, 4, 16)
    return x.permute(0, 1, 2, 4, 5, 3).reshape(N, -1)


def _unpack_keys(x, G, hd):
    N = x.shape[0]
    x = x.reshape(N, G, hd // 16, 4, 16, 16).permute(0, 1, 2, 5, 3, 4).reshape(N, G, 4, hd // 4, 4, 16)
    return x.permute(0, 2, 5, 1, 4, 3).reshape(N, PAGE, G, hd)


def _pack_values(x):
    """[N][64][G][hd] one-byte values in the page's order: [G][hd / 16][64 lanes][16], lane = dim % 16 + 16 ((t / 4) % 4),
    byte 4 (t / 16) + t % 4 of piece dim / 16."""
    N, _, G, hd = x.shape
    return x.reshape(N, 4, 4, 4, G, hd // 16, 16).permute(0, 4, 5, 2, 6, 1, 3).reshape(N, -1)


def _unpack_values(x, G, hd):
    N = x.shape[0]
    return x.reshape(N, G, hd // 16, 4, 16, 4, 4).permute(0, 5, 3, 6, 1, 2, 4).reshape(N, PAGE, G, hd)


def _pack_pool(kc, ks, vc, vs):
    N, _, G, hd = kc.shape
    n = G * PAGE * hd
    pool = torch.zeros(N, _page_bytes(G, hd), dtype=torch.uint8, device=kc.device)
    pool[:, :n] = _pack_keys(kc.view(torch.uint8))
    pool[:, n:2 * n] = _pack_values(vc.view(torch.uint8))
    pool[:, 2 * n:2 * n + 8 * G] = torch.stack([ks, vs], 2).reshape(N, -1).view(torch.uint8)
    return pool


def _vis_words(case):
    """[R][8] 64-bit words: bit j of a row's mask is the j-th row of its sequence."""
    rows = _lengths(case)[1]
    bits = torch.zeros(sum(rows), 512, dtype=torch.bool)
    at, seen = 0, {}
    for n in rows:
        if n not in seen:
            seen[n] = _visible(n, case["tree"])
        bits[at:at + n, :n] = seen[n]
        at += n
    weights = (torch.ones(64, dtype=torch.int64) << torch.arange(64)).view(1, 1, 64)
    return (bits.view(-1, 8, 64).long() * weights).sum(2).contiguous().cuda()


def _logits(case, seed):
    """Logits of spread 2.5; rows on a stride that is longer than the vocabulary, every seventh one masked in part."""
    g, R, V = _gen(seed, 5), case["rows"], case["vocab"]
    x = _normal(g, R, (V + 63) // 64 * 64, std=2.5).to(TYPES[case["x"]])
    if case["masked"]:
        x[torch.rand(x.shape, device="cuda", generator=g) < 0.3] = -math.inf
    tokens = torch.randint(0, V, (R,), device="cuda", generator=g, dtype=torch.int32)
    tokens[torch.rand(R, device="cuda", generator=g) < 0.1] = -1    # rows without a token
    x[torch.arange(R, device="cuda"), tokens.clamp(min=0).long()] = 6.0
    return x[:, :V], tokens


def prepare(case, seed):
    s = {"case": case}
    if case["kind"] in ("logprobs", "loss"):
        R, V = case["rows"], case["vocab"]
        s["x"], s["tokens"] = _logits(case, seed)
        s["logprob"], s["entropy"] = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
        s["norm"] = torch.zeros(R, 2, device="cuda")     # a row's maximum, and the logarithm of its sum relative to it
        if case["kind"] == "loss":
            g = _gen(seed, 6)
            s["g_logprob"], s["g_entropy"] = _normal(g, R), _normal(g, R, std=0.1)
            s["grad"] = torch.zeros(R, V, dtype=TYPES[case["x"]], device="cuda")
        else:
            s["top_ids"] = torch.zeros(R, case["k"], dtype=torch.int32, device="cuda")
            s["top_logprob"] = torch.zeros(R, case["k"], device="cuda")
        return s
    H, G, hd, _ = DIMS[case["dims"]]
    ctx, rows = _lengths(case)
    start = _starts(rows)
    R = start[-1]
    s["table"], s["n_pages"] = _page_table(case, seed)
    s["ctx"], s["start"], s["flags"] = _ints(ctx), _ints(start), _ints([0])
    if case["kind"] == "attention":
        q, pages, _ = _attention_inputs(case, seed)
        s["q"], s["kv"] = q, _pack_pool(*pages)
        s["vis"] = _vis_words(case) if case["tree"] else None
        s["out"] = torch.zeros(q.shape[0], (R + 15) // 16 * 16 * H * hd, dtype=q.dtype, device="cuda")
        return s
    x = _append_inputs(case, seed)
    s["q"], s["k"], s["v"] = x[:, :H * hd], x[:, H * hd:(H + G) * hd], x[:, (H + G) * hd:]
    s["kv"] = _random_pool(case, seed, s["n_pages"])
    act = TYPES[case["act"]]
    s["q_out"] = torch.zeros(2 if case["act"] == "bf16" else 1, R, H, hd, dtype=act, device="cuda")
    # draft rows of a tree share positions: the depth below the committed tokens
    s["pos"] = _ints([c + d for c, n in zip(ctx, rows) for d in _depths(n, True)]) if case["tree"] else None
    if case["kv"] == "e4m3":
        # the blocks that the call writes into, read back from their first token on
        s["ctx0"] = _ints([c // PAGE * PAGE for c in ctx])
        back = _starts([c % PAGE + n for c, n in zip(ctx, rows)])
        s["start0"], s["back"] = _ints(back), back[-1]
        s["k_back"], s["v_back"] = (torch.zeros(back[-1], G * hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


# ---- one pass -------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"append": _own_append, "attention": _own_attention}.get(kind, _own_logprobs)(s)
    return {"append": _plain_append, "attention": _plain_attention}.get(kind, _plain_logprobs)(s)


def _own_batch(s, key="batch", ctx="ctx", start="start", n_rows=None):
    """The batch's descriptor, made at the first pass as a program makes it when its buffers are."""
    if key not in s:
        from paper_2512_14681_amd import jf
        lens, rows = _lengths(s["case"])
        extra = PAGE if key != "batch" else 0
        s[key] = jf.Batch(s[start], s[ctx], s["table"], n_rows or sum(rows), max(rows) + extra,
                          max(c + n for c, n in zip(lens, rows)), s["n_pages"])
    return s[key]


def _own_append(s):
    from paper_2512_14681_amd import jf
    c = s["case"]
    H, G, hd, base = DIMS[c["dims"]]
    kv = {"f32": jf.JF_F32, "bf16": jf.JF_BF16, "e4m3": jf.JF_E4M3}[c["kv"]]
    act = jf.JF_F32 if c["act"] == "f32" else jf.JF_BF16
    jf.kv_append(_own_batch(s), H, G, hd, kv, s["kv"], s["k"], s["v"], d_q=s["q"], d_q_out=s["q_out"], act_dtype=act,
                 d_pos=s["pos"], rope_base=base, d_flags=s["flags"])
    q = s["q_out"][0] if c["act"] == "f32" else torch.sum(s["q_out"], 0, dtype=torch.float32)
    if c["kv"] != "e4m3":
        return [q, s["kv"]]
    back = _own_batch(s, "batch0", "ctx0", "start0", s["back"])
    jf.kv_read(back, G, hd, kv, s["kv"], s["k_back"], s["v_back"], d_flags=s["flags"])
    return [q, s["k_back"], s["v_back"]]


def _own_attention(s):
    from paper_2512_14681_amd import jf
    c = s["case"]
    H, G, hd, _ = DIMS[c["dims"]]
    b = _own_batch(s)
    if "ws" not in s:
        s["ws"] = torch.empty(jf.attention_kv8_ws_bytes(b, H, G, hd), dtype=torch.uint8, device="cuda")
    jf.attention_kv8(b, H, G, hd, jf.JF_F32 if c["act"] == "f32" else jf.JF_BF16, s["q"], s["kv"], s["out"], s["ws"],
                     d_vis=s["vis"], d_flags=s["flags"])
    # the value the planes stand for
    return [s["out"][0] if c["act"] == "f32" else torch.sum(s["out"], 0, dtype=torch.float32)]


def _own_logprobs(s):
    from paper_2512_14681_amd import jf
    c = s["case"]
    k = c.get("k", 0)
    if "ws" not in s:
        s["ws"] = torch.empty(jf.token_logprobs_ws_bytes(c["rows"], c["vocab"], k), dtype=torch.uint8, device="cuda")
    if c["kind"] == "loss":
        jf.token_logprobs(s["x"], s["ws"], d_tokens=s["tokens"], d_logprob=s["logprob"], d_entropy=s["entropy"],
                          d_norm=s["norm"])
        jf.token_logprobs_grad(s["x"], s["norm"], s["grad"], d_tokens=s["tokens"], d_entropy=s["entropy"],
                               d_g_logprob=s["g_logprob"], d_g_entropy=s["g_entropy"])
        return [s["logprob"], s["entropy"], s["grad"]]
    jf.token_logprobs(s["x"], s["ws"], d_tokens=s["tokens"], k=k, d_logprob=s["logprob"], d_entropy=s["entropy"],
                      d_norm=s["norm"], d_top_ids=s["top_ids"], d_top_logprob=s["top_logprob"])
    return [s["logprob"], s["entropy"], s["norm"], s["top_ids"], s["top_logprob"]]


# ---- the plain forms ------------------------------------------------------------------
def _slots(s):
    """Of every row: its sequence, its slot in that sequence and its physical page."""
    start, ctx, R = s["start"].long(), s["ctx"].long(), s["k" if "k" in s else "q"].shape[-3 if "out" in s else 0]
    r = torch.arange(R, device="cuda")
    seq = torch.searchsorted(start[1:], r, right=True)
    slot = ctx[seq] + r - start[seq]
    return seq, slot, s["table"].long()[seq, slot // PAGE]


def _rotate(x, cs, sn):
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)


def _plain_append(s):
    c = s["case"]
    H, G, hd, base = DIMS[c["dims"]]
    seq, slot, page = _slots(s)
    R = len(slot)
    pos = slot if s["pos"] is None else s["pos"].long()
    ang = pos[:, None].double() * base ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    cs, sn = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    q = _rotate(s["q"].float().reshape(R, H, hd), cs, sn)
    k = _rotate(s["k"].float().reshape(R, G, hd), cs, sn)
    v = s["v"].float().reshape(R, G, hd)
    q = _planes(q, c["act"]).to(torch.float32).sum(0)
    if c["kv"] != "e4m3":
        pool, t = s["kv"], slot % PAGE
        keys = pool[:, :G * PAGE * hd].view(-1, G, PAGE, hd)
        values = pool[:, G * PAGE * hd:].view(-1, G, hd, PAGE)
        keys[page, :, t] = k.to(pool.dtype)
        values[page, :, :, t] = v.to(pool.dtype)
        return [q, pool]
    # the pages written into, each with the tokens it keeps (slots below the committed length) and its new ones
    touched, which = torch.unique(page, return_inverse=True)
    N, t = len(touched), slot % PAGE
    block = torch.zeros(N, dtype=torch.int64, device="cuda")
    block[which] = slot // PAGE * PAGE
    owner = torch.zeros(N, dtype=torch.int64, device="cuda")
    owner[which] = seq
    kept = (s["ctx"].long()[owner] - block).clamp(0, PAGE)
    old = s["kv"][touched]
    n = G * PAGE * hd
    scales = old[:, 2 * n:2 * n + 8 * G].contiguous().view(torch.float32).view(N, G, 2)
    keep = torch.arange(PAGE, device="cuda") < kept[:, None]
    fresh = torch.zeros(N, PAGE, dtype=torch.bool, device="cuda")
    fresh[which, t] = True
    new = old.clone()
    outs = []
    for i, (rows, unpack, pack) in enumerate(((k, _unpack_keys, _pack_keys), (v, _unpack_values, _pack_values))):
        codes = unpack(old[:, i * n:(i + 1) * n].contiguous().view(torch.float8_e4m3fn), G, hd).float()
        x = torch.zeros(N, PAGE, G, hd, device="cuda")
        x[which, t] = rows
        amax = x.abs().amax((1, 3))
        need = torch.exp2(torch.ceil(torch.log2(torch.where(amax > 0, amax / F8_MAX, 1.0))))
        sc = torch.where(kept[:, None] > 0, torch.maximum(need, scales[:, :, i]), need)
        x = torch.where(fresh[:, :, None, None], x, codes * scales[:, None, :, i, None])
        q8 = (x / sc[:, None, :, None]).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn)
        was = unpack(old[:, i * n:(i + 1) * n].contiguous(), G, hd)
        q8 = torch.where((fresh | keep)[:, :, None, None], q8.view(torch.uint8), was)
        new[:, i * n:(i + 1) * n] = pack(q8)
        new[:, 2 * n:2 * n + 8 * G].view(N, G, 2, 4)[:, :, i] = sc.contiguous().view(torch.uint8).view(N, G, 4)
        outs.append(q8.view(torch.float8_e4m3fn).float() * sc[:, None, :, None])
    s["kv"][touched] = new
    # back from the blocks' first tokens on, sequence by sequence
    start0 = s["start0"].long()
    r = torch.arange(s["back"], device="cuda")
    sq = torch.searchsorted(start0[1:], r, right=True)
    at = s["ctx0"].long()[sq] + r - start0[sq]
    index = torch.searchsorted(touched, s["table"].long()[sq, at // PAGE])
    return [q] + [o[index, at % PAGE].reshape(len(r), G * hd).to(torch.bfloat16) for o in outs]


def _gemm_layout(x):
    """[R][K] in the GEMM-input layout of include/jf.h: rows padded to 16 with zeros, 16 x 128 blocks in matrix-core order."""
    R, K = x.shape
    x = torch.nn.functional.pad(x, (0, 0, 0, -R % 16)).reshape(-1, 16, K // 128, 4, 4, 8)
    return x.permute(0, 2, 4, 3, 1, 5).reshape(-1)


def _plain_attention(s):
    c = s["case"]
    H, G, hd, _ = DIMS[c["dims"]]
    n, B = G * PAGE * hd, c["seqs"]
    start, ctx = s["start"].long(), s["ctx"].long()
    seq, _, _ = _slots(s)
    R, most = len(seq), c["rows"]
    # every sequence's cache, padded to the longest
    table = s["table"].long()
    T = table.shape[1] * PAGE
    pages = s["kv"][table.reshape(-1)]
    sc = pages[:, 2 * n:2 * n + 8 * G].contiguous().view(torch.float32).view(-1, 1, G, 2)
    keys = _unpack_keys(pages[:, :n].contiguous().view(torch.float8_e4m3fn), G, hd).float() * sc[..., 0, None]
    values = _unpack_values(pages[:, n:2 * n].contiguous().view(torch.float8_e4m3fn), G, hd).float() * sc[..., 1, None]
    keys, values = (x.reshape(B, T, G, hd).transpose(1, 2) for x in (keys, values))
    # the rows, padded to the longest sequence's
    within = torch.arange(R, device="cuda") - start[seq]
    q = torch.zeros(B, most, H, hd, device="cuda")
    q[seq, within] = s["q"].float().sum(0)
    q = q.view(B, most, G, H // G, hd).permute(0, 2, 3, 1, 4).reshape(B, G, -1, hd)
    j = torch.arange(T, device="cuda")
    own_row = j - ctx[:, None]                                   # [B][T]: the in-step row in that slot
    if s["vis"] is None:
        seen = own_row[:, None] <= torch.arange(most, device="cuda")[None, :, None]
    else:
        words = torch.zeros(B, most, 8, dtype=torch.int64, device="cuda")
        words[seq, within] = s["vis"]
        o = own_row.clamp(0, 511)
        bits = torch.gather(words, 2, (o // 64)[:, None].expand(B, most, T)) >> (o % 64)[:, None] & 1
        seen = (bits == 1) & (own_row[:, None] >= 0) | (own_row[:, None] < 0)
    seen &= own_row[:, None] < (start[1:] - start[:-1])[:, None, None]
    scores = torch.matmul(q, keys.transpose(2, 3).contiguous()) / math.sqrt(hd)
    scores = scores.view(B, G, H // G, most, T).masked_fill_(~seen[:, None, None], -math.inf)
    scores = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    total = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores.view(B, G, -1, T), values.contiguous()).view(B, G, H // G, most, hd)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, most, H * hd)[seq, within]
    return [_planes(_gemm_layout(o), c["act"]).to(torch.float32).sum(0)]


def _plain_logprobs(s):
    c = s["case"]
    x, tok = s["x"].float(), s["tokens"].long()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    p = e / total
    norm = torch.cat([m, torch.log(total)], 1)
    lp = x - m - norm[:, 1:]
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    logprob = torch.where(tok >= 0, lp.gather(1, tok.clamp(min=0)[:, None])[:, 0], 0.0)
    if c["kind"] == "loss":
        hot = torch.arange(c["vocab"], device="cuda")[None] == tok[:, None]
        g = s["g_logprob"][:, None] * torch.where(tok[:, None] >= 0, hot.float() - p, 0.0)
        g -= s["g_entropy"][:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
        return [logprob, entropy, g.to(s["x"].dtype)]
    best, ids = torch.sort(x, dim=1, descending=True, stable=True)    # ties: the lowest index first
    k = c["k"]
    return [logprob, entropy, norm, ids[:, :k].to(torch.int32), best[:, :k] - m - norm[:, 1:]]


# ---- what a pass cannot do without ----------------------------------------------------
def work(case):
    if case["kind"] in ("logprobs", "loss"):
        R, V, e = case["rows"], case["vocab"], 2 if case["x"] == "bf16" else 4
        by = R * V * e + R * 16 + R * case.get("k", 0) * 8
        if case["kind"] == "loss":      # the logits again, now that their sums are known, and the gradient
            return {"bytes": by + 2 * R * V * e, "flops": 10.0 * R * V}
        return {"bytes": by, "flops": 5.0 * R * V}
    H, G, hd, _ = DIMS[case["dims"]]
    ctx, rows = _lengths(case)
    R = sum(rows)
    if case["kind"] == "attention":
        pairs = sum(n * c + int(_visible(n, case["tree"]).sum()) for c, n in zip(ctx, rows))
        cache = sum(c + n for c, n in zip(ctx, rows)) * G * hd * 2
        return {"bytes": cache + R * H * hd * 8, "flops": 4 * H * hd * pairs}
    e, ex = {"f32": 4, "bf16": 2, "e4m3": 1}[case["kv"]], 4 if case["x"] == "f32" else 2
    by = R * (H + 2 * G) * hd * ex + R * H * hd * 4 + R * 2 * G * hd * e
    if case["kv"] == "e4m3":            # the blocks written into, read back
        by += sum(c % PAGE + n for c, n in zip(ctx, rows)) * 2 * G * hd * (1 + 2)
    return {"bytes": by, "flops": 6.0 * R * (H + G) * hd}


# ---- the same in 64 bits --------------------------------------------------------------
def _round_e4m3(x):
    """To the nearest value that an e4m3 number can have (3 bits behind the point, exponents from -6 on), ties to even."""
    _, e = torch.frexp(x.clamp(-F8_MAX, F8_MAX))
    step = torch.ldexp(torch.ones_like(x), (e - 4).clamp(min=-9))
    return torch.round(x.clamp(-F8_MAX, F8_MAX) / step) * step


def _block_scale(top):
    """The smallest power of two that brings `top` down to the largest e4m3 value."""
    m, e = math.frexp(top / F8_MAX)
    return 1.0 if top == 0 else math.ldexp(1.0, e - 1 if m == 0.5 else e)


def _exact_append(case, seed):
    f64 = torch.float64
    H, G, hd, base = DIMS[case["dims"]]
    ctx, rows = _lengths(case)
    start = _starts(rows)
    table, n_pages = _page_table(case, seed)
    x = _append_inputs(case, seed).to(f64)
    pos = torch.tensor([c + (d if case["tree"] else i) for c, n in zip(ctx, rows)
                        for i, d in enumerate(_depths(n, case["tree"]))], device="cuda", dtype=f64)
    freq = torch.tensor([base ** (-2.0 * i / hd) for i in range(hd // 2)], device="cuda", dtype=f64)
    turn = torch.polar(torch.ones(len(pos), hd // 2, device="cuda", dtype=f64), pos[:, None] * freq[None])[:, None]

    def rotate(y):     # a pair is a complex number, turned by its angle
        y = y.reshape(len(y), -1, hd)
        z = torch.complex(y[..., :hd // 2].contiguous(), y[..., hd // 2:].contiguous()) * turn
        return torch.cat([z.real, z.imag], -1)

    q, k = rotate(x[:, :H * hd]), rotate(x[:, H * hd:(H + G) * hd])
    v = x[:, (H + G) * hd:].reshape(-1, G, hd)
    pool = _random_pool(case, seed, n_pages)
    n = G * PAGE * hd
    if case["kv"] != "e4m3":
        pool = pool.to(f64)
        for s, (c, r) in enumerate(zip(ctx, rows)):
            for b in range(c // PAGE, (c + r - 1) // PAGE + 1):
                lo, hi = max(c, b * PAGE), min(c + r, (b + 1) * PAGE)
                i, t = start[s] + lo - c, lo - b * PAGE
                at = pool[int(table[s, b])]
                at[:n].view(G, PAGE, hd)[:, t:t + hi - lo] = k[i:i + hi - lo].transpose(0, 1)
                at[n:].view(G, hd, PAGE)[:, :, t:t + hi - lo] = v[i:i + hi - lo].permute(1, 2, 0)
        return [q, pool]
    out = [[], []]
    tab = table.tolist()
    first = torch.tensor([tab[s][c // PAGE] for s, c in enumerate(ctx)], device="cuda")
    kept = pool[first]
    scales = kept[:, 2 * n:2 * n + 8 * G].contiguous().view(torch.float32).view(-1, G, 2).to(f64)
    for i, (new, unpack) in enumerate(((k, _unpack_keys), (v, _unpack_values))):
        codes = unpack(kept[:, i * n:(i + 1) * n].contiguous().view(torch.float8_e4m3fn), G, hd).to(f64)
        # tops of every block of every sequence, in one list
        spans = [(s, b, max(c, b * PAGE), min(c + r, (b + 1) * PAGE)) for s, (c, r) in enumerate(zip(ctx, rows))
                 for b in range(c // PAGE, (c + r - 1) // PAGE + 1)]
        tops = torch.stack([new[start[s] + lo - ctx[s]:start[s] + hi - ctx[s]].abs().amax((0, 2)) for s, _, lo, hi in spans])
        need = torch.tensor([[_block_scale(t) for t in r] for r in tops.tolist()], device="cuda", dtype=f64)
        for (s, b, lo, hi), sc in zip(spans, need):
            old = lo % PAGE       # only a sequence's first block holds earlier tokens
            if old:
                sc = torch.maximum(sc, scales[s, :, i])
                was = codes[s, :old] * scales[s, None, :, i, None]
                out[i].append(_round_e4m3(was / sc[:, None]) * sc[:, None])
            fresh = new[start[s] + lo - ctx[s]:start[s] + hi - ctx[s]]
            out[i].append(_round_e4m3(fresh / sc[:, None]) * sc[:, None])
    return [q] + [torch.cat(o).reshape(-1, G * hd) for o in out]


def _exact_attention(case, seed):
    f64 = torch.float64
    H, G, hd, _ = DIMS[case["dims"]]
    ctx, rows = _lengths(case)
    start = _starts(rows)
    q, (kc, ks, vc, vs), table = _attention_inputs(case, seed)
    q = q.to(f64).sum(0)
    out = torch.zeros(start[-1], H, hd, device="cuda", dtype=f64)
    for s, (c, n) in enumerate(zip(ctx, rows)):
        ids = table[s, :(c + n + PAGE - 1) // PAGE].long()
        keys = (kc[ids].to(f64) * ks[ids].to(f64)[:, None, :, None]).reshape(-1, G, hd)[:c + n]
        values = (vc[ids].to(f64) * vs[ids].to(f64)[:, None, :, None]).reshape(-1, G, hd)[:c + n]
        mask = torch.cat([torch.ones(n, c, dtype=torch.bool), _visible(n, case["tree"])], 1).cuda()
        rq = q[start[s]:start[s] + n]
        for g in range(G):
            h0, h1 = g * (H // G), (g + 1) * (H // G)
            sc = torch.tensordot(rq[:, h0:h1], keys[:, g], dims=([2], [1])) / math.sqrt(hd)
            w = torch.softmax(sc.masked_fill(~mask[:, None], -math.inf), 2)
            out[start[s]:start[s] + n, h0:h1] = torch.tensordot(w, values[:, g], dims=([2], [0]))
    R, K = start[-1], H * hd
    flat = torch.zeros((R + 15) // 16 * 16, K, device="cuda", dtype=f64)
    flat[:R] = out.reshape(R, K)
    # element (row, col) of the GEMM-input layout
    col = torch.arange(K, device="cuda")
    row = torch.arange(len(flat), device="cuda")[:, None]
    at = ((row // 16 * (K // 128) + col // 128) * 2048 + col % 32 // 8 * 512 + (row % 16 + 16 * (col % 128 // 32)) * 8
          + col % 8)
    res = torch.zeros(flat.numel(), device="cuda", dtype=f64)
    res[at.reshape(-1)] = flat.reshape(-1)
    return [res]


def _exact_logprobs(case, seed):
    x, tok = _logits(case, seed)
    lp = torch.log_softmax(x.double(), 1)
    p = torch.exp(lp)
    entropy = torch.special.entr(p).sum(1)
    picked = lp[torch.arange(len(tok), device="cuda"), tok.clamp(min=0).long()]
    logprob = picked * (tok >= 0)
    if case["kind"] == "loss":
        g = _gen(seed, 6)
        g_lp, g_h = _normal(g, len(tok)).double(), _normal(g, len(tok), std=0.1).double()
        grad = -p * (g_lp * (tok >= 0))[:, None]
        grad[torch.arange(len(tok), device="cuda"), tok.clamp(min=0).long()] += g_lp * (tok >= 0)
        return [logprob, entropy, grad + (torch.special.entr(p) - p * entropy[:, None]) * g_h[:, None]]
    top = torch.topk(lp, case["k"], 1).values
    m = x.double().max(1).values
    return [logprob, entropy, torch.stack([m, torch.logsumexp(x.double(), 1) - m], 1), None, top]


def exact(case, seed):
    return {"append": _exact_append, "attention": _exact_attention}.get(case["kind"], _exact_logprobs)(case, seed)
