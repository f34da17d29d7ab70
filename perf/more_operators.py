"""The component operators of training on sampled groups: causal attention over packed sequences with its gradient,
attention of a batch whose sequences share long prefixes, and a clipped policy loss with its gradient.

Each case is one pass through one of them, as a program that samples from a model and trains it calls it.  Where ``own``
is false ``run`` computes the same in elementary torch operations.  All inputs are made on the GPU from the seed; how
long each sequence is belongs to the case.
"""
import math
import random

import torch

own = False

# Attention dimensions (query heads, KV heads, head_dim) of the repository's decoder shapes.
DIMS = {
    "7b": (28, 4, 128),     # the benchmark's decoder shape
    "mid": (16, 4, 128),    # the mid-size bf16 decoder of the tests
    "small": (16, 2, 64),   # generic: head_dim 64
    "tiny": (4, 4, 32),     # the tests' fp32 decoder: every query head has keys of its own
}
PAGE = 64               # tokens of a cache page
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CLIP_LOW, CLIP_HIGH, KL_WEIGHT, ENTROPY_WEIGHT, SCALE = 0.2, 0.28, 0.04, 0.001, 1.0


def listed():
    return [
        # A short prompt: the smallest call, launch and host time.
        {"name": "causal_rows64", "kind": "causal", "dims": "7b", "x": "bf16", "seqs": 1, "rows": 64},
        # A prompt of ordinary length.
        {"name": "causal_rows2048", "kind": "causal", "dims": "7b", "x": "bf16", "seqs": 1, "rows": 2048},
        # The prompts of sixteen requests, ragged, one behind the other.
        {"name": "causal_ragged16", "kind": "causal", "dims": "mid", "x": "bf16", "seqs": 16, "rows": 1500},
        # A long prompt: bound by the matrix cores.
        {"name": "causal_rows8192", "kind": "causal", "dims": "7b", "x": "bf16", "seqs": 1, "rows": 8192},
        # A training sequence, forward and backward.
        {"name": "train_rows4096", "kind": "train", "dims": "7b", "x": "bf16", "seqs": 1, "rows": 4096},
        # Nine answers packed into one training row, a small decoder.
        {"name": "train_ragged9", "kind": "train", "dims": "small", "x": "bf16", "seqs": 9, "rows": 1000},
        # Two sequences of odd lengths in fp32: the tests' decoder.
        {"name": "train_tiny_f32", "kind": "train", "dims": "tiny", "x": "f32", "seqs": 2, "rows": 333},
        # One decoding step of 64 samples of one prompt of 8192 tokens.
        {"name": "shared_batch64", "kind": "shared", "dims": "7b", "x": "bf16", "groups": 1, "seqs": 64, "pages": 128,
         "ctx": 500, "rows": 1, "tree": False},
        # Draft blocks of 13 rows under tree masks: five prompts of up to 2048 tokens, eight samples of each.
        {"name": "shared_groups5", "kind": "shared", "dims": "mid", "x": "bf16", "groups": 5, "seqs": 8, "pages": 32,
         "ctx": 777, "rows": 13, "tree": True},
        # A step of three samples in fp32: the smallest call.
        {"name": "shared_small_f32", "kind": "shared", "dims": "small", "x": "f32", "groups": 1, "seqs": 3, "pages": 5,
         "ctx": 70, "rows": 2, "tree": False},
        # The tokens of a small training batch.
        {"name": "policy_rows512", "kind": "policy", "seqs": 8, "rows": 64, "mean": "seqs", "adv": "seq"},
        # A large batch of samples, advantages of their own for every token.
        {"name": "policy_rows1m", "kind": "policy", "seqs": 1024, "rows": 1500, "mean": "tokens", "adv": "row"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["causal", "causal", "causal", "train", "train", "train", "shared", "shared", "shared", "policy"])
    if kind == "policy":
        seqs = _log_int(rng, 1, 1024)
        return {"kind": kind, "seqs": seqs, "rows": _log_int(rng, 1, min(8192, (1 << 20) // seqs)),
                "mean": rng.choice(["tokens", "seqs", "sum"]), "adv": rng.choice(["seq", "row"])}
    c = {"kind": kind, "dims": rng.choice(["7b", "7b", "mid", "small", "tiny"])}
    c["x"] = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "shared":
        c["groups"] = _log_int(rng, 1, 8)
        c["seqs"] = _log_int(rng, 1, 64 // c["groups"])
        c["pages"] = _log_int(rng, 1, 256 // c["groups"])
        c["ctx"] = _log_int(rng, 1, 2000)
        c["rows"] = _log_int(rng, 1, max(1, min(128, 512 // (c["groups"] * c["seqs"]))))
        c["tree"] = rng.random() < 0.4
        return c
    # as much work as the largest case at most: the fp32 matrix rate is a sixteenth of the bf16 one
    c["seqs"] = _log_int(rng, 1, 32)
    H, _, hd = DIMS[c["dims"]]
    pairs = (2.2e11 if kind == "causal" else 0.9e11) / (16 if c["x"] == "f32" else 1) / (2 * H * hd)
    c["rows"] = _log_int(rng, 1, min(8192, int(math.sqrt(2 * pairs / c["seqs"]))))
    return c


# ---- lengths --------------------------------------------------------------------------
def _rng(case):
    return random.Random("/".join(f"{k}={v}" for k, v in sorted(case.items()) if k != "name"))


def _rows(case):
    """Rows of each packed sequence: the first has the case's, the others down to a quarter of them."""
    rng, n = _rng(case), case["rows"]
    return [n] + [rng.randint((n + 3) // 4, n) for _ in range(case["seqs"] - 1)]


def _groups(case):
    """[(shared pages, [(tokens of a sequence's own, rows)])] of each group: the first has the case's sizes, the others
    down to a quarter of them."""
    rng = _rng(case)

    def some(n):
        return rng.randint((n + 3) // 4, n)
    out = []
    for g in range(case["groups"]):
        pages, seqs = (case["pages"], case["seqs"]) if g == 0 else (some(case["pages"]), some(case["seqs"]))
        out.append((pages, [(case["ctx"], case["rows"]) if g == i == 0 else (rng.randint(case["ctx"] // 4, case["ctx"]),
                                                                             some(case["rows"])) for i in range(seqs)]))
    return out


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _parents(n, tree):
    """A row's parent among its sequence's rows: a chain, or half a chain and branches of 8 under the first row."""
    half = (n + 1) // 2
    if not tree:
        return list(range(-1, n - 1))
    return [i - 1 if i < half or (i - half) % 8 else (0 if i else -1) for i in range(n)]


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


def _causal_inputs(case, seed):
    """(rows of a fused projection [R][(H + 2 G) hd]: rotated queries and keys, values; gradient of the outputs)."""
    H, G, hd = DIMS[case["dims"]]
    g, R = _gen(seed, 1), sum(_rows(case))
    x = _normal(g, R, (H + 2 * G) * hd)
    x[:, :H * hd] *= 1.5
    return x.to(TYPES[case["x"]]), _normal(g, R, H * hd, dtype=TYPES[case["x"]]) if case["kind"] == "train" else None


def _tables(case, seed):
    """(page table [sequences][stride], pages of the pool): pages scattered over the pool, a group's first ones shared."""
    groups = _groups(case)
    need = [pages + (c + r + PAGE - 1) // PAGE for pages, seqs in groups for c, r in seqs]
    total = sum(pages + sum((c + r + PAGE - 1) // PAGE for c, r in seqs) for pages, seqs in groups) + 3
    perm = torch.randperm(total, device="cuda", generator=_gen(seed, 2)).to(torch.int32)
    table = torch.zeros(len(need), max(need), dtype=torch.int32, device="cuda")
    at = s = 0
    for pages, seqs in groups:
        shared, at = perm[at:at + pages], at + pages
        for c, r in seqs:
            n = (c + r + PAGE - 1) // PAGE
            table[s, :pages], table[s, pages:pages + n] = shared, perm[at:at + n]
            at, s = at + n, s + 1
    return table, total


def _planes(x, kind):
    """An fp32 tensor as activation planes: hi and lo bf16, or one fp32 plane."""
    if kind == "f32":
        return x[None]
    hi = x.to(torch.bfloat16)
    return torch.stack([hi, (x - hi.float()).to(torch.bfloat16)])


def _shared_inputs(case, seed):
    """(q planes [P][R][H][hd], cache pages: keys [G][64][hd], then values [G][hd][64])."""
    H, G, hd = DIMS[case["dims"]]
    _, n_pages = _tables(case, seed)
    g = _gen(seed, 3)
    R = sum(r for _, seqs in _groups(case) for _, r in seqs)
    q = _planes(_normal(g, R, H, hd, std=2.0), case["x"]).contiguous()
    return q, _normal(g, n_pages, 2 * G * PAGE * hd, dtype=TYPES[case["x"]])


def _vis_words(case):
    """[R][8] 64-bit words: bit j of a row's mask is the j-th row of its sequence."""
    rows = [r for _, seqs in _groups(case) for _, r in seqs]
    bits = torch.zeros(sum(rows), 512, dtype=torch.bool)
    at, seen = 0, {}
    for n in rows:
        if n not in seen:
            seen[n] = _visible(n, case["tree"])
        bits[at:at + n, :n] = seen[n]
        at += n
    weights = (torch.ones(64, dtype=torch.int64) << torch.arange(64)).view(1, 1, 64)
    return (bits.view(-1, 8, 64).long() * weights).sum(2).contiguous().cuda()


def _policy_inputs(case, seed):
    """(tokens, log probabilities now / when sampled / of the reference, entropies, advantages); a quarter of the rows
    belong to prompts and have no token."""
    g, R = _gen(seed, 4), sum(_rows(case))
    lp = -torch.empty(R, device="cuda").exponential_(1.2, generator=g)
    old, ref = (torch.clamp(lp + _normal(g, R, std=s), max=0.0) for s in (0.15, 0.3))
    tokens = torch.randint(0, 152064, (R,), device="cuda", generator=g, dtype=torch.int32)
    tokens[torch.rand(R, device="cuda", generator=g) < 0.25] = -1
    entropy = torch.empty(R, device="cuda").exponential_(0.8, generator=g)
    return tokens, lp, old, ref, entropy, _normal(g, R if case["adv"] == "row" else case["seqs"])


def prepare(case, seed):
    s = {"case": case}
    if case["kind"] == "policy":
        s["tokens"], s["lp"], s["old"], s["ref"], s["entropy"], s["adv"] = _policy_inputs(case, seed)
        s["start"] = _ints(_starts(_rows(case)))
        s["stats"] = torch.zeros(6, device="cuda")
        s["g_lp"], s["g_entropy"] = torch.zeros_like(s["lp"]), torch.zeros_like(s["lp"])
        return s
    H, G, hd = DIMS[case["dims"]]
    if case["kind"] == "shared":
        groups = _groups(case)
        seqs = [(pages, c, r) for pages, members in groups for c, r in members]
        s["q"], s["kv"] = _shared_inputs(case, seed)
        s["table"], s["n_pages"] = _tables(case, seed)
        s["ctx"] = _ints([pages * PAGE + c for pages, c, _ in seqs])
        s["start"] = _ints(_starts([r for _, _, r in seqs]))
        s["seq_start"] = _ints(_starts([len(members) for _, members in groups]))
        s["shared"] = _ints([pages for pages, _ in groups])
        s["vis"] = _vis_words(case) if case["tree"] else None
        R = sum(r for _, _, r in seqs)
        s["out"] = torch.zeros(s["q"].shape[0], (R + 15) // 16 * 16 * H * hd, dtype=s["q"].dtype, device="cuda")
        s["flags"] = _ints([0])
        return s
    s["x"], s["g_out"] = _causal_inputs(case, seed)
    R = len(s["x"])
    s["start"], s["flags"] = _ints(_starts(_rows(case))), _ints([0])
    s["out"] = torch.zeros(R, H * hd, dtype=s["x"].dtype, device="cuda")
    s["lse"] = torch.zeros(H, R, device="cuda")
    if case["kind"] == "train":
        s["g_x"] = torch.zeros_like(s["x"])
    return s


# ---- one pass -------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"shared": _own_shared, "policy": _own_policy}.get(kind, _own_causal)(s)
    return {"shared": _plain_shared, "policy": _plain_policy}.get(kind, _plain_causal)(s)


def _split(x, dims):
    """The queries, keys and values in rows of a fused projection."""
    H, G, hd = DIMS[dims]
    return x[:, :H * hd], x[:, H * hd:(H + G) * hd], x[:, (H + G) * hd:]


def _own_causal(s):
    from paper_2512_14681_amd import jf
    c = s["case"]
    H, G, hd = DIMS[c["dims"]]
    q, k, v = _split(s["x"], c["dims"])
    jf.attention_causal(s["start"], H, G, hd, q, k, v, s["out"], d_lse=s["lse"], d_flags=s["flags"])
    if c["kind"] == "causal":
        return [s["out"], s["lse"]]
    if "ws" not in s:
        n = jf.attention_causal_grad_ws_bytes(len(s["start"]) - 1, len(s["x"]), H, G, hd)
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    g_q, g_k, g_v = _split(s["g_x"], c["dims"])
    jf.attention_causal_grad(s["start"], H, G, hd, q, k, v, s["out"], s["lse"], s["g_out"], g_q, g_k, g_v, s["ws"],
                             d_flags=s["flags"])
    return [s["out"], s["g_x"]]


def _own_shared(s):
    from paper_2512_14681_amd import jf
    c = s["case"]
    H, G, hd = DIMS[c["dims"]]
    if "batch" not in s:    # made at the first pass, as a program makes them when its buffers are
        groups = _groups(c)
        seqs = [(pages, n, r) for pages, members in groups for n, r in members]
        s["batch"] = jf.Batch(s["start"], s["ctx"], s["table"], sum(r for _, _, r in seqs), max(r for _, _, r in seqs),
                              max(pages * PAGE + n + r for pages, n, r in seqs), s["n_pages"])
        s["prefix"] = jf.Prefix(s["seq_start"], s["shared"], max(sum(r for _, r in members) for _, members in groups),
                                max(pages for pages, _ in groups))
        s["ws"] = torch.empty(jf.attention_shared_ws_bytes(s["batch"], s["prefix"], H, G, hd), dtype=torch.uint8,
                              device="cuda")
    jf.attention_shared(s["batch"], s["prefix"], H, G, hd, jf.JF_F32 if c["x"] == "f32" else jf.JF_BF16, s["q"], s["kv"],
                        s["out"], s["ws"], d_vis=s["vis"], d_flags=s["flags"])
    # the value the planes stand for
    return [s["out"][0] if c["x"] == "f32" else torch.sum(s["out"], 0, dtype=torch.float32)]


def _own_policy(s):
    from paper_2512_14681_amd import jf
    c = s["case"]
    if "ws" not in s:
        n = jf.policy_loss_ws_bytes(c["seqs"], len(s["lp"]))
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    mean = {"tokens": jf.JF_MEAN_TOKENS, "seqs": jf.JF_MEAN_SEQS, "sum": jf.JF_SUM}[c["mean"]]
    jf.policy_loss(s["start"], s["tokens"], s["lp"], s["old"], s["adv"], s["stats"], s["ws"], d_ref_logprob=s["ref"],
                   d_entropy=s["entropy"], d_g_logprob=s["g_lp"], d_g_entropy=s["g_entropy"], clip_low=CLIP_LOW,
                   clip_high=CLIP_HIGH, kl_weight=KL_WEIGHT, entropy_weight=ENTROPY_WEIGHT, scale=SCALE, mean=mean,
                   adv_rows=c["adv"] == "row")
    return [s["stats"], s["g_lp"], s["g_entropy"]]


# ---- the plain forms ------------------------------------------------------------------
def _plain_causal(s):
    c = s["case"]
    H, G, hd = DIMS[c["dims"]]
    q, k, v = (t.float() for t in _split(s["x"], c["dims"]))
    out, lse = torch.zeros_like(q), torch.zeros(H, len(q), device="cuda")
    train = c["kind"] == "train"
    if train:
        g_out = s["g_out"].float()
        g_x = torch.zeros_like(s["x"], dtype=torch.float32)
        g_q, g_k, g_v = _split(g_x, c["dims"])
    at = 0
    for n in _rows(c):
        rows, m = slice(at, at + n), H // G
        at += n

        def heads(t, m):       # [G][m n][hd]: the rows of a group's heads one after the other
            return t[rows].reshape(n, G, m, hd).permute(1, 2, 0, 3).reshape(G, m * n, hd).contiguous()

        def back(t, m):
            return t.reshape(G, m, n, hd).permute(2, 0, 1, 3).reshape(n, G * m * hd)
        qs, ks, vs = heads(q, m), heads(k, 1), heads(v, 1)
        p = torch.matmul(qs, ks.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(hd)).view(G, m, n, n)
        future = torch.ones(n, n, dtype=torch.bool, device="cuda").triu_(1)
        p.masked_fill_(future, -math.inf)
        top = p.amax(-1, keepdim=True)
        p = p.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        lse[:, rows] = (top + torch.log(total)).view(H, n)
        p = p.div_(total).view(G, m * n, n)
        o = torch.matmul(p, vs)
        out[rows] = back(o, m)
        if train:
            do = heads(g_out, m)
            d = torch.matmul(do, vs.transpose(1, 2).contiguous())
            d = d.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(hd))
            g_v[rows] = back(torch.matmul(p.transpose(1, 2).contiguous(), do), 1)
            g_q[rows] = back(torch.matmul(d, ks), m)
            g_k[rows] = back(torch.matmul(d.transpose(1, 2).contiguous(), qs), 1)
    if train:
        return [out.to(s["x"].dtype), g_x.to(s["x"].dtype)]
    return [out.to(s["x"].dtype), lse]


def _gemm_layout(x):
    """[R][K] in the GEMM-input layout of include/jf.h: rows padded to 16 with zeros, 16 x 128 blocks in matrix-core order."""
    R, K = x.shape
    x = torch.nn.functional.pad(x, (0, 0, 0, -R % 16)).reshape(-1, 16, K // 128, 4, 4, 8)
    return x.permute(0, 2, 4, 3, 1, 5).reshape(-1)


def _plain_shared(s):
    """Every sequence's cache, padded to the longest, as if nothing were shared."""
    c = s["case"]
    H, G, hd = DIMS[c["dims"]]
    m, n = H // G, G * PAGE * hd
    start, ctx, table = s["start"].long(), s["ctx"].long(), s["table"].long()
    B, T, R = len(ctx), table.shape[1] * PAGE, s["q"].shape[1]
    most = max(r for _, members in _groups(c) for _, r in members)
    pages = s["kv"][table.reshape(-1)]
    keys = pages[:, :n].float().view(B, -1, G, PAGE, hd).permute(0, 2, 1, 3, 4).reshape(B, G, T, hd)
    values = pages[:, n:].float().view(B, -1, G, hd, PAGE).permute(0, 2, 1, 4, 3).reshape(B, G, T, hd)
    r = torch.arange(R, device="cuda")
    seq = torch.searchsorted(start[1:], r, right=True)
    within = r - start[seq]
    q = torch.zeros(B, most, H, hd, device="cuda")
    q[seq, within] = s["q"].float().sum(0)
    q = q.view(B, most, G, m, hd).permute(0, 2, 3, 1, 4).reshape(B, G, -1, hd)
    own_row = torch.arange(T, device="cuda") - ctx[:, None]      # [B][T]: the in-step row in that slot
    if s["vis"] is None:
        seen = own_row[:, None] <= torch.arange(most, device="cuda")[None, :, None]
    else:
        words = torch.zeros(B, most, 8, dtype=torch.int64, device="cuda")
        words[seq, within] = s["vis"]
        o = own_row.clamp(0, 511)
        bits = torch.gather(words, 2, (o // 64)[:, None].expand(B, most, T)) >> (o % 64)[:, None] & 1
        seen = (bits == 1) & (own_row[:, None] >= 0) | (own_row[:, None] < 0)
    seen &= own_row[:, None] < (start[1:] - start[:-1])[:, None, None]
    scores = torch.matmul(q, keys.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(hd))
    scores = scores.view(B, G, m, most, T).masked_fill_(~seen[:, None, None], -math.inf)
    scores = scores.sub_(scores.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores.view(B, G, -1, T), values).view(B, G, m, most, hd)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, most, H * hd)[seq, within]
    return [_planes(_gemm_layout(o), c["x"]).to(torch.float32).sum(0)]


def _plain_policy(s):
    """Differences of log probabilities are taken in 64 bits: ratios lie next to the borders, KL terms next to 0."""
    c = s["case"]
    start, R = s["start"].long(), len(s["lp"])
    seq = torch.searchsorted(start[1:], torch.arange(R, device="cuda"), right=True)
    valid = s["tokens"] >= 0
    lp = s["lp"].double()
    adv = s["adv"].double()
    adv = adv if c["adv"] == "row" else adv[seq]
    ratio = torch.exp(lp - s["old"].double())
    clipped = ((adv > 0) & (ratio > 1 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - CLIP_LOW))
    policy = -torch.minimum(ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
    k = s["ref"].double() - lp
    kl = torch.expm1(k) - k
    if c["mean"] == "tokens":
        w = valid / valid.sum().clamp(min=1).double()
    elif c["mean"] == "seqs":
        count = torch.zeros(c["seqs"], dtype=torch.float64, device="cuda").index_add_(0, seq, valid.double())
        w = valid / (count[seq] * (count > 0).sum()).clamp(min=1)
    else:
        w = valid.double()
    entropy = s["entropy"].double()
    loss = SCALE * (w * (policy + KL_WEIGHT * kl - ENTROPY_WEIGHT * entropy)).sum()
    stats = torch.stack([loss, (w * policy).sum(), (w * kl).sum(), (w * entropy).sum(), (w * clipped).sum(),
                         valid.sum().double()])
    g = SCALE * w * (torch.where(clipped, 0.0, -adv * ratio) - KL_WEIGHT * torch.expm1(k))
    return [stats.float(), g.float(), (-SCALE * ENTROPY_WEIGHT * w).float()]


# ---- what a pass cannot do without ----------------------------------------------------
def work(case):
    if case["kind"] == "policy":
        R = sum(_rows(case))
        return {"bytes": R * (5 * 4 + 8 + (4 if case["adv"] == "row" else 0)), "flops": 40.0 * R}
    H, G, hd = DIMS[case["dims"]]
    e = 2 if case["x"] == "bf16" else 4
    if case["kind"] == "shared":
        pairs = slots = R = 0
        for pages, members in _groups(case):
            slots += pages * PAGE
            for c, r in members:
                pairs += r * (pages * PAGE + c) + int(_visible(r, case["tree"]).sum())
                slots += c + r
                R += r
        return {"bytes": slots * 2 * G * hd * e + R * H * hd * 8, "flops": 4.0 * H * hd * pairs}
    rows = _rows(case)
    R, pairs = sum(rows), sum(n * (n + 1) // 2 for n in rows)
    by, fl = R * (2 * H + 2 * G) * hd * e + R * H * 4, 4.0 * H * hd * pairs
    if case["kind"] == "train":     # the gradient of the outputs and the outputs, and q, k, v again; their gradients
        return {"bytes": by + R * (4 * H + 4 * G) * hd * e, "flops": fl + 10.0 * H * hd * pairs}
    return {"bytes": by, "flops": fl}


# ---- the same in 64 bits --------------------------------------------------------------
def _exact_causal(case, seed):
    H, G, hd = DIMS[case["dims"]]
    x, g_out = _causal_inputs(case, seed)
    R = len(x)
    out = torch.zeros(R, H, hd, dtype=torch.float64, device="cuda")
    lse = torch.zeros(H, R, dtype=torch.float64, device="cuda")
    g_x = torch.zeros(R, H + 2 * G, hd, dtype=torch.float64, device="cuda")
    at = 0
    for n in _rows(case):
        here = x[at:at + n].double().reshape(n, H + 2 * G, hd)
        past = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for h in range(H):
            g = h // (H // G)
            q, k, v = (here[:, i].clone().requires_grad_(case["kind"] == "train") for i in (h, H + g, H + G + g))
            score = torch.mm(q, k.t()) / math.sqrt(hd)
            score = torch.where(past, score, -math.inf)
            o = torch.mm(torch.softmax(score, 1), v)
            out[at:at + n, h], lse[h, at:at + n] = o.detach(), torch.logsumexp(score.detach(), 1)
            if case["kind"] == "train":
                grads = torch.autograd.grad(o, (q, k, v), g_out[at:at + n, h * hd:(h + 1) * hd].double())
                for i, grad in zip((h, H + g, H + G + g), grads):
                    g_x[at:at + n, i] += grad
        at += n
    out = out.reshape(R, -1)
    return [out, g_x.reshape(R, -1)] if case["kind"] == "train" else [out, lse]


def _exact_shared(case, seed):
    H, G, hd = DIMS[case["dims"]]
    q, pool = _shared_inputs(case, seed)
    table, _ = _tables(case, seed)
    q = q.double().sum(0)
    R, n = len(q), G * PAGE * hd
    flat = torch.zeros((R + 15) // 16 * 16, H * hd, dtype=torch.float64, device="cuda")
    at = s = 0
    for pages, members in _groups(case):
        for c, r in members:
            T = pages * PAGE + c
            ids = table[s, :(T + r + PAGE - 1) // PAGE].long()
            keys = pool[ids, :n].double().view(-1, G, PAGE, hd)
            values = pool[ids, n:].double().view(-1, G, hd, PAGE)
            mask = torch.cat([torch.ones(r, T, dtype=torch.bool), _visible(r, case["tree"])], 1).cuda()
            for h in range(H):
                g = h // (H // G)
                score = torch.mm(q[at:at + r, h], keys[:, g].reshape(-1, hd)[:T + r].t()) / math.sqrt(hd)
                w = torch.softmax(score.masked_fill(~mask, -math.inf), 1)
                v = values[:, g].transpose(1, 2).reshape(-1, hd)[:T + r]
                flat[at:at + r, h * hd:(h + 1) * hd] = torch.mm(w, v)
            at, s = at + r, s + 1
    # element (row, col) of the GEMM-input layout
    K = H * hd
    col = torch.arange(K, device="cuda")
    row = torch.arange(len(flat), device="cuda")[:, None]
    to = ((row // 16 * (K // 128) + col // 128) * 2048 + col % 32 // 8 * 512 + (row % 16 + 16 * (col % 128 // 32)) * 8
          + col % 8)
    res = torch.zeros(flat.numel(), device="cuda", dtype=torch.float64)
    res[to.reshape(-1)] = flat.reshape(-1)
    return [res]


def _exact_policy(case, seed):
    tokens, lp, old, ref, entropy, adv = _policy_inputs(case, seed)
    lens = torch.tensor(_rows(case), device="cuda")
    lp, entropy = (t.double().requires_grad_() for t in (lp, entropy))
    if case["adv"] == "seq":
        adv = adv.repeat_interleave(lens)
    adv, has = adv.double(), (tokens >= 0).double()
    if case["mean"] == "sum":
        w = has
    elif case["mean"] == "tokens":
        w = has / max(float(has.sum()), 1.0)
    else:
        parts = [p / p.sum() if bool(p.sum() > 0) else p for p in torch.split(has, lens.tolist())]
        w = torch.cat(parts) / max(sum(bool(p.sum() > 0) for p in parts), 1)
    ratio = torch.exp(lp - old.double())
    low, high = ratio * adv, torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
    policy = (w * -torch.where(low <= high, low, high)).sum()
    cut = (w * ((ratio > 1 + CLIP_HIGH) * (adv > 0) + (ratio < 1 - CLIP_LOW) * (adv < 0))).sum()
    kl = (w * (torch.exp(ref.double() - lp) - 1 - (ref.double() - lp))).sum()
    mean_entropy = (w * entropy).sum()
    loss = SCALE * (policy + KL_WEIGHT * kl - ENTROPY_WEIGHT * mean_entropy)
    g_lp, g_entropy = torch.autograd.grad(loss, (lp, entropy))
    return [torch.stack([loss, policy, kl, mean_entropy, cut, has.sum()]).detach(), g_lp, g_entropy]


def exact(case, seed):
    return {"shared": _exact_shared, "policy": _exact_policy}.get(case["kind"], _exact_causal)(case, seed)
