"""GPU parity of the paged-cache component calls (jf_kv_append, jf_kv_read,
jf_attention_kv8) against oracle/batch.py in 64 bits, at the lengths, masks,
strides and page tables where they can go wrong.

Bounds.  A rotated value u cos a - w sin a: the angle's fraction of a turn is
rounded to 24 bits (at most 2^-26 turns, 2^-23 radians), sine and cosine to
2^-23, and three operations to 2^-24 each, together below 2^-20 (|u| + |w|).
Storing rounds once more, by half a step of the type.
"""
import numpy as np
import pytest

from oracle import batch as ob

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}    # half a step relative to the value


@pytest.fixture(scope="module")
def tj():
    import torch
    from paper_2512_14681_amd import jf
    assert torch.cuda.is_available()
    return torch, jf


def types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16}


def codes(jf):
    return {"f32": jf.JF_F32, "bf16": jf.JF_BF16, "e4m3": jf.JF_E4M3}


class Seqs:
    """Ragged sequences: row starts, lengths, a scattered page table (entries past a sequence's pages are bad)."""

    def __init__(self, tj, ctx, rows, spare=2, seed=0, pad_before=0, pad_after=0, bounds=None):
        torch, jf = tj
        self.ctx, self.rows = list(ctx), list(rows)
        self.start = (pad_before + np.concatenate([[0], np.cumsum(rows)])).astype(np.int32)
        self.R = int(self.start[-1]) + pad_after
        need = [-(-(c + r) // 64) for c, r in zip(ctx, rows)]
        self.n_pages = sum(need) + spare
        perm = np.random.default_rng(seed).permutation(self.n_pages)
        self.table = np.full((len(ctx), max(max(need), 1) + 1), -7, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = perm[at:at + n]
            at += n
        i32 = dict(dtype=torch.int32, device="cuda")
        self.d_start, self.d_ctx = torch.tensor(self.start, **i32), torch.tensor(self.ctx, **i32)
        self.d_table = torch.tensor(self.table, **i32)
        self.max_rows = max(max(rows), 1)
        self.max_ctx = min(max(c + r for c, r in zip(ctx, rows)) + 5, 64 * self.table.shape[1])
        if bounds:
            self.max_rows, self.max_ctx = bounds
        self.batch = jf.Batch(self.d_start, self.d_ctx, self.d_table, self.R, self.max_rows, self.max_ctx,
                              self.n_pages)
        self.flags = torch.zeros(1, **i32)


def rows_input(torch, rng, R, cols, x, pad, offset):
    """(device view [R][cols] on a longer stride and an odd offset, its values in 64 bits)."""
    dt = types(torch)[x]
    buf = torch.tensor(rng.normal(size=(R * (cols + pad) + offset,)), dtype=torch.float32).to(dt).cuda()
    view = buf[offset:offset + R * (cols + pad)].view(R, cols + pad)[:, :cols]
    return view, view.double().cpu().numpy()


LENGTHS = [
    # (ctx, rows): one token, page borders, ragged, empty sequences, several pages
    ([0], [1]), ([63], [1]), ([64], [1]), ([1], [130]), ([0, 5, 60, 64, 127], [64, 59, 9, 1, 0]),
    ([10, 0, 200, 33], [0, 0, 3, 300]),
]


@pytest.mark.parametrize("hd,G,grp,x,kv,act", [
    (32, 4, 1, "f32", "f32", "f32"), (64, 2, 8, "bf16", "bf16", "bf16"), (128, 4, 7, "f32", "bf16", "bf16"),
    (32, 4, 2, "bf16", "e4m3", "f32"), (64, 1, 2, "f32", "e4m3", "bf16"), (128, 4, 7, "bf16", "e4m3", "bf16"),
    (128, 1, 3, "f32", "e4m3", "f32")])
@pytest.mark.parametrize("case", range(len(LENGTHS)))
def test_append_and_read(tj, hd, G, grp, x, kv, act, case):
    torch, jf = tj
    ctx, rows = LENGTHS[case]
    H = G * grp
    rng = np.random.default_rng([hd, G, case, len(x), len(kv)])
    # odd strides and offsets in every second case; two rows of padding on either side
    odd = case % 2
    S = Seqs(tj, ctx, rows, seed=case, pad_before=2, pad_after=2)
    q, q64 = rows_input(torch, rng, S.R, H * hd, x, 3 * odd, odd)
    k, k64 = rows_input(torch, rng, S.R, G * hd, x, 5 * odd, 3 * odd)
    v, v64 = rows_input(torch, rng, S.R, G * hd, x, odd, odd)
    pos = np.concatenate([[0, 0]] + [c + np.arange(r) // 2 for c, r in zip(ctx, rows)] + [[0, 0]]).astype(np.int32)
    use_pos, base = case in (1, 3), (0.0 if case == 2 else 1e4)
    # the cache before: values, or random codes on scales of 2^-9 .. 2^-5
    if kv == "e4m3":
        raw = rng.integers(0, 256, (S.n_pages, ob.page_bytes(G, hd))).astype(np.uint8)
        raw[(raw & 127) == 127] -= 64
        n = 2 * G * 64 * hd
        raw[:, n:n + 8 * G] = (2.0 ** rng.integers(-9, -4, (S.n_pages, 2 * G))).astype(np.float32).view(np.uint8)
        pool = torch.tensor(raw).cuda()
        want = ob.Pool8(raw, G, hd)
    else:
        pool = torch.tensor(rng.normal(size=(S.n_pages, 2 * G * 64 * hd)), dtype=torch.float32).to(types(torch)[kv]).cuda()
        want = ob.PoolDense(pool.double().cpu().numpy(), G, hd)
    before = pool.clone()
    planes = 2 if act == "bf16" else 1
    q_out = torch.full((planes, S.R, H, hd), 7.0, dtype=types(torch)[act], device="cuda")
    jf.kv_append(S.batch, H, G, hd, codes(jf)[kv], pool, k, v, d_q=q, d_q_out=q_out, act_dtype=codes(jf)[act],
                 d_pos=torch.tensor(pos).cuda() if use_pos else None, rope_base=base, d_flags=S.flags)
    assert int(S.flags) == 0
    ob.append(want, S.start, ctx, S.table, k64.reshape(-1, G, hd), v64.reshape(-1, G, hd), base,
              pos if use_pos else None)
    # queries
    slots = pos if use_pos else np.concatenate([[0, 0]] + [c + np.arange(r) for c, r in zip(ctx, rows)] + [[0, 0]])
    lo, hi = S.start[0], S.start[-1]
    w = ob.rotate(q64.reshape(-1, H, hd), slots, base)[lo:hi]
    mag = np.abs(q64.reshape(-1, H, 2, hd // 2)).sum(2)[lo:hi]
    mag = np.concatenate([mag, mag], -1)
    got = q_out.double().sum(0).cpu().numpy()[lo:hi]
    # two bf16 planes leave half a step of the second: 2^-16 of the value
    assert (np.abs(got - w) <= 2.0 ** -20 * mag + (2.0 ** -16 if act == "bf16" else HALF["f32"]) * np.abs(w)).all()
    assert bool((q_out[:, :lo] == 7).all()) and bool((q_out[:, hi:] == 7).all())
    # the cache: every slot that no row names as it was, the others within the bound
    kmag = np.abs(k64.reshape(-1, G, 2, hd // 2)).sum(2)
    kmag = np.concatenate([kmag, kmag], -1)
    if kv == "e4m3":
        got_pool = ob.Pool8(pool.cpu().numpy(), G, hd)
        assert np.array_equal(got_pool.raw[:, 2 * G * 64 * hd:], want.raw[:, 2 * G * 64 * hd:])   # scales, padding
    else:
        got_pool = ob.PoolDense(pool.double().cpu().numpy(), G, hd)
    touched = set()
    for s, (c, r) in enumerate(zip(ctx, rows)):
        for p in range(c // 64, -(-(c + r) // 64) if r else c // 64):
            t0, t1 = max(c - 64 * p, 0), min(c + r - 64 * p, 64)
            page = S.table[s, p]
            touched.add(int(page))
            i0 = S.start[s] + 64 * p + t0 - c
            for g in range(G):
                for kind in (0, 1):
                    a, b = got_pool.values(page, g, kind), want.values(page, g, kind)
                    assert np.array_equal(a[:t0], b[:t0]) and np.array_equal(a[t1:], b[t1:])
                    x64 = (v64.reshape(-1, G, hd) if kind else ob.rotate(k64.reshape(-1, G, hd), slots, base))[i0:i0 + t1 - t0, g]
                    rot = 0.0 if kind else 2.0 ** -20 * kmag[i0:i0 + t1 - t0, g]
                    if kv == "e4m3":
                        step = np.maximum(2.0 ** -4 * np.abs(x64), 2.0 ** -10 * got_pool.scale(page, g, kind))
                    else:
                        step = HALF[kv] * np.abs(x64) if not (kind and kv == x) else 0.0
                    assert (np.abs(a[t0:t1] - x64) <= step + 2 * rot).all(), (s, p, g, kind)
    rest = [p for p in range(S.n_pages) if p not in touched]
    assert bool((pool[rest].view(torch.uint8) == before[rest].view(torch.uint8)).all())
    # read back: what the pool holds, rounded once to the rows' type
    for xt in ("f32", "bf16"):
        ko = torch.full((S.R, G * hd + 3), 5.0, dtype=types(torch)[xt], device="cuda")
        vo = torch.full((S.R, G * hd), 5.0, dtype=types(torch)[xt], device="cuda")
        jf.kv_read(S.batch, G, hd, codes(jf)[kv], pool, ko[:, :G * hd], vo, d_flags=S.flags)
        assert bool((ko[:, G * hd:] == 5).all()) and bool((ko[:lo] == 5).all()) and bool((vo[hi:] == 5).all())
        for s, (c, r) in enumerate(zip(ctx, rows)):
            for kind, o in ((0, ko[:, :G * hd]), (1, vo)):
                held = ob.gather(got_pool, S.table[s], c + r, G, kind)[c:] if r else np.zeros((0, G, hd))
                a = o[S.start[s]:S.start[s + 1]].double().cpu().numpy().reshape(-1, G, hd)
                b = torch.tensor(held).to(types(torch)[xt]).double().numpy()
                assert np.array_equal(a, b)
    assert int(S.flags) == 0


def test_far_positions_turn_exactly(tj):
    """Angles of positions up to 2^30 - 1: the bound above, with no loss in the turns."""
    torch, jf = tj
    hd, R = 128, 40
    rng = np.random.default_rng(5)
    S = Seqs(tj, [0], [R])
    pos = rng.integers(1 << 20, 1 << 30, R).astype(np.int32)
    pos[-1] = (1 << 30) - 1
    k, k64 = rows_input(torch, rng, R, hd, "f32", 0, 0)
    pool = torch.zeros(S.n_pages, 2 * 64 * hd, device="cuda")
    jf.kv_append(S.batch, 1, 1, hd, jf.JF_F32, pool, k, k, d_pos=torch.tensor(pos).cuda(), rope_base=1e6)
    got = ob.PoolDense(pool.double().cpu().numpy(), 1, hd).values(S.table[0, 0], 0, 0)[:R]
    # the oracle's own angles, in 64 bits, are off by 2^30 radians * 2^-53 and more: they are formed as turns
    # with the integer part taken out exactly
    from fractions import Fraction
    x = k64
    for i in range(0, hd // 2, 9):
        f = Fraction(float(1e6 ** (-2.0 * i / hd) / (2 * np.pi)))
        for r in range(R):
            t = f * int(pos[r])
            a = 2 * np.pi * float(t - round(t))
            u, w = x[r, i], x[r, i + hd // 2]
            # 2^30 * 2^-53 turns from the product in 64 bits, 2 pi of them radians: below 2^-20
            bound = 2.0 ** -19 * (abs(u) + abs(w))
            assert abs(got[r, i] - (u * np.cos(a) - w * np.sin(a))) <= bound
            assert abs(got[r, i + hd // 2] - (w * np.cos(a) + u * np.sin(a))) <= bound


def test_special_values_in_an_8bit_page(tj):
    """Infinities saturate, NaN stays, neither sets the scale; zeros get scale 1; a larger token later
    requantises the kept ones; a page begun anew takes a new scale; the same call twice changes nothing."""
    torch, jf = tj
    G, hd = 1, 32
    S = Seqs(tj, [0], [4])
    pool = torch.zeros(S.n_pages, ob.page_bytes(G, hd), dtype=torch.uint8, device="cuda")
    x = torch.zeros(4, hd, device="cuda")
    jf.kv_append(S.batch, 4, G, hd, jf.JF_E4M3, pool, x, x)
    p = ob.Pool8(pool.cpu().numpy(), G, hd)
    page = S.table[0, 0]
    assert p.scale(page, 0, 0) == p.scale(page, 0, 1) == 1.0
    x[0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.5])
    jf.kv_append(S.batch, 4, G, hd, jf.JF_E4M3, pool, x, x)
    p = ob.Pool8(pool.cpu().numpy(), G, hd)
    for kind in (0, 1):
        assert p.scale(page, 0, kind) == 2.0 ** -7              # 3.5 = 448 * 2^-7
        got = p.values(page, 0, kind)[0, :4]
        assert got[0] == 3.5 and got[1] == -3.5 and np.isnan(got[2]) and got[3] == 3.5
    # two more tokens after these four, the second one large
    S.d_ctx.fill_(4)
    S.d_start.copy_(torch.tensor([0, 2]))
    y = torch.zeros(2, hd, device="cuda")
    y[1, 0] = 1000.0
    for _ in range(2):
        b2 = jf.Batch(S.d_start, S.d_ctx, S.d_table, 2, 2, 64, S.n_pages)
        jf.kv_append(b2, 4, G, hd, jf.JF_E4M3, pool, y, y)
        p2 = ob.Pool8(pool.cpu().numpy(), G, hd)
        want = ob.Pool8(p.raw, G, hd)
        want.append(page, 0, 0, 4, y.double().cpu().numpy())
        want.append(page, 0, 1, 4, y.double().cpu().numpy())
        assert p2.scale(page, 0, 0) == 4.0 and np.isnan(p2.values(page, 0, 0)[0, 2])
        nan = np.isnan(want.values(page, 0, 0))
        for kind in (0, 1):
            a, b = p2.values(page, 0, kind), want.values(page, 0, kind)
            assert np.array_equal(np.isnan(a), nan) and np.array_equal(a[~nan], b[~nan])
    # from the first token on: the old scale is forgotten
    S.d_ctx.fill_(0)
    jf.kv_append(b2, 4, G, hd, jf.JF_E4M3, pool, y[:2] * 0.001, y[:2] * 0.001)
    assert ob.Pool8(pool.cpu().numpy(), G, hd).scale(page, 0, 0) == 2.0 ** -8


def test_what_does_not_fit_is_left_alone(tj):
    """A length, a row range or a page beyond the host's bounds raises its flag and moves nothing of that
    sequence; the sequences beside it are served."""
    torch, jf = tj
    G, hd = 2, 64
    x = torch.randn(6, G * hd, device="cuda")
    q = torch.zeros(1, 6, 4, hd, device="cuda")

    def run(S, H=4):
        pool = torch.zeros(S.n_pages, ob.page_bytes(G, hd), dtype=torch.uint8, device="cuda")
        ko, vo = (torch.full((6, G * hd), 9.0, device="cuda") for _ in range(2))
        out = torch.full((1, 16 * H * hd), 9.0, device="cuda")
        ws = torch.empty(jf.attention_kv8_ws_bytes(S.batch, H, G, hd), dtype=torch.uint8, device="cuda")
        seen = []
        for call in (lambda: jf.kv_append(S.batch, H, G, hd, jf.JF_E4M3, pool, x, x, d_flags=S.flags),
                     lambda: jf.kv_read(S.batch, G, hd, jf.JF_E4M3, pool, ko, vo, d_flags=S.flags),
                     lambda: jf.attention_kv8(S.batch, H, G, hd, jf.JF_F32, q, pool, out, ws, d_flags=S.flags)):
            S.flags.zero_()
            call()
            seen.append(int(S.flags))
        return seen, pool, ko

    for spoil, flag in ((lambda S: S.d_ctx[0].fill_(-1), 2), (lambda S: S.d_ctx[0].fill_(1 << 29), 2),
                        (lambda S: S.d_ctx[0].fill_(2147483647), 2),
                        (lambda S: S.d_start[0].fill_(-3), 2), (lambda S: S.d_start[0].fill_(4), 2),
                        (lambda S: S.d_table[0, 0].fill_(S.n_pages), jf.JF_FLAG_BAD_PAGE),
                        (lambda S: S.d_table[0, 0].fill_(-1), jf.JF_FLAG_BAD_PAGE),
                        (lambda S: S.d_table[0, 0].fill_(1 << 30), jf.JF_FLAG_BAD_PAGE)):
        S = Seqs(tj, [0, 3], [3, 3], seed=3)
        spoil(S)
        seen, pool, ko = run(S)
        assert seen == [flag] * 3
        other = int(S.table[1, 0])
        untouched = [p for p in range(S.n_pages) if p != other]
        assert bool((pool[untouched] == 0).all()) and bool((pool[other] != 0).any())
        assert bool((ko[:3] == 9).all()) and bool((ko[3:] != 9).any())
    # more rows than max_rows says, more than the tensors hold
    S = Seqs(tj, [0, 3], [3, 3], seed=3, bounds=(2, 64))
    seen, pool, ko = run(S)
    assert seen == [2] * 3 and bool((pool == 0).all()) and bool((ko == 9).all())
    S = Seqs(tj, [0, 3], [3, 3], seed=3)
    S.d_start[2].fill_(7)
    seen, pool, ko = run(S)
    assert seen == [2] * 3 and bool((ko[3:] == 9).all()) and bool((ko[:3] != 9).any())


# ---- attention -----------------------------------------------------------------------
def tree(n, kind, rng):
    """[n][n] bool masks of the in-step slots."""
    vis = np.tril(np.ones((n, n), bool))
    if kind == "tree":
        vis = np.zeros((n, n), bool)
        for i in range(n):
            par = int(rng.integers(-1, i)) if i else -1
            if par >= 0:
                vis[i] = vis[par]
            vis[i, i] = True
    elif kind == "any":                     # not only what came before: any set of the in-step slots, some empty
        vis = rng.random((n, n)) < 0.3
        vis[::5] = False
    return vis


def vis_words(torch, S, masks):
    bits = np.zeros((S.R, 512), bool)
    bits[:, :] = True                       # bits of slots past the sequence's rows are set: they mean nothing
    for s, m in enumerate(masks):
        bits[S.start[s]:S.start[s + 1], :m.shape[1]] = m
    w = np.packbits(bits.reshape(S.R, 8, 64), axis=2, bitorder="little").view(np.uint64).reshape(S.R, 8)
    return torch.tensor(w.view(np.int64)).cuda()


def rows_of_layout(jf, flat, R, K):
    return jf.act_unlayout(flat, R, K)


def attention_case(tj, hd, G, grp, act, ctx, rows, kind, seed, qstd=1.0, nan_outside=True):
    """Runs the call and checks every row against the oracle within a derived bound."""
    torch, jf = tj
    H = G * grp
    rng = np.random.default_rng(seed)
    S = Seqs(tj, ctx, rows, seed=seed, pad_before=1, pad_after=1)
    raw = np.full((S.n_pages, ob.page_bytes(G, hd)), 0x7F if nan_outside else 0, np.uint8)   # NaN where nothing is written
    pool = ob.Pool8(raw, G, hd)
    for s, (c, r) in enumerate(zip(ctx, rows)):
        kv = rng.normal(size=(2, c + r, G, hd)) * np.exp2(rng.integers(-2, 3, (2, c + r, 1, 1)))
        ob.append(pool, [0, c + r], [0], [S.table[s]], kv[0], kv[1])
    d_pool = torch.tensor(pool.raw).cuda()
    q = rng.normal(size=(S.R, H, hd)).astype(np.float32) * qstd
    tq = torch.tensor(q).cuda()
    if act == "bf16":
        h = tq.to(torch.bfloat16)
        planes = torch.stack([h, (tq - h.float()).to(torch.bfloat16)])
    else:
        planes = tq[None].contiguous()
    q64 = planes.double().sum(0).cpu().numpy()
    masks = [tree(r, kind, rng) for r in rows]
    K, Rp = H * hd, (S.R + 15) // 16 * 16
    out = torch.full((planes.shape[0], Rp * K), 3.0, dtype=planes.dtype, device="cuda")
    ws = torch.full((jf.attention_kv8_ws_bytes(S.batch, H, G, hd),), 0xFF, dtype=torch.uint8, device="cuda")
    d_vis = None if kind == "causal" else vis_words(torch, S, masks)
    jf.attention_kv8(S.batch, H, G, hd, codes(jf)[act], planes, d_pool, out, ws, d_vis=d_vis, d_flags=S.flags)
    assert int(S.flags) == 0
    got = jf.act_unlayout(out.double().sum(0).cpu().numpy(), S.R, K).reshape(S.R, H, hd)
    filler = 3.0 * planes.shape[0]
    assert (got[:1] == filler).all() and (got[S.R - 1:] == filler).all()
    for s, (c, r) in enumerate(zip(ctx, rows)):
        if not r:
            continue
        k = ob.gather(pool, S.table[s], c + r, G, 0)
        v = ob.gather(pool, S.table[s], c + r, G, 1)
        rq = q64[S.start[s]:S.start[s + 1]]
        want = ob.attention(rq, k, v, c, masks[s])
        a = got[S.start[s]:S.start[s + 1]]
        # A score: Q in two fp16 terms leaves 2^-20 of the row's largest element, the products of hd terms
        # are summed in fp32, and the exponent's argument rounds to 2^-23 of the score.
        kk, vmax = np.abs(k).sum(2).max(0), np.abs(v).max((0, 2))            # by KV head
        qm = np.abs(rq).max(2).reshape(r, G, grp)
        score = qm * kk[None, :, None] / np.sqrt(hd)
        d = score * (2.0 ** -20 + hd * 2.0 ** -24) + score * 2.0 ** -23 + 2.0 ** -22
        # Weights in two fp16 terms: 2^-20; sums over the pages in fp32: one rounding a page, 64 inside one.
        rel = 2 * d + 2.0 ** -20 + ((c + r) / 64 + 64) * 2.0 ** -24
        bound = (rel * vmax[None, :, None]).reshape(r, H)[..., None]
        bound = bound + np.abs(want) * (2.0 ** -16 if act == "bf16" else 2.0 ** -24)
        assert (np.abs(a - want) <= bound).all(), (s, float((np.abs(a - want) / bound).max()))
    return S, got


@pytest.mark.parametrize("hd,G,grp,act", [(32, 4, 1, "f32"), (64, 2, 8, "f32"), (64, 2, 8, "bf16"),
                                          (128, 4, 7, "bf16"), (128, 1, 1, "f32"), (32, 1, 4, "bf16"),
                                          (64, 2, 3, "bf16")])
@pytest.mark.parametrize("ctx,rows,kind", [
    ([0], [1], "causal"), ([63], [1], "causal"), ([64], [1], "causal"), ([0, 1, 64, 130, 257], [1, 1, 1, 1, 1], "causal"),
    ([700], [1], "causal"), ([0], [70], "causal"), ([37, 0, 100], [13, 0, 5], "tree"), ([100, 64], [20, 64], "any"),
    ([0, 250], [9, 33], "any")])
def test_attention(tj, hd, G, grp, act, ctx, rows, kind):
    attention_case(tj, hd, G, grp, act, ctx, rows, kind, seed=len(ctx) + hd)


@pytest.mark.parametrize("hd,G,grp,act,ctx,rows,kind", [
    (128, 2, 7, "bf16", [300], [200], "tree"), (128, 1, 4, "f32", [0], [512], "causal"),
    (64, 1, 2, "bf16", [65], [512], "any"), (32, 4, 1, "bf16", [500, 3], [200, 129], "tree"),
    (128, 1, 2, "bf16", [9000], [3], "causal"), (64, 2, 8, "f32", [20000], [1], "causal")])
def test_attention_many_rows_and_long_prefixes(tj, hd, G, grp, act, ctx, rows, kind):
    attention_case(tj, hd, G, grp, act, ctx, rows, kind, seed=hd + rows[0])


@pytest.mark.parametrize("hd,G,grp,act", [(128, 4, 7, "bf16"), (64, 2, 8, "f32"), (32, 1, 8, "bf16")])
@pytest.mark.parametrize("ctx,rows,kind", [([0], [4], "causal"), ([900, 0, 63, 130], [4, 1, 0, 3], "tree"),
                                           ([5000, 64], [3, 4], "any"), ([60, 61, 62], [4, 4, 4], "causal")])
def test_attention_of_short_drafts(tj, hd, G, grp, act, ctx, rows, kind):
    """17 to 32 queries of a KV head, some sequences with fewer."""
    attention_case(tj, hd, G, grp, act, ctx, rows, kind, seed=grp + len(ctx))


@pytest.mark.parametrize("qstd", [0.0, 1e-30, 8.0, 1e4])
def test_attention_scores_of_any_size(tj, qstd):
    """From queries of zero (the mean of the values) to scores of which one takes all."""
    attention_case(tj, 64, 2, 4, "f32", [150], [5], "causal", seed=11, qstd=qstd)


def test_attention_rows_that_see_nothing(tj):
    torch, jf = tj
    S, got = attention_case(tj, 64, 2, 2, "bf16", [0, 0], [11, 70], "any", seed=4)
    assert (got[S.start[0]] == 0).all() and (got[S.start[1] + 5] == 0).all()


@pytest.mark.parametrize("rows", [1, 6, 30])
def test_attention_skips_a_bad_pages_slots(tj, rows):
    """A table entry beyond the pool, while page 0 holds NaN scales: what attention over the other pages gives."""
    torch, jf = tj
    G, grp, hd, C = 2, 4, 64, 200
    rng = np.random.default_rng(rows)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = np.array([[3, 5, 1, 4]], np.int32)
    pool = ob.Pool8(np.zeros((6, ob.page_bytes(G, hd)), np.uint8), G, hd)
    kv = rng.normal(size=(2, C + rows, G, hd))
    ob.append(pool, [0, C + rows], [0], table, kv[0], kv[1])
    k, v = (ob.gather(pool, table[0], C + rows, G, kind) for kind in (0, 1))
    n = 2 * G * 64 * hd
    pool.raw[0, :n] = 0x7F
    pool.raw[0, n:n + 8 * G] = np.full(2 * G, np.nan, np.float32).view(np.uint8)
    q = torch.tensor(rng.normal(size=(1, rows, G * grp, hd)), dtype=torch.float32).cuda()
    bad = table.copy()
    bad[0, 1] = 6
    flags = torch.zeros(1, **i32)
    b = jf.Batch(torch.tensor([0, rows], **i32), torch.tensor([C], **i32), torch.tensor(bad).cuda(), rows, rows, 256, 6)
    out = torch.zeros(1, (rows + 15) // 16 * 16 * G * grp * hd, device="cuda")
    ws = torch.empty(jf.attention_kv8_ws_bytes(b, G * grp, G, hd), dtype=torch.uint8, device="cuda")
    jf.attention_kv8(b, G * grp, G, hd, jf.JF_F32, q, torch.tensor(pool.raw).cuda(), out, ws, d_flags=flags)
    assert int(flags) == jf.JF_FLAG_BAD_PAGE
    got = jf.act_unlayout(out[0].cpu().numpy(), rows, G * grp * hd).reshape(rows, G * grp, hd)
    rest = np.r_[0:64, 128:C + rows]
    want = ob.attention(q[0].double().cpu().numpy(), k[rest], v[rest], C - 64, np.tril(np.ones((rows, rows), bool)))
    # scores below 16 in all: 2 (16 (2^-20 + 64 2^-24 + 2^-23)) of the largest value, and the sums
    assert np.abs(got - want).max() <= (2 * 16 * (2.0 ** -20 + 2.0 ** -18 + 2.0 ** -23) + 80 * 2.0 ** -24) * np.abs(v).max()


@pytest.mark.parametrize("rows", [6, 100])
def test_attention_nan_reaches_only_the_rows_that_see_it(tj, rows):
    """NaN in a key (every output of the rows that see it) and in one dim of a value (that dim of them)."""
    torch, jf = tj
    G, grp, hd, C = 1, 4, 32, 70
    rng = np.random.default_rng(8)
    S = Seqs(tj, [C], [rows])
    pool = ob.Pool8(np.zeros((S.n_pages, ob.page_bytes(G, hd)), np.uint8), G, hd)
    kv = rng.normal(size=(2, C + rows, G, hd))
    kv[0, C + 2, 0, 7] = np.nan
    kv[1, C + 4, 0, 9] = np.nan
    ob.append(pool, [0, C + rows], [0], S.table, kv[0], kv[1])
    vis = np.tril(np.ones((rows, rows), bool))
    vis[:, 2] = vis[:, 4] = False
    vis[3, 2] = vis[5, 4] = True
    q = torch.tensor(rng.normal(size=(1, rows, grp, hd)), dtype=torch.float32).cuda()
    out = torch.zeros(1, (rows + 15) // 16 * 16 * grp * hd, device="cuda")
    ws = torch.empty(jf.attention_kv8_ws_bytes(S.batch, grp, G, hd), dtype=torch.uint8, device="cuda")
    jf.attention_kv8(S.batch, grp, G, hd, jf.JF_F32, q, torch.tensor(pool.raw).cuda(), out, ws,
                     d_vis=vis_words(torch, S, [vis]))
    nan = np.isnan(jf.act_unlayout(out[0].cpu().numpy(), rows, grp * hd).reshape(rows, grp, hd))
    want = np.zeros((rows, grp, hd), bool)
    want[3] = True
    want[5, :, 9] = True
    assert np.array_equal(nan, want)


def test_attention_prefix_nan_is_seen_by_all(tj):
    torch, jf = tj
    G, hd = 1, 128
    S = Seqs(tj, [64], [1])
    pool = ob.Pool8(np.zeros((S.n_pages, ob.page_bytes(G, hd)), np.uint8), G, hd)
    v = np.ones((65, G, hd))
    v[3, 0, 100] = np.nan
    ob.append(pool, [0, 65], [0], S.table, np.ones((65, G, hd)), v)
    out = torch.zeros(1, 16 * hd, device="cuda")
    ws = torch.empty(jf.attention_kv8_ws_bytes(S.batch, 1, G, hd), dtype=torch.uint8, device="cuda")
    jf.attention_kv8(S.batch, 1, G, hd, jf.JF_F32, torch.ones(1, 1, 1, hd, device="cuda"), torch.tensor(pool.raw).cuda(),
                     out, ws)
    got = jf.act_unlayout(out[0].cpu().numpy(), 1, hd)[0]
    assert np.isnan(got[100]) and not np.isnan(np.delete(got, 100)).any()


def test_pages_beyond_32_bit_offsets(tj):
    """A pool of 4.6 GB: pages at its end hold the sequence."""
    torch, jf = tj
    G, hd, C = 4, 128, 150
    pb = jf.kv_page_bytes(G, hd, jf.JF_E4M3)
    n_pages = (1 << 32) // pb + 5000
    pool = torch.zeros(n_pages, pb, dtype=torch.uint8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.tensor([[n_pages - 1, n_pages - 3000, n_pages - 2]], **i32)
    small = torch.tensor([[0, 2, 1]], **i32)
    pool2 = torch.zeros(3, pb, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(C, 3, G * hd, device="cuda", generator=g)
    outs = []
    for t, p in ((table, pool), (small, pool2)):
        b = jf.Batch(torch.tensor([0, C], **i32), torch.tensor([0], **i32), t, C, C, 192, p.shape[0])
        q = torch.empty(1, C, G, hd, device="cuda")
        jf.kv_append(b, G, G, hd, jf.JF_E4M3, p, x[:, 0], x[:, 1], d_q=x[:, 2], d_q_out=q, act_dtype=jf.JF_F32,
                     rope_base=1e4)
        out = torch.zeros(1, 160 * G * hd, device="cuda")
        ws = torch.empty(jf.attention_kv8_ws_bytes(b, G, G, hd), dtype=torch.uint8, device="cuda")
        jf.attention_kv8(b, G, G, hd, jf.JF_F32, q, p, out, ws)
        ko, vo = (torch.empty(C, G * hd, device="cuda") for _ in range(2))
        jf.kv_read(b, G, hd, jf.JF_E4M3, p, ko, vo)
        outs.append((out, ko, vo))
    for a, b in zip(*outs):
        assert bool((a == b).all())
    assert bool((pool[n_pages - 1] == pool2[0]).all()) and int((pool[:100] != 0).sum()) == 0
    assert float(outs[0][0].abs().sum()) > 0


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_read_into_rows_on_8_byte_boundaries(tj, hd):
    """bf16 rows whose starts are multiples of 8 bytes, not of 16, and of 4: the values are those of plain rows."""
    torch, jf = tj
    G, C, n = 3, 50, 90
    S = Seqs(tj, [C], [n])
    pool = torch.zeros(S.n_pages, jf.kv_page_bytes(G, hd, jf.JF_E4M3), dtype=torch.uint8, device="cuda")
    first = jf.Batch(torch.tensor([0, C + n], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda(), S.d_table,
                     C + n, C + n, 64 * S.d_table.shape[1], S.n_pages)
    x = torch.randn(C + n, 2, G * hd, device="cuda")
    jf.kv_append(first, G, G, hd, jf.JF_E4M3, pool, x[:, 0], x[:, 1])
    want = [torch.empty(n, G * hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    jf.kv_read(S.batch, G, hd, jf.JF_E4M3, pool, *want)
    assert bool((want[0] != 0).any()) and bool((want[1] != 0).any())
    for pad, at in ((4, 4), (4, 0), (1, 2)):
        flat = torch.full((2, n * (G * hd + pad) + at), 9.0, dtype=torch.bfloat16, device="cuda")
        rows = [f[at:].view(n, G * hd + pad) for f in flat]
        jf.kv_read(S.batch, G, hd, jf.JF_E4M3, pool, rows[0][:, :G * hd], rows[1][:, :G * hd])
        for r, w in zip(rows, want):
            assert bool((r[:, :G * hd] == w).all()) and bool((r[:, G * hd:] == 9).all())
        assert bool((flat[:, :at] == 9).all())


def test_shared_prefix_pages(tj):
    """Two sequences whose first pages are the same: each sees them, and appends to its own last page."""
    torch, jf = tj
    G, hd = 2, 64
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros(4, jf.kv_page_bytes(G, hd, jf.JF_E4M3), dtype=torch.uint8, device="cuda")
    x = torch.randn(64, 2, G * hd, device="cuda")
    one = jf.Batch(torch.tensor([0, 64], **i32), torch.tensor([0], **i32), torch.tensor([[2]], **i32), 64, 64, 64, 4)
    jf.kv_append(one, G, G, hd, jf.JF_E4M3, pool, x[:, 0], x[:, 1])
    shared = pool[2].clone()
    both = jf.Batch(torch.tensor([0, 1, 2], **i32), torch.tensor([64, 64], **i32), torch.tensor([[2, 0], [2, 3]], **i32),
                    2, 1, 128, 4)
    y = x[:1, 0].repeat(2, 1)
    jf.kv_append(both, G, G, hd, jf.JF_E4M3, pool, y, y)
    assert bool((pool[2] == shared).all()) and bool((pool[0] == pool[3]).all())
    q = torch.randn(1, 1, G, hd, device="cuda").repeat(1, 2, 1, 1).contiguous()
    out = torch.zeros(1, 16 * G * hd, device="cuda")
    ws = torch.empty(jf.attention_kv8_ws_bytes(both, G, G, hd), dtype=torch.uint8, device="cuda")
    jf.attention_kv8(both, G, G, hd, jf.JF_F32, q, pool, out, ws)
    got = jf.act_unlayout(out[0].cpu().numpy(), 2, G * hd)
    assert np.array_equal(got[0], got[1]) and np.abs(got[0]).sum() > 0


def test_bf16_cache_feeds_the_engines_attention(tj):
    """A bf16 pool that jf_kv_append filled is what jf_attention reads: a rotated prefix and a draft of 5 rows."""
    torch, jf = tj
    H, G, hd, C, n = 8, 2, 64, 100, 5
    rng = np.random.default_rng(21)
    S = Seqs(tj, [0], [C], spare=1)
    S2 = Seqs(tj, [C], [n], spare=1)
    xk, k64 = rows_input(torch, rng, C + n, G * hd, "f32", 0, 0)
    xv, v64 = rows_input(torch, rng, C + n, G * hd, "f32", 0, 0)
    xq, q64 = rows_input(torch, rng, C + n, H * hd, "f32", 0, 0)
    pool = torch.zeros(S2.n_pages, 2 * G * 64 * hd, dtype=torch.bfloat16, device="cuda")
    b1 = jf.Batch(S.d_start, S.d_ctx, S2.d_table, C, C, 128, S2.n_pages)
    jf.kv_append(b1, H, G, hd, jf.JF_BF16, pool, xk[:C], xv[:C], rope_base=1e4)
    q = torch.empty(2, n, H, hd, dtype=torch.bfloat16, device="cuda")
    jf.kv_append(S2.batch, H, G, hd, jf.JF_BF16, pool, xk[C:], xv[C:], d_q=xq[C:], d_q_out=q, rope_base=1e4)
    out = torch.zeros(2, 16 * H * hd, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(jf.lib().jf_attention_ws_bytes(H, hd, n), dtype=torch.uint8, device="cuda")
    jf.check(jf.lib().jf_attention(H, G, hd, jf.JF_BF16, C, n, jf._ptr(q), jf._ptr(pool), jf._ptr(S2.d_table), None,
                                   jf._ptr(out), jf._ptr(ws), jf._stream()))
    got = jf.act_unlayout(out.double().sum(0).cpu().numpy(), n, H * hd).reshape(n, H, hd)
    held = ob.PoolDense(pool.double().cpu().numpy(), G, hd)
    k, v = (ob.gather(held, S2.table[0], C + n, G, kind) for kind in (0, 1))
    want = ob.attention(q.double().sum(0).cpu().numpy(), k, v, C, np.tril(np.ones((n, n), bool)))
    # the engine's attention: 16-bit terms of q and of the weights; scores below 8, values below 5
    assert np.abs(got - want).max() <= 2.0 ** -12
    rot = ob.rotate(k64.reshape(-1, G, hd), np.arange(C + n), 1e4)
    assert np.abs(k - rot).max() <= 2.0 ** -8 * np.abs(rot).max() * 1.01


# ---- streams, captures -----------------------------------------------------------------
def test_captured_calls_follow_the_devices_lengths(tj):
    """Append and attention of a growing batch, captured once on a stream of their own: replays take new
    lengths and rows, and equal the eager calls; two captures share one workspace."""
    torch, jf = tj
    G, grp, hd, B, steps = 2, 4, 64, 3, 70
    H = G * grp
    i32 = dict(dtype=torch.int32, device="cuda")
    start = torch.arange(B + 1, **i32)
    table = torch.arange(B * 3, **i32).view(B, 3)
    ctx, pool = torch.zeros(B, **i32), torch.zeros(B * 3, jf.kv_page_bytes(G, hd, jf.JF_E4M3), dtype=torch.uint8, device="cuda")
    b = jf.Batch(start, ctx, table, B, 1, 192, B * 3)
    x = torch.zeros(B, (H + 2 * G) * hd, device="cuda")
    q = torch.zeros(1, B, H, hd, device="cuda")
    out, out2 = (torch.zeros(1, 16 * H * hd, device="cuda") for _ in range(2))
    ws = torch.empty(jf.attention_kv8_ws_bytes(b, H, G, hd), dtype=torch.uint8, device="cuda")

    def one(o, x_, q_, pool_, b_, ws_):
        jf.kv_append(b_, H, G, hd, jf.JF_E4M3, pool_, x_[:, H * hd:(H + G) * hd], x_[:, (H + G) * hd:],
                     d_q=x_[:, :H * hd], d_q_out=q_, act_dtype=jf.JF_F32, rope_base=1e4)
        jf.attention_kv8(b_, H, G, hd, jf.JF_F32, q_, pool_, o, ws_)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one(out, x, q, pool, b, ws)
        pool.zero_()
        torch.cuda.synchronize()
        graphs = []
        for o in (out, out2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                one(o, x, q, pool, b, ws)
            graphs.append(graph)
        ectx, epool = torch.zeros(B, **i32), torch.zeros_like(pool)
        eb = jf.Batch(start, ectx, table, B, 1, 192, B * 3)
        eq, eo, ews = torch.zeros_like(q), torch.zeros_like(out), torch.empty_like(ws)
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        for i in range(steps):
            x.copy_(torch.randn(x.shape, device="cuda", generator=g) * (1 + i))
            ctx.fill_(i)
            ectx.fill_(i)
            ctx[1] = ectx[1] = 2 * i
            graphs[0].replay()
            graphs[1].replay()
            one(eo, x, eq, epool, eb, ews)
            torch.cuda.synchronize()
            assert bool((out == eo).all()) and bool((out2 == eo).all()) and bool((pool == epool).all()), i
    assert float(out.abs().sum()) > 0


def test_calls_on_two_streams_at_once(tj):
    """Streams that are named, not current, each with its own workspace: what the calls give alone."""
    torch, jf = tj
    G, grp, hd, C = 2, 4, 64, 1500
    H = G * grp
    sets = []
    for seed, rows in ((1, 1), (2, 70)):
        S = Seqs(tj, [C, 300], [rows, rows], seed=seed)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        pool = torch.randint(0, 100, (S.n_pages, jf.kv_page_bytes(G, hd, jf.JF_E4M3)), dtype=torch.uint8, device="cuda",
                             generator=g)
        n = 2 * G * 64 * hd
        pool[:, n:n + 8 * G] = torch.ones(2 * G).view(torch.uint8).cuda()
        x = torch.randn(S.R, (H + 2 * G) * hd, device="cuda", generator=g)
        q = torch.empty(1, S.R, H, hd, device="cuda")
        out = torch.zeros(1, (S.R + 15) // 16 * 16 * H * hd, device="cuda")
        ws = torch.empty(jf.attention_kv8_ws_bytes(S.batch, H, G, hd), dtype=torch.uint8, device="cuda")
        sets.append((S, pool, x, q, out, ws))

    def one(S, pool, x, q, out, ws, stream):
        jf.kv_append(S.batch, H, G, hd, jf.JF_E4M3, pool, x[:, H * hd:(H + G) * hd], x[:, (H + G) * hd:],
                     d_q=x[:, :H * hd], d_q_out=q, act_dtype=jf.JF_F32, rope_base=1e4, stream=stream)
        jf.attention_kv8(S.batch, H, G, hd, jf.JF_F32, q, pool, out, ws, stream=stream)
    alone = []
    for a in sets:
        one(*a, None)
        alone.append((a[4].clone(), a[1].clone()))
        a[4].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(20):                     # the rows once more into the same slots: the same pages
        for a, st in zip(sets, streams):
            one(*a, st)
    torch.cuda.synchronize()
    for a, (o, pool) in zip(sets, alone):
        assert bool((a[4] == o).all()) and bool((a[1] == pool).all()) and float(o.abs().sum()) > 0
