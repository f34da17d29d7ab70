"""jf_attention_shared against softmax attention of every sequence by itself in 64 bits.

Tolerances, from the arithmetic: queries, keys and values are what the planes and the cache hold.  A score is a sum of
head_dim products (twice as many for two planes) in fp32, off by at most e = 2 hd 2^-24 sum |q k| / sqrt(hd); a weight is
off by 2 e + n 2^-24 relative, and enters the second product in two bf16 terms, whose rest is at most 2^-17 of it (2^-24
in fp32); the output is stored in two terms again.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

DIMS = {"7b": (28, 4, 128), "grp3": (6, 2, 64), "tiny": (4, 4, 32), "wide": (8, 1, 128), "grp8": (16, 2, 64)}
PAGE = 64


def _torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def visible(n, tree, empty=()):
    """[n][n] bool: a chain, or every third row a branch of row 0; rows of `empty` see nothing in the step."""
    vis = np.tril(np.ones((n, n), bool))
    if tree:
        for i in range(1, n):
            vis[i] = vis[0] if i % 3 == 0 else vis[i - 1]
            vis[i, i] = True
    for i in empty:
        vis[i] = False
    return vis


def words(masks):
    out = np.zeros((sum(len(m) for m in masks), 8), np.uint64)
    at = 0
    for m in masks:
        for i, row in enumerate(m):
            for j in np.flatnonzero(row):
                out[at + i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        at += len(m)
    return out


class Call:
    """groups: [(shared pages, [(committed tokens beyond the shared ones, rows)])]; loners: sequences of no group behind
    them.  Pages are scattered; what no sequence's slots hold is NaN."""

    def __init__(self, groups, dims, name, seed=0, loners=(), tree=False, empty=(), pad=(0, 0), std=2.0):
        torch = _torch()
        from paper_2512_14681_amd import jf
        self.H, self.G, self.hd = H, G, hd = DIMS[dims]
        self.name, self.code = name, jf.JF_F32 if name == "f32" else jf.JF_BF16
        dt = torch.float32 if name == "f32" else torch.bfloat16
        rng = np.random.default_rng(seed)
        members = [(p, c, r) for p, seqs in groups for c, r in seqs] + [(0, c, r) for c, r in loners]
        need = [(p * PAGE + c + r + PAGE - 1) // PAGE for p, c, r in members]
        total = sum(p for p, _ in groups) + sum(n - p for n, (p, _, _) in zip(need, members)) + 2
        perm = rng.permutation(total)
        stride = max(need + [1])
        table = np.full((len(members), stride), -1, np.int32)   # entries past a sequence's pages are no pages
        at = s = 0
        for p, seqs in list(groups) + [(0, [m]) for m in loners]:
            shared, at = perm[at:at + p], at + p
            for _ in seqs:
                own = need[s] - p
                table[s, :p], table[s, p:need[s]] = shared, perm[at:at + own]
                at, s = at + own, s + 1
        self.members, self.table_np = members, table
        R = pad[0] + sum(r for _, _, r in members) + pad[1]
        self.R, self.pad = R, pad
        starts = pad[0] + np.cumsum([0] + [r for _, _, r in members])
        self.starts = starts
        self.masks = [visible(r, tree, [e for e in empty if e < r]) for _, _, r in members]
        k = torch.full((total, G, PAGE, hd), math.nan, dtype=torch.float64)
        v = torch.full((total, G, PAGE, hd), math.nan, dtype=torch.float64)
        for s, (p, c, r) in enumerate(members):
            for b in range(need[s]):
                n = min(p * PAGE + c + r - b * PAGE, PAGE)
                for t in (k, v):
                    t[table[s, b], :, :n] = torch.from_numpy(rng.standard_normal((G, n, hd)))
        self.k, self.v = k.to(dt).double(), v.to(dt).double()
        pool = torch.cat([k.to(dt).reshape(total, -1), v.to(dt).transpose(2, 3).reshape(total, -1)], 1)
        self.kv = pool.contiguous().cuda()
        q = torch.from_numpy(rng.standard_normal((R, H, hd)) * std).float()
        if name == "f32":
            planes = q[None]
        else:
            hi = q.to(dt)
            planes = torch.stack([hi, (q - hi.float()).to(dt)])
        self.q64 = planes.double().sum(0)
        self.q = planes.contiguous().cuda()
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
        self.start, self.table = i32(starts), i32(table)
        self.ctx = i32([p * PAGE + c for p, c, _ in members])
        self.seq_start, self.pages = i32(np.cumsum([0] + [len(m) for _, m in groups])), i32([p for p, _ in groups])
        self.vis = torch.from_numpy(np.concatenate([np.zeros((pad[0], 8), np.uint64), words(self.masks),
                                                    np.zeros((pad[1], 8), np.uint64)]).view(np.int64)).cuda()
        self.use_vis = tree or len(empty) > 0
        self.flags = i32([0])
        self.bounds = dict(max_rows=max([r for _, _, r in members] + [1]),
                           max_ctx=max([p * PAGE + c + r for p, c, r in members] + [1]), n_pages=total)
        self.group_rows = max([sum(r for _, r in m) for _, m in groups] + [0])
        self.max_pages = max([p for p, _ in groups] + [0])
        self.out = torch.full((planes.shape[0], (R + 15) // 16 * 16 * H * hd), 7.0, dtype=dt, device="cuda")

    def descriptors(self, **kw):
        from paper_2512_14681_amd import jf
        b = dict(self.bounds, **{k: v for k, v in kw.items() if k in self.bounds})
        batch = jf.Batch(self.start, self.ctx, self.table, self.R, b["max_rows"], b["max_ctx"], b["n_pages"])
        prefix = jf.Prefix(self.seq_start, self.pages, kw.get("group_rows", self.group_rows),
                           kw.get("max_pages", self.max_pages))
        return batch, prefix

    def run(self, shared=True, stream=None, **kw):
        torch = _torch()
        from paper_2512_14681_amd import jf
        batch, prefix = self.descriptors(**kw)
        prefix = prefix if shared else None
        ws = torch.full((jf.attention_shared_ws_bytes(batch, prefix, self.H, self.G, self.hd),), 255, dtype=torch.uint8,
                        device="cuda")
        self.keep = (batch, prefix, ws)
        jf.attention_shared(batch, prefix, self.H, self.G, self.hd, self.code, self.q, self.kv, self.out, ws,
                            d_vis=self.vis if self.use_vis else None, d_flags=self.flags, stream=stream)
        return self

    def result(self):
        """[R][H][hd], float64."""
        from paper_2512_14681_amd import jf
        flat = self.out.double().sum(0).cpu().numpy()
        return _torch().from_numpy(jf.act_unlayout(flat, self.R, self.H * self.hd)).reshape(self.R, self.H, self.hd)

    def reference(self, drop=()):
        """(value, bound) of the rows of all sequences; slots of the physical pages in `drop` are seen by nobody."""
        torch = _torch()
        H, G, hd = self.H, self.G, self.hd
        f, u = 2.0 ** -24, 2.0 ** -17 if self.name == "bf16" else 2.0 ** -24
        out, bound = torch.zeros(self.R, H, hd, dtype=torch.float64), torch.zeros(self.R, H, hd, dtype=torch.float64)
        for s, (p, c, r) in enumerate(self.members):
            T = p * PAGE + c
            ids = self.table_np[s, :(T + r + PAGE - 1) // PAGE]
            keep = np.repeat(~np.isin(ids, drop), PAGE)[:T + r]
            mask = torch.from_numpy(np.concatenate([np.ones((r, T), bool), self.masks[s]], 1) & keep)
            k = self.k[np.maximum(ids, 0)].transpose(0, 1).reshape(G, -1, hd)[:, :T + r]
            v = self.v[np.maximum(ids, 0)].transpose(0, 1).reshape(G, -1, hd)[:, :T + r]
            k, v = (torch.where(torch.from_numpy(keep)[:, None], t, 0.0) for t in (k, v))
            rows = slice(int(self.starts[s]), int(self.starts[s]) + r)
            for h in range(H):
                q, kk, vv = self.q64[rows, h], k[h // (H // G)], v[h // (H // G)]
                sc = (q @ kk.T) / math.sqrt(hd)
                e = 2 * hd * f * float((q.abs() @ kk.abs().T).max()) / math.sqrt(hd)
                w = torch.softmax(sc.masked_fill(~mask, -math.inf), 1)
                w = torch.where(mask.any(1, keepdim=True), w, torch.zeros_like(w))
                out[rows, h] = w @ vv
                mag = w @ vv.abs()
                bound[rows, h] = (2 * e + (T + r + 32) * f + u) * mag + u * (w @ vv).abs() + 1e-30
        return out, bound

    def check(self, drop=()):
        value, bound = self.reference(drop)
        got = self.result()
        lo, hi = self.pad[0], self.R - self.pad[1]
        err = (got - value).abs()[lo:hi]
        assert bool((err <= bound[lo:hi]).all()), (float((err / bound[lo:hi]).max()), float(err.max()))
        for rows in (got[:lo], got[hi:]):
            assert bool((rows == 7.0 * self.out.shape[0]).all())
        assert int(self.flags) == 0


GROUPS = [
    [(1, [(0, 1)])],                                             # one sequence, nothing of its own but the row
    [(2, [(63, 1), (0, 1), (64, 1)])],                           # page borders
    [(1, [(5, 1)] * 40)],                                        # more rows than one tile holds
    [(7, [(130, 3), (1, 5), (300, 1)]), (0, [(70, 2)]), (3, [(0, 4), (9, 4)])],
    [(9, [(20, 33), (700, 17)])],
    [(5, [(0, 130)])],                                           # rows past two pages
]


@pytest.mark.parametrize("groups", GROUPS, ids=range(len(GROUPS)))
@pytest.mark.parametrize("dims,name", [("7b", "bf16"), ("grp3", "bf16"), ("tiny", "f32"), ("wide", "f32"), ("tiny", "bf16"),
                                       ("grp8", "f32")])
@pytest.mark.parametrize("tree", [False, True])
def test_matches_64_bits(groups, dims, name, tree):
    Call(groups, dims, name, seed=len(groups), tree=tree).run().check()


def test_long_prefix_many_samples():
    """Prefixes in many parts, and sequences that are split too."""
    Call([(70, [(1500, 1)] * 9), (33, [(10, 2)] * 20)], "7b", "bf16", seed=3).run().check()
    Call([(40, [(900, 1)] * 3)], "grp8", "f32", seed=4).run().check()


@pytest.mark.parametrize("dims,name", [("7b", "bf16"), ("tiny", "f32")])
def test_few_rows_over_many_parts(dims, name):
    Call([(80, [(300, 1)] * 2), (75, [(1, 3), (1200, 1)])], dims, name, seed=12).run().check()


def test_shared_parts_beside_many_sequences():
    """The sequences' own pages alone take all places of the chip; the shared ones come in parts all the same."""
    Call([(36, [(40, 8)] * 64)], "7b", "bf16", seed=13).run().check()


def test_sequences_of_no_group():
    Call([(3, [(10, 2), (100, 1)])], "grp3", "bf16", seed=5, loners=[(0, 1), (200, 7), (64, 1)]).run().check()
    Call([], "grp3", "bf16", seed=6, loners=[(33, 2), (200, 7)]).run().check()


def test_nothing_shared_by_request():
    """Without a prefix, and with a prefix of no pages: the same sequences, each by itself."""
    groups = [(3, [(10, 2), (100, 1)]), (1, [(0, 3)])]
    for name in ("bf16", "f32"):
        Call(groups, "grp3", name, seed=7).run(shared=False).check()
        c = Call(groups, "grp3", name, seed=7)
        c.pages.zero_()
        c.run().check()
        c = Call(groups, "grp3", name, seed=7)
        c.pages.zero_()
        c.run(max_pages=0).check()


def test_more_groups_than_lanes():
    groups = [(1 + g % 2, [(g % 5, 1)] * (g % 3)) for g in range(150)]
    Call(groups, "tiny", "bf16", seed=8).run().check()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_rows_that_see_nothing_are_zeros(name):
    """Rows with an empty mask and no committed tokens; the others beside them as ever."""
    c = Call([], "grp3", name, seed=9, loners=[(0, 5), (0, 40)], empty=(0, 3)).run()
    c.check()
    got = c.result()
    for r in (0, 3, 5, 8):
        assert bool((got[r] == 0).all())


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [4, 60])
def test_what_a_row_does_not_see_does_not_reach_it(name, rows):
    """A NaN or an infinity in a draft row's key and value reaches the rows that see it alone (slots past the rows hold
    NaN in every test here)."""
    c = Call([(2, [(30, rows), (5, 2)])], "grp3", name, seed=10, tree=True)
    value, bound = c.reference()
    for bad, dim in ((math.nan, 3), (math.inf, 40)):
        slot = 30 + 2                                  # in-step row 2 of the first sequence, in its own first page
        page = int(c.table_np[0, 2])
        n = c.G * PAGE * c.hd
        values = c.kv[page, n:].view(c.G, c.hd, PAGE)
        values[0, dim, slot] = bad
    c.run()
    got = c.result()
    sees = c.masks[0][:, 2]
    ok = ((got - value).abs() <= bound).numpy()
    for i in range(rows):
        for h in range(3):
            hit = got[i, h]
            if sees[i]:
                # two bf16 planes hold no infinity: hi = inf, lo = inf - inf
                assert math.isnan(float(hit[3])) and not math.isfinite(float(hit[40])), i
                ok[i, h, 3] = ok[i, h, 40] = True
    assert ok.all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 30])   # slots below 128: 1 + slot / 128 is a bf16 number
def test_scores_beyond_what_fp32_tells_apart(name, rows):
    """Scores of 2^31 and more, in even steps, the largest in the shared pages or in a sequence's own: it has all the
    weight; sums of values of 2^126 have a mean that fits."""
    torch = _torch()
    for sign in (1, -1):
        c = Call([(1, [(30, rows), (3, 2)])], "grp3", name, seed=20)
        n = c.G * PAGE * c.hd
        c.q.zero_()
        c.q[0, :, :, 0] = 2.0 ** 17
        c.q64 = c.q.double().sum(0).cpu()
        for s, (p, ctx, r) in enumerate(c.members):
            for b in range((p * PAGE + ctx + r + PAGE - 1) // PAGE):
                slots = torch.arange(b * PAGE, b * PAGE + PAGE)
                page = int(c.table_np[s, b])
                c.k[page] = 0.0
                c.k[page, :, :, 0] = sign * 2.0 ** 17 * (1 + slots / 128)
                c.v[page] = torch.where(c.v[page].isnan(), c.v[page], 2.0 ** 126 * torch.sign(c.v[page]))
        c.kv[:, :n] = c.k.reshape(len(c.k), -1).to(c.kv.dtype).cuda()
        c.kv[:, n:] = c.v.transpose(2, 3).reshape(len(c.v), -1).to(c.kv.dtype).cuda()
        c.run()
        got = c.result()
        for s, (p, ctx, r) in enumerate(c.members):
            for i in range(r):
                at = p * PAGE + ctx + i if sign > 0 else 0
                v = c.v[int(c.table_np[s, at // PAGE]), :, at % PAGE].repeat_interleave(c.H // c.G, 0)
                assert bool((got[int(c.starts[s]) + i] == v).all()), (sign, s, i)
        c.q.zero_()      # equal scores: the mean
        c.q64 = c.q.double().sum(0).cpu()
        c.flags.zero_()
        c.run().check()


def test_bad_pages_are_skipped():
    """Entries outside the pool: flagged, their slots seen by nobody; a shared page's by the whole group."""
    from paper_2512_14681_amd import jf
    for rows in (1, 30):
        c = Call([(6, [(10, rows), (200, rows)])], "grp3", "bf16", seed=11)
        c.table_np[:, 3] = -1
        c.table_np[1, 7] = 1 << 30
        c.table.copy_(_torch().from_numpy(c.table_np))
        c.table_np[:, 3] = c.table_np[1, 7] = -7     # never a page's number
        c.run()
        value, bound = c.reference(drop=[-7])
        assert bool(((c.result() - value).abs() <= bound).all())
        assert int(c.flags) == jf.JF_FLAG_BAD_PAGE


@pytest.mark.parametrize("what", ["ctx", "pages", "max_pages", "group_rows", "max_rows", "seq_start"])
def test_beyond_the_bounds(what):
    """A group or sequence beyond what the host announced: flagged, its rows left as they were, the others computed."""
    from paper_2512_14681_amd import jf
    c = Call([(4, [(10, 2), (100, 1)]), (2, [(0, 3), (70, 2), (1, 1)])], "grp3", "bf16", seed=12)
    kw, left = {}, []
    if what == "ctx":           # sequence 0 has fewer tokens than it is said to share
        c.ctx[0] = 4 * PAGE - 1
        left = [0]
    elif what == "pages":
        c.pages[1] = -1
        left = [2, 3, 4]
    elif what == "max_pages":
        kw, left = dict(max_pages=3), [0, 1]
    elif what == "group_rows":
        kw, left = dict(group_rows=5), [2, 3, 4]
    elif what == "max_rows":
        kw, left = dict(max_rows=2), [2]
    else:
        c.seq_start[1] = 6       # the first group ends behind the last sequence, the second before its start
        left = [0, 1, 2, 3, 4]
    value, bound = c.reference()
    c.run(**kw)
    got = c.result()
    for s, (_, _, r) in enumerate(c.members):
        rows = slice(int(c.starts[s]), int(c.starts[s]) + r)
        if s in left:
            assert bool((got[rows] == 14.0).all()), s
        else:
            assert bool(((got[rows] - value[rows]).abs() <= bound[rows]).all()), s
    assert int(c.flags) == jf.JF_FLAG_CAPACITY


def test_padding_rows_stay():
    Call([(3, [(10, 2), (100, 1)])], "grp3", "bf16", seed=13, pad=(5, 20)).run().check()
    Call([(3, [(10, 50), (100, 1)])], "grp3", "f32", seed=13, pad=(1, 3)).run().check()


def test_an_appended_cache():
    """jf_kv_append writes the samples' pages, jf_attention_shared reads them: a step of a serving program."""
    torch = _torch()
    from paper_2512_14681_amd import jf
    c = Call([(3, [(10, 2), (63, 3)]), (1, [(0, 1)])], "grp3", "bf16", seed=14)
    batch, prefix = c.descriptors()
    H, G, hd = c.H, c.G, c.hd
    g = torch.Generator().manual_seed(1)
    new = torch.randn(c.R, (H + 2 * G) * hd, generator=g).cuda()
    q_out = torch.zeros_like(c.q)
    jf.kv_append(batch, H, G, hd, jf.JF_BF16, c.kv, new[:, H * hd:(H + G) * hd], new[:, (H + G) * hd:], d_q=new[:, :H * hd],
                 d_q_out=q_out, act_dtype=jf.JF_BF16, rope_base=0.0, d_flags=c.flags)
    c.q.copy_(q_out)
    c.q64 = q_out.double().sum(0).cpu()
    k = new[:, H * hd:(H + G) * hd].to(torch.bfloat16).double().cpu().view(c.R, G, hd)
    v = new[:, (H + G) * hd:].to(torch.bfloat16).double().cpu().view(c.R, G, hd)
    for s, (p, ctx, r) in enumerate(c.members):
        for i in range(r):
            slot, row = p * PAGE + ctx + i, int(c.starts[s]) + i
            page = c.table_np[s, slot // PAGE]
            c.k[page, :, slot % PAGE], c.v[page, :, slot % PAGE] = k[row], v[row]
    c.run().check()


def test_captured_with_new_lengths():
    """A captured call takes the lengths, groups and pages that the device holds at every replay."""
    torch = _torch()
    a = Call([(4, [(10, 2), (100, 1)]), (2, [(0, 3), (70, 2)])], "grp3", "bf16", seed=15)
    a.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    held = a.keep
    first = a.result()
    a.out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert bool((a.result() == first).all())
    a.pages.copy_(torch.tensor([3, 0], dtype=torch.int32))      # the same tokens, fewer of them shared
    a.out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    a.check()
    a.ctx.sub_(torch.tensor([5, 20, 1, 0], dtype=torch.int32, device="cuda"))
    a.members = [(p, c - d, r) for (p, c, r), d in zip(a.members, (5, 20, 1, 0))]
    a.members[2] = (1, PAGE - 1, 3)                              # 2 pages less one token
    graph.replay()
    torch.cuda.synchronize()
    # rows past the shortened contexts now see other slots as their own: those of the tokens that were cut off
    a.check()
    del held


def test_two_streams_at_once():
    torch = _torch()
    calls = [Call([(8, [(300, 2)] * 6)], "7b", "bf16", seed=s) for s in (16, 17)]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for c, s in zip(calls, streams):
            s.wait_stream(torch.cuda.current_stream())
            c.run(stream=s)
        torch.cuda.synchronize()
        for c in calls:
            c.check()


def test_same_bits_every_time():
    calls = [Call([(20, [(300, 2)] * 9)], "7b", "bf16", seed=18).run().result() for _ in range(3)]
    for c in calls[1:]:
        assert bool((c == calls[0]).all())
