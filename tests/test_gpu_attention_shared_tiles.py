"""jf_attention_shared where test_gpu_attention_shared.py, whose oracle and tolerances these are, does not go: both forms of
its kernel (one tile of queries a workgroup, or four) for the shared pages and the sequences' own, in each type and head_dim
(test_attention_plans_cpu.py holds that these calls take them); row starts and groups that cannot be."""
import math

import pytest

from test_attention_plans_cpu import SHARED_TILES
from test_gpu_attention_shared import DIMS, PAGE, Call, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("end", [20, 51])
def test_a_member_with_rows_beyond_its_groups(name, end):
    """Row starts that go beyond the group's end and come back: the first sequence fits the host's bounds by itself, but
    not among the group's rows, which is all that the group's part of the work covers.  It is left as it was, flagged, as
    the second is, whose rows end before they start."""
    from paper_2512_14681_amd import jf
    c = Call([(2, [(10, 50), (5, 3)])], "grp3", name, seed=21, pad=(0, 4))
    c.start.copy_(_torch().tensor([0, 52 if end == 51 else 50, end], dtype=_torch().int32))
    c.run(max_rows=52, max_ctx=3 * PAGE)
    assert bool((c.result() == 7.0 * c.out.shape[0]).all())
    assert int(c.flags) == jf.JF_FLAG_CAPACITY


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("before", [0, 70])
def test_groups_that_overlap(name, before):
    """Group starts that decrease and leave a group over sequences of an earlier one, behind none or more groups than a
    wave looks at in one go: the earlier one is computed, what only the later one holds is left as it was."""
    from paper_2512_14681_amd import jf
    torch = _torch()
    c = Call([(1, [(g % 7, 1)]) for g in range(before)] + [(2, [(10, 3), (70, 1), (0, 2), (33, 2)]), (1, [(5, 1)]),
                                                           (3, [(1, 2), (100, 2)])], "grp3", name, seed=22)
    n = before
    # groups n: sequences n .. n + 3; n + 1: ends before it starts; n + 2: n + 2 .. n + 6
    c.seq_start[n + 1:].copy_(torch.tensor([n + 4, n + 2, n + 7], dtype=torch.int32))
    c.pages[n + 2] = 0           # nothing else is wrong with it
    value, bound = c.reference()
    c.run(group_rows=20)
    got = c.result()
    last = int(c.starts[n + 4])
    assert bool(((got[:last] - value[:last]).abs() <= bound[:last]).all())
    assert bool((got[last:] == 7.0 * c.out.shape[0]).all())
    assert int(c.flags) == jf.JF_FLAG_CAPACITY


# ---- both forms on either side ----------------------------------------------------------
def tile_call(wide, name, hd, **kw):
    groups, loners, H, G = SHARED_TILES[wide]
    DIMS[f"tiles{hd}"] = (H, G, hd)
    return Call(groups, f"tiles{hd}", name, loners=loners, **kw)


FORMS = pytest.mark.parametrize("wide", SHARED_TILES, ids=str)
TYPES = pytest.mark.parametrize("name,hd", [(n, d) for n in ("bf16", "f32") for d in (32, 64, 128)])


@FORMS
@TYPES
@pytest.mark.parametrize("tree", [False, True])
def test_every_form(wide, name, hd, tree):
    tile_call(wide, name, hd, seed=31, tree=tree).run().check()


@FORMS
@TYPES
def test_rows_that_see_nothing_in_the_step(wide, name, hd):
    tile_call(wide, name, hd, seed=32, empty=(0, 2, 33)).run().check()


@FORMS
@TYPES
@pytest.mark.parametrize("shared", [True, False])
def test_bad_pages(wide, name, hd, shared):
    """Entries outside the pool among the shared pages (the first, one in the middle, the last: seen by none of the group)
    or among a sequence's own, whose last one holds the step's rows: flagged, their slots seen by nobody."""
    from paper_2512_14681_amd import jf
    c = tile_call(wide, name, hd, seed=33)
    bad = []
    for s, (p, ctx, r) in enumerate(c.members):
        need = (p * PAGE + ctx + r + PAGE - 1) // PAGE
        for i, b in enumerate(sorted({0, p // 2, p - 1}) if shared and p else () if shared else sorted({p, need - 1})):
            bad.append((s, b, (-1, 1 << 30, -7)[(s + i) % 3]))
    for s, b, entry in bad:
        c.table_np[s, b] = entry
    c.table.copy_(_torch().from_numpy(c.table_np))
    for s, b, _ in bad:
        c.table_np[s, b] = -7       # never a page's number
    c.run()
    value, bound = c.reference(drop=[-7])
    assert bool(((c.result() - value).abs() <= bound).all())
    assert int(c.flags) == jf.JF_FLAG_BAD_PAGE


@FORMS
@TYPES
def test_what_a_row_does_not_see_does_not_reach_it(wide, name, hd):
    """A NaN and an infinity in a row's value, in the largest sequence's own pages, reach the rows that see it alone, in
    their dims of their KV head."""
    torch = _torch()
    c = tile_call(wide, name, hd, seed=34, tree=True)
    value, bound = c.reference()
    s = max(range(len(c.members)), key=lambda i: c.members[i][2])
    p, ctx, rows = c.members[s]
    at = p * PAGE + ctx + 2                                   # in-step row 2
    n = c.G * PAGE * c.hd
    values = c.kv[int(c.table_np[s, at // PAGE]), n:].view(c.G, c.hd, PAGE)
    values[0, 3, at % PAGE], values[0, c.hd - 12, at % PAGE] = math.nan, math.inf
    c.run()
    got = c.result()
    ok = ((got - value).abs() <= bound).numpy()
    grp = c.H // c.G
    seen = 0
    for i in range(rows):
        row = int(c.starts[s]) + i
        if c.masks[s][i, 2]:
            seen += 1
            # two bf16 planes hold no infinity: hi = inf, lo = inf - inf
            assert bool(got[row, :grp, 3].isnan().all()) and not bool(got[row, :grp, c.hd - 12].isfinite().any()), i
            ok[row, :grp, [3, c.hd - 12]] = True
    assert ok.all() and 0 < seen < rows
    assert int(c.flags) == 0


def rising(slots, name, first=2.0 ** 17):
    """Numbers of the type, each 2^-7 or 2^-8 above the one of the slot before."""
    torch = _torch()
    bits = torch.tensor(first).to(torch.bfloat16).view(torch.int16).int() + slots.int()
    return bits.to(torch.int16).view(torch.bfloat16).double()


@FORMS
@TYPES
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_beyond_what_fp32_tells_apart(wide, name, hd, sign):
    """Scores from 2^30 on, 2^22 and more apart, the largest in the shared pages or in a sequence's own: it has all the
    weight (in two terms, and the result too: 2^-17 each, 2^-24 in fp32; product, quotient, merges: 12 steps of 2^-24);
    sums of values of 2^126 have a mean that fits.  Equal scores share the weight."""
    torch = _torch()
    c = tile_call(wide, name, hd, seed=35)
    n = c.G * PAGE * c.hd
    c.q.zero_()
    c.q[0, :, :, 0] = 2.0 ** 17
    c.q64 = c.q.double().sum(0).cpu()
    for s, (p, ctx, r) in enumerate(c.members):
        for b in range((p * PAGE + ctx + r + PAGE - 1) // PAGE):
            page = int(c.table_np[s, b])
            c.k[page] = 0.0
            c.k[page, :, :, 0] = sign * rising(torch.arange(b * PAGE, b * PAGE + PAGE), name)
            c.v[page] = torch.where(c.v[page].isnan(), c.v[page], 2.0 ** 126 * torch.sign(c.v[page]))
    c.kv[:, :n] = c.k.reshape(len(c.k), -1).to(c.kv.dtype).cuda()
    c.kv[:, n:] = c.v.transpose(2, 3).reshape(len(c.v), -1).to(c.kv.dtype).cuda()
    c.run()
    got = c.result()
    u = 2.0 ** -17 if name == "bf16" else 2.0 ** -24
    for s, (p, ctx, r) in enumerate(c.members):
        for i in range(r):
            at = p * PAGE + ctx + i if sign > 0 else 0
            v = c.v[int(c.table_np[s, at // PAGE]), :, at % PAGE].repeat_interleave(c.H // c.G, 0)
            err = (got[int(c.starts[s]) + i] - v).abs()
            assert bool((err <= (2 * u + 12 * 2.0 ** -24) * v.abs()).all()), (s, i)
    c.q.zero_()
    c.q64 = c.q.double().sum(0).cpu()
    c.flags.zero_()
    c.run().check()


def test_a_batch_of_wide_steps_without_a_prefix():
    """The plain batched attention over a bf16 or fp32 cache: nobody shares, some sequences' rows fill four tiles."""
    for name, hd in (("bf16", 128), ("f32", 64)):
        DIMS[f"tiles{hd}"] = (16, 2, hd)
        Call([], f"tiles{hd}", name, seed=36, loners=[(700, 140), (0, 129), (64, 1), (3, 512)]).run(shared=False).check()


@pytest.mark.parametrize("loners", [[(10, 140)] * 60, [(10, 1), (90, 3)] * 150], ids=["four tiles", "one"])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_batches_whose_pages_are_not_split(loners, name):
    """So many sequences that each one's pages are one part: outputs without a merge."""
    from paper_2512_14681_amd import jf
    c = Call([], "grp8", name, seed=37, loners=loners)
    assert jf.attention_shared_ws_bytes(c.descriptors()[0], None, c.H, c.G, c.hd) == 256
    c.run(shared=False).check()
