"""jf_attention_causal and its gradient where test_gpu_attention_causal.py, whose oracle and tolerances these are, does not
go: every kernel there is (blocks of 128, 64 and 32 rows of each type and head_dim; test_attention_plans_cpu.py holds that
these calls run on them), long sequences, far strides, row starts that leave sequences over each other, gradients of scores
that are no numbers."""
import math

import numpy as np
import pytest

from test_attention_plans_cpu import CAUSAL_BLOCKS, CAUSAL_SHARES
from test_gpu_attention_causal import DIMS, Call, _torch, case, close, dtype_of, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("starts,used", [
    ([0, 100, 50, 120], [(0, 100)]),
    ([0, 200, 150, 300, 410], [(0, 200), (300, 410)]),
    ([5, 60, 20, 70, 80, 10, 30], [(5, 60), (70, 80)]),
    ([0, 90, -3, 40, 90, 180, 500, 170, 200], [(0, 90), (90, 180)]),
])
@pytest.mark.parametrize("dims,name", [("grp3", "bf16"), ("tiny", "f32")])
def test_sequences_that_overlap(dims, name, starts, used):
    """Row starts that decrease, flagged: of the sequences that remain the earlier one has the rows, one that starts before
    its end is left alone, and no row is written twice."""
    from paper_2512_14681_amd import jf
    R = 410
    c = case([R], dims, name, seed=41)
    call = Call(c, starts, dims, name)
    call.forward()
    call.backward()
    got = call.results()
    assert int(call.flags) == jf.JF_FLAG_CAPACITY
    free = [True] * R
    for a, b in used:
        free[a:b] = [False] * (b - a)
        part = {n: (t[:, a:b] if n == "lse" else t[a:b]) for n, t in got.items()}
        close(part, reference({n: t[a:b] for n, t in c.items()}, [b - a], dims, name))
    for n in ("out", "dq", "dk", "dv"):
        assert bool((got[n][free] == 7.0).all()), n
    assert bool((got["lse"][:, free] == 7.0).all())


@pytest.mark.parametrize("dims,name", [("grp3", "bf16"), ("grp3", "f32"), ("tiny", "f32"), ("tiny", "bf16"), ("wide", "bf16")])
def test_a_nan_score_makes_gradients_nan(dims, name):
    """A NaN in row 70's query of one head: by the formulas the gradients of that query, and of the keys and values up to
    row 70 of the KV head that it reads, are NaN.  Values behind it, other KV heads, other rows' queries and the other
    sequence have what they have without it."""
    lens, at = [100, 141], 170   # row 70 of the second sequence
    c = case(lens, dims, name, seed=42)
    want = reference(c, lens, dims, name)
    H, G, hd = DIMS[dims]
    c["q"][at, 5] = math.nan
    call = Call(c, [0, 100, 241], dims, name)
    call.forward()
    call.backward()
    got = call.results()
    assert bool(got["dq"][at, :hd].isnan().all())
    for n in ("dk", "dv"):
        assert bool(got[n][100:at + 1, :hd].isnan().all()), n
    for n in ("dq", "dk", "dv"):
        ok = (got[n] - want[n][0]).abs() <= want[n][1]
        if n == "dq":
            ok[at, :hd] = True
        else:       # dk: 0 times the query, where a key is behind the row
            ok[100:241 if n == "dk" else at + 1, :hd] = True
        assert bool(ok.all()), n


# ---- every kernel -----------------------------------------------------------------------
def dims_of(H, G, hd):
    """The name of these dimensions in the oracle's table."""
    name = f"{H}+2x{G}x{hd}"
    DIMS[name] = (H, G, hd)
    return name


def block_case(name, hd, n, seed, std=1.5):
    """(lengths, starts, dims, inputs) of the call that runs on blocks of 32 n rows."""
    lens, H, G = CAUSAL_BLOCKS[name, hd, n]
    dims = dims_of(H, G, hd)
    return lens, np.cumsum([0] + lens).tolist(), dims, case(lens, dims, name, seed=seed, std=std)


BLOCKS = pytest.mark.parametrize("name,hd,n", CAUSAL_BLOCKS, ids=lambda x: str(x))


@BLOCKS
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (0, 3)])
def test_every_block_height(name, hd, n, offset, pad):
    """Rows on 16-byte boundaries, which go to LDS by themselves, and others, which pass registers."""
    lens, starts, dims, c = block_case(name, hd, n, seed=51)
    call = Call(c, starts, dims, name, offset=offset, pad=pad)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
    assert int(call.flags) == 0


@pytest.mark.parametrize("parts", CAUSAL_SHARES)
def test_shares_of_heads(parts):
    name, lens, H, G, hd = CAUSAL_SHARES[parts]
    dims = dims_of(H, G, hd)
    c = case(lens, dims, name, seed=52)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))


@BLOCKS
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
def test_later_rows_do_not_reach_earlier_ones(name, hd, n, where, bad):
    """An infinity or NaN in a key or value of the first sequence's row 333: the rows before it, the other sequences and the
    heads of other KV heads are as they were; what sees a value shows it in its dim alone (no weight is below e^-60)."""
    lens, starts, dims, c = block_case(name, hd, n, seed=53)
    at, dim = 333, 5
    value, bound = reference(c, lens, dims, name)["out"]
    c[where][at, dim] = bad
    call = Call(c, starts, dims, name)
    call.forward()
    got = call.results()["out"]
    H, G, _ = DIMS[dims]
    grp = H // G
    ok = (got - value).abs() <= bound
    first = got[at:lens[0], :grp * hd].reshape(-1, grp, hd)
    if where == "v":
        assert bool((first[:, :, dim].isnan() if math.isnan(bad) else first[:, :, dim] == bad).all())
        ok[at:lens[0], dim:grp * hd:hd] = True
    else:
        if math.isnan(bad):
            assert bool(first.isnan().all())
        ok[at:lens[0], :grp * hd] = True
    assert bool(ok.all())


@BLOCKS
def test_a_nan_score_reaches_its_gradients_alone(name, hd, n):
    """A NaN in row 333's query of the first head: the gradients of that query, and of the keys and values up to row 333 of
    the KV head that it reads, are NaN.  Values behind it, other KV heads, other rows' queries and the other sequences have
    what they have without it."""
    lens, starts, dims, c = block_case(name, hd, n, seed=54)
    at = 333
    want = reference(c, lens, dims, name)
    c["q"][at, 5] = math.nan
    call = Call(c, starts, dims, name)
    call.forward()
    call.backward()
    got = call.results()
    assert bool(got["dq"][at, :hd].isnan().all())
    for which in ("dq", "dk", "dv"):
        ok = (got[which] - want[which][0]).abs() <= want[which][1]
        if which == "dq":
            ok[at, :hd] = True
        else:       # dk: 0 times the query, where a key is behind the row
            assert bool(got[which][:at + 1, :hd].isnan().all()), which
            ok[:lens[0] if which == "dk" else at + 1, :hd] = True
        assert bool(ok.all()), which


def rising(n, name, first=2.0 ** 17):
    """n numbers of the type from `first` on, each 2^-7 or 2^-8 above the one before."""
    torch = _torch()
    bits = torch.tensor(first).to(torch.bfloat16).view(torch.int16).int() + torch.arange(n, dtype=torch.int32)
    return bits.to(torch.int16).view(torch.bfloat16).to(dtype_of(name))


@BLOCKS
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_beyond_what_fp32_tells_apart(name, hd, n, sign):
    """Scores from 2^30 on, 2^22 and more apart (the products are exact): the largest one that a row sees has all the weight.
    The weight and the result are rounded to the type (u each); the weight's product, the quotient and their product are
    fp32's (6 steps of 2^-24 at most).  Equal scores share the weight.  The gradients there have no digits but stay finite."""
    torch = _torch()
    lens, starts, dims, c = block_case(name, hd, n, seed=55)
    H, G, _ = DIMS[dims]
    u, f = 2.0 ** -8 if name == "bf16" else 2.0 ** -24, 2.0 ** -24
    for t in ("q", "k"):
        c[t].zero_()
    c["q"][:, ::hd] = 2.0 ** 17
    v = c["v"].double().reshape(-1, G, hd).repeat_interleave(H // G, 1).reshape(-1, H * hd)
    for a, b in zip(starts, starts[1:]):
        c["k"][a:b, ::hd] = sign * rising(b - a, name)[:, None]
    call = Call(c, starts, dims, name)
    call.forward()
    call.backward()
    got = call.results()
    largest = torch.cat([torch.arange(a, b) if sign > 0 else torch.full((b - a,), a) for a, b in zip(starts, starts[1:])])
    assert bool(((got["out"] - v[largest]).abs() <= (2 * u + 6 * f) * (1 + u) * v[largest].abs()).all())
    assert all(bool(got[t].isfinite().all()) for t in got)
    c["k"][:, ::hd] = sign * 2.0 ** 17
    call = Call(c, starts, dims, name)
    call.forward()
    got = call.results()["out"]
    for a, b in zip(starts, starts[1:]):
        count = torch.arange(1, b - a + 1)[:, None]
        mean, mag = v[a:b].cumsum(0) / count, v[a:b].abs().cumsum(0) / count
        assert bool(((got[a:b] - mean).abs() <= (2 * u + 500 * f) * (mag + mean.abs())).all())


@BLOCKS
def test_values_next_to_the_largest(name, hd, n):
    """Sums of many values of 2^127 have a mean that fits, whatever the order of the maxima."""
    torch = _torch()
    lens, starts, dims, c = block_case(name, hd, n, seed=56)
    c["v"] = (2.0 ** 127 * torch.sign(c["v"].double() + 2.5)).to(c["v"].dtype)
    value, bound = reference(dict(c, do=c["do"] * 0), lens, dims, name)["out"]
    call = Call(c, starts, dims, name)
    call.forward()
    assert bool(((call.results()["out"] - value).abs() <= bound).all())


# ---- far sizes --------------------------------------------------------------------------
def test_long_sequences_of_the_benchmark_heads():
    """More than a thousand rows of 28 and 4 heads of 128 dims, a few beside them: the 128-row kernels."""
    lens = [1100, 37, 700]
    c = case(lens, "7b", "bf16", seed=57)
    call = Call(c, np.cumsum([0] + lens).tolist(), "7b", "bf16")
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, "7b", "bf16"))


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_a_sequence_of_more_blocks_than_are_looked_through(name):
    """More than 256 blocks of 32 rows beside a short sequence on either side: one sequence after the other."""
    lens, dims = [45, 8300, 33], dims_of(1, 1, 32)
    c = case(lens, dims, name, seed=58)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))


@pytest.mark.parametrize("which", ["all", "do"])
@pytest.mark.parametrize("beyond", [0, 16])
@pytest.mark.parametrize("name,heads,lens", [("bf16", (6, 2, 64), [130, 3]), ("f32", (6, 2, 32), [130, 3]),
                                             ("bf16", (28, 4, 128), [130, 3] + [1] * 30)])
def test_rows_far_apart(name, heads, lens, beyond, which):
    """Strides of 2^22 elements, whose steps of 128 rows are within 31-bit offsets, and of 16 bytes more."""
    torch = _torch()
    dims = dims_of(*heads)
    c = case(lens, dims, name, seed=59)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    ld = 2 ** 22 + beyond // dtype_of(name).itemsize
    raw = torch.full((call.R * ld,), 7.0, dtype=dtype_of(name), device="cuda")
    at = 0
    for t in ("q", "k", "v", "do", "out", "dq", "dk", "dv") if which == "all" else ("do",):
        old = getattr(call, t)
        far = torch.as_strided(raw, old.shape, (ld, 1), at)
        at += old.shape[1]
        far.copy_(old)
        setattr(call, t, far)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
