"""jf_attention_causal and its gradient where test_gpu_attention_causal.py, whose oracle and tolerances these are, does not
go: row starts that leave sequences over each other, gradients of scores that are no numbers."""
import math

import pytest

from test_gpu_attention_causal import DIMS, Call, case, close, reference

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
