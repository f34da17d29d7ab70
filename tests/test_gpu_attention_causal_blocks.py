"""jf_attention_causal and its gradient where test_gpu_attention_causal.py, whose oracle and tolerances these are, does not
go: row starts that leave sequences over each other."""
import pytest

from test_gpu_attention_causal import Call, case, close, reference

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
