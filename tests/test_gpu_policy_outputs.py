"""jf_policy_loss where only some of its outputs are asked for: the others are what they are with all of them."""
import pytest

from test_gpu_policy_loss import Call, case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [20, 6000])     # one launch, and several
@pytest.mark.parametrize("mean", ["tokens", "seqs", "sum"])
@pytest.mark.parametrize("without", [("g_lp",), ("g_entropy",), ("g_lp", "g_entropy")])
def test_without_some_gradients(size, mean, without):
    c = case([size, size // 2, 3], seed=3, mean=mean, before=2, after=3)
    full, some = Call(c), Call(c)
    full.run()
    kept = {n: getattr(some, n) for n in without}
    for n in without:
        setattr(some, n, None)
    some.run()
    for n in ("stats", "g_lp", "g_entropy"):
        if n not in without:
            assert bool((getattr(some, n) == getattr(full, n)).all()), n
    for t in kept.values():
        assert bool((t == 7.0).all())
    assert int(some.flags) == 0
