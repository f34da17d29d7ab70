"""jf_attention_shared where it goes wrong most easily: row starts and groups that cannot be.  The oracle and its
tolerances are those of test_gpu_attention_shared.py."""
import pytest

from test_gpu_attention_shared import PAGE, Call, _torch

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
