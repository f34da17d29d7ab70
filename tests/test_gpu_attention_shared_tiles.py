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
