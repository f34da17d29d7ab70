"""Ties of the alternatives between -0 and +0, which are one value: the lowest id comes first, whatever the sign and
however the row is split."""
import numpy as np
import pytest

from oracle import batch as ob

pytestmark = pytest.mark.gpu


def top_ids(x, k):
    import torch
    from paper_2512_14681_amd import jf
    R, V = x.shape
    ids, lp = torch.empty(R, k, dtype=torch.int32, device="cuda"), torch.empty(R, k, device="cuda")
    ws = torch.empty(jf.token_logprobs_ws_bytes(R, V, k), dtype=torch.uint8, device="cuda")
    jf.token_logprobs(x, ws, k=k, d_top_ids=ids, d_top_logprob=lp)
    return ids.cpu().numpy(), lp.cpu().numpy()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,V", [(1, 3), (2, 700), (3, 9000), (1100, 9000), (2, 152064)])
@pytest.mark.parametrize("few", [False, True])
def test_signed_zeros_tie(dtype, R, V, few):
    """few: a -0, a +0 and another -0 in places far apart among negative logits; else half of all logits are zeros."""
    import torch
    rng = np.random.default_rng([R, V, few])
    x = -1.0 - rng.random((R, V))
    if few:
        at = np.sort(rng.random((R, V)).argpartition(min(3, V) - 1, 1)[:, :3], 1)
        np.put_along_axis(x, at, np.array([-0.0, 0.0, -0.0])[None], 1)
    else:
        zero = rng.random((R, V)) < 0.5
        x = np.where(zero, np.where(rng.random((R, V)) < 0.5, -0.0, 0.0), x)
    d = torch.tensor(x, dtype=torch.float32).to(getattr(torch, dtype)).cuda()
    x = d.double().cpu().numpy()
    for k in (1, 3, 20):
        ids, lp = top_ids(d, k)
        for r in range(0, R, max(R // 7, 1)):
            want = np.lexsort((np.arange(V), -x[r]))[:k]
            assert np.array_equal(ids[r][:len(want)], want), (k, r)
            m = x[r].max()
            ls = np.log(np.exp(x[r] - m).sum())
            # (x - m) - log s in fp32, the sum of fp32 exponentials: 2^-20 of numbers below 16
            assert np.abs(lp[r][:len(want)] - (x[r][want] - m - ls)).max() <= 2.0 ** -16


def test_the_row_of_three():
    import torch
    x = torch.tensor([[-0.0, 0.0, -1.0]], device="cuda")
    assert top_ids(x, 3)[0].tolist() == [[0, 1, 2]]
    assert ob.token_logprobs(x.double().cpu().numpy(), [-1], 3)[3].tolist() == [[0, 1, 2]]
