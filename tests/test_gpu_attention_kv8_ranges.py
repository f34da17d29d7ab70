"""jf_attention_kv8 where the numbers of a cache lie far apart: what a row does not see changes nothing for it, and what it
sees counts relative to the largest value that it sees.

Bounds, per row and KV head: a score from queries in two fp16 terms (2^-20 of the row's largest element), hd products summed
in fp32 and the exponent's argument rounded to 2^-23; weights in two fp16 terms (2^-20); sums over the pages in fp32.  All
relative to the largest value among the slots that the row sees."""
import numpy as np
import pytest

from oracle import batch as ob

pytestmark = pytest.mark.gpu


def words(vis):
    import torch
    bits = np.zeros((len(vis), 512), bool)
    bits[:, :vis.shape[1]] = vis
    w = np.packbits(bits.reshape(len(vis), 8, 64), axis=2, bitorder="little").view(np.uint64).reshape(len(vis), 8)
    return torch.tensor(w.view(np.int64)).cuda()


def attend(G, grp, hd, C, vis, k, v, q):
    """(outputs [rows][H][hd], keys and values as the pool holds them) of one sequence."""
    import torch
    from paper_2512_14681_amd import jf
    n, H = len(vis), G * grp
    pages = -(-(C + n) // 64)
    table = np.random.default_rng(n).permutation(pages + 1)[None, :pages].astype(np.int32)
    pool = ob.Pool8(np.zeros((pages + 1, ob.page_bytes(G, hd)), np.uint8), G, hd)
    ob.append(pool, [0, C + n], [0], table, k, v)
    i32 = dict(dtype=torch.int32, device="cuda")
    b = jf.Batch(torch.tensor([0, n], **i32), torch.tensor([C], **i32), torch.tensor(table, **i32), n, n, 64 * pages, pages + 1)
    out = torch.zeros((n + 15) // 16 * 16 * H * hd, device="cuda")
    ws = torch.empty(jf.attention_kv8_ws_bytes(b, H, G, hd), dtype=torch.uint8, device="cuda")
    jf.attention_kv8(b, H, G, hd, jf.JF_F32, torch.tensor(q[None], dtype=torch.float32).cuda(), torch.tensor(pool.raw).cuda(),
                     out, ws, d_vis=words(vis))
    held = [ob.gather(pool, table[0], C + n, G, kind) for kind in (0, 1)]
    return jf.act_unlayout(out.cpu().numpy(), n, H * hd).reshape(n, H, hd), held


def check(G, grp, hd, C, vis, k, v, q):
    q = np.asarray(q, np.float32).astype(np.float64)
    got, (hk, hv) = attend(G, grp, hd, C, vis, k, v, q)
    want = ob.attention(q, hk, hv, C, vis)
    sees = np.concatenate([np.ones((len(vis), C), bool), vis], 1)
    for i in range(len(vis)):
        js = np.nonzero(sees[i])[0]
        if not len(js):
            assert (got[i] == 0).all()
            continue
        for h in range(G * grp):
            kk, vv = hk[js, h // grp], hv[js, h // grp]
            score = np.abs(q[i, h]).max() * np.abs(kk).sum(1).max() / np.sqrt(hd)
            d = score * (2.0 ** -20 + hd * 2.0 ** -24) + score * 2.0 ** -23 + 2.0 ** -22
            rel = 2 * d + 2.0 ** -20 + (sees.shape[1] / 64 + 64) * 2.0 ** -24
            bound = rel * np.abs(vv).max() + np.abs(want[i, h]) * 2.0 ** -24
            assert (np.abs(got[i, h] - want[i, h]) <= bound).all(), (i, h)


@pytest.mark.parametrize("big", [1e4, 1e12, 1e30])
@pytest.mark.parametrize("hd,grp,C,n", [(64, 4, 0, 200), (128, 7, 70, 150), (32, 2, 130, 300), (64, 1, 60, 14), (128, 2, 0, 140)])
def test_values_that_a_row_does_not_see(hd, grp, C, n, big):
    """Some rows' values are `big` times the others' and visible to those rows alone, in pages before and after."""
    rng = np.random.default_rng([hd, n])
    G = 2
    vis = np.zeros((n, n), bool)
    large = np.zeros(n, bool)
    large[[0, 3, n // 2, n - 1]] = True
    for i in range(n):
        vis[i, max(i - 3, 0):i + 1] = True
    vis &= ~large[None] | np.eye(n, dtype=bool)
    vis[5] = False
    k = rng.normal(size=(C + n, G, hd))
    v = rng.normal(size=(C + n, G, hd))
    v[C:][large] *= big
    check(G, grp, hd, C, vis, k, v, rng.normal(size=(n, G * grp, hd)))


@pytest.mark.parametrize("big", [1e4, 1e12, 1e30])
@pytest.mark.parametrize("n", [1, 4, 40])
def test_scales_apart_in_pages_that_all_rows_see(n, big):
    """Committed pages of values `big` apart, large ones first, last and between."""
    rng = np.random.default_rng(n)
    G, grp, hd, C = 2, 4, 64, 64 * 12 + 5
    v = rng.normal(size=(C + n, G, hd))
    v[128:192] *= big
    v[600:640] *= big
    check(G, grp, hd, C, np.tril(np.ones((n, n), bool)), rng.normal(size=(C + n, G, hd)), v, rng.normal(size=(n, G * grp, hd)))


@pytest.mark.parametrize("qs,ks", [(1e-30, 1e-15), (1e-25, 1e-25), (0.0, 1e-30), (1e-38, 1e-30)])
@pytest.mark.parametrize("hd,grp,C,n", [(64, 4, 70, 3), (128, 7, 0, 2), (32, 2, 100, 40), (128, 2, 64, 150)])
def test_scores_below_the_smallest_number(hd, grp, C, n, qs, ks):
    """Queries and keys so small that every score is 0: the mean of the values that a row sees, no more of the others."""
    rng = np.random.default_rng([hd, n])
    G = 2
    vis = np.tril(rng.random((n, n)) < 0.6)
    vis[0] = False
    check(G, grp, hd, C, vis, rng.normal(size=(C + n, G, hd)) * ks, rng.normal(size=(C + n, G, hd)),
          rng.normal(size=(n, G * grp, hd)) * qs)


@pytest.mark.parametrize("qs,ks", [(1e5, 1.0), (1e8, 1.0), (1e9, 3.0), (1e10, 1e3), (1e15, 1e15)])
@pytest.mark.parametrize("hd,grp,C,n", [(64, 4, 700, 3), (128, 7, 300, 2), (32, 2, 100, 40), (128, 2, 640, 150)])
def test_scores_of_any_size(hd, grp, C, n, qs, ks):
    """Scores far beyond what fp32 tells apart: nothing overflows, and the outputs are means of the values that a row sees."""
    rng = np.random.default_rng([hd, n])
    G = 2
    vis = np.tril(rng.random((n, n)) < 0.6)
    vis[0] = False
    check(G, grp, hd, C, vis, rng.normal(size=(C + n, G, hd)) * ks, rng.normal(size=(C + n, G, hd)),
          rng.normal(size=(n, G * grp, hd)) * qs)


@pytest.mark.parametrize("hd,grp,C,n", [(64, 4, 700, 3), (128, 7, 300, 2), (32, 2, 100, 40), (128, 2, 640, 150)])
@pytest.mark.parametrize("vs", [1e30, 1e35, 2e37, 1e-30])
def test_values_of_any_size(hd, grp, C, n, vs):
    """Values close to fp32's largest: their mean is a number, whatever the sum of the weights."""
    rng = np.random.default_rng([hd, n])
    G = 2
    check(G, grp, hd, C, np.tril(np.ones((n, n), bool)), rng.normal(size=(C + n, G, hd)),
          np.clip(rng.normal(size=(C + n, G, hd)), -4, 4) * vs, rng.normal(size=(n, G * grp, hd)))
