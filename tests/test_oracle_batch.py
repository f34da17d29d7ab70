"""Pins of oracle/batch.py: the e4m3 rounding against the type's own
conversion, the page layout as a permutation, the rotation as complex turns,
the log probabilities against torch in 64 bits, and the gradient against
differences."""
import numpy as np
import pytest
import torch

from oracle import batch as ob


def test_e4m3_values_and_rounding():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ob.E4M3, want, equal_nan=True)
    pos = ob.E4M3[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([pos, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), [1e30, np.inf]])
    x = np.concatenate([x, -x])
    # in 64 bits on both sides of the midpoints; the type's conversion takes
    # fp32, where the neighbours collapse onto them
    f = x.astype(np.float32)
    ok = f.astype(np.float64) == x
    want = torch.from_numpy(np.clip(f, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert ok.sum() > 400 and np.array_equal(ob.round_e4m3(x)[ok], want[ok])
    n = len(pos) + len(mid)
    below, above = ob.round_e4m3(x[n:n + len(mid)]), ob.round_e4m3(x[n + len(mid):n + 2 * len(mid)])
    assert np.array_equal(below, np.arange(126)) and np.array_equal(above, np.arange(1, 127))
    assert ob.round_e4m3(np.array([np.nan]))[0] == 127


@pytest.mark.parametrize("top,scale", [(0.0, 1.0), (448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (223.9, 0.5),
                                       (224.1, 1.0), (1.0, 2.0 ** -8), (0.875, 2.0 ** -9)])
def test_block_scale(top, scale):
    assert ob.block_scale(np.array([0.0, -top, np.nan, np.inf])) == scale


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_page_layout_is_a_permutation(hd):
    t, i = np.meshgrid(np.arange(64), np.arange(hd), indexing="ij")
    for off in (ob.key_offset(t, i, hd), ob.value_offset(t, i)):
        assert sorted(off.reshape(-1).tolist()) == list(range(64 * hd))
    assert ob.page_bytes(4, hd) % 128 == 0 and ob.page_bytes(4, hd) >= 8 * 64 * hd + 32


def test_append_keeps_and_requantises():
    G, hd = 2, 32
    pool = ob.Pool8(np.zeros((2, ob.page_bytes(G, hd)), np.uint8), G, hd)
    rng = np.random.default_rng(0)
    a = rng.normal(size=(10, G, hd))
    ob.append(pool, [0, 10], [0], [[1, 0]], a, a)
    first = pool.values(1, 0, 0)[:10]
    assert np.abs(first - a[:, 0]).max() <= 2.0 ** -4 * np.abs(a).max()
    big = 100 * rng.normal(size=(60, G, hd))       # on into the next page, on a larger scale
    ob.append(pool, [0, 60], [10], [[1, 0]], big, big)
    got = ob.gather(pool, [1, 0], 70, G, 1)
    assert np.abs(got[10:] - big).max() <= 2.0 ** -4 * np.abs(big).max()
    # a power of two larger leaves what stays in the normal range as it was
    normal = np.abs(first) >= 2.0 ** -6 * pool.scale(1, 0, 0)
    assert normal.mean() > 0.5 and np.array_equal(pool.values(1, 0, 0)[:10][normal], first[normal])


def test_rotation_is_a_turn():
    rng = np.random.default_rng(1)
    x, pos = rng.normal(size=(5, 3, 64)), np.array([0, 1, 77, 100000, 1000001])
    y = ob.rotate(x, pos, 1e4)
    z = (x[..., :32] + 1j * x[..., 32:]) * np.exp(1j * pos[:, None, None] * 1e4 ** (-np.arange(32) / 32))
    assert np.allclose(y, np.concatenate([z.real, z.imag], -1), rtol=0, atol=1e-9)
    assert np.array_equal(y[0], x[0]) and np.array_equal(ob.rotate(x, pos, 0.0), x)


def test_logprobs_against_torch():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(6, 97)) * 3
    x[1, ::3] = -np.inf
    x[3] = np.round(x[3])                          # ties
    tok = np.array([5, 1, -1, 96, 0, 200])
    lp, ent, norm, ids, top = ob.token_logprobs(x, tok, 7)
    want = torch.log_softmax(torch.from_numpy(x), 1)
    assert np.allclose(lp[[0, 1, 3, 4]], [want[r, tok[r]] for r in (0, 1, 3, 4)], atol=1e-12)
    assert lp[2] == 0 and np.isnan(lp[5])
    p = want.exp()
    assert np.allclose(ent, torch.special.entr(p).sum(1), atol=1e-12)
    assert np.allclose(norm.sum(1), torch.logsumexp(torch.from_numpy(x), 1), atol=1e-12)
    vals, order = torch.sort(torch.from_numpy(x), dim=1, descending=True, stable=True)
    assert np.array_equal(ids, order[:, :7]) and np.allclose(top, torch.gather(want, 1, order[:, :7]), atol=1e-12)
    bad = np.array([[-np.inf] * 4, [1, np.nan, 0, 0], [np.inf, 0, 0, 0]])
    lp, ent, norm, ids, top = ob.token_logprobs(bad, [0, 0, 0], 2)
    assert np.isnan(lp).all() and np.isnan(ent).all() and np.isnan(top).all() and (ids == -1).all()


def test_gradient_against_differences():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(4, 23))
    x[2, 5] = -np.inf
    tok, g, h = np.array([3, 22, 0, -1]), np.array([1.5, -0.25, 0.0, 2.0]), np.array([0.0, 0.7, -1.1, 0.3])

    def loss(y):
        lp, ent, *_ = ob.token_logprobs(y, tok, 0)
        return (g * lp + h * ent).sum()
    grad, d = ob.token_logprobs_grad(x, tok, g, h), 1e-6
    for r in range(4):
        for j in range(23):
            if x[r, j] == -np.inf:
                assert grad[r, j] == 0
                continue
            up, down = x.copy(), x.copy()
            up[r, j] += d
            down[r, j] -= d
            # a difference over 2 d: truncation d^2, rounding 2^-52 * |loss| / d
            assert abs((loss(up) - loss(down)) / (2 * d) - grad[r, j]) < 1e-8
