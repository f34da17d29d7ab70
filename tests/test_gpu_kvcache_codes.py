"""The codes that jf_kv_append writes into an e4m3 page are those of the exact values: values are divided by a power of two
and rounded once, keys are turned in 64 bits and rounded once.

A turned key u cos a - w sin a: the oracle's angle is off by some 2^-53 of its radians, below 2^-40 for positions here, the
kernel's sine and cosine by 1.2e-10 (their polynomials' first left-out terms, (pi / 4)^12 / 12! and (pi / 4)^13 / 13!), so both
are within EPS (|u| + |w|) of each other with EPS = 2.5e-10.  A code may differ only where the value is that close to the
middle between two."""
import numpy as np
import pytest

from oracle import batch as ob

pytestmark = pytest.mark.gpu
EPS = 2.5e-10
MIDDLES = (ob.E4M3[:126] + ob.E4M3[1:127]) / 2


def middle_distance(a):
    """Distance of |a| to the nearest middle between two e4m3 values."""
    a = np.abs(a)
    i = np.clip(np.searchsorted(MIDDLES, a), 1, len(MIDDLES) - 1)
    return np.minimum(np.abs(a - MIDDLES[i - 1]), np.abs(a - MIDDLES[i]))


def append(k, v, G, hd, base, ctx=0, pos=None, x="float32"):
    """The rows [n][G][hd] after ctx committed tokens (scale 2^-20, codes 0) in a pool of their own: (pool, page table)."""
    import torch
    from paper_2512_14681_amd import jf
    n = len(k)
    pages = -(-(ctx + n) // 64)
    table = np.random.default_rng(n).permutation(pages)[None].astype(np.int32)
    raw = np.zeros((pages, ob.page_bytes(G, hd)), np.uint8)
    raw[:, 2 * G * 64 * hd:][:, :8 * G] = np.full((pages, 2 * G), 2.0 ** -20, np.float32).view(np.uint8)
    i32 = dict(dtype=torch.int32, device="cuda")
    b = jf.Batch(torch.tensor([0, n], **i32), torch.tensor([ctx], **i32), torch.tensor(table, **i32), n, n, 64 * pages, pages)
    d = torch.tensor(raw).cuda()
    rows = [torch.tensor(t.reshape(n, G * hd), dtype=torch.float32).to(getattr(torch, x)).cuda() for t in (k, v)]
    jf.kv_append(b, G, G, hd, jf.JF_E4M3, d, *rows, rope_base=base,
                 d_pos=None if pos is None else torch.tensor(pos, **i32))
    want = ob.Pool8(raw, G, hd)
    ob.append(want, [0, n], [ctx], table, *(r.double().cpu().numpy().reshape(n, G, hd) for r in rows), base, pos)
    return ob.Pool8(d.cpu().numpy(), G, hd), want, table[0]


def compare(got, want, table, k, G, hd, base, ctx=0, pos=None):
    """Scales and value codes equal; key codes equal except where 64 bits cannot tell.  Returns how many those are."""
    n = len(k)
    slots = ctx + np.arange(n)
    turned = ob.rotate(k, slots if pos is None else pos, base)
    mag = np.abs(k.reshape(n, G, 2, hd // 2)).sum(2)
    mag = np.concatenate([mag, mag], -1)
    unsure = 0
    o = 2 * G * 64 * hd
    assert np.array_equal(got.raw[:, o:], want.raw[:, o:])
    for p, page in enumerate(table):
        for g in range(G):
            at = got.at[1][g]
            assert np.array_equal(got.raw[page, at], want.raw[page, at])
            at = got.at[0][g]
            differ = got.raw[page, at] != want.raw[page, at]
            mine = np.nonzero(slots // 64 == p)[0]
            t = slots[mine] % 64
            s = got.scale(page, g, 0)
            near = np.zeros((64, hd), bool)
            near[t] = middle_distance(turned[mine, g] / s) <= EPS * mag[mine, g] / s
            near[t] &= bool(base) & (turned[mine, g] != k[mine, g])     # what is not turned is exact
            assert not (differ & ~near).any(), (p, g)
            unsure += int(near.sum())
    return unsure


@pytest.mark.parametrize("hd,G,ctx,n,base", [(128, 4, 0, 4000, 1e6), (64, 2, 1000, 3000, 1e4), (32, 4, 63, 500, 1e4),
                                             (128, 1, 10, 700, 0.0)])
@pytest.mark.parametrize("x", ["float32", "bfloat16"])
def test_codes_are_those_of_the_exact_values(hd, G, ctx, n, base, x):
    import torch
    rng = np.random.default_rng([hd, n])
    k, v = (torch.tensor(rng.normal(size=(n, G, hd)) * np.exp2(rng.integers(-4, 5, (n, G, 1))), dtype=torch.float32)
            .to(getattr(torch, x)).double().numpy() for _ in range(2))
    got, want, table = append(k, v, G, hd, base, ctx, x=x)
    unsure = compare(got, want, table, k, G, hd, base, ctx)
    # a middle is met within EPS |k| / scale by one element in some 10^7
    assert unsure <= 3


def directed(base, hd, seed):
    """Keys [64][1][hd] of tokens at positions 1 .. 64 whose first halves turn to within 2^-26 .. 2^-37 of a middle between
    two codes of scale 1, to either side, and never nearer than the kernel's 64 bits can tell."""
    rng = np.random.default_rng(seed)
    half, n = hd // 2, 64
    pos = 1 + np.arange(n)
    ang = pos[:, None] * base ** (-2.0 * np.arange(half) / hd)
    c, s = np.cos(ang), np.sin(ang)
    k = np.zeros((n, 1, hd))
    left = np.ones((n, half), bool)
    for _ in range(400):
        middle = MIDDLES[rng.integers(40, 112, (n, half))]
        w = np.float32(rng.normal(size=(n, half)) * middle / 4).astype(np.float64)
        with np.errstate(divide="ignore", invalid="ignore"):
            u = np.float32((middle + w * s) / c).astype(np.float64)
        y = u * c - w * s
        off = np.abs(y - middle)
        ok = left & (np.abs(u) < 300) & (off < 2.0 ** -26 * middle) & (off > 2 * EPS * (np.abs(u) + np.abs(w)))
        k[:, 0, :half][ok], k[:, 0, half:][ok] = u[ok], w[ok]
        left &= ~ok
    k[0, 0, :half], k[0, 0, half:] = 0.0, 0.0
    # sets the scale: turned back by its own angle, it is 300 exactly enough to lie between 224 and 448
    k[0, 0, 0], k[0, 0, half] = 300 * c[0, 0], -300 * s[0, 0]
    return np.float32(k).astype(np.float64), pos.astype(np.int32), ~left


@pytest.mark.parametrize("hd,base", [(128, 1e6), (64, 1e4), (32, 1e4)])
def test_keys_next_to_the_middle_between_two_codes(hd, base):
    """A key rounded to 32 bits first lies on the middle itself, and goes to the even code whatever side it came from."""
    k, pos, found = directed(base, hd, hd)
    assert found.mean() > 0.3
    turned = ob.rotate(k, pos, base)
    assert ob.block_scale(turned) == 1.0
    exact = ob.round_e4m3(turned)
    twice = ob.round_e4m3(np.float32(turned).astype(np.float64))
    wrong = int((exact != twice).sum())
    assert wrong > 0.02 * found.sum()          # what one more rounding would get wrong
    got, want, table = append(k, k, 1, hd, base, 0, pos)
    assert got.scale(table[0], 0, 0) == 1.0
    compare(got, want, table, k, 1, hd, base, 0, pos)


@pytest.mark.parametrize("hd,base", [(128, 1e6), (64, 1e4)])
def test_keys_of_an_fp32_cache_are_rounded_once(hd, base):
    """Half a step of fp32 and the 64-bit arithmetic's EPS: no more."""
    import torch
    from paper_2512_14681_amd import jf
    n, G = 3000, 2
    rng = np.random.default_rng(hd)
    k = torch.tensor(rng.normal(size=(n, G, hd)), dtype=torch.float32)
    pages = -(-n // 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.arange(pages, **i32)[None]
    b = jf.Batch(torch.tensor([0, n], **i32), torch.zeros(1, **i32), table, n, n, 64 * pages, pages)
    pool = torch.zeros(pages, 2 * G * 64 * hd, device="cuda")
    d = k.view(n, G * hd).cuda()
    jf.kv_append(b, G, G, hd, jf.JF_F32, pool, d, d, rope_base=base)
    got = ob.gather(ob.PoolDense(pool.double().cpu().numpy(), G, hd), list(range(pages)), n, G, 0)
    k = k.double().numpy()
    want = ob.rotate(k, np.arange(n), base)
    mag = np.abs(k.reshape(n, G, 2, hd // 2)).sum(2)
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + EPS * np.concatenate([mag, mag], -1)).all()


@pytest.mark.parametrize("hd,G", [(32, 3), (64, 2), (128, 2)])
@pytest.mark.parametrize("t0", [1, 3, 17, 63])
def test_zeros_hold_nobody_to_their_scale(hd, G, t0):
    """Tokens of 0 (either sign) get scale 1; small ones appended after them get their own, whatever stands in the slots
    behind.  Kept NaN and saturated infinities, which have scale 1 for want of finite values, keep it."""
    import torch
    from paper_2512_14681_amd import jf
    rng = np.random.default_rng([hd, t0])
    n = 70 - t0
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.tensor([[1, 0]], **i32)
    for kept in (0.0, -0.0, np.nan, np.inf, "one"):
        raw = rng.integers(0, 127, (2, ob.page_bytes(G, hd))).astype(np.uint8)      # what an earlier sequence left
        d, want = torch.tensor(raw).cuda(), ob.Pool8(raw, G, hd)
        first = np.zeros((t0, G, hd))
        first[:, 0] = 300.0 if kept == "one" else kept      # head 0 alone; a value that has scale 1 by itself
        rest = rng.normal(size=(n, G, hd)) * 2.0 ** -12
        for at, rows in ((0, first), (t0, np.float32(rest).astype(np.float64))):
            b = jf.Batch(torch.tensor([0, len(rows)], **i32), torch.tensor([at], **i32), table, len(rows), len(rows), 128, 2)
            x = torch.tensor(rows.reshape(len(rows), -1), dtype=torch.float32).cuda()
            jf.kv_append(b, G, G, hd, jf.JF_E4M3, d, x, -x)
            ob.append(want, [0, len(rows)], [at], [[1, 0]], rows, -rows)
        got = ob.Pool8(d.cpu().numpy(), G, hd)
        for g in range(G):
            for kind in (0, 1):
                small = g > 0 or kept == 0
                assert (got.scale(1, g, kind) == 1) == (not small) and got.scale(1, g, kind) <= 1
                a, b = (np.concatenate([w.values(1, g, kind), w.values(0, g, kind)])[:70] for w in (got, want))
                assert np.array_equal(a, b, equal_nan=True)
                if small:       # half a step of the values that are not subnormal on their scale
                    x = rest[:, g] * (-1 if kind else 1)
                    assert (np.abs(a[t0:64] - x[:64 - t0]) <= 2.0 ** -4 * np.abs(x[:64 - t0]) + 2.0 ** -10 * got.scale(1, g, kind)).all()
        assert np.array_equal(got.raw[0, :2 * G * 64 * hd], want.raw[0, :2 * G * 64 * hd])
