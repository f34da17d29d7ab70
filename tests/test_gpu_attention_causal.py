"""jf_attention_causal and jf_attention_causal_grad against softmax attention in 64 bits.

Tolerances, from the arithmetic (u = half a step of the type: bf16 2^-8, fp32 2^-24):
* scores: sums of head_dim products in fp32, off by at most hd 2^-24 sum |q k| / sqrt(hd) = e; a weight p is off by
  2 e + n 2^-24 relative (score, sum) and a few steps of exp2, and is rounded to the type for the second product (u);
* out: off by (u + w) sum p |v| with w the weights' error, then rounded (u |out|);
* dv: the same with p^T and do;
* D = out . do takes the rounded out: off by u |out| |do| and out's own error times |do|, summed over head_dim;
* ds = p (dp - D): w |ds| + u |ds| + p (D's error + hd 2^-24 |do| |v|); dq and dk are sums of it times |k| and |q|, rounded.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

DIMS = {"7b": (28, 4, 128), "grp3": (6, 2, 64), "tiny": (4, 4, 32), "wide": (8, 1, 128), "one": (1, 1, 64)}


def _torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def dtype_of(name):
    torch = _torch()
    return torch.float32 if name == "f32" else torch.bfloat16


def rows(shape, name, seed, std=1.0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std).to(dtype_of(name))


def case(lens, dims, name, seed=0, std=1.5):
    H, G, hd = DIMS[dims]
    R = sum(lens)
    return dict(q=rows((R, H * hd), name, seed, std), k=rows((R, G * hd), name, seed + 1), v=rows((R, G * hd), name, seed + 2),
                do=rows((R, H * hd), name, seed + 3))


def reference(c, lens, dims, name):
    """{output: (value, bound)} in 64 bits on the CPU; rows of the sequences one after the other."""
    torch = _torch()
    H, G, hd = DIMS[dims]
    u, f = (2.0 ** -8 if name == "bf16" else 2.0 ** -24), 2.0 ** -24
    x = {n: t.double() for n, t in c.items()}
    out = {n: [torch.zeros_like(x[s]), torch.zeros_like(x[s])] for n, s in
           (("out", "q"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    R = len(x["q"])
    out["lse"] = [torch.zeros(H, R, dtype=torch.float64), torch.zeros(H, R, dtype=torch.float64)]
    sc, at = 1 / math.sqrt(hd), 0
    for n in filter(None, lens):
        rs = slice(at, at + n)
        at += n
        past = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(H):
            g = h // (H // G)
            hs, gs = slice(h * hd, (h + 1) * hd), slice(g * hd, (g + 1) * hd)
            q, k, v, do = x["q"][rs, hs], x["k"][rs, gs], x["v"][rs, gs], x["do"][rs, hs]
            s = (q @ k.T) * sc
            e = hd * f * float((q.abs() @ k.abs().T).max()) * sc
            w = 2 * e + (n + 16) * f
            s = s.masked_fill(~past, -math.inf)
            p = torch.softmax(s, 1)
            o = p @ v
            mag = p @ v.abs()
            err_o = (u + w + n * f) * mag
            out["out"][0][rs, hs], out["out"][1][rs, hs] = o, err_o + u * (o.abs() + err_o)
            out["lse"][0][h, rs] = torch.logsumexp(s, 1)
            out["lse"][1][h, rs] = w + 4 * f * out["lse"][0][h, rs].abs() + 4 * f
            D = (o * do).sum(1, keepdim=True)
            err_D = ((err_o + u * (o.abs() + err_o)) * do.abs()).sum(1, keepdim=True) + hd * f * (o * do).abs().sum(1, keepdim=True)
            dp = do @ v.T
            ds = p * (dp - D)
            err_ds = (u + w) * ds.abs() + p * (err_D + hd * f * (do.abs() @ v.abs().T))
            out["dq"][0][rs, hs] = ds @ k * sc
            out["dq"][1][rs, hs] = ((err_ds + n * f * ds.abs()) @ k.abs()) * sc
            out["dk"][0][rs, gs] += ds.T @ q * sc
            out["dk"][1][rs, gs] += ((err_ds + n * f * ds.abs()).T @ q.abs()) * sc
            out["dv"][0][rs, gs] += p.T @ do
            out["dv"][1][rs, gs] += ((u + w + n * f) * p).T @ do.abs()
    for n in ("dq", "dk", "dv"):
        out[n][1] += u * (out[n][0].abs() + out[n][1]) + 1e-30
    return {n: tuple(p) for n, p in out.items()}


class Call:
    """Device buffers of one call: rows of a fused projection unless `ld` gives every tensor a stride of its own."""

    def __init__(self, c, starts, dims, name, offset=0, pad=0, fill=7.0):
        torch = _torch()
        self.dims, self.name = dims, name
        H, G, hd = DIMS[dims]
        R = len(c["q"])
        self.R = R
        t = dtype_of(name)

        def buf(width):
            """[R][width] at `offset` elements past a 16-byte boundary, rows `pad` elements further apart."""
            ld = width + pad
            raw = torch.full((R * ld + 64,), fill, dtype=t, device="cuda")
            return torch.as_strided(raw, (R, width), (ld, 1), offset)
        fused = buf((H + 2 * G) * hd)
        self.q, self.k, self.v = fused[:, :H * hd], fused[:, H * hd:(H + G) * hd], fused[:, (H + G) * hd:]
        for dst, src in ((self.q, "q"), (self.k, "k"), (self.v, "v")):
            dst.copy_(c[src])
        self.do, self.out = buf(H * hd), buf(H * hd)
        self.do.copy_(c["do"])
        self.out.fill_(fill)
        grads = buf((H + 2 * G) * hd)
        grads.fill_(fill)
        self.dq, self.dk, self.dv = grads[:, :H * hd], grads[:, H * hd:(H + G) * hd], grads[:, (H + G) * hd:]
        self.lse = torch.full((H, R), fill, device="cuda")
        self.start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.flags = torch.zeros(1, dtype=torch.int32, device="cuda")
        from paper_2512_14681_amd import jf
        self.ws = torch.full((jf.attention_causal_grad_ws_bytes(len(starts) - 1, R, H, G, hd),), 255, dtype=torch.uint8,
                             device="cuda")

    def forward(self, **kw):
        from paper_2512_14681_amd import jf
        jf.attention_causal(self.start, *DIMS[self.dims], self.q, self.k, self.v, self.out, d_lse=self.lse,
                            d_flags=self.flags, **kw)

    def backward(self, **kw):
        from paper_2512_14681_amd import jf
        jf.attention_causal_grad(self.start, *DIMS[self.dims], self.q, self.k, self.v, self.out, self.lse, self.do, self.dq,
                                 self.dk, self.dv, self.ws, d_flags=self.flags, **kw)

    def results(self):
        _torch().cuda.synchronize()
        return {n: getattr(self, n).double().cpu() for n in ("out", "lse", "dq", "dk", "dv")}


def close(got, want, keep=None):
    for n, (value, bound) in want.items():
        g = got[n]
        err = (g - value).abs()
        worst = float((err / bound.clamp(min=1e-300)).max()) if err.numel() else 0.0
        assert bool((err <= bound).all()), (n, worst, float(err.max()))


LENS = [[1], [2], [31], [32], [33], [63], [64], [65], [127], [128], [129], [200], [500], [1, 1, 1], [5, 0, 130, 64, 1, 0, 77]]


@pytest.mark.parametrize("lens", LENS, ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("dims,name", [("grp3", "bf16"), ("tiny", "f32"), ("wide", "bf16"), ("tiny", "bf16"), ("one", "f32")])
def test_matches_64_bits(lens, dims, name):
    c = case(lens, dims, name)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
    assert int(call.flags) == 0


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_7b_heads(name):
    lens = [150, 260]
    c = case(lens, "7b", name, seed=5)
    call = Call(c, [0, 150, 410], "7b", name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, "7b", name))


@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (0, 8), (8, 4)])
@pytest.mark.parametrize("dims,name", [("grp3", "bf16"), ("wide", "f32"), ("tiny", "f32"), ("tiny", "bf16")])
def test_any_stride_and_alignment(dims, name, offset, pad):
    lens = [70, 135]
    c = case(lens, dims, name, seed=9)
    call = Call(c, [0, 70, 205], dims, name, offset=offset, pad=pad)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
    # what lies between the rows stays
    if pad:
        torch = _torch()
        for t in (call.out, call.dq):
            H, G, hd = DIMS[dims]
            width = H * hd if t is call.out else (H + 2 * G) * hd
            gaps = torch.as_strided(t, (call.R - 1, pad), (width + pad, 1), offset + width)
            assert bool((gaps == 7.0).all())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_rows_outside_the_sequences_stay(name):
    """Padding before the first and behind the last sequence: NaN there is neither read nor written."""
    torch = _torch()
    lens, dims = [40, 90], "grp3"
    c = case([13] + lens + [150], dims, name, seed=3)
    inner = {n: t[13:143] for n, t in c.items()}
    for t in c.values():
        t[:13] = math.nan
        t[143:] = math.nan
    call = Call(c, [13, 53, 143], dims, name)
    call.forward()
    call.backward()
    got = call.results()
    for n in ("out", "dq", "dk", "dv"):
        assert bool((got[n][:13] == 7.0).all()) and bool((got[n][143:] == 7.0).all()), n
        got[n] = got[n][13:143]
    assert bool((got["lse"][:, :13] == 7.0).all()) and bool((got["lse"][:, 143:] == 7.0).all())
    got["lse"] = got["lse"][:, 13:143]
    close(got, reference(inner, lens, dims, name))
    assert int(call.flags) == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_later_rows_do_not_reach_earlier_ones(name, where, bad):
    """An infinity or NaN in a row's key or value leaves the rows before it, and other sequences, as they are."""
    lens, dims, at = [100, 141], "grp3", 170   # row 70 of the second sequence
    c = case(lens, dims, name, seed=4)
    want = reference(c, lens, dims, name)
    c[where][at, 5] = bad
    call = Call(c, [0, 100, 241], dims, name)
    call.forward()
    got = call.results()
    value, bound = want["out"]
    assert bool(((got["out"][:at] - value[:at]).abs() <= bound[:at]).all())
    H, G, hd = DIMS[dims]
    first = got["out"][at:, :3 * hd].reshape(-1, 3, hd)     # the heads that read KV head 0
    if where == "v":     # dim 5 of what sees it is as it is, the rest as before (no weight here is below e^-60)
        assert bool((first[:, :, 5].isnan() if math.isnan(bad) else first[:, :, 5] == bad).all())
        ok = (got["out"] - value).abs() <= bound
        ok[at:, 5:3 * hd:hd] = True
        assert bool(ok.all())
    elif math.isnan(bad):
        assert bool(first.isnan().all())


def test_scores_of_minus_infinity_have_no_weight():
    """A key of -inf leaves a row with other keys a mean of these, and a row that sees only it zeros and -inf."""
    torch = _torch()
    lens, dims, name = [40], "one", "f32"
    c = case(lens, dims, name, seed=8)
    c["q"].abs_()
    c["k"][0] = -math.inf
    call = Call(c, [0, 40], dims, name)
    call.forward()
    got = call.results()
    assert bool((got["out"][0] == 0).all()) and float(got["lse"][0, 0]) == -math.inf
    rest = {n: t[1:] for n, t in c.items()}
    value, bound = reference(rest, [39], dims, name)["out"]
    assert bool(((got["out"][1:] - value).abs() <= bound).all())


def test_large_scores():
    """Scores of thousands: the running maximum keeps the weights in range."""
    lens, dims, name = [300], "grp3", "f32"
    c = case(lens, dims, name, seed=6, std=300.0)
    call = Call(c, [0, 300], dims, name)
    call.forward()
    got = call.results()
    value, bound = reference(c, lens, dims, name)["out"]
    assert bool(((got["out"] - value).abs() <= bound).all())


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_beyond_what_fp32_tells_apart(name, sign):
    """Scores of 2^31 and more (exact in fp32), in even steps of 2^25: the largest one that a row sees has all the weight;
    equal ones share it.  The gradients there have no digits but stay finite."""
    torch = _torch()
    dims, n, hd = "one", 60, 64
    c = case([n], dims, name, seed=31)
    for t in ("q", "k"):
        c[t].zero_()
    c["q"][:, 0] = 2.0 ** 17
    c["k"][:, 0] = sign * 2.0 ** 17 * (1 + torch.arange(n) / 64)
    call = Call(c, [0, n], dims, name)
    call.forward()
    call.backward()
    got = call.results()
    v = c["v"].double()
    assert bool((got["out"] == (v if sign > 0 else v[:1].expand(n, -1))).all())
    assert all(bool(got[t].isfinite().all()) for t in got)
    c["k"][:, 0] = sign * 2.0 ** 17
    call = Call(c, [0, n], dims, name)
    call.forward()
    u = 2.0 ** -8 if name == "bf16" else 2.0 ** -24
    mean = v.cumsum(0) / torch.arange(1, n + 1)[:, None]
    mag = v.abs().cumsum(0) / torch.arange(1, n + 1)[:, None]
    assert bool(((call.results()["out"] - mean).abs() <= (2 * u + 100 * 2.0 ** -24) * (mag + mean.abs())).all())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_log_sums_of_equal_scores_have_their_digits(name):
    """Scores of zero: row i's lse is ln(i + 1).  Its sum is exact; the logarithm to base 2 is off by 2 steps of 2^-24 at
    most, ln 2 and the product by one each, all relative to the result; 6 cover terms of second order."""
    torch = _torch()
    dims, n = "grp3", 700
    c = case([n], dims, name, seed=36)
    c["q"].zero_()
    call = Call(c, [0, n], dims, name)
    call.forward()
    want = torch.log(torch.arange(1, n + 1, dtype=torch.float64))
    assert bool(((call.results()["lse"] - want).abs() <= 6 * 2.0 ** -24 * want).all())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_values_next_to_the_largest(name):
    """Sums of many values of 2^127 have a mean that fits, whatever the order of the maxima."""
    torch = _torch()
    dims, n = "grp3", 500
    c = case([n], dims, name, seed=32)
    c["v"] = (2.0 ** 127 * torch.sign(c["v"].double() + 2.5)).to(c["v"].dtype)
    want = reference(dict(c, do=c["do"] * 0), [n], dims, name)["out"]
    call = Call(c, [0, n], dims, name)
    call.forward()
    got = call.results()["out"]
    assert bool(((got - want[0]).abs() <= want[1]).all())


def test_thousands_of_short_sequences():
    torch = _torch()
    g = torch.Generator().manual_seed(33)
    lens = torch.randint(0, 4, (5000,), generator=g).tolist()
    lens[4000] = 300
    dims, name = "one", "bf16"
    c = case(lens, dims, name, seed=34)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
    assert int(call.flags) == 0


@pytest.mark.parametrize("lens", [[0] * 90 + [1, 5], [1] * 60 + [0] * 60 + [70], [0, 3] * 50 + [0] * 100 + [2] * 3],
                         ids=["front", "middle", "mixed"])
def test_more_sequences_than_rows(lens):
    """Empty sequences among more than 64: the last ones' blocks have numbers beyond the rows'."""
    dims, name = "grp3", "bf16"
    c = case(lens, dims, name, seed=36)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
    assert int(call.flags) == 0


def test_bad_starts_among_many_sequences():
    """More than 64 sequences: flagged, and nothing outside the good ones is written."""
    from paper_2512_14681_amd import jf
    R, dims, name = 300, "grp3", "bf16"
    c = case([R], dims, name, seed=35)
    starts = list(range(0, 3 * 80, 3)) + [500, 250, 260]
    call = Call(c, starts, dims, name)
    call.forward()
    call.backward()
    got = call.results()
    assert int(call.flags) == jf.JF_FLAG_CAPACITY
    assert bool((got["out"][260:] == 7.0).all()) and bool((got["dk"][260:] == 7.0).all())


@pytest.mark.parametrize("starts", [[0, 300, 410], [0, -5, 410], [-1, 200, 410], [0, 200, 411], [0, 250, 200], [50, 411, 60, 90]])
def test_bad_starts_are_flagged_and_left_alone(starts):
    """Sequences inside the rows are computed; what does not fit raises JF_FLAG_CAPACITY, nothing outside is written."""
    from paper_2512_14681_amd import jf
    dims, name, R = "grp3", "bf16", 410
    c = case([R], dims, name, seed=2)
    call = Call(c, starts, dims, name)
    call.forward()
    call.backward()
    got = call.results()
    ok = [0 <= a <= b <= R for a, b in zip(starts, starts[1:])]
    assert int(call.flags) == (0 if all(ok) else jf.JF_FLAG_CAPACITY)
    covered = np.zeros(R, bool)
    for good, a, b in zip(ok, starts, starts[1:]):
        if good:
            covered[a:b] = True
            part = {n: t[a:b] for n, t in c.items()}
            want = reference(part, [b - a], dims, name)["out"]
            assert bool(((got["out"][a:b] - want[0]).abs() <= want[1]).all())
    for n in ("out", "dq", "dk", "dv"):
        assert bool((got[n][~covered] == 7.0).all()), n


def test_the_gradient_is_that_of_differences():
    """Central differences of sum(g out) in 64 bits, of the reference itself, against the kernels' gradient along random
    directions: off by the bounds of test_matches_64_bits and by what the difference quotient leaves (step^2)."""
    torch = _torch()
    lens, dims, name = [37, 70], "grp3", "f32"
    c = case(lens, dims, name, seed=12)
    call = Call(c, [0, 37, 107], dims, name)
    call.forward()
    call.backward()
    got = call.results()
    want = reference(c, lens, dims, name)
    for which in ("q", "k", "v"):
        g = torch.Generator().manual_seed(7)
        direction = torch.randn(c[which].shape, generator=g, dtype=torch.float64)
        step, total = 1e-4, []
        for sign in (1, -1):
            moved = {n: t.double() for n, t in c.items()}
            moved[which] = moved[which] + sign * step * direction
            total.append(float((reference(moved, lens, dims, name)["out"][0] * moved["do"]).sum()))
        quotient = (total[0] - total[1]) / (2 * step)
        along = float((got["d" + which] * direction).sum())
        bound = float((want["d" + which][1] * direction.abs()).sum()) + 1e-4 * abs(quotient) + 1e-4
        assert abs(along - quotient) <= bound, (which, along, quotient, bound)


def test_same_bits_every_time():
    lens, dims, name = [300, 211], "7b", "bf16"
    c = case(lens, dims, name, seed=1)
    first = None
    for _ in range(3):
        call = Call(c, [0, 300, 511], dims, name)
        call.forward()
        call.backward()
        got = call.results()
        first = first or got
        for n in got:
            assert bool((got[n] == first[n]).all()), n


def test_captured_with_new_lengths():
    """A captured forward and backward pass takes the lengths that the device holds at every replay, between the
    program's own work."""
    torch = _torch()
    dims, name, R = "grp3", "bf16", 260
    c = case([R], dims, name, seed=13)
    call = Call(c, [0, 100, 260], dims, name)
    call.forward()
    call.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.forward()
        call.backward()
    for starts in ([0, 100, 260], [0, 37, 200], [5, 5, 70], [0, 100, 260]):
        call.start.copy_(torch.tensor(starts, dtype=torch.int32))
        for t in (call.out, call.dq, call.dk, call.dv):
            t.fill_(7.0)
        graph.replay()
        got = call.results()
        eager = Call(c, starts, dims, name)
        eager.forward()
        eager.backward()
        want = eager.results()
        for n in ("out", "dq", "dk", "dv"):
            assert bool((got[n] == want[n]).all()), (starts, n)


def test_on_a_stream_of_its_own():
    torch = _torch()
    lens, dims, name = [90, 61], "grp3", "bf16"
    c = case(lens, dims, name, seed=15)
    call = Call(c, [0, 90, 151], dims, name)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call.forward(stream=s)
    call.backward(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    close(call.results(), reference(c, lens, dims, name))


def test_many_short_sequences():
    """More sequences than lanes, empty ones among them, across the boundaries of 64 of them."""
    torch = _torch()
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 9, (200,), generator=g).tolist()
    dims, name = "tiny", "bf16"
    c = case(lens, dims, name, seed=21)
    call = Call(c, np.cumsum([0] + lens).tolist(), dims, name)
    call.forward()
    call.backward()
    close(call.results(), reference(c, lens, dims, name))
    assert int(call.flags) == 0


def test_nothing_to_do():
    torch = _torch()
    from paper_2512_14681_amd import jf
    x = torch.zeros(0, 64, device="cuda")
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    jf.attention_causal(start, 1, 1, 64, x, x, x, x.clone())
    c = case([5], "one", "f32")
    call = Call(c, [0], "one", "f32")
    call.forward()
    call.backward()
    assert bool((call.results()["out"] == 7.0).all())
