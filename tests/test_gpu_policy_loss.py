"""jf_policy_loss against the formulas in 64 bits (numpy, row by row).

Tolerances: everything is computed in 64 bits and rounded once to fp32, so results are off by 2^-24 relative and what 64
bits lose: 2^-48 of the sums' terms."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def expected(c):
    """{name: array} by the formulas of jf.h."""
    starts, tok = c["starts"], c["tokens"]
    R, S = len(c["lp"]), len(starts) - 1
    seq = np.full(R, -1)
    for s in range(S):
        seq[starts[s]:starts[s + 1]] = s
    valid = (seq >= 0) & (tok != -1)
    lp, old, ref, ent = (np.asarray(c[n], np.float64) for n in ("lp", "old", "ref", "entropy"))
    adv = np.asarray(c["adv"], np.float64)
    adv = adv if c["adv_rows"] else adv[np.maximum(seq, 0)]
    n_s = np.bincount(seq[valid], minlength=S) if S else np.zeros(0)
    w = np.zeros(R)
    if valid.any():
        w[valid] = {"tokens": 1 / valid.sum(), "seqs": 1 / (n_s[seq[valid]] * (n_s > 0).sum()), "sum": 1.0}[c["mean"]]
    with np.errstate(all="ignore"):
        r = np.exp(lp - old)
        cut = ((adv > 0) & (r > 1 + c["high"])) | ((adv < 0) & (r < 1 - c["low"]))
        used = np.where(cut, np.where(adv > 0, 1 + c["high"], 1 - c["low"]), r)
        policy = np.where(adv == 0, 0.0, -used * adv)
        k = (ref - lp) if c["use_ref"] else np.zeros(R)
        series = k * k * (0.5 + k * (1 / 6 + k * (1 / 24 + k * (1 / 120 + k / 720))))
        kl = np.where(np.abs(k) < 0.02, series, np.expm1(k) - k)
        g = np.where(cut | (adv == 0), 0.0, -adv * r) - c["beta"] * np.expm1(k)
    terms = [np.where(valid, w * t, 0.0) for t in (policy, kl, ent if c["use_entropy"] else np.zeros(R), cut * 1.0)]
    p, kk, h, cl = (t.sum() for t in terms)
    loss = c["scale"] * (p + c["beta"] * kk - (c["ent_w"] * h if c["use_entropy"] else 0.0))
    mags = [np.abs(t).sum() for t in terms]
    mags = [abs(c["scale"]) * (mags[0] + abs(c["beta"]) * mags[1] + abs(c["ent_w"]) * mags[2])] + mags + [R]
    return dict(stats=np.array([loss, p, kk, h, cl, valid.sum()]), mags=np.array(mags),
                g_lp=np.where(valid, c["scale"] * w * np.where(valid, g, 0), 0.0),
                g_entropy=np.where(valid, -c["scale"] * c["ent_w"] * w, 0.0), inside=seq >= 0)


def case(lens, seed=0, mean="tokens", adv_rows=False, before=0, after=0, spread=0.2, none=0.3, **kw):
    rng = np.random.default_rng(seed)
    starts = before + np.cumsum([0] + list(lens))
    R = int(starts[-1]) + after
    lp = -rng.exponential(1.0, R)
    c = dict(starts=starts, lp=lp, old=lp + rng.normal(0, spread, R), ref=lp + rng.normal(0, 0.4, R),
             entropy=rng.exponential(1.0, R), tokens=np.where(rng.random(R) < none, -1, rng.integers(0, 99, R)),
             adv=rng.normal(0, 1, R if adv_rows else len(lens)), mean=mean, adv_rows=adv_rows, low=0.2, high=0.3, beta=0.05,
             ent_w=0.01, scale=2.0, use_ref=True, use_entropy=True)
    for n in ("lp", "old", "ref", "entropy", "adv"):
        c[n] = c[n].astype(np.float32)
    c.update(kw)
    return c


class Call:
    def __init__(self, c):
        torch = _torch()
        from paper_2512_14681_amd import jf
        self.c = c
        f = lambda n: torch.from_numpy(np.ascontiguousarray(c[n], np.float32)).cuda()
        i = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()
        self.lp, self.old, self.ref, self.entropy, self.adv = (f(n) for n in ("lp", "old", "ref", "entropy", "adv"))
        self.start, self.tokens, self.flags = i(c["starts"]), i(c["tokens"]), i([0])
        self.stats = torch.full((6,), 7.0, device="cuda")
        self.g_lp, self.g_entropy = (torch.full_like(self.lp, 7.0) for _ in range(2))
        self.ws = torch.full((jf.policy_loss_ws_bytes(len(c["starts"]) - 1, len(c["lp"])),), 255, dtype=torch.uint8,
                             device="cuda")

    def run(self, **kw):
        from paper_2512_14681_amd import jf
        c = self.c
        jf.policy_loss(self.start, self.tokens, self.lp, self.old, self.adv, self.stats, self.ws,
                       d_ref_logprob=self.ref if c["use_ref"] else None,
                       d_entropy=self.entropy if c["use_entropy"] else None, d_g_logprob=self.g_lp,
                       d_g_entropy=self.g_entropy if c["use_entropy"] else None, clip_low=c["low"], clip_high=c["high"],
                       kl_weight=c["beta"], entropy_weight=c["ent_w"], scale=c["scale"],
                       mean={"tokens": jf.JF_MEAN_TOKENS, "seqs": jf.JF_MEAN_SEQS, "sum": jf.JF_SUM}[c["mean"]],
                       adv_rows=c["adv_rows"], d_flags=self.flags, **kw)
        return self

    def check(self):
        _torch().cuda.synchronize()
        want = expected(self.c)
        f = 2.0 ** -24
        got = self.stats.double().cpu().numpy()
        assert (np.abs(got - want["stats"]) <= f * np.abs(want["stats"]) + 2.0 ** -48 * want["mags"]).all(), (got, want["stats"])
        inside = want["inside"]
        names = ("g_lp", "g_entropy") if self.c["use_entropy"] else ("g_lp",)
        for n in names:
            g = getattr(self, n).double().cpu().numpy()
            assert (g[~inside] == 7.0).all(), n
            w = want[n][inside]
            assert (np.abs(g[inside] - w) <= f * np.abs(w) * (1 + 1e-6) + 1e-44).all(), n
        assert int(self.flags) == 0
        return got


LENS = [[1], [3, 0, 5], [64] * 8, [0, 0, 1, 0], [700, 1, 2000, 64], [5000], [1, 4100, 0, 3, 900], [2] * 3000, [37] * 5000]


@pytest.mark.parametrize("lens", LENS, ids=range(len(LENS)))
@pytest.mark.parametrize("mean", ["tokens", "seqs", "sum"])
@pytest.mark.parametrize("adv_rows", [False, True])
def test_matches_64_bits(lens, mean, adv_rows):
    Call(case(lens, seed=len(lens), mean=mean, adv_rows=adv_rows)).run().check()


@pytest.mark.parametrize("size", [1, 3000])
@pytest.mark.parametrize("mean", ["tokens", "seqs"])
def test_padding_rows_stay(size, mean):
    c = case([size, 40, size], seed=3, mean=mean, before=11, after=17)
    for n in ("lp", "old", "ref", "entropy"):
        c[n][:11] = np.nan
        c[n][-17:] = np.nan
    Call(c).run().check()


@pytest.mark.parametrize("size", [20, 6000])
@pytest.mark.parametrize("mean", ["tokens", "seqs", "sum"])
def test_no_tokens_at_all(size, mean):
    got = Call(case([size, size], seed=4, mean=mean, none=1.1)).run().check()
    assert (got == 0).all()


@pytest.mark.parametrize("size", [20, 6000])
def test_rows_without_a_token_count_nowhere(size):
    """What they hold is not looked at: NaN among them reaches nothing."""
    c = case([size, size], seed=5, mean="seqs")
    hole = c["tokens"] == -1
    for n in ("lp", "old", "ref", "entropy"):
        c[n][hole] = np.nan
    Call(c).run()
    call = Call(c).run()
    clean = dict(c, **{n: np.where(hole, np.float32(0), c[n]) for n in ("lp", "old", "ref", "entropy")})
    call.c = clean
    call.check()


def test_without_reference_and_entropy():
    for size in (100, 5000):
        Call(case([size, 9], seed=6, use_ref=False)).run().check()
        Call(case([size, 9], seed=6, use_entropy=False)).run().check()


def test_borders_are_those_of_64_bits():
    """Ratios a step of fp32 around the borders, where a rounded ratio would lie on the wrong side."""
    n = 4000
    old = np.full(n, -1.5, np.float32)
    up, down = -1.5 + math.log(1.3), -1.5 + math.log(0.8)
    lp = np.concatenate([np.float32(up) + (np.arange(n // 2) - n // 4) * np.spacing(np.float32(1.3)) * 0.25,
                         np.float32(down) + (np.arange(n // 2) - n // 4) * np.spacing(np.float32(1.7))]).astype(np.float32)
    c = case([n // 2, n // 2], seed=7, none=-1.0, lp=lp, old=old, adv=np.array([1.5, -0.5], np.float32))
    got = Call(c).run().check()
    assert 0.2 < got[4] < 0.8


def test_extreme_values():
    """Probabilities of 0 now or before, an advantage of 0 beside an infinite ratio, no upper border."""
    lp = np.array([-math.inf, -0.5, -0.5, -200.0, -0.0, -1e-30], np.float32)
    old = np.array([-0.5, -math.inf, -math.inf, -1.0, -1000.0, -0.0], np.float32)
    adv = np.array([1.0, 0.0, -1.0, -1.0, 0.0, 1.0], np.float32)
    c = case([6], seed=8, adv_rows=True, lp=lp, old=old, adv=adv, none=-1.0, use_ref=False)
    torch = _torch()
    call = Call(c).run()
    torch.cuda.synchronize()
    g = call.g_lp.cpu().numpy()
    w = 2.0 / 6
    assert g[0] == 0.0                                    # ratio 0
    assert g[1] == 0.0 and g[4] == 0.0                    # no advantage
    assert g[2] == math.inf and call.stats[0].item() == math.inf
    assert g[3] == 0.0                                    # clipped from below
    assert abs(g[5] + w) < 1e-6
    c = case([50, 6000], seed=9, high=math.inf, low=1.0, spread=1.0)
    Call(c).run().check()
    assert Call(c).run().check()[4] == 0                  # nothing is clipped


def test_the_gradient_is_that_of_differences():
    """Central differences of the loss in 64 bits, away from the borders."""
    c = case([40, 25], seed=10, mean="seqs")
    call = Call(c).run()
    call.check()
    g, gh = call.g_lp.double().cpu().numpy(), call.g_entropy.double().cpu().numpy()
    r = np.exp(c["lp"].astype(np.float64) - c["old"])
    for i in range(65):
        if min(abs(r[i] - 1.3), abs(r[i] - 0.8)) < 1e-3:
            continue
        for name, got in (("lp", g), ("entropy", gh)):
            side = []
            for step in (1e-5, -1e-5):
                moved = dict(c, **{name: c[name].astype(np.float64)})
                moved[name][i] += step
                side.append(expected(moved)["stats"][0])
            quotient = (side[0] - side[1]) / 2e-5
            assert abs(got[i] - quotient) <= 1e-6 * (abs(quotient) + 0.1), (name, i)


@pytest.mark.parametrize("starts", [[0, 30, 20, 60], [-1, 20, 60], [0, 20, 61], [0, 5000, 4999, 6000], [0, 100, 6001]])
def test_bad_starts(starts):
    from paper_2512_14681_amd import jf
    R = 60 if starts[-1] < 100 else 6000
    c = case([R], seed=11, mean="seqs")
    c["starts"], c["adv"] = np.array(starts), np.ones(len(starts) - 1, np.float32)
    call = Call(c).run()
    _torch().cuda.synchronize()
    assert bool(call.stats.isnan().all()) and int(call.flags) == jf.JF_FLAG_CAPACITY
    assert bool((call.g_lp == 7.0).all()) and bool((call.g_entropy == 7.0).all())


def test_nothing_to_do():
    torch = _torch()
    c = case([5], seed=12)
    call = Call(c)
    call.start = call.start[:1].contiguous()
    call.adv = call.adv[:0].contiguous()
    call.run()
    torch.cuda.synchronize()
    assert bool((call.stats == 0).all()) and bool((call.g_lp == 7.0).all())


@pytest.mark.parametrize("mean", ["tokens", "seqs"])
def test_captured_and_replayed(mean):
    """Every replay, with new data and lengths between them, equals the eager call; the workspace is not cleared."""
    torch = _torch()
    for lens in ([30, 50], [5000, 900, 1]):
        call = Call(case(lens, seed=13, mean=mean))
        call.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call.run()
        for seed in range(3):
            c = case(lens, seed=20 + seed, mean=mean)
            c["starts"] = c["starts"].copy()
            c["starts"][1] -= seed
            for t, n in ((call.lp, "lp"), (call.old, "old"), (call.ref, "ref"), (call.entropy, "entropy"), (call.adv, "adv")):
                t.copy_(torch.from_numpy(c[n]))
            call.tokens.copy_(torch.from_numpy(c["tokens"].astype(np.int32)))
            call.start.copy_(torch.from_numpy(c["starts"].astype(np.int32)))
            call.c = c
            call.ws.fill_(255)
            graph.replay()
            call.check()
            graph.replay()
            call.check()


def test_from_logits_to_their_gradient():
    """jf_token_logprobs -> jf_policy_loss -> jf_token_logprobs_grad: the gradient of the whole, against 64-bit autograd.
    The log probabilities that the loss takes are fp32 (off by 2^-23 |x| and a few steps), so the chain is off by e = 1e-5
    of each row's gradient where no ratio lies that close to a border."""
    torch = _torch()
    from paper_2512_14681_amd import jf
    R, V, lens = 48, 1000, [20, 28]
    g = torch.Generator().manual_seed(2)
    x = torch.randn(R, V, generator=g) * 2
    tokens = torch.randint(0, V, (R,), generator=g, dtype=torch.int32)
    tokens[::7] = -1
    lp64 = torch.log_softmax(x.double(), 1)
    picked = lp64[torch.arange(R), tokens.clamp(min=0).long()]
    old = (picked + torch.randn(R, generator=g, dtype=torch.float64) * 0.2).float()
    ref = (picked + torch.randn(R, generator=g, dtype=torch.float64) * 0.2).float()
    adv = torch.tensor([1.0, -0.7])
    d = {n: t.cuda() for n, t in dict(x=x, tokens=tokens, old=old, ref=ref, adv=adv).items()}
    start = torch.tensor([0, 20, 48], dtype=torch.int32, device="cuda")
    lp, ent, norm, stats = (torch.zeros(n, device="cuda") for n in (R, R, 2 * R, 6))
    g_lp, g_ent, grad = torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda"), torch.zeros(R, V, device="cuda")
    ws = torch.empty(jf.token_logprobs_ws_bytes(R, V), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(jf.policy_loss_ws_bytes(2, R), dtype=torch.uint8, device="cuda")
    jf.token_logprobs(d["x"], ws, d_tokens=d["tokens"], d_logprob=lp, d_entropy=ent, d_norm=norm)
    jf.policy_loss(start, d["tokens"], lp, d["old"], d["adv"], stats, ws2, d_ref_logprob=d["ref"], d_entropy=ent,
                   d_g_logprob=g_lp, d_g_entropy=g_ent, kl_weight=0.1, entropy_weight=0.02)
    jf.token_logprobs_grad(d["x"], norm, grad, d_tokens=d["tokens"], d_entropy=ent, d_g_logprob=g_lp, d_g_entropy=g_ent)
    torch.cuda.synchronize()
    y = x.double().requires_grad_()
    lp64 = torch.log_softmax(y, 1)
    has = (tokens != -1).double()
    picked = lp64[torch.arange(R), tokens.clamp(min=0).long()]
    H = -(lp64.exp() * lp64).sum(1)
    a = adv.double()[torch.tensor([0] * 20 + [1] * 28)]
    r = torch.exp(picked - old.double())
    assert float(torch.minimum((r - 1.2).abs(), (r - 0.8).abs()).detach().min()) > 1e-5
    k = ref.double() - picked
    loss = (has * (-torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.1 * (k.exp() - k - 1) - 0.02 * H)).sum() / has.sum()
    loss.backward()
    assert abs(float(stats[0]) - loss.item()) < 1e-5 * (1 + abs(loss.item()))
    err = (grad.double().cpu() - y.grad).norm(dim=1)
    assert bool((err <= 1e-5 * y.grad.norm(dim=1) + 1e-9).all()), float(err.max())


@pytest.mark.parametrize("size", [20, 6000])
def test_weights_of_zero_leave_their_terms_out(size):
    """The KL term and the entropy, infinite in places, are only reported."""
    c = case([size], seed=9, beta=0.0, ent_w=0.0, none=0.0)
    c["ref"][::3] = -np.inf
    c["ref"][1] = 500.0  # e^k beyond fp32's largest
    c["entropy"][2] = np.inf
    call = Call(c).run()
    got, g = call.stats.cpu().numpy(), call.g_lp.cpu().numpy()
    assert np.isinf(got[2]) and np.isinf(got[3])
    c["use_ref"] = c["use_entropy"] = False
    alone = Call(c).run()
    assert (g == alone.g_lp.cpu().numpy()).all()
    assert got[0] == alone.stats.cpu().numpy()[0] and np.isfinite(got[0])
