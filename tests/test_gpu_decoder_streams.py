"""decode.Decoder with a model on a stream of its own that is not the current one, and busy: what it gives without."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tiny():
    import torch
    import jf_inputs
    from paper_2512_14681_amd import jf
    shape = jf_inputs.MODEL_SHAPES["tiny"]
    return torch, jf, jf_inputs, shape, jf_inputs.model_weights(shape, seed=0)


def test_a_model_on_its_own_stream(tiny):
    torch, jf, jf_inputs, shape, w = tiny
    from paper_2512_14681_amd import decode
    prompt = jf_inputs.prompt(1, 20, shape["vocab"])
    toks = jf_inputs.token_ids(9, 1, 21, shape["vocab"])
    own = torch.cuda.Stream()
    work = torch.randn(4096, 4096, device="cuda")
    plain = decode.Decoder(jf.Model(shape, w, max_rows=8, max_ctx=128))
    named = decode.Decoder(jf.Model(shape, w, max_rows=8, max_ctx=128, stream=own))
    loops = {"score": lambda d: d.score(prompt, toks, k=3), "ar": lambda d: d.generate_ar(prompt, 12),
             "jacobi": lambda d: d.generate_jacobi(prompt, 4, 12),
             "multiblock": lambda d: d.generate_multiblock(prompt, 4, 2, 0.85, 12, n_cand=0)[0],
             "trajectories": lambda d: d.collect_trajectories(prompt, 4, 3)}
    for name, loop in loops.items():
        plain.reset()
        want = loop(plain)
        named.reset()
        torch.cuda.synchronize()
        with torch.cuda.stream(own):            # some milliseconds that the loop's first calls stand behind
            for _ in range(8):
                y = work @ work
        got = loop(named)
        assert float(y[0, 0]) == float(y[0, 0])
        for a, b in zip(want if isinstance(want, tuple) else (want,), got if isinstance(got, tuple) else (got,)):
            a, b = (x.cpu().numpy() if torch.is_tensor(x) else np.asarray(x) for x in (a, b))
            assert np.array_equal(a, b), name
        assert named.length() == plain.length(), name


def test_score_with_alternatives_of_a_named_stream(tiny):
    """The alternatives' ids and the refusals, next to the log probabilities that the oracle's decoder gives."""
    torch, jf, jf_inputs, shape, w = tiny
    from oracle import batch as ob, jacobi as ojac
    from oracle.model import DecoderOracle
    from paper_2512_14681_amd import decode
    prompt = jf_inputs.prompt(1, 20, shape["vocab"])
    toks = jf_inputs.token_ids(9, 1, 21, shape["vocab"])
    dec = decode.Decoder(jf.Model(shape, w, max_rows=8, max_ctx=128, stream=torch.cuda.Stream()))
    for bad in ([shape["vocab"]], [-1]):
        with pytest.raises(ValueError):
            dec.score(prompt, bad)
    lp, _, ids, top = dec.score(prompt, toks, k=3)
    back = ojac.TransformerBackend(DecoderOracle(shape, w))
    back.prefill(list(prompt[:-1]))
    feed = [int(prompt[-1])] + [int(t) for t in toks[:-1]]
    back.step(feed, ojac.linear_segments(len(feed)))
    wlp, _, _, wids, wtop = ob.token_logprobs(np.asarray(back.last[1], np.float64), toks, 4)
    # fp32 logits of the tiny decoder are within 2^-12 of the oracle's: alternatives closer than twice that may swap
    assert np.abs(lp - wlp).max() <= 2.0 ** -11 and np.abs(top - wtop[:, :3]).max() <= 2.0 ** -11
    apart = -np.diff(wtop, axis=1) > 2.0 ** -10
    clear = apart & np.concatenate([np.ones((len(toks), 1), bool), apart[:, :2]], 1)
    assert clear.mean() > 0.9 and np.array_equal(ids[clear], wids[:, :3][clear])
