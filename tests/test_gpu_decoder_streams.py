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
