"""What the binding remembers between calls, without a GPU: sizes and parameters by their values, never by the object that
holds them (a tensor that changes in place is the same object)."""
import os
import types

import pytest

from paper_2512_14681_amd import jf

STREAM = types.SimpleNamespace(cuda_stream=0)


@pytest.fixture
def policies(monkeypatch):
    """The parameters that jf_policy_loss was called with; host tensors pass for the GPU's."""
    if not os.path.exists(jf.LIB_PATH):
        pytest.skip("libjf.so not built (python -m paper_2512_14681_amd.build)")
    jf._types()
    seen = []
    real = jf.lib()

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)

            def call(*args):
                p = args[0]._obj
                seen.append({n: getattr(p, n) for n, _ in jf.JfPolicy._fields_})
                return jf.JF_OK
            return call
    monkeypatch.setattr(jf, "lib", lambda: Lib())
    monkeypatch.setattr(jf, "_current_device", lambda: -1)   # what host tensors answer
    return seen


def policy(**kw):
    import torch
    z = lambda k=10: torch.zeros(k)
    jf.policy_loss(torch.tensor([0, 4, 10], dtype=torch.int32), None, z(), z(), z(2), z(6),
                   torch.zeros(jf.policy_loss_ws_bytes(2, 10), dtype=torch.uint8), d_entropy=z(), stream=STREAM, **kw)


@pytest.mark.parametrize("name", ["clip_low", "clip_high", "kl_weight", "entropy_weight", "scale"])
def test_a_weight_in_a_tensor_is_read_at_every_call(policies, name):
    """A weight that a program anneals in place counts as what it is at the call."""
    import numpy as np
    import torch
    for held in (torch.tensor(0.25), torch.tensor(0.25, dtype=torch.float64), np.array(0.25)):
        del policies[:]
        for value in (0.25, 0.5, 0.125):
            held[...] = value
            policy(**{name: held})
        policy(**{name: 0.75})
        assert [p[name] for p in policies] == [0.25, 0.5, 0.125, 0.75]


def test_the_mean_in_a_tensor_is_read_at_every_call(policies):
    import torch
    held = torch.tensor(jf.JF_MEAN_TOKENS)
    for value in (jf.JF_MEAN_TOKENS, jf.JF_SUM, jf.JF_MEAN_SEQS):
        held.fill_(value)
        policy(mean=held)
    assert [p["mean"] for p in policies] == [jf.JF_MEAN_TOKENS, jf.JF_SUM, jf.JF_MEAN_SEQS]
    with pytest.raises(TypeError):
        policy(mean=0.5)


def test_sizes_are_those_of_the_counts_at_the_call():
    """A count in a tensor that grew asks for the workspace of the larger count."""
    import torch
    if not os.path.exists(jf.LIB_PATH):
        pytest.skip("libjf.so not built (python -m paper_2512_14681_amd.build)")
    i32 = dict(dtype=torch.int32)
    batch = jf.Batch(torch.tensor([0, 2], **i32), torch.zeros(1, **i32), torch.zeros(1, 1000, **i32), 2, 2, 64000, 3)
    for size, counts in ((lambda n: jf.attention_causal_grad_ws_bytes(1, n, 4, 2, 64), (100, 9000)),
                         (lambda n: jf.attention_causal_grad_ws_bytes(1, 100, n, 2, 64), (4, 64)),
                         (lambda n: jf.policy_loss_ws_bytes(n, 100), (1, 90000)),
                         (lambda n: jf.token_logprobs_ws_bytes(1000, 152064, n), (0, 20)),
                         (lambda n: jf.attention_shared_ws_bytes(batch, None, n, 2, 64), (4, 64)),
                         (lambda n: jf.attention_kv8_ws_bytes(batch, n, 2, 64), (4, 64))):
        want = [size(n) for n in counts]
        assert want[0] < want[1]
        held = torch.tensor(counts[0])
        got = [size(held)]
        held.fill_(counts[1])
        assert got + [size(held)] == want
