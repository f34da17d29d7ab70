"""decode.Decoder's host side without a GPU: a model that writes down its calls, host tensors, and streams that only
remember who waited for whom."""
import contextlib
import types

import pytest

from paper_2512_14681_amd import decode, jf

V, ROWS = 50, 4


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append(("wait", self.name, other.name))


class Cuda:
    def __init__(self, log):
        self.log, self.at = log, Stream("callers", log)

    def current_stream(self):
        return self.at

    @contextlib.contextmanager
    def stream(self, s):
        was, self.at = self.at, s
        try:
            yield
        finally:
            self.at = was


class Torch:
    """torch with its GPU tensors on the host; every tensor made is noted with the stream it is made on."""

    def __init__(self, log):
        self.log, self.cuda = log, Cuda(log)

    def __getattr__(self, name):
        import torch
        real = getattr(torch, name)
        if name not in ("as_tensor", "empty", "zeros", "full"):
            return real

        def make(*a, **k):
            k.pop("device", None)
            self.log.append((name, self.cuda.at.name))
            return real(*a, **k)
        return make


class Model:
    """Accepts one row of every step; `flags` of the steps in turn."""

    def __init__(self, t, stream, flags=()):
        self.t, self.stream, self.flags = t, stream, list(flags)
        self.cfg, self.V = types.SimpleNamespace(max_rows=ROWS), V
        self.committed = []

    def note(self, name):
        self.t.log.append((name, (self.stream or self.t.cuda.at).name))

    def jf_prefill(self, d_tokens, d_pending):
        self.note("prefill")
        d_pending.fill_(7)

    def jf_jacobi_step(self, d_draft, n, mode, seed, d_argmax, d_result, d_next, d_logits=None):
        self.note("step")
        d_result[0], d_result[2] = 1, 7
        d_result[3] = self.flags.pop(0) if self.flags else 0
        d_argmax[:n] = 7

    def jf_commit_kv(self, d_path, d_result, max_commit=0):
        self.note("commit")
        self.committed.append(int(d_result[0]))


def decoder(monkeypatch, own=True, flags=()):
    import torch
    log = []
    t = Torch(log)
    d = decode.Decoder.__new__(decode.Decoder)
    d.t, d.m, d.V = t, Model(t, Stream("models", log) if own else None, flags), V
    d.d_io = torch.zeros(4 + 2 * ROWS, dtype=torch.int32)
    d.d_result, d.d_argmax, d.d_pending = d.d_io[:4], d.d_io[4:4 + ROWS], torch.zeros(1, dtype=torch.int32)
    d.d_tokens, d.d_next, d.h_stage = (torch.zeros(ROWS, dtype=torch.int32) for _ in range(3))
    d.trace = []
    monkeypatch.setattr(jf, "token_logprobs", lambda *a, **k: log.append(("logprobs", k["stream"].name if k["stream"]
                                                                           else t.cuda.at.name)))
    monkeypatch.setattr(jf, "trajectory_record", lambda *a, stream=None: log.append(("record", "models")))
    return d, log


LOOPS = {"prefill": lambda d: d.prefill([1, 2, 3]), "ar": lambda d: d.generate_ar([1, 2, 3], 3),
         "jacobi": lambda d: d.generate_jacobi([1, 2, 3], 2, 3), "score": lambda d: d.score([1, 2, 3], [4, 5, 6, 7, 8], k=2)}


@pytest.mark.parametrize("loop", LOOPS)
def test_loops_run_on_the_models_stream(monkeypatch, loop):
    """A model with a stream of its own: everything a loop makes and calls is on it, between two waits."""
    d, log = decoder(monkeypatch)
    LOOPS[loop](d)
    assert log[0] == ("wait", "models", "callers") and log[-1] == ("wait", "callers", "models")
    assert {e[1] for e in log if e[0] != "wait"} == {"models"} and d.t.cuda.at.name == "callers"


def test_loops_leave_the_current_stream_alone(monkeypatch):
    """A model without a stream works on the current one: nobody waits."""
    d, log = decoder(monkeypatch, own=False)
    LOOPS["score"](d)
    assert {e[1] for e in log} == {"callers"} and not [e for e in log if e[0] == "wait"]
    assert d.m.committed == [4, 1]


def test_callers_wait_for_a_loop_that_fails(monkeypatch):
    d, log = decoder(monkeypatch)
    with pytest.raises(ValueError):
        d.score([1], [2])
    assert log[-1] == ("wait", "callers", "models") and d.t.cuda.at.name == "callers"


@pytest.mark.parametrize("flags", [[0, jf.JF_FLAG_CAPACITY], [jf.JF_FLAG_SYNC, 0], [jf.JF_FLAG_BAD_TOKEN]])
def test_score_raises_what_any_step_flagged(monkeypatch, flags):
    """Every step writes its own flags: those of an earlier one are not lost."""
    d, _ = decoder(monkeypatch, own=False, flags=flags)
    with pytest.raises(RuntimeError, match=f"bits {max(flags)}"):
        d.score([1, 2, 3], [4, 5, 6, 7, 8])
    d.score([1, 2, 3], [4, 5, 6, 7, 8])


@pytest.mark.parametrize("prompt,tokens", [([1, V], [2]), ([1, -1], [2]), ([1, 2], [3, V, 4]), ([1, 2], [-1]),
                                           ([1, 2], [2 ** 32 + 3]), (range(2 ** 40, 2 ** 40 + 3), [1])])
def test_score_refuses_ids_that_are_no_tokens(monkeypatch, prompt, tokens):
    """A step would read them as id 0 and go on from there."""
    d, log = decoder(monkeypatch, own=False)
    with pytest.raises(ValueError, match="token ids"):
        d.score(prompt, tokens)
    assert log == []
