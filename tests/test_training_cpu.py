"""Refusals and sizes of the causal attention, shared-prefix attention and policy loss calls, without a GPU: they are
decided on the host before any HIP call, in the library and in its binding."""
import ctypes
import os
import types

import pytest

from paper_2512_14681_amd import jf

P = ctypes.c_void_p(4096)        # aligned, never dereferenced: every call below is refused or does nothing
ODD = ctypes.c_void_p(4104)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(jf.LIB_PATH):
        pytest.skip("libjf.so not built (python -m paper_2512_14681_amd.build)")
    return jf.lib()


# ---- the library ----------------------------------------------------------------------
def causal(L, n_seqs=2, n_rows=9, start=P, H=4, G=2, hd=64, dt=1, q=P, ld_q=256, k=P, ld_k=128, v=P, ld_v=128, out=P, ld_out=256):
    return L.jf_attention_causal(n_seqs, n_rows, start, H, G, hd, dt, q, ld_q, k, ld_k, v, ld_v, out, ld_out, P, None, None)


def causal_grad(L, n_seqs=2, n_rows=9, start=P, H=4, G=2, hd=64, dt=1, q=P, ld_q=256, k=P, ld_k=128, v=P, ld_v=128, out=P,
                ld_out=256, lse=P, go=P, ld_go=256, gq=P, ld_gq=256, gk=P, ld_gk=128, gv=P, ld_gv=128, ws=P):
    return L.jf_attention_causal_grad(n_seqs, n_rows, start, H, G, hd, dt, q, ld_q, k, ld_k, v, ld_v, out, ld_out, lse, go,
                                      ld_go, gq, ld_gq, gk, ld_gk, gv, ld_gv, ws, None, None)


@pytest.mark.parametrize("call", [causal, causal_grad])
@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), jf.JF_E_DTYPE), (dict(n_seqs=-1), jf.JF_E_INVAL), (dict(n_rows=-1), jf.JF_E_INVAL),
    (dict(H=3), jf.JF_E_SHAPE), (dict(G=0), jf.JF_E_SHAPE), (dict(H=0), jf.JF_E_SHAPE), (dict(hd=48), jf.JF_E_SHAPE),
    (dict(start=None), jf.JF_E_INVAL), (dict(q=None), jf.JF_E_INVAL), (dict(k=None), jf.JF_E_INVAL),
    (dict(v=None), jf.JF_E_INVAL), (dict(out=None), jf.JF_E_INVAL), (dict(ld_q=255), jf.JF_E_SHAPE),
    (dict(ld_k=127), jf.JF_E_SHAPE), (dict(ld_v=127), jf.JF_E_SHAPE), (dict(ld_out=255), jf.JF_E_SHAPE),
    (dict(n_rows=(1 << 30) + 1), jf.JF_E_CAPACITY), (dict(n_rows=1 << 29), jf.JF_E_CAPACITY),
    (dict(n_rows=0, q=None, start=None), jf.JF_OK), (dict(n_seqs=0, q=None, start=None), jf.JF_OK),
])
def test_causal_refusals(L, call, kw, status):
    assert call(L, **kw) == status
    assert status == jf.JF_OK or L.jf_last_error().decode()


@pytest.mark.parametrize("kw,status", [
    *((dict([(n, None)]), jf.JF_E_INVAL) for n in ("lse", "go", "gq", "gk", "gv", "ws")), (dict(ws=ODD), jf.JF_E_INVAL),
    (dict(ld_go=255), jf.JF_E_SHAPE), (dict(ld_gq=255), jf.JF_E_SHAPE), (dict(ld_gk=127), jf.JF_E_SHAPE),
    (dict(ld_gv=127), jf.JF_E_SHAPE),
])
def test_causal_grad_refusals(L, kw, status):
    assert causal_grad(L, **kw) == status


def test_causal_grad_workspace(L):
    f = L.jf_attention_causal_grad_ws_bytes
    assert f(1, 100, 4, 2, 48) == 0 and f(-1, 100, 4, 2, 64) == 0 and f(1, 100, 3, 2, 64) == 0
    assert f(0, 100, 4, 2, 64) > 0 and f(1, 0, 4, 2, 64) > 0
    # two floats a row and head; shares of the heads' gradients where there are few workgroups
    for n in (1, 100, 8192, 1 << 20):
        assert f(1, n, 28, 4, 128) >= n * 28 * 8
        assert f(1, n, 4, 4, 32) < n * 4 * 8 + 1024
    assert f(1, 4096, 28, 4, 128) >= 4096 * (28 * 8 + 2 * 28 * 128 * 4)


def batch(**kw):
    c = dict(n_seqs=2, n_rows=4, max_rows=2, max_ctx=128, n_pages=8, table_stride=2, d_row_start=4096, d_ctx=4096,
             d_page_table=4096)
    c.update(kw)
    return jf.JfBatch(**c)


def prefix(**kw):
    c = dict(n_groups=1, max_rows=4, max_pages=2, d_seq_start=4096, d_pages=4096)
    c.update(kw)
    return jf.JfPrefix(**c)


def shared(L, b=None, p=None, H=4, G=2, hd=64, dt=1, q=P, kv=P, out=P, ws=P, vis=None):
    return L.jf_attention_shared(ctypes.byref(b or batch()), ctypes.byref(p or prefix()), H, G, hd, dt, q, kv, vis, out, ws,
                                 None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), jf.JF_E_DTYPE), (dict(H=3), jf.JF_E_SHAPE), (dict(hd=48), jf.JF_E_SHAPE),
    (dict(H=1, G=1), jf.JF_E_SHAPE), (dict(q=None), jf.JF_E_INVAL), (dict(kv=None), jf.JF_E_INVAL),
    (dict(out=None), jf.JF_E_INVAL), (dict(ws=None), jf.JF_E_INVAL), (dict(q=ODD), jf.JF_E_INVAL),
    (dict(kv=ODD), jf.JF_E_INVAL), (dict(out=ODD), jf.JF_E_INVAL), (dict(ws=ODD), jf.JF_E_INVAL),
    (dict(b=batch(n_seqs=-1)), jf.JF_E_INVAL), (dict(b=batch(n_pages=0)), jf.JF_E_CAPACITY),
    (dict(b=batch(max_ctx=129)), jf.JF_E_CAPACITY), (dict(b=batch(d_ctx=None)), jf.JF_E_INVAL),
    (dict(b=batch(max_rows=513, n_rows=1024, max_ctx=640, table_stride=10)), jf.JF_E_CAPACITY),
    (dict(p=prefix(n_groups=-1)), jf.JF_E_INVAL), (dict(p=prefix(max_rows=-1)), jf.JF_E_INVAL),
    (dict(p=prefix(max_pages=-1)), jf.JF_E_INVAL), (dict(p=prefix(max_pages=3)), jf.JF_E_CAPACITY),
    (dict(p=prefix(d_seq_start=None)), jf.JF_E_INVAL), (dict(p=prefix(d_pages=None)), jf.JF_E_INVAL),
    (dict(p=prefix(n_groups=1 << 30)), jf.JF_E_CAPACITY),
    (dict(b=batch(n_seqs=1 << 30, n_rows=1 << 29)), jf.JF_E_CAPACITY),
    (dict(b=batch(n_rows=0), q=None), jf.JF_OK), (dict(b=batch(n_seqs=0), ws=None), jf.JF_OK),
    (dict(b=batch(max_rows=0), p=prefix(d_pages=None)), jf.JF_OK),
])
def test_shared_refusals(L, kw, status):
    assert shared(L, **kw) == status
    b, p = kw.get("b") or batch(), kw.get("p") or prefix()
    n = L.jf_attention_shared_ws_bytes(ctypes.byref(b), ctypes.byref(p), kw.get("H", 4), kw.get("G", 2), kw.get("hd", 64))
    if "b" in kw or "p" in kw or set(kw) & {"H", "hd"}:
        assert (n > 0) == (status == jf.JF_OK)


def test_shared_without_prefix(L):
    assert L.jf_attention_shared(None, None, 4, 2, 64, 1, P, P, None, P, P, None, None) == jf.JF_E_INVAL
    b = batch()
    assert L.jf_attention_shared(ctypes.byref(b), None, 4, 2, 64, 1, None, P, None, P, P, None, None) == jf.JF_E_INVAL
    one = L.jf_attention_shared_ws_bytes(ctypes.byref(b), None, 4, 2, 64)
    two = L.jf_attention_shared_ws_bytes(ctypes.byref(b), ctypes.byref(prefix()), 4, 2, 64)
    assert 0 < one <= two


def policy(L, p=None, n_seqs=2, n_rows=9, start=P, tokens=P, lp=P, old=P, ref=P, entropy=P, adv=P, stats=P, g=P, ge=P, ws=P, **kw):
    c = dict(clip_low=0.2, clip_high=0.2, kl_weight=0.1, entropy_weight=0.0, scale=1.0, mean=0, adv_rows=0)
    c.update(kw)
    return L.jf_policy_loss(ctypes.byref(jf.JfPolicy(**c)), n_seqs, n_rows, start, tokens, lp, old, ref, entropy, adv, stats,
                            g, ge, ws, None, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=-1), jf.JF_E_INVAL), (dict(n_rows=-1), jf.JF_E_INVAL), (dict(n_rows=(1 << 22) + 1), jf.JF_E_CAPACITY),
    (dict(n_seqs=(1 << 22) + 1), jf.JF_E_CAPACITY), (dict(clip_low=-0.1), jf.JF_E_INVAL), (dict(clip_low=1.1), jf.JF_E_INVAL),
    (dict(clip_low=NAN), jf.JF_E_INVAL), (dict(clip_high=-0.1), jf.JF_E_INVAL), (dict(clip_high=NAN), jf.JF_E_INVAL),
    (dict(kl_weight=INF), jf.JF_E_INVAL), (dict(entropy_weight=NAN), jf.JF_E_INVAL), (dict(scale=INF), jf.JF_E_INVAL),
    (dict(mean=3), jf.JF_E_INVAL), (dict(adv_rows=2), jf.JF_E_INVAL), (dict(start=None), jf.JF_E_INVAL),
    (dict(lp=None), jf.JF_E_INVAL), (dict(old=None), jf.JF_E_INVAL), (dict(adv=None), jf.JF_E_INVAL),
    (dict(stats=None), jf.JF_E_INVAL), (dict(ws=None), jf.JF_E_INVAL), (dict(ws=ODD), jf.JF_E_INVAL),
    (dict(entropy=None), jf.JF_E_INVAL),      # its gradient is asked for
])
def test_policy_refusals(L, kw, status):
    assert policy(L, **kw) == status
    assert L.jf_last_error().decode()


def test_policy_workspace(L):
    f = L.jf_policy_loss_ws_bytes
    assert L.jf_policy_loss(None, 1, 1, P, P, P, P, P, P, P, P, P, P, P, None, None) == jf.JF_E_INVAL
    assert f(-1, 4) == 0 and f(4, (1 << 22) + 1) == 0 and f(0, 0) > 0
    assert f(1000, 1 << 20) >= 1000 * 4 + 1024 * (4 + 40)


# ---- the binding ----------------------------------------------------------------------
STREAM = types.SimpleNamespace(cuda_stream=0)


@pytest.fixture
def calls(monkeypatch):
    """The names of the library calls that were reached; host tensors pass for the GPU's."""
    jf._types()
    seen = []
    real = jf.lib()

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(real, name)
            return lambda *a: seen.append(name) or jf.JF_OK
    monkeypatch.setattr(jf, "lib", lambda: Lib())
    monkeypatch.setattr(jf, "_current_device", lambda: -1)   # what host tensors answer
    return seen


def causal_args(n=10, H=4, G=2, hd=32):
    import torch
    z = lambda w: torch.zeros(n, w)
    return dict(d_row_start=torch.tensor([0, 4, n], dtype=torch.int32), n_heads=H, n_kv_heads=G, head_dim=hd, d_q=z(H * hd),
                d_k=z(G * hd), d_v=z(G * hd), d_out=z(H * hd), d_lse=torch.zeros(H, n), stream=STREAM)


def grad_args():
    import torch
    a = causal_args()
    a.update(d_g_out=a["d_q"].clone(), d_g_q=a["d_q"].clone(), d_g_k=a["d_k"].clone(), d_g_v=a["d_k"].clone(),
             d_ws=torch.zeros(jf.attention_causal_grad_ws_bytes(2, 10, 4, 2, 32), dtype=torch.uint8))
    return a


def test_binding_of_causal_attention(calls):
    import torch
    jf.attention_causal(**causal_args())
    jf.attention_causal_grad(**grad_args())
    assert calls == ["jf_attention_causal", "jf_attention_causal_grad"]
    del calls[:]
    for make, call, names in ((causal_args, jf.attention_causal, ("d_q", "d_k", "d_v", "d_out")),
                              (grad_args, jf.attention_causal_grad, ("d_q", "d_k", "d_v", "d_out", "d_g_out", "d_g_q",
                                                                     "d_g_k", "d_g_v"))):
        for name in names:
            for wrong in (lambda t: t.to(torch.bfloat16), lambda t: t[:, :-1], lambda t: t.t().contiguous().t(),
                          lambda t: t.reshape(-1), lambda t: t.half(), lambda t: t[:9] if name != "d_q" else t.half()):
                a = make()
                a[name] = wrong(a[name])
                with pytest.raises((TypeError, ValueError)):
                    call(**a)
        for name, wrong in (("d_lse", lambda t: t[:, :-1].contiguous()), ("d_lse", lambda t: t.double()),
                            ("d_row_start", lambda t: t.long()), ("d_row_start", lambda t: t[::2]),
                            ("d_row_start", lambda t: t[:0])):
            a = make()
            a[name] = wrong(a[name])
            with pytest.raises((TypeError, ValueError)):
                call(**a)
    a = grad_args()
    a["d_ws"] = a["d_ws"][:-1]
    with pytest.raises(ValueError):
        jf.attention_causal_grad(**a)
    with pytest.raises(jf.JfError):
        jf.attention_causal_grad_ws_bytes(1, 10, 4, 3, 32)
    with pytest.raises(jf.JfError):
        jf.attention_causal_grad_ws_bytes(1, 2 ** 32 + 10, 4, 2, 32)
    assert calls == []


def shared_args(act, n=5, H=4, G=2, hd=32):
    import torch
    i32 = dict(dtype=torch.int32)
    b = jf.Batch(torch.tensor([0, 2, n], **i32), torch.zeros(2, **i32), torch.zeros(2, 10, **i32), n, 3, 640, 3)
    p = jf.Prefix(torch.tensor([0, 2], **i32), torch.zeros(1, **i32), n, 4)
    code, dt, planes = (jf.JF_F32, torch.float32, 1) if act == "f32" else (jf.JF_BF16, torch.bfloat16, 2)
    return dict(batch=b, prefix=p, n_heads=H, n_kv_heads=G, head_dim=hd, dtype=code,
                d_q=torch.zeros(planes, n, H, hd, dtype=dt), d_kv=torch.zeros(3 * 2 * G * 64 * hd, dtype=dt),
                d_out=torch.zeros(planes, 16 * H * hd, dtype=dt),
                d_ws=torch.zeros(jf.attention_shared_ws_bytes(b, p, H, G, hd), dtype=torch.uint8),
                d_vis=torch.zeros(n, 8, dtype=torch.int64), stream=STREAM)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_binding_of_shared_attention(calls, act):
    import torch
    jf.attention_shared(**shared_args(act))
    a = shared_args(act)
    a["prefix"] = None
    jf.attention_shared(**a)
    assert calls == ["jf_attention_shared"] * 2
    other = torch.bfloat16 if act == "f32" else torch.float32
    for name, wrong in (("d_q", lambda t: t.to(other)), ("d_q", lambda t: t[:, :-1].contiguous()),
                        ("d_kv", lambda t: t[:-1]), ("d_out", lambda t: t[:, :-1].contiguous()),
                        ("d_out", lambda t: t.to(other)), ("d_ws", lambda t: t[:-1]), ("d_vis", lambda t: t[:-1])):
        a = shared_args(act)
        a[name] = wrong(a[name])
        with pytest.raises((TypeError, ValueError)):
            jf.attention_shared(**a)
    i32 = dict(dtype=torch.int32)
    for start, pages in ((torch.zeros(2, **i32), torch.zeros(2, **i32)), (torch.zeros(3), torch.zeros(2, **i32)),
                         (torch.zeros(3, **i32), torch.zeros(4, **i32)[::2])):
        with pytest.raises((TypeError, ValueError)):
            jf.Prefix(start, pages, 1, 1)
    with pytest.raises(jf.JfError):
        jf.Prefix(torch.zeros(2, **i32), torch.zeros(1, **i32), 2 ** 32 + 1, 1)
    b = shared_args(act)["batch"]
    with pytest.raises(jf.JfError):
        jf.attention_shared_ws_bytes(b, None, 4, 3, 32)
    with pytest.raises(jf.JfError):
        jf.attention_shared_ws_bytes(b, jf.Prefix(torch.zeros(2, **i32), torch.zeros(1, **i32), 5, 11), 4, 2, 32)
    assert len(calls) == 2


def test_workspaces_of_two_prefixes_differ(calls):
    """A batch remembers workspace sizes: one prefix's is not another's."""
    import torch
    i32 = dict(dtype=torch.int32)
    b = jf.Batch(torch.tensor([0, 2], **i32), torch.zeros(1, **i32), torch.zeros(1, 1000, **i32), 2, 2, 64000, 3)
    small = jf.Prefix(torch.tensor([0, 1], **i32), torch.zeros(1, **i32), 2, 4)
    large = jf.Prefix(torch.tensor([0, 1], **i32), torch.zeros(1, **i32), 2, 900)
    sizes = [jf.attention_shared_ws_bytes(b, p, 4, 2, 32) for p in (None, small, large, small, None)]
    L = jf.lib()
    direct = [L.jf_attention_shared_ws_bytes(b.ref, p and p.ref, 4, 2, 32) for p in (None, small, large, small, None)]
    assert sizes == direct and sizes[0] != sizes[1]
    n = jf.attention_kv8_ws_bytes(b, 4, 2, 32)
    assert n == jf.lib().jf_attention_kv8_ws_bytes(b.ref, 4, 2, 32)


def policy_args(n=10):
    import torch
    z = lambda k=n: torch.zeros(k)
    return dict(d_row_start=torch.tensor([0, 4, n], dtype=torch.int32), d_tokens=torch.zeros(n, dtype=torch.int32),
                d_logprob=z(), d_old_logprob=z(), d_advantage=z(2), d_stats=z(6), d_ref_logprob=z(), d_entropy=z(),
                d_g_logprob=z(), d_g_entropy=z(), d_ws=torch.zeros(jf.policy_loss_ws_bytes(2, n), dtype=torch.uint8),
                stream=STREAM)


def test_binding_of_the_policy_loss(calls):
    import torch
    jf.policy_loss(**policy_args())
    a = policy_args()
    a.update(d_advantage=torch.zeros(10), adv_rows=True, d_tokens=None, d_ref_logprob=None, d_entropy=None, d_g_logprob=None,
             d_g_entropy=None)
    jf.policy_loss(**a)
    assert calls == ["jf_policy_loss"] * 2
    for name in ("d_tokens", "d_old_logprob", "d_stats", "d_ref_logprob", "d_entropy", "d_g_logprob", "d_g_entropy", "d_ws",
                 "d_advantage", "d_logprob"):
        for wrong in (lambda t: t[:-1], lambda t: t.double(), lambda t: t.repeat(2)[::2]):
            a = policy_args()
            if name == "d_logprob" and wrong(a[name]).dtype == torch.float32 and wrong(a[name]).is_contiguous():
                continue      # fewer rows are fewer rows
            a[name] = wrong(a[name])
            if name == "d_ws" and a[name].nbytes >= policy_args()["d_ws"].nbytes and a[name].is_contiguous():
                continue
            with pytest.raises((TypeError, ValueError)):
                jf.policy_loss(**a)
    a = policy_args()
    with pytest.raises(TypeError):
        jf.policy_loss(**dict(a, adv_rows=True))      # two advantages for ten rows
    with pytest.raises(jf.JfError):
        jf.policy_loss_ws_bytes(2, (1 << 22) + 1)
    assert len(calls) == 2
