"""Refusals and sizes of the batch and log-probability calls without a GPU:
they are decided on the host before any HIP call."""
import ctypes
import os

import pytest

from paper_2512_14681_amd import jf
from oracle import batch as ob

P = ctypes.c_void_p(4096)        # aligned, never dereferenced: every call below is refused or does nothing
ODD = ctypes.c_void_p(4104)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(jf.LIB_PATH):
        pytest.skip("libjf.so not built (python -m paper_2512_14681_amd.build)")
    return jf.lib()


def batch(**kw):
    c = dict(n_seqs=2, n_rows=4, max_rows=2, max_ctx=128, n_pages=8, table_stride=2, d_row_start=4096, d_ctx=4096,
             d_page_table=4096)
    c.update(kw)
    return jf.JfBatch(**c)


def append(L, b=None, H=4, G=2, hd=64, kv=jf.JF_E4M3, x=jf.JF_F32, act=jf.JF_BF16, q=P, ld_q=256, k=P, ld_k=128, v=P,
           ld_v=128, pos=None, base=1e4, d_kv=P, q_out=P):
    b = batch() if b is None else b
    return L.jf_kv_append(ctypes.byref(b), H, G, hd, kv, x, act, q, ld_q, k, ld_k, v, ld_v, pos, base, d_kv, q_out,
                          None, None)


def read(L, b=None, G=2, hd=64, kv=jf.JF_E4M3, x=jf.JF_BF16, d_kv=P, k=P, ld_k=128, v=P, ld_v=128):
    b = batch() if b is None else b
    return L.jf_kv_read(ctypes.byref(b), G, hd, kv, x, d_kv, k, ld_k, v, ld_v, None, None)


def attend(L, b=None, H=4, G=2, hd=64, act=jf.JF_BF16, q=P, kv=P, vis=None, out=P, ws=P):
    b = batch() if b is None else b
    return L.jf_attention_kv8(ctypes.byref(b), H, G, hd, act, q, kv, vis, out, ws, None, None)


BAD_BATCHES = [
    (dict(n_seqs=-1), jf.JF_E_INVAL), (dict(n_rows=-1), jf.JF_E_INVAL), (dict(n_pages=-1), jf.JF_E_INVAL),
    (dict(max_ctx=129), jf.JF_E_CAPACITY), (dict(max_rows=129), jf.JF_E_CAPACITY),
    (dict(max_ctx=(1 << 30) + 1, table_stride=1 << 30), jf.JF_E_CAPACITY),
    (dict(n_pages=0), jf.JF_E_CAPACITY), (dict(d_row_start=None), jf.JF_E_INVAL), (dict(d_ctx=None), jf.JF_E_INVAL),
    (dict(d_page_table=None), jf.JF_E_INVAL),
]


@pytest.mark.parametrize("fields,status", BAD_BATCHES)
def test_bad_batches_are_refused(L, fields, status):
    for call in (append, read, attend):
        assert call(L, batch(**fields)) == status, call.__name__
        assert L.jf_last_error().decode()


def test_append_refusals(L):
    assert L.jf_kv_append(None, 4, 2, 64, 2, 0, 1, P, 256, P, 128, P, 128, None, 1e4, P, P, None, None) == jf.JF_E_INVAL
    assert append(L, hd=48) == jf.JF_E_SHAPE
    assert append(L, H=3) == jf.JF_E_SHAPE
    assert append(L, G=0) == jf.JF_E_SHAPE
    assert append(L, kv=3) == jf.JF_E_DTYPE
    assert append(L, x=jf.JF_E4M3) == jf.JF_E_DTYPE
    assert append(L, act=jf.JF_E4M3) == jf.JF_E_DTYPE
    for base in (1.0, -1.0, 0.5, float("inf"), float("nan")):
        assert append(L, base=base) == jf.JF_E_INVAL
    for name in ("k", "v", "d_kv", "q_out"):
        assert append(L, **{name: None}) == jf.JF_E_INVAL
    assert append(L, d_kv=ODD) == jf.JF_E_INVAL
    assert append(L, q_out=ODD) == jf.JF_E_INVAL
    for name in ("ld_k", "ld_v"):
        assert append(L, **{name: 127}) == jf.JF_E_SHAPE
    assert append(L, ld_q=255) == jf.JF_E_SHAPE
    big = batch(n_seqs=4096, max_rows=1 << 20, max_ctx=1 << 20, table_stride=1 << 14, n_rows=1 << 20)
    assert append(L, big) == jf.JF_E_CAPACITY
    assert "launch" in L.jf_last_error().decode()


def test_read_refusals(L):
    assert read(L, kv=5) == jf.JF_E_DTYPE
    assert read(L, x=jf.JF_E4M3) == jf.JF_E_DTYPE
    assert read(L, hd=96) == jf.JF_E_SHAPE
    for name in ("d_kv", "k", "v"):
        assert read(L, **{name: None}) == jf.JF_E_INVAL
    assert read(L, d_kv=ODD) == jf.JF_E_INVAL
    assert read(L, ld_v=64) == jf.JF_E_SHAPE


def test_attention_refusals(L):
    assert attend(L, act=jf.JF_E4M3) == jf.JF_E_DTYPE
    assert attend(L, hd=16) == jf.JF_E_SHAPE
    assert attend(L, H=1, G=1, hd=64) == jf.JF_E_SHAPE      # 64 columns are no GEMM input
    assert attend(L, H=5) == jf.JF_E_SHAPE
    wide = dict(max_ctx=1024, table_stride=16, n_rows=2000)
    assert attend(L, batch(max_rows=jf.JF_MAX_ROWS + 1, **wide)) == jf.JF_E_CAPACITY
    for name in ("q", "kv", "out", "ws"):
        assert attend(L, **{name: None}) == jf.JF_E_INVAL
        assert attend(L, **{name: ODD}) == jf.JF_E_INVAL
    b = batch(max_rows=jf.JF_MAX_ROWS + 1, **wide)
    assert L.jf_attention_kv8_ws_bytes(ctypes.byref(b), 4, 2, 64) == 0
    assert L.jf_attention_kv8_ws_bytes(None, 4, 2, 64) == 0


@pytest.mark.parametrize("field", ["n_seqs", "n_rows", "max_rows"])
def test_empty_batches_do_nothing(L, field):
    b = batch(**{field: 0, "d_row_start": None, "d_ctx": None, "d_page_table": None})
    assert append(L, b, k=None, v=None, d_kv=None) == jf.JF_OK
    assert read(L, b, d_kv=None) == jf.JF_OK
    assert attend(L, b, q=None) == jf.JF_OK
    assert L.jf_attention_kv8_ws_bytes(ctypes.byref(b), 4, 2, 64) > 0


def test_page_and_workspace_bytes(L):
    for G in (1, 2, 4, 7):
        for hd in (32, 64, 128):
            assert L.jf_kv_page_bytes(G, hd, jf.JF_F32) == 2 * G * 64 * hd * 4
            assert L.jf_kv_page_bytes(G, hd, jf.JF_BF16) == 2 * G * 64 * hd * 2
            assert L.jf_kv_page_bytes(G, hd, jf.JF_E4M3) == ob.page_bytes(G, hd)
    assert L.jf_kv_page_bytes(4, 96, 2) == L.jf_kv_page_bytes(0, 64, 2) == L.jf_kv_page_bytes(4, 64, 3) == 0
    # enough for fewer rows too, whatever their split
    for V in (1, 4097, 50257, 152064):
        most = 0
        for R in list(range(1, 300)) + [499, 500, 511, 512, 1023, 1024, 1025, 4096]:
            n = L.jf_token_logprobs_ws_bytes(R, V, 8)
            assert n >= most
            most = n
    assert L.jf_token_logprobs_ws_bytes(0, 10, 0) == 0
    assert L.jf_token_logprobs_ws_bytes(4, 10, jf.JF_MAX_TOP + 1) == 0


def logprobs(L, R=4, V=100, dtype=jf.JF_F32, x=P, ld=100, tok=P, k=2, lp=P, ws=P):
    return L.jf_token_logprobs(R, V, dtype, x, ld, tok, k, lp, None, None, None, None, ws, None)


def grad(L, R=4, V=100, dtype=jf.JF_F32, x=P, ld=100, tok=P, norm=P, ent=P, g=P, h=P, out=ODD, ld_g=100):
    return L.jf_token_logprobs_grad(R, V, dtype, x, ld, tok, norm, ent, g, h, out, ld_g, None)


def test_logprob_refusals(L):
    for call in (logprobs, grad):
        assert call(L, dtype=jf.JF_E4M3) == jf.JF_E_DTYPE
        assert call(L, V=0) == jf.JF_E_SHAPE
        assert call(L, R=-1) == jf.JF_E_SHAPE
        assert call(L, ld=99) == jf.JF_E_SHAPE
        assert call(L, V=(1 << 30) + 1, ld=1 << 31) == jf.JF_E_CAPACITY
        assert call(L, R=(1 << 22) + 1) == jf.JF_E_CAPACITY
        assert call(L, x=None) == jf.JF_E_INVAL
        assert call(L, tok=None) == jf.JF_E_INVAL
        assert call(L, R=0, x=None) == jf.JF_OK
    for k in (-1, jf.JF_MAX_TOP + 1):
        assert logprobs(L, k=k) == jf.JF_E_SHAPE
    assert logprobs(L, ws=None) == jf.JF_E_INVAL
    assert logprobs(L, ws=ODD) == jf.JF_E_INVAL
    for name in ("norm", "ent", "out"):
        assert grad(L, **{name: None}) == jf.JF_E_INVAL
    assert grad(L, ld_g=99) == jf.JF_E_SHAPE
    assert grad(L, out=P, ld_g=101) == jf.JF_E_INVAL        # in place on another stride
    assert grad(L, R=1 << 20, V=152064, ld=152064, ld_g=152064) == jf.JF_E_CAPACITY


def test_binding_checks_its_tensors():
    import torch
    i32 = dict(dtype=torch.int32)
    with pytest.raises(TypeError):
        jf.Batch(torch.zeros(3), torch.zeros(2, **i32), torch.zeros(2, 1, **i32), 4, 2, 64, 1)
    with pytest.raises(ValueError):
        jf.Batch(torch.zeros(2, **i32), torch.zeros(2, **i32), torch.zeros(2, 1, **i32), 4, 2, 64, 1)
    with pytest.raises(ValueError):
        jf.Batch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, **i32), 4, 2, 64, 1)
    with pytest.raises(TypeError):
        jf.token_logprobs(torch.zeros(4, 8, dtype=torch.float16), None)
    with pytest.raises(TypeError):
        jf.token_logprobs(torch.zeros(8, 4).t(), None)
    with pytest.raises(TypeError):
        jf.token_logprobs_grad(torch.zeros(4, 8), None, torch.zeros(4, 8, dtype=torch.bfloat16))


def test_binding_refuses_tensors_elsewhere(monkeypatch):
    """Host tensors, short vectors and other types never reach the library as addresses."""
    import torch
    jf._types()
    monkeypatch.setattr(jf, "_current_device", lambda: 0)
    x, i32 = torch.zeros(4, 8), dict(dtype=torch.int32)
    with pytest.raises(ValueError, match="on cpu"):
        jf.token_logprobs(x, torch.zeros(1024, dtype=torch.uint8))
    with pytest.raises(TypeError, match="int32"):
        jf._vec(0, torch.zeros(4, dtype=torch.int64), torch.int32, 4)
    for bad in (torch.zeros(3), torch.zeros(8)[::2], torch.zeros(4, dtype=torch.bfloat16)):
        with pytest.raises((TypeError, ValueError)):
            jf._vec(0, bad, torch.float32, 4)
    b = jf.Batch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 1, **i32), 4, 2, 64, 1)
    with pytest.raises(ValueError, match="batch is on"):
        jf.kv_read(b, 1, 32, jf.JF_BF16, x, torch.zeros(4, 32), torch.zeros(4, 32))


def test_binding_refuses_short_tensors(monkeypatch):
    """Fewer rows than the batch has, narrow rows, small pools and strided outputs never reach the library."""
    import torch
    jf._types()
    monkeypatch.setattr(jf, "_current_device", lambda: -1)   # what host tensors answer
    i32 = dict(dtype=torch.int32)
    G, hd, n = 2, 32, 4
    for kv, dtype in ((jf.JF_F32, torch.float32), (jf.JF_BF16, torch.bfloat16), (jf.JF_E4M3, torch.uint8)):
        b = jf.Batch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 1, **i32), n, 2, 64, 3)
        assert jf._pool_bytes(b, G, hd, kv) == 3 * jf.kv_page_bytes(G, hd, kv)
        pool = torch.zeros(jf._pool_bytes(b, G, hd, kv) // torch.zeros(1, dtype=dtype).element_size(), dtype=dtype)
        rows, q = torch.zeros(n, G * hd), torch.zeros(n, 4 * hd)
        out = torch.zeros(n, 4, hd)
        ok = dict(d_kv=pool, d_k=rows, d_v=rows, d_q=q, d_q_out=out)
        for bad in (dict(d_k=rows[1:]), dict(d_v=rows[:, 1:]), dict(d_q=q[:3]), dict(d_q=q[:, :96]),
                    dict(d_kv=pool[:-1]), dict(d_q_out=out[1:]), dict(d_q_out=out.transpose(0, 1))):
            with pytest.raises(ValueError, match="expected"):
                jf.kv_append(b, 4, G, hd, kv, act_dtype=jf.JF_F32, **{**ok, **bad})
        for bad in (dict(d_k=rows[1:]), dict(d_v=rows[:, 1:]), dict(d_kv=pool[:-1])):
            with pytest.raises(ValueError, match="expected"):
                jf.kv_read(b, G, hd, kv, **{**{k: ok[k] for k in ("d_kv", "d_k", "d_v")}, **bad})
    ok = dict(d_q=out, d_kv=pool, d_out=out, d_ws=None, d_vis=torch.zeros(n, jf.JF_VIS_WORDS, dtype=torch.int64))
    for bad in (dict(d_q=out[1:]), dict(d_kv=pool[:-1]), dict(d_out=out[1:]), dict(d_vis=ok["d_vis"][1:]),
                dict(d_q=out.transpose(0, 1)), dict(d_ws=torch.zeros(jf.attention_kv8_ws_bytes(b, 4, G, hd) // 4 - 1))):
        with pytest.raises(ValueError, match="expected"):
            jf.attention_kv8(b, 4, G, hd, jf.JF_F32, **{**ok, **bad})
    x = torch.zeros(3, 5000)
    with pytest.raises(ValueError, match="expected"):
        jf.token_logprobs(x, torch.zeros(jf.token_logprobs_ws_bytes(3, 5000, 4) - 1, dtype=torch.uint8), k=4)


def test_batch_takes_a_loose_bound_on_the_rows():
    """More rows a sequence than the slots allow: the call itself refuses it, the binding takes the slots' bound."""
    import torch
    i32 = dict(dtype=torch.int32)
    b = jf.Batch(torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 1, **i32), 4, 70, 33, 3)
    assert (b.c.max_rows, b.c.max_ctx) == (33, 33)
    assert jf.attention_kv8_ws_bytes(b, 4, 2, 64) > 0
