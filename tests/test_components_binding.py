"""What the binding of the component calls lets through to the library, on host tensors and with the library's entry
points replaced by ones that write down their arguments."""
import types

import pytest

from paper_2512_14681_amd import jf


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


STREAM = types.SimpleNamespace(cuda_stream=0)


def batch(n_rows, max_rows=None, max_ctx=640):
    import torch
    i32 = dict(dtype=torch.int32)
    return jf.Batch(torch.tensor([0, n_rows], **i32), torch.zeros(1, **i32), torch.zeros(1, 10, **i32), n_rows,
                    max_rows or n_rows, max_ctx, 3)


def layout_offset(row, col, K):
    """The GEMM-input layout of include/jf.h: 16-row tiles of 128-column blocks."""
    c = col % 128
    return ((row // 16) * (K // 128) + col // 128) * 2048 + (c % 32) // 8 * 512 + (row % 16 + 16 * (c // 32)) * 8 + c % 8


@pytest.mark.parametrize("n", [1, 4, 15, 16, 17, 100])
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_attention_output_holds_whole_tiles(calls, n, act):
    """d_out is written in tiles of 16 rows, its second plane behind whole tiles: a tensor of the rows alone is refused."""
    import torch
    H, G, hd = 4, 2, 32
    K, Rp = H * hd, (n + 15) // 16 * 16
    code, dt, planes = (jf.JF_F32, torch.float32, 1) if act == "f32" else (jf.JF_BF16, torch.bfloat16, 2)
    last = (planes - 1) * Rp * K + max(layout_offset(n - 1, c, K) for c in range(K))
    assert last < planes * Rp * K and (last >= planes * n * K or n % 16 == 0)
    b = batch(n)
    args = dict(d_q=torch.zeros(planes, n, H, hd, dtype=dt),
                d_kv=torch.zeros(3 * jf.kv_page_bytes(G, hd, jf.JF_E4M3), dtype=torch.uint8),
                d_ws=torch.zeros(jf.attention_kv8_ws_bytes(b, H, G, hd), dtype=torch.uint8), stream=STREAM)
    for short in [planes * Rp * K - 1] + [planes * n * K] * (n % 16 != 0):
        with pytest.raises(ValueError, match="expected"):
            jf.attention_kv8(b, H, G, hd, code, d_out=torch.zeros(short, dtype=dt), **args)
    assert calls == []
    jf.attention_kv8(b, H, G, hd, code, d_out=torch.zeros(planes, Rp * K, dtype=dt), **args)
    assert calls == ["jf_attention_kv8"]


@pytest.mark.parametrize("act,other", [("f32", "bf16"), ("bf16", "f32"), ("f32", "f16"), ("bf16", "i32")])
def test_activation_planes_are_of_the_named_type(calls, act, other):
    """act_dtype says what the queries and outputs hold; a tensor of another type is refused, bytes are taken."""
    import torch
    H, G, hd, n = 4, 2, 32, 16
    dts = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32}
    code = {"f32": jf.JF_F32, "bf16": jf.JF_BF16}[act]
    b, size = batch(n), 4 * n * H * hd

    def planes(dt):
        return torch.zeros(size, dtype=torch.uint8).view(dt)
    pool = torch.zeros(3 * jf.kv_page_bytes(G, hd, jf.JF_E4M3), dtype=torch.uint8)
    rows = torch.zeros(n, G * hd)
    ws = torch.zeros(jf.attention_kv8_ws_bytes(b, H, G, hd), dtype=torch.uint8)

    def append(q_out):
        jf.kv_append(b, H, G, hd, jf.JF_E4M3, pool, rows, rows, d_q=torch.zeros(n, H * hd), d_q_out=q_out, act_dtype=code,
                     stream=STREAM)

    def attend(q, out):
        jf.attention_kv8(b, H, G, hd, code, q, pool, out, ws, stream=STREAM)
    right, wrong = planes(dts[act]), planes(dts[other])
    for call in (lambda: append(wrong), lambda: attend(wrong, right), lambda: attend(right, wrong)):
        with pytest.raises(TypeError, match="expected"):
            call()
    assert calls == []
    for t in (right, planes(torch.uint8)):
        append(t)
        attend(t, t.clone())
    assert calls == ["jf_kv_append", "jf_attention_kv8"] * 2


def test_the_types_appear_after_what_calls_need(monkeypatch):
    """Another thread that finds the table of types filled finds the device and stream functions too."""
    names = ("_I32", "_F32", "_U8", "_current_device", "_raw_stream")
    jf._types()
    for name in names:
        monkeypatch.delattr(jf, name)

    class Table(dict):
        def update(self, *a):
            assert all(hasattr(jf, name) for name in names)
            super().update(*a)
    monkeypatch.setattr(jf, "_DTYPES", Table())
    assert len(jf._types()) == 2


def test_counts_beyond_32_bits_are_refused(calls):
    """2^32 + 8 logits are not 8: the library's arguments have 32 bits (meta tensors, nothing is allocated)."""
    import torch
    V = 2 ** 32 + 8
    x, g = (torch.empty(1, V, dtype=torch.bfloat16, device="meta") for _ in range(2))
    norm, one = torch.zeros(1, 2), torch.zeros(1)
    for call in (lambda: jf.token_logprobs(x, None, k=1),
                 lambda: jf.token_logprobs_ws_bytes(3, V, 0), lambda: jf.token_logprobs_ws_bytes(2 ** 32 + 3, 8, 0),
                 lambda: jf.token_logprobs_ws_bytes(3, 8, 2 ** 32 + 1),
                 lambda: jf.token_logprobs_grad(x, norm, g, d_g_logprob=one, d_tokens=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(jf.JfError) as e:
            call()
        assert e.value.status == jf.JF_E_CAPACITY
    i32 = dict(dtype=torch.int32)
    three = torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros(1, 10, **i32)
    for bounds in ((2 ** 32 + 4, 4, 640, 3), (4, 4, 2 ** 32 + 640, 3), (4, 4 - 2 ** 32, 640, 3), (4, 4, 640, 2 ** 31)):
        with pytest.raises(jf.JfError) as e:
            jf.Batch(*three, *bounds)
        assert e.value.status == jf.JF_E_CAPACITY
    assert calls == []
