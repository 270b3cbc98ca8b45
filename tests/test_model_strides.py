"""Tensors of heads whose strides go backwards, which the C entry points take and
torch cannot express: the same bits as from the tensors turned round."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2409_07704_amd._native import AttentionDesc, Heads, QkDesc

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
CODE = {F32: 0, F16: 1, BF16: 2}


@pytest.fixture(scope="module")
def mas():
    import paper_2409_07704_amd as m

    m.lib()
    return m


def plain(x):
    return Heads(x.data_ptr(), x.stride(0), x.stride(1), x.stride(2))


def backwards(x, dims):
    """mas_heads of x flipped along `dims` (of 0, 1, 2): the same memory from its other end."""
    data, strides = x.data_ptr(), list(x.stride()[:3])
    for d in dims:
        data += (x.shape[d] - 1) * strides[d] * x.element_size()
        strides[d] = -strides[d]
    return Heads(data, *strides)


def rand(gen, *shape, dtype):
    return torch.randn(shape, generator=gen).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("B,T,Hq,Hk,D", [
    (2, 200, 4, 2, 64),   # few rows and keys, whole tiles and a cut one
    (2, 1, 8, 2, 128),    # a step
    (3, 70, 6, 2, 40),    # a group of three
    (90, 150, 6, 3, 64),  # tiles that a workgroup shares
    (90, 150, 3, 3, 128),
])
def test_attention(mas, dtype, B, T, Hq, Hk, D):
    print(f"[gpu-case] strides that go backwards B={B} T={T} Hq={Hq} Hk={Hk} D={D} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(D + T)
    q, g = (rand(gen, B, T, Hq, D, dtype=dtype) for _ in range(2))
    k, v = (rand(gen, B, T, Hk, D, dtype=dtype) for _ in range(2))
    L, s = mas.lib(), torch.cuda.current_stream().cuda_stream
    desc = AttentionDesc(B, T, T, Hq, Hk, D, CODE[dtype], 1, 1, D**-0.5, 0.0, None, None, None, None, None)
    n = L.mas_attention_workspace_bytes(desc, 1)
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    ptr = ctypes.c_void_p(ws.data_ptr() + -ws.data_ptr() % 256)

    def run(view, q, k, v, g):
        out, dq = (torch.full_like(q, 7.0) for _ in range(2))
        dk, dv = (torch.full_like(k, 7.0) for _ in range(2))
        lse = torch.full((B, Hq, T), 7.0, device="cuda")
        assert L.mas_attention(desc, view(q), view(k), view(v), view(out), lse.data_ptr(), ptr, n, s) == 0
        assert L.mas_attention_backward(desc, view(g), view(q), view(k), view(v), view(out), lse.data_ptr(), view(dq), view(dk),
                                        view(dv), ptr, n, s) == 0
        torch.cuda.synchronize()
        return out, dq, dk, dv, lse

    for dims in ((1,), (2,), (0, 1, 2)):
        back = run(lambda x: backwards(x, dims), q, k, v, g)
        want = run(plain, *(x.flip(dims).contiguous() for x in (q, k, v, g)))
        for name, x, y in zip(("out", "dq", "dk", "dv"), back, want):
            assert torch.equal(x.flip(dims), y), (dims, name)
        assert torch.equal(back[4], want[4]), dims


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 7])
def test_norm_and_rotation(mas, dtype, D):
    B, T, Hq, Hk, R = 2, 33, 4, 2, D // 2 * 2
    print(f"[gpu-case] norm, strides that go backwards D={D} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(D)
    q, gq = (rand(gen, B, T, Hq, D, dtype=dtype) for _ in range(2))
    k, gk = (rand(gen, B, T, Hk, D, dtype=dtype) for _ in range(2))
    cos, sin = (rand(gen, T, R // 2, dtype=F32) for _ in range(2))
    L, s = mas.lib(), torch.cuda.current_stream().cuda_stream
    desc = QkDesc(B, T, Hq, Hk, D, R, T, CODE[dtype], 0, 1e-6, None, None, cos.data_ptr(), sin.data_ptr(), None, None)
    n = L.mas_qk_norm_rope_workspace_bytes(B, T, Hq, Hk, D)
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    ptr = ctypes.c_void_p(ws.data_ptr() + -ws.data_ptr() % 256)

    def run(view, q, k, gq, gk):
        outs = [torch.full_like(x, 7.0) for x in (q, k, q, k)]
        dw = torch.full((2, D), 7.0, device="cuda")
        assert L.mas_qk_norm_rope(desc, view(q), view(k), view(outs[0]), view(outs[1]), s) == 0
        assert L.mas_qk_norm_rope_backward(desc, view(gq), view(gk), view(q), view(k), view(outs[2]), view(outs[3]),
                                           dw[0].data_ptr(), dw[1].data_ptr(), ptr, n, s) == 0
        torch.cuda.synchronize()
        return outs, dw

    for dims in ((1,), (0, 1)):
        back, dw = run(lambda x: backwards(x, dims), q, k, gq, gk)
        want, dw2 = run(plain, *(x.flip(dims).contiguous() for x in (q, k, gq, gk)))
        for x, y in zip(back, want):
            assert torch.equal(x.flip(dims), y), dims
        assert torch.equal(dw, dw2)
