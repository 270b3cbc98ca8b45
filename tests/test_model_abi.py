"""Host-side checks of the operators around the alignment: what their C entry
points refuse before anything touches the GPU."""
from __future__ import annotations

import ctypes

import pytest

import paper_2409_07704_amd as mas
from paper_2409_07704_amd import _native
from paper_2409_07704_amd._native import AttentionDesc, Heads, QkDesc

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: validation fails first
H = Heads(0x10000, 64, 64, 64)
NULL, SHAPE, WORKSPACE, VALUE = 1, 2, 3, 6


def attention(**change):
    d = dict(B=1, Tq=8, Tk=8, Hq=2, Hk=1, D=64, dtype=2, causal=1, N=1, scale=0.1, cap=0.0)
    return AttentionDesc(**dict(d, **change))


BAD_ATTENTION = [
    (dict(B=0), SHAPE), (dict(Tq=0), SHAPE), (dict(Tk=-1), SHAPE), (dict(Hk=0), SHAPE), (dict(Hq=3, Hk=2), SHAPE),
    (dict(D=0), SHAPE), (dict(D=129), SHAPE), (dict(Tq=1 << 30, Hq=4), SHAPE), (dict(B=1 << 22, Tq=64), SHAPE),
    (dict(Tq=1 << 20, Hq=256), SHAPE), (dict(N=0, doc_start=0x10000), SHAPE), (dict(N=2, prefix=0x10000), SHAPE),
    (dict(dtype=3), VALUE), (dict(dtype=-1), VALUE), (dict(scale=float("inf")), VALUE), (dict(cap=float("nan")), VALUE),
    (dict(cap=-2.0), VALUE), (dict(causal=0, prefix=0x10000), VALUE),
]


@pytest.mark.parametrize("change,code", BAD_ATTENTION)
def test_attention_descriptions(change, code):
    L, d = mas.lib(), attention(**change)
    assert L.mas_attention_workspace_bytes(d, 0) == 0
    assert L.mas_attention(d, H, H, H, H, None, FAKE, 1 << 40, None) == code
    assert L.mas_attention_backward(d, H, H, H, H, H, FAKE, H, H, H, FAKE, 1 << 40, None) == code


def test_attention_pointers_and_workspaces():
    L, d, no = mas.lib(), attention(), Heads()
    for n in range(4):
        heads = [H] * 4
        for missing in (None, no):
            heads[n] = missing
            assert L.mas_attention(d, *heads, None, FAKE, 1 << 40, None) == NULL
    assert L.mas_attention(None, H, H, H, H, None, FAKE, 1 << 40, None) == NULL
    for n in range(8):
        heads = [H] * 8
        heads[n] = no
        args = heads[:5] + [FAKE] + heads[5:]
        assert L.mas_attention_backward(d, *args, FAKE, 1 << 40, None) == NULL
    assert L.mas_attention_backward(d, H, H, H, H, H, None, H, H, H, FAKE, 1 << 40, None) == NULL
    assert L.mas_attention(d, H, Heads(0x10001, 64, 64, 64), H, H, None, FAKE, 1 << 40, None) == VALUE
    # Short calls over long keys need room for their parts; so do all gradients.
    long = attention(Tk=4096)
    n = L.mas_attention_workspace_bytes(long, 0)
    assert n > 256 and n % 256 == 0 and L.mas_attention_workspace_bytes(long, 1) >= n
    assert L.mas_attention(long, H, H, H, H, None, None, 0, None) == WORKSPACE
    assert L.mas_attention(long, H, H, H, H, None, FAKE, 256, None) == WORKSPACE
    assert L.mas_attention(long, H, H, H, H, None, ctypes.c_void_p(0x10010), n, None) == WORKSPACE
    assert L.mas_attention_backward(d, H, H, H, H, H, FAKE, H, H, H, FAKE, 16, None) == WORKSPACE


def qk(**change):
    d = dict(B=1, T=4, Hq=2, Hk=1, D=64, R=64, P=16, dtype=2, interleaved=0, eps=1e-6, cos=0x10000, sin=0x10000)
    return QkDesc(**dict(d, **change))


@pytest.mark.parametrize("change,code", [
    (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(Hq=0), SHAPE), (dict(Hk=-1), SHAPE), (dict(D=0, R=0), SHAPE),
    (dict(D=257), SHAPE), (dict(R=66), SHAPE), (dict(R=63), SHAPE), (dict(R=-2), SHAPE), (dict(P=0), SHAPE),
    (dict(B=1 << 20, T=17), SHAPE), (dict(dtype=5), VALUE), (dict(eps=-1e-6), VALUE), (dict(eps=float("nan")), VALUE),
    (dict(cos=None), NULL), (dict(sin=None), NULL),
])
def test_norm_and_rotation_descriptions(change, code):
    L, d = mas.lib(), qk(**change)
    assert L.mas_qk_norm_rope(d, H, H, H, H, None) == code
    assert L.mas_qk_norm_rope_backward(d, H, H, H, H, H, H, None, None, FAKE, 1 << 40, None) == code


def test_norm_and_rotation_pointers_and_workspaces():
    L, d, no = mas.lib(), qk(), Heads()
    for n in range(4):
        heads = [H] * 4
        heads[n] = no
        assert L.mas_qk_norm_rope(d, *heads, None) == NULL
    for n in range(6):
        heads = [H] * 6
        heads[n] = None
        assert L.mas_qk_norm_rope_backward(d, *heads, None, None, FAKE, 1 << 40, None) == NULL
    assert L.mas_qk_norm_rope(None, H, H, H, H, None) == NULL
    assert L.mas_qk_norm_rope(d, Heads(0x10001, 64, 64, 64), H, H, H, None) == VALUE
    assert L.mas_qk_norm_rope_workspace_bytes(1, 4, 2, 1, 64) % 256 == 0
    for bad in ((0, 4, 2, 1, 64), (1, 0, 2, 1, 64), (1, 4, 0, 1, 64), (1, 4, 2, -1, 64), (1, 4, 2, 1, 257)):
        assert L.mas_qk_norm_rope_workspace_bytes(*bad) == 0
    assert L.mas_qk_norm_rope_backward(d, H, H, H, H, H, H, None, None, None, 0, None) == WORKSPACE
    assert L.mas_qk_norm_rope_backward(d, H, H, H, H, H, H, None, None, FAKE, 64, None) == WORKSPACE


def test_aligned_loss():
    L = mas.lib()

    def call(shape=(1, 2, 3, 4), pointers=(FAKE, FAKE, FAKE, FAKE, FAKE), loss=FAKE, ws=(FAKE, 1 << 40)):
        return L.mas_align_loss(*pointers, *shape, loss, FAKE, FAKE, FAKE, *ws, None)

    for n in (0, 2, 3):
        p = [FAKE] * 5
        p[n] = None
        assert call(pointers=p) == NULL
    assert call(loss=None) == NULL
    for shape in ((0, 2, 3, 4), (1, 0, 3, 4), (1, 2, 0, 4), (1, 2, 3, 0), (1, 2, 3, 1 << 17), (1 << 20, 8, 8, 4), (1 << 15, 2, 1 << 15, 4)):
        assert call(shape=shape) == SHAPE
        assert mas.mas_align_loss_workspace_bytes(*shape) == 0
    n = mas.mas_align_loss_workspace_bytes(2, 10, 500, 80)
    assert n > 0 and n % 256 == 0
    assert call((2, 10, 500, 80), ws=(None, 0)) == WORKSPACE
    assert call((2, 10, 500, 80), ws=(ctypes.c_void_p(0x10010), n)) == WORKSPACE
    assert call((2, 10, 500, 80), ws=(FAKE, 256)) == WORKSPACE


def test_binding_refuses_host_tensors():
    import torch

    x = torch.zeros(1, 2, 2, 8)
    with pytest.raises(TypeError):
        mas.mas_attention(x, x, x)
    with pytest.raises(TypeError):
        mas.mas_qk_norm_rope(x, x, None, None, None, None)
    m = torch.zeros(1, 2, 8)
    with pytest.raises(TypeError):
        mas.mas_align_loss(m, None, m, torch.zeros(1, 3, dtype=torch.int32))


def test_structures_match_the_header():
    """Sizes as the C compiler lays them out."""
    assert ctypes.sizeof(Heads) == 32
    assert ctypes.sizeof(AttentionDesc) == 11 * 4 + 4 + 5 * 8
    assert ctypes.sizeof(QkDesc) == 10 * 4 + 6 * 8
    assert set(_native._DTYPES.values()) == {0, 1, 2}
