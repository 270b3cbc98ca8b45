"""The kernels that large batches take (tiles that a workgroup shares, workgroups of
eight waves, pairs of waves for dk and dv) against 64 bits, forward and backward: every
width, groups of heads that divide a tile and others, ragged lengths, documents,
prefixes, caps and distances.

Ten different items are repeated until the workgroups are as many as those kernels
want (256 of 128 rows, of 256 rows with eight waves, of 64 keys).  The ten are compared
with 64 bits, the others with them, bit for bit."""
from __future__ import annotations

import pytest
import torch

from ._attention import check, reference
from .test_model_attention import BF16, F16, F32, _ints, make, mas  # noqa: F401

pytestmark = pytest.mark.gpu

ITEMS = 10


def compare(mas, copies, q, k, v, g, label, **args):
    print(f"[gpu-case] large {label} {copies} x q{tuple(q.shape)} k{tuple(k.shape)} {q.dtype} {sorted(n for n in args)}", flush=True)
    many = lambda x: x.repeat(copies, *[1] * (x.dim() - 1))
    per_item = ("t_q", "t_k", "doc_start", "prefix")
    wide = {n: many(x) if n in per_item else x for n, x in args.items()}
    Q, K, V, G = (many(x) for x in (q, k, v, g))
    fill = lambda x: torch.full_like(x, 7.0)
    lse = torch.full((Q.shape[0], Q.shape[2], Q.shape[1]), 7.0, device="cuda")
    out, dq, dk, dv = fill(Q), fill(Q), fill(K), fill(V)
    mas.mas_attention(Q, K, V, out=out, lse_out=lse, **wide)
    mas.mas_attention_backward(G, Q, K, V, out, lse, dq=dq, dk=dk, dv=dv, **wide)
    want = reference(q, k, v, g, **args)
    for name, x in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(x[:ITEMS], want[name], f"{label} {name}")
        assert torch.equal(x, many(x[:ITEMS])), f"{label} {name}: copies of an item differ"


def lengths(T):
    return _ints([T, 0, 1, T - 1, T // 2, 33, 64, T, 2, T - 7])


def documents(T):
    """Starts of three documents an item, some empty, some leaving places out."""
    return _ints([[0, T // 3, T // 3, T], [0, 0, 0, 0], [0, 1, 1, 1], [0, 65, 70, T - 1], [5, 20, T // 2, T // 2],
                  [0, 10, 20, 33], [0, 1, 63, 64], [0, 0, T, T], [0, 1, 2, 2], [0, T // 2, T - 9, T - 9]])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D", [32, 40, 64, 72, 96, 100, 128])
@pytest.mark.parametrize("T,Hq,Hk,copies", [
    (200, 1, 1, 13),  # 130 pairs: 260 workgroups of 128 rows, 130 of 256
    (300, 1, 1, 13),  # 390, and 260 of 256 rows; five tiles of keys and of rows
    (70, 6, 2, 13),   # groups of three: 260 pairs of 210 rows
    (45, 8, 1, 26),   # groups of eight: 260 pairs of 360 rows
])
def test_sizes_and_groups(mas, dtype, D, T, Hq, Hk, copies):
    q, k, v, g = make(ITEMS, T, T, Hq, Hk, D, dtype, T + D)
    lens = lengths(T)
    compare(mas, copies, q, k, v, g, "ragged", t_q=lens, t_k=lens, causal=True)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_masks_and_biases(mas, dtype, D):
    T = 150
    q, k, v, g = make(ITEMS, T, T, 2, 1, D, dtype, D)
    lens, docs = lengths(T), documents(T)
    prefix = _ints([[5, 1, 200], [3, 0, 0], [0, 0, 0], [64, 2, 7], [1, 1, 1], [0, 9, 0], [1, 40, 1], [0, 0, 70], [1, 1, 0], [75, 3, 1]])
    slope = torch.tensor([0.03, 0.5], device="cuda")
    compare(mas, 26, q, k, v, g, "documents", t_q=lens, t_k=lens, causal=True, doc_start=docs, prefix=prefix, slope=slope, cap=5.0)
    compare(mas, 26, q, k, v, g, "documents both ways", t_q=lens, t_k=lens, doc_start=docs, cap=30.0)
    compare(mas, 26, q, k, v, g, "prefix", t_q=lens, t_k=lens, causal=True, prefix=_ints([[7 * n] for n in range(ITEMS)]))
    compare(mas, 26, q, k, v, g, "distances", slope=slope)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,Tq,Tk", [(64, 70, 200), (128, 90, 260), (128, 200, 60), (40, 260, 1)])
def test_queries_and_keys_of_different_lengths(mas, dtype, D, Tq, Tk):
    """Queries that are the last of more keys, and more queries than keys."""
    q, k, v, g = make(ITEMS, Tq, Tk, 4, 2, D, dtype, Tq)
    t_q = _ints([Tq, 0, 1, Tq, Tq // 2, 33, 64, 7, 2, Tq - 7])
    t_k = _ints([Tk, Tk, 0, Tk // 2, Tk, 1, Tk, 7, Tk, Tk])
    compare(mas, 26, q, k, v, g, "causal", t_q=t_q, t_k=t_k, causal=True, slope=torch.full((4,), 0.02, device="cuda"))
    compare(mas, 26, q, k, v, g, "all", t_q=t_q, t_k=t_k, cap=20.0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_padding_may_hold_anything(mas, dtype, D):
    T = 300
    q, k, v, g = make(ITEMS, T, T, 1, 1, D, dtype, 5)
    lens = lengths(T)
    run = lambda *x: compare(mas, 13, *x, "padding", t_q=lens, t_k=lens, causal=True)
    for bad in (float("nan"), float("inf")):
        dirty = [x.clone() for x in (q, k, v, g)]
        for x in dirty:
            for b, n in enumerate(lens.tolist()):
                x[b, n:] = bad
        run(*dirty)
