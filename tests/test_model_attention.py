"""mas_attention and mas_attention_backward on the GPU against 64 bits, with
bounds that follow the operations; masks that leave rows empty, lengths of zero
and one, odd head sizes, strides and alignments, long caches, non-finite values
in hidden places, streams and graphs."""
from __future__ import annotations

import pytest
import torch

from ._attention import check, reference

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


@pytest.fixture(scope="module")
def mas():
    import paper_2409_07704_amd as m

    m.lib()
    return m


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _rand(gen, *shape, dtype):
    return torch.randn(shape, generator=gen, dtype=torch.float32).to(dtype).cuda()


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(B, Tq, Tk, Hq, Hk, D, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    return (_rand(gen, B, Tq, Hq, D, dtype=dtype), _rand(gen, B, Tk, Hk, D, dtype=dtype),
            _rand(gen, B, Tk, Hk, D, dtype=dtype), _rand(gen, B, Tq, Hq, D, dtype=dtype))


def run_and_check(mas, q, k, v, dout, label, **args):
    _say(f"{label} q{tuple(q.shape)} k{tuple(k.shape)} {q.dtype} " + " ".join(f"{n}={x.tolist() if isinstance(x, torch.Tensor) and x.numel() < 9 else '...' if isinstance(x, torch.Tensor) else x}" for n, x in args.items()))
    B, Tq, Hq, D = q.shape
    fill = lambda x: torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
    out, lse = fill(q), torch.full((B, Hq, Tq), 7.0, device="cuda")
    mas.mas_attention(q, k, v, out=out, lse_out=lse, **args)
    want = reference(q, k, v, dout, **args)
    check(out, want["out"], label + " out")
    check(lse, want["lse"], label + " lse")
    if dout is None:
        return out, lse
    dq, dk, dv = fill(q), fill(k), fill(v)
    mas.mas_attention_backward(dout, q, k, v, out, lse, dq=dq, dk=dk, dv=dv, **args)
    for name, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(x, want[name], f"{label} {name}")
    return out, lse, dq, dk, dv


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 2, 31, 33, 64, 129, 200])
def test_lengths_around_tiles(mas, dtype, T):
    run_and_check(mas, *make(2, T, T, 2, 2, 64, dtype, T), "plain")
    run_and_check(mas, *make(1, T, T, 2, 1, 32, dtype, T), "causal", causal=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [1, 7, 8, 24, 40, 80, 96, 100, 128])
def test_head_sizes(mas, dtype, D):
    """Whole and broken 16-byte rows, every padded width."""
    run_and_check(mas, *make(2, 70, 70, 4, 2, D, dtype, D), "head size", causal=True)


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (6, 2), (5, 1), (16, 2), (64, 1)])
def test_shared_heads(mas, Hq, Hk):
    """Groups of heads that are and are not powers of two, up to 64 to a key head."""
    run_and_check(mas, *make(2, 37, 37, Hq, Hk, 32, BF16, Hq), "groups", causal=True)
    run_and_check(mas, *make(1, 21, 53, Hq, Hk, 64, F32, Hq), "groups", slope=0.1 + torch.rand(Hq, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B", [20, 30])
def test_gradients_in_one_launch_and_in_two(mas, dtype, B):
    """Few items: 40 pairs of 3 blocks of rows and 3 of keys, 240 workgroups; and 60, 360."""
    lens = _ints([96, 0, 1, 33, 65] * (B // 5))
    run_and_check(mas, *make(B, 96, 96, 2, 2, 72, dtype, B), "launches", t_q=lens, t_k=lens, causal=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("big", [False, True])
def test_masks_and_biases(mas, dtype, big):
    """Documents, prefixes, caps and distances together, on a few items (waves take
    turns at the keys) and on many (shared tiles)."""
    B = 150 if big else 3
    q, k, v, g = make(B, 130, 130, 2, 1, 32, dtype, 3)
    lens = _ints([130, 0, 1] * (B // 3))
    docs = _ints([[0, 40, 41, 41, 130], [0, 0, 0, 0, 0], [0, 1, 1, 1, 1]] * (B // 3))
    prefix = _ints([[5, 1, 0, 200], [3, 0, 0, 0], [0, 0, 0, 0]] * (B // 3))
    slope = _ints([1, 2]).float() * 0.03
    run_and_check(mas, q, k, v, g, "docs", t_q=lens, t_k=lens, causal=True, doc_start=docs, prefix=prefix, slope=slope, cap=3.0)
    run_and_check(mas, q, k, v, g, "docs both ways", t_q=lens, t_k=lens, doc_start=docs, cap=20.0)
    run_and_check(mas, q, k, v, g, "prefix", t_q=lens, t_k=lens, causal=True, prefix=_ints([[17], [3], [200]] * (B // 3)))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_see_nothing(mas, dtype):
    """Places before the first document, between documents' table ends and past the
    last one; queries longer than the keys; lengths outside the extents."""
    q, k, v, g = make(4, 75, 75, 2, 2, 64, dtype, 5)
    docs = _ints([[10, 20, 50], [0, 0, 0], [75, 75, 75], [-5, 30, 200]])
    out, lse, dq, dk, dv = run_and_check(mas, q, k, v, g, "gaps", causal=True, doc_start=docs)
    assert bool((out[0, :10] == 0).all()) and bool((out[0, 50:] == 0).all()) and bool((out[1:3] == 0).all())
    assert bool((lse[1:3] == -float("inf")).all()) and bool((dq[1:3] == 0).all()) and bool((dk[1:3] == 0).all())
    run_and_check(mas, q, k, v, g, "queries before the first key", causal=True, t_q=_ints([75, 60, 3, -4]), t_k=_ints([30, 0, 99, 75]))
    run_and_check(mas, q, k, v, g, "other lengths", t_q=_ints([75, 60, 3, 500]), t_k=_ints([30, 0, 99, -1]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Tq,Tk,Hq,Hk,D", [(1, 1, 4, 2, 64), (1, 700, 16, 2, 128), (3, 2111, 8, 1, 64), (5, 4096, 3, 3, 80), (8, 300, 32, 4, 32)])
def test_steps_over_a_cache(mas, dtype, Tq, Tk, Hq, Hk, D):
    """A few queries at the end of caches of different lengths: keys split and joined."""
    B = 3
    q, k, v, _ = make(B, Tq, Tk, Hq, Hk, D, dtype, Tk)
    lens = _ints([Tk, max(Tk // 3, 1), Tq])
    run_and_check(mas, q, k, v, None, "step", t_k=lens, causal=True, slope=torch.full((Hq,), 0.01, device="cuda"))
    run_and_check(mas, q, k, v, None, "step", t_k=lens, cap=10.0)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_training_over_a_cache(mas, dtype):
    """Gradients where queries are the last of more keys."""
    q, k, v, g = make(2, 40, 333, 4, 2, 64, dtype, 9)
    run_and_check(mas, q, k, v, g, "tail", t_q=_ints([40, 7]), t_k=_ints([333, 101]), causal=True)


def test_scales(mas):
    q, k, v, g = make(1, 66, 66, 2, 2, 32, F32, 11)
    for scale in (0.0, -0.3, 2.0):
        run_and_check(mas, q, k, v, g, "scale", scale=scale)
    run_and_check(mas, q, k, v, g, "scale", scale=-0.3, cap=1.5, causal=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(mas, dtype):
    """Scores of hundreds: the running maximum moves by more than an exponent holds."""
    q, k, v, _ = make(1, 200, 200, 2, 2, 64, dtype, 12)
    ramp = torch.linspace(0.1, 40.0, 200, device="cuda")[None, :, None, None]
    k = (k.float() * ramp).to(dtype)
    run_and_check(mas, q, k, v, None, "ramp", scale=1.0, causal=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(mas, dtype):
    """Heads sliced from one projection, transposed layouts, keys shared by all
    items (stride 0), and rows that start off 16-byte boundaries."""
    gen = torch.Generator().manual_seed(13)
    B, T, Hq, Hk, D = 2, 90, 4, 2, 64
    qkv = _rand(gen, B, T, Hq + 2 * Hk, D, dtype=dtype)
    g = _rand(gen, B, Hq, T, D, dtype=dtype).transpose(1, 2)
    run_and_check(mas, qkv[:, :, :Hq], qkv[:, :, Hq : Hq + Hk], qkv[:, :, Hq + Hk :], g, "one projection", causal=True)
    k = _rand(gen, 1, T, Hk, D, dtype=dtype).expand(B, T, Hk, D)
    v = _rand(gen, Hk, T, 1, D, dtype=dtype).permute(2, 1, 0, 3).expand(B, T, Hk, D)
    run_and_check(mas, qkv[:, :, :Hq], k, v, g, "shared keys")
    off = _rand(gen, B, T, Hq, D + 3, dtype=dtype)[..., 1 : D + 1]
    run_and_check(mas, off, off[:, :, :Hk], off[:, :, Hk:], off, "off boundaries", causal=True)


def test_outputs_in_place_of_a_projection(mas):
    """Gradients written into the slices of one tensor; the rest stays."""
    q, k, v, g = make(2, 50, 50, 4, 2, 32, BF16, 14)
    lse = torch.empty((2, 4, 50), device="cuda")
    out = mas.mas_attention(q, k, v, causal=True, lse_out=lse)
    want = mas.mas_attention_backward(g, q, k, v, out, lse, causal=True)
    both = torch.full((2, 50, 9, 32), 5.0, dtype=BF16, device="cuda")
    mas.mas_attention_backward(g, q, k, v, out, lse, causal=True, dq=both[:, :, :4], dk=both[:, :, 4:6], dv=both[:, :, 6:8])
    for x, y in zip(want, (both[:, :, :4], both[:, :, 4:6], both[:, :, 6:8])):
        assert torch.equal(x, y)
    assert bool((both[:, :, 8] == 5.0).all())


@pytest.mark.parametrize("Tq", [1, 200])
def test_offsets_past_32_bits(mas, Tq):
    """A cache whose tokens lie 40000 elements apart: the last is 2^32 bytes on."""
    gen = torch.Generator().manual_seed(15)
    Tk, D, apart = 60000, 32, 40000
    store = torch.empty(Tk * apart, dtype=BF16, device="cuda")
    k = store.as_strided((1, Tk, 1, D), (0, apart, D, 1))
    v = store.as_strided((1, Tk, 1, D), (0, apart, D, 1), 64)
    k.copy_(torch.randn((1, Tk, 1, D), generator=gen))
    v.copy_(torch.randn((1, Tk, 1, D), generator=gen))
    q = _rand(gen, 1, Tq, 1, D, dtype=BF16)
    _say(f"long cache Tq={Tq}")
    assert (Tk - 1) * apart * 2 > 2**32
    out = mas.mas_attention(q, k, v, causal=True)
    assert torch.equal(out, mas.mas_attention(q, k.contiguous(), v.contiguous(), causal=True))


@pytest.mark.parametrize("dtype", TYPES)
def test_padding_may_hold_anything(mas, dtype):
    q, k, v, g = make(2, 100, 100, 2, 2, 64, dtype, 16)
    lens = _ints([100, 37])
    args = dict(t_q=lens, t_k=lens, causal=True)
    want = run_and_check(mas, q, k, v, g, "clean padding", **args)
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        q2, k2, v2, g2 = (x.clone() for x in (q, k, v, g))
        for x in (q2, k2, v2, g2):
            x[1, 37:] = bad
        got = run_and_check(mas, q2, k2, v2, g2, f"padding {bad}", **args)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,D", [(1, 130, 64), (150, 200, 40)])
def test_hidden_values_may_hold_anything(mas, dtype, B, T, D):
    """Non-finite keys and values that only later queries see leave earlier ones as
    they are; queries that see such a value get it in its channel."""
    q, k, v, _ = make(B, T, T, 4, 2, D, dtype, 17)
    t = T // 2 + 3
    _say(f"hidden {dtype} B={B} T={T} D={D}")
    want = reference(q[:1], k[:1], v[:1], causal=True)["out"]
    for bad in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        k2[:, t:] = bad
        v2[:, t:] = bad
        out = mas.mas_attention(q, k2, v2, causal=True)
        check(out[:1, :t], (want[0][:, :t], want[1][:, :t]), f"before {bad}")
        v2 = v.clone()
        v2[:, t, :, 3] = bad
        out = mas.mas_attention(q, k, v2, causal=True)
        hit = out[:, t:, :, 3]
        assert bool(hit.isnan().all()) if bad != bad else bool((hit == bad).all())
        out[:, t:, :, 3] = 0
        value, bound = want[0].clone(), want[1]
        value[:, t:, :, 3] = 0
        check(out[:1], (value, bound), f"around {bad}")


def test_malformed_documents_stay_inside_the_tensors(mas):
    """A table that is no table: results are unspecified, but nothing else changes."""
    B, T, H, D = 4, 100, 2, 32
    q, k, v, g = make(B, T, T, H, H, D, BF16, 18)
    docs = torch.randint(-300, 300, (B, 9), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    prefix = torch.randint(-300, 2**31 - 1, (B, 8), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    n = B * T * H * D
    _say("malformed documents")
    guards = [torch.full((n + 256,), 3.0, dtype=BF16, device="cuda") for _ in range(4)]
    out, dq, dk, dv = (x[128 : 128 + n].view(B, T, H, D) for x in guards)
    lse = torch.full((B * H * T + 64,), 3.0, device="cuda")
    mas.mas_attention(q, k, v, causal=True, doc_start=docs, prefix=prefix, out=out, lse_out=lse[32:-32].view(B, H, T))
    mas.mas_attention_backward(g, q, k, v, out, lse[32:-32].view(B, H, T), causal=True, doc_start=docs, prefix=prefix, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    for x in guards + [lse]:
        e = 128 if x.dtype == BF16 else 32
        assert bool((x[:e] == 3.0).all()) and bool((x[-e:] == 3.0).all())


def test_gradients_against_differences(mas):
    """Central differences of the kernel's own forward pass, in fp32."""
    q, k, v, g = make(2, 40, 40, 4, 2, 32, F32, 19)
    args = dict(causal=True, cap=4.0, slope=torch.full((4,), 0.05, device="cuda"), doc_start=_ints([[0, 25, 40]] * 2),
                prefix=_ints([[6, 3]] * 2))
    lse = torch.empty((2, 4, 40), device="cuda")
    out = mas.mas_attention(q, k, v, lse_out=lse, **args)
    grads = mas.mas_attention_backward(g, q, k, v, out, lse, **args)
    gen = torch.Generator().manual_seed(20)
    for n, (x, dx) in enumerate(zip((q, k, v), grads)):
        for _ in range(3):
            d, h = _rand(gen, *x.shape, dtype=F32), 2.0**-6
            f = []
            for sign in (h, -h):
                moved = [q, k, v]
                moved[n] = x + sign * d
                f.append((mas.mas_attention(*moved, **args).double() * g.double()).sum())
            # Differences err by h^2 times a third derivative (about the size of the sum
            # of the parts' absolute values) and by fp32 over 2 h.
            size = (dx.double() * d.double()).abs().sum()
            assert abs((f[0] - f[1]) / (2 * h) - (dx.double() * d.double()).sum()) <= (h * h + 2.0**-18 / h) * size


@pytest.mark.parametrize("Tq,Tk", [(300, 300), (1, 3000)])
def test_repeated_calls_other_streams_and_workspaces(mas, Tq, Tk):
    """Identical bits from repeated calls, on a stream of their own, with the
    caller's workspace or the call's."""
    q, k, v, g = make(2, Tq, Tk, 4, 2, 64, BF16, 21)
    lse = torch.empty((2, 4, Tq), device="cuda")
    ws = torch.empty(mas.mas_attention_workspace_bytes(q, k, backward=True), dtype=torch.uint8, device="cuda")
    out = mas.mas_attention(q, k, v, causal=True, lse_out=lse, workspace=ws)
    grads = mas.mas_attention_backward(g, q, k, v, out, lse, causal=True, workspace=ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    lse2 = torch.empty_like(lse)
    for how in (stream, stream.cuda_stream):
        out2 = mas.mas_attention(q, k, v, causal=True, lse_out=lse2, stream=how)
        again = mas.mas_attention_backward(g, q, k, v, out2, lse2, causal=True, stream=how)
        torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(grads, again))


def test_rows_do_not_depend_on_their_company(mas):
    """A query's bits are the same whatever other queries and items there are."""
    q, k, v, _ = make(2, 256, 256, 2, 2, 64, BF16, 22)
    out = mas.mas_attention(q, k, v)
    q2 = q.clone()
    q2[:, 100:] *= 30.0
    q2[1] = 0
    assert torch.equal(mas.mas_attention(q2, k, v)[0, :100], out[0, :100])


def test_captured_in_a_graph(mas):
    q, k, v, g = make(2, 200, 200, 4, 2, 64, F16, 23)
    lse = torch.empty((2, 4, 200), device="cuda")
    bufs = [torch.empty_like(x) for x in (q, q, k, v)]
    ws = torch.empty(mas.mas_attention_workspace_bytes(q, k, backward=True), dtype=torch.uint8, device="cuda")

    def step():
        mas.mas_attention(q, k, v, causal=True, out=bufs[0], lse_out=lse, workspace=ws)
        mas.mas_attention_backward(g, q, k, v, bufs[0], lse, causal=True, dq=bufs[1], dk=bufs[2], dv=bufs[3], workspace=ws)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for seed in range(3):
        for x, y in zip((q, k, v, g), make(2, 200, 200, 4, 2, 64, F16, 30 + seed)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in bufs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, bufs))


def test_the_binding_refuses(mas):
    q, k, v, g = make(2, 8, 8, 4, 2, 32, BF16, 24)
    lse = torch.empty((2, 4, 8), device="cuda")
    for bad, error in (
        (lambda: mas.mas_attention(q.cpu(), k, v), TypeError),
        (lambda: mas.mas_attention(q, k.half(), v), TypeError),
        (lambda: mas.mas_attention(q.double(), k.double(), v.double()), TypeError),
        (lambda: mas.mas_attention(q, k, v[:, :7]), ValueError),
        (lambda: mas.mas_attention(q[0], k, v), ValueError),
        (lambda: mas.mas_attention(q.transpose(2, 3), k, v), ValueError),
        (lambda: mas.mas_attention(q, k, v, t_k=_ints([8])), ValueError),
        (lambda: mas.mas_attention(q, k, v, t_k=torch.ones(2, device="cuda")), TypeError),
        (lambda: mas.mas_attention(q, k, v, doc_start=_ints([0, 8])), ValueError),
        (lambda: mas.mas_attention(q, k, v, lse_out=lse[:, :, :7]), ValueError),
        (lambda: mas.mas_attention(q[:, :, :3], k, v), mas.MasError),  # 3 heads over 2
        (lambda: mas.mas_attention(q, k, v, cap=-1.0), mas.MasError),
        (lambda: mas.mas_attention(q, k, v, scale=float("nan")), mas.MasError),
        (lambda: mas.mas_attention(q, k, v, prefix=_ints([[1], [1]])), mas.MasError),  # without causal
        (lambda: mas.mas_attention_backward(g, q, k, v, q, None), TypeError),
        (lambda: mas.mas_attention_backward(g, q, k, v, q, lse, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")), mas.MasError),
    ):
        with pytest.raises(error):
            bad()
