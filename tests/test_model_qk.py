"""mas_qk_norm_rope and its backward pass on the GPU against 64 bits: types, head
sizes that are and are not whole pieces, partial turns of both kinds, positions,
padding, strides, in place, and sums of weights' gradients."""
from __future__ import annotations

import pytest
import torch

from ._attention import TINY, UNIT, check

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E = UNIT[F32]


@pytest.fixture(scope="module")
def mas():
    import paper_2409_07704_amd as m

    m.lib()
    return m


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(B, T, Hq, Hk, D, R, dtype, seed=0, P=64):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    qkv = r(B, T, Hq + 2 * Hk, D).to(dtype).cuda()
    angle = torch.arange(P, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(R // 2, dtype=torch.float64) / max(R // 2, 1))
    return dict(q=qkv[:, :, :Hq], k=qkv[:, :, Hq : Hq + Hk], wq=(1 + 0.3 * r(D)).cuda(), wk=(1 + 0.3 * r(D)).cuda(),
                cos=torch.cos(angle).float().cuda(), sin=torch.sin(angle).float().cuda(),
                gq=r(B, T, Hq, D).to(dtype).cuda(), gk=r(B, T, Hk, D).to(dtype).cuda())


def reference(x, w, dz, cos, sin, R, interleaved, pos, t_x, eps):
    """{name: (value, bound)} of y, dx and dw in 64 bits.  Bounds: fp32 sums of D
    terms, some ten fp32 operations an element, results rounded once; dw is an
    fp32 sum whose chains are at most 700 additions."""
    u, tiny = UNIT[x.dtype], TINY[x.dtype] + 1e-30
    x, dz, cos, sin = (a.cpu().double() for a in (x, dz, cos, sin))
    B, T, H, D = x.shape
    w = torch.ones(D, dtype=torch.float64) if w is None else w.cpu().double()
    at = torch.arange(T).expand(B, T) if pos is None else pos.cpu().long()
    at = at.clamp(0, cos.shape[0] - 1)
    keep = torch.ones((B, T), dtype=torch.bool) if t_x is None else torch.arange(T) < t_x.cpu().clamp(0, T)[:, None]
    keep = keep[:, :, None, None]
    a = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
    b = a + (1 if interleaved else R // 2)
    c, s = cos[at][:, :, None], sin[at][:, :, None]

    def turn(y, s):
        z, size = y.clone(), y.abs()
        z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        size = size.clone()
        size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
        return z, size

    clean = torch.where(keep, x, 0.0)
    r = (clean.square().mean(3, keepdim=True) + eps).rsqrt()
    h = torch.where(keep, clean * r, 0.0)
    y, size = turn(h * w, s)
    few = (D + 16) * E
    dy, dsize = turn(torch.where(keep, dz, 0.0), -s)
    g = dy * w
    mean, msize = (g * h).mean(3, keepdim=True), (dsize * w.abs() * h.abs()).mean(3, keepdim=True)
    dx = torch.where(keep, r * (g - h * mean), 0.0)
    dxsize = torch.where(keep, r * (dsize * w.abs() + h.abs() * msize), 0.0)
    prod, psize = dy * h, dsize * h.abs()
    return {"y": (y, u * y.abs() + few * size + tiny), "dx": (dx, u * dx.abs() + 3 * few * dxsize + tiny),
            "dw": (prod.sum((0, 1, 2)), (few + 700 * E) * psize.sum((0, 1, 2)) + 1e-30)}


def run_and_check(mas, st, R, label, interleaved=False, pos=None, t_x=None, eps=1e-6, weights=True):
    print(f"[gpu-case] {label} q{tuple(st['q'].shape)} k{tuple(st['k'].shape)} R={R} {st['q'].dtype} interleaved={interleaved}", flush=True)
    wq, wk = (st["wq"], st["wk"]) if weights else (None, None)
    rest = (wq, wk, st["cos"] if R else None, st["sin"] if R else None)
    args = dict(pos=pos, t_x=t_x, eps=eps, interleaved=interleaved)
    fill = lambda x: torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
    q, k = mas.mas_qk_norm_rope(st["q"], st["k"], *rest, q_out=fill(st["q"]), k_out=fill(st["k"]), **args)
    dq, dk, dwq, dwk = mas.mas_qk_norm_rope_backward(st["gq"], st["gk"], st["q"], st["k"], *rest, dq=fill(st["q"]), dk=fill(st["k"]), **args)
    for n, w, y, dx, dw in (("q", wq, q, dq, dwq), ("k", wk, k, dk, dwk)):
        want = reference(st[n], w, st["g" + n], st["cos"], st["sin"], R, interleaved, pos, t_x, eps)
        for name, got in (("y", y), ("dx", dx), ("dw", dw)):
            check(got, want[name], f"{label} {n} {name}")
    return q, k, dq, dk, dwq, dwk


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R", [(2, 2), (7, 6), (32, 32), (40, 40), (64, 32), (80, 40), (96, 48), (100, 20), (128, 128), (192, 0), (250, 50), (256, 256)])
def test_head_sizes_and_turns(mas, dtype, interleaved, D, R):
    run_and_check(mas, make(2, 9, 3, 2, D, R, dtype, D), R, "sizes", interleaved)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,Hq,Hk", [(1, 1, 1, 1), (64, 1, 16, 4), (3, 203, 2, 2), (2, 700, 8, 1)])
def test_batches(mas, dtype, B, T, Hq, Hk):
    lens = _ints([T, 0, 1, T + 5, -3, T // 2][:B] if B <= 6 else list(range(B)))
    st = make(B, T, Hq, Hk, 64, 64, dtype, T, P=1024)
    run_and_check(mas, st, 64, "padding", t_x=lens)
    run_and_check(mas, st, 64, "no weights", weights=False)


def test_many_rows(mas):
    """More tokens than groups of lanes: groups that walk over all heads of a token,
    and outputs large enough to be stored around the caches."""
    st = make(8, 4200, 9, 3, 64, 64, BF16, 1, P=4200)
    assert st["q"].shape[0] * 4200 > 32768 and 8 * 4200 * 12 * 64 * 2 < 64 << 20
    run_and_check(mas, st, 64, "many rows")
    st = make(12, 4200, 9, 3, 64, 64, BF16, 2, P=4200)
    assert 12 * 4200 * 12 * 64 * 2 > 64 << 20
    run_and_check(mas, st, 64, "large outputs", interleaved=True)


def test_positions(mas):
    """Positions per token; those outside the tables take the nearest row."""
    pos = torch.randint(-20, 90, (4, 33), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    for R, D in ((64, 64), (6, 7)):
        run_and_check(mas, make(4, 33, 4, 2, D, R, BF16, 4), R, "positions", pos=pos)


def test_queries_alone_and_eps_zero(mas):
    st = make(2, 17, 5, 1, 64, 64, F32, 5)
    q, k = mas.mas_qk_norm_rope(st["q"], None, st["wq"], None, st["cos"], st["sin"], eps=0.0)
    assert k is None
    check(q, reference(st["q"], st["wq"], st["gq"], st["cos"], st["sin"], 64, False, None, None, 0.0)["y"], "queries alone")
    dq, dk, dwq, dwk = mas.mas_qk_norm_rope_backward(st["gq"], None, st["q"], None, st["wq"], None, st["cos"], st["sin"], eps=0.0)
    assert dk is None and dwk is None
    check(dwq, reference(st["q"], st["wq"], st["gq"], st["cos"], st["sin"], 64, False, None, None, 0.0)["dw"], "queries alone dw")


@pytest.mark.parametrize("dtype", [F32, F16])
def test_strides_alignment_and_in_place(mas, dtype):
    B, T, H, D = 2, 21, 3, 64
    gen = torch.Generator().manual_seed(6)
    st = make(B, T, H, H, D, D, dtype, 7)
    wide = torch.randn((B, T, 2 * H, D + 3), generator=gen).to(dtype).cuda()
    off = dict(st, q=wide[:, :, :H, 1 : D + 1], k=wide[:, :, H:, 1 : D + 1])
    run_and_check(mas, off, D, "off boundaries")
    turned = dict(st, q=torch.randn((B, H, T, D), generator=gen).to(dtype).cuda().transpose(1, 2), k=wide[:, :, :1, :D].expand(B, T, H, D))
    run_and_check(mas, turned, D, "transposed, shared heads")
    for R, inter in ((D, False), (D, True), (20, False)):
        rest = (st["wq"], st["wk"], st["cos"][:, : R // 2].contiguous(), st["sin"][:, : R // 2].contiguous())
        q, k = st["q"].clone(), st["k"].clone()
        want = mas.mas_qk_norm_rope(q, k, *rest, interleaved=inter)
        back = mas.mas_qk_norm_rope_backward(st["gq"], st["gk"], q, k, *rest, interleaved=inter)
        gq, gk = st["gq"].clone(), st["gk"].clone()
        again = mas.mas_qk_norm_rope_backward(gq, gk, q, k, *rest, interleaved=inter, dq=gq, dk=gk)
        assert all(torch.equal(x, y) for x, y in zip(back, again))
        mas.mas_qk_norm_rope(q, k, *rest, interleaved=inter, q_out=q, k_out=k)
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_written_into_a_cache(mas):
    """New keys go to their place in a longer cache; the rest of it stays."""
    st = make(3, 2, 4, 2, 64, 64, BF16, 8)
    cache = torch.full((3, 50, 2, 64), 5.0, dtype=BF16, device="cuda")
    want = mas.mas_qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["cos"], st["sin"])
    mas.mas_qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["cos"], st["sin"], k_out=cache[:, 30:32])
    assert torch.equal(cache[:, 30:32], want[1])
    cache[:, 30:32] = 5.0
    assert bool((cache == 5.0).all())


@pytest.mark.parametrize("D", [64, 7])
def test_padding_may_hold_anything(mas, D):
    lens, R = _ints([3, 9]), D // 2 * 2
    st = make(2, 9, 4, 2, D, R, F16, 9)
    want = run_and_check(mas, st, R, "clean", t_x=lens)
    for bad in (float("nan"), float("inf")):
        st2 = {n: x.clone() for n, x in st.items()}
        for n in ("q", "k", "gq", "gk"):
            st2[n][0, 3:] = bad
        assert all(torch.equal(x, y) for x, y in zip(run_and_check(mas, st2, R, "dirty", t_x=lens), want))


def test_gradients_against_differences(mas):
    st = make(2, 5, 3, 2, 32, 16, F32, 10)
    rest = (st["cos"], st["sin"])
    grads = mas.mas_qk_norm_rope_backward(st["gq"], st["gk"], st["q"], st["k"], st["wq"], st["wk"], *rest)
    names, gen = ("q", "k", "wq", "wk"), torch.Generator().manual_seed(11)
    for n, dx in zip(names, grads):
        d, h, f = torch.randn(st[n].shape, generator=gen).cuda(), 2.0**-7, []
        for sign in (h, -h):
            at = dict(st, **{n: st[n] + sign * d})
            y = mas.mas_qk_norm_rope(at["q"], at["k"], at["wq"], at["wk"], *rest)
            f.append((y[0].double() * st["gq"].double()).sum() + (y[1].double() * st["gk"].double()).sum())
        # Third derivatives are a few times the first; fp32 errs by 2^-20 of the parts over 2 h.
        size = (dx.double() * d.double()).abs().sum()
        assert abs((f[0] - f[1]) / (2 * h) - (dx.double() * d.double()).sum()) <= (8 * h * h + 2.0**-19 / h) * size


def test_repeated_calls_streams_and_graph(mas):
    st = make(4, 300, 4, 2, 64, 64, BF16, 12, P=512)
    args = (st["wq"], st["wk"], st["cos"], st["sin"])
    ws = torch.empty(mas.mas_qk_norm_rope_workspace_bytes(st["q"], st["k"]), dtype=torch.uint8, device="cuda")
    q, k, gq, gk = (st[n].contiguous() for n in ("q", "k", "gq", "gk"))
    outs = [torch.empty_like(x) for x in (q, k, q, k)] + [torch.empty(64, device="cuda") for _ in range(2)]

    def step():
        mas.mas_qk_norm_rope(q, k, *args, q_out=outs[0], k_out=outs[1])
        mas.mas_qk_norm_rope_backward(gq, gk, q, k, *args, dq=outs[2], dk=outs[3], dwq=outs[4], dwk=outs[5], workspace=ws)

    step()
    first = [x.clone() for x in outs]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    alone = mas.mas_qk_norm_rope_backward(gq, gk, q, k, *args, stream=stream)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(alone, first[2:]))
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for scale in (1.0, 2.0, 0.5):
        gq.copy_(st["gq"] * scale)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, outs))


def test_the_binding_refuses(mas):
    st = make(2, 4, 2, 2, 32, 32, BF16, 13)
    rest = (st["wq"], st["wk"], st["cos"], st["sin"])
    for bad, error in (
        (lambda: mas.mas_qk_norm_rope(st["q"].cpu(), st["k"], *rest), TypeError),
        (lambda: mas.mas_qk_norm_rope(st["q"], st["k"].float(), *rest), TypeError),
        (lambda: mas.mas_qk_norm_rope(st["q"], st["k"], st["wq"].half(), *rest[1:]), TypeError),
        (lambda: mas.mas_qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["cos"], None), ValueError),
        (lambda: mas.mas_qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["cos"], st["sin"][:3].contiguous()), ValueError),
        (lambda: mas.mas_qk_norm_rope(st["q"], st["k"], *rest, pos=_ints([1, 2])), ValueError),
        (lambda: mas.mas_qk_norm_rope(st["q"], st["k"], *rest, eps=-1.0), mas.MasError),
        (lambda: mas.mas_qk_norm_rope(st["q"][..., :20], st["k"][..., :20], None, None, st["cos"], st["sin"]), mas.MasError),
        (lambda: mas.mas_qk_norm_rope_backward(st["gq"], st["gk"], st["q"], st["k"], *rest, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), mas.MasError),
    ):
        with pytest.raises(error):
            bad()
