"""mas_align_loss on the GPU against 64 bits: alignments with long and short
rows, rows cut by every boundary of the work, items without an alignment, odd
channel counts and alignments, weights, and each output alone."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import synth

from ._attention import check

pytestmark = pytest.mark.gpu

E = 2.0**-24


@pytest.fixture(scope="module")
def mas():
    import paper_2409_07704_amd as m

    m.lib()
    return m


def make(rows, S, D, seed=0, sigma=True):
    """rows: per item the number of frames of each text row."""
    gen = torch.Generator().manual_seed(seed)
    B, T = len(rows), len(rows[0])
    table = torch.zeros((B, T + 1), dtype=torch.int32)
    table[:, 1:] = torch.tensor(rows, dtype=torch.int32).cumsum(1)
    r = lambda *s: torch.randn(s, generator=gen).cuda()
    return dict(mu=r(B, T, D), log_sigma=0.3 * r(B, T, D) if sigma else None, z=r(B, S, D) * 1.5, row_start=table.cuda(),
                item_weight=0.1 + torch.rand(B, generator=gen).cuda())


def reference(mu, log_sigma, z, row_start, item_weight):
    """{name: (value, bound)}; fp32 operations, and sums whose chains of additions
    are at most the frames of a row, or 400 for the loss."""
    mu, z, table = mu.cpu().double(), z.cpu().double(), row_start.cpu().tolist()
    B, T, D = mu.shape
    ls = torch.zeros_like(mu) if log_sigma is None else log_sigma.cpu().double()
    weight = torch.ones(B, dtype=torch.float64) if item_weight is None else item_weight.cpu().double()
    out = {n: (torch.zeros(s, dtype=torch.float64), torch.full(s, 1e-30, dtype=torch.float64))
           for n, s in (("loss", (B,)), ("dmu", mu.shape), ("dlog_sigma", mu.shape), ("dz", z.shape))}
    few = 16 * E
    for b in range(B):
        for i in range(T):
            lo, hi = table[b][i], table[b][i + 1]
            if hi <= lo:
                continue
            r, w = z[b, lo:hi] - mu[b, i], torch.exp(-2 * ls[b, i])
            # The subtraction's rounding is relative to its operands.
            size = (r.abs() + z[b, lo:hi].abs() + mu[b, i].abs()) * w
            n = few + (hi - lo) * E
            out["loss"][0][b] += (0.5 * math.log(2 * math.pi) + ls[b, i] + 0.5 * r * r * w).sum()
            out["loss"][1][b] += (few + 400 * E) * (1 + ls[b, i].abs() + r.abs() * size).sum()
            out["dz"][0][b, lo:hi] = weight[b] * r * w
            out["dz"][1][b, lo:hi] += weight[b] * few * size
            out["dmu"][0][b, i] = -weight[b] * (r * w).sum(0)
            out["dmu"][1][b, i] += weight[b] * n * size.sum(0)
            out["dlog_sigma"][0][b, i] = weight[b] * (1 - r * r * w).sum(0)
            out["dlog_sigma"][1][b, i] += weight[b] * 2 * n * (1 + r.abs() * size).sum(0)
    return out


def run_and_check(mas, st, label):
    B, T, D = st["mu"].shape
    S = st["z"].shape[1]
    print(f"[gpu-case] {label} B={B} T={T} S={S} D={D}", flush=True)
    fill = lambda *s: torch.full(s, 7.0, device="cuda")
    got = mas.mas_align_loss(st["mu"], st["log_sigma"], st["z"], st["row_start"], item_weight=st["item_weight"],
                             loss_out=fill(B), dmu=fill(B, T, D), dlog_sigma=fill(B, T, D), dz=fill(B, S, D))
    want = reference(**st)
    for name, x in zip(("loss", "dmu", "dlog_sigma", "dz"), got):
        check(x, want[name], f"{label} {name}")
    return got


@pytest.mark.parametrize("D", [1, 3, 4, 60, 80, 128, 130, 192, 256, 260, 300])
@pytest.mark.parametrize("sigma", [False, True])
def test_channels(mas, D, sigma):
    run_and_check(mas, make([[1, 5, 0, 30, 2, 0], [3, 3, 3, 3, 3, 3], [0] * 6], 45, D, D, sigma), "channels")


@pytest.mark.parametrize("D", [5, 80, 192])
def test_shapes_of_alignments(mas, D):
    """One row with every frame, one frame a row, long rows in the middle: rows cut
    by runs, by chunks and by neither."""
    S = 1111
    one, each, middle = [S] + [0] * 400, [1] * 401, [1] * 200 + [700] + [1] * 200
    steps = [0] * 401
    for i in range(0, 401, 13):
        steps[i] = i % 70
    run_and_check(mas, make([one, each, middle, steps, [0] * 400 + [S]], S, D, 1), "alignments")


def test_lengths_of_one(mas):
    run_and_check(mas, make([[1]], 1, 80, 2), "one frame")
    run_and_check(mas, make([[0]], 1, 80, 3), "no frame")
    run_and_check(mas, make([[0, 1], [1, 1]], 3, 7, 4), "few frames")


@pytest.mark.parametrize("B,T,S,D", [(16, 128, 512, 80), (32, 300, 2050, 192)])
def test_batches(mas, B, T, S, D):
    """Batches that fill the chip (long runs of frames) and small ones (short runs)."""
    gen = np.random.default_rng(5)
    rows = []
    for b in range(B):
        t, s = int(gen.integers(1, T + 1)), int(gen.integers(T, S + 1))
        n = np.bincount(gen.integers(0, t, s), minlength=T)
        rows.append(n.tolist())
    run_and_check(mas, make(rows, S, D, 6), "batch")


def test_alignments_of_the_search(mas):
    """With the tables that mas_search writes, invalid items among them, the loss is
    the alignment's score of mas_loglik's values with the sign turned."""
    mu, ls, z, tx, ty = synth.gauss_inputs("tts-b16-t128-s512", log_sigma_scale=0.2)
    tx, ty = tx.copy(), ty.copy()
    tx[0], ty[1], tx[2], ty[2] = 0, 0, 100, 50
    mu, ls, z, x, y = (torch.from_numpy(a).cuda() for a in (mu, ls, z, tx, ty))
    B, T, D = mu.shape
    value = mas.mas_loglik(mu, ls, z, x, y, value_out=torch.zeros((B, T, z.shape[1]), device="cuda"))
    score = torch.empty(B, device="cuda")
    table = mas.mas_search(value, x, y, score_out=score)
    st = dict(mu=mu, log_sigma=ls, z=z, row_start=table, item_weight=None)
    loss = run_and_check(mas, st, "search")[0]
    assert bool((loss[:3] == 0).all())
    # Both are fp32: the producer's cells and a score of up to 512 additions.
    assert bool(((loss + score)[3:].abs() <= 1e-5 * score[3:].abs() + 512 * 64 * E * 80).all())


def test_unaligned_pointers(mas):
    st = make([[3, 4, 0, 40]], 50, 80, 7)
    for n in ("mu", "log_sigma", "z"):
        flat = torch.empty(st[n].numel() + 1, device="cuda")
        flat[1:] = st[n].reshape(-1)
        st[n] = flat[1:].view(st[n].shape)
        assert st[n].data_ptr() % 16 != 0
    run_and_check(mas, st, "unaligned")


def test_each_output_alone(mas):
    st = make([[3, 0, 40, 90], [1, 1, 1, 1]], 140, 80, 8)
    args = (st["mu"], st["log_sigma"], st["z"], st["row_start"])
    all_ = mas.mas_align_loss(*args)
    assert torch.equal(mas.mas_align_loss(*args, gradients=False)[0], all_[0])
    for n, name in enumerate(("dmu", "dlog_sigma", "dz"), 1):
        buf = torch.full_like(all_[n], 7.0)
        got = mas.mas_align_loss(*args, gradients=False, **{name: buf})
        assert torch.equal(buf, all_[n]) and torch.equal(got[0], all_[0])
        assert [x is None for x in got[1:]] == [i != n for i in (1, 2, 3)]


def test_padding_may_hold_anything(mas):
    st = make([[3, 4, 0, 0], [0, 0, 0, 0]], 20, 80, 9)
    want = run_and_check(mas, st, "clean")
    for bad in (float("nan"), float("inf")):
        st2 = {n: x.clone() for n, x in st.items()}
        st2["z"][0, 7:] = st2["z"][1] = st2["mu"][0, 2:] = st2["mu"][1] = st2["log_sigma"][0, 2:] = bad
        got = mas.mas_align_loss(st2["mu"], st2["log_sigma"], st2["z"], st2["row_start"], item_weight=st2["item_weight"])
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_malformed_table_stays_inside_the_tensors(mas):
    B, T, S, D = 3, 40, 300, 16
    st = make([[1] * T] * B, S, D, 10)
    st["row_start"] = torch.randint(-50, S + 50, (B, T + 1), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    print("[gpu-case] malformed row_start", flush=True)
    guards = [torch.full((n + 128,), 3.0, device="cuda") for n in (B, B * T * D, B * T * D, B * S * D)]
    loss, dmu, dls, dz = (g[64:-64] for g in guards)
    mas.mas_align_loss(st["mu"], st["log_sigma"], st["z"], st["row_start"], loss_out=loss, dmu=dmu.view(B, T, D),
                       dlog_sigma=dls.view(B, T, D), dz=dz.view(B, S, D))
    torch.cuda.synchronize()
    for g in guards:
        assert bool((g[:64] == 3.0).all()) and bool((g[-64:] == 3.0).all())


def test_gradients_against_differences(mas):
    st = make([[2, 5, 0, 9], [1, 1, 8, 0]], 18, 12, 11)
    args = ("mu", "log_sigma", "z")
    grads = dict(zip(("mu", "log_sigma", "z"), mas.mas_align_loss(**st)[1:]))
    gen = torch.Generator().manual_seed(12)
    for n in args:
        d, h, f = torch.randn(st[n].shape, generator=gen).cuda(), 2.0**-6, []
        for sign in (h, -h):
            loss = mas.mas_align_loss(**dict(st, **{n: st[n] + sign * d}), gradients=False)[0]
            f.append((loss.double() * st["item_weight"].double()).sum())
        # The loss is a square in mu and z and an exponential in log_sigma, whose third
        # derivative is 4 times the first; fp32 errs by 2^-18 of the loss over 2 h.
        size = (grads[n].double() * d.double()).abs().sum()
        off = abs((f[0] - f[1]) / (2 * h) - (grads[n].double() * d.double()).sum())
        assert off <= 4 * 4 * h * h * size * float(d.abs().max()) ** 2 + 2.0**-18 * abs(f[0]) / h


def test_repeated_calls_streams_and_graph(mas):
    gen = np.random.default_rng(13)
    rows = [np.bincount(gen.integers(0, 100, 500), minlength=100).tolist() for _ in range(4)]
    st = make(rows, 520, 80, 14)
    B, T, S, D = 4, 100, 520, 80
    ws = torch.empty(mas.mas_align_loss_workspace_bytes(B, T, S, D), dtype=torch.uint8, device="cuda")
    bufs = dict(loss_out=torch.empty(B, device="cuda"), dmu=torch.empty(B, T, D, device="cuda"),
                dlog_sigma=torch.empty(B, T, D, device="cuda"), dz=torch.empty(B, S, D, device="cuda"), workspace=ws)
    step = lambda: mas.mas_align_loss(**st, **bufs)
    first = [x.clone() for x in step()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    alone = mas.mas_align_loss(**st, stream=stream)
    stream.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(alone, first))
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for scale in (1.0, 2.0, 0.5):
        st["z"].mul_(scale)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (bufs["loss_out"], bufs["dmu"], bufs["dlog_sigma"], bufs["dz"])]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_the_binding_refuses(mas):
    st = make([[3, 4]], 8, 16, 15)
    args = (st["mu"], st["log_sigma"], st["z"], st["row_start"])
    for bad, error in (
        (lambda: mas.mas_align_loss(args[0].cpu(), *args[1:]), TypeError),
        (lambda: mas.mas_align_loss(args[0].half(), *args[1:]), TypeError),
        (lambda: mas.mas_align_loss(args[0], args[1][:, :1], *args[2:]), ValueError),
        (lambda: mas.mas_align_loss(*args[:2], args[2][..., :8], args[3]), ValueError),
        (lambda: mas.mas_align_loss(*args[:3], args[3].long()), TypeError),
        (lambda: mas.mas_align_loss(*args[:3], None), TypeError),
        (lambda: mas.mas_align_loss(*args, item_weight=torch.ones(2, device="cuda")), ValueError),
        (lambda: mas.mas_align_loss(args[0][0], *args[1:]), ValueError),
        (lambda: mas.mas_align_loss(*args, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), mas.MasError),
    ):
        with pytest.raises(error):
            bad()
