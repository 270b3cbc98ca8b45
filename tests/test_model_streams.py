"""Memory that a call brings along (a workspace, an output) belongs to the stream that
the call runs on: freed while the stream still works, it may only go to later work of
that stream."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mas():
    import paper_2409_07704_amd as m

    m.lib()
    return m


@pytest.mark.parametrize("raw", [False, True])
def test_allocations_belong_to_the_calls_stream(mas, monkeypatch, raw):
    print(f"[gpu-case] streams raw={raw}", flush=True)
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=gen).cuda()
    B, T, S, D = 3, 20, 50, 8
    mu, z, value = r(B, T, D), r(B, S, D), r(B, T, S)
    tx, ty = (torch.full((B,), n, dtype=torch.int32, device="cuda") for n in (T, S))
    rs = mas.mas_search(value, tx, ty)
    path = mas.mas_forward_ex(value, tx, ty)
    want = {"search": rs, "forward_ex": path, "sentinel": mas.mas_forward_sentinel(value, tx, ty, -1e9), "static": mas.mas_forward_static(value, tx, ty),
            "forward": mas.mas_forward(value, tx, ty), "expand_path": mas.mas_expand_path(rs, S), "expand_text": mas.mas_expand_text(mu, rs, S),
            "loglik": mas.mas_loglik(mu, None, z, tx, ty)}
    qkv = r(1, 40, 2, 32)
    want["attention"] = mas.mas_attention(qkv, qkv, qkv)
    stream = torch.cuda.Stream()
    how = stream.cuda_stream if raw else stream
    torch.cuda.synchronize()
    seen, empty = [], torch.empty

    def spy(*args, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", spy)
    got = {"search": mas.mas_search(value, tx, ty, stream=how), "forward_ex": mas.mas_forward_ex(value, tx, ty, stream=how),
           "sentinel": mas.mas_forward_sentinel(value, tx, ty, -1e9, stream=how), "static": mas.mas_forward_static(value, tx, ty, stream=how),
           "forward": mas.mas_forward(value, tx, ty, stream=how), "expand_path": mas.mas_expand_path(rs, S, stream=how),
           "expand_text": mas.mas_expand_text(mu, rs, S, stream=how), "loglik": mas.mas_loglik(mu, None, z, tx, ty, stream=how),
           "attention": mas.mas_attention(qkv, qkv, qkv, stream=how)}
    mas.Workspace(B, T, S, stream=how)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert len(seen) >= 12 and set(seen) == {stream.cuda_stream}
    assert torch.cuda.current_stream() != stream
    for n, x in got.items():
        if n != "loglik":  # (cells outside the band are left as they were)
            assert torch.equal(x, want[n]), n
