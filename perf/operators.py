"""The operators around the alignment that a text encoder and its training step
need, as cases to time: attention over text tokens and speech frames, the norm
and rotation of its queries and keys, and the aligned loss with its gradients.

Sizes are the repository's synthetic batches (items of up to 128 ... 1024 text
rows, 512 ... 4096 frames, 80 or 192 channels: 2 heads of 96, 3 of 64) and
generic head layouts.  Lengths are ragged, evenly spread from half the padded
length up to it in an order that the seed decides, unless a case says "full".

`run` computes the plain form in 32 bits, or, where `own` is true, calls the
library.
"""
import math

import torch

own = False

DEVICE = "cuda"
LOG_2PI = math.log(2.0 * math.pi)
EPS = 1e-6
DOC_WEIGHTS = (3, 1, 4, 1, 5, 9, 2, 6)


def listed():
    return [
        # Serving, one item: the newest frame looks back over its own frames.  Latency counts.
        _attend("step b1 k2048", B=1, Tq=1, Tk=2048, Hq=16, Hk=2, D=128, dtype="bfloat16"),
        # Serving, a full batch of streams with caches of different lengths, scores capped.
        _attend("step b64 k4096", B=64, Tq=1, Tk=4096, Hq=16, Hk=4, D=64, dtype="float16", cap=30.0, lengths="ragged"),
        # Text encoder at inference: every token sees its whole sentence, nearer ones more.
        _attend("text b32 t512", B=32, Tq=512, Tk=512, Hq=2, Hk=2, D=96, dtype="float16", slope=True, lengths="ragged"),
        # Frames at inference, the longest items of the benchmark batch, shared heads: the largest forward pass.
        _attend("frames b8 t4096", B=8, Tq=4096, Tk=4096, Hq=16, Hk=4, D=128, dtype="bfloat16", causal=True),
        # A small training batch in fp32, as the alignment itself runs.
        _attend("train b16 t128 fp32", train=True, B=16, Tq=128, Tk=128, Hq=2, Hk=2, D=96, dtype="float32", lengths="ragged"),
        # The benchmark batch's text in training, several sentences packed into an item, each with a prompt that all of it sees.
        _attend("train docs b64 t1001", train=True, B=64, Tq=1001, Tk=1001, Hq=3, Hk=3, D=64, dtype="bfloat16",
                causal=True, docs=5, prefix=True, lengths="ragged"),
        # Frames in training: long items, shared heads, capped scores and a distance bias.
        _attend("train frames b4 t4096", train=True, B=4, Tq=4096, Tk=4096, Hq=8, Hk=2, D=128, dtype="bfloat16",
                causal=True, slope=True, cap=50.0),
        # The newest frame of every stream, on its way into the cache.
        _qk("qk step b64", B=64, T=1, Hq=16, Hk=4, D=64, R=64, dtype="float16"),
        # Odd sizes: fp32, a part of the channels turned, pairs side by side.
        _qk("qk train b16 t203 fp32", train=True, B=16, T=203, Hq=2, Hk=2, D=96, R=48, dtype="float32", interleaved=True, lengths="ragged"),
        # Frames in training.
        _qk("qk train b8 t4096", train=True, B=8, T=4096, Hq=16, Hk=4, D=128, R=128, dtype="bfloat16"),
        # The loss of a small batch of mel frames under unit-variance Gaussians.
        _loss("loss b16 t128 s512", B=16, T=128, S=512, D=80, sigma=False, lengths="ragged"),
        # The loss of the benchmark batch, latent frames under Gaussians with their own log-sigmas.
        _loss("loss b64 t1024 s4096", B=64, T=1024, S=4096, D=192, sigma=True, lengths="ragged"),
    ]


def _attend(name=None, train=False, causal=False, cap=0.0, slope=False, docs=0, prefix=False, lengths="full", **sizes):
    case = dict(do="attend", train=train, causal=causal, cap=cap, slope=slope, docs=docs, prefix=prefix,
                lengths=lengths, **sizes)
    return dict(case, name=name) if name else case


def _qk(name=None, train=False, interleaved=False, lengths="full", **sizes):
    case = dict(do="qk", train=train, interleaved=interleaved, lengths=lengths, **sizes)
    return dict(case, name=name) if name else case


def _loss(name=None, lengths="full", **sizes):
    case = dict(do="loss", lengths=lengths, **sizes)
    return dict(case, name=name) if name else case


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    do = rng.choice(["step", "attend", "train", "train", "qk", "qk_train", "loss"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    lengths = rng.choice(["ragged", "ragged", "full"])
    Hk = rng.choice([1, 2, 2, 3, 4])
    Hq = Hk * rng.choice([1, 1, 2, 4, 8])
    D = rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
    if do in ("attend", "train", "step"):
        extra = dict(Hq=Hq, Hk=Hk, D=D, dtype=dtype, lengths=lengths, cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                     slope=rng.random() < 0.4)
        while True:
            B = log_int(1, 64)
            if do == "step":
                Tk = log_int(16, 8192)
                Tq = min(rng.choice([1, 1, 1, 2, 5, 8]), Tk // 2)
                if B * Tk * Hk * D <= 64 * 4096 * 4 * 64:
                    return _attend(B=B, Tq=Tq, Tk=Tk, causal=True, **extra)
                continue
            T = log_int(16, 4096)
            # fp32 products run at a sixteenth of the 16-bit rate.
            limit = 4 * 4096 * 4096 * 8 * 128 * (1 if do == "train" else 2) / 2
            if B * T * T * Hq * D * (8 if dtype == "float32" else 1) <= limit:
                break
        docs = rng.choice([0, 0, rng.randint(2, 8)])
        causal = rng.random() < 0.6
        return _attend(train=do == "train", B=B, Tq=T, Tk=T, causal=causal, docs=min(docs, T // 4),
                       prefix=causal and rng.random() < 0.4, **extra)
    if do in ("qk", "qk_train"):
        while True:
            B, T = log_int(1, 64), log_int(1, 4096)
            if B * T * (Hq + Hk) * D <= 8 * 4096 * 20 * 128 // (2 if dtype == "float32" else 1):
                break
        return _qk(train=do == "qk_train", B=B, T=T, Hq=Hq, Hk=Hk, D=D, R=rng.choice([D, D, D // 2]), dtype=dtype,
                   interleaved=rng.random() < 0.3, lengths=lengths)
    while True:
        B, T = log_int(1, 64), log_int(8, 2048)
        S = min(8192, int(T * rng.uniform(1.5, 6.0)))
        D = rng.choice([80, 80, 100, 192, rng.randint(1, 192)])
        if B * S * D <= 64 * 4096 * 192:
            return _loss(B=B, T=T, S=S, D=D, sigma=rng.random() < 0.6, lengths=lengths)


# ---------------------------------------------------------------- inputs
def _lens(case, n):
    """The items' lengths, without their order."""
    B = case["B"]
    if case["lengths"] == "full":
        return [n] * B
    return [max(1, n // 2 + (n - n // 2) * (i + 1) // B) for i in range(B)]


def _doc_starts(t, docs, turn):
    """Starts of an item's documents, and its length last."""
    w = [DOC_WEIGHTS[(i + turn) % len(DOC_WEIGHTS)] for i in range(docs)]
    starts, total = [0], 0
    for x in w:
        total += x
        starts.append(total * t // sum(w))
    return starts


def _shuffled(values, seed):
    order = torch.randperm(len(values), generator=torch.Generator().manual_seed(seed))
    return [values[i] for i in order.tolist()]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).to(DEVICE)


def _slopes(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=DEVICE)


def _normal(shape, gen, dtype):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(getattr(torch, dtype))


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    st = {"case": case}
    {"attend": _prepare_attend, "qk": _prepare_qk, "loss": _prepare_loss}[case["do"]](case, seed, gen, st)
    return st


def _prepare_attend(case, seed, gen, st):
    B, Tq, Tk, Hq, Hk, D, dtype = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "D", "dtype"))
    if Tq == Tk:
        # One projection makes queries, keys and values of a token: the heads are slices of its rows.
        qkv = _normal((B, Tq, Hq + 2 * Hk, D), gen, dtype)
        st["q"], st["k"], st["v"] = qkv[:, :, :Hq], qkv[:, :, Hq : Hq + Hk], qkv[:, :, Hq + Hk :]
    else:
        st["q"] = _normal((B, Tq, Hq, D), gen, dtype)
        st["k"], st["v"] = _normal((B, Tk, Hk, D), gen, dtype), _normal((B, Tk, Hk, D), gen, dtype)
    lens = _shuffled(_lens(case, Tk), seed)
    st["args"] = {"causal": case["causal"], "cap": case["cap"], "slope": _slopes(Hq) if case["slope"] else None}
    if case["lengths"] != "full":
        st["args"]["t_k"] = _ints(lens)
        if Tq == Tk:
            st["args"]["t_q"] = st["args"]["t_k"]
    starts = [_doc_starts(t, case["docs"] or 1, seed + b) for b, t in enumerate(lens)]
    if case["docs"]:
        st["args"]["doc_start"] = _ints(starts)
    if case["prefix"]:
        st["args"]["prefix"] = _ints([[(hi - lo) // 4 for lo, hi in zip(s, s[1:])] for s in starts])
    if case["train"]:
        st["dout"] = _normal((B, Tq, Hq, D), gen, dtype)
    if own:
        import paper_2409_07704_amd as mas

        n = mas.mas_attention_workspace_bytes(st["q"], st["k"], backward=case["train"])
        st["buffers"] = {"workspace": torch.empty(n, dtype=torch.uint8, device=DEVICE)}
        st["out"] = torch.empty_like(st["q"], memory_format=torch.contiguous_format)
        if case["train"]:
            st["lse"] = torch.empty((B, Hq, Tq), device=DEVICE)
            for x in "qkv":
                st["buffers"]["d" + x] = torch.empty_like(st[x], memory_format=torch.contiguous_format)


def _prepare_qk(case, seed, gen, st):
    B, T, Hq, Hk, D, R, dtype = (case[k] for k in ("B", "T", "Hq", "Hk", "D", "R", "dtype"))
    qkv = _normal((B, T, Hq + 2 * Hk, D), gen, dtype)
    st["q"], st["k"] = qkv[:, :, :Hq], qkv[:, :, Hq : Hq + Hk]
    st["wq"] = 1.0 + 0.1 * torch.randn(D, generator=gen, device=DEVICE)
    st["wk"] = 1.0 + 0.1 * torch.randn(D, generator=gen, device=DEVICE)
    P = max(T, 8192)
    angle = torch.arange(P, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(R // 2, dtype=torch.float64) / (R // 2))
    st["cos"], st["sin"] = torch.cos(angle).float().to(DEVICE), torch.sin(angle).float().to(DEVICE)
    st["args"] = {"eps": EPS, "interleaved": case["interleaved"]}
    if not case["train"] and T < 16:  # new tokens of streams that are at different places
        first = torch.randint(0, P - T + 1, (B, 1), generator=torch.Generator().manual_seed(seed))
        st["args"]["pos"] = (first + torch.arange(T)).to(torch.int32).to(DEVICE)
    if case["lengths"] != "full":
        st["args"]["t_x"] = _ints(_shuffled(_lens(case, T), seed))
    if case["train"]:
        st["dq_out"], st["dk_out"] = _normal((B, T, Hq, D), gen, dtype), _normal((B, T, Hk, D), gen, dtype)
    if own:
        import paper_2409_07704_amd as mas

        st["q_out"], st["k_out"] = (torch.empty_like(st[x], memory_format=torch.contiguous_format) for x in "qk")
        if case["train"]:
            n = mas.mas_qk_norm_rope_workspace_bytes(st["q"], st["k"])
            st["buffers"] = {"workspace": torch.empty(n, dtype=torch.uint8, device=DEVICE)}
            for x in "qk":
                st["buffers"]["d" + x] = torch.empty_like(st[x], memory_format=torch.contiguous_format)
                st["buffers"]["dw" + x] = torch.empty(D, device=DEVICE)


def _prepare_loss(case, seed, gen, st):
    B, T, S, D = (case[k] for k in ("B", "T", "S", "D"))
    ty = _shuffled(_lens(case, S), seed)
    tx = [min(x, y) for x, y in zip(_shuffled(_lens(case, T), seed + 1), ty)]
    # A monotone alignment: one frame for every text row, the others spread at random.
    i = torch.arange(T)
    x, y = torch.tensor(tx)[:, None], torch.tensor(ty)[:, None]
    w = (torch.rand((B, T), generator=torch.Generator().manual_seed(seed), dtype=torch.float64) + 0.15) * (i < x)
    last = torch.where(i < x, (torch.cumsum(w, 1) / w.sum(1, keepdim=True) * (y - x)).long() + i + 1, y)
    last = torch.where(i == x - 1, y, torch.minimum(last, y))
    st["row_start"] = torch.cat([torch.zeros((B, 1), dtype=torch.long), last], 1).to(torch.int32).to(DEVICE)
    row = torch.searchsorted(st["row_start"][:, 1:].contiguous(), torch.arange(S, dtype=torch.int32, device=DEVICE).expand(B, S).contiguous(), right=True)
    st["mu"] = torch.randn((B, T, D), generator=gen, device=DEVICE)
    st["log_sigma"] = 0.2 * torch.randn((B, T, D), generator=gen, device=DEVICE) - 0.3 if case["sigma"] else None
    st["z"] = 0.8 * torch.randn((B, S, D), generator=gen, device=DEVICE)
    st["z"] += torch.gather(st["mu"], 1, row.clamp(max=T - 1)[:, :, None].expand(B, S, D))
    st["item_weight"] = torch.full((B,), 1.0 / sum(ty), device=DEVICE)
    if own:
        import paper_2409_07704_amd as mas

        n = mas.mas_align_loss_workspace_bytes(B, T, S, D)
        st["buffers"] = {"workspace": torch.empty(n, dtype=torch.uint8, device=DEVICE),
                         "loss_out": torch.empty(B, device=DEVICE), "dmu": torch.empty_like(st["mu"]),
                         "dlog_sigma": torch.empty_like(st["mu"]) if case["sigma"] else None,
                         "dz": torch.empty_like(st["z"])}


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if not own:
        return {"attend": _plain_attend, "qk": _plain_qk, "loss": _plain_loss}[case["do"]](st)
    import paper_2409_07704_amd as mas

    if case["do"] == "loss":
        loss, dmu, dls, dz = mas.mas_align_loss(st["mu"], st["log_sigma"], st["z"], st["row_start"],
                                                item_weight=st["item_weight"], **st["buffers"])
        out = {"loss": loss, "dmu": dmu, "dz": dz}
        return dict(out, dlog_sigma=dls) if case["sigma"] else out
    if case["do"] == "qk":
        rest = (st["wq"], st["wk"], st["cos"], st["sin"])
        q, k = mas.mas_qk_norm_rope(st["q"], st["k"], *rest, q_out=st["q_out"], k_out=st["k_out"], **st["args"])
        if not case["train"]:
            return {"q": q, "k": k}
        dq, dk, dwq, dwk = mas.mas_qk_norm_rope_backward(st["dq_out"], st["dk_out"], st["q"], st["k"], *rest,
                                                         **st["args"], **st["buffers"])
        return {"q": q, "k": k, "dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    qkv = (st["q"], st["k"], st["v"])
    if not case["train"]:
        return {"out": mas.mas_attention(*qkv, out=st["out"], **st["buffers"], **st["args"])}
    out = mas.mas_attention(*qkv, out=st["out"], lse_out=st["lse"], workspace=st["buffers"]["workspace"], **st["args"])
    dq, dk, dv = mas.mas_attention_backward(st["dout"], *qkv, out, st["lse"], **st["buffers"], **st["args"])
    return {"out": out, "dq": dq, "dk": dk, "dv": dv}


def _visible(case, args):
    """Which key a query sees, [B or 1, Tq, Tk], and the distance between them."""
    Tq, Tk = case["Tq"], case["Tk"]
    t_q = args["t_q"][:, None] if "t_q" in args else torch.tensor([[Tq]], device=DEVICE)
    t_k = args["t_k"][:, None] if "t_k" in args else torch.tensor([[Tk]], device=DEVICE)
    i, j = torch.arange(Tq, device=DEVICE)[None], torch.arange(Tk, device=DEVICE)[None]
    place = (i + t_k - t_q)[:, :, None]
    see = ((i < t_q)[:, :, None] & (j < t_k)[:, None]).expand(-1, Tq, Tk)
    hidden = None
    if case["causal"]:
        hidden = j[:, None] > place
    if "doc_start" in args:
        table = args["doc_start"]
        doc = torch.searchsorted(table, torch.arange(Tk, dtype=torch.int32, device=DEVICE).expand(len(table), Tk).contiguous(), right=True) - 1
        see = see & (doc[:, :, None] == doc[:, None])
        if "prefix" in args:
            n = doc.clamp(max=case["docs"] - 1)
            hidden = hidden & (j >= torch.gather(table + torch.nn.functional.pad(args["prefix"], (0, 1)), 1, n))[:, None]
    elif "prefix" in args:
        hidden = hidden & (j >= args["prefix"])[:, None]
    if hidden is not None:
        see = see & ~hidden
    return see, (place - j[:, None]).abs()


def _plain_attend(st):
    case, args = st["case"], st["args"]
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "D"))
    G, cap, scale = Hq // Hk, case["cap"], 1.0 / math.sqrt(case["D"])
    see, distance = _visible(case, args)
    see = see[:, None, None]
    q = st["q"].float().transpose(1, 2).reshape(B, Hk, G * Tq, D)
    k, v = (st[x].float().transpose(1, 2).contiguous() for x in "kv")
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, Hk, G, Tq, Tk).mul_(scale)
    bend = None
    if cap:
        t = torch.tanh(s.div_(cap))
        s = t * cap
        bend = t.square_().neg_().add_(1.0) if case["train"] else None
    if case["slope"]:
        s -= args["slope"].view(Hk, G, 1, 1) * distance[:, None, None]
    s.masked_fill_(~see, -math.inf)
    top = s.amax(4, keepdim=True)
    p = torch.exp(s.sub_(top.masked_fill(top == -math.inf, 0.0)))
    total = p.sum(4, keepdim=True)
    p = p.div_(total.masked_fill(total == 0.0, 1.0)).view(B, Hk, G * Tq, Tk)
    out = torch.matmul(p, v)
    back = lambda x, H: x.view(B, H, -1, D).transpose(1, 2).to(st["q"].dtype).contiguous()
    if not case["train"]:
        return {"out": back(out, Hq)}
    do = st["dout"].float().transpose(1, 2).reshape(B, Hk, G * Tq, D)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    delta = (do * out).sum(3, keepdim=True)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_(delta).mul_(p).mul_(scale)
    if cap:
        ds.mul_(bend.view(B, Hk, G * Tq, Tk))
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q)
    return {"out": back(out, Hq), "dq": back(dq, Hq), "dk": back(dk, Hk), "dv": back(dv, Hk)}


def _plain_turn(x, c, s, R, interleaved):
    a, b = (x[..., :R:2], x[..., 1:R:2]) if interleaved else (x[..., : R // 2], x[..., R // 2 : R])
    y = x.clone()
    if interleaved:
        y[..., :R:2], y[..., 1:R:2] = a * c - b * s, b * c + a * s
    else:
        y[..., : R // 2], y[..., R // 2 : R] = a * c - b * s, b * c + a * s
    return y


def _plain_qk(st):
    case, args = st["case"], st["args"]
    T, R, inter = case["T"], case["R"], case["interleaved"]
    pos = args["pos"].long() if "pos" in args else torch.arange(T, device=DEVICE)[None]
    c, s = st["cos"][pos][:, :, None], st["sin"][pos][:, :, None]
    keep = (torch.arange(T, device=DEVICE) < args["t_x"][:, None])[:, :, None, None] if "t_x" in args else None
    out = {}
    for x in "qk":
        a, w = st[x].float(), st["w" + x]
        r = torch.rsqrt(a.square().mean(3, keepdim=True) + EPS)
        h = a * r
        y = _plain_turn(h * w, c, s, R, inter)
        out[x] = (y if keep is None else y * keep).to(st[x].dtype)
        if case["train"]:
            dy = _plain_turn(st["d" + x + "_out"].float(), c, -s, R, inter)
            if keep is not None:
                dy *= keep
            out["dw" + x] = (dy * h).sum((0, 1, 2))
            g = dy * w
            out["d" + x] = (r * (g - h * (g * h).mean(3, keepdim=True))).to(st[x].dtype)
    return {n: out[n] for n in (("q", "k", "dq", "dk", "dwq", "dwk") if case["train"] else ("q", "k"))}


def _plain_loss(st):
    case, mu, z, table = st["case"], st["mu"], st["z"], st["row_start"]
    B, T, S, D = (case[k] for k in ("B", "T", "S", "D"))
    j = torch.arange(S, dtype=torch.int32, device=DEVICE).expand(B, S).contiguous()
    keep = (j < table[:, T:])[:, :, None]
    row = (torch.searchsorted(table[:, 1:].contiguous(), j, right=True).clamp(max=T - 1)
           + T * torch.arange(B, device=DEVICE)[:, None]).view(-1)
    r = z - mu.view(B * T, D)[row].view(B, S, D)
    dz = r * keep
    cost = 0.5 * LOG_2PI
    if case["sigma"]:
        ls = st["log_sigma"].view(B * T, D)[row].view(B, S, D)
        dz *= torch.exp(-2.0 * ls)
        cost = cost + ls
    loss = ((cost + 0.5 * r * dz) * keep).sum((1, 2))
    weight = st["item_weight"][:, None, None]
    out = {"loss": loss}
    if case["sigma"]:
        dls = torch.zeros((B * T, D), device=DEVICE)
        out["dlog_sigma"] = dls.index_add_(0, row, ((keep.float() - r * dz) * weight).view(-1, D)).view(B, T, D)
    dz *= weight
    out["dmu"] = torch.zeros((B * T, D), device=DEVICE).index_add_(0, row, -dz.view(-1, D)).view(B, T, D)
    out["dz"] = dz
    return {n: out[n] for n in ("loss", "dmu", "dz", "dlog_sigma") if n in out}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    B = case["B"]
    if case["do"] == "loss":
        T, S, D = case["T"], case["S"], case["D"]
        frames = sum(_lens(case, S))
        rows = sum(_lens(case, T))
        two = 2 if case["sigma"] else 1
        # Every output element is written, the zeros of the padding too.
        return {"bytes": 4 * D * (frames + two * rows + B * S + two * B * T) + 4 * B * (T + 1), "flops": 10 * D * frames}
    size = getattr(torch, case["dtype"]).itemsize
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if case["do"] == "qk":
        T, R = case["T"], case["R"]
        used, held = sum(_lens(case, T)) * (Hq + Hk) * D, B * T * (Hq + Hk) * D
        table = 4 * R * (B * T if not case["train"] and T < 16 else T)
        n = 3 if case["train"] else 1  # reads of x, and of the gradient; writes of x, and of its gradient
        return {"bytes": size * ((2 if n == 3 else 1) * used + (2 if n == 3 else 1) * held) + table, "flops": 8 * n * used}
    Tq, Tk = case["Tq"], case["Tk"]
    pairs = 0
    for t in _lens(case, Tk):
        if Tq != Tk:
            n = min(Tq, t)  # of a shorter cache, the first queries see nothing
            pairs += n * t - n * (n - 1) // 2 if case["causal"] else Tq * t
            continue
        starts = _doc_starts(t, case["docs"] or 1, 0)
        for lo, hi in zip(starts, starts[1:]):
            n, m = hi - lo, (hi - lo) // 4 if case["prefix"] else 0
            pairs += n * (n + 1) // 2 + m * (m - 1) // 2 if case["causal"] else n * n
    keys = sum(_lens(case, Tk)) * Hk * D
    rows = (sum(_lens(case, Tk)) if Tq == Tk else B * Tq) * Hq * D
    out = B * Tq * Hq * D
    if not case["train"]:
        return {"bytes": size * (rows + 2 * keys + out), "flops": 4 * Hq * D * pairs}
    return {"bytes": size * (2 * rows + 2 * keys + 2 * out + 2 * B * Tk * Hk * D), "flops": 14 * Hq * D * pairs}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"attend": _exact_attend, "qk": _exact_qk, "loss": _exact_loss}[case["do"]](case, st)


def _exact_attend(case, st):
    """Item by item and head by head; gradients by differentiation of the definition."""
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "D"))
    args = st["args"]
    names = ("q", "k", "v") if case["train"] else ()
    out = {"out": torch.zeros((B, Tq, Hq, D), dtype=torch.float64, device=DEVICE)}
    for x in names:
        out["d" + x] = torch.zeros(st[x].shape, dtype=torch.float64, device=DEVICE)
    for b in range(B):
        nk = int(args["t_k"][b]) if "t_k" in args else Tk
        nq = int(args["t_q"][b]) if "t_q" in args else Tq
        place = torch.arange(nq, device=DEVICE) + (nk - nq)
        key = torch.arange(nk, device=DEVICE)
        allowed = torch.ones((nq, nk), dtype=torch.bool, device=DEVICE)
        if case["causal"]:
            allowed = key[None] <= place[:, None]
        lo = args["doc_start"][b].tolist() if "doc_start" in args else [0, nk]
        if "prefix" in args:
            for n, m in enumerate(args["prefix"][b].tolist()):
                allowed |= ((key >= lo[n]) & (key < lo[n] + m))[None]
        same = torch.zeros_like(allowed)
        for n in range(len(lo) - 1):
            inside = lambda x: (x >= lo[n]) & (x < lo[n + 1])
            same |= inside(place)[:, None] & inside(key)[None]
        if "doc_start" in args:
            allowed &= same
        for h in range(Hq):
            hk = h * Hk // Hq
            q, k, v = (st[x][b, : nq if x == "q" else nk, h if x == "q" else hk].double().requires_grad_(case["train"]) for x in "qkv")
            with torch.set_grad_enabled(case["train"]):
                s = (q @ k.T.contiguous()) / D ** 0.5
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["slope"]:
                    s = s - args["slope"][h].double() * (place[:, None] - key[None]).abs()
                e = torch.exp(s - s.detach().masked_fill(~allowed, -1e300).amax(1, keepdim=True)).masked_fill(~allowed, 0.0)
                o = (e / e.sum(1, keepdim=True).clamp(min=1e-300)) @ v
            out["out"][b, :nq, h] = o.detach()
            if case["train"]:
                grads = torch.autograd.grad(o, (q, k, v), st["dout"][b, :nq, h].double())
                out["dq"][b, :nq, h] = grads[0]
                out["dk"][b, :nk, hk] += grads[1]
                out["dv"][b, :nk, hk] += grads[2]
    return out


def _exact_qk(case, st):
    B, T, R = case["B"], case["T"], case["R"]
    first = (torch.arange(0, R, 2) if case["interleaved"] else torch.arange(R // 2)).to(DEVICE)
    second = first + (1 if case["interleaved"] else R // 2)
    out = {}
    for b in range(B):
        n = int(st["args"]["t_x"][b]) if "t_x" in st["args"] else T
        pos = st["args"]["pos"][b].long() if "pos" in st["args"] else torch.arange(T, device=DEVICE)
        turn = torch.complex(st["cos"].double(), st["sin"].double())[pos[:n], None]
        for x in "qk":
            a = st[x][b, :n].double().requires_grad_(case["train"])
            w = st["w" + x].double().requires_grad_(case["train"])
            with torch.set_grad_enabled(case["train"]):
                y = a / torch.sqrt((a * a).mean(2, keepdim=True) + EPS) * w
                z = torch.complex(y[..., first], y[..., second]) * turn
                y = y.index_copy(2, first, z.real).index_copy(2, second, z.imag)
            full = out.setdefault(x, torch.zeros(st[x].shape, dtype=torch.float64, device=DEVICE))
            full[b, :n] = y.detach()
            if case["train"]:
                ga, gw = torch.autograd.grad(y, (a, w), st["d" + x + "_out"][b, :n].double())
                out.setdefault("d" + x, torch.zeros_like(full))[b, :n] = ga
                out["dw" + x] = out.get("dw" + x, 0.0) + gw
    return out


def _exact_loss(case, st):
    B, T, S, D = (case[k] for k in ("B", "T", "S", "D"))
    shape = lambda n: torch.zeros((B, n, D), dtype=torch.float64, device=DEVICE)
    out = {"loss": torch.zeros(B, dtype=torch.float64, device=DEVICE), "dmu": shape(T), "dz": shape(S)}
    if case["sigma"]:
        out["dlog_sigma"] = shape(T)
    for b in range(B):
        held = (st["row_start"][b, 1:] - st["row_start"][b, :-1]).long()
        n = int(held.sum())
        mu, z = (st[x][b].double().requires_grad_() for x in ("mu", "z"))
        ls = (st["log_sigma"][b] if case["sigma"] else torch.zeros_like(st["mu"][b])).double().requires_grad_()
        with torch.enable_grad():
            m, l = (torch.repeat_interleave(x, held, 0) for x in (mu, ls))
            loss = (0.5 * LOG_2PI + l + 0.5 * ((z[:n] - m) / torch.exp(l)) ** 2).sum()
            grads = torch.autograd.grad(loss * st["item_weight"][b].double(), (mu, z, ls))
        out["loss"][b] = loss.detach()
        out["dmu"][b], out["dz"][b] = grads[0], grads[1]
        if case["sigma"]:
            out["dlog_sigma"][b] = grads[2]
    return out
