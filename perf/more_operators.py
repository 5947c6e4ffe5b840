"""The operators of softmax attention on the sizes they are timed at.

A layer of exact attention over an event stream or a batch of point clouds, in
training and with a kept cache: norms of queries and keys with the rotation by
their positions, attention over packed sequences with its gradients, the pages
of a cache for new tokens, and attention of new tokens over those pages.

`run()` computes a case in plain torch operations, or, where `own` is true, by
the library's calls.  `exact()` recomputes it in float64 by another way.
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_SCORES = 4_300_000_000  # of a plain form, padded to its longest sequences (17 GB)
MOST_FLOPS = 1.3e12


# ---------------------------------------------------------------- cases
def listed():
    return [
        # Queries and keys of a 300k-event recording, by time, row and column.
        dict(name="qk_events_300k_bf16", op="qk", train=False, n=300_000, hq=4, hk=4, d=64, s0=16,
             s1=8, s2=8, events=True, interleaved=True, dtype="bf16"),
        # The gradients of a batch of 32 clouds of 1024 points; part of a head turns.
        dict(name="qk_grad_points_32768", op="qk", train=True, n=32_768, hq=8, hk=2, d=96, s0=11,
             s1=11, s2=10, events=False, interleaved=False, dtype="f32"),
        # One small cloud (256 points), all points with all: the latency of a single example.
        dict(name="attn_cloud_256", op="attn", train=False, causal=False, b=1, lq=256, lk=256,
             hq=4, hk=4, dk=64, dv=64, dtype="f32"),
        # 32 prompts of different lengths, heads in groups.
        dict(name="attn_prompts_32x1024_bf16", op="attn", train=False, causal=True, b=32, lq=1024,
             lk=1024, hq=8, hk=2, dk=128, dv=128, dtype="bf16"),
        # One recording of 32768 events.
        dict(name="attn_events_32768_bf16", op="attn", train=False, causal=True, b=1, lq=32_768,
             lk=32_768, hq=4, hk=4, dk=64, dv=64, dtype="bf16"),
        # The gradients of down-sampled points that see their whole clouds.
        dict(name="attn_grad_clouds_down", op="attn", train=True, causal=False, b=32, lq=301,
             lk=1024, hq=4, hk=4, dk=64, dv=64, dtype="f32"),
        # The gradients of a long sequence, heads in groups.
        dict(name="attn_grad_16384_bf16", op="attn", train=True, causal=True, b=1, lq=16_384,
             lk=16_384, hq=8, hk=2, dk=128, dv=128, dtype="bf16"),
        # The next token of one stream: latency.
        dict(name="paged_1x4095_bf16", op="paged", b=1, ctx=4095, new=1, page=16, hq=8, hk=2,
             dk=128, dv=128, dtype="bf16"),
        # The next token of each of 64 streams.
        dict(name="paged_64x8000_bf16", op="paged", b=64, ctx=8000, new=1, page=64, hq=8, hk=2,
             dk=128, dv=128, dtype="bf16"),
        # Chunks of new events behind what their streams have kept, pages of an odd size.
        dict(name="paged_chunks_12x300_bf16", op="paged", b=12, ctx=5000, new=300, page=48, hq=4,
             hk=4, dk=64, dv=64, dtype="bf16"),
        # Pages for the next token of each of 64 streams.
        dict(name="pages_64x1_bf16", op="pages", b=64, ctx=2000, new=1, page=16, hk=2, dk=128,
             dv=128, short=False, dtype="bf16"),
        # Pages for 64 prompts of float32 channels.
        dict(name="pages_64x1000", op="pages", b=64, ctx=100, new=1000, page=32, hk=4, dk=64,
             dv=64, short=False, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


HEADS = [(1, 1), (2, 2), (4, 4), (8, 8), (8, 2), (6, 3), (3, 1), (12, 2), (16, 1)]
CHANNELS = [(32, 32), (64, 64), (64, 64), (128, 128), (128, 128), (96, 96), (40, 72), (128, 64),
            (33, 31), (16, 16)]


def draw(rng):
    op = rng.choice(["qk", "qk", "attn", "attn", "attn", "attn", "paged", "paged", "pages"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    hq, hk = rng.choice(HEADS)
    if op == "qk":
        d = rng.choice([16, 32, 40, 64, 64, 96, 128, 128])
        s = [max(1, d // 6 - rng.randint(0, 2)) for _ in range(3)]
        return dict(op=op, train=rng.random() < 0.5,
                    n=_log_int(rng, 1, min(300_000, 70_000_000 // (d * (hq + hk)))), hq=hq, hk=hk,
                    d=d, s0=s[0], s1=s[1], s2=s[2], events=rng.random() < 0.5,
                    interleaved=rng.random() < 0.5, dtype=dtype)
    dk, dv = rng.choice(CHANNELS)
    if op == "attn":
        case = dict(op=op, train=rng.random() < 0.5, causal=rng.random() < 0.6, b=1, lq=1, lk=1,
                    hq=hq, hk=hk, dk=dk, dv=dv, dtype=dtype)
        pairs = 10 ** rng.uniform(3, 9.3)  # of queries and keys, over heads and sequences
        most = MOST_FLOPS / ((10 if case["train"] else 4) * max(dk, dv))
        pairs = min(pairs, MOST_SCORES / 2.5, most / 1.2)
        case["b"] = min(_log_int(rng, 1, 300), max(1, int(pairs / hq)))
        length = math.sqrt(pairs / hq / case["b"])
        ratio = 1.0 if rng.random() < 0.6 else 2 ** rng.uniform(-2, 2)
        case["lq"] = max(1, int(length * math.sqrt(ratio)))
        case["lk"] = max(1, int(length / math.sqrt(ratio)))
        return case
    row = hk * (dk + dv)
    page = rng.choice([1, 5, 16, 16, 32, 48, 64, 64, 128, 256])
    b = _log_int(rng, 1, 256)
    if op == "paged":
        ctx = _log_int(rng, 1, min(40_000, 130_000_000 // (row * b)))
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 1024)
        most = min(MOST_SCORES / 2.5, MOST_FLOPS / (4 * max(dk, dv)))
        new = max(1, min(new, int(most / (b * hq * (ctx + new)))))
        return dict(op=op, b=b, ctx=ctx, new=new, page=page, hq=hq, hk=hk, dk=dk, dv=dv,
                    dtype=dtype)
    ctx = _log_int(rng, 1, min(4000, 60_000_000 // (row * b)))
    new = 1 if rng.random() < 0.5 else _log_int(rng, 2, min(4000, max(2, 30_000_000 // (row * b))))
    return dict(op=op, b=b, ctx=ctx, new=new, page=page, hk=hk, dk=dk, dv=dv,
                short=rng.random() < 0.3, dtype=dtype)


# ---------------------------------------------------------------- lengths of sequences
def _lengths(b, mean, least=0):
    """b lengths from half of the mean to one and a half of it; of many, an empty one and one
    of a single token."""
    if b == 1 or mean == 1:
        return [mean] * b
    lens = [mean // 2 + (2 * i + 1) * mean // (2 * b) for i in range(b)]
    if b >= 8:
        lens[0], lens[1] = 0, 1
    return [max(least, x) for x in lens]


def _pair_lengths(case):
    """Of the queries and of the keys, sequence by sequence.  Keys of their own lengths: the
    most queries meet the fewest keys."""
    lq = _lengths(case["b"], case["lq"])
    if case["lk"] == case["lq"]:
        return lq, lq
    return lq, _lengths(case["b"], case["lk"])[::-1]


def _cache_lengths(case):
    """Of the kept tokens and of the new ones."""
    kept = _lengths(case["b"], case["ctx"])
    new = [case["new"]] * case["b"] if case["new"] == 1 else _lengths(case["b"], case["new"])[::-1]
    return kept, new


def _visible(q, k, causal):
    """Pairs that count, of q queries whose last sees the last of k keys."""
    if not causal:
        return q * k
    first = max(0, q - k)  # queries before the first key
    m = q - first
    return m * (k - q + first) + m * (m + 1) // 2


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op == "qk":
        values = case["n"] * (case["hq"] + case["hk"]) * case["d"]
        pairs = case["s0"] + case["s1"] + case["s2"]
        grads = 8 * case["d"] if case["train"] else 0
        return {"bytes": (3 if case["train"] else 2) * values * e + 12 * case["n"] + 4 * pairs
                + 8 * case["d"] + grads,
                "flops": (14 if case["train"] else 6) * values}
    hk, dk, dv = case["hk"], case["dk"], case["dv"]
    if op == "pages":
        kept, new = _cache_lengths(case)
        held = sum(-(-(a + n) // case["page"]) for a, n in zip(kept, new))
        return {"bytes": sum(new) * (2 * hk * (dk + dv) * e + 8) + 8 * held + 12 * case["b"],
                "flops": sum(new)}
    hq = case["hq"]
    if op == "paged":
        kept, new = _cache_lengths(case)
        n = sum(new)
        rows = sum(a + c for a, c in zip(kept, new) if c)
        pairs = sum(_visible(c, a + c, True) for a, c in zip(kept, new))
        return {"bytes": (n * hq + rows * hk) * (dk + dv) * e + 4 * rows // case["page"],
                "flops": 2 * (dk + dv) * hq * pairs}
    lq, lk = _pair_lengths(case)
    n, m = sum(lq), sum(lk)
    pairs = sum(_visible(a, c, case["causal"]) for a, c in zip(lq, lk))
    io = (n * hq + m * hk) * (dk + dv) * e + 4 * n * hq  # q, k, v, o and lse
    if case["train"]:  # do beside them, and three gradients
        return {"bytes": io + n * hq * (dk + dv) * e + m * hk * (dk + dv) * e,
                "flops": 2 * (3 * dk + 2 * dv) * hq * pairs}
    return {"bytes": io, "flops": 2 * (dk + dv) * hq * pairs}


# ---------------------------------------------------------------- inputs
def _splits(lens):
    return torch.tensor([0] + lens).cumsum(0).to(torch.int32)


def prepare(case, seed):
    host = torch.Generator().manual_seed(int(seed))
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    s = {"case": case}
    if case["op"] == "qk":
        return _prepare_qk(case, s, normal, gen, dt)
    b, hk, dk, dv = case["b"], case["hk"], case["dk"], case["dv"]
    order = torch.randperm(b, generator=host).tolist()  # which sequence comes when
    s["scale"] = dk ** -0.5
    if case["op"] == "attn":
        lq, lk = _pair_lengths(case)
        s["most_q"], s["most_k"] = max(lq), max(lk)
        s["splits"] = _splits([lq[i] for i in order]).to(DEVICE)
        s["k_splits"] = (None if case["lk"] == case["lq"]
                         else _splits([lk[i] for i in order]).to(DEVICE))
        n, m = sum(lq), sum(lk)
        s["q"], s["k"], s["v"] = (normal(n, case["hq"], dk).to(dt), normal(m, hk, dk).to(dt),
                                  normal(m, hk, dv).to(dt))
        s["q"] *= 1.5  # some keys stand out
        if case["train"]:
            s["do"] = normal(n, case["hq"], dv).to(dt)
            # what the forward pass left
            s["o"], s["lse"] = _plain_attn(s)
        return s
    kept, new = _cache_lengths(case)
    kept, new = [kept[i] for i in order], [new[i] for i in order]
    page = case["page"]
    held = [-(-a // page) for a in kept]
    after = [-(-(a + c) // page) for a, c in zip(kept, new)]
    most = max(after) + 2  # pages that a stream's row of the table has room for
    n_pages = sum(after) + 3
    s["splits"] = None if case["new"] == 1 else _splits(new).to(DEVICE)
    s["k_pages"], s["v_pages"] = (normal(n_pages, page, hk, d).to(dt) for d in (dk, dv))
    perm = torch.randperm(n_pages, generator=host).to(torch.int32)
    n = sum(new)
    counts = torch.tensor(after if case["op"] == "paged" else held)
    there = torch.arange(most)[None, :] < counts[:, None]
    table = torch.full((b, most), -1, dtype=torch.int32)
    table[there] = perm[:int(counts.sum())]
    s["table"] = table.to(DEVICE)
    if case["op"] == "paged":
        s["lengths"] = torch.tensor([a + c for a, c in zip(kept, new)], dtype=torch.int32).to(DEVICE)
        s["most_q"] = max(new)
        s["q"] = (1.5 * normal(n, case["hq"], dk)).to(dt)
        return s
    s["lengths"] = torch.tensor(kept, dtype=torch.int32).to(DEVICE)
    free = perm[int(counts.sum()):]
    if case["short"]:  # the pool has not enough
        free = free[:max(1, (sum(after) - sum(held)) // 2)]
    s["free"] = free.contiguous().to(DEVICE)
    s["k"], s["v"] = normal(n, hk, dk).to(dt), normal(n, hk, dv).to(dt)
    return s


def _prepare_qk(case, s, normal, gen, dt):
    n, d = case["n"], case["d"]
    s["q"], s["k"] = normal(n, case["hq"], d).to(dt), normal(n, case["hk"], d).to(dt)
    s["q_weight"], s["k_weight"] = 1 + 0.2 * normal(d), 1 + 0.2 * normal(d)
    if case["train"]:
        s["dq"], s["dk"] = normal(n, case["hq"], d).to(dt), normal(n, case["hk"], d).to(dt)
    s["sections"] = (case["s0"], case["s1"], case["s2"])
    if case["events"]:  # time, row and column of events on a 128 x 128 sensor
        t = torch.sort(torch.randint(0, 100_000, (n,), device=DEVICE, generator=gen)).values
        xy = torch.randint(0, 128, (n, 2), device=DEVICE, generator=gen)
        s["positions"] = torch.cat([t[:, None], xy], 1).to(torch.int32)
        extents = (100_000.0, 128.0, 128.0)
    else:  # points on an ellipsoid
        x = normal(n, 3)
        s["positions"] = x / x.norm(dim=1, keepdim=True) * torch.tensor([1.0, 0.8, 0.6],
                                                                        device=DEVICE)
        extents = (1.0, 1.0, 1.0)
    # the fastest pair turns by 60 over its axis' extent, the slowest by 0.5
    s["freqs"] = torch.cat([60.0 / e * (0.5 / 60) ** (torch.arange(m) / max(1, m - 1))
                            for m, e in zip(s["sections"], extents)]).to(DEVICE, torch.float32)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2012_01170_amd as sbc

    case = s["case"]
    if case["op"] == "qk":
        if case["train"]:
            return sbc.qk_norm_rotary_backward(
                s["dq"], s["dk"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["positions"],
                s["freqs"], s["sections"], interleaved=case["interleaved"], eps=EPS)
        return sbc.qk_norm_rotary_forward(s["q"], s["k"], s["q_weight"], s["k_weight"],
                                          s["positions"], s["freqs"], s["sections"],
                                          interleaved=case["interleaved"], eps=EPS)
    if case["op"] == "attn":
        if case["train"]:
            return sbc.softmax_attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"],
                                                  s["lse"], splits=s["splits"],
                                                  k_splits=s["k_splits"], scale=s["scale"],
                                                  causal=case["causal"])
        return sbc.softmax_attention_forward(s["q"], s["k"], s["v"], splits=s["splits"],
                                             k_splits=s["k_splits"], scale=s["scale"],
                                             causal=case["causal"])
    if case["op"] == "paged":
        return sbc.softmax_attention_paged(s["q"], s["k_pages"], s["v_pages"], s["table"],
                                           s["lengths"], splits=s["splits"], scale=s["scale"])
    table, slots, lengths, needed = sbc.cache_slots(s["lengths"], s["table"], s["free"],
                                                    case["page"], splits=s["splits"],
                                                    n=s["k"].shape[0])
    sbc.cache_append(s["k"], s["v"], s["k_pages"], s["v_pages"], slots)
    return table, slots, lengths, needed, s["k_pages"], s["v_pages"]


def _run_plain(s):
    op, train = s["case"]["op"], s["case"].get("train")
    if op == "qk":
        return _plain_qk_grad(s) if train else _plain_qk(s)
    if op == "attn":
        return _plain_attn_grad(s) if train else _plain_attn(s)
    return _plain_paged(s) if op == "paged" else _plain_pages(s)


# norms and rotation
def _plain_angles(s):
    p, (s0, s1, s2) = s["positions"].double(), s["sections"]
    angle = torch.cat([p[:, 0:1].expand(-1, s0), p[:, 1:2].expand(-1, s1),
                       p[:, 2:3].expand(-1, s2)], 1) * s["freqs"].double()
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _plain_turn(f, cos, sin, interleaved):
    m = cos.shape[-1]
    a, b = (f[..., 0:2 * m:2], f[..., 1:2 * m:2]) if interleaved else (f[..., :m], f[..., m:2 * m])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, f[..., 2 * m:]], -1)


def _plain_unit(x):
    f = x.float()
    rstd = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    return f * rstd, rstd


def _plain_qk(s):
    cos, sin = _plain_angles(s)
    inter = s["case"]["interleaved"]
    q, k = _plain_unit(s["q"])[0] * s["q_weight"], _plain_unit(s["k"])[0] * s["k_weight"]
    return (_plain_turn(q, cos, sin, inter).to(s["q"].dtype),
            _plain_turn(k, cos, sin, inter).to(s["k"].dtype))


def _plain_one_grad(dy, x, w, cos, sin, inter):
    g = _plain_turn(dy.float(), cos, -sin, inter)
    xn, rstd = _plain_unit(x)
    gw = g * w
    dx = rstd * (gw - xn * (gw * xn).mean(-1, keepdim=True))
    return dx.to(x.dtype), (g * xn).flatten(0, 1).sum(0)


def _plain_qk_grad(s):
    cos, sin = _plain_angles(s)
    inter = s["case"]["interleaved"]
    dq, dqw = _plain_one_grad(s["dq"], s["q"], s["q_weight"], cos, sin, inter)
    dk, dkw = _plain_one_grad(s["dk"], s["k"], s["k_weight"], cos, sin, inter)
    return dq, dk, dqw, dkw


# attention over sequences that are padded to the longest
def _plain_pad(x, splits, most):
    """[n, h, d] -> [b, h, most, d] in float32, zero past a sequence's end"""
    at = splits[:-1].long()[:, None] + torch.arange(most, device=x.device)
    ok = at < splits[1:, None]
    x = x[at.clamp(max=max(0, x.shape[0] - 1))].float() if x.shape[0] else x.new_zeros(
        *at.shape, *x.shape[1:], dtype=torch.float32)
    return torch.where(ok[..., None, None], x, 0.0).transpose(1, 2).contiguous()


def _plain_pack(x, splits, like):
    """back again, in the type of `like` [n, h, d]"""
    i = torch.arange(like.shape[0], device=like.device)
    seq = torch.searchsorted(splits[1:].long().contiguous(), i, right=True)
    return x[seq, :, i - splits.long()[seq]].to(like.dtype)


def _plain_seen(lq, lk, most_q, most_k, causal):
    """[b, 1, 1, most_q, most_k]: whether a query sees a key"""
    i = torch.arange(most_q, device=lq.device)[None, :, None]
    j = torch.arange(most_k, device=lq.device)[None, None, :]
    lq, lk = lq[:, None, None], lk[:, None, None]
    seen = (i < lq) & (j < lk)
    if causal:
        seen = seen & (j <= i + lk - lq)
    return seen[:, None, None]


def _plain_scores(q, k, seen, scale):
    """q [b, hk, g, lq, d], k [b, hk, lk, d] -> scores, -inf where a query sees no key"""
    b, hk, g, lq, d = q.shape
    x = torch.matmul(q.view(b, hk, g * lq, d), k.transpose(2, 3).contiguous())
    return x.view(b, hk, g, lq, -1).mul_(scale).masked_fill_(~seen, -math.inf)


def _plain_softmax_product(x, v):
    """scores [b, hk, g, lq, lk] (overwritten) and v -> o [b, hk, g, lq, dv], lse"""
    b, hk, g, lq, lk = x.shape
    if lk == 0:
        return x.new_zeros(b, hk, g, lq, v.shape[-1]), x.new_full((b, hk, g, lq), -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(b, hk, g * lq, lk), v).view(b, hk, g, lq, -1)
    return torch.where(total > 0, o / total, 0.0), (top + torch.log(total)).squeeze(-1)


def _plain_attn_in(s):
    case, hk = s["case"], s["case"]["hk"]
    splits = s["splits"]
    k_splits = splits if s["k_splits"] is None else s["k_splits"]
    q = _plain_pad(s["q"], splits, s["most_q"])
    b, hq, lq, d = q.shape
    seen = _plain_seen(splits[1:] - splits[:-1], k_splits[1:] - k_splits[:-1], s["most_q"],
                       s["most_k"], case["causal"])
    return (q.view(b, hk, hq // hk, lq, d), _plain_pad(s["k"], k_splits, s["most_k"]),
            _plain_pad(s["v"], k_splits, s["most_k"]), seen, splits, k_splits)


def _plain_attn(s):
    q, k, v, seen, splits, _ = _plain_attn_in(s)
    o, lse = _plain_softmax_product(_plain_scores(q, k, seen, s["scale"]), v)
    like = s["q"].new_empty(s["q"].shape[0], s["q"].shape[1], v.shape[-1])
    return (_plain_pack(o.flatten(1, 2), splits, like),
            _plain_pack(lse.flatten(1, 2)[..., None], splits,
                        like[..., :1].float()).squeeze(-1).contiguous())


def _plain_attn_grad(s):
    q, k, v, seen, splits, k_splits = _plain_attn_in(s)
    b, hk, g, lq, dk = q.shape
    pad = lambda x: _plain_pad(x, splits, lq).view(b, hk, g, lq, -1)  # noqa: E731
    do, o, lse = pad(s["do"]), pad(s["o"]), pad(s["lse"][..., None])
    p = _plain_scores(q, k, seen, s["scale"])
    p = p.sub_(lse).exp_().masked_fill_(~seen, 0.0)  # (rows without a key have no lse)
    rows = lambda x: x.reshape(b, hk, g * lq, -1)  # noqa: E731
    dv = torch.matmul(rows(p).transpose(2, 3), rows(do))
    ds = torch.matmul(rows(do), v.transpose(2, 3).contiguous()).view(p.shape)
    ds = ds.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq = torch.matmul(rows(ds), k).view(b, hk * g, lq, dk)
    dk_ = torch.matmul(rows(ds).transpose(2, 3), rows(q))
    return (_plain_pack(dq, splits, s["q"]), _plain_pack(dk_, k_splits, s["k"]),
            _plain_pack(dv, k_splits, s["v"]))


# a cache in pages
def _plain_new(s):
    """The splits of the new tokens"""
    if s["splits"] is not None:
        return s["splits"]
    return torch.arange(s["table"].shape[0] + 1, device=s["table"].device, dtype=torch.int32)


def _plain_paged(s):
    hk = s["case"]["hk"]
    splits, table = _plain_new(s), s["table"].clamp(min=0).long()
    b = table.shape[0]
    most = table.shape[1] * s["k_pages"].shape[1]
    k = s["k_pages"][table].float().view(b, most, hk, -1).transpose(1, 2).contiguous()
    v = s["v_pages"][table].float().view(b, most, hk, -1).transpose(1, 2).contiguous()
    q = _plain_pad(s["q"], splits, s["most_q"])
    q = q.view(b, hk, q.shape[1] // hk, *q.shape[2:])
    seen = _plain_seen(splits[1:] - splits[:-1], s["lengths"], s["most_q"], most, True)
    o, _ = _plain_softmax_product(_plain_scores(q, k, seen, s["scale"]), v)
    like = s["q"].new_empty(s["q"].shape[0], s["q"].shape[1], v.shape[-1])
    return _plain_pack(o.flatten(1, 2), splits, like)


def _plain_pages(s):
    page, table, free = s["case"]["page"], s["table"], s["free"]
    splits, lens = _plain_new(s).long(), s["lengths"].long()
    b, most = table.shape
    after = lens + splits[1:] - splits[:-1]
    held = ((lens + page - 1) // page).clamp(max=most)
    need = ((after + page - 1) // page).clamp(max=most) - held
    upto = torch.cumsum(need, 0)
    at = torch.arange(most, device=table.device)
    rank = (upto - need)[:, None] + at - held[:, None]  # of a page among those handed out
    fresh = (at >= held[:, None]) & (at < (held + need)[:, None])
    given = torch.where(rank < free.shape[0], free[rank.clamp(0, free.shape[0] - 1)], -1)
    table = torch.where(fresh, given, table)
    i = torch.arange(s["k"].shape[0], device=table.device)
    seq = torch.searchsorted(splits[1:].contiguous(), i, right=True)
    pos = lens[seq] + i - splits[seq]
    where = pos // page
    p = torch.where(where < most, table[seq, where.clamp(max=most - 1)], -1).long()
    slots = torch.where(p >= 0, p * page + pos % page, -1)
    ok = slots >= 0
    for pages, rows in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        pages.view(-1, *rows.shape[1:])[slots[ok]] = rows[ok]
    return (table, slots, after.to(torch.int32), upto[-1:].to(torch.int32), s["k_pages"],
            s["v_pages"])


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "qk":
        return _exact_qk(s)
    if case["op"] == "attn":
        return _exact_attn(s)
    return _exact_paged(s) if case["op"] == "paged" else _exact_pages(s)


def _exact_qk(s):
    case = s["case"]
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(s["sections"])).to(DEVICE)
    angle = s["positions"].double()[:, axis] * s["freqs"].double()
    m = axis.numel()
    i = torch.arange(m, device=DEVICE)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + m)

    def turn(x, angle):
        z = torch.complex(x[..., first], x[..., second])
        z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    out, sums = [], []
    for name in ("q", "k"):
        x, w = s[name].double(), s[name + "_weight"].double()
        d = x.shape[-1]
        square = (x * x).sum(-1, keepdim=True) / d + EPS
        if not case["train"]:
            out.append(turn(x * w / torch.sqrt(square), angle))
            continue
        g = turn(s["d" + name].double(), -angle)
        # through the product, and through the norm in its denominator
        dx = g * w / torch.sqrt(square) - x * ((g * w * x).sum(-1, keepdim=True) / d) * square ** -1.5
        out.append(dx)
        sums.append((g * x / torch.sqrt(square)).sum((0, 1)))
    return (*out, *sums)


def _exact_sequence(q, k, v, causal, scale, grad=None):
    """One sequence: q [hq, n, dk], k [hk, m, dk], v in float64, in blocks of queries.  grad:
    (do, o, lse) [hq, n, ...] for the gradients."""
    hq, n, _ = q.shape
    hk, m, _ = k.shape
    group = torch.arange(hq, device=q.device) // (hq // hk)
    T = lambda x: x.transpose(-1, -2).contiguous()  # noqa: E731
    o = torch.zeros(hq, n, v.shape[-1], dtype=torch.float64, device=q.device)
    lse = torch.full((hq, n), -math.inf, dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    step = max(16, min(4096, 500_000_000 // max(1, hq * m)))
    for i in range(0, n, step):
        j = min(i + step, n)
        upto = min(m, j + m - n) if causal else m
        if upto <= 0:
            continue
        K, V = k[:, :upto][group], v[:, :upto][group]
        x = torch.matmul(q[:, i:j], T(K)) * scale
        if causal:
            row = torch.arange(i, j, device=q.device)[:, None] + (m - n)
            hidden = torch.arange(upto, device=q.device)[None, :] > row
            x = torch.where(hidden, -math.inf, x)
        if grad is None:
            lse[:, i:j] = torch.logsumexp(x, -1)
            some = lse[:, i:j] > -math.inf
            p = torch.where(some[..., None], torch.exp(x - lse[:, i:j, None]), 0.0)
            o[:, i:j] = torch.matmul(p, V)
            continue
        do, was, stat = (y[:, i:j] for y in grad)
        p = torch.where(x > -math.inf, torch.exp(x - stat[..., None]), 0.0)
        ds = p * (torch.matmul(do, T(V)) - (do * was).sum(-1, keepdim=True)) * scale
        dq[:, i:j] = torch.matmul(ds, K)
        dk[:, :upto].index_add_(0, group, torch.matmul(T(ds), q[:, i:j].contiguous()))
        dv[:, :upto].index_add_(0, group, torch.matmul(T(p), do.contiguous()))
    return (o, lse) if grad is None else (dq, dk, dv)


def _exact_attn(s):
    case = s["case"]
    splits = s["splits"].tolist()
    k_splits = splits if s["k_splits"] is None else s["k_splits"].tolist()
    f = lambda x: x.double().transpose(0, 1).contiguous()  # noqa: E731
    q, k, v = f(s["q"]), f(s["k"]), f(s["v"])
    grad = (f(s["do"]), f(s["o"]), s["lse"].double().t().contiguous()) if case["train"] else None
    parts = []
    for a, b, c, d in zip(splits, splits[1:], k_splits, k_splits[1:]):
        parts.append(_exact_sequence(q[:, a:b], k[:, c:d], v[:, c:d], case["causal"], s["scale"],
                                     None if grad is None else [x[:, a:b] for x in grad]))
    return tuple(torch.cat(x, 1).transpose(0, 1) for x in zip(*parts))


def _exact_paged(s):
    case = s["case"]
    lengths, table = s["lengths"].tolist(), s["table"].long()
    splits = list(range(len(lengths) + 1)) if s["splits"] is None else s["splits"].tolist()
    parts = []
    for b, n in enumerate(lengths):
        x = s["q"][splits[b]:splits[b + 1]].double().transpose(0, 1).contiguous()
        if x.shape[1] == 0:
            continue
        pages = table[b, :-(-n // case["page"])]
        k, v = (p[pages].flatten(0, 1)[:n].double().transpose(0, 1).contiguous()
                for p in (s["k_pages"], s["v_pages"]))
        parts.append(_exact_sequence(x, k, v, True, s["scale"])[0])
    return torch.cat(parts, 1).transpose(0, 1)


def _exact_pages(s):
    """The rows' places one stream after another; of the whole numbers nothing is computed."""
    page, table = s["case"]["page"], s["table"].tolist()
    free, lens = s["free"].tolist(), s["lengths"].tolist()
    splits = list(range(len(lens) + 1)) if s["splits"] is None else s["splits"].tolist()
    k, v = s["k_pages"].double().flatten(0, 1), s["v_pages"].double().flatten(0, 1)
    to, rows = [], []
    for b, n in enumerate(lens):
        row = table[b][:-(-n // page)]
        for i in range(splits[b], splits[b + 1]):
            if n // page == len(row):
                row.append(free.pop(0) if free and len(row) < len(table[b]) else -1)
            if row[n // page] >= 0:
                to.append(row[n // page] * page + n % page)
                rows.append(i)
            n += 1
    if to:
        to, rows = torch.tensor(to, device=DEVICE), torch.tensor(rows, device=DEVICE)
        k[to], v[to] = s["k"].double()[rows], s["v"].double()[rows]
    shape = s["k_pages"].shape[:3]
    return None, None, None, None, k.view(*shape, -1), v.view(*shape, -1)
