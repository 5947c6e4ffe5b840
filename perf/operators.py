"""The sequence operators on the sizes they are timed at.

A layer over an event stream or a batch of point clouds, next to the library's
convolutions: layer norm, rotary positions with several axes (time and pixel of
an event, coordinates of a point), and linear attention with a decay for each
head, forward, backward and as a step of one token.

`run()` computes a case in plain torch operations, or, where `own` is true, by
the library's calls.  `exact()` recomputes it in float64 by another way.
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-5
CHUNK = 128  # tokens that the plain form of the attention takes at once
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # The features of one small cloud (256 outputs, 32 channels): the latency of a
        # single example.
        dict(name="norm_256x32", op="norm", train=False, n=256, c=32, bias=True, dtype="f32"),
        # A 1M-event recording of 64 bf16 channels.
        dict(name="norm_events_1m_bf16", op="norm", train=False, n=1_000_000, c=64, bias=True,
             dtype="bf16"),
        # The gradients of a norm over a batch of 32 clouds of 1024 points.
        dict(name="norm_grad_32768x64", op="norm", train=True, n=32_768, c=64, bias=True,
             dtype="f32"),
        # Wide rows of an odd length, without a bias.
        dict(name="norm_grad_12007x1001_bf16", op="norm", train=True, n=12_007, c=1001,
             bias=False, dtype="bf16"),
        # Queries and keys of a batch of 32 clouds turned by the points' coordinates.
        dict(name="rotary_points_32768", op="rotary", train=False, n=32_768, hq=4, hk=4, d=64,
             s0=11, s1=11, s2=10, events=False, interleaved=False, dtype="f32"),
        # The gradients of queries and keys of a 300k-event recording: time, row, column.
        dict(name="rotary_grad_events_300k_bf16", op="rotary", train=True, n=300_000, hq=4, hk=4,
             d=64, s0=16, s1=8, s2=8, events=True, interleaved=True, dtype="bf16"),
        # Prompts of different lengths that go on from a kept state, which is wanted after
        # them too (decay by position).
        dict(name="attn_prompts_32768", op="attn", train=False, n=32_768, b=32, h=4, dk=64, dv=64,
             times=False, state=True, dtype="f32"),
        # One 300k-event recording, decayed by the events' times.
        dict(name="attn_events_300k_bf16", op="attn", train=False, n=300_000, b=1, h=4, dk=64,
             dv=64, times=True, state=False, dtype="bf16"),
        # Its gradients.
        dict(name="attn_grad_events_300k_bf16", op="attn", train=True, n=300_000, b=1, h=4, dk=64,
             dv=64, times=True, state=False, dtype="bf16"),
        # A training batch of short sequences, odd in every size.
        dict(name="attn_grad_11003_odd", op="attn", train=True, n=11_003, b=37, h=3, dk=40, dv=72,
             times=False, state=False, dtype="f32"),
        # One token of one stream: the latency of a live sensor.
        dict(name="step_1", op="step", b=1, h=4, dk=64, dv=64, times=True, dtype="f32"),
        # One token for each of 512 streams.
        dict(name="step_512_bf16", op="step", b=512, h=8, dk=64, dv=64, times=True,
             dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "rotary", "rotary", "attn", "attn", "attn", "step"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "norm":
        c = _log_int(rng, 8, 4096)
        return dict(op=op, train=rng.random() < 0.5, n=_log_int(rng, 1, max(2, 24_000_000 // c)),
                    c=c, bias=rng.random() < 0.7, dtype=dtype)
    if op == "rotary":
        d = rng.choice([16, 32, 40, 64, 64, 96, 128])
        hq, hk = rng.choice([(1, 1), (2, 2), (4, 4), (8, 8), (8, 2), (6, 3), (3, 1)])
        s = [max(1, d // 6 - rng.randint(0, 2)) for _ in range(3)]
        return dict(op=op, train=rng.random() < 0.5,
                    n=_log_int(rng, 16, min(300_000, 70_000_000 // (d * (hq + hk)))), hq=hq, hk=hk,
                    d=d, s0=s[0], s1=s[1], s2=s[2], events=rng.random() < 0.5,
                    interleaved=rng.random() < 0.5, dtype=dtype)
    h = rng.choice([1, 2, 3, 4, 6, 8])
    dk, dv = rng.choice([(32, 32), (64, 64), (64, 64), (40, 72), (128, 128), (64, 128), (33, 31)])
    if op == "attn":
        train = rng.random() < 0.5
        most = 38_000_000 // (h * (dk + dv)) // (2 if dtype == "f32" else 1)
        n = _log_int(rng, 64, min(200_000, most // 2 if train else most))
        return dict(op=op, train=train, n=n, b=min(n, _log_int(rng, 1, 256)), h=h, dk=dk, dv=dv,
                    times=rng.random() < 0.5, state=not train and rng.random() < 0.5, dtype=dtype)
    return dict(op=op, b=_log_int(rng, 1, max(1, 16_000_000 // (h * dk * dv))), h=h, dk=dk, dv=dv,
                times=rng.random() < 0.5, dtype=dtype)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        n, c = case["n"], case["c"]
        if case["train"]:  # x, dy -> dx; mean, rstd, the weight and its gradients
            return {"bytes": 3 * n * c * e + 8 * n + 12 * c, "flops": 14 * n * c}
        return {"bytes": 2 * n * c * e + 8 * n + 8 * c, "flops": 8 * n * c}
    if case["op"] == "rotary":
        values = case["n"] * (case["hq"] + case["hk"]) * case["d"]
        pairs = case["s0"] + case["s1"] + case["s2"]
        return {"bytes": 2 * values * e + 12 * case["n"] + 4 * pairs,
                "flops": case["n"] * pairs * (6 * (case["hq"] + case["hk"]) + 20)}
    h, dk, dv = case["h"], case["dk"], case["dv"]
    if case["op"] == "step":
        b = case["b"]
        return {"bytes": b * h * (8 * dk * dv + (2 * dk + 2 * dv) * e) + (12 * b if case["times"] else 0),
                "flops": 5 * b * h * dk * dv}
    n = case["n"]
    io = n * h * (2 * dk + 2 * dv) * e + (4 * n if case["times"] else 0)
    # the recurrence: a rank-one update and a product with the state per token
    flops = 4 * n * h * dk * dv
    if case["train"]:
        return {"bytes": io + n * h * (2 * dk + dv) * e, "flops": 3 * flops}
    states = 2 * case["b"] * h * dk * dv * 4 if case["state"] else 0
    return {"bytes": io + states, "flops": flops}


# ---------------------------------------------------------------- inputs
def _splits(n, b, g):
    """b sequences of different lengths, some of them perhaps empty, that make n tokens."""
    cuts = torch.sort(torch.randint(0, n + 1, (b - 1,), generator=g)).values
    return torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([n])]).to(torch.int32)


def prepare(case, seed):
    host = torch.Generator().manual_seed(int(seed))
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=gen)

    s = {"case": case}
    if case["op"] == "norm":
        n, c = case["n"], case["c"]
        # channels of different spread and place, as a convolution gives them
        s["x"] = (normal(n, c) * (0.5 + normal(c).abs()) + normal(c)).to(dt)
        s["weight"] = 1 + 0.2 * normal(c)
        s["bias"] = 0.2 * normal(c) if case["bias"] else None
        if case["train"]:
            s["dy"] = normal(n, c).to(dt)
            x = s["x"].float()  # the statistics that the forward pass left
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt(x.var(1, correction=0) + EPS)
        return s
    if case["op"] == "rotary":
        n = case["n"]
        s["q"], s["k"] = (normal(n, case["hq"], case["d"]).to(dt),
                          normal(n, case["hk"], case["d"]).to(dt))
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
    h, dk, dv = case["h"], case["dk"], case["dv"]
    n = case["b"] if case["op"] == "step" else case["n"]
    s["scale"] = dk ** -0.5
    s["q"], s["k"], s["v"] = (normal(n, h, dk).to(dt), normal(n, h, dk).to(dt),
                              normal(n, h, dv).to(dt))
    # from a fast head to a slow one; in the unit of the times, else per token
    fast, slow = (1 / 500, 1 / 20_000) if case["times"] else (1 / 8, 1 / 512)
    s["rates"] = fast * (slow / fast) ** (torch.arange(h, device=DEVICE) / max(1, h - 1))
    s["t"] = s["state"] = s["state_time"] = None
    if case["op"] == "step":
        s["state"] = 4 * normal(n, h, dk, dv)
        s["next_state"] = torch.empty_like(s["state"])
        s["next_time"] = None
        if case["times"]:
            s["state_time"] = torch.randint(0, 50_000, (n,), device=DEVICE, generator=gen).int()
            s["t"] = s["state_time"] + torch.randint(0, 500, (n,), device=DEVICE,
                                                     generator=gen).int()
            s["next_time"] = torch.empty_like(s["t"])
        return s
    s["splits"] = _splits(n, case["b"], host).to(DEVICE)
    if case["times"]:  # sorted over all sequences, so sorted in each
        s["t"] = torch.sort(torch.randint(50_000, 150_000, (n,), device=DEVICE,
                                          generator=gen)).values.int()
    if case["state"]:
        s["state"] = 4 * normal(case["b"], h, dk, dv)
        if case["times"]:
            s["state_time"] = torch.full((case["b"],), 49_000, device=DEVICE, dtype=torch.int32)
    if case["train"]:
        s["do"] = normal(n, h, dv).to(dt)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2012_01170_amd as sbc

    case = s["case"]
    if case["op"] == "norm":
        if case["train"]:
            return sbc.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"],
                                           need_dbias=case["bias"])
        return sbc.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=EPS)
    if case["op"] == "rotary":
        call = sbc.rotary_backward if case["train"] else sbc.rotary_forward
        return call(s["q"], s["k"], s["positions"], s["freqs"], s["sections"],
                    interleaved=case["interleaved"])
    if case["op"] == "step":
        return sbc.linear_attention_step(s["q"], s["k"], s["v"], s["rates"], s["state"], t=s["t"],
                                         state_time=s["state_time"], scale=s["scale"],
                                         out_state=s["next_state"], out_time=s["next_time"])
    if case["train"]:
        return sbc.linear_attention_backward(s["do"], s["q"], s["k"], s["v"], s["rates"],
                                             splits=s["splits"], t=s["t"], scale=s["scale"])
    return sbc.linear_attention_forward(s["q"], s["k"], s["v"], s["rates"], splits=s["splits"],
                                        t=s["t"], scale=s["scale"], state=s["state"],
                                        state_time=s["state_time"], return_state=case["state"])


def _run_plain(s):
    case = s["case"]
    if case["op"] == "norm":
        return _plain_norm_grad(s) if case["train"] else _plain_norm(s)
    if case["op"] == "rotary":
        return _plain_rotary(s)
    if case["op"] == "step":
        return _plain_step(s)
    return _plain_attn_grad(s) if case["train"] else _plain_attn(s)


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = torch.rsqrt((x * x).mean(1) + EPS)
    y = x * rstd[:, None] * s["weight"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["x"].dtype), mean, rstd


def _plain_norm_grad(s):
    dy = s["dy"].float()
    xn = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"]
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xn * (g * xn).mean(1, keepdim=True))
    return (dx.to(s["x"].dtype), (dy * xn).sum(0), dy.sum(0) if s["case"]["bias"] else None)


def _plain_turn(x, cos, sin, interleaved):
    m = cos.shape[-1]
    f = x.float()
    a, b = (f[..., 0:2 * m:2], f[..., 1:2 * m:2]) if interleaved else (f[..., :m], f[..., m:2 * m])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, f[..., 2 * m:]], -1).to(x.dtype)


def _plain_rotary(s):
    case = s["case"]
    s0, s1, s2 = s["sections"]
    p = s["positions"].float()
    angle = torch.cat([p[:, 0:1].expand(-1, s0), p[:, 1:2].expand(-1, s1),
                       p[:, 2:3].expand(-1, s2)], 1) * s["freqs"]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if case["train"]:
        sin = -sin
    return (_plain_turn(s["q"], cos, sin, case["interleaved"]),
            _plain_turn(s["k"], cos, sin, case["interleaved"]))


def _plain_step(s):
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if s["t"] is None:
        decay = torch.exp(-s["rates"])[None, :, None, None]
    else:
        gap = (s["t"] - s["state_time"]).float()
        decay = torch.exp(-s["rates"] * gap[:, None])[:, :, None, None]
    new = decay * s["state"] + k[..., :, None] * v[..., None, :]
    o = s["scale"] * (q[..., :, None] * new).sum(2)
    return o.to(s["q"].dtype), new, None if s["t"] is None else s["t"].clone()


# The attention in chunks of CHUNK tokens of one sequence: pairs in a chunk directly, pairs of
# chunks by the chunks' sums of k v^T (and q do^T), brought to the chunk's end (start).
def _plain_chunks(s):
    n, dev = s["q"].shape[0], s["q"].device
    sp = s["splits"].long()
    b = sp.shape[0] - 1
    count = (sp[1:] - sp[:-1] + CHUNK - 1) // CHUNK
    upto = torch.cumsum(count, 0)
    c = torch.arange(n // CHUNK + b, device=dev)  # no fewer than there are
    seq = torch.searchsorted(upto, c, right=True)
    there = seq < b
    seq = seq.clamp(max=b - 1)
    first = sp[seq] + (c - (upto - count)[seq]) * CHUNK
    token = first[:, None] + torch.arange(CHUNK, device=dev)
    ok = there[:, None] & (token < sp[seq + 1][:, None])
    token = torch.minimum(token, sp[seq + 1][:, None] - 1).clamp(0, n - 1)
    if s["t"] is None:  # the position in the sequence
        t = token - sp[seq][:, None]
    else:
        t = s["t"].long()[token]
    return {"seq": torch.where(there, seq, -1 - c), "token": token, "ok": ok, "t": t,
            "there": there, "splits": sp}


def _plain_load(x, ch):
    """[n, h, d] -> [h, chunks, CHUNK, d], zero where a chunk has no token."""
    return (x.float()[ch["token"]] * ch["ok"][..., None, None]).permute(2, 0, 1, 3).contiguous()


def _plain_store(x, ch, like):
    n = like.shape[0]
    out = torch.empty(n + 1, *like.shape[1:], dtype=like.dtype, device=like.device)
    out[torch.where(ch["ok"], ch["token"], n)] = x.permute(1, 2, 0, 3).to(like.dtype)
    return out[:n]  # the last row takes the places without a token


def _plain_decays(s, ch):
    r = s["rates"][:, None, None]
    t, ok = ch["t"], ch["ok"]
    start, end = t[:, 0], t[:, -1]  # places without a token repeat the last one's time
    gap = (t[:, :, None] - t[:, None, :]).float()
    lower = torch.ones(CHUNK, CHUNK, device=t.device, dtype=torch.bool).tril()
    pair = torch.where(lower, torch.exp(-r[..., None] * gap.clamp(min=0)), 0.0)
    head = torch.exp(-r * (t - start[:, None]).float())       # of a token from its chunk's start
    tail = torch.exp(-r * (end[:, None] - t).float()) * ok    # of a token to its chunk's end
    c = torch.arange(t.shape[0], device=t.device)
    before = (ch["seq"][:, None] == ch["seq"][None, :]) & (c[:, None] > c[None, :])
    far = (start[:, None] - end[None, :]).float()
    chunk = torch.where(before, torch.exp(-r * far.clamp(min=0)), 0.0)  # [h, chunk, earlier one]
    return {"gap": gap, "pair": pair, "head": head, "tail": tail, "chunk": chunk, "far": far}


def _plain_attn(s):
    ch = _plain_chunks(s)
    d = _plain_decays(s, ch)
    q, k, v = _plain_load(s["q"], ch), _plain_load(s["k"], ch), _plain_load(s["v"], ch)
    h, m, _, dk = q.shape
    dv = v.shape[-1]
    sums = torch.matmul((k * d["tail"][..., None]).transpose(2, 3).contiguous(), v)
    came = torch.matmul(d["chunk"], sums.view(h, m, dk * dv)).view(h, m, dk, dv)
    r = s["rates"][:, None]
    if s["state"] is not None:
        seq = ch["seq"].clamp(min=0)
        t0 = (torch.full((s["state"].shape[0],), -1, device=q.device) if s["t"] is None
              else s["state_time"].long())
        kept = torch.exp(-r * (ch["t"][:, 0] - t0[seq]).float()) * ch["there"]
        came = came + kept[..., None, None] * s["state"].transpose(0, 1)[:, seq]
    o = torch.matmul(torch.matmul(q, k.transpose(2, 3).contiguous()) * d["pair"], v)
    o = o + torch.matmul(q, came) * d["head"][..., None]
    o = _plain_store(o * s["scale"], ch, s["v"])
    if s["state"] is None:
        return o
    sp = ch["splits"]
    b = sp.shape[0] - 1
    empty = sp[1:] == sp[:-1]
    at = (sp[1:] - 1).clamp(min=0)
    last = at - sp[:-1] if s["t"] is None else s["t"].long()[at]
    last = torch.where(empty, t0, last)
    mine = torch.arange(b, device=q.device)[:, None] == ch["seq"][None, :]
    left = torch.exp(-r[..., None] * (last[:, None] - ch["t"][None, :, -1]).float().clamp(min=0))
    new = torch.matmul(torch.where(mine, left, 0.0), sums.view(h, m, dk * dv)).view(h, b, dk, dv)
    new = new + torch.exp(-r * (last - t0).float())[..., None, None] * s["state"].transpose(0, 1)
    return o, new.transpose(0, 1).contiguous(), None if s["t"] is None else last.int()


def _plain_attn_grad(s):
    ch = _plain_chunks(s)
    d = _plain_decays(s, ch)
    q, k = _plain_load(s["q"], ch), _plain_load(s["k"], ch)
    v, do = _plain_load(s["v"], ch), _plain_load(s["do"], ch) * s["scale"]
    h, m, _, dk = q.shape
    dv = v.shape[-1]
    kt = (k * d["tail"][..., None]).transpose(2, 3).contiguous()
    qh = (q * d["head"][..., None]).transpose(2, 3).contiguous()
    sums, back = torch.matmul(kt, v), torch.matmul(qh, do)  # [dk, dv] of every chunk
    flat = lambda x: x.view(h, m, dk * dv)  # noqa: E731
    came = torch.matmul(d["chunk"], flat(sums)).view(h, m, dk, dv)
    goes = torch.matmul(d["chunk"].transpose(1, 2).contiguous(), flat(back)).view(h, m, dk, dv)
    a = torch.matmul(q, k.transpose(2, 3).contiguous()) * d["pair"]
    g = torch.matmul(do, v.transpose(2, 3).contiguous())
    ag = a * g
    g = g * d["pair"]
    at, gt = a.transpose(2, 3).contiguous(), g.transpose(2, 3).contiguous()
    dq = torch.matmul(g, k) + d["head"][..., None] * torch.matmul(
        do, came.transpose(2, 3).contiguous())
    dk_ = torch.matmul(gt, q) + d["tail"][..., None] * torch.matmul(
        v, goes.transpose(2, 3).contiguous())
    dv_ = torch.matmul(at, do) + d["tail"][..., None] * torch.matmul(k, goes)
    # the rates: every pair's term times its gap, inside a chunk and between chunks
    since = (ch["t"] - ch["t"][:, :1]).float()
    until = (ch["t"][:, -1:] - ch["t"]).float()
    back1 = torch.matmul(qh * since[:, None, :], do)
    sums1 = torch.matmul(kt * until[:, None, :], v)
    over = lambda x, y: torch.matmul(flat(x), flat(y).transpose(1, 2).contiguous())  # noqa: E731
    between = d["chunk"] * (over(back1, sums) + over(back, sums1) + d["far"] * over(back, sums))
    drates = -(ag * d["gap"]).sum((1, 2, 3)) - between.sum((1, 2))
    return (_plain_store(dq, ch, s["q"]), _plain_store(dk_, ch, s["k"]),
            _plain_store(dv_, ch, s["v"]), drates)


# ---------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "rotary":
        return _exact_rotary(s)
    if case["op"] == "step":
        return _exact_step(s)
    return _exact_attn(s)


def _exact_norm(s):
    x, w = s["x"].double(), s["weight"].double()
    c = x.shape[1]
    if not s["case"]["train"]:
        mean = x.sum(1) / c
        var = ((x - mean[:, None]) ** 2).sum(1) / c
        y = (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * w
        return (y if s["bias"] is None else y + s["bias"].double()), mean, 1 / torch.sqrt(var + EPS)
    dy, r = s["dy"].double(), s["rstd"].double()[:, None]
    u = x - s["mean"].double()[:, None]
    g = dy * w * r
    # through x - mean and through the spread
    dx = g - u * r * r * ((g * u).sum(1, keepdim=True) / c)
    dx = dx - g.sum(1, keepdim=True) / c
    return dx, (dy * u * r).sum(0), dy.sum(0) if s["case"]["bias"] else None


def _exact_rotary(s):
    case = s["case"]
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(s["sections"])).to(DEVICE)
    angle = s["positions"].double()[:, axis] * s["freqs"].double()
    if case["train"]:
        angle = -angle
    m = axis.numel()
    i = torch.arange(m, device=DEVICE)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + m)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]
    out = []
    for x in (s["q"], s["k"]):
        x = x.double()
        z = torch.complex(x[..., first], x[..., second]) * unit
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_step(s):
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    gap = (torch.ones(q.shape[0], device=DEVICE) if s["t"] is None
           else s["t"].long() - s["state_time"].long()).double()
    keep = torch.exp(-gap[:, None] * s["rates"].double())
    new = torch.empty_like(s["state"], dtype=torch.float64)
    torch.mul(k.unsqueeze(3), v.unsqueeze(2), out=new)
    new += s["state"].double() * keep[:, :, None, None]
    o = torch.matmul(q.unsqueeze(2), new).squeeze(2) * s["scale"]
    return o, new, None if s["t"] is None else s["t"].long()


def _exact_attn(s):
    """Sequence by sequence, in blocks: forwards with the state, its derivative by the rates
    and the queries' gradient; backwards with the state's gradient."""
    case, step = s["case"], 512
    h, dk, dv = case["h"], case["dk"], case["dv"]
    splits = s["splits"].tolist()
    if sum(-(-(b - a) // step) for a, b in zip(splits, splits[1:])) > 1500:
        return None
    f = lambda x: x.double().transpose(0, 1).contiguous()  # noqa: E731
    q, k, v = f(s["q"]), f(s["k"]), f(s["v"])
    rate = s["rates"].double()[:, None]
    n = q.shape[1]
    time = torch.arange(n, device=DEVICE).double() if s["t"] is None else s["t"].double()
    T = lambda x: x.transpose(-1, -2).contiguous()  # noqa: E731
    train = case["train"]
    o = torch.zeros_like(v)
    if train:
        do = f(s["do"]) * s["scale"]
        dq, dk_, dv_ = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        drates = torch.zeros(h, dtype=torch.float64, device=DEVICE)
    states, times = [], []
    for b in range(len(splits) - 1):
        lo, hi = splits[b], splits[b + 1]
        if s["state"] is not None:
            S = s["state"][b].double()
            if s["t"] is None:
                now = torch.tensor(float(lo - 1), dtype=torch.float64, device=DEVICE)
            else:
                now = s["state_time"][b].double()
        else:
            S = torch.zeros(h, dk, dv, dtype=torch.float64, device=DEVICE)
            now = time[lo] if lo < hi else torch.zeros((), dtype=torch.float64, device=DEVICE)
        S1 = torch.zeros_like(S)
        blocks = [(i, min(i + step, hi)) for i in range(lo, hi, step)]
        for i, j in blocks:
            t = time[i:j]
            gap = (t[:, None] - t[None, :])
            D = torch.tril(torch.exp(-rate[..., None] * gap.clamp(min=0)))
            e = torch.exp(-rate * (t - now))[..., None]
            Q, K, V = q[:, i:j].contiguous(), k[:, i:j].contiguous(), v[:, i:j].contiguous()
            A = torch.matmul(Q, T(K)) * D
            if train:
                G = do[:, i:j].contiguous()
                B = torch.matmul(G, T(V))
                dq[:, i:j] = torch.matmul(B * D, K) + e * torch.matmul(G, T(S))
                grown = e * torch.matmul(Q, S1) - e * (t - now)[:, None] * torch.matmul(Q, S)
                drates += (grown * G).sum((1, 2)) - (A * B * gap).sum((1, 2))
            else:
                o[:, i:j] = torch.matmul(A, V) + e * torch.matmul(Q, S)
            over = torch.exp(-rate * (t[-1] - now))[..., None]
            w = torch.exp(-rate * (t[-1] - t))[..., None]
            S1 = over * (S1 - (t[-1] - now) * S) - torch.matmul(T(K * w * (t[-1] - t)[:, None]), V)
            S = over * S + torch.matmul(T(K * w), V)
            now = t[-1]
        states.append(S)
        times.append(now)
        if train and blocks:
            R = torch.zeros_like(S)
            now = time[hi - 1]
            for i, j in reversed(blocks):
                t = time[i:j]
                D = torch.tril(torch.exp(-rate[..., None] * (t[:, None] - t[None, :]).clamp(min=0)))
                Q, K, V = q[:, i:j].contiguous(), k[:, i:j].contiguous(), v[:, i:j].contiguous()
                G = do[:, i:j].contiguous()
                w = torch.exp(-rate * (now - t))[..., None]
                dk_[:, i:j] = torch.matmul(T(torch.matmul(G, T(V)) * D), Q) + w * torch.matmul(V, T(R))
                dv_[:, i:j] = torch.matmul(T(torch.matmul(Q, T(K)) * D), G) + w * torch.matmul(K, R)
                R = (torch.exp(-rate * (now - t[0]))[..., None] * R
                     + torch.matmul(T(Q * torch.exp(-rate * (t - t[0]))[..., None]), G))
                now = t[0]
    back = lambda x: x.transpose(0, 1)  # noqa: E731
    if train:
        return back(dq), back(dk_), back(dv_), drates
    o = back(o) * s["scale"]
    if s["state"] is None:
        return o
    return o, torch.stack(states), None if s["t"] is None else torch.stack(times).long()
