#!/usr/bin/env python3
"""A layer over a whole event stream on top of the event convolution: trained on a
recording, then run event by event.

    python examples/event_attention.py [--events 4096] [--steps 60]

The convolution sees an event's 3 x 3 pixels over a short window.  The layer that
follows mixes the whole past: layer norm, one projection to queries, keys and
values, rotary positions by time, row and column, linear attention whose heads
forget at learned rates, a projection back, and the residual.  The target is the
activity of the event's side of the sensor so far, which no window holds.

Gradients are the library's, put together by hand; torch does the projections,
the loss and Adam.  Afterwards the stream is fed in three parts: the first half
as a prompt that leaves its state, then one event at a time.
"""
import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2012_01170_amd as sbc  # noqa: E402

WIDTH = HEIGHT = 32
DURATION = 20_000
MEMORY = 2_000.0        # the target's decay time
HEADS, DIM, CHANNELS = 2, 32, 32
SECTIONS = (8, 4, 4)    # pairs of a head that turn with time, row and column


def make_events(n, seed, device):
    """A stream whose activity moves between the sensor's halves, and its target."""
    g = torch.Generator().manual_seed(seed)
    t = torch.sort(torch.randint(0, DURATION, (n,), generator=g)).values
    right = torch.rand(n, generator=g) < 0.5 + 0.45 * torch.sin(t / 900.0)
    px = torch.randint(0, WIDTH // 2, (n,), generator=g) + right * (WIDTH // 2)
    py = torch.randint(0, HEIGHT, (n,), generator=g)
    gap = (t[:, None] - t[None, :]).double()
    same = (right[:, None] == right[None, :]) & (torch.ones(n, n).tril(-1) > 0)
    target = torch.where(same, torch.exp(-gap.clamp(min=0) / MEMORY), 0.0).sum(1)
    target = (target / target.mean() - 1).float()
    i = lambda x: x.to(device, torch.int32)  # noqa: E731
    return i(px), i(py), i(t), target.to(device)[:, None]


class EventAttention:
    """The layer: parameters, forward, backward (into .grad), and a step of one event."""

    def __init__(self, device, seed=0):
        g = torch.Generator().manual_seed(seed)
        p = lambda *shape: torch.randn(*shape, generator=g).to(device)  # noqa: E731
        inner = HEADS * DIM
        self.norm_w, self.norm_b = torch.ones(CHANNELS, device=device), torch.zeros(CHANNELS,
                                                                                    device=device)
        self.w_qkv = p(CHANNELS, 3 * inner) / math.sqrt(CHANNELS)
        self.w_out = p(inner, CHANNELS) / math.sqrt(inner)
        self.log_rates = torch.log(torch.tensor([1 / 300.0, 1 / 1500.0], device=device))
        # a quarter turn between neighbouring pixels at most, and over 100 time units
        turn = [torch.logspace(0, -2, m) for m in SECTIONS]
        self.freqs = torch.cat([turn[0] * 0.015, turn[1] * 1.5, turn[2] * 1.5]).to(device)
        self.scale = 0.02 * DIM ** -0.5  # (some hundred events last)

    def parameters(self):
        return [self.norm_w, self.norm_b, self.w_qkv, self.w_out, self.log_rates]

    def _qkv(self, x, positions, stats):
        y, mean, rstd = sbc.layer_norm_forward(x, self.norm_w, self.norm_b, stats=stats)
        qkv = (y @ self.w_qkv).view(x.shape[0], 3, HEADS, DIM)
        q, k, v = qkv[:, 0], qkv[:, 1], qkv[:, 2]
        sbc.rotary_forward(q, k, positions, self.freqs, SECTIONS, inplace=True)
        return y, mean, rstd, q, k, v

    def forward(self, x, positions, t, state=None, state_time=None, return_state=False):
        y, mean, rstd, q, k, v = self._qkv(x, positions, stats=True)
        o = sbc.linear_attention_forward(q, k, v, self.log_rates.exp(), t=t, scale=self.scale,
                                         state=state, state_time=state_time,
                                         return_state=return_state)
        o, kept = (o[0], o[1:]) if return_state else (o, None)
        out = x + o.flatten(1) @ self.w_out
        self.saved = (x, y, mean, rstd, q, k, v, o, positions, t)
        return (out, *kept) if return_state else out

    def backward(self, dout):
        x, y, mean, rstd, q, k, v, o, positions, t = self.saved
        rates = self.log_rates.exp()
        self.w_out.grad = o.flatten(1).t() @ dout
        do = (dout @ self.w_out.t()).view_as(o)
        dqkv = torch.empty(x.shape[0], 3, HEADS, DIM, device=x.device)
        dq, dk, dqkv[:, 2], drates = sbc.linear_attention_backward(do, q, k, v, rates, t=t,
                                                                   scale=self.scale)
        self.log_rates.grad = drates * rates
        dqkv[:, 0], dqkv[:, 1] = sbc.rotary_backward(dq, dk, positions, self.freqs, SECTIONS,
                                                     inplace=True)
        dqkv = dqkv.flatten(1)
        self.w_qkv.grad = y.t() @ dqkv
        dx, self.norm_w.grad, self.norm_b.grad = sbc.layer_norm_backward(
            dqkv @ self.w_qkv.t(), x, self.norm_w, mean, rstd)
        return dx + dout

    def step(self, x, positions, t, state, state_time):
        """One event: its output, the state (updated in place) and its time."""
        _, _, _, q, k, v = self._qkv(x, positions, stats=False)
        o, state, state_time = sbc.linear_attention_step(
            q, k, v, self.log_rates.exp(), state, t=t, state_time=state_time, scale=self.scale,
            out_state=state)
        return x + o.flatten(1) @ self.w_out, state, state_time


def main(events=4096, steps=60, seed=0, log=print):
    dev = torch.device("cuda:0")
    px, py, t, target = make_events(events, seed, dev)
    positions = torch.stack([t, py, px], 1)
    # the convolution's part: neighbours and their transpose, features from the polarity
    csr, csc = sbc.neighbour_search_events_csc(px, py, t, WIDTH, HEIGHT, 1000)
    geometry = sbc.Geometry("event8", tau=500.0, px=px, py=py, t=t)
    g = torch.Generator().manual_seed(seed + 1)
    F = torch.randn(events, 8, generator=g).to(dev)
    side = torch.where(px >= WIDTH // 2, 1.0, -1.0)
    W = (0.3 * torch.randn(8, 8, CHANNELS, generator=g)).to(dev)
    embed = torch.randn(1, CHANNELS, generator=g).to(dev)
    layer = EventAttention(dev, seed)
    w_read = (torch.randn(CHANNELS, 1, generator=g) / math.sqrt(CHANNELS)).to(dev)
    params = [W, embed, w_read, *layer.parameters()]
    adam = torch.optim.Adam(params, lr=5e-3)

    def features():
        return sbc.conv_forward(csr, F, W, geometry=geometry) + side[:, None] * embed

    losses = []
    for i in range(steps):
        x = features()
        out = layer.forward(x, positions, t)
        error = out @ w_read - target
        losses.append(float((error * error).mean()))
        derr = 2 * error / events
        w_read.grad = out.t() @ derr
        dx = layer.backward(derr @ w_read.t())
        embed.grad = (side[:, None] * dx).sum(0, keepdim=True)
        W.grad = sbc.conv_backward(csr, csc, F, W, dx, geometry=geometry, need_dF=False)[1]
        adam.step()
        if i % 10 == 0 or i == steps - 1:
            log(f"step {i:3d}  loss {losses[-1]:.4f}  memory of the heads "
                + ", ".join(f"{1 / r:.0f}" for r in layer.log_rates.exp().tolist()))

    # deployment: a prompt, then event by event
    x = features()
    whole = layer.forward(x, positions, t)
    half = events // 2
    first, state, time = layer.forward(x[:half], positions[:half], t[:half], return_state=True)
    worst = float((first - whole[:half]).abs().max())
    for i in range(half, min(events, half + 64)):
        out, state, time = layer.step(x[i:i + 1], positions[i:i + 1], t[i:i + 1], state, time)
        worst = max(worst, float((out - whole[i:i + 1]).abs().max()))
    worst /= float(whole.abs().max())
    log(f"event by event against the whole stream: {worst:.1e} of the largest output")
    return losses, worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--events", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    main(a.events, a.steps)
