"""A small decoder that reads a network's feature maps, as an example of the operators (``operators``) together.

A ``mafat.Network`` whose last layer is a linear 1x1 convolution of ``2 * kv_heads * head_dim`` channels leaves, for every
position of a frame, its key and its value side by side.  Rows of tokens, of any number of requests about those frames,
attend to them:

    h = h + delta                                   add_rms_norm: the sum, and its norm in 8 bits
    q = norm(h) Wq^T (+ the request's adapter)      linear8
    o = attention(q, keys, values of its frame)     cross_attention
    delta = norm(o) Wo^T (+ the request's adapter)  add_rms_norm, linear8

per layer, and a last norm.  Every layer reads the same keys and values, where the network left them.

A layer may first mix the tokens of each request, in order, by a memory of constant size that the request keeps:

    q, k, v, g = norm(h) Wm^T                       add_rms_norm, linear8
    q, k turned by the tokens' positions            rotary, in place
    o = linear attention with decays                decay_attention, and the request's state after it
    delta = (norm by head(o) * silu(g)) Wn^T        block_norm into 8 bits, linear8
    h = h + scale * norm(delta), and its norm       block_norm, for the layer's own query projection
"""
from __future__ import annotations

import torch

from . import operators as O


def to_f8_rows(w):
    """A float matrix as e4m3 rows and their scales (what linear8 takes as weights), once, when weights are loaded."""
    scale = w.abs().amax(1).float() / 448
    scale = torch.where(scale < 2.0 ** -100, torch.ones_like(scale), scale)
    return (w.float() / scale[:, None]).to(O.F8), scale


def draw_params(width, q_heads, head_dim, layers, seed=0, adapters=0, rank=8, device="cuda", mix_heads=0, mix_dim=0):
    """Random weights of a Reader: a list of layers, and the last norm's gain.  With mix_heads heads of mix_dim, every layer
    mixes the requests' tokens first."""
    gen = torch.Generator().manual_seed(seed)
    inner = q_heads * head_dim

    def randn(*shape):
        return torch.randn(shape, generator=gen)

    def linear(n, k):
        d = dict(zip(("w", "scale"), (t.to(device) for t in to_f8_rows(randn(n, k) / k ** 0.5))))
        d["adapters"] = None
        if adapters:
            d["adapters"] = ((randn(adapters, rank, k) / k ** 0.5).bfloat16().to(device),
                             (0.3 * randn(adapters, n, rank) / rank ** 0.5).bfloat16().to(device),
                             (0.5 + torch.rand(adapters, generator=gen)).to(device))
        return d

    def gain(n):
        return (1 + 0.1 * randn(n)).to(device)

    def mix():
        n = mix_heads * mix_dim
        # heads that forget within some ten to some thousand tokens
        decay = torch.log1p(-2.0 ** -(4 + 6 * torch.arange(mix_heads) / max(mix_heads - 1, 1)))
        return {"gain": gain(width), "qkvg": linear(4 * n, width), "log_decay": decay.to(device), "o_gain": gain(n),
                "o": linear(width, n), "after_gain": gain(width), "scale": (0.5 + 0.1 * randn(width)).to(device)}

    params = {"layers": [{"gain": gain(width), "q": linear(inner, width), "o_gain": gain(inner), "o": linear(width, inner)}
                         for _ in range(layers)], "gain": gain(width)}
    if mix_heads:
        for p in params["layers"]:
            p["mix"] = mix()
    return params


class Reader:
    """Layers of cross attention from rows of tokens to the feature maps of a batch of frames."""

    def __init__(self, params, q_heads, kv_heads, head_dim, eps=1e-6, mix_heads=0, mix_dim=0):
        self.params, self.q_heads, self.kv_heads, self.head_dim, self.eps = params, q_heads, kv_heads, head_dim, eps
        self.mix_heads, self.mix_dim = mix_heads, mix_dim
        # Formed on the host and there when this returns: a run may be recorded by a graph, or be on any stream.
        self.turns = O.rotary_turns(mix_dim // 2, device="cpu").to(params["gain"].device) if mix_heads else None

    def states(self, y):
        """Keys and values, [frames, positions, kv_heads, head_dim] each, in a network's output [frames, h, w, channels]."""
        frames, h, w, c = y.shape
        if c != 2 * self.kv_heads * self.head_dim:
            raise ValueError(f"the maps have {c} channels, not 2 * {self.kv_heads} * {self.head_dim}")
        kv = y.view(frames, h * w, 2, self.kv_heads, self.head_dim)
        return kv[:, :, 0], kv[:, :, 1]

    def memory(self, slots, device="cuda"):
        """Empty memories of `slots` requests for layers that mix: float32 [layers, slots, mix_heads, mix_dim, mix_dim]."""
        return torch.zeros(len(self.params["layers"]), slots, self.mix_heads, self.mix_dim, self.mix_dim, device=device)

    def _mix(self, p, h, x, scale, next_gain, positions, offsets, states, slots):
        """The sum after the tokens of each request are mixed, and its norm in 8 bits with `next_gain`."""
        rows, heads, dim = h.shape[0], self.mix_heads, self.mix_dim
        n = heads * dim
        all_ = O.linear8(x, scale, p["qkvg"]["w"], p["qkvg"]["scale"])
        q, k, v = (all_[:, i * n:(i + 1) * n].view(rows, heads, dim) for i in range(3))
        O.rotary(q, positions, self.turns, k=k, in_place=True)
        o = O.decay_attention(q, k, v, p["log_decay"], states=states, slots=slots, offsets=offsets)
        _, x, scale = O.block_norm(o.view(rows, n), after_gain=p["o_gain"], groups=heads, gate=all_[:, 3 * n:], before=False,
                                   eps=self.eps)
        delta = O.linear8(x, scale, p["o"]["w"], p["o"]["scale"])
        return O.block_norm(delta, after_gain=p["after_gain"], scale=p["scale"], residual=h, before_gain=next_gain, eps=self.eps)

    def run(self, tokens, y, q_offsets=None, row_adapter=None, k_lengths=None, key_mask=None, positions=None, offsets=None,
            memory=None, slots=None):
        """tokens: bfloat16 [rows, width], as y has to be, frame by frame; q_offsets: int32 [frames + 1], the frames' rows (None: as many
        each); row_adapter: int32 [rows], the adapter of each row's request, for layers that have adapters (None: without
        them).  For layers that mix: positions: int32 [rows], of the tokens in their requests; offsets: int32 [requests + 1],
        the requests' rows (None: as many each, of as many requests as slots or else memory has places, which have to be given
        then); memory: what memory() gives, updated in place (None: every request starts without one, and none is kept); slots:
        int32 [requests], each request's place in it (None: request i has place i).
        Returns the normed rows."""
        if row_adapter is not None and not any(p[i]["adapters"] for p in self.params["layers"] for i in ("q", "o")):
            raise ValueError("row_adapter names adapters, but no layer has any")
        mixes = any("mix" in p for p in self.params["layers"])
        if mixes and (positions is None or not self.mix_heads):
            raise ValueError("layers that mix need positions, and a reader with mix_heads and mix_dim")
        if mixes and offsets is None and memory is None:
            raise ValueError("layers that mix need offsets, or a memory, to tell the requests' rows apart")
        if not mixes and any(t is not None for t in (positions, offsets, memory, slots)):
            raise ValueError("positions, offsets, memory and slots are for layers that mix, but no layer does")
        k, v = self.states(y)
        rows, h, delta = tokens.shape[0], tokens, None

        def linear(x, scale, p):
            ad = p["adapters"] if row_adapter is not None else None
            return O.linear8(x, scale, p["w"], p["scale"], adapters=ad, row_adapter=row_adapter if ad is not None else None)

        for i, p in enumerate(self.params["layers"]):
            gain = p["mix"]["gain"] if "mix" in p else p["gain"]
            if delta is None:
                _, x, scale = O.add_rms_norm(h, gain, eps=self.eps)
            else:
                h, x, scale = O.add_rms_norm(delta, gain, h, eps=self.eps)
            if "mix" in p:
                h, x, scale = self._mix(p["mix"], h, x, scale, p["gain"], positions, offsets,
                                        None if memory is None else memory[i], slots)
            q = linear(x, scale, p["q"]).view(rows, self.q_heads, self.head_dim)
            o, _ = O.cross_attention(q, k, v, q_offsets=q_offsets, k_lengths=k_lengths, key_mask=key_mask)
            _, x, scale = O.add_rms_norm(o.view(rows, -1), p["o_gain"], eps=self.eps)
            delta = linear(x, scale, p["o"])
        return O.add_rms_norm(delta, self.params["gain"], h, eps=self.eps, out="bf16")[1]
