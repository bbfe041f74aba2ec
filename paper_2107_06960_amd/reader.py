"""A small decoder that reads a network's feature maps, as an example of the operators (``operators``) together.

A ``mafat.Network`` whose last layer is a linear 1x1 convolution of ``2 * kv_heads * head_dim`` channels leaves, for every
position of a frame, its key and its value side by side.  Rows of tokens, of any number of requests about those frames,
attend to them:

    h = h + delta                                   add_rms_norm: the sum, and its norm in 8 bits
    q = norm(h) Wq^T (+ the request's adapter)      linear8
    o = attention(q, keys, values of its frame)     cross_attention
    delta = norm(o) Wo^T (+ the request's adapter)  add_rms_norm, linear8

per layer, and a last norm.  Every layer reads the same keys and values, where the network left them.
"""
from __future__ import annotations

import torch

from . import operators as O


def to_f8_rows(w):
    """A float matrix as e4m3 rows and their scales (what linear8 takes as weights), once, when weights are loaded."""
    scale = w.abs().amax(1).float() / 448
    scale = torch.where(scale < 2.0 ** -100, torch.ones_like(scale), scale)
    return (w.float() / scale[:, None]).to(O.F8), scale


def draw_params(width, q_heads, head_dim, layers, seed=0, adapters=0, rank=8, device="cuda"):
    """Random weights of a Reader: a list of layers, and the last norm's gain."""
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

    return {"layers": [{"gain": gain(width), "q": linear(inner, width), "o_gain": gain(inner), "o": linear(width, inner)}
                       for _ in range(layers)], "gain": gain(width)}


class Reader:
    """Layers of cross attention from rows of tokens to the feature maps of a batch of frames."""

    def __init__(self, params, q_heads, kv_heads, head_dim, eps=1e-6):
        self.params, self.q_heads, self.kv_heads, self.head_dim, self.eps = params, q_heads, kv_heads, head_dim, eps

    def states(self, y):
        """Keys and values, [frames, positions, kv_heads, head_dim] each, in a network's output [frames, h, w, channels]."""
        frames, h, w, c = y.shape
        if c != 2 * self.kv_heads * self.head_dim:
            raise ValueError(f"the maps have {c} channels, not 2 * {self.kv_heads} * {self.head_dim}")
        kv = y.view(frames, h * w, 2, self.kv_heads, self.head_dim)
        return kv[:, :, 0], kv[:, :, 1]

    def run(self, tokens, y, q_offsets=None, row_adapter=None, k_lengths=None, key_mask=None):
        """tokens: bfloat16 [rows, width], as y has to be, frame by frame; q_offsets: int32 [frames + 1], the frames' rows (None: as many
        each); row_adapter: int32 [rows], the adapter of each row's request, for layers that have adapters (None: without
        them).  Returns the normed rows."""
        if row_adapter is not None and not any(p[i]["adapters"] for p in self.params["layers"] for i in ("q", "o")):
            raise ValueError("row_adapter names adapters, but no layer has any")
        k, v = self.states(y)
        rows, h, delta = tokens.shape[0], tokens, None

        def linear(x, scale, p):
            ad = p["adapters"] if row_adapter is not None else None
            return O.linear8(x, scale, p["w"], p["scale"], adapters=ad, row_adapter=row_adapter if ad is not None else None)

        for p in self.params["layers"]:
            if delta is None:
                _, x, scale = O.add_rms_norm(h, p["gain"], eps=self.eps)
            else:
                h, x, scale = O.add_rms_norm(delta, p["gain"], h, eps=self.eps)
            q = linear(x, scale, p["q"]).view(rows, self.q_heads, self.head_dim)
            o, _ = O.cross_attention(q, k, v, q_offsets=q_offsets, k_lengths=k_lengths, key_mask=key_mask)
            _, x, scale = O.add_rms_norm(o.view(rows, -1), p["o_gain"], eps=self.eps)
            delta = linear(x, scale, p["o"])
        return O.add_rms_norm(delta, self.params["gain"], h, eps=self.eps, out="bf16")[1]
