"""The operators of a reader's tokens among themselves: rotary positions, linear attention with a decay for each head whose
state a request keeps, and the norms after and before a block with its gate and residual scale.

Sizes: the model widths, head counts and head sizes that the reader's other operators are measured at, feature maps of
19x19 positions as the YOLOv2 stack gives them, odd and ragged ones among them.

A case: ``op`` and its sizes.
  rotary: rows, hq and hk heads of queries and keys (hk 0: queries alone), d, rot (how many of d turn), axes of a position,
          layout ("half", "interleaved"), stretch (factor by which positions are longer than trained ones), span (largest
          position), dtype.
  block:  rows, cols, dtype, after (whether the block's output is normed, in `groups` equal parts of a row), gate ("none",
          "silu", "sigmoid"), scaled (a residual scale for each column), residual, before (the next block's norm), out
          ("f8", "bf16", "f32").
  decay:  requests, rows (tokens of all requests together), hq and hkv heads, dk and dv, dtype, ragged (requests have
          different numbers of tokens, none among them), by_row (a decay for each token and head, or one for each head).
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": F8}
SIZE = {"f32": 4, "bf16": 2, "f8": 1}
F8_MAX = 448.0
EPS = 1e-6


def _rotary(rows, hq, hk, d, rot, axes=1, layout="half", stretch=1.0, span=4096, dtype="bf16", name=None):
    c = {"op": "rotary", "rows": rows, "hq": hq, "hk": hk, "d": d, "rot": rot, "axes": axes, "layout": layout,
         "stretch": stretch, "span": span, "dtype": dtype}
    return dict(c, name=name) if name else c


def _block(rows, cols, dtype="bf16", after=True, groups=1, gate="none", scaled=True, residual=True, before=True, out="f8",
           name=None):
    c = {"op": "block", "rows": rows, "cols": cols, "dtype": dtype, "after": after, "groups": groups, "gate": gate,
         "scaled": scaled, "residual": residual, "before": before, "out": out}
    return dict(c, name=name) if name else c


def _decay(requests, rows, hq, hkv, dk, dv, dtype="bf16", ragged=False, by_row=False, name=None):
    c = {"op": "decay", "requests": requests, "rows": rows, "hq": hq, "hkv": hkv, "dk": dk, "dv": dv, "dtype": dtype,
         "ragged": ragged, "by_row": by_row}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One decode step of four requests: a launch's latency.
        _rotary(4, 8, 2, 64, 64, name="rotary_step"),
        # Keys of three frames' 19x19 maps by their row and column, part of an odd-sized head, full precision.
        _rotary(1083, 0, 6, 80, 48, axes=2, layout="interleaved", span=19, dtype="f32", name="rotary_map_f32"),
        # Prompts of many requests far into long contexts: bound by memory.
        _rotary(16384, 32, 8, 128, 128, stretch=16.0, span=1 << 20, name="rotary_prompts"),
        # Between two blocks in one decode step of four requests: a launch's latency.
        _block(4, 1024, name="block_step"),
        # The output of a prompt's heads, normed by head and gated, into the 8 bits that a projection takes.
        _block(4096, 2048, groups=16, gate="silu", scaled=False, residual=False, before=False, name="block_heads"),
        # An odd width in full precision.
        _block(1083, 1001, "f32", gate="sigmoid", out="f32", name="block_odd_f32"),
        # Between two blocks, prompts of many requests: bound by memory.
        _block(16384, 4096, name="block_prompts"),
        # One token of one request.
        _decay(1, 1, 8, 8, 64, 64, name="decay_token"),
        # A decode step of 64 requests: every state is read and written once.
        _decay(64, 64, 16, 16, 128, 128, name="decay_step"),
        # Prompts of eight requests of different lengths: the largest product.
        _decay(8, 16384, 16, 16, 128, 128, ragged=True, name="decay_prompts"),
        # One long prompt, few heads that pairs of query heads share, a decay for each token: a long axis for few heads.
        _decay(1, 65536, 8, 4, 128, 128, by_row=True, name="decay_long"),
        # Ragged prompts in float32 with odd head sizes.
        _decay(3, 397, 6, 3, 80, 48, "f32", ragged=True, by_row=True, name="decay_odd_f32"),
    ]


def draw(rng):
    """One more case of the ranges above."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    for _ in range(1000):
        op = rng.choice(["rotary", "block", "decay", "decay"])
        if op == "rotary":
            d = rng.choice([32, 64, 64, 128, 128, 256, 40, 80, 96, 2 * log(8, 128)])
            rot = rng.choice([d, d, d // 2 // 2 * 2, 2 * rng.randint(1, d // 2)])
            hk = rng.choice([0, 1, 2, 4, 8])
            case = _rotary(log(1, 16384), rng.choice([hk * rng.choice([1, 2, 4]), log(1, 64)]) if hk else log(1, 64), hk, d, rot,
                           rng.choice([1, 1, 2, 3]), rng.choice(["half", "interleaved"]), rng.choice([1.0, 1.0, 4.0, 32.0]),
                           log(16, 1 << 22), rng.choice(["bf16", "bf16", "f32"]))
        elif op == "block":
            dtype = rng.choice(["bf16", "bf16", "f32"])
            groups = rng.choice([1, 1, 4, 8, 16, 32])
            cols = rng.choice([log(64, 8192), 8 * log(8, 1024), rng.choice([256, 512, 1024, 2048, 4096])])
            if groups > 1:
                cols = groups * rng.choice([64, 128, 256, log(16, 256)])
            residual = rng.random() < 0.7
            case = _block(log(1, 16384), cols, dtype, rng.random() < 0.8, groups, rng.choice(["none", "none", "silu", "sigmoid"]),
                          rng.random() < 0.5, residual, rng.random() < (0.8 if residual else 0.3),
                          rng.choice(["f8", "f8", dtype]))
        else:
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            hkv = rng.choice([1, 2, 3, 4, 8, 16])
            dk, dv = (rng.choice([32, 64, 64, 128, 128, 128, 256, 40, 80, 96, log(16, 256)]) for _ in range(2))
            if rng.random() < 0.6:
                dv = dk
            requests = rng.choice([1, log(1, 16), log(1, 256)])
            rows = rng.choice([requests, log(requests, 16 * requests), log(requests, 65536)])
            case = _decay(requests, rows, hkv * rng.choice([1, 1, 2, 4]), hkv, dk, dv, dtype, rows > 1 and rng.random() < 0.5,
                          rng.random() < 0.5)
            # the plain form pads every request to the longest and holds a state for every 64 tokens
            if requests * rows * (1 if case["ragged"] else 1 / requests) * hkv * max(dk * dv / 64, 256) > 2 ** 31:
                continue
        w = work(case)
        # no more than the largest listed case of the same operator (float32 products run at a fraction of the rate)
        most = {"rotary": (3.4e8, 1e12), "block": (4.7e8, 1e12), "decay": (2.8e8, 1.8e10)}[op]
        if op == "decay" and case["dtype"] == "f32":
            most = (2.8e8, 4e9)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return case
    raise RuntimeError("no case drawn")


def work(case):
    """Each input once and each output once."""
    c = case
    if c["op"] == "rotary":
        values = c["rows"] * (c["hq"] + c["hk"]) * c["d"]
        bytes_ = 2 * values * SIZE[c["dtype"]] + 4 * c["rows"] * c["axes"] + 4 * c["axes"] * c["rot"]
        return {"bytes": bytes_, "flops": 3 * c["rows"] * (c["hq"] + c["hk"]) * c["rot"]}
    if c["op"] == "block":
        size = SIZE[c["dtype"]]
        a_row = c["cols"] * (size * (1 + (c["gate"] != "none") + 2 * c["residual"]) + SIZE[c["out"]])
        a_row += 4 if c["out"] == "f8" else 0
        return {"bytes": c["rows"] * a_row + 4 * c["cols"] * (c["after"] + c["scaled"] + c["before"]),
                "flops": c["rows"] * c["cols"] * (4 * c["after"] + 4 * c["before"] + 6 * (c["gate"] != "none") + 2)}
    size = SIZE[c["dtype"]]
    states = min(c["requests"], c["rows"]) * c["hkv"] * c["dk"] * c["dv"]
    bytes_ = c["rows"] * (c["hq"] + c["hkv"]) * (c["dk"] + c["dv"]) * size + 8 * states
    bytes_ += 4 * c["hkv"] * (c["rows"] if c["by_row"] else 1)
    return {"bytes": bytes_, "flops": 2 * c["rows"] * (c["hq"] + c["hkv"]) * c["dk"] * c["dv"]}


def prepare(case, seed):
    """Activations, positions and states on the GPU, as the layers and steps before leave them."""
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)

    dt = DTYPES[c["dtype"]]
    if c["op"] == "rotary":
        # queries and keys side by side in the rows of one projection
        x = (1.5 * randn(c["rows"], c["hq"] + c["hk"], c["d"])).to(dt)
        pairs, stretch = c["rot"] // 2, c["stretch"]
        i = torch.arange(pairs, device="cuda", dtype=torch.float64)
        freq = 10000.0 ** (-i / pairs)
        # frequencies that turn seldom within trained lengths are stretched, those that turn often are kept
        keep = ((freq * 4096 / (2 * math.pi) - 1) / 31).clamp(0, 1)
        turns = freq * (keep + (1 - keep) / stretch) / (2 * math.pi)
        # pair i belongs to axis i modulo axes
        axis = torch.arange(c["axes"], device="cuda")[:, None] == torch.arange(pairs, device="cuda") % c["axes"]
        q, k = (x[:, :c["hq"]], x[:, c["hq"]:]) if c["hq"] and c["hk"] else (x, None)
        return dict(c, q=q, k_=k, turns=turns * axis, magnitude=0.1 * math.log(stretch) + 1,
                    positions=ints(0, c["span"], c["rows"], c["axes"]))
    if c["op"] == "block":
        rows, cols = c["rows"], c["cols"]
        wide = torch.exp(0.5 * randn(cols))  # some channels are larger than others
        return dict(c, x=(randn(rows, cols) * wide).to(dt), gate_=randn(rows, cols).to(dt) if c["gate"] != "none" else None,
                    after_gain=1 + 0.2 * randn(cols) if c["after"] else None,
                    before_gain=1 + 0.2 * randn(cols) if c["before"] else None,
                    scale_=0.5 + 0.1 * randn(cols) if c["scaled"] else None,
                    residual_=(2 * randn(rows, cols) * wide).to(dt) if c["residual"] else None)
    n, rows, hkv = c["requests"], c["rows"], c["hkv"]
    s = dict(c, q=randn(rows, c["hq"], c["dk"]).to(dt), k=randn(rows, hkv, c["dk"]).to(dt), v=randn(rows, hkv, c["dv"]).to(dt),
             offsets=None, scale=c["dk"] ** -0.5)
    if c["ragged"]:
        cut = ints(0, rows + 1, n - 1)
        ends = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        s["offsets"] = torch.sort(torch.cat([ends, cut])).values.to(torch.int32)
    elif rows % n:
        s["offsets"] = (torch.arange(n + 1, device="cuda") * rows // n).to(torch.int32)  # as many each, but for the rest
    # heads forget within some ten to some thousand tokens
    rate = 2.0 ** -(3 + 8 * torch.rand(hkv, generator=gen, device="cuda"))
    s["log_decay"] = -rate * torch.nn.functional.softplus(2 * randn(rows, hkv)) if c["by_row"] else -rate
    # the requests' states anywhere in a pool with room for a few more
    s["states"] = 3 * randn(n + 3, hkv, c["dk"], c["dv"])
    s["slots"] = torch.randperm(n + 3, generator=gen, device="cuda")[:n].to(torch.int32)
    return s


def run(state):
    s = state
    if own:
        from paper_2107_06960_amd import operators as O
        if s["op"] == "rotary":
            q, k = O.rotary(s["q"], s["positions"], s["turns"], k=s["k_"], interleaved=s["layout"] == "interleaved",
                            magnitude=s["magnitude"])
            return {"q": q, "k": k}
        if s["op"] == "block":
            total, y, scale = O.block_norm(s["x"], after=s["after"], after_gain=s["after_gain"], groups=s["groups"],
                                           gate=s["gate_"], act="silu" if s["gate"] == "none" else s["gate"],
                                           scale=s["scale_"], residual=s["residual_"], before=s["before"],
                                           before_gain=s["before_gain"], eps=EPS, out=s["out"])
            return {"sum": total, "y": y, "scale": scale}
        y = O.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], states=s["states"], slots=s["slots"],
                              offsets=s["offsets"], scale=s["scale"])
        return {"y": y, "states": s["states"]}
    return {"rotary": _plain_rotary, "block": _plain_block, "decay": _plain_decay}[s["op"]](s)


def _plain_rotary(s):
    angle = 2 * math.pi * (s["positions"].double() @ s["turns"])
    cos, sin = (s["magnitude"] * angle.cos()).float()[:, None], (s["magnitude"] * angle.sin()).float()[:, None]
    rot = s["rot"]

    def turned(x):
        f = x[..., :rot].float()
        a, b = (f[..., 0::2], f[..., 1::2]) if s["layout"] == "interleaved" else (f[..., :rot // 2], f[..., rot // 2:])
        a, b = a * cos - b * sin, b * cos + a * sin
        f = torch.stack([a, b], -1).flatten(-2) if s["layout"] == "interleaved" else torch.cat([a, b], -1)
        return torch.cat([f.to(x.dtype), x[..., rot:]], -1)

    return {"q": turned(s["q"]), "k": None if s["k_"] is None else turned(s["k_"])}


def _plain_block(s):
    u = s["x"].float()
    if s["after"]:
        parts = u.reshape(s["rows"], s["groups"], -1)
        u = (parts * torch.rsqrt((parts * parts).mean(-1, keepdim=True) + EPS)).reshape(u.shape) * s["after_gain"]
    if s["gate"] != "none":
        g = s["gate_"].float()
        u = u * ((g if s["gate"] == "silu" else 1) / (1 + torch.exp(-g)))
    if s["scaled"]:
        u = u * s["scale_"]
    total = None
    if s["residual"]:
        u = u + s["residual_"].float()
        total = u.to(s["x"].dtype)
    if s["before"]:
        u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * s["before_gain"]
    if s["out"] != "f8":
        return {"sum": total, "y": u.to(DTYPES[s["out"]]), "scale": None}
    most = u.abs().amax(-1)
    scale = torch.where(most == 0, 1.0, most / F8_MAX)
    return {"sum": total, "y": (u / scale[:, None]).to(F8), "scale": scale}


def _requests_rows(s):
    """Row numbers of each request's tokens, padded to the longest, and which of them are there."""
    n, rows, dev = s["requests"], s["rows"], s["q"].device
    if s["offsets"] is None:
        at = torch.arange(rows, device=dev).reshape(n, rows // n)
        return at, torch.ones_like(at, dtype=torch.bool)
    off = s["offsets"].long()
    at = off[:-1, None] + torch.arange(int((off[1:] - off[:-1]).max()), device=dev)
    return at.clamp(max=rows - 1), at < off[1:, None]


def _plain_decay(s):
    at, there = _requests_rows(s)
    n, t = at.shape
    hkv, dk, dv = s["hkv"], s["dk"], s["dv"]
    g = s["hq"] // hkv
    step = min(64, t)  # tokens of a chunk
    m = -(-t // step)
    pad = m * step - t

    def chunks(x):
        """[rows, heads, ...] -> [requests, heads, chunks, step, ...], zeros where no token is."""
        x = torch.where(there.reshape(n, t, *[1] * (x.dim() - 1)), x[at], 0)
        x = torch.cat([x, x.new_zeros(n, pad, *x.shape[2:])], 1).reshape(n, m, step, *x.shape[2:])
        return x.movedim(3, 1).contiguous()

    q, k, v = chunks(s["q"].float()), chunks(s["k"].float()), chunks(s["v"].float())
    decay = s["log_decay"].double()
    c = chunks(decay if s["by_row"] else decay.expand(s["rows"], hkv)).cumsum(-1)  # of the chunk's tokens so far
    q = q.reshape(n, hkv, g, m, step, dk)
    # within the chunks
    inside = torch.exp((c[..., :, None] - c[..., None, :]).masked_fill_(
        ~torch.ones(step, step, dtype=torch.bool, device=q.device).tril(), -math.inf)).float()
    y = ((q @ k.transpose(-1, -2).contiguous()[:, :, None]) * inside[:, :, None]) @ v[:, :, None]
    # what every chunk adds to the state, and the states ahead of every chunk and after the last
    kv = (k * torch.exp(c[..., -1:] - c).float()[..., None]).transpose(-1, -2).contiguous() @ v
    upto = torch.cat([c.new_zeros(n, hkv, 1), c[..., -1].cumsum(-1)], -1)
    before = torch.arange(m, device=q.device) < torch.arange(m + 1, device=q.device)[:, None]
    across = torch.exp((upto[..., :, None] - upto[..., None, 1:]).masked_fill_(~before, -math.inf)).float()
    slots = s["slots"].long()
    states = (across @ kv.reshape(n, hkv, m, dk * dv)).reshape(n, hkv, m + 1, dk, dv)
    states = states + torch.exp(upto).float()[..., None, None] * s["states"][slots][:, :, None]
    y = y + torch.exp(c).float()[:, :, None, ..., None] * (q @ states[:, :, None, :-1])
    s["states"][slots] = states[:, :, -1]
    y = (s["scale"] * y).reshape(n, hkv * g, m * step, dv)[:, :, :t].transpose(1, 2)
    return {"y": y[there].to(s["q"].dtype), "states": s["states"]}


def exact(case, seed):
    """The operators in float64, before any rounding of the outputs (8-bit values: what they stand for before they are
    rounded to 8 bits)."""
    s = prepare(case, seed)
    if s["op"] == "rotary":
        i = torch.arange(s["rot"] // 2, device="cuda")
        first = 2 * i if s["layout"] == "interleaved" else i
        second = first + 1 if s["layout"] == "interleaved" else i + s["rot"] // 2
        turns = sum(s["positions"][:, a, None].double() * s["turns"][a] for a in range(s["axes"]))
        by = torch.polar(torch.full_like(turns, s["magnitude"]), 2 * math.pi * (turns - turns.round()))[:, None]

        def turned(x):
            y = x.double()
            z = torch.complex(y[..., first], y[..., second]) * by
            y[..., first], y[..., second] = z.real, z.imag
            return y

        return {"q": turned(s["q"]), "k": None if s["k_"] is None else turned(s["k_"])}
    if s["op"] == "block":
        u = s["x"].double()
        if s["after"]:
            parts = u.reshape(-1, s["cols"] // s["groups"])
            u = (parts / (parts.square().sum(1, keepdim=True) / parts.shape[1] + EPS).sqrt()).reshape(u.shape)
            u = u * s["after_gain"].double()
        if s["gate"] != "none":
            g = s["gate_"].double()
            u = u * torch.sigmoid(g) * (g if s["gate"] == "silu" else 1.0)
        if s["scaled"]:
            u = u * s["scale_"].double()
        h = u + s["residual_"].double() if s["residual"] else u
        y = h
        if s["before"]:
            y = h / (h.square().sum(-1, keepdim=True) / h.shape[1] + EPS).sqrt() * s["before_gain"].double()
        total = h if s["residual"] else None
        if s["out"] != "f8":
            return {"sum": total, "y": y, "scale": None}
        scale = y.abs().amax(-1) / F8_MAX
        scale[scale == 0] = 1
        return {"sum": total, "y": y / scale[:, None], "scale": scale}
    # token after token, all requests at once
    n, rows = s["requests"], s["rows"]
    off = [i * rows // n for i in range(n + 1)] if s["offsets"] is None else s["offsets"].tolist()
    lengths = [b - a for a, b in zip(off, off[1:])]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    a = s["log_decay"].double().exp()
    slots = s["slots"].tolist()
    states = s["states"].double()
    y = torch.zeros(rows, s["hq"], s["dv"], dtype=torch.float64, device="cuda")
    order = sorted(range(n), key=lambda i: -lengths[i])
    mine = states[[slots[i] for i in order]]  # longest first: after t tokens a leading part of them goes on
    first = torch.tensor([off[i] for i in order], device="cuda")
    q = q.reshape(rows, s["hkv"], -1, s["dk"]) * s["scale"]
    for t in range(max(lengths)):
        on = sum(length > t for length in lengths)
        at = first[:on] + t
        now = mine[:on]
        now *= (a[at] if s["by_row"] else a.expand(on, -1))[:, :, None, None]
        now += k[at][..., None] * v[at][:, :, None]
        y[at] = (q[at][..., None] * now[:, :, None]).sum(-2).reshape(on, s["hq"], s["dv"])
    states[[slots[i] for i in order]] = mine
    return {"y": y, "states": states}
