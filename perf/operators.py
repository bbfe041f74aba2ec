"""The operators of a decoder that reads a network's feature maps: residual addition with RMS norm into 8 bits, the
8-bit projection with the low-rank adapters of many requests, and cross attention from the requests' tokens to the
positions of the frames.

Sizes: feature maps of 19x19, 38x38 and 76x76 positions as the YOLOv2 stack gives them, model widths, head sizes and
ranks as decoders have them, odd and ragged ones among them.

A case: ``op`` and its sizes.
  norm:   rows, cols, dtype of the residual stream, residual (whether there is one to add), out ("f8", "bf16", "f32").
  linear: rows, k, n, adapters (0: none), rank, grouped (rows of one adapter next to each other, or every row its
          own), bias.
  cross:  frames, rows (queries of all frames together), s positions, hq and hkv heads, d, dtype, ragged (frames have
          different numbers of queries and of valid positions), mask ("none", "keys": by frame, "rows": by query),
          lse.
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f8": F8}
SIZE = {"f32": 4, "bf16": 2, "f8": 1}
F8_MAX = 448.0
EPS = 1e-6


def _norm(rows, cols, dtype, residual, out, name=None):
    d = {"op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual, "out": out}
    return dict(d, name=name) if name else d


def _linear(rows, k, n, adapters=0, rank=0, grouped=False, bias=False, name=None):
    d = {"op": "linear", "rows": rows, "k": k, "n": n, "adapters": adapters, "rank": rank, "grouped": grouped,
         "bias": bias}
    return dict(d, name=name) if name else d


def _cross(frames, rows, s, hq, hkv, d, dtype="bf16", ragged=False, mask="none", lse=False, name=None):
    c = {"op": "cross", "frames": frames, "rows": rows, "s": s, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype,
         "ragged": ragged, "mask": mask, "lse": lse}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One decode step of four requests: a launch's latency.
        _norm(4, 1024, "bf16", True, "f8", name="norm_step"),
        # The network's own feature map (three frames of 19x19) of an odd width, full precision, nothing to add.
        _norm(1083, 1001, "f32", False, "f32", name="norm_map_odd_f32"),
        # Prompts of many requests at once: bound by memory.
        _norm(16384, 4096, "bf16", True, "f8", name="norm_prompts"),
        # One decode step of four requests without adapters: the weights are read for four rows.
        _linear(4, 2048, 2048, name="linear_step"),
        # A decode step of 64 requests, each with its own of 16 adapters in any order, and a bias.
        _linear(64, 4096, 4096, 16, 16, bias=True, name="linear_adapters_step"),
        # Ragged prompts: odd rows and outputs, a width that is no multiple of a tile, grouped adapters.
        _linear(1083, 1360, 1001, 5, 8, grouped=True, name="linear_ragged"),
        # Long prompts of eight requests, an adapter each: the largest product.
        _linear(8192, 4096, 4096, 8, 32, grouped=True, name="linear_prompts"),
        # One token of one request about one frame.
        _cross(1, 1, 1444, 8, 2, 64, name="cross_token"),
        # A decode step of 64 requests about eight frames, several a frame, maps of different sizes.
        _cross(8, 64, 1444, 32, 8, 128, ragged=True, name="cross_step_ragged"),
        # Four requests, each about 45 frames in a row: a long axis for few rows.
        _cross(4, 4, 64980, 16, 4, 128, mask="keys", name="cross_long"),
        # Prompts that read the 76x76 map of two frames: the largest call.
        _cross(2, 4096, 5776, 16, 16, 128, name="cross_prompts"),
        # Ragged prompts in float32 with an odd head size, every query its own region of the map, some of them empty.
        _cross(3, 397, 361, 6, 3, 80, "f32", ragged=True, mask="rows", lse=True, name="cross_regions_f32"),
    ]


def draw(rng):
    """One more case of the ranges above."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    for _ in range(1000):
        op = rng.choice(["norm", "linear", "linear", "cross", "cross"])
        if op == "norm":
            dtype = rng.choice(["bf16", "bf16", "f32"])
            cols = rng.choice([log(64, 8192), 8 * log(8, 1024), rng.choice([256, 512, 1024, 2048, 4096])])
            case = _norm(log(1, 16384), cols, dtype, rng.random() < 0.6, rng.choice(["f8", "f8", dtype]))
        elif op == "linear":
            adapters = rng.choice([0, 0, 1, log(2, 64)])
            rank = rng.choice([4, 8, 16, 32, 64]) if adapters else 0
            n = rng.choice([log(64, 8192), 16 * log(4, 512)])
            rows = rng.choice([log(1, 64), log(1, 8192)])
            case = _linear(rows, 16 * log(8, 512), n, adapters, rank, adapters > 0 and rng.random() < 0.5,
                           rng.random() < 0.3)
        else:
            hkv = rng.choice([1, 2, 3, 4, 8])
            d = rng.choice([32, 64, 64, 128, 128, 256, 40, 80, 96])
            frames = log(1, 16)
            rows = rng.choice([frames, log(frames, 64 * frames), log(frames, 2048 * frames)])
            case = _cross(frames, rows, rng.choice([361, 1444, 5776, log(1, 64980)]), hkv * rng.choice([1, 2, 4, 8]),
                          hkv, d, rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.random() < 0.5,
                          rng.choice(["none", "none", "keys", "rows"]), rng.random() < 0.3)
            if case["mask"] == "rows" and rows * case["s"] > 2 ** 27 or rows * case["hq"] * case["s"] > 5e8:
                continue
        w = work(case)
        # no more than the largest listed case of the same operator (float32 products run at a fraction of the rate)
        most = {"norm": (4.8e8, 1e12), "linear": (4.8e8, 2.8e11), "cross": (5.4e8, 2e11)}[op]
        if case.get("dtype") == "f32" and op == "cross":
            most = (2.7e8, 2e10)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return case
    raise RuntimeError("no case drawn")


def work(case):
    """Each input once and each output once."""
    c = case
    if c["op"] == "norm":
        size = SIZE[c["dtype"]]
        a_row = c["cols"] * (size * (3 if c["residual"] else 1) + SIZE[c["out"]]) + (4 if c["out"] == "f8" else 0)
        return {"bytes": c["rows"] * a_row + 4 * c["cols"], "flops": 6 * c["rows"] * c["cols"]}
    if c["op"] == "linear":
        met = min(c["adapters"], c["rows"])
        bytes_ = c["rows"] * (c["k"] + 4 + 2 * c["n"]) + c["n"] * (c["k"] + 4)
        bytes_ += 2 * met * c["rank"] * (c["k"] + c["n"])
        return {"bytes": bytes_, "flops": 2 * c["rows"] * (c["n"] * c["k"] + c["rank"] * (c["n"] + c["k"]))}
    size = SIZE[c["dtype"]]
    # ragged frames have half of the positions on average
    keys = c["s"] * (0.5 if c["ragged"] else 1.0)
    bytes_ = 2 * c["rows"] * c["hq"] * c["d"] * size + 2 * c["frames"] * keys * c["hkv"] * c["d"] * size
    if c["mask"] != "none":
        bytes_ += (c["frames"] if c["mask"] == "keys" else c["rows"]) * keys
    return {"bytes": int(bytes_), "flops": int(4 * c["rows"] * c["hq"] * keys * c["d"])}


def _to_f8(x):
    """Rows in 8 bits: the values that are stored, and a scale per row."""
    scale = x.abs().amax(-1) / F8_MAX
    return (x / scale[:, None]).to(F8), scale


def prepare(case, seed):
    """Activations, weights and adapters on the GPU, as the layers before leave them."""
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if c["op"] == "norm":
        dt = DTYPES[c["dtype"]]
        wide = torch.exp(0.5 * randn(c["cols"]))  # some channels are larger than others
        return dict(c, x=(randn(c["rows"], c["cols"]) * wide).to(dt), gain=1 + 0.2 * randn(c["cols"]),
                    residual=(2 * randn(c["rows"], c["cols"]) * wide).to(dt) if c["residual"] else None)
    if c["op"] == "linear":
        x8, x_scale = _to_f8(randn(c["rows"], c["k"]))
        w8, w_scale = _to_f8(randn(c["n"], c["k"]) / math.sqrt(c["k"]))
        s = dict(c, x8=x8, x_scale=x_scale, w8=w8, w_scale=w_scale, bias_=0.1 * randn(c["n"]) if c["bias"] else None,
                 a=None, b=None, factor=None, row_adapter=None)
        if c["adapters"]:
            n, r = c["adapters"], c["rank"]
            s["a"] = (randn(n, r, c["k"]) / math.sqrt(c["k"])).bfloat16()
            s["b"] = (0.3 * randn(n, c["n"], r) / math.sqrt(r)).bfloat16()
            s["factor"] = 0.5 + torch.rand(n, generator=gen, device="cuda")
            # one row in n + 1 has no adapter (-1); grouped: requests one after another
            at = torch.randint(-1, n, (c["rows"],), generator=gen, device="cuda", dtype=torch.int32)
            s["row_adapter"] = torch.sort(at).values if c["grouped"] else at
        return s
    dt, f, s_ = DTYPES[c["dtype"]], c["frames"], c["s"]
    # keys and values side by side in the channels, as a network's last 1x1 layer gives them
    kv = randn(f, s_, 2, c["hkv"], c["d"]).to(dt)
    s = dict(c, q=(1.5 * randn(c["rows"], c["hq"], c["d"])).to(dt), k=kv[:, :, 0], v=kv[:, :, 1], q_offsets=None,
             k_lengths=None, key_mask=None, row_mask=None)
    if c["ragged"]:
        cut = torch.randint(0, c["rows"] + 1, (f - 1,), generator=gen, device="cuda", dtype=torch.int32)
        ends = torch.tensor([0, c["rows"]], dtype=torch.int32, device="cuda")
        s["q_offsets"] = torch.sort(torch.cat([ends, cut])).values.to(torch.int32)
        s["k_lengths"] = torch.randint(0, s_ + 1, (f,), generator=gen, device="cuda", dtype=torch.int32)
    elif c["rows"] % f:
        # as many queries for each frame, but for the rest
        s["q_offsets"] = (torch.arange(f + 1, device="cuda") * c["rows"] // f).to(torch.int32)
    if c["mask"] == "keys":
        s["key_mask"] = torch.rand(f, s_, generator=gen, device="cuda") < 0.9
    elif c["mask"] == "rows":
        # a query's region: a run of positions, of length zero for some
        lo = torch.randint(0, s_ + 1, (c["rows"], 1), generator=gen, device="cuda")
        at = torch.arange(s_, device="cuda")
        s["row_mask"] = (at >= lo) & (at < lo + s_ // 2)
    return s


def run(state):
    s = state
    if own:
        from paper_2107_06960_amd import operators as O
        if s["op"] == "norm":
            total, y, scale = O.add_rms_norm(s["x"], s["gain"], s["residual"], eps=EPS, out=s["out"])
            return {"sum": total, "y": y, "scale": scale}
        if s["op"] == "linear":
            adapters = (s["a"], s["b"], s["factor"]) if s["adapters"] else None
            return O.linear8(s["x8"], s["x_scale"], s["w8"], s["w_scale"], bias=s["bias_"], adapters=adapters,
                             row_adapter=s["row_adapter"])
        y, lse = O.cross_attention(s["q"], s["k"], s["v"], q_offsets=s["q_offsets"], k_lengths=s["k_lengths"],
                                   key_mask=s["key_mask"], row_mask=s["row_mask"], lse=s["lse"])
        return {"y": y, "lse": lse}
    return {"norm": _plain_norm, "linear": _plain_linear, "cross": _plain_cross}[s["op"]](s)


def _plain_norm(s):
    x, total = s["x"], None
    if s["residual"] is not None:
        x = total = (x.float() + s["residual"].float()).to(x.dtype)
    h = x.float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["gain"]
    if s["out"] != "f8":
        return {"sum": total, "y": y.to(DTYPES[s["out"]]), "scale": None}
    most = y.abs().amax(-1)
    scale = torch.where(most == 0, 1.0, most / F8_MAX)
    return {"sum": total, "y": (y / scale[:, None]).to(F8), "scale": scale}


def _plain_linear(s):
    x = s["x8"].float() * s["x_scale"][:, None]
    y = x @ (s["w8"].float() * s["w_scale"][:, None]).t()
    if s["bias_"] is not None:
        y = y + s["bias_"]
    if s["adapters"]:
        n, r, k = s["a"].shape
        u = (x @ s["a"].float().reshape(n * r, k).t()).reshape(-1, n, r)
        mine = s["row_adapter"][:, None] == torch.arange(n, device=x.device)
        u = u * (mine * s["factor"])[:, :, None]
        y = y + u.reshape(-1, n * r) @ s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    return y.bfloat16()


def _plain_cross(s):
    q, f, s_, hkv, d = s["q"].float(), s["frames"], s["s"], s["hkv"], s["d"]
    rows, g = s["rows"], s["hq"] // s["hkv"]
    # every frame's queries in a block of its own, as many slots as rows could need
    if s["q_offsets"] is None:
        t = rows // f
        slots = torch.arange(rows, device=q.device)
        block = slots.reshape(f, t)
    else:
        off = s["q_offsets"].long()
        t = int((off[1:] - off[:-1]).max())
        block = off[:-1, None] + torch.arange(t, device=q.device)
        frame = (torch.arange(rows, device=q.device)[:, None] >= off[1:]).sum(1)
        slots = frame * t + torch.arange(rows, device=q.device) - off[frame]
        block = block.clamp(max=rows - 1)
    qf = q[block].reshape(f, t, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(f, hkv, g * t, d)
    kf = s["k"].float().permute(0, 2, 3, 1).contiguous()
    vf = s["v"].float().permute(0, 2, 1, 3).contiguous()
    z = (qf @ kf).reshape(f, hkv, g, t, s_) / math.sqrt(d)
    if s["k_lengths"] is not None:
        z = z.masked_fill((torch.arange(s_, device=q.device) >= s["k_lengths"][:, None])[:, None, None, None], -math.inf)
    if s["key_mask"] is not None:
        z = z.masked_fill(~s["key_mask"][:, None, None, None], -math.inf)
    if s["row_mask"] is not None:
        z = z.masked_fill(~s["row_mask"][block][:, None, None], -math.inf)
    most = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(f, hkv, g * t, s_) @ vf).reshape(f, hkv, g, t, d) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(f * t, hkv * g, d)[slots]
    lse = None
    if s["lse"]:
        lse = (most + torch.log(total)).permute(0, 3, 1, 2, 4).reshape(f * t, hkv * g)[slots]
    return {"y": o.to(s["q"].dtype), "lse": lse}


def exact(case, seed):
    """The operators in float64, before any rounding of the outputs (8-bit values: what they stand for before they are
    rounded to 8 bits)."""
    s = prepare(case, seed)
    if s["op"] == "norm":
        h, total = s["x"].double(), None
        if s["residual"] is not None:
            total = h + s["residual"].double()
            h = total.to(s["x"].dtype).double()  # the norm is that of the sum as it is stored
        y = h / (h.square().sum(-1, keepdim=True) / h.shape[1] + EPS).sqrt() * s["gain"].double()
        if s["out"] != "f8":
            return {"sum": total, "y": y, "scale": None}
        scale = y.abs().amax(-1) / F8_MAX
        scale[scale == 0] = 1
        return {"sum": total, "y": y / scale[:, None], "scale": scale}
    if s["op"] == "linear":
        x = s["x8"].double().mul_(s["x_scale"].double()[:, None])
        y = x @ s["w8"].double().mul_(s["w_scale"].double()[:, None]).t().contiguous()
        if s["bias_"] is not None:
            y += s["bias_"].double()
        for i in range(s["adapters"]):
            at = (s["row_adapter"] == i).nonzero()[:, 0]
            if at.numel():
                u = x[at] @ s["a"][i].double().t().contiguous()
                y[at] += s["factor"][i].double() * (u @ s["b"][i].double().t().contiguous())
        return y
    rows, f, g = s["rows"], s["frames"], s["hq"] // s["hkv"]
    off = [i * rows // f for i in range(f + 1)] if s["q_offsets"] is None else s["q_offsets"].tolist()
    lens = [s["s"]] * f if s["k_lengths"] is None else s["k_lengths"].tolist()
    y = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for i in range(f):
        a, b, n = off[i], off[i + 1], lens[i]
        if a == b or n == 0:
            continue
        for h in range(s["hq"]):
            k, v = s["k"][i, :n, h // g].double(), s["v"][i, :n, h // g].double()
            z = s["q"][a:b, h].double() @ k.t().contiguous() / math.sqrt(s["d"])
            if s["key_mask"] is not None:
                z[:, ~s["key_mask"][i, :n]] = -math.inf
            if s["row_mask"] is not None:
                z[~s["row_mask"][a:b, :n]] = -math.inf
            some = z.amax(-1) > -math.inf
            lse[a:b, h] = torch.logsumexp(z, -1)
            y[a:b, h] = torch.where(some[:, None], torch.softmax(z, -1) @ v, 0.0)
    return {"y": y, "lse": lse if s["lse"] else None}
