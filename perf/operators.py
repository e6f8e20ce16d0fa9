"""The operators around the skip-aware attention call of a transformer layer, as timed cases.

    "rotary"    queries and keys as a projection leaves them -> normalised over the head or over the whole token, turned
                by the token's position on the axes time, height and width, and laid out for the attention call
    "residual"  a branch's output y -> normalised, gated and added to the residual stream x, whose norm, scaled and
                shifted, is the next branch's input h

each forwards and backwards, through the public entry points of ``paper_2511_11062_amd.layer``.

A "rotary" case has

    batch, heads_q, heads_k, head_dim      (heads_k < heads_q: shared key heads)
    frames, height, width, text            the latent grid in raster order and the text tokens behind it
    tokens, start                          tokens of the call and the first one's place in that order
    far                                    positions come from a tensor and start here; None: from the grid
    norm       "none", "head" (over head_dim) or "row" (over all heads of the token)
    halves     pair i is (i, i + pairs); otherwise (2i, 2i + 1)
    pairs      pairs turned, in three sections, one for each axis; what is left of the head stays as it is
    source     "bnhd" or "packed": q, k and v side by side in one projection's result;  target  "bhnd" or "bnhd"

and a "residual" case batch, tokens, dim, tokens_per_mod (tokens that share a row of gate, scale and shift), the norms of
the branch ("post") and of the stream ("pre"): "none", "layer" or "rms", weights of both or none, and the stream's type.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_THETA = 10000.0
_EPS = 1e-6
_SCALE = 0.75  # of the residual branch


def _rotary(name, way, batch, heads, head_dim, grid, *, text=0, tokens=None, start=0, far=None, dtype="bf16",
            weights="f32", norm="none", halves=False, pairs=None, source="bnhd", target="bhnd"):
    c = {"op": "rotary", "way": way, "batch": batch, "heads_q": heads[0], "heads_k": heads[1], "head_dim": head_dim,
         "frames": grid[0], "height": grid[1], "width": grid[2], "text": text,
         "tokens": grid[0] * grid[1] * grid[2] + text if tokens is None else tokens, "start": start, "far": far,
         "dtype": dtype, "weights": weights, "norm": norm, "halves": halves,
         "pairs": head_dim // 2 if pairs is None else pairs, "source": source, "target": target}
    return dict(c, name=name) if name else c


def _residual(name, way, batch, tokens, dim, *, tokens_per_mod=None, dtype="bf16", stream="f32", params="f32",
              post="none", pre="layer", weights=False):
    c = {"op": "residual", "way": way, "batch": batch, "tokens": tokens, "dim": dim,
         "tokens_per_mod": tokens if tokens_per_mod is None else tokens_per_mod, "dtype": dtype, "stream": stream,
         "params": params, "post": post, "pre": pre, "weights": weights}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token for each of three requests far into their sequences, shared key heads, positions from a tensor:
        # latency and launches only
        _rotary("rotary_one_token", "fwd", 3, (16, 4), 128, (1, 1, 1), far=1 << 20, norm="head", halves=True,
                target="bnhd"),
        # the tiny configuration
        _rotary("rotary_tiny", "fwd", 1, (2, 2), 128, (2, 32, 32)),
        # a ragged low-resolution preview with text behind it, batch of two (guidance), out of one packed projection,
        # part of the head turned
        _rotary("rotary_preview", "fwd", 2, (6, 2), 64, (2, 24, 31), text=99, dtype="f16", weights="f16", norm="head",
                halves=True, pairs=24, source="packed"),
        # the 12-head layer; norm over the token, as the layers of that model have it
        _rotary("rotary_12_heads", "fwd", 1, (12, 12), 128, (21, 30, 52), norm="row"),
        # the 40-head layer of the benchmark
        _rotary("rotary_40_heads", "fwd", 1, (40, 40), 128, (21, 60, 60), norm="row"),
        # training the 12-head layer
        _rotary("rotary_bwd_12_heads", "bwd", 1, (12, 12), 128, (21, 30, 52), norm="row"),
        # training in 32 bits with a head that is no power of two, an odd number of tokens, a norm over the head
        _rotary("rotary_bwd_ragged", "bwd", 2, (5, 5), 72, (3, 31, 41), text=77, dtype="f32", norm="head",
                source="packed", target="bnhd"),
        # the first block of a chunk of a few tokens: latency and launches only
        _residual("residual_chunk", "fwd", 2, 17, 256),
        # the 12-head layer: stream in 32 bits, one row of gate, scale and shift for the sample
        _residual("residual_12_heads", "fwd", 1, 32760, 1536),
        # the 40-head layer: stream in 16 bits, norms before and behind the block, modulated frame by frame
        _residual("residual_40_heads", "fwd", 1, 75600, 5120, tokens_per_mod=3600, stream="bf16", post="rms", pre="rms",
                  weights=True),
        # training the 12-head layer
        _residual("residual_bwd_12_heads", "bwd", 1, 32760, 1536),
        # training with a width and a number of tokens that are odd, frame by frame, all norms and weights
        _residual("residual_bwd_ragged", "bwd", 2, 3913, 1111, tokens_per_mod=1271, dtype="f16", stream="f16",
                  params="f16", post="rms", pre="layer", weights=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        way = rng.choice(["fwd", "bwd"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        batch = rng.choice([1, 1, 2, 3])
        tokens = _log(rng, 1, 118800)
        if rng.random() < 0.5:
            heads_q = _log(rng, 1, 40)
            heads_k = rng.choice([heads_q, heads_q, max(1, heads_q // 4)])
            head_dim = rng.choice([128, 128, 128, 64, 72, 80, 96, 256])
            frames = min(33, tokens, _log(rng, 1, 33))
            height = max(1, round(math.sqrt(tokens / frames) * rng.uniform(0.6, 1.0)))
            width = max(1, round(tokens / (frames * height)))
            text = rng.choice([0, 0, rng.randint(1, 300)])
            whole = frames * height * width + text
            chunk = rng.random() < 0.2
            n = _log(rng, 1, whole) if chunk else whole
            c = _rotary(None, way, batch, (heads_q, heads_k), head_dim, (frames, height, width), text=text, tokens=n,
                        start=rng.randint(0, whole - n), far=rng.choice([None, None, None, rng.randint(0, 1 << 20)]),
                        dtype=dtype, weights=rng.choice(["f32", dtype]), norm=rng.choice(["none", "head", "row", "row"]),
                        halves=rng.random() < 0.4, pairs=rng.choice([head_dim // 2] * 3 + [head_dim // 4]),
                        source=rng.choice(["bnhd", "packed"]), target=rng.choice(["bhnd", "bnhd"]))
        else:
            dim = 128 * _log(rng, 1, 64) if rng.random() < 0.7 else _log(rng, 65, 8191)
            c = _residual(None, way, batch, tokens, dim,
                          tokens_per_mod=rng.choice([None, None, max(1, tokens // rng.randint(2, 33))]), dtype=dtype,
                          stream=rng.choice(["f32", dtype]), params=rng.choice(["f32", dtype]),
                          post=rng.choice(["none", "none", "rms", "layer"]), pre=rng.choice(["layer", "layer", "rms"]),
                          weights=rng.random() < 0.4)
        if work(c)["bytes"] <= most:
            return c


def _sections(pairs):
    """Pairs of each axis: time gets what an even split leaves over."""
    side = pairs // 3
    return pairs - 2 * side, side, side


def _elements(case):
    return case["batch"] * case["tokens"] * (case["heads_q"] + case["heads_k"]) * case["head_dim"]


def work(case):
    size = _BYTES[case["dtype"]]
    bwd = case["way"] == "bwd"
    if case["op"] == "rotary":
        n = _elements(case)
        normed = case["norm"] != "none"
        # forwards: in and out; backwards: the results' gradients in and the inputs' out, under a norm the inputs too
        total = n * size * (3 if bwd and normed else 2)
        params = (case["heads_q"] + case["heads_k"] if case["norm"] == "row" else 2) * case["head_dim"] if normed else 0
        total += params * (_BYTES[case["weights"]] + (4 if bwd else 0)) + 3 * case["pairs"] * 8
        if case["far"] is not None:
            total += case["batch"] * case["tokens"] * 3 * 4
        return {"bytes": float(total), "flops": float(n * ((12 if bwd else 6) if normed else 3))}
    n, dim = case["batch"] * case["tokens"], case["dim"]
    groups = case["batch"] * -(-case["tokens"] // case["tokens_per_mod"])
    wide = _BYTES[case["stream"]]
    vectors = 3 if case["weights"] else 0
    # forwards x, y -> x_out, h; backwards dh, dx_out, x_out, y -> dx, dy and the parameters' gradients
    total = n * dim * ((3 * wide + 3 * size) if bwd else (2 * wide + 2 * size))
    total += (groups * 3 + vectors) * dim * _BYTES[case["params"]]
    if bwd:
        total += (groups * 3 + vectors) * dim * 4
    return {"bytes": float(total), "flops": float(n * dim * (30 if bwd else 14))}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFF)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _frequencies(case):
    """[3][pairs] radians per position, 64 bits: pair i of an axis' n pairs turns by theta^(-i/n), the others' not at all."""
    f = torch.zeros(3, case["pairs"], dtype=torch.float64)
    at = 0
    for axis, n in enumerate(_sections(case["pairs"])):
        f[axis, at:at + n] = torch.pow(torch.tensor(_THETA, dtype=torch.float64), -torch.arange(n, dtype=torch.float64) / n)
        at += n
    return f.cuda()


def _grid_positions(case):
    """[tokens, 3] places of the call's tokens on the grid; tokens behind the grid stand at its origin."""
    t = torch.arange(case["start"], case["start"] + case["tokens"], device="cuda")
    area, width = case["height"] * case["width"], case["width"]
    pos = torch.stack([t // area, t % area // width, t % width], dim=1)
    return pos * (t < case["frames"] * area)[:, None]


def _packed(case, g, std):
    """q and k [B,N,H,d] views of what the projection left, whose channels differ in size."""
    b, n, hq, hk, d = (case[x] for x in ("batch", "tokens", "heads_q", "heads_k", "head_dim"))
    kind = _TYPES[case["dtype"]]

    def make(heads):
        return (_randn(g, b, n, heads, d) * std * torch.exp(0.5 * _randn(g, heads, d))).to(kind)

    if case["source"] == "packed":
        x = make(hq + 2 * hk)
        return x[:, :, :hq], x[:, :, hq:hq + hk]
    return make(hq), make(hk)


def _target(case, heads, std=None, g=None):
    b, n, d = case["batch"], case["tokens"], case["head_dim"]
    shape = (b, heads, n, d) if case["target"] == "bhnd" else (b, n, heads, d)
    kind = _TYPES[case["dtype"]]
    return torch.empty(shape, dtype=kind, device="cuda") if g is None else (std * _randn(g, *shape)).to(kind)


def _prepare_rotary(case, seed):
    g = _gen(seed)
    q, k = _packed(case, g, 1.5)
    s = {"case": case, "q": q, "k": k, "freqs": _frequencies(case), "positions": None, "weights": (None, None)}
    if case["far"] is not None:  # [B,3,N]: time goes on from request to request, height and width stay on the grid
        pos = _grid_positions(case).t().repeat(case["batch"], 1, 1)
        first = case["far"] + torch.randint(0, 4096, (case["batch"],), generator=g, device="cuda")
        pos[:, 0] += first[:, None]
        s["positions"] = pos.to(torch.int32).contiguous()
    if case["norm"] != "none":
        shapes = [(h, case["head_dim"]) if case["norm"] == "row" else (case["head_dim"],)
                  for h in (case["heads_q"], case["heads_k"])]
        s["weights"] = tuple((1.0 + 0.2 * _randn(g, *shape)).to(_TYPES[case["weights"]]) for shape in shapes)
    heads = (case["heads_q"], case["heads_k"])
    if case["way"] == "fwd":
        s["out"] = [_target(case, h) for h in heads]
    else:
        s["grad"] = [_target(case, h, 0.01, g) for h in heads]
        s["dx"] = [torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (q, k)]
        s["dw"] = [None if w is None else torch.empty(w.shape, dtype=torch.float32, device="cuda") for w in s["weights"]]
    return s


def _prepare_residual(case, seed):
    g = _gen(seed)
    b, n, dim = case["batch"], case["tokens"], case["dim"]
    groups = -(-n // case["tokens_per_mod"])
    kind, wide, par = _TYPES[case["dtype"]], _TYPES[case["stream"]], _TYPES[case["params"]]
    # a residual stream: channels of different size and mean, some of them large
    size = torch.exp(0.7 * _randn(g, dim))
    x = (_randn(g, b, n, dim) * size + 0.5 * _randn(g, dim) * size).to(wide)
    s = {"case": case, "x": x, "y": (1.5 * _randn(g, b, n, dim)).to(kind)}
    # gate, scale and shift as the modulation's projection leaves them, side by side
    mod = (0.3 * _randn(g, b, groups, 3, dim)).to(par)
    s["gate"], s["scale"], s["shift"] = (mod[:, :, i] for i in range(3))
    s["post_weight"] = s["pre_weight"] = s["pre_bias"] = None
    if case["weights"]:
        s["post_weight"], s["pre_weight"] = ((1.0 + 0.2 * _randn(g, dim)).to(par) for _ in range(2))
        s["pre_bias"] = (0.1 * _randn(g, dim)).to(par)
    if case["way"] == "fwd":
        s["x_out"], s["h"] = torch.empty_like(x), torch.empty_like(s["y"])
    else:  # x is here what the forward pass left in the stream
        s["dh"] = (0.01 * _randn(g, b, n, dim)).to(kind)
        s["dx_out"] = (0.01 * _randn(g, b, n, dim)).to(wide)
        s["dx"], s["dy"] = torch.empty_like(x), torch.empty_like(s["y"])
        s["dmod"] = torch.empty(3, b, groups, dim, dtype=torch.float32, device="cuda")
        s["dvec"] = torch.empty(3, dim, dtype=torch.float32, device="cuda") if case["weights"] else None
    return s


def prepare(case, seed):
    s = _prepare_rotary(case, seed) if case["op"] == "rotary" else _prepare_residual(case, seed)
    if own:
        from paper_2511_11062_amd import layer
        s["layer"] = layer
        kinds = {"bf16": layer.LITE_ATTN_BF16, "f16": layer.LITE_ATTN_F16, "f32": layer.LITE_ATTN_F32}
        norms = {"none": layer.LITE_ATTN_NORM_NONE, "head": layer.LITE_ATTN_NORM_HEAD, "row": layer.LITE_ATTN_NORM_ROW,
                 "layer": layer.LITE_ATTN_NORM_LAYER, "rms": layer.LITE_ATTN_NORM_RMS}
        if case["op"] == "rotary":
            s["desc"] = layer.make_rotary_desc(
                case["batch"], case["tokens"], case["heads_q"], case["heads_k"], case["head_dim"],
                dtype=kinds[case["dtype"]], weight_dtype=kinds[case["weights"]], norm=norms[case["norm"]],
                halves=case["halves"], pairs=case["pairs"], grid=(case["frames"], case["height"], case["width"]), eps=_EPS)
            need = layer.lite_attn_rotary_bwd_workspace(s["desc"]) if case["way"] == "bwd" else 0
        else:
            s["desc"] = layer.make_residual_desc(
                case["batch"], case["tokens"], case["dim"], dtype=kinds[case["dtype"]],
                stream_dtype=kinds[case["stream"]], param_dtype=kinds[case["params"]], post_norm=norms[case["post"]],
                pre_norm=norms[case["pre"]], post_eps=_EPS, pre_eps=_EPS, residual_scale=_SCALE,
                tokens_per_mod=case["tokens_per_mod"])
            need = layer.lite_attn_residual_norm_bwd_workspace(s["desc"]) if case["way"] == "bwd" else 0
        s["workspace"] = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    return s


def _heads(t, layout):
    """A tensor's address and its strides over batch, heads and tokens."""
    if layout == "bhnd":
        return t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)
    return t.data_ptr(), t.stride(0), t.stride(2), t.stride(1)


def _rows(t):
    return t.data_ptr(), t.stride(0), t.stride(1)


def _at(t):
    return 0 if t is None else t.data_ptr()


def _own_rotary(s):
    case, layer = s["case"], s["layer"]
    stream = torch.cuda.current_stream().cuda_stream
    pos = s["positions"]
    where = {"positions": _at(pos), "positions_stride_b": 0 if pos is None else pos.stride(0),
             "token_start": case["start"], "hip_stream": stream}
    q, k = _heads(s["q"], "bnhd"), _heads(s["k"], "bnhd")
    wq, wk = s["weights"]
    if case["way"] == "fwd":
        qo, ko = s["out"]
        layer.lite_attn_rotary_fwd(s["desc"], q, k, _heads(qo, case["target"]), _heads(ko, case["target"]),
                                   s["freqs"].data_ptr(), q_weight=_at(wq), k_weight=_at(wk), **where)
        return {"q": qo, "k": ko}
    gq, gk = s["grad"]
    dq, dk = s["dx"]
    dwq, dwk = s["dw"]
    layer.lite_attn_rotary_bwd(s["desc"], q, k, _heads(gq, case["target"]), _heads(gk, case["target"]),
                               _heads(dq, "bnhd"), _heads(dk, "bnhd"), s["freqs"].data_ptr(), q_weight=_at(wq),
                               k_weight=_at(wk), dq_weight=_at(dwq), dk_weight=_at(dwk),
                               workspace=s["workspace"].data_ptr(), workspace_bytes=s["workspace"].numel(), **where)
    grads = {"dq": dq, "dk": dk}
    return grads if dwq is None else dict(grads, dq_weight=dwq, dk_weight=dwk)


def _own_residual(s):
    case, layer = s["case"], s["layer"]
    stream = torch.cuda.current_stream().cuda_stream
    params = {"gate": _rows(s["gate"]), "scale": _rows(s["scale"]), "post_weight": _at(s["post_weight"]),
              "pre_weight": _at(s["pre_weight"]), "pre_bias": _at(s["pre_bias"]), "hip_stream": stream}
    if case["way"] == "fwd":
        layer.lite_attn_residual_norm_fwd(s["desc"], _rows(s["x"]), _rows(s["y"]), _rows(s["x_out"]), _rows(s["h"]),
                                          shift=_rows(s["shift"]), **params)
        return {"x_out": s["x_out"], "h": s["h"]}
    dgate, dscale, dshift = s["dmod"]
    out = {"dx": s["dx"], "dy": s["dy"], "dgate": dgate, "dscale": dscale, "dshift": dshift}
    if s["dvec"] is not None:
        out["dpost_weight"], out["dpre_weight"], out["dpre_bias"] = s["dvec"]
    layer.lite_attn_residual_norm_bwd(s["desc"], _rows(s["dh"]), _rows(s["dx_out"]), _rows(s["x"]), _rows(s["y"]),
                                      _rows(s["dx"]), _rows(s["dy"]), dgate=_at(dgate), dscale=_at(dscale),
                                      dshift=_at(dshift), dpost_weight=_at(out.get("dpost_weight")),
                                      dpre_weight=_at(out.get("dpre_weight")), dpre_bias=_at(out.get("dpre_bias")),
                                      workspace=s["workspace"].data_ptr(), workspace_bytes=s["workspace"].numel(),
                                      **params)
    return out


def _turn(x, cos, sin, halves):
    """x [B,N,H,d] with its first 2 * pairs entries turned by cos, sin [B or 1, N, pairs]."""
    pairs = cos.shape[-1]
    cos, sin = cos[:, :, None], sin[:, :, None]
    if halves:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    return turned if 2 * pairs == x.shape[-1] else torch.cat([turned, x[..., 2 * pairs:]], dim=-1)


def _plain_rotary(s):
    case = s["case"]
    pos = _grid_positions(case)[None] if s["positions"] is None else s["positions"].transpose(1, 2)
    pos = pos.double()
    angle = sum(pos[:, :, a, None] * s["freqs"][a] for a in range(3))
    cos, sin = angle.cos().float(), angle.sin().float()
    over = {"head": (3,), "row": (2, 3)}.get(case["norm"])
    bhnd = case["target"] == "bhnd"
    outs = {}
    for name, x, w, at in (("q", s["q"], s["weights"][0], 0), ("k", s["k"], s["weights"][1], 1)):
        x = x.float()
        if over is not None:
            r = torch.rsqrt((x * x).mean(dim=over, keepdim=True) + _EPS)
            w = w.float()
        if case["way"] == "fwd":
            z = x if over is None else x * r * w
            z = _turn(z, cos, sin, case["halves"]).to(_TYPES[case["dtype"]])
            outs[name] = z.transpose(1, 2).contiguous() if bhnd else z
            continue
        dz = s["grad"][at].float()
        dz = _turn(dz.transpose(1, 2) if bhnd else dz, cos, -sin, case["halves"])
        if over is not None:
            n = x * r
            outs["d%s_weight" % name] = (dz * n).sum(dim=(0, 1) if case["norm"] == "row" else (0, 1, 2))
            dn = dz * w
            dz = r * (dn - n * (dn * n).mean(dim=over, keepdim=True))
        outs["d" + name] = dz.to(_TYPES[case["dtype"]])
    return outs


def _normed(x, kind):
    """(n, r): x normalised over its last axis and what it was multiplied with."""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + _EPS)
    return x * r, r


def _normed_back(dn, n, r, kind):
    if kind == "none":
        return dn
    d = dn - n * (dn * n).mean(dim=-1, keepdim=True)
    if kind == "layer":
        d = d - dn.mean(dim=-1, keepdim=True)
    return d * r


def _plain_residual(s):
    case = s["case"]
    per, tokens = case["tokens_per_mod"], case["tokens"]
    kind, wide = _TYPES[case["dtype"]], _TYPES[case["stream"]]

    def spread(t):  # a row of modulation for every token
        t = t.float()
        return t if t.shape[1] == 1 else t.repeat_interleave(per, dim=1)[:, :tokens]

    gate, scale = spread(s["gate"]), spread(s["scale"])
    w2 = 1.0 if s["post_weight"] is None else s["post_weight"].float()
    w1 = 1.0 if s["pre_weight"] is None else s["pre_weight"].float()
    b1 = 0.0 if s["pre_bias"] is None else s["pre_bias"].float()
    ny, ry = _normed(s["y"].float(), case["post"])
    if case["way"] == "fwd":
        x_out = s["x"].float() + _SCALE * gate * (ny * w2)
        n, _ = _normed(x_out, case["pre"])
        h = (n * w1 + b1) * (1.0 + scale) + spread(s["shift"])
        return {"x_out": x_out.to(wide), "h": h.to(kind)}

    def gathered(t):  # sums over the tokens of a row of modulation
        groups = s["gate"].shape[1]
        if groups == 1:
            return t.sum(dim=1, keepdim=True)
        short = groups * per - tokens
        if short:
            t = torch.nn.functional.pad(t, (0, 0, 0, short))
        return t.view(t.shape[0], groups, per, -1).sum(dim=2)

    n, r = _normed(s["x"].float(), case["pre"])
    dh = s["dh"].float()
    da = dh * (1.0 + scale)
    dx = s["dx_out"].float() + _normed_back(da * w1, n, r, case["pre"])
    dp = _SCALE * dx * gate
    out = {"dx": dx.to(wide), "dy": _normed_back(dp * w2, ny, ry, case["post"]).to(kind),
           "dgate": gathered(_SCALE * dx * (ny * w2)), "dscale": gathered(dh * (n * w1 + b1)), "dshift": gathered(dh)}
    if case["weights"]:
        out["dpost_weight"] = (dp * ny).sum(dim=(0, 1))
        out["dpre_weight"] = (da * n).sum(dim=(0, 1))
        out["dpre_bias"] = da.sum(dim=(0, 1))
    return out


def run(state):
    if state["case"]["op"] == "rotary":
        return _own_rotary(state) if own else _plain_rotary(state)
    return _own_residual(state) if own else _plain_residual(state)


def _exact_rotary(case, s):
    """Pair by pair as multiplication of complex numbers, the gradients by differentiating that."""
    if s["positions"] is not None:
        pos = s["positions"].permute(0, 2, 1).double()
    else:
        pos = torch.zeros(1, case["tokens"], 3, dtype=torch.float64, device="cuda")
        t = case["start"] + torch.arange(case["tokens"], device="cuda")
        on = t < case["frames"] * case["height"] * case["width"]
        for axis, size in ((2, case["width"]), (1, case["height"]), (0, case["frames"])):
            pos[0, :, axis] = torch.where(on, t % size, 0).double()
            t = torch.div(t, size, rounding_mode="floor")
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos @ s["freqs"])[:, :, None]
    pairs, out = case["pairs"], {}
    for x, name, at in ((s["q"], "q", 0), (s["k"], "k", 1)):
        bwd, w = case["way"] == "bwd", s["weights"][at]
        x = x.double().requires_grad_(bwd)
        w = None if w is None else w.double().requires_grad_(bwd)
        z = x
        if w is not None:
            power = x.square().mean(dim=3, keepdim=True)
            if case["norm"] == "row":
                power = power.mean(dim=2, keepdim=True)
            z = x / (power + _EPS).sqrt() * w
        head, rest = z[..., :2 * pairs], z[..., 2 * pairs:]
        split = (2, pairs) if case["halves"] else (pairs, 2)
        head = head.unflatten(-1, split)
        if case["halves"]:
            head = head.transpose(-1, -2)
        head = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
        if case["halves"]:
            head = head.transpose(-1, -2)
        z = torch.cat([head.flatten(-2), rest], dim=-1)
        if case["target"] == "bhnd":
            z = z.permute(0, 2, 1, 3)
        if not bwd:
            out[name] = z.contiguous()
            continue
        leaves = [x] if w is None else [x, w]
        grads = torch.autograd.grad(z, leaves, s["grad"][at].double())
        out["d" + name] = grads[0]
        if w is not None:
            out["d%s_weight" % name] = grads[1]
    return out


def _exact_residual(case, s):
    """The definition in 64 bits, the gradients by differentiating it."""
    bwd = case["way"] == "bwd"
    group = torch.arange(case["tokens"], device="cuda") // case["tokens_per_mod"]
    names = [x for x in ("gate", "scale", "shift", "post_weight", "pre_weight", "pre_bias") if s[x] is not None]
    p = {x: s[x].double().requires_grad_(bwd) for x in names}

    def norm(t, kind):
        if kind == "none":
            return t
        var, mean = torch.var_mean(t, dim=-1, keepdim=True, correction=0)
        if kind == "layer":
            return (t - mean) / (var + _EPS).sqrt()
        return t / (var + mean.square() + _EPS).sqrt()

    def step(y):  # what the branch adds to the stream
        z = norm(y, case["post"])
        return _SCALE * p["gate"][:, group] * (z * p["post_weight"] if "post_weight" in p else z)

    def block(x):
        z = norm(x, case["pre"])
        if "pre_weight" in p:
            z = z * p["pre_weight"] + p["pre_bias"]
        return z + z * p["scale"][:, group] + p["shift"][:, group]

    y = s["y"].double().requires_grad_(bwd)
    if not bwd:
        x = s["x"].double() + step(y)
        return {"x_out": x, "h": block(x)}
    x = s["x"].double().requires_grad_()
    front = [x] + [p[n] for n in ("scale", "shift", "pre_weight", "pre_bias") if n in p]
    got = torch.autograd.grad(block(x), front, s["dh"].double())
    dx = got[0] + s["dx_out"].double()
    back = [y, p["gate"]] + ([p["post_weight"]] if "post_weight" in p else [])
    low = torch.autograd.grad(step(y), back, dx)
    out = {"dx": dx, "dy": low[0], "dgate": low[1], "dscale": got[1], "dshift": got[2]}
    if case["weights"]:
        out["dpost_weight"], out["dpre_weight"], out["dpre_bias"] = low[2], got[3], got[4]
    return out


def exact(case, seed):
    s = _prepare_rotary(case, seed) if case["op"] == "rotary" else _prepare_residual(case, seed)
    return _exact_rotary(case, s) if case["op"] == "rotary" else _exact_residual(case, s)
