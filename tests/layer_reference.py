"""Plain definitions in 64 bits of the operators of paper_2511_11062_amd.layer, and what the tests of them share."""
import torch

from paper_2511_11062_amd import layer

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
KINDS = {"bf16": layer.LITE_ATTN_BF16, "f16": layer.LITE_ATTN_F16, "f32": layer.LITE_ATTN_F32}
NORMS = {"none": layer.LITE_ATTN_NORM_NONE, "head": layer.LITE_ATTN_NORM_HEAD, "row": layer.LITE_ATTN_NORM_ROW,
         "rms": layer.LITE_ATTN_NORM_RMS, "layer": layer.LITE_ATTN_NORM_LAYER}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def stream():
    return torch.cuda.current_stream().cuda_stream


def heads_view(t):
    """(address, stride_b, stride_h, stride_n) of a tensor indexed [batch, heads, tokens, head_dim]."""
    assert t.stride(3) == 1 or t.shape[3] == 1
    return t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)


def rows_view(t):
    return None if t is None else (t.data_ptr(), t.stride(0), t.stride(1))


def at(t):
    return 0 if t is None else t.data_ptr()


def half_step(kind, ref):
    """What rounding a result once to its type may be off by, subnormal results included."""
    info = torch.finfo(kind)
    return torch.maximum(ref.abs() * (info.eps / 2), torch.full_like(ref, info.tiny * info.eps / 2))


def check(name, got, ref, slack):
    """|got - ref| within half a step of the type and `slack` of 32-bit arithmetic (a tensor or a number), everywhere."""
    off = (got.double() - ref).abs()
    bound = half_step(got.dtype, ref.abs() + slack) + slack
    assert torch.isfinite(got).all(), name
    worst = (off / bound.clamp_min(1e-300)).max().item() if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3f of its bound" % (name, worst)


# ---- rotary ----

def grid_positions(grid, start, n):
    f, h, w = grid
    rows = []
    for t in range(start, start + n):
        rows.append((t // (h * w), t % (h * w) // w, t % w) if t < f * h * w else (0, 0, 0))
    return torch.tensor(rows, dtype=torch.float64, device="cuda").reshape(n, 3)


def rotary(x, w, freqs, positions, norm, halves, eps):
    """x [B,H,N,d] (64 bits); positions [B or 1,N,3]; -> [B,H,N,d]."""
    if norm != "none":
        mean = (x * x).mean(dim=(1, 3) if norm == "row" else 3, keepdim=True)
        x = x / torch.sqrt(mean + eps)
        if w is not None:
            x = x * (w[:, None] if norm == "row" else w)
    pairs = freqs.shape[1]
    angle = (positions[:, :, :, None] * freqs[None, None]).sum(dim=2)[:, None]  # [B,1,N,pairs]
    if halves:
        ia = torch.arange(pairs, device=x.device)
        ib = ia + pairs
    else:
        ia = 2 * torch.arange(pairs, device=x.device)
        ib = ia + 1
    a, b = x[..., ia], x[..., ib]
    out = x.clone()
    out[..., ia] = a * angle.cos() - b * angle.sin()
    out[..., ib] = a * angle.sin() + b * angle.cos()
    return out


def partner_sum(x, pairs, halves):
    """|a| + |b| of each entry's pair, for entries that are turned; |x| for the others."""
    x = x.abs()
    out = x.clone()
    i = torch.arange(pairs, device=x.device)
    ia, ib = (i, i + pairs) if halves else (2 * i, 2 * i + 1)
    out[..., ia] = out[..., ib] = x[..., ia] + x[..., ib]
    return out


# ---- residual ----

def normed(x, kind, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)


def spread(t, per, n):
    """A row of modulation for each token: [B,G,D] -> [B,N,D]."""
    return t[:, torch.arange(n, device=t.device) // per]
