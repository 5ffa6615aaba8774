"""Contexts and 64-bit references for the GPU tests of the differential layers' operators."""
import math

from paper_2505_23317_amd import synth

EPS32 = 2.0 ** -24
HALF_STEP = {"bf16": 2.0 ** -8, "f32": EPS32}   # of one rounding, relative to the value
MODELS = {64: 2, 256: 8, 384: 6, 768: 12, 1024: 16}
LN_EPS = 1e-5


def encoder(d, rows, frames=1, dtype="bf16", heads=None, ffn=128):
    """A context of that width whose one layer is never run."""
    from paper_2505_23317_amd import cfdetr
    cfg = synth.Config("operators", frames, 32, 32, (32,), d, heads or MODELS[d], 1, ffn, "bf16")
    return cfdetr.Encoder(cfg, synth.make_weights(cfg, 1), act_dtype=dtype, max_batch=frames, max_tokens_total=max(rows, frames))


def act(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def normal(seed, *shape, std=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda") * std


def offsets(lengths):
    import torch
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")


def diff_attention(q, k, v, nq, nk, heads, lam, head_g, dtype, scale=None, mask=None):
    """(rows, bound of the error of the library's), both [n_q, d] in 64 bits.

    Bound.  With u the half step of the probabilities' type and e the relative error that a
    logit's 32-bit products (d_head terms, their sum, the scale) leave in a probability, a map's row is off by
    (u + 2 e + n 2^-24) sum p |v| at most, the sum of probabilities in the divisor included (n keys added in 32 bits).
    The norm divides by the root mean square r of the row: an element off by D_i and a row off by D make
    (D_i + |o_i| rms(D) / r) g / r; rounding the result adds its half step.  A twentieth is for products of these.
    """
    import torch
    d = q.shape[1]
    dh = d // heads
    scale = dh ** -0.5 if scale is None else scale
    out = torch.zeros(q.shape[0], d, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    q0 = k0 = 0
    u = HALF_STEP[dtype] if dtype == "bf16" else 0.0
    for a, b in zip(nq, nk):
        keys = torch.arange(k0, k0 + b, device="cuda")
        if mask is not None:
            keys = keys[mask[keys] != 0]
        qf, kf, vf = q[q0:q0 + a].double(), k[keys].double(), v[keys].double()
        for h in range(heads // 2 if len(keys) and a else 0):
            cols = slice(2 * h * dh, 2 * (h + 1) * dh)
            o, err = 0.0, 0.0
            for m, weight in ((0, 1.0), (1, -float(lam[h]))):
                c = slice((2 * h + m) * dh, (2 * h + m + 1) * dh)
                kt = kf[:, c].t().contiguous()
                p = torch.softmax(scale * (qf[:, c] @ kt), 1)
                e = (dh + 4) * EPS32 * scale * (qf[:, c].abs() @ kt.abs()).amax(1, keepdim=True)
                o = o + weight * (p @ vf[:, cols])
                err = err + abs(weight) * (u + 2 * e + len(keys) * EPS32) * (p @ vf[:, cols].abs())
            if head_g is not None:
                r = torch.sqrt(o.square().mean(1, keepdim=True) + LN_EPS)
                g = head_g.double()
                err = (err + o.abs() * torch.sqrt(err.square().mean(1, keepdim=True)) / r) * g.abs() / r + 64 * EPS32 * (o / r * g).abs()
                o = o / r * g
            out[q0:q0 + a, cols] = o
            bound[q0:q0 + a, cols] = 1.05 * err + (HALF_STEP[dtype] + 4 * EPS32) * o.abs()
        q0 += a
        k0 += b
    return out, bound


def within(got, want, bound, what=""):
    off = (got.double() - want).abs()
    worst = (off / bound.clamp_min(1e-300)).max().item() if off.numel() else 0.0
    assert bool((off <= bound).all()), f"{what}: {worst:.3g} times the bound, at most {off.max().item():.3g}"
    return worst


def turned(x, pos, freq, heads, interleaved):
    """Rows [M, d] with their pairs turned, in 64 bits, and for every feature the length of its pair."""
    import torch
    M, d = x.shape
    y = x.double().view(M, heads, d // heads).clone()
    size = y.abs()
    n, n_axes = freq.numel(), pos.shape[1]
    angle = pos.double()[:, torch.arange(n, device="cuda") * n_axes // n] * freq
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    first = slice(0, 2 * n, 2) if interleaved else slice(0, n)
    second = slice(1, 2 * n, 2) if interleaved else slice(n, 2 * n)
    a, b = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    size[..., first] = size[..., second] = torch.hypot(a, b)
    return y.reshape(M, d), size.reshape(M, d)


def log2e_over(dh):
    return 1.4426950408889634 / math.sqrt(dh)
