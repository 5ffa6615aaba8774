"""The operators of a differential encoder layer, as calls that can be timed.

A layer of that form is x -> LayerNorm -> query/key/value product -> rotary positions on the
queries and keys -> differential attention -> output product -> norm, gate, residual and the
next norm in one step.  The three operators between its matrix products are called here one at
a time, as a program does that keeps a context, its weights and its buffers:

  rotary     rotated queries and keys of a batch of token rows
  attention  differential attention of query rows over the token rows of their frames
  norm       norm of a block's output, gate, scaled residual, and the norm in front of the next

With ``own`` false ``run`` computes the same from elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

EPS = 1e-5
# widths and heads of the encoder's configurations: (d_model, heads)
_MODELS = [(64, 2), (256, 8), (384, 6), (768, 12)]


# ---- cases -----------------------------------------------------------------------------
def _rotary(name, width, heads, rows, dtype="bf16", axes=2, part=1.0, interleaved=False, far=0, factor=1.0, by_parts=False):
    """`far`: the largest position of one axis; 0: cell centres of a frame, two axes."""
    c = {"op": "rotary", "width": width, "heads": heads, "rows": rows, "dtype": dtype, "axes": axes, "part": part,
         "interleaved": interleaved, "far": far, "factor": factor, "by_parts": by_parts}
    return dict(c, name=name) if name else c


def _attention(name, width, heads, frames, lo, hi, queries=0, dtype="bf16", masked=0.0, norm=True):
    """Frames of lo..hi tokens; `queries` rows a frame read them (0: the tokens themselves do).  `masked`: share
    of the tokens that no query may read; then the first of several frames has none left."""
    c = {"op": "attention", "width": width, "heads": heads, "frames": frames, "tokens_lo": lo, "tokens_hi": hi,
         "queries": queries, "dtype": dtype, "masked": masked, "norm": norm}
    return dict(c, name=name) if name else c


def _norm(name, width, rows, frames=1, dtype="bf16", post="rms", pre="layer", gate="shared", scale=1.0):
    c = {"op": "norm", "width": width, "rows": rows, "frames": frames, "dtype": dtype, "post": post, "pre": pre,
         "gate": gate, "scale": scale}
    return dict(c, name=name) if name else c


def listed():
    return [
        # Object queries of one frame in a decoder layer: the smallest call, latency.
        _rotary("rotary_queries", 256, 8, 300),
        # The tokens of four high-resolution frames, partly refined, two axes, pairs half a head apart.
        _rotary("rotary_high_res", 384, 6, 24470),
        # A long sequence of track tokens in the check mode: far positions of one axis, half of every head rotated
        # in neighbouring pairs, frequencies stretched by parts beyond the trained length.
        _rotary("rotary_long_f32", 768, 12, 16063, "f32", axes=1, part=0.5, interleaved=True, far=1_000_003, factor=8.0,
                by_parts=True),
        # One tiny fp32 frame: the check mode on a few tokens.
        _attention("attention_tiny_f32", 64, 2, 1, 43, 43, dtype="f32"),
        # Six cameras with different refined shares, head width 32.
        _attention("attention_six", 256, 8, 6, 400, 1600),
        # The worst case of a scheduler: eight high-resolution frames, everything refined.
        _attention("attention_high_res", 384, 6, 8, 6400, 6400),
        # Three granularities on twelve cameras, ragged.
        _attention("attention_three_level", 768, 12, 12, 523, 2467),
        # Object queries of four frames over their tokens, a third of them masked (the vehicle's own body,
        # occluded sensors), one frame without any.
        _attention("attention_queries", 384, 6, 4, 1600, 6400, queries=300, masked=0.33),
        # One pooling query over the tokens that a long clip has left: a single row, many keys.
        _attention("attention_pooled", 768, 12, 1, 50_001, 50_001, queries=1),
        # One camera's coarse grid: few rows, latency.
        _norm("norm_one_camera", 256, 400),
        # A gate for every frame, LayerNorm on both sides, scaled residual, in the check mode.
        _norm("norm_frames_f32", 768, 5003, frames=12, dtype="f32", post="layer", gate="frame", scale=1.25),
        # Coarse and fine sequences of eight high-resolution frames together.
        _norm("norm_high_res", 384, 64000, frames=8),
    ]


def draw(rng: random.Random):
    def log_uniform(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    width, heads = rng.choice(_MODELS)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    op = rng.choice(["rotary", "attention", "attention", "norm"])
    if op == "rotary":
        far = 0 if rng.random() < 0.6 else log_uniform(1000, 1_000_003)
        return _rotary(None, width, heads, min(log_uniform(1, 60_000), 18_000_000 // width), dtype, 2 if far == 0 else 1,
                       rng.choice([1.0, 1.0, 0.5]), rng.random() < 0.5, far, rng.choice([1.0, 4.0, 8.0]), rng.random() < 0.5)
    if op == "norm":
        return _norm(None, width, min(log_uniform(1, 60_000), 24_000_000 // width), rng.randint(1, 16), dtype,
                     rng.choice(["rms", "layer", "none"]), rng.choice(["layer", "rms", "none"]),
                     rng.choice(["shared", "frame", "none"]), rng.choice([1.0, 1.25]))
    frames = max(1, log_uniform(0.7, 12.4))
    queries = rng.choice([0, 0, 0, 1, log_uniform(2, 600)])
    hi = log_uniform(8, 6400 if queries != 1 else 60_000)
    if dtype == "f32":
        hi, queries = min(hi, 2000), min(queries, 200)
    if queries == 1:
        frames = min(frames, max(1, 100_000 // hi))
    lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
    c = _attention(None, width, heads, frames, lo, hi, queries, dtype, rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.9), 2)]),
                   rng.random() < 0.8)
    most = work(listed()[5])["flops"]
    if dtype == "f32":
        most //= 20
    while c["frames"] > 1 and work(c)["flops"] > most:
        c["frames"] -= 1
    while work(c)["flops"] > most:
        c["tokens_hi"] = c["tokens_hi"] * 3 // 4
        c["tokens_lo"] = min(c["tokens_lo"], c["tokens_hi"])
    return c


def _tokens(case):
    """Tokens of every frame, spread over the case's range, every second one odd."""
    n, lo, hi = case["frames"], case["tokens_lo"], case["tokens_hi"]
    return [min(hi, (lo + (hi - lo) * i // max(1, n - 1)) | (i & 1)) for i in range(n)]


def _queries(case):
    return [case["queries"]] * case["frames"] if case["queries"] else _tokens(case)


def _open_keys(case):
    """About how many tokens of every frame a query may read."""
    t = [n * (1.0 - case["masked"]) for n in _tokens(case)]
    if case["masked"] and len(t) > 1:
        t[0] = 0.0
    return t


def work(case):
    d, size = case["width"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "rotary":
        rows = case["rows"]
        pairs = case["heads"] * (_rot_dim(case) // 2)
        return {"bytes": rows * (4 * d * size + 4 * case["axes"]), "flops": 2 * rows * pairs * 6}
    if case["op"] == "norm":
        outs = size if case["pre"] != "none" else 0
        return {"bytes": case["rows"] * d * (8 + size + outs), "flops": case["rows"] * d * 14}
    dh, heads = d // case["heads"], case["heads"] // 2
    q, k = _queries(case), _open_keys(case)
    # two logits and one product with the values for every query, key and differential head
    flops = sum(a * b for a, b in zip(q, k)) * heads * 8 * dh
    return {"bytes": int(size * d * (2 * sum(q) + 2 * sum(k))) + (sum(_tokens(case)) if case["masked"] else 0),
            "flops": int(flops)}


# ---- inputs ----------------------------------------------------------------------------
def _rot_dim(case):
    return int(case["width"] // case["heads"] * case["part"])


def _frequencies(case):
    """Frequencies of the pairs of a head, in double precision on the host."""
    n, axes = _rot_dim(case) // 2, case["axes"]
    base, trained, keep, stretch = 10000.0, 4096.0, 32.0, 1.0
    out = []
    for i in range(n):
        f = base ** (-(i % (n // axes)) * axes / n)
        if case["by_parts"]:
            w = (trained * f / (2 * math.pi) - stretch) / (keep - stretch)
            w = min(1.0, max(0.0, w))
            f = f * (w + (1.0 - w) / case["factor"])
        else:
            f = f / case["factor"]
        out.append(f)
    return out


def _inputs(case, seed):
    """What the program has in hand, whichever side computes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, heads = case["width"], case["heads"] if "heads" in case else 0
    act = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    s = {}
    if case["op"] == "rotary":
        rows = case["rows"]
        # the projection's rows: queries, keys and values side by side
        s["qkv"] = normal(rows, 3 * d).to(act)
        if case["far"]:
            at = torch.rand(rows, 1, generator=g, device="cuda", dtype=torch.float64) * case["far"]
            s["pos"] = at.floor().float()
        else:
            # cell centres on a grid of half cells
            s["pos"] = torch.randint(0, 160, (rows, 2), generator=g, device="cuda").float() + 0.5
        s["q_scale"] = 1.4426950408889634 / math.sqrt(d // heads)
    elif case["op"] == "norm":
        rows = case["rows"]
        s["x"] = normal(rows, d, std=2.0)
        s["block"] = normal(rows, d, std=0.7).to(act)
        for name in ("post", "pre"):
            s[name + "_g"] = 1.0 + normal(d, std=0.1) if case[name] != "none" else None
            s[name + "_b"] = normal(d, std=0.1) if case[name] == "layer" else None
        frames = case["frames"]
        s["gate"] = normal(frames, d, std=0.3) if case["gate"] == "frame" else normal(d, std=0.3) if case["gate"] == "shared" else None
        cut = sorted(torch.randint(0, rows + 1, (frames - 1,), generator=g, device="cuda").tolist())
        s["cu"] = torch.tensor([0, *cut, rows], dtype=torch.int32, device="cuda") if case["gate"] == "frame" else None
    else:
        nq, nk = _queries(case), _tokens(case)
        if case["queries"]:
            s["q"] = normal(sum(nq), d, std=1.5).to(act)
            kv = torch.cat([normal(sum(nk), d, std=1.5), normal(sum(nk), d)], 1).to(act)
            s["k"], s["v"] = kv[:, :d], kv[:, d:]
        else:
            qkv = torch.cat([normal(sum(nk), 2 * d, std=1.5), normal(sum(nk), d)], 1).to(act)
            s["q"], s["k"], s["v"] = qkv[:, :d], qkv[:, d:2 * d], qkv[:, 2 * d:]
        for name, n in (("cu_q", nq), ("cu_k", nk)):
            s[name] = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")
        s["lengths"] = (nq, nk)
        s["mask"] = None
        if case["masked"]:
            s["mask"] = (torch.rand(sum(nk), generator=g, device="cuda") >= case["masked"]).to(torch.uint8)
            if len(nk) > 1:
                s["mask"][:nk[0]] = 0
        s["lambda"] = 0.2 + 0.7 * torch.rand(heads // 2, generator=g, device="cuda")
        s["head_g"] = 0.5 + normal(2 * (d // heads), std=0.05) if case["norm"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    d = case["width"]
    act = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if case["op"] == "rotary":
        s["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        s["out"] = torch.empty(case["rows"], 2 * d, dtype=act, device="cuda")
    elif case["op"] == "norm":
        s["x_out"] = torch.empty_like(s["x"])
        s["normed"] = torch.empty(case["rows"], d, dtype=act, device="cuda") if case["pre"] != "none" else None
    else:
        s["out"] = torch.empty(s["q"].shape[0], d, dtype=act, device="cuda")
    if own:
        _own_state(case, s)
    return s


# ---- one pass --------------------------------------------------------------------------
def run(s):
    if own:
        return _own_run(s)
    return {"rotary": _plain_rotary, "norm": _plain_norm, "attention": _plain_attention}[s["case"]["op"]](s)


def _own_state(case, s):
    """The context of a program with this model, and the frequencies as the library lays them out."""
    from paper_2505_23317_amd import cfdetr, synth

    d, op = case["width"], case["op"]
    heads = case.get("heads") or dict(_MODELS)[d]
    rows = max(s["q"].shape[0], s["k"].shape[0]) if op == "attention" else case["rows"]
    frames = case.get("frames", 1)
    cfg = synth.Config("operators", frames, 32, 32, (32,), d, heads, 1, 2 * d, "bf16")
    s["enc"] = cfdetr.Encoder(cfg, synth.make_weights(cfg, 1), act_dtype=case["dtype"], max_batch=frames,
                              max_tokens_total=max(rows, frames))
    if op == "rotary":
        s["params"] = cfdetr.rotary_params(rot_dim=_rot_dim(case), n_axes=case["axes"], interleaved=case["interleaved"],
                                           factor=case["factor"], trained_len=4096.0 if case["by_parts"] else 0.0,
                                           keep_turns=32.0, stretch_turns=1.0)
        s["freq"] = torch.tensor(cfdetr.cfdetr_rotary_frequencies(s["params"]), dtype=torch.float64, device="cuda")
    elif op == "norm":
        s["params"] = cfdetr.norm_residual_params(post=case["post"], pre=case["pre"], post_g=s["post_g"], post_b=s["post_b"],
                                                  pre_g=s["pre_g"], pre_b=s["pre_b"], gate=s["gate"], cu_seqlens=s["cu"],
                                                  res_scale=case["scale"])


def _own_run(s):
    case, enc = s["case"], s["enc"]
    d = case["width"]
    if case["op"] == "rotary":
        qkv, out = s["qkv"], s["out"]
        enc.rotary(s["params"], s["freq"], s["pos"], qkv[:, :d], out[:, :d], qkv[:, d:2 * d], out[:, d:], q_scale=s["q_scale"])
        return out
    if case["op"] == "norm":
        enc.norm_residual(s["params"], s["x"], s["block"], s["x_out"], s["normed"])
        return (s["x_out"],) if s["normed"] is None else (s["x_out"], s["normed"])
    enc.diff_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["lambda"], s["out"], head_g=s["head_g"], key_mask=s["mask"])
    return s["out"]


def _plain_rotary(s):
    case, out = s["case"], s["out"]
    d, heads, rows = case["width"], case["heads"], case["rows"]
    n = _rot_dim(case) // 2
    per = n // case["axes"]
    at = s["pos"].double().repeat_interleave(per, dim=1)
    angle = at * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for i, scale in ((0, s["q_scale"]), (1, 1.0)):
        x = s["qkv"][:, i * d:(i + 1) * d].float().view(rows, heads, d // heads)
        y = x.clone()
        if case["interleaved"]:
            a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
            y[..., 0:2 * n:2], y[..., 1:2 * n:2] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = x[..., :n], x[..., n:2 * n]
            y[..., :n], y[..., n:2 * n] = a * cos - b * sin, a * sin + b * cos
        out[:, i * d:(i + 1) * d] = (y * scale).reshape(rows, d).to(out.dtype)
    return out


def _normed(x, kind, g, b):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x * (x * x).mean(-1, keepdim=True).add(EPS).rsqrt() * g
    return y + b if kind == "layer" else y


def _plain_norm(s):
    case = s["case"]
    y = _normed(s["block"].float(), case["post"], s["post_g"], s["post_b"])
    if case["gate"] == "shared":
        y = y * s["gate"]
    elif case["gate"] == "frame":
        y = y * s["gate"].repeat_interleave(s["cu"].diff().long(), dim=0, output_size=case["rows"])
    x = s["x"] * case["scale"] + y
    if case["pre"] == "none":
        return (x,)
    return x, _normed(x, case["pre"], s["pre_g"], s["pre_b"]).to(s["block"].dtype)


def _plain_attention(s):
    case, out = s["case"], s["out"]
    d = case["width"]
    dh, heads = d // case["heads"], case["heads"] // 2
    scale = 1.0 / math.sqrt(dh)
    q0 = k0 = 0
    for nq, nk in zip(*s["lengths"]):
        q = s["q"][q0:q0 + nq].float().view(nq, 2 * heads, dh).transpose(0, 1).contiguous() * scale
        k = s["k"][k0:k0 + nk].float().view(nk, 2 * heads, dh).permute(1, 2, 0).contiguous()
        v = s["v"][k0:k0 + nk].float().view(nk, heads, 2 * dh).transpose(0, 1).contiguous()
        mask = None if s["mask"] is None else s["mask"][k0:k0 + nk] != 0
        for h in range(heads):
            logits = torch.bmm(q[2 * h:2 * h + 2], k[2 * h:2 * h + 2])
            if mask is not None:
                logits = logits.masked_fill(~mask, -math.inf)
            p = (logits - logits.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
            p = p / p.sum(-1, keepdim=True).clamp_min(1e-30)
            o = torch.mm(p[0] - s["lambda"][h] * p[1], v[h])
            if s["head_g"] is not None:
                o = o * (o * o).mean(-1, keepdim=True).add(EPS).rsqrt() * s["head_g"]
            out[q0:q0 + nq, 2 * h * dh:2 * (h + 1) * dh] = o.to(out.dtype)
        q0 += nq
        k0 += nk
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    return _exact_attention(case, s)


def _exact_rotary(case, s):
    """Every pair as a complex number, turned by its angle."""
    d, heads, rows = case["width"], case["heads"], case["rows"]
    r = _rot_dim(case)
    n = r // 2
    freq = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    axis = torch.arange(n, device="cuda") * case["axes"] // n
    angle = s["pos"].double()[:, axis] * freq
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    parts = []
    for i, scale in ((0, s["q_scale"]), (1, 1.0)):
        x = s["qkv"][:, i * d:(i + 1) * d].double().reshape(rows, heads, d // heads)
        head, rest = x[..., :r], x[..., r:]
        pairs = head.reshape(rows, heads, n, 2) if case["interleaved"] else head.reshape(rows, heads, 2, n).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.reshape(rows, heads, r) if case["interleaved"] else z.transpose(-1, -2).reshape(rows, heads, r)
        parts.append(torch.cat([z, rest], -1).reshape(rows, d) * scale)
    return torch.cat(parts, 1)


def _exact_norm(case, s):
    def norm(x, kind, g, b):
        if kind == "layer":
            mean, var = x.mean(1, keepdim=True), x.var(1, unbiased=False, keepdim=True)
            return (x - mean) / torch.sqrt(var + EPS) * g.double() + b.double()
        if kind == "rms":
            return x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS) * g.double()
        return x

    y = norm(s["block"].double(), case["post"], s["post_g"], s["post_b"])
    if case["gate"] != "none":
        gate = s["gate"].double()
        if case["gate"] == "frame":
            row = torch.arange(case["rows"], device="cuda")
            gate = gate[torch.searchsorted(s["cu"][1:].long(), row, right=True)]
        y = y * gate
    x = case["scale"] * s["x"].double() + y
    return (x,) if case["pre"] == "none" else (x, norm(x, case["pre"], s["pre_g"], s["pre_b"]))


def _exact_attention(case, s):
    d, heads = case["width"], case["heads"] // 2
    dh = d // case["heads"]
    out = torch.zeros(s["q"].shape[0], d, dtype=torch.float64, device="cuda")
    cu_q, cu_k = s["cu_q"].tolist(), s["cu_k"].tolist()
    for f in range(case["frames"]):
        keys = torch.arange(cu_k[f], cu_k[f + 1], device="cuda")
        if s["mask"] is not None:
            keys = keys[s["mask"][keys] != 0]
        if keys.numel() == 0:
            continue
        k, v = s["k"][keys].double(), s["v"][keys].double()
        for a in range(cu_q[f], cu_q[f + 1], 2048):
            b = min(a + 2048, cu_q[f + 1])
            q = s["q"][a:b].double()
            for h in range(heads):
                c = 2 * h * dh
                maps = [torch.softmax((q[:, c + m * dh:c + (m + 1) * dh] @ k[:, c + m * dh:c + (m + 1) * dh].t()) * dh ** -0.5, 1)
                        for m in (0, 1)]
                o = (maps[0] - s["lambda"][h].double() * maps[1]) @ v[:, c:c + 2 * dh]
                if s["head_g"] is not None:
                    o = o / torch.sqrt(o.square().mean(1, keepdim=True) + EPS) * s["head_g"].double()
                out[a:b, c:c + 2 * dh] = o
    return out
