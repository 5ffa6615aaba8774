"""The operators of a paged stream memory, as calls that can be timed.

A memory keeps the keys and values of tokens beyond the call that made them: those of the last frames of a camera,
of an object's track, of a clip.  It is cut into pages that streams take and give back; how many tokens a stream has
is known on the GPU alone.  Its operators are called here one at a time, as a program does that keeps a context and
its buffers:

  advance    tokens forgotten and tokens new: pages given back and taken, the new tokens' slots
  rotary     queries and keys turned by positions of three axes (time, row, column)
  append     new keys (turned on the way) and values written into their slots
  attention  one new token of every stream over all that its stream holds

With ``own`` false ``run`` computes the same from elementary torch operations, in 32 bits (angles in 64).
"""
import math
import random

import numpy as np
import torch

own = False

# widths and heads of the encoder's configurations: (d_model, heads), and how many key heads they may share
_MODELS = [(64, 2), (256, 8), (384, 6), (768, 12)]
_KEY_HEADS = {2: (2, 1), 8: (8, 4, 2, 1), 6: (6, 3, 2, 1), 12: (12, 6, 4, 3, 2, 1)}


# ---- cases -----------------------------------------------------------------------------
def _advance(name, streams, held, new, page, ended=0.0, window=False):
    """held, new: the fewest and the most tokens that a stream holds and gets.  ended: share of the streams whose
    tokens are all forgotten first.  window: every stream forgets as many tokens as it gets."""
    c = {"op": "advance", "streams": streams, "held_lo": held[0], "held_hi": held[1], "new_lo": new[0], "new_hi": new[1],
         "page": page, "ended": ended, "window": window}
    return dict(c, name=name) if name else c


def _rotary(name, width, heads, key_heads, rows, dtype="bf16", part=1.0, interleaved=False, in_turn=False, shared=False, far=1000):
    """far: the largest position in time.  in_turn: the axes' pairs one after the other, not in blocks.  shared: one
    ladder of frequencies over the whole head, not one for every axis."""
    c = {"op": "rotary", "width": width, "heads": heads, "key_heads": key_heads, "rows": rows, "dtype": dtype, "part": part,
         "interleaved": interleaved, "in_turn": in_turn, "shared": shared, "far": far}
    return dict(c, name=name) if name else c


def _append(name, width, heads, key_heads, rows, page, dtype="bf16", turned=True, padding=0.0):
    """padding: share of the rows that have no slot."""
    c = {"op": "append", "width": width, "heads": heads, "key_heads": key_heads, "rows": rows, "page": page, "dtype": dtype,
         "turned": turned, "padding": padding}
    return dict(c, name=name) if name else c


def _attention(name, width, heads, key_heads, streams, held, page, dtype="bf16", masked=0.0):
    """masked: share of the tokens that are not read; then the first of several streams has none left."""
    c = {"op": "attention", "width": width, "heads": heads, "key_heads": key_heads, "streams": streams, "held_lo": held[0],
         "held_hi": held[1], "page": page, "dtype": dtype, "masked": masked}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token for each of 300 tracked objects: the smallest call, latency.
        _advance("advance_tracks", 300, (1, 700), (1, 1), 16),
        # The tokens of a new frame of six cameras, differently refined; as many of the oldest are forgotten.
        _advance("advance_cameras", 6, (4000, 16000), (400, 1600), 64, window=True),
        # Many tracks, a quarter of them lost and replaced by clips that are read in at once.
        _advance("advance_refill", 1024, (100, 3000), (1, 1200), 32, ended=0.25),
        # Track tokens of one frame: latency.
        _rotary("rotary_tracks", 256, 8, 8, 300),
        # Tokens of four high-resolution frames, partly refined, key heads shared by three query heads each.
        _rotary("rotary_frames", 384, 6, 2, 24470),
        # A long clip in the check mode: far times, half of every head rotated in neighbouring pairs, axes in turn.
        _rotary("rotary_clip_f32", 768, 12, 12, 16063, "f32", part=0.5, interleaved=True, in_turn=True, shared=True, far=1_000_003),
        # The tracks' tokens into their pages.
        _append("append_tracks", 256, 8, 8, 300, 16),
        # Three granularities on twelve cameras, a batch whose last rows are padding.
        _append("append_frames", 768, 12, 12, 24470, 64, padding=0.1),
        # The check mode on the memory of one short track.
        _attention("attention_track_f32", 64, 2, 2, 1, (43, 43), 16, "f32"),
        # Every tracked object's token over its own past, a few to many frames.
        _attention("attention_tracks", 256, 8, 8, 300, (1, 900), 16),
        # A clip's pooling token over all that the clip has left: a single row, many keys.
        _attention("attention_clip", 768, 12, 12, 1, (200_003, 200_003), 64),
        # A token for each of 24 cameras over their last frames; six query heads share a key head; a fifth of the
        # tokens masked (the vehicle's own body, occluded sensors), one camera without any left.
        _attention("attention_cameras", 768, 12, 2, 24, (8000, 64000), 64, masked=0.2),
    ]


def _log_uniform(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng: random.Random):
    op = rng.choice(["advance", "rotary", "append", "attention", "attention"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    if op == "advance":
        streams, held = _log_uniform(rng, 1, 1500), _log_uniform(rng, 1, 60_000)
        new = _log_uniform(rng, 1, 4000)
        # no more tokens than the largest listed case has
        held, new = max(1, min(held, 3_000_000 // streams)), max(1, min(new, 1_000_000 // streams))
        kind = rng.choice(["grow", "window", "ended"])
        return _advance(None, streams, (rng.randint(0, held), held), (rng.choice([0, 1, new]), new), page,
                        round(rng.uniform(0.05, 1.0), 2) if kind == "ended" else 0.0, kind == "window")
    width, heads = rng.choice(_MODELS)
    key_heads = rng.choice((heads,) + _KEY_HEADS[heads])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if op == "rotary":
        return _rotary(None, width, heads, key_heads, min(_log_uniform(rng, 1, 60_000), 12_000_000 // width), dtype, rng.choice([1.0, 1.0, 0.5]),
                       rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5, _log_uniform(rng, 10, 1_000_003))
    if op == "append":
        return _append(None, width, heads, key_heads, min(_log_uniform(rng, 1, 60_000), 18_000_000 // width), page, dtype,
                       rng.random() < 0.7, rng.choice([0.0, round(rng.uniform(0.01, 0.9), 2)]))
    streams = _log_uniform(rng, 1, 512)
    held = _log_uniform(rng, 1, 200_000)
    c = _attention(None, width, heads, key_heads, streams, (int(held * rng.uniform(0.0, 1.0)), held), page, dtype,
                   rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.9), 2)]))
    most = work(listed()[10])
    while any(work(c)[k] > most[k] for k in most):
        c["streams"] = max(1, c["streams"] * 3 // 4)
        c["held_hi"] = max(1, c["held_hi"] * 7 // 8)
        c["held_lo"] = min(c["held_lo"], c["held_hi"])
    return c


def _spread(n, lo, hi):
    """Lengths from lo to hi, more short ones than long ones, every second odd."""
    return [max(lo, min(hi, int(lo + (hi - lo) * (i / max(1, n - 1)) ** 2) | (i & 1))) for i in range(n)]


def _held(case):
    n = case["streams"]
    return _spread(n, case["held_lo"], case["held_hi"]) if n > 1 else [case["held_hi"]]


def _news(case):
    n = case["streams"]
    return _spread(n, case["new_lo"], case["new_hi"])[::-1] if n > 1 else [case["new_hi"]]


def _ended(case):
    """Every k-th stream has ended."""
    n, share = case["streams"], case["ended"]
    return [int((i + 1) * share) > int(i * share) for i in range(n)]


def work(case):
    op = case["op"]
    if op == "advance":
        n, p = case["streams"], case["page"]
        taken = given = kept = 0
        for h, w, e in zip(_held(case), _news(case), _ended(case)):
            d = h if e else min(h, w) if case["window"] else 0
            taken += (h - d + w + p - 1) // p - (h - d + p - 1) // p
            given += d // p
            kept += (h - d + p - 1) // p if e or case["window"] else 0
        # a stream's span, offset and what it forgets; a page's number read and written; kept numbers where the new
        # table is another one
        moved = case["window"] or case["ended"] > 0
        return {"bytes": n * (24 if moved else 20) + 4 * sum(_news(case)) + 8 * (taken + given) + (8 * kept if moved else 0), "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    dh = case["width"] // case["heads"]
    keys = dh * case["key_heads"]
    if op == "rotary":
        pairs = (case["heads"] + case["key_heads"]) * _rot_dim(case) // 2
        return {"bytes": case["rows"] * (2 * size * (case["width"] + keys) + 12), "flops": case["rows"] * pairs * 6}
    if op == "append":
        real = case["rows"] - int(case["rows"] * case["padding"])
        turn = case["turned"]
        return {"bytes": real * (4 * size * keys + 4 + (12 if turn else 0)) + 4 * (case["rows"] - real),
                "flops": real * keys * 3 if turn else 0}
    held = sum(_held(case))
    if case["masked"] and case["streams"] > 1:
        held -= _held(case)[0]
    read = held * (1.0 - case["masked"])
    return {"bytes": int(read * 2 * keys * size) + 2 * case["streams"] * case["width"] * size + (sum(_held(case)) if case["masked"] else 0)
                     + 4 * (sum(_held(case)) // case["page"] + 3 * case["streams"]),
            "flops": int(read * 4 * case["width"])}


# ---- inputs ----------------------------------------------------------------------------
def _rot_dim(case):
    return int(case["width"] // case["heads"] * case.get("part", 1.0))


def _sections(case):
    """Pairs of time, row and column: a quarter, and what is left in halves."""
    n = _rot_dim(case) // 2
    t = n // 4
    return [t, (n - t) // 2, n - t - (n - t) // 2]


def _axes_and_frequencies(case):
    """Axis and frequency of every pair of a head, in double precision on the host."""
    sections = _sections(case)
    n = sum(sections)
    if case.get("in_turn"):
        left, axis = list(sections), []
        while len(axis) < n:
            for a in range(3):
                if left[a]:
                    left[a] -= 1
                    axis.append(a)
    else:
        axis = [a for a in range(3) for _ in range(sections[a])]
    freq, seen = [], [0, 0, 0]
    for i, a in enumerate(axis):
        freq.append(10000.0 ** (-i / n) if case.get("shared") else 10000.0 ** (-seen[a] / sections[a]))
        seen[a] += 1
    return axis, freq


def _streams_state(held, new, page, rng):
    """Streams that have taken and given back pages for a while: where they begin, which pages they hold, which are free."""
    held = np.asarray(held, dtype=np.int64)
    n = len(held)
    cols = int((int(held.max()) + int(max(new)) + page - 1) // page + 2)
    first = np.where(held > 0, rng.integers(0, cols * page, n), 0)
    lo, hi = first // page, (first + held + page - 1) // page
    count = np.where(held > 0, hi - lo, 0)
    used = int(count.sum())
    n_pages = sum(int(x + page - 1) // page + 1 for x in (*held, *new)) + 8
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((n, cols), -1, dtype=np.int32)
    row = np.repeat(np.arange(n), count)
    within = np.arange(used) - np.repeat(np.cumsum(count) - count, count)
    table[row, (lo[row] + within) % cols] = ids[:used]
    head = int(rng.integers(0, n_pages))
    free = np.full(n_pages, -1, dtype=np.int32)
    free[(head + np.arange(n_pages - used)) % n_pages] = ids[used:]
    return {"span": np.stack([first, held], 1).astype(np.int32), "table": table, "free": free,
            "pool": np.array([head, n_pages - used], dtype=np.int32), "n_pages": n_pages, "cols": cols}


def _slots_of(state, page, b):
    """Slots of all tokens that stream b holds, in order (host)."""
    first, held = (int(x) for x in state["span"][b])
    at = first + np.arange(held, dtype=np.int64)
    return state["table"][b, (at // page) % state["cols"]].astype(np.int64) * page + at % page


def _groups(lengths):
    """Neighbouring streams that are taken together: at most 2^18 tokens with their padding."""
    groups, a = [], 0
    for b in range(1, len(lengths) + 1):
        if b == len(lengths) or (b + 1 - a) * max(lengths[a:b + 1]) > 1 << 18:
            groups.append((a, b))
            a = b
    return groups


def _inputs(case, seed):
    """What the program has in hand, whichever side computes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    op, s = case["op"], {}
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if op == "advance":
        page = case["page"]
        order = rng.permutation(case["streams"])
        held, new, ended = (np.asarray(f(case))[order] for f in (_held, _news, _ended))
        host = _streams_state(held, new, page, rng)
        s.update({k: up(host[k]) for k in ("span", "table", "free", "pool")})
        s.update({k: host[k] for k in ("n_pages", "cols")})
        s["n_new"] = int(new.sum())
        s["cu"] = up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        s["drop"] = None
        if case["window"] or case["ended"] > 0:
            s["drop"] = up(np.where(ended, held, np.minimum(held, new) if case["window"] else 0).astype(np.int32))
        return s
    act = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    d, keys = case["width"], case["width"] // case["heads"] * case["key_heads"]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(act)

    if op in ("rotary", "append"):
        rows = case["rows"]
        # the projection's rows: queries, keys and values side by side
        s["qkv"] = normal(rows, d + 2 * keys)
        time = (torch.rand(rows, 1, generator=g, device="cuda", dtype=torch.float64) * case.get("far", 1000)).floor().float()
        # cell centres on a grid of half cells
        cell = torch.randint(0, 160, (rows, 2), generator=g, device="cuda").float() + 0.5
        s["pos"] = torch.cat([time, cell], 1).contiguous()
        s["q_scale"] = 1.4426950408889634 / math.sqrt(d // case["heads"])
        if op == "append":
            page = case["page"]
            real = rows - int(rows * case["padding"])
            n_pages = (real + page - 1) // page + 1 + rows // (4 * page)
            # as pages were taken: tokens in order inside a page, pages anywhere
            ids = rng.permutation(n_pages)
            at = np.arange(real) + int(rng.integers(0, page))
            slots = np.full(rows, -1, dtype=np.int32)
            slots[:real] = ids[at // page] * page + at % page
            s["slots"], s["n_pages"] = up(slots), n_pages
            s["k_cache"], s["v_cache"] = (normal(n_pages * page, keys) for _ in range(2))
        return s
    page = case["page"]
    held = np.asarray(_held(case))
    host = _streams_state(held, [0], page, rng)
    s.update({k: up(host[k]) for k in ("span", "table")})
    s.update({k: host[k] for k in ("n_pages", "cols")})
    s["q"] = normal(case["streams"], d, std=1.5)
    s["k_cache"], s["v_cache"] = normal(host["n_pages"] * page, keys, std=1.5), normal(host["n_pages"] * page, keys)
    s["slots_of"] = [up(_slots_of(host, page, b)) for b in range(case["streams"])]
    s["mask"] = None
    if case["masked"]:
        s["mask"] = (torch.rand(host["n_pages"] * page, generator=g, device="cuda") >= case["masked"]).to(torch.uint8)
        if case["streams"] > 1:
            s["mask"][s["slots_of"][0]] = 0
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if op == "advance":
        # what a step writes beside the old state, so that the step can be taken again; where nothing is forgotten the
        # table is added to in place
        s["span_out"], s["pool_out"] = torch.empty_like(s["span"]), torch.empty_like(s["pool"])
        s["table_out"] = s["table"] if s["drop"] is None else torch.full_like(s["table"], -1)
        s["slots"] = torch.empty(s["n_new"], dtype=torch.int32, device="cuda")
    else:
        act = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        if op in ("rotary", "append"):
            axis, freq = _axes_and_frequencies(case)
            s["axis"] = torch.tensor(axis, dtype=torch.uint8, device="cuda")
            s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        if op == "rotary":
            keys = case["width"] // case["heads"] * case["key_heads"]
            s["out"] = torch.empty(case["rows"], case["width"] + keys, dtype=act, device="cuda")
        if op == "attention":
            s["lengths"] = _held(case)
            s["groups"] = _groups(s["lengths"])
            s["out"] = torch.empty(case["streams"], case["width"], dtype=act, device="cuda")
    if own:
        _own_state(case, s)
    return s


# ---- one pass --------------------------------------------------------------------------
def run(s):
    if own:
        return _own_run(s)
    return {"advance": _plain_advance, "rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention}[s["case"]["op"]](s)


def _context(width, heads, dtype, memory, made={}):
    """The context of a program with this model and memory: made once, whatever inputs come (sizes and work space are all it has of them)."""
    from paper_2505_23317_amd import cfdetr, synth

    key = (width, heads, dtype, memory)
    if key not in made:
        cfg = synth.Config("operators", 1, 32, 32, (32,), width, heads, 1, 2 * width, "bf16")
        made[key] = cfdetr.Encoder(cfg, synth.make_weights(cfg, 1), act_dtype=dtype, max_batch=1, max_tokens_total=64)
        if memory:
            made[key].attach_memory(*memory)
    return made[key]


def _rotation(rot_dim, pairs, in_turn, shared, interleaved, made={}):
    """Parameters of a rotation and the pairs' table as the library lays it out, which depend on no input."""
    from paper_2505_23317_amd import cfdetr

    key = (rot_dim, pairs, in_turn, shared, interleaved)
    if key not in made:
        params = cfdetr.rotary_axes_params(rot_dim=rot_dim, pairs=pairs, in_turn=in_turn, shared_ladder=shared, interleaved=interleaved)
        freq, axis = cfdetr.cfdetr_rotary_axes_table(params)
        made[key] = (params, torch.tensor(freq, dtype=torch.float64, device="cuda"), torch.tensor(axis, dtype=torch.uint8, device="cuda"))
    return made[key]


def _own_state(case, s):
    op = case["op"]
    memory = None
    if op != "rotary":
        memory = (case["page"], s["n_pages"], s.get("cols", 1), case.get("streams", 1), case.get("key_heads"))
    s["enc"] = _context(case.get("width", 256), case.get("heads", 8), case.get("dtype", "bf16"), memory)
    if op in ("rotary", "append"):
        s["params"], s["freq"], s["axis"] = _rotation(_rot_dim(case), tuple(_sections(case)), case.get("in_turn", False),
                                                      case.get("shared", False), case.get("interleaved", False))


def _own_run(s):
    case, enc = s["case"], s["enc"]
    op = case["op"]
    if op == "advance":
        enc.memory_advance(s["cu"], s["span"], s["table"], s["pool"], s["free"], s["slots"], drop=s["drop"], span_out=s["span_out"],
                           table_out=s["table_out"], pool_out=s["pool_out"])
        return s["slots"], s["span_out"], s["table_out"], s["pool_out"], s["free"]
    if op == "attention":
        enc.memory_attention(s["q"], s["k_cache"], s["v_cache"], s["span"], s["table"], s["out"], key_mask=s["mask"])
        return s["out"]
    d, qkv = case["width"], s["qkv"]
    keys = d // case["heads"] * case["key_heads"]
    if op == "rotary":
        out = s["out"]
        enc.rotary_axes(s["params"], s["freq"], s["axis"], s["pos"], qkv[:, :d], out[:, :d], qkv[:, d:d + keys], out[:, d:],
                        q_scale=s["q_scale"])
        return out
    turn = (s["params"], s["freq"], s["axis"], s["pos"]) if case["turned"] else ()
    enc.memory_append(qkv[:, d:d + keys], qkv[:, d + keys:], s["slots"], s["k_cache"], s["v_cache"], *turn)
    return s["k_cache"], s["v_cache"]


def _plain_advance(s):
    page, cols, n_pages = s["case"]["page"], s["cols"], s["n_pages"]
    first, held = s["span"].long().unbind(1)
    new = s["cu"].long().diff()
    drop = torch.zeros_like(held) if s["drop"] is None else torch.minimum(s["drop"].long(), held)
    pages = lambda n: (n + page - 1) // page
    gone = drop == held
    lo = first // page
    first2, held2 = torch.where(gone, 0, first + drop), held - drop
    given = torch.where(gone, torch.where(held > 0, pages(first + held) - lo, 0), first2 // page - lo)
    first2 = torch.where(first2 >= cols * page, first2 - cols * page, first2)
    have = torch.where(gone, 0, pages(first2 + held2))      # page behind the last one held
    taken = pages(first2 + held2 + new) - have
    head, n_free = s["pool"].long().unbind()
    # numbers of a ring's places from a page on, for every stream
    col = torch.arange(cols, device="cuda")
    table, free = s["table"], s["free"]
    back = (col - lo[:, None]) % cols
    to = (head + n_free + (given.cumsum(0) - given)[:, None] + back) % n_pages
    ring = torch.cat([free, free[:1]])
    ring[torch.where(back < given[:, None], to, n_pages).flatten()] = table.flatten()
    ahead = (col - have[:, None]) % cols
    take = free[(head + (taken.cumsum(0) - taken)[:, None] + ahead) % n_pages]
    kept = (col - (first2 // page)[:, None]) % cols < torch.where(gone, 0, have - first2 // page)[:, None]
    out = torch.where(ahead < taken[:, None], take, torch.where(kept, table, s["table_out"]))
    row = torch.repeat_interleave(torch.arange(new.shape[0], device="cuda"), new, output_size=s["n_new"])
    at = (first2 + held2)[row] + torch.arange(s["n_new"], device="cuda") - s["cu"].long()[row]
    s["slots"].copy_(out[row, (at // page) % cols].long() * page + at % page)
    s["span_out"].copy_(torch.stack([first2, held2 + new], 1))
    s["pool_out"].copy_(torch.stack([(head + taken.sum()) % n_pages, n_free - taken.sum() + given.sum()]))
    s["table_out"].copy_(out)
    free.copy_(ring[:n_pages])
    return s["slots"], s["span_out"], s["table_out"], s["pool_out"], free


def _turned(x, case, s):
    """Rows of heads, their rotated features turned."""
    rows, n = x.shape[0], _rot_dim(case) // 2
    angle = s["pos"].double()[:, s["axis"].long()] * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float().view(rows, -1, case["width"] // case["heads"])
    y = x.clone()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case.get("interleaved") else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    return y.reshape(rows, -1)


def _plain_rotary(s):
    case, d, out = s["case"], s["case"]["width"], s["out"]
    keys = d // case["heads"] * case["key_heads"]
    out[:, :d] = (_turned(s["qkv"][:, :d], case, s) * s["q_scale"]).to(out.dtype)
    out[:, d:] = _turned(s["qkv"][:, d:d + keys], case, s).to(out.dtype)
    return out


def _plain_append(s):
    case, d = s["case"], s["case"]["width"]
    keys = d // case["heads"] * case["key_heads"]
    k, v = s["qkv"][:, d:d + keys], s["qkv"][:, d + keys:]
    if case["turned"]:
        k = _turned(k, case, s).to(k.dtype)
    real = s["slots"] >= 0
    at = s["slots"][real].long()
    s["k_cache"][at] = k[real]
    s["v_cache"][at] = v[real]
    return s["k_cache"], s["v_cache"]


def _plain_attention(s):
    case, out = s["case"], s["out"]
    dh, hk, page = case["width"] // case["heads"], case["key_heads"], case["page"]
    first, held = s["span"].long().unbind(1)
    table = s["table"].long()
    for a, b in s["groups"]:
        # streams of similar lengths, padded to the longest of them
        n, longest = b - a, max(1, max(s["lengths"][a:b]))
        t = torch.arange(longest, device="cuda")
        p = first[a:b, None] + t
        open_ = t < held[a:b, None]
        at = torch.where(open_, table[a:b].gather(1, (p // page) % s["cols"]) * page + p % page, 0)
        if s["mask"] is not None:
            open_ = open_ & (s["mask"][at] != 0)
        q = s["q"][a:b].float().view(n * hk, -1, dh) * dh ** -0.5
        k = s["k_cache"][at].float().view(n, longest, hk, dh).permute(0, 2, 3, 1).reshape(n * hk, dh, longest)
        v = s["v_cache"][at].float().view(n, longest, hk, dh).transpose(1, 2).reshape(n * hk, longest, dh)
        logits = torch.bmm(q, k.contiguous()).view(n, -1, longest).masked_fill(~open_[:, None], -math.inf)
        w = (logits - logits.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
        w = w / w.sum(-1, keepdim=True).clamp_min(1e-30)
        out[a:b] = torch.bmm(w.view(n * hk, -1, longest), v.contiguous()).reshape(n, -1).to(out.dtype)
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"advance": _exact_advance, "rotary": _exact_rotary, "append": _exact_append, "attention": _exact_attention}[case["op"]](case, s)


def _exact_advance(case, s):
    """Streams one after the other, pages one by one."""
    page, cols, n_pages = case["page"], s["cols"], s["n_pages"]
    span, table, free, pool, cu = (s[k].cpu().numpy().copy() for k in ("span", "table", "free", "pool", "cu"))
    drop = np.zeros(case["streams"], dtype=np.int64) if s["drop"] is None else s["drop"].cpu().numpy()
    table_out = table if s["drop"] is None else np.full_like(table, -1)
    old = table.copy()
    head, n_free = (int(x) for x in pool)
    tail, slots, given = head + n_free, np.empty(s["n_new"], dtype=np.int32), 0
    for b in range(case["streams"]):
        first, held = (int(x) for x in span[b])
        d, n = int(drop[b]), int(cu[b + 1] - cu[b])
        pages = list(range(first // page, (first + held + page - 1) // page)) if held else []
        left = pages if d == 0 else [] if d == held else [j for j in pages if (j + 1) * page > first + d]
        for j in pages[:len(pages) - len(left)]:
            free[tail % n_pages] = old[b, j % cols]
            tail += 1
            given += 1
        for j in left:
            table_out[b, j % cols] = old[b, j % cols]
        first, held = (0, 0) if d == held else (first + d, held - d)
        if first >= cols * page:
            first -= cols * page
            left = [j - cols for j in left]
        end = left[-1] + 1 if left else 0
        at = np.arange(first + held, first + held + n)
        while end * page < first + held + n:
            table_out[b, end % cols] = free[head % n_pages]
            head += 1
            n_free -= 1
            end += 1
        slots[cu[b]:cu[b + 1]] = table_out[b, (at // page) % cols] * page + at % page
        span[b] = first, held + n
    pool[:] = head % n_pages, n_free + given
    return tuple(torch.from_numpy(a).double().cuda() for a in (slots, span, table_out, pool, free))


def _exact_turned(x, case, s):
    """Every pair as a complex number, turned by its angle."""
    axis, freq = _axes_and_frequencies(case)
    n, rows, dh = len(axis), x.shape[0], case["width"] // case["heads"]
    angle = torch.stack([s["pos"][:, a].double() * f for a, f in zip(axis, freq)], 1)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    x = x.double().reshape(rows, -1, dh)
    head, rest = x[..., :2 * n], x[..., 2 * n:]
    pairs = head.unflatten(-1, (n, 2)) if case.get("interleaved") else head.unflatten(-1, (2, n)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.flatten(-2) if case.get("interleaved") else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, rest], -1).reshape(rows, -1)


def _exact_rotary(case, s):
    d = case["width"]
    keys = d // case["heads"] * case["key_heads"]
    return torch.cat([_exact_turned(s["qkv"][:, :d], case, s) * s["q_scale"], _exact_turned(s["qkv"][:, d:d + keys], case, s)], 1)


def _exact_append(case, s):
    d = case["width"]
    keys = d // case["heads"] * case["key_heads"]
    k, v = s["qkv"][:, d:d + keys].double(), s["qkv"][:, d + keys:].double()
    if case["turned"]:
        k = _exact_turned(k, case, s)
    out = []
    for cache, rows in ((s["k_cache"], k), (s["v_cache"], v)):
        cache = cache.double()
        have = torch.nonzero(s["slots"] >= 0).flatten()
        out.append(cache.index_copy(0, s["slots"][have].long(), rows[have]))
    return tuple(out)


def _exact_attention(case, s):
    dh = case["width"] // case["heads"]
    group = case["heads"] // case["key_heads"]
    out = torch.zeros(case["streams"], case["width"], dtype=torch.float64, device="cuda")
    for b, at in enumerate(s["slots_of"]):
        if s["mask"] is not None:
            at = at[s["mask"][at] != 0]
        if at.numel() == 0:
            continue
        for h in range(case["heads"]):
            c, kc = slice(h * dh, (h + 1) * dh), slice(h // group * dh, (h // group + 1) * dh)
            p = torch.softmax(s["k_cache"][at, kc].double() @ s["q"][b, c].double() / math.sqrt(dh), 0)
            out[b, c] = p @ s["v_cache"][at, kc].double()
    return out
