"""A paged stream memory in plain Python, page by page, and what its operators compute in 64 bits."""
import copy
import math

import numpy as np

import differential_reference as T


class State:
    """What cfdetr_memory_advance works on, as numpy arrays and integers."""

    def __init__(self, streams, page, n_pages, cols):
        self.page, self.n_pages, self.cols = page, n_pages, cols
        self.span = np.zeros((streams, 2), dtype=np.int32)
        self.table = np.full((streams, cols), -7, dtype=np.int32)
        self.pool = np.array([0, n_pages], dtype=np.int32)
        self.free = np.arange(n_pages, dtype=np.int32)

    def copy(self):
        return copy.deepcopy(self)

    def pages(self, b):
        """Positions' pages that a stream holds, oldest first."""
        first, held = (int(x) for x in self.span[b])
        return [] if held == 0 else list(range(first // self.page, (first + held - 1) // self.page + 1))

    def slots(self, b):
        first, held = (int(x) for x in self.span[b])
        return [int(self.table[b, p // self.page % self.cols]) * self.page + p % self.page for p in range(first, first + held)]

    def free_list(self):
        head, n = (int(x) for x in self.pool)
        return [int(self.free[(head + i) % self.n_pages]) for i in range(n)]

    def check(self):
        """Every page has one owner: a stream, at one place of its table, or the list of free ones."""
        owned = [int(self.table[b, j % self.cols]) for b in range(len(self.span)) for j in self.pages(b)]
        assert sorted(owned + self.free_list()) == list(range(self.n_pages))
        for b in range(len(self.span)):
            assert len(self.pages(b)) <= self.cols and 0 <= self.span[b, 0] < self.cols * self.page


def step(old, drop, new):
    """(state behind a step, slots of the new tokens), or None where the step is refused."""
    s, slots = old.copy(), []
    head, n_free = (int(x) for x in old.pool)
    back, front = [], 0
    for b in range(len(old.span)):
        first, held = (int(x) for x in old.span[b])
        d, n = int(drop[b]), int(new[b])
        if d < 0 or n < 0:
            return None
        pages = old.pages(b)
        if d >= held:
            gone, pages, first, held = pages, [], 0, 0
            back += [int(old.table[b, j % s.cols]) for j in gone]
        else:
            first, held = first + d, held - d
            back += [int(old.table[b, j % s.cols]) for j in pages if j < first // s.page]
            pages = [j for j in pages if j >= first // s.page]
            if first >= s.cols * s.page:
                first, pages = first - s.cols * s.page, [j - s.cols for j in pages]
        begin = first // s.page
        for p in range(first + held, first + held + n):
            j = p // s.page
            if j not in pages[-1:]:
                if front == n_free or j - begin >= s.cols:
                    return None
                s.table[b, j % s.cols] = old.free[(head + front) % s.n_pages]
                front += 1
                pages = [j]
            slots.append(int(s.table[b, j % s.cols]) * s.page + p % s.page)
        s.span[b] = first, held + n
    for i, page in enumerate(back):
        s.free[(head + n_free + i) % s.n_pages] = page
    s.pool[:] = (head + front) % s.n_pages, n_free - front + len(back)
    return s, slots


def random_step(rng, s, most_new):
    """What a step forgets and adds: nothing, a little, up to a page's end, everything, more than everything."""
    drop, new = [], []
    for b in range(len(s.span)):
        first, held = (int(x) for x in s.span[b])
        to_page = min(held, s.page - first % s.page)
        drop.append(int(rng.choice([0, 0, 1, to_page, held, 2 ** 31 - 1, rng.integers(0, held + 1)])))
        left = 0 if drop[-1] >= held else held - drop[-1]
        first = 0 if left == 0 else first + drop[-1]
        room = max(0, s.cols * s.page - first % s.page - left)
        fill = (-(first + left)) % s.page
        new.append(int(min(room, rng.choice([0, 0, 1, fill, fill + 1, rng.integers(0, most_new + 1)]))))
    return drop, new


# ---- attention ---------------------------------------------------------------------------
def attention(q, k_cache, v_cache, slots, heads, kv_heads, dtype, scale=None, mask=None):
    """(rows, bound of the error of the library's), both [B, d] in 64 bits; slots: those of every stream's tokens.

    Bound.  A logit's products (d_head of them, the scale) are rounded in 32 bits: off by (d_head + 4) 2^-24 times
    scale sum |q k|, the largest of a row's logits making e.  The probability of a token is then off by 2 e, and 4 * 2^-24 more for
    the exponentials; n of them are added in 32 bits, under weights and alone (n 2^-24 twice).  So a row is off by
    (4 e + (8 + 2 n) 2^-24) sum p |v|, and by half a step of its type once it is rounded.  Where query heads share a key head,
    bf16 weights are operands of a matrix product and so rounded to bf16, the sum that divides is of the weights as they were:
    a weight w_t becomes w_t (1 + r_t), |r_t| <= 2^-8, and the row sum w_t (1 + r_t) v_t / sum w_t is off by
    sum p_t |r_t v_t| <= 2^-8 sum p |v|, `u`.
    """
    import torch
    d = q.shape[1]
    dh = d // heads
    group = heads // kv_heads
    scale = dh ** -0.5 if scale is None else scale
    u = T.HALF_STEP["bf16"] if dtype == "bf16" and group > 1 else 0.0
    out = torch.zeros(q.shape[0], d, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    for b, at in enumerate(slots):
        at = torch.as_tensor(at, dtype=torch.int64, device="cuda")
        if mask is not None:
            at = at[mask[at] != 0]
        n = at.numel()
        if n == 0:
            continue
        k = k_cache[at].double().view(n, kv_heads, dh).repeat_interleave(group, 1).transpose(0, 1)
        v = v_cache[at].double().view(n, kv_heads, dh).repeat_interleave(group, 1).transpose(0, 1)
        qf = q[b].double().view(heads, dh, 1)
        logits = torch.bmm(k.contiguous(), qf)[..., 0] * scale
        size = torch.bmm(k.abs().contiguous(), qf.abs())[..., 0].amax(1, keepdim=True) * scale
        p = torch.softmax(logits, 1)[:, None]
        row = torch.bmm(p, v.contiguous())[:, 0]
        weight = torch.bmm(p, v.abs().contiguous())[:, 0]
        e = (dh + 4) * T.EPS32 * size
        err = weight * (4 * e + (8 + 2 * n) * T.EPS32 + u)
        out[b] = row.reshape(-1)
        bound[b] = (err + T.HALF_STEP[dtype] * (row.abs() + err)).reshape(-1) * 1.05 + 1e-30
    return out, bound


# ---- rotary positions ----------------------------------------------------------------------
def axes_table(pairs, in_turn, shared, base=10000.0):
    """(axis, frequency) of every pair, from the definition."""
    if in_turn:
        rounds = [[a for a in range(len(pairs)) if r < pairs[a]] for r in range(max(pairs))]
        axis = [a for r in rounds for a in r]
    else:
        axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    n, freq = len(axis), []
    for i, a in enumerate(axis):
        freq.append(math.pow(base, -i / n) if shared else math.pow(base, -axis[:i].count(a) / pairs[a]))
    return axis, freq


def turned(x, pos, axis, freq, heads, interleaved):
    """(features turned, length of each feature's pair), [rows, heads * d_head] in 64 bits."""
    import torch
    rows, n = x.shape[0], len(axis)
    x = x.double().reshape(rows, heads, -1)
    angle = pos.double()[:, torch.tensor(axis, device=x.device)] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    i = torch.arange(n, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    a, b = x[..., ia], x[..., ib]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia] = size[..., ib] = (a * a + b * b).sqrt()
    return y.reshape(rows, -1), size.reshape(rows, -1)
