"""Attention of one new token of every stream over a paged memory, against softmax over the held tokens in 64 bits: shared key
heads, lengths from none to long, pages that end inside a tile, rings that go round, masks; and the refusals."""
import math

import numpy as np
import pytest

import differential_reference as T
import stream_memory_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _memory(rng, lengths, page, spare=5):
    """Streams of those lengths whose rings have gone round, on pages anywhere."""
    cols = max(lengths) // page + 3
    s = R.State(len(lengths), page, sum(n // page + 2 for n in lengths) + spare, cols)
    ids = iter(rng.permutation(s.n_pages))
    for b, n in enumerate(lengths):
        s.span[b] = (rng.integers(0, cols * page) if n else 0), n
        for j in s.pages(b):
            s.table[b, j % cols] = next(ids)
    return s


class Case:
    def __init__(self, d, kv, lengths, page, dtype, seed=1, heads=None, std=1.5, together=False):
        import torch
        rng = np.random.default_rng(seed)
        self.heads, self.kv, self.dtype, self.d = heads or T.MODELS[d], kv, dtype, d
        self.s = _memory(rng, lengths, page)
        self.enc = T.encoder(d, 8, dtype=dtype, heads=heads)
        self.enc.attach_memory(page, self.s.n_pages, self.s.cols, len(lengths), kv)
        kd, n = d // self.heads * kv, page * self.s.n_pages
        self.q = T.normal(seed, len(lengths), d, std=std).to(T.act(dtype))
        # keys and values in columns of wider rows, a strip between them
        rows = T.normal(seed + 1, n, 2 * kd + 16).to(T.act(dtype))
        self.k, self.v = rows[:, :kd], rows[:, kd + 16:]
        if together:
            self.k, self.v = self.k.contiguous(), self.v.contiguous()
        self.k.mul_(std)
        self.span, self.table = (torch.from_numpy(x).cuda() for x in (self.s.span, self.s.table))
        self.slots = [self.s.slots(b) for b in range(len(lengths))]
        self.mask = None
        # slots that no stream holds, and columns between, may hold anything
        unused = np.setdiff1d(np.arange(n), np.concatenate([np.asarray(x, dtype=np.int64) for x in self.slots]))
        self.k[torch.from_numpy(unused).cuda()] = math.nan
        self.v[torch.from_numpy(unused).cuda()] = math.inf

    def run(self, out=None, q=None, **kw):
        import torch
        if out is None:
            out = torch.empty(self.q.shape[0], self.d, device="cuda").to(T.act(self.dtype))
        self.enc.memory_attention(self.q if q is None else q, self.k, self.v, self.span, self.table, out, key_mask=self.mask, **kw)
        return out

    def check(self, got, scale=None):
        want, bound = R.attention(self.q, self.k, self.v, self.slots, self.heads, self.kv, self.dtype, scale, self.mask)
        return T.within(got, want, bound, "rows")


@pytest.mark.parametrize("d,kv,dtype", [(64, 2, "bf16"), (64, 1, "bf16"), (64, 2, "f32"), (64, 1, "f32"), (256, 8, "bf16"), (256, 4, "bf16"), (256, 2, "bf16"),
                                        (256, 1, "bf16"), (256, 4, "f32"), (384, 6, "bf16"), (384, 3, "bf16"), (384, 2, "bf16"), (384, 1, "f32"),
                                        (768, 12, "bf16"), (768, 4, "bf16"), (768, 1, "bf16"), (768, 3, "f32"), (1024, 16, "bf16"), (1024, 2, "bf16")])
@pytest.mark.parametrize("page", (8, 64))
def test_head_layouts(K, d, kv, dtype, page):
    """Lengths round a page's and a tile's end, among them none."""
    case = Case(d, kv, [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 129, 255, 257, 500, 0], page, dtype)
    case.check(case.run())
    case.enc.sync_status()
    case.enc.close()


@pytest.mark.parametrize("heads,d", [(32, 1024), (10, 320), (5, 320), (14, 448), (7, 448), (9, 576), (3, 192), (20, 640), (1, 64)])
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_numbers_of_heads(K, heads, d, dtype):
    """Every divisor of the heads as their number of key heads, odd groups among them."""
    for kv in (n for n in range(1, heads + 1) if heads % n == 0):
        case = Case(d, kv, [130, 1, 77], 16, dtype, seed=kv, heads=heads)
        case.check(case.run())
        case.enc.close()


@pytest.mark.parametrize("d,kv,lengths,page,dtype", [
    (768, 12, [50_001], 64, "bf16"), (768, 2, [30_000, 3, 9_999], 256, "bf16"), (256, 8, [20_011, 0, 1], 16, "bf16"), (64, 1, [70_000], 1024, "bf16"),
    (64, 2, [9_001], 8, "f32"), (384, 2, [6_000, 6_001, 5_999], 32, "f32"), (256, 8, [1_000_003], 1024, "bf16"),
])
def test_long_streams(K, d, kv, lengths, page, dtype):
    case = Case(d, kv, lengths, page, dtype)
    got = case.run()
    case.check(got)
    for _ in range(3):   # the same bits again
        assert (case.run() == got).all()
    case.enc.sync_status()
    case.enc.close()


@pytest.mark.parametrize("streams,d,kv,most", [(300, 256, 8, 120), (1000, 64, 2, 40), (4096, 64, 1, 9), (700, 768, 4, 30), (513, 384, 6, 60)])
def test_many_streams(K, streams, d, kv, most):
    rng = np.random.default_rng(streams)
    case = Case(d, kv, rng.integers(0, most, streams).tolist(), 8, "bf16")
    case.check(case.run())
    case.enc.sync_status()
    case.enc.close()


def test_one_long_stream_among_short_ones(K):
    case = Case(256, 2, [3] * 60 + [40_000] + [0, 17] * 20, 32, "bf16")
    case.check(case.run())
    case.enc.close()


@pytest.mark.parametrize("d,kv,dtype", [(256, 8, "bf16"), (768, 2, "bf16"), (384, 6, "f32"), (64, 1, "bf16")])
def test_masks(K, d, kv, dtype):
    """Masked tokens hold no numbers; streams whose mask leaves nothing, one token, the first or the last."""
    import torch
    case = Case(d, kv, [300, 300, 1, 129, 129, 2000, 64, 5], 16, dtype)
    case.mask = (torch.rand(case.k.shape[0], generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") > 0.3).to(torch.uint8)
    case.mask[case.slots[0]] = 0
    case.mask[case.slots[2]] = 0
    for b, one in ((3, 0), (4, -1), (6, 17)):
        case.mask[case.slots[b]] = 0
        case.mask[case.slots[b][one]] = 255
    shut = case.mask == 0
    case.k[shut], case.v[shut] = math.nan, math.inf
    out = torch.full((10, d), 9.0, device="cuda").to(T.act(dtype))
    case.run(out[1:-1])
    case.check(out[1:-1])
    assert not out[1].any() and not out[3].any() and (out[0] == 9).all() and (out[-1] == 9).all()
    for b, one in ((3, 0), (4, -1), (6, 17)):   # a single token's values, as they are
        v = case.v[case.slots[b][one]].view(kv, -1).repeat_interleave(case.heads // kv, 0).reshape(-1)
        assert torch.equal(out[1 + b], v)
    case.enc.sync_status()
    case.enc.close()


@pytest.mark.parametrize("d,kv,dtype", [(256, 8, "bf16"), (768, 2, "bf16"), (384, 6, "f32")])
def test_logits_of_every_size(K, d, kv, dtype):
    """Peaked rows, equal logits, logits that go up and down along a stream by hundreds, all far below 0."""
    import torch
    case = Case(d, kv, [700, 700, 700, 900, 40], 16, dtype, std=1.0)
    s = case.slots
    case.k[s[0]] *= 30
    case.k[s[1]] = 0
    for step in range(700):   # towards one key, ever nearer, and the opposite for the next stream
        if step % 7 == 0:
            case.k[s[2][step]] = case.k[s[2][699]] * (step / 70)
    far = case.q[4].view(case.kv, -1, d // case.heads).sum(1).reshape(-1)
    case.k[s[4]] = -20 * far
    got = case.run()
    # (equal logits: the mean of the values)
    mean = case.v[s[1]].double().view(700, kv, -1).repeat_interleave(case.heads // kv, 1).mean(0).reshape(-1)
    want, bound = R.attention(case.q, case.k, case.v, s, case.heads, kv, dtype)
    T.within(got, want, bound)
    assert (want[1] - mean).abs().max() < 1e-12
    case.enc.close()


def test_scale(K):
    import torch
    case = Case(256, 8, [77, 500], 16, "bf16")
    case.check(case.run(softmax_scale=0.03), 0.03)
    case.check(case.run(softmax_scale=0.0), math.log(2.0))
    # in place, and queries in columns of wider rows
    wide = torch.zeros(2, 800, device="cuda", dtype=torch.bfloat16)
    wide[:, 256:512] = case.q
    want = case.run()
    case.run(wide[:, 256:512], wide[:, 256:512])
    assert torch.equal(wide[:, 256:512], want) and not wide[:, :256].any() and not wide[:, 512:].any()
    case.enc.close()


def test_streams_on_the_same_pages(K):
    """A copied state: several streams read the same slots, fewer streams than the context may have."""
    import torch
    case = Case(256, 2, [900, 40, 3, 7, 1], 16, "bf16")
    case.span[1:3], case.table[1:3] = case.span[0].clone(), case.table[0].clone()
    case.span[2, 1] = 500   # (the first of them)
    case.q[1] = case.q[0]
    case.slots[1:3] = case.slots[0], case.slots[0][:500]
    out = torch.empty(4, 256, device="cuda", dtype=torch.bfloat16)
    case.enc.memory_attention(case.q[:4], case.k, case.v, case.span[:4], case.table[:4], out)
    want, bound = R.attention(case.q[:4], case.k, case.v, case.slots[:4], 8, 2, "bf16")
    T.within(out, want, bound)
    assert torch.equal(out[0], out[1])
    case.enc.sync_status()
    case.enc.close()


@pytest.mark.parametrize("d,kv,dtype", [(256, 8, "bf16"), (768, 2, "bf16"), (384, 6, "f32")])
def test_values_that_are_no_numbers_stay_where_they_belong(K, d, kv, dtype):
    """A query that is none makes its own row none, a key its stream's rows of its head, a value its column; no other."""
    import torch
    case = Case(d, kv, [300, 300, 300, 2000, 40], 16, dtype)
    dh, group = d // case.heads, case.heads // kv
    want = case.run()
    case.q[1, 3] = math.nan
    case.k[case.slots[2][17], dh * (kv - 1)] = math.nan
    case.v[case.slots[3][1999], 5] = math.inf
    got = case.run()
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[1, :dh] = True
    bad[2, d - dh * group:] = True
    for g in range(group):
        bad[3, g * dh + 5] = True
    assert (torch.isfinite(got) == ~bad).all() and torch.equal(got[~bad], want[~bad])
    case.enc.close()


def test_two_contexts_on_two_streams(K):
    """Long streams in pieces, on both at once: each has its own work space."""
    import torch
    cases = [Case(256, 8, [20_000, 3, 9_000], 16, "bf16", seed=1), Case(256, 2, [9_000, 15_000], 32, "bf16", seed=2)]
    want = [c.run() for c in cases]
    sides = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(6):
        for side, c, o in zip(sides, cases, outs):
            with torch.cuda.stream(side):
                o.append(c.run())
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x, w) for x in o)
    for c in cases:
        c.enc.sync_status()
        c.enc.close()


def test_rows_past_32_bits(K):
    """A cache of more than 4 GiB, a stream whose pages lie at both of its ends."""
    import torch
    page, n_pages, d = 1024, 2100, 1024
    enc = T.encoder(d, 8)
    enc.attach_memory(page, n_pages, 8, 1)
    k, v = (torch.empty(page * n_pages, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))   # 4.4 GB each
    s = R.State(1, page, n_pages, 8)
    s.span[0], s.table[0, :4] = (1000, 3000), (2099, 0, 2048, 1023)
    at = s.slots(0)
    rows = torch.tensor(at, device="cuda")
    k[rows], v[rows] = T.normal(1, 3000, d).bfloat16(), T.normal(2, 3000, d).bfloat16()
    q, out = T.normal(3, 1, d).bfloat16(), torch.empty(1, d, device="cuda", dtype=torch.bfloat16)
    enc.memory_attention(q, k, v, torch.from_numpy(s.span).cuda(), torch.from_numpy(s.table).cuda(), out)
    want, bound = R.attention(q, k, v, [at], 16, 16, "bf16")
    T.within(out, want, bound)
    enc.close()


def test_page_numbers_that_are_none(K):
    """Their tokens count as masked, and the status says so."""
    import torch
    case = Case(256, 8, [100, 64], 16, "bf16")
    for bad in (-1, case.s.n_pages, 2 ** 31 - 1, -2 ** 31):
        pages = case.s.pages(0)
        table = case.table.clone()
        column = pages[1] % case.s.cols
        table[0, column] = bad
        out = torch.empty(2, 256, device="cuda", dtype=torch.bfloat16)
        case.enc.memory_attention(case.q, case.k, case.v, case.span, table, out)
        with pytest.raises(K.CfdetrError) as e:
            case.enc.sync_status()
        assert e.value.status == K.CFDETR_ECAPACITY
        first = int(case.s.span[0, 0])
        left = [x for i, x in enumerate(case.slots[0]) if (first + i) // 16 % case.s.cols != column]
        want, bound = R.attention(case.q, case.k, case.v, [left, case.slots[1]], 8, 8, "bf16")
        T.within(out, want, bound)
    case.enc.sync_status()
    case.enc.close()


@pytest.mark.parametrize("span", [(-1, 5), (0, -1), (10 ** 9, 1), (0, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1), (1, None)])
def test_spans_that_are_none(K, span):
    """Nothing is written, and the status says so."""
    import torch
    case = Case(64, 2, [30, 20, 10], 8, "bf16")
    ring = case.s.cols * 8
    case.span[1] = torch.tensor((span[0], ring if span[1] is None else span[1]), dtype=torch.int32)
    out = torch.full((3, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    case.run(out)
    with pytest.raises(K.CfdetrError) as e:
        case.enc.sync_status()
    assert e.value.status == K.CFDETR_ECAPACITY and (out == 7).all()
    case.enc.close()


def test_refusals(K):
    import torch
    enc = T.encoder(64, 8)
    x = torch.zeros(64, 80, device="cuda", dtype=torch.bfloat16)
    i = torch.zeros(64, dtype=torch.int32, device="cuda")
    p, ld, n = x.data_ptr(), 80, i.data_ptr()

    def call(q=p, q_ld=ld, B=2, k=p, k_ld=ld, v=p, v_ld=ld, span=n, table=n, mask=None, scale=0.1, out=p, out_ld=ld):
        K.cfdetr_memory_attention(enc.ctx, q, q_ld, B, k, k_ld, v, v_ld, span, table, mask, scale, out, out_ld, enc._stream())

    with pytest.raises(K.CfdetrError) as e:
        call()
    assert e.value.status == K.CFDETR_EINVAL
    enc.attach_memory(8, 4, 4, 2, 1)
    call()
    assert not x.any()
    for bad, status in ((dict(B=0), K.CFDETR_EINVAL), (dict(B=-1), K.CFDETR_EINVAL), (dict(B=3), K.CFDETR_ECAPACITY), (dict(scale=-1.0), K.CFDETR_EINVAL),
                        (dict(scale=math.nan), K.CFDETR_EINVAL), (dict(scale=math.inf), K.CFDETR_EINVAL),
                        *((dict([(name, value)]), K.CFDETR_EINVAL) for name in ("q", "k", "v", "out", "span", "table") for value in (None, p + 2)),
                        (dict(span=n + 4), K.CFDETR_EINVAL), (dict(mask=n + 4), K.CFDETR_EINVAL), (dict(q_ld=56), K.CFDETR_EINVAL), (dict(k_ld=24), K.CFDETR_EINVAL), (dict(v_ld=36), K.CFDETR_EINVAL),
                        (dict(out_ld=88), K.CFDETR_EINVAL), (dict(k_ld=(1 << 24) + 8), K.CFDETR_EINVAL)):
        with pytest.raises(K.CfdetrError) as e:
            call(**bad)
        assert e.value.status == status and K.cfdetr_last_error(enc.ctx), bad
    enc.sync_status()
    enc.close()
