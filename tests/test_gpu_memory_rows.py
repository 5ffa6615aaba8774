"""Rotary positions of several axes, and rows into the slots of a memory of streams, against the formulas in 64 bits."""
import math

import numpy as np
import pytest

import differential_reference as T
import stream_memory_reference as R

pytestmark = pytest.mark.gpu

# What a feature may be off, relative to its pair's length: the angle's last 32 bits (half a step of half a turn, in
# radians: 2^-25 2 pi < 2^-22), sine, cosine, two products and a sum in 32 bits (4 units), the scale (1).
PAIR = 2.0 ** -22 + 8 * T.EPS32


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _positions(rows, axes, far, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, far, (rows, axes), generator=g, device="cuda").float() + (0.5 if far < 1000 else 0.0)


def _table(K, params):
    import torch
    freq, axis = K.cfdetr_rotary_axes_table(params)
    return torch.tensor(freq, dtype=torch.float64, device="cuda"), torch.tensor(axis, dtype=torch.uint8, device="cuda")


CASES = [
    # d, key heads, rows, dtype, pairs, in_turn, shared, interleaved, far
    (64, 2, 1, "bf16", (4, 6, 6), False, False, False, 160), (64, 1, 67, "f32", (2, 3, 3), True, False, True, 100),
    (256, 8, 300, "bf16", (4, 6, 6), True, True, False, 160), (256, 1, 17, "bf16", (8,), False, False, True, 16_000_000),
    (384, 2, 1001, "bf16", (8, 12, 12), False, True, True, 4000), (384, 6, 5, "f32", (6, 9, 9), True, False, False, 1_000_003),
    (768, 12, 129, "bf16", (1, 13, 1, 1), True, False, False, 160), (768, 4, 40, "f32", (8, 12, 12), True, True, True, 1_000_003),
    (1024, 16, 33, "bf16", (12, 12), False, False, False, 4000), (1024, 16, 9, "f32", (8, 8, 8, 8), True, False, False, 160),
]


@pytest.mark.parametrize("d,kv,rows,dtype,pairs,in_turn,shared,interleaved,far", CASES)
def test_turned_against_the_formula(K, d, kv, rows, dtype, pairs, in_turn, shared, interleaved, far):
    import torch
    enc, heads = T.encoder(d, 8, dtype=dtype), T.MODELS[d]
    dh = d // heads
    kd = kv * dh
    params = K.rotary_axes_params(2 * sum(pairs), pairs, in_turn, shared, interleaved)
    freq, axis = _table(K, params)
    want_axis, want_freq = R.axes_table(pairs, in_turn, shared)
    pos = _positions(rows, len(pairs), far, 1)
    qkv = T.normal(2, rows, d + 2 * kd).to(T.act(dtype))
    q, k = qkv[:, :d], qkv[:, d:d + kd]
    scale = T.log2e_over(dh)
    out = torch.full((rows + 2, d + kd + 64), 7.0, device="cuda").to(T.act(dtype))   # rows apart, others around them
    enc.rotary_axes(params, freq, axis, pos, q, out[1:-1, :d], k, out[1:-1, d:d + kd], q_scale=scale)
    for x, got, n, s in ((q, out[1:-1, :d], heads, scale), (k, out[1:-1, d:d + kd], kv, 1.0)):
        want, size = R.turned(x, pos, want_axis, want_freq, n, interleaved)
        T.within(got, want * s, (want.abs() * T.HALF_STEP[dtype] + size * PAIR + want.abs() * T.EPS32) * s * 1.001, "features")
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, d + kd:] == 7).all()
    if 2 * sum(pairs) < dh:   # features behind the rotated ones are as they were
        assert torch.equal(out[1:-1, d:d + kd].reshape(rows, kv, dh)[..., 2 * sum(pairs):], k.reshape(rows, kv, dh)[..., 2 * sum(pairs):])
    # in place, and queries alone, the same bits
    own = qkv.clone()
    enc.rotary_axes(params, freq, axis, pos, own[:, :d], own[:, :d], own[:, d:d + kd], own[:, d:d + kd], q_scale=scale)
    assert torch.equal(own[:, :d + kd], out[1:-1, :d + kd]) and torch.equal(own[:, d + kd:], qkv[:, d + kd:])
    alone = torch.empty(rows, d, device="cuda").to(T.act(dtype))
    enc.rotary_axes(params, freq, axis, pos, q, alone, q_scale=scale)
    assert torch.equal(alone, out[1:-1, :d])
    enc.close()


def test_one_axis_of_text(K):
    """Three equal positions with a shared ladder turn as one axis does, whatever the axes' shares."""
    import torch
    enc = T.encoder(256, 50)
    x, t = T.normal(3, 50, 256).bfloat16(), _positions(50, 1, 5000, 2)
    plain, axes = torch.empty_like(x), torch.empty_like(x)
    one = K.rotary_params(32, 1)
    enc.rotary(one, torch.tensor(K.cfdetr_rotary_frequencies(one), dtype=torch.float64, device="cuda"), t, x, plain)
    for in_turn in (False, True):
        params = K.rotary_axes_params(32, (3, 7, 6), in_turn, True)
        enc.rotary_axes(params, *_table(K, params), t.repeat(1, 3), x, axes)
        assert torch.equal(plain, axes)
    enc.close()


def test_axes_that_are_none_count_as_the_last(K):
    import torch
    enc = T.encoder(64, 8)
    params = K.rotary_axes_params(32, (8, 8))
    freq, axis = _table(K, params)
    x, pos, a, b = T.normal(1, 8, 64).bfloat16(), _positions(8, 2, 100, 1), *(torch.empty(8, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    enc.rotary_axes(params, freq, axis, pos, x, a)
    enc.rotary_axes(params, freq, torch.where(axis == 1, 255, 0).to(torch.uint8), pos, x, b)
    assert torch.equal(a, b)
    enc.close()


def _slots(rng, rows, n_slots, padding):
    at = rng.permutation(n_slots)[:rows].astype(np.int32)
    at[rng.permutation(rows)[:padding]] = -1 - rng.integers(0, 5)
    return at


@pytest.mark.parametrize("d,kv,rows,dtype,pairs,interleaved,padding", [
    (64, 2, 1, "bf16", (4, 6, 6), False, 0), (64, 1, 67, "f32", (2, 3, 3), True, 9), (256, 8, 300, "bf16", (4, 6, 6), False, 0),
    (384, 3, 1001, "bf16", (8, 12, 12), True, 1000), (384, 1, 50, "f32", (6, 9, 9), False, 3), (768, 12, 129, "bf16", None, False, 5),
    (768, 4, 40, "f32", None, False, 0), (1024, 16, 33, "bf16", (8, 8, 8, 8), False, 33),
])
def test_appended(K, d, kv, rows, dtype, pairs, interleaved, padding):
    """Keys as cfdetr_rotary_axes turns them, values as they are, no other row touched."""
    import torch
    enc, heads, page, n_pages = T.encoder(d, 8, dtype=dtype), T.MODELS[d], 8, (rows + 40) // 8
    enc.attach_memory(page, n_pages, 4, 1, kv)
    kd = d // heads * kv
    rng = np.random.default_rng(rows)
    at = _slots(rng, rows, page * n_pages, padding)
    slots, have = torch.from_numpy(at).cuda(), torch.from_numpy(np.flatnonzero(at >= 0)).cuda()
    kvr = T.normal(2, rows, 2 * kd + 16).to(T.act(dtype))
    k, v = kvr[:, :kd], kvr[:, kd + 16:]
    for x in (k, v):   # values that are no numbers are copied bit by bit, and stay in their pair where they are turned
        x[0, 1], x[-1, -1] = math.nan, -math.inf
    args, want = (), k
    if pairs:
        params = K.rotary_axes_params(2 * sum(pairs), pairs, True, False, interleaved)
        args = (params, *_table(K, params), _positions(rows, len(pairs), 160, 1))
        want = torch.empty(rows, kd, device="cuda").to(T.act(dtype))
        enc.rotary_axes(*args, T.normal(1, rows, d).to(T.act(dtype)), torch.empty(rows, d, device="cuda").to(T.act(dtype)), k, want)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    cache = torch.full((page * n_pages, 2 * kd + 32), 7.0, device="cuda").to(T.act(dtype))   # keys and values side by side
    expected = cache.clone()
    expected[slots[have].long(), :kd] = want[have]
    expected[slots[have].long(), kd + 32:] = v[have]
    enc.memory_append(k, v, slots, cache[:, :kd], cache[:, kd + 32:], *args)
    assert torch.equal(cache.view(bits), expected.view(bits))
    enc.sync_status()
    enc.close()


def test_slots_beyond_the_memory(K):
    import torch
    enc = T.encoder(64, 8)
    enc.attach_memory(8, 4, 4, 1)
    k = T.normal(1, 4, 64).bfloat16()
    cache = torch.zeros(2, 40, 64, device="cuda", dtype=torch.bfloat16)   # (8 rows more than the memory has)
    slots = torch.tensor([3, 32, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    enc.memory_append(k, k, slots, cache[0, :32], cache[1, :32])
    with pytest.raises(K.CfdetrError) as e:
        enc.sync_status()
    assert e.value.status == K.CFDETR_ECAPACITY
    for c in cache:
        assert torch.equal(c[3], k[0])
        c[3] = 0
        assert not c.any()
    enc.close()


def test_rows_past_32_bits(K):
    """Slots whose rows begin beyond 2^32 bytes of a cache."""
    import torch
    enc = T.encoder(1024, 8)
    page, n_pages = 1024, 2100
    enc.attach_memory(page, n_pages, 4, 1)
    cache = torch.empty(page * n_pages, 1024, device="cuda", dtype=torch.bfloat16)   # 4.4 GB
    at = [0, 1_048_575, 1_048_576, 2_097_151, 2_097_152, page * n_pages - 1]
    slots = torch.tensor(at, dtype=torch.int32, device="cuda")
    k = T.normal(1, 6, 1024).bfloat16()
    cache[slots.long()] = 0
    enc.memory_append(k, k, slots, cache, cache)
    assert torch.equal(cache[slots.long()], k)
    enc.close()


def test_more_rows_than_a_slice(K):
    """From 2^23 rows on a call has several launches."""
    import torch
    enc = T.encoder(64, 8)
    rows = (1 << 23) + 5
    params = K.rotary_axes_params(32, (4, 6, 6))
    freq, axis = _table(K, params)
    pos = _positions(rows, 3, 160, 1)
    x = torch.randn(rows, 64, device="cuda", dtype=torch.bfloat16)
    out, part = torch.empty_like(x), torch.empty_like(x[-9:])
    enc.rotary_axes(params, freq, axis, pos, x, out)
    enc.rotary_axes(params, freq, axis, pos[-9:], x[-9:], part)
    assert torch.equal(part, out[-9:])
    enc.attach_memory(1024, 8300, 4, 1)
    slots = torch.randperm(8300 * 1024, device="cuda", dtype=torch.int32)[:rows]
    cache = torch.zeros(8300 * 1024, 128, device="cuda", dtype=torch.bfloat16)
    enc.memory_append(x, x, slots, cache[:, :64], cache[:, 64:], params, freq, axis, pos)
    assert torch.equal(cache[slots.long(), :64], out) and torch.equal(cache[slots.long(), 64:], x)
    enc.sync_status()
    enc.close()


def test_refusals(K):
    import torch
    enc = T.encoder(64, 8)
    params = K.rotary_axes_params(32, (4, 6, 6))
    freq, axis = _table(K, params)
    pos, x = torch.zeros(8, 3, device="cuda"), torch.zeros(8, 80, device="cuda", dtype=torch.bfloat16)
    slots = torch.zeros(8, dtype=torch.int32, device="cuda")
    p, ld = x.data_ptr(), 80

    def turn(params=params, freq=freq.data_ptr(), axis=axis.data_ptr(), pos=pos.data_ptr(), M=8, q=p, q_ld=ld, qo=p, qo_ld=ld, scale=1.0, k=None,
             k_ld=0, ko=None, ko_ld=0, kh=2):
        K.cfdetr_rotary_axes(enc.ctx, params, freq, axis, pos, M, q, q_ld, qo, qo_ld, scale, k, k_ld, ko, ko_ld, kh, enc._stream())

    def append(params=params, freq=freq.data_ptr(), axis=axis.data_ptr(), pos=pos.data_ptr(), M=8, k=p, k_ld=ld, v=p, v_ld=ld, slots=slots.data_ptr(),
               kc=p, kc_ld=ld, vc=p, vc_ld=ld):
        K.cfdetr_memory_append(enc.ctx, params, freq, axis, pos, M, k, k_ld, v, v_ld, slots, kc, kc_ld, vc, vc_ld, enc._stream())

    def refused(call, **kw):
        with pytest.raises(K.CfdetrError) as e:
            call(**kw)
        assert e.value.status == K.CFDETR_EINVAL and K.cfdetr_last_error(enc.ctx), kw

    turn(M=0, q=None, qo=None, freq=None, axis=None, pos=None)
    refused(append)   # no memory yet
    enc.attach_memory(8, 1, 1, 1, 1)
    append(M=0, k=None, v=None, slots=None, kc=None, vc=None, freq=None, axis=None, pos=None)
    bad_params = [K.rotary_axes_params(48, (8, 8, 8)), K.rotary_axes_params(8, (4,)), K.rotary_axes_params(32, (4, 6, 6), interleaved=2)]
    none, five = K.rotary_axes_params(32, (16,)), K.rotary_axes_params(32, (16,))
    none.n_axes, five.n_axes = 0, 5
    for kw in [dict(params=b) for b in (*bad_params, none, five)] + [dict(freq=None), dict(axis=None), dict(pos=None), dict(M=-1),
                                                                     dict(freq=freq.data_ptr() + 4), dict(pos=pos.data_ptr() + 2)]:
        refused(turn, **kw)
        refused(append, **kw)
    for kw in (dict(q=None), dict(qo=None), dict(q=p + 2), dict(q_ld=60), dict(qo_ld=84), dict(scale=math.inf), dict(scale=math.nan), dict(k=p), dict(ko=p),
               dict(k=p, k_ld=ld, ko=p, ko_ld=ld + 8), dict(k=p, k_ld=63, ko=p, ko_ld=ld), dict(k=p, k_ld=ld, ko=p, ko_ld=ld, kh=0),
               dict(k=p, k_ld=ld, ko=p, ko_ld=ld, kh=3), dict(qo_ld=(1 << 24) + 8)):
        refused(turn, **kw)
    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(kc=None), dict(vc=None), dict(k=p + 8), dict(vc=p + 2), dict(slots=slots.data_ptr() + 2),
               dict(k_ld=24), dict(v_ld=31), dict(kc_ld=33), dict(vc_ld=(1 << 24) + 8)):
        refused(append, **kw)
        refused(append, **dict(kw, params=None, freq=None, axis=None, pos=None))
    enc.sync_status()
    enc.close()
