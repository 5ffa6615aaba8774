"""Differential attention against its definition in 64 bits: lengths from one token on, empty frames, strides, masks that leave
little or nothing, single queries over many keys, logits far from zero, repeated calls; and the refusals."""
import math

import pytest

import differential_reference as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _inputs(d, nq, nk, dtype, std=1.5, cross=False, seed=1):
    import torch
    act = T.act(dtype)
    if cross:
        q = T.normal(seed, sum(nq), d, std=std).to(act)
        kv = torch.cat([T.normal(seed + 1, sum(nk), d, std=std), T.normal(seed + 2, sum(nk), d)], 1).to(act)
        return q, kv[:, :d], kv[:, d:]
    qkv = torch.cat([T.normal(seed, sum(nq), 2 * d, std=std), T.normal(seed + 2, sum(nq), d)], 1).to(act)
    return qkv[:, :d], qkv[:, d:2 * d], qkv[:, 2 * d:]


def _run(K, d, nq, nk, dtype="bf16", norm=True, mask=None, std=1.5, scale=None, heads=None, enc=None, qkv=None):
    import torch
    heads = heads or T.MODELS[d]
    own = enc is None
    enc = enc or T.encoder(d, max(sum(nq), sum(nk)), len(nq), dtype, heads)
    q, k, v = qkv or _inputs(d, nq, nk, dtype, std, cross=nq != nk)
    lam = 0.2 + 0.7 * torch.rand(heads // 2, generator=torch.Generator().manual_seed(3)).cuda()
    g = 0.5 + T.normal(4, 2 * d // heads, std=0.1) if norm else None
    out = torch.full((sum(nq) + 2, d + 8), 7.0, device="cuda").to(T.act(dtype))
    enc.diff_attention(q, k, v, T.offsets(nq), T.offsets(nk), lam, out[1:-1, :d], g, mask, scale)
    enc.sync_status()
    want, bound = T.diff_attention(q, k, v, nq, nk, heads, lam, g, dtype, scale, mask)
    worst = T.within(out[1:-1, :d], want, bound, f"{d} {nq} {nk}")
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, d:] == 7).all()
    again = torch.full_like(out, 7.0)
    enc.diff_attention(q, k, v, T.offsets(nq), T.offsets(nk), lam, again[1:-1, :d], g, mask, scale)
    assert torch.equal(again.view(torch.int16 if dtype == "bf16" else torch.int32), out.view(torch.int16 if dtype == "bf16" else torch.int32))
    if own:
        enc.close()
    print(f"{worst:.3f} of the bound", flush=True)
    return out[1:-1, :d]


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d", (64, 256, 384, 768))
def test_frames_of_every_length(K, d, dtype):
    """One token, both sides of a tile and of a unit of keys, empty frames at either end."""
    _run(K, d, *[[0, 1, 2, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 200, 0]] * 2, dtype)


@pytest.mark.parametrize("norm", (True, False))
@pytest.mark.parametrize("d,nq,nk", [
    (256, [300, 0, 7, 1], [1, 33, 0, 517]), (384, [1], [5003]), (768, [1, 1], [4100, 37]), (64, [2, 1, 0], [0, 3000, 9]),
    (384, [65, 300], [1601, 64]), (1024, [5], [777]),
])
def test_queries_over_other_rows(K, d, nq, nk, norm):
    _run(K, d, nq, nk, norm=norm)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d,nq,nk", [
    (256, [2] * 20, [i * 397 % 4100 for i in range(20)]), (64, [5, 1, 1], [9000, 1, 0]), (384, [200, 3, 0, 40], [1025, 6000, 31, 2999]),
    (256, [600, 1, 0, 1], [3000, 0, 500, 4000]), (64, [33] * 40, [(i * 613) % 2300 for i in range(40)]), (768, [1, 1], [30_000, 100]),
])
def test_runs_of_ragged_frames(K, d, nq, nk, dtype):
    """Frames whose keys are cut into runs, of one run, and without keys, in one call."""
    _run(K, d, nq, nk, dtype)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d,nq,nk", [(768, [1], [9001]), (256, [40], [5000]), (384, [33, 2], [4000, 3001]), (256, [40, 1], [5000, 3])])
def test_long_frames_without_a_key_left(K, d, nq, nk, dtype):
    import torch
    mask = torch.zeros(sum(nk), dtype=torch.uint8, device="cuda")
    assert not _run(K, d, nq, nk, dtype, mask=mask).any()
    mask[sum(nk) - 1] = 1
    assert _run(K, d, nq, nk, dtype, mask=mask)[-1].any()


@pytest.mark.parametrize("heads,frames", [(12, 12), (12, 9), (2, 60)])
def test_tiles_that_do_not_divide_by_the_xcds(K, heads, frames):
    n = [300 + f % 3 for f in range(frames)]
    _run(K, 32 * heads if heads == 2 else 64 * heads, n, [130 + 7 * f for f in range(frames)], heads=heads)


@pytest.mark.parametrize("d,n", [(256, [1600, 901, 1333, 400]), (384, [2500, 37]), (768, [1100, 1, 640])])
def test_longer_frames(K, d, n):
    _run(K, d, n, n)


# Frames of every length about a unit of 32 keys and a tile of 128 queries, often enough for the kernel of many queries (rows times
# heads from 16,384 on, on 256 CUs: eight wavefronts a tile, beyond 32,768 four), empty ones between them.
EDGES = [0, 1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 0, 160, 255, 256, 257, 300, 513, 0]


MANY = (20_000, 40_000)


def _many(d, rows):
    n, heads = [], T.MODELS[d] // 2
    while sum(n) * heads < rows:
        n += EDGES
    return n[:63] + [rows // heads - sum(n[:63])] if len(n) > 64 else n


@pytest.mark.parametrize("norm", (True, False))
@pytest.mark.parametrize("d", (64, 256, 384, 768, 1024))
@pytest.mark.parametrize("rows", MANY)
def test_many_queries(K, d, norm, rows):
    n = _many(d, rows)
    _run(K, d, n, n, norm=norm, scale=0.2 if norm else None)


@pytest.mark.parametrize("d", (256, 384))
@pytest.mark.parametrize("rows", MANY)
def test_many_queries_over_other_rows(K, d, rows):
    n = _many(d, rows)
    _run(K, d, n, [(7 * m + 3) % 211 for m in n])


@pytest.mark.parametrize("d,share", [(256, 0.5), (384, 0.1), (384, 0.95)])
@pytest.mark.parametrize("rows", MANY)
def test_many_queries_masked(K, d, share, rows):
    import torch
    n = _many(d, rows)
    q, k, v = (x.clone() for x in _inputs(d, n, n, "bf16"))
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    mask = (torch.rand(sum(n), generator=g, device="cuda") >= share).to(torch.uint8)
    mask[sum(n[:20]):sum(n[:21])] = 0
    k[mask == 0], v[mask == 0] = math.nan, math.inf
    out = _run(K, d, n, n, mask=mask, qkv=(q, k, v))
    assert not out[sum(n[:20]):sum(n[:21])].any()


def test_many_frames(K):
    """As many as a context takes, most of them short."""
    n = [(i * 37) % 91 for i in range(64)]
    _run(K, 256, n, n)
    _run(K, 64, n, n, "f32")


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d", (256, 384))
def test_single_queries_over_many_keys(K, d, dtype):
    _run(K, d, [1], [20_011], dtype)
    _run(K, d, [1, 3, 2], [9000, 1, 30], dtype)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d,nq,nk", [(256, [33, 200, 64, 5], [33, 200, 64, 5]), (384, [300, 300, 3], [2100, 5000, 70]), (768, [1], [9001])])
@pytest.mark.parametrize("share", (0.05, 0.5, 0.97))
def test_masks(K, d, nq, nk, dtype, share):
    """Masked rows hold what no row may: they are not read.  One frame has no key left."""
    import torch
    q, k, v = _inputs(d, nq, nk, dtype, cross=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    mask = (torch.rand(sum(nk), generator=g, device="cuda") >= share).to(torch.uint8) * 3
    if len(nk) > 1:
        mask[nk[0]:nk[0] + nk[1]] = 0
    k[mask == 0], v[mask == 0] = math.nan, math.inf
    out = _run(K, d, nq, nk, dtype, mask=mask, qkv=(q, k, v))
    if len(nk) > 1:
        assert not out[nq[0]:nq[0] + nq[1]].any()


def test_masks_that_leave_everything_or_nothing(K):
    import torch
    n = [70, 2049, 1]
    q, k, v = _inputs(256, n, n, "bf16")
    enc = T.encoder(256, sum(n), 3)
    lam, out = torch.full((4,), 0.4, device="cuda"), torch.empty(sum(n), 256, device="cuda").bfloat16()
    plain = torch.empty_like(out)
    cu = T.offsets(n)
    enc.diff_attention(q, k, v, cu, cu, lam, plain)
    enc.diff_attention(q, k, v, cu, cu, lam, out, key_mask=torch.ones(sum(n), dtype=torch.uint8, device="cuda"))
    assert torch.equal(out, plain)
    enc.diff_attention(q, k, v, cu, cu, lam, out, head_g=torch.ones(64, device="cuda"), key_mask=torch.zeros(sum(n), dtype=torch.uint8, device="cuda"))
    assert not out.any()
    enc.diff_attention(q[:5], k[:0], v[:0], T.offsets([2, 3]), T.offsets([0, 0]), lam, out[:5], head_g=torch.ones(64, device="cuda"))
    assert not out[:5].any()
    enc.sync_status()
    enc.close()


@pytest.mark.parametrize("n", ([1, 63, 64, 65, 129, 200, 1000], [1500] * 2, [1, 63, 65, 129, 200, 1000] * 6,
                               [1, 63, 65, 129, 200, 1000] * 10))
@pytest.mark.parametrize("level", (-400.0, -90.0, 90.0, 400.0))
@pytest.mark.parametrize("d", (256, 384))
def test_logits_far_from_zero(K, d, n, level):
    """Every logit of a query lies around `level`, in powers of two, and its keys a few units apart: what a
    softmax relative to 0 cannot hold at the outer levels.  Whole numbers, so that products in bf16 are exact."""
    import torch
    heads, dh = T.MODELS[d], d // T.MODELS[d]
    q, k, v = (x.clone() for x in _inputs(d, n, n, "bf16"))
    q.view(sum(n), heads, dh)[:, :, 0], k.view(sum(n), heads, dh)[:, :, 0] = 16.0, level / 16.0
    q.view(sum(n), heads, dh)[:, :, 1:], k.view(sum(n), heads, dh)[:, :, 1:] = 1.0, 0.0
    k.view(sum(n), heads, dh)[:, :, 1] = torch.randint(-4, 5, (sum(n), heads), generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    # queries of the second half of the rows see the opposite level
    q.view(sum(n), heads, dh)[sum(n) // 2:, 0, 0] = -16.0
    _run(K, d, n, n, qkv=(q, k, v), scale=math.log(2.0))
    _run(K, d, [5] * len(n), n, qkv=(q[:5 * len(n)].contiguous(), k, v), scale=math.log(2.0))


def test_one_key_far_above_the_others(K):
    """It is in the last, ragged unit of keys."""
    n = [65, 300, 1025]
    q, k, v = (x.clone() for x in _inputs(256, n, n, "bf16", std=0.5))
    q[:, ::32] = 8.0
    k[:, ::32] = 0.0
    for end in (65, 365, 1390):
        k[end - 1, ::32] = 30.0
    _run(K, 256, n, n, qkv=(q, k, v))


@pytest.mark.parametrize("n", ([65, 300, 1025], [1500] * 4, [1500] * 8))
@pytest.mark.parametrize("d", (256, 384))
def test_values_and_weights_that_are_large_together(K, d, n):
    """Base-2 logits about 60 and values of 2^90: neither the sums nor the rows may pass what 32 bits hold."""
    import torch
    heads, dh = T.MODELS[d], d // T.MODELS[d]
    q, k, v = (x.clone() for x in _inputs(d, n, n, "bf16"))
    q.view(sum(n), heads, dh)[:, :, 0], k.view(sum(n), heads, dh)[:, :, 0] = 16.0, 60.0 / 16.0
    q.view(sum(n), heads, dh)[:, :, 1:], k.view(sum(n), heads, dh)[:, :, 1:] = 1.0, 0.0
    k.view(sum(n), heads, dh)[:, :, 1] = torch.randint(-4, 5, (sum(n), heads), generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    v *= 2.0 ** 90
    _run(K, d, n, n, qkv=(q, k, v), scale=math.log(2.0), norm=False)


def test_scale_in_the_queries(K):
    """softmax_scale 0 takes base-2 logits: the same as ln 2."""
    import torch
    n = [100, 33]
    q, k, v = _inputs(384, n, n, "bf16", std=0.5)
    enc = T.encoder(384, 133, 2)
    cu, lam = T.offsets(n), torch.full((3,), 0.5, device="cuda")
    a, b = (torch.empty(133, 384, device="cuda").bfloat16() for _ in range(2))
    enc.diff_attention(q, k, v, cu, cu, lam, a, softmax_scale=0.0)
    want, bound = T.diff_attention(q, k, v, n, n, 6, lam, None, "bf16", math.log(2.0))
    T.within(a, want, bound)
    # in place of the queries
    own = q.clone()
    enc.diff_attention(own, k, v, cu, cu, lam, b, softmax_scale=0.0)
    enc.diff_attention(own, k, v, cu, cu, lam, own, softmax_scale=0.0)
    assert torch.equal(a, b) and torch.equal(own, a)
    enc.close()


def test_no_numbers_stay_in_their_frame(K):
    import torch
    n = [40, 40, 200]
    q, k, v = (x.clone() for x in _inputs(256, n, n, "bf16"))
    k[45, 3], v[130, 70] = math.nan, math.inf
    enc = T.encoder(256, 280, 3)
    out = torch.empty(280, 256, device="cuda").bfloat16()
    enc.diff_attention(q, k, v, T.offsets(n), T.offsets(n), torch.full((4,), 0.5, device="cuda"), out, softmax_scale=0.01)
    bad = ~torch.isfinite(out)
    assert bad[40:80, :64].all() and not bad[:40].any() and not bad[40:80, 64:].any()
    assert bad[80:, 70].all() and bad[80:].sum() == 200
    enc.close()


@pytest.mark.parametrize("d", (256, 384))
@pytest.mark.parametrize("more", (0, 6001))
def test_no_numbers_among_many_queries(K, d, more):
    """A value that is no number reaches its column of the rows of its frame, the last key's too."""
    import torch
    n = [3000, 129, 3000, 97] + [more] * (more > 0)
    q, k, v = (x.clone() for x in _inputs(d, n, n, "bf16", std=0.3))
    k[10, 3], v[3000 + 128, 70], v[6129 + 96, 5] = math.nan, math.inf, -math.inf
    w = 2 * d // T.MODELS[d]
    enc = T.encoder(d, sum(n), len(n))
    out = torch.empty(sum(n), d, device="cuda").bfloat16()
    enc.diff_attention(q, k, v, T.offsets(n), T.offsets(n), torch.full((T.MODELS[d] // 2,), 0.0, device="cuda"), out)
    bad = ~torch.isfinite(out)
    assert bad[:3000, :w].all() and not bad[:3000, w:].any() and not bad[3129:6129].any()
    assert (out[3000:3129, 70] == math.inf).all() and bad[3000:3129].sum() == 129
    assert (out[6129:6226, 5] == -math.inf).all() and bad[6129:].sum() == 97
    enc.close()


def test_bad_offsets_write_nothing(K):
    import torch
    n = [40, 60]
    q, k, v = _inputs(256, n, n, "bf16")
    enc = T.encoder(256, 100, 2)
    lam = torch.full((4,), 0.5, device="cuda")
    good = T.offsets(n)
    mask = torch.ones(100, dtype=torch.uint8, device="cuda")
    for cu in ([0, 60, 40], [0, 40, 101], [1, 40, 100], [0, -5, 100]):
        bad = torch.tensor(cu, dtype=torch.int32, device="cuda")
        for a, b, m in ((bad, good, None), (good, bad, None), (good, bad, mask)):
            out = torch.full((100, 256), 3.0, device="cuda").bfloat16()
            enc.diff_attention(q, k, v, a, b, lam, out, key_mask=m)
            with pytest.raises(K.CfdetrError) as e:
                enc.sync_status()
            assert e.value.status == K.CFDETR_ECAPACITY and (out == 3).all()
    enc.sync_status()
    enc.close()


def test_rows_behind_the_last_frame(K):
    import torch
    q, k, v = _inputs(256, [100], [100], "bf16")
    enc = T.encoder(256, 100, 2)
    out = torch.full((100, 256), 3.0, device="cuda").bfloat16()
    enc.diff_attention(q, k, v, T.offsets([30, 40]), T.offsets([20, 50]), torch.full((4,), 0.5, device="cuda"), out)
    assert (out[70:] == 3).all() and not (out[:70] == 3).all(1).any()
    enc.close()


def test_refusals(K):
    import torch
    enc = T.encoder(64, 32, 2)
    x = torch.zeros(32, 192, device="cuda", dtype=torch.bfloat16)
    cu, lam, g = T.offsets([16, 16]), torch.ones(1, device="cuda"), torch.ones(64, device="cuda")
    p, ld = x.data_ptr(), 192

    def call(q=p, q_ld=ld, n_q=32, k=p + 128, k_ld=ld, v=p + 256, v_ld=ld, n_k=32, cu_q=cu.data_ptr(), cu_k=cu.data_ptr(), B=2, mask=None,
             lam=lam.data_ptr(), g=g.data_ptr(), scale=1.0, out=p, out_ld=ld):
        K.cfdetr_diff_attention(enc.ctx, q, q_ld, n_q, k, k_ld, v, v_ld, n_k, cu_q, cu_k, B, mask, lam, g, scale, out, out_ld, enc._stream())

    call()
    call(n_q=0, q=None, out=None)
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(cu_q=None), dict(cu_k=None), dict(lam=None), dict(B=0), dict(n_q=-1),
               dict(n_k=-1), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(q_ld=60), dict(k_ld=196), dict(v=p + 2), dict(g=g.data_ptr() + 4),
               dict(out_ld=200)):
        with pytest.raises(K.CfdetrError) as e:
            call(**kw)
        assert e.value.status == K.CFDETR_EINVAL and K.cfdetr_last_error(enc.ctx)
    for kw in (dict(B=3), dict(n_q=33), dict(n_k=33)):
        with pytest.raises(K.CfdetrError) as e:
            call(**kw)
        assert e.value.status == K.CFDETR_ECAPACITY
    odd = T.encoder(192, 32, 2, heads=3)
    with pytest.raises(K.CfdetrError) as e:
        K.cfdetr_diff_attention(odd.ctx, p, ld, 32, p, ld, p, ld, 32, cu.data_ptr(), cu.data_ptr(), 2, None, lam.data_ptr(), None, 1.0, p, ld, 0)
    assert e.value.status == K.CFDETR_ESHAPE
    rows = [x[:, i * 64:(i + 1) * 64] for i in range(3)]
    for bad in (dict(q=rows[0].float()), dict(k=rows[1][:, :32]), dict(cu_q=cu.long()), dict(cu_k=cu[:2]), dict(lambda_=lam.double()),
                dict(lambda_=torch.ones(2, device="cuda")), dict(head_g=g[:32]), dict(key_mask=torch.ones(31, dtype=torch.uint8, device="cuda")),
                dict(out=rows[0][:31]), dict(v=rows[2].cpu())):
        kw = dict(dict(q=rows[0], k=rows[1], v=rows[2], cu_q=cu, cu_k=cu, lambda_=lam, out=rows[0]), **bad)
        with pytest.raises(ValueError):
            enc.diff_attention(**kw)
    enc.sync_status()
    odd.close()
    enc.close()
