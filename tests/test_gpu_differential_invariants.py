"""What the encode calls promise of their results bit for bit, of contexts with attached differential layers: a frame's rows do not
depend on an earlier run of the context, on the frame's batch, on the call it comes from, or on padding; and a captured pass gives on every
replay what an eager one gives."""
import numpy as np
import pytest

from paper_2505_23317_amd import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


# Frames of 400 to 2,400 tokens: one of them is few queries, all of them are many for 256 CUs (rows times heads on both
# sides of 16,384, tiles of 128 on both sides of one a CU).
CFGS = {
    64: synth.Config("same64", 3, 128, 128, (16, 8), 64, 2, 2, 128, "bf16", box_rule="poisson", box_lambda=3.0, side_lo=16, side_hi=90),
    256: synth.Config("same256", 6, 320, 480, (16, 8), 256, 8, 2, 512, "bf16", box_rule="fraction", frac_lo=0.0, frac_hi=1.0, side_lo=32, side_hi=160),
    384: synth.Config("same384", 6, 320, 480, (32, 16, 8), 384, 6, 2, 768, "bf16", box_rule="tiered", box_lambda=9.0, side_lo=32, side_hi=160),
    768: synth.Config("same768", 4, 256, 256, (16, 8), 768, 12, 1, 1536, "bf16", box_rule="fraction", frac_lo=0.0, frac_hi=1.0, side_lo=32, side_hi=160),
}
FORMS = [(64, "bf16"), (256, "bf16"), (384, "bf16"), (768, "bf16"), (64, "f32"), (256, "f32"), (384, "f32")]


def _encoder(K, cfg, dtype, seed=5):
    """A context of that shape; logits have a spread of a few units (sharp), so that a running maximum moves often."""
    rng = np.random.default_rng(seed)
    enc = K.Encoder(cfg, synth.make_weights(cfg, 4, sharp=True), act_dtype=dtype)
    diff = {"lambda": rng.uniform(0.2, 0.9, (cfg.layers, cfg.heads // 2)).astype(np.float32)}
    for name, n in (("head_g", 2 * cfg.d_head), ("post1_g", cfg.d), ("post2_g", cfg.d), ("gate1", cfg.d), ("gate2", cfg.d)):
        diff[name] = (0.5 + 0.1 * rng.standard_normal((cfg.layers, n))).astype(np.float32)
    enc.attach_differential(diff, K.rotary_params(cfg.d_head, base=100.0))
    return enc


def _frames(wl, lo, hi):
    """Frames lo..hi of a workload, as arguments of upload_images and upload_boxes."""
    a, b = int(wl["box_offsets"][lo]), int(wl["box_offsets"][hi])
    return wl["images"][lo:hi], wl["boxes"][a:b], wl["tier"][a:b], wl["box_offsets"][lo:hi + 1] - wl["box_offsets"][lo]


def _upload(enc, images, boxes, tier, offsets):
    return enc.upload_images(images), enc.upload_boxes(boxes, tier, offsets)


def _merged(enc, img, boxes):
    out = enc.alloc_outputs(img.shape[0])
    enc.multilevel_batch(img, img.shape[0], *boxes, out)
    enc.sync_status()
    return out


def _three_calls(enc, img, boxes):
    B = img.shape[0]
    out = enc.alloc_outputs(B)
    enc.coarse_encode(img, B, out["x0_cache"], out["y_coarse"])
    enc.select_fine(*boxes, B, out["tok_desc"], out["cu_seqlens"])
    enc.fine_encode(img, B, out["tok_desc"], out["cu_seqlens"], out["x0_cache"], out["y_mixed"])
    enc.sync_status()
    return out


def _same(a, b, what):
    import torch
    assert torch.equal(a["cu_seqlens"], b["cu_seqlens"])
    n = int(a["cu_seqlens"][-1])
    for k, x, y in (("y_coarse", a["y_coarse"], b["y_coarse"]), ("y_mixed", a["y_mixed"][:n], b["y_mixed"][:n])):
        differ = int((x != y).any(1).sum())
        assert torch.equal(x, y), f"{what}: {differ} of {x.shape[0]} rows of {k} differ"


@pytest.mark.parametrize("d,dtype", FORMS)
def test_earlier_runs_do_not_show(K, d, dtype):
    """Small, large and small batches in turn: the first of each has another run's row count, or none, to go by."""
    cfg = CFGS[d]
    wl = synth.make_workload(cfg, seed=3)
    enc = _encoder(K, cfg, dtype)
    batches = [_upload(enc, *_frames(wl, 0, 1)), _upload(enc, *_frames(wl, 0, cfg.B))]
    for form in (_merged, _three_calls):
        first = {}
        for i in (0, 1, 1, 0, 0, 1):
            out = form(enc, *batches[i])
            print(f"{d} {dtype} {form.__name__}: {int(out['cu_seqlens'][-1])} tokens", flush=True)
            _same(first.setdefault(i, out), out, f"{form.__name__}, batch {i} again")
    enc.close()


@pytest.mark.parametrize("d,dtype", FORMS)
def test_one_call_gives_what_three_give(K, d, dtype):
    cfg = CFGS[d]
    wl = synth.make_workload(cfg, seed=4)
    enc = _encoder(K, cfg, dtype)
    for lo, hi in ((0, cfg.B), (1, 2)):
        img, boxes = _upload(enc, *_frames(wl, lo, hi))
        _same(_merged(enc, img, boxes), _three_calls(enc, img, boxes), f"frames {lo} to {hi}")
    enc.close()


@pytest.mark.parametrize("d,dtype", FORMS)
def test_a_batch_gives_what_its_frames_give_alone(K, d, dtype):
    import torch
    cfg = CFGS[d]
    wl = synth.make_workload(cfg, seed=6)
    enc, alone = _encoder(K, cfg, dtype), _encoder(K, synth.replace(cfg, B=1), dtype)
    whole = _merged(enc, *_upload(enc, *_frames(wl, 0, cfg.B)))
    cu = whole["cu_seqlens"].tolist()
    for f in range(cfg.B):
        for one in (enc, alone):   # with room for the batch, and for one frame
            got = _merged(one, *_upload(one, *_frames(wl, f, f + 1)))
            n = cu[f + 1] - cu[f]
            assert got["cu_seqlens"].tolist() == [0, n]
            assert torch.equal(got["y_mixed"][:n], whole["y_mixed"][cu[f]:cu[f + 1]]), f"frame {f}, {n} tokens"
            assert torch.equal(got["y_coarse"], whole["y_coarse"][f * enc.n0:(f + 1) * enc.n0]), f"frame {f}, coarse"
    enc.close()
    alone.close()


@pytest.mark.parametrize("cfg_id,frames", [(3, 6), (4, 4), (5, 8)])
def test_the_configurations_frame_by_frame(K, cfg_id, frames):
    """With as many rows as the contractions have tiles for: first and last frame alone, the batch twice, and in three calls."""
    import torch
    cfg = synth.replace(synth.config(cfg_id), B=frames, layers=2)
    wl = synth.make_workload(cfg, seed=11)
    enc, alone = _encoder(K, cfg, "bf16"), _encoder(K, synth.replace(cfg, B=1), "bf16")
    img, boxes = _upload(enc, *_frames(wl, 0, frames))
    whole = _merged(enc, img, boxes)
    cu = whole["cu_seqlens"].tolist()
    print(f"config {cfg_id}: {cu[-1]} mixed tokens, {frames * enc.n0} coarse ones", flush=True)
    _same(whole, _merged(enc, img, boxes), "again")
    _same(whole, _three_calls(enc, img, boxes), "three calls")
    for f in (0, frames - 1):
        got = _merged(alone, *_upload(alone, *_frames(wl, f, f + 1)))
        assert torch.equal(got["y_mixed"][:cu[f + 1] - cu[f]], whole["y_mixed"][cu[f]:cu[f + 1]]), f"frame {f}"
        assert torch.equal(got["y_coarse"], whole["y_coarse"][f * enc.n0:(f + 1) * enc.n0]), f"frame {f}, coarse"
    enc.close()
    alone.close()


@pytest.mark.parametrize("extra", (0, 37))
@pytest.mark.parametrize("d,dtype", FORMS)
def test_padding_does_not_show(K, d, dtype, extra):
    import torch
    cfg = CFGS[d]
    wl = synth.make_workload(cfg, seed=7)
    enc = _encoder(K, cfg, dtype)
    img, boxes = _upload(enc, *_frames(wl, 0, 3))
    out = _three_calls(enc, img, boxes)
    cu = out["cu_seqlens"].tolist()
    t_pad = max(max(b - a for a, b in zip(cu, cu[1:])), enc.n0)
    t_pad = min(t_pad + extra, enc.max_tokens // 3)
    padded = torch.zeros(3 * t_pad, cfg.d, device="cuda")
    enc.fine_encode_padded(img, 3, out["tok_desc"], out["cu_seqlens"], out["x0_cache"], t_pad, padded)
    enc.sync_status()
    print(f"{d} {dtype}: {cu} padded to {t_pad}", flush=True)
    for f in range(3):
        n = cu[f + 1] - cu[f]
        got, want = padded[f * t_pad:f * t_pad + n], out["y_mixed"][cu[f]:cu[f + 1]]
        assert torch.equal(got, want), f"frame {f}: {int((got != want).any(1).sum())} of {n} rows differ"
    assert torch.isfinite(padded).all()
    enc.close()


@pytest.mark.parametrize("d,dtype", [(256, "bf16"), (384, "bf16"), (256, "f32")])
def test_captured_and_replayed(K, d, dtype):
    """The coarse and the fine pass: every replay against the eager result, with other frames, token sets, eager passes and waits
    between them."""
    import torch
    cfg = CFGS[d]
    loads = [synth.make_workload(cfg, seed=s) for s in (8, 9, 10)]
    enc = _encoder(K, cfg, dtype)
    img = enc.upload_images(loads[0]["images"]).clone()
    out = enc.alloc_outputs(cfg.B)

    def put(wl):
        img.copy_(enc.upload_images(wl["images"]))
        enc.select_fine(*enc.upload_boxes(wl["boxes"], wl["tier"], wl["box_offsets"]), cfg.B, out["tok_desc"], out["cu_seqlens"])

    def call(to):
        enc.coarse_encode(img, cfg.B, to["x0_cache"], to["y_coarse"])
        enc.fine_encode(img, cfg.B, out["tok_desc"], out["cu_seqlens"], to["x0_cache"], to["y_mixed"])

    put(loads[0])
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in (0, 1, 2, 1, 0):
        put(loads[i])
        eager = dict(enc.alloc_outputs(cfg.B), cu_seqlens=out["cu_seqlens"])
        call(eager)
        torch.cuda.synchronize()
        for k in ("x0_cache", "y_coarse", "y_mixed"):
            out[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        _same(eager, out, f"replay with frames {i}")
    enc.sync_status()
    enc.close()


def test_hidden_rows_that_no_product_takes_are_refused_when_attached(K):
    """32,768 rows and 65,536 hidden columns are 4 GiB, which the contractions do not address: refused before anything is enqueued.
    The context goes on with what it was: a coarse pass of plain layers."""
    cfg = synth.replace(CFGS[64], B=1, layers=1, ffn=65_536)
    weights = synth.make_weights(cfg, 4)
    n0 = cfg.n_cells(0)
    diff = {"lambda": np.full((1, 1), 0.5, np.float32)}
    for tokens, fits in ((32_767 - n0, True), (32_768 - n0, False)):
        enc = K.Encoder(cfg, weights, max_tokens_total=tokens)
        if fits:
            enc.attach_differential(diff, K.rotary_params(32))
        else:
            with pytest.raises(K.CfdetrError) as e:
                enc.attach_differential(diff, K.rotary_params(32))
            assert e.value.status == K.CFDETR_ECAPACITY and "hidden rows" in str(e.value)
        img, boxes = _upload(enc, *_frames(synth.make_workload(CFGS[64], seed=3), 0, 1))
        out = enc.alloc_outputs(1)
        enc.coarse_encode(img, 1, out["x0_cache"], out["y_coarse"])
        if fits:
            enc.multilevel_batch(img, 1, *boxes, out)
        enc.sync_status()
        assert np.isfinite(out["y_coarse"].cpu().numpy()).all()
        enc.close()
