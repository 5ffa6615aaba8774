"""The memory's operators together, as a program strings them: streams that grow, slide and end, fed by the selection's own
offsets; captured and replayed on other lengths; two graphs and two states on one context; another stream; beside the encoder."""
import numpy as np
import pytest

import differential_reference as T
import stream_memory_reference as R
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


class Program:
    """One layer over the memory of B streams: every step forgets, makes room, turns and writes the new tokens, and asks with one
    token a stream.  Expected results come from a plain record of what every stream has been given."""

    def __init__(self, K, d, kv, B, page, n_pages, cols, capacity, dtype="bf16", enc=None):
        import torch
        self.heads, self.kv, self.d, self.dtype, self.page = T.MODELS[d], kv, d, dtype, page
        self.dh, self.kd = d // self.heads, d // self.heads * kv
        self.enc = enc or T.encoder(d, 8, dtype=dtype)
        if enc is None:
            self.enc.attach_memory(page, n_pages, cols, B, kv)
        self.m = self.enc.alloc_memory(B)
        n = self.dh // 2
        self.pairs = (n // 4, n // 4, n // 2)
        self.params = K.rotary_axes_params(self.dh, self.pairs, in_turn=True)
        freq, axis = K.cfdetr_rotary_axes_table(self.params)
        self.freq, self.axis = torch.tensor(freq, dtype=torch.float64, device="cuda"), torch.tensor(axis, dtype=torch.uint8, device="cuda")
        zeros = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype, device="cuda")
        act = T.act(dtype)
        self.cu, self.drop, self.slots = zeros(B + 1), zeros(B), zeros(capacity)
        self.rows, self.pos = zeros(capacity, 2 * self.kd, dtype=act), zeros(capacity, 3, dtype=torch.float32)
        self.q, self.q_pos = zeros(B, d, dtype=act), zeros(B, 3, dtype=torch.float32)
        self.turned, self.out = zeros(B, d, dtype=act), zeros(B, d, dtype=act)
        self.state = R.State(B, page, self.m["free_pages"].numel(), self.m["table"].shape[1])
        self.kept = [([], []) for _ in range(B)]   # keys (turned, in 64 bits) and values of every stream

    def call(self):
        enc, m = self.enc, self.m
        enc.memory_advance(self.cu, m["span"], m["table"], m["pool"], m["free_pages"], self.slots, drop=self.drop)
        enc.memory_append(self.rows[:, :self.kd], self.rows[:, self.kd:], self.slots, m["k_cache"], m["v_cache"], self.params, self.freq,
                          self.axis, self.pos)
        enc.rotary_axes(self.params, self.freq, self.axis, self.q_pos, self.q, self.turned, q_scale=T.log2e_over(self.dh))
        enc.memory_attention(self.turned, m["k_cache"], m["v_cache"], m["span"], m["table"], self.out, softmax_scale=0.0)

    def feed(self, seed, drop, new):
        import torch
        capacity = self.slots.numel()
        self.cu.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
        self.drop.copy_(torch.tensor(drop, dtype=torch.int32))
        self.rows.copy_(T.normal(seed, capacity, 2 * self.kd))
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.pos.copy_(torch.randint(0, 100, (capacity, 3), generator=g, device="cuda").float() + seed)
        self.q.copy_(T.normal(seed + 1000, *self.q.shape, std=1.5))
        self.q_pos.copy_(torch.randint(0, 100, self.q_pos.shape, generator=g, device="cuda").float() + seed)

    def record(self, drop, new):
        """The step in plain Python, with the rows fed to the device."""
        self.state, slots = R.step(self.state, drop, new)
        axis, freq = R.axes_table(self.pairs, True, False)
        k, size = R.turned(self.rows[:, :self.kd], self.pos, axis, freq, self.kv, False)
        at = 0
        for b, n in enumerate(new):
            keys, values = self.kept[b]
            gone = min(len(keys), int(drop[b]))
            del keys[:gone], values[:gone]
            keys += [k[i].cpu() for i in range(at, at + n)]
            values += [self.rows[i, self.kd:].cpu() for i in range(at, at + n)]
            at += n
        return slots

    def check(self, slots):
        import torch
        m = self.m
        assert self.slots[:len(slots)].tolist() == slots and (self.slots[len(slots):] == -1).all()
        assert (m["span"].cpu().numpy() == self.state.span).all() and (m["pool"].cpu().numpy() == self.state.pool).all()
        # the caches hold what the streams were given: values as they were, keys turned (half a step of the type, and 2^-20 of
        # a pair's length for 32-bit angles and products), and the rows are the softmax over these
        held = [self.state.slots(b) for b in range(len(self.kept))]
        for at, (keys, values) in zip(held, self.kept):
            assert len(at) == len(keys)
            if not at:
                continue
            rows = torch.tensor(at, device="cuda")
            assert torch.equal(m["v_cache"][rows], torch.stack(values).cuda())
            want = torch.stack(keys).cuda()
            T.within(m["k_cache"][rows], want, want.abs() * T.HALF_STEP[self.dtype] + 2.0 ** -18)
        axis, freq = R.axes_table(self.pairs, True, False)
        scale = T.log2e_over(self.dh)
        want, size = R.turned(self.q, self.q_pos, axis, freq, self.heads, False)
        T.within(self.turned, want * scale, (want.abs() * T.HALF_STEP[self.dtype] + size * 2.0 ** -20) * scale * 1.001)
        want, bound = R.attention(self.turned, m["k_cache"], m["v_cache"], held, self.heads, self.kv, self.dtype, np.log(2.0))
        T.within(self.out, want, bound)


@pytest.mark.parametrize("d,kv,B,page,n_pages,cols,most,dtype", [(256, 8, 6, 16, 120, 16, 40, "bf16"), (768, 2, 3, 64, 30, 7, 150, "bf16"), (64, 1, 40, 8, 200, 4, 6, "f32"),
                                                                 (384, 3, 2, 8, 400, 180, 500, "bf16")])
def test_steps_in_a_row(K, d, kv, B, page, n_pages, cols, most, dtype):
    p = Program(K, d, kv, B, page, n_pages, cols, 3 * B * most, dtype)
    rng = np.random.default_rng(B)
    made = 0
    for i in range(8):
        drop, new = R.random_step(rng, p.state, most)
        if R.step(p.state, drop, new) is None:
            new = [n // 8 for n in new]
            if R.step(p.state, drop, new) is None:
                continue
        p.feed(i, drop, new)
        p.call()
        p.check(p.record(drop, new))
        made += 1
    p.enc.sync_status()
    assert made >= 4
    p.enc.close()


def test_captured_and_replayed(K):
    """The same graph on other lengths, with eager steps and waits between: every step as expected."""
    import torch
    p = Program(K, 256, 4, 5, 16, 150, 16, 400)
    rng = np.random.default_rng(2)
    p.feed(50, [0] * 5, [3, 0, 20, 1, 2])
    p.call()
    p.check(p.record([0] * 5, [3, 0, 20, 1, 2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call()
    made = 0
    for i in range(9):
        drop, new = R.random_step(rng, p.state, 60)
        if R.step(p.state, drop, new) is None:
            continue
        p.feed(i, drop, new)
        if i % 3 == 2:
            p.call()
        else:
            graph.replay()
        torch.cuda.synchronize()
        p.check(p.record(drop, new))
        made += 1
    p.enc.sync_status()
    assert made >= 5
    p.enc.close()


def test_two_states_and_graphs_of_one_context(K):
    """They share the context's work space and are replayed in turn; long streams, so that sums are split."""
    import torch
    a = Program(K, 256, 8, 4, 16, 4000, 2000, 30_000)
    b = Program(K, 256, 8, 4, 16, 4000, 2000, 30_000, enc=a.enc)
    steps = [([0, 0, 0, 0], [9000, 11, 7000, 1]), ([4000, 2, 0, 1], [1, 1, 1, 1]), ([0] * 4, [1, 0, 1, 5000])]
    graphs = []
    for p, first in ((a, 0), (b, 1)):
        new = [n + 37 * first for n in steps[0][1]]
        p.feed(first, steps[0][0], new)
        p.call()
        p.record(steps[0][0], new)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.call()
        graphs.append(g)
    for i, (drop, new) in enumerate(steps[1:] * 2):
        order = ((a, graphs[0]), (b, graphs[1]))
        for p, _ in order:
            p.feed(10 * i, drop, new)
        for p, g in order if i % 2 else order[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for p, _ in order:
            p.check(p.record(drop, new))
    a.enc.sync_status()
    a.enc.close()


def test_another_stream(K):
    """The calls go to the current stream, behind what it holds."""
    import torch
    p = Program(K, 256, 8, 3, 16, 300, 100, 3000)
    drop, new = [0, 0, 0], [1000, 1, 500]
    p.feed(1, drop, new)
    rows = p.rows.clone()
    p.rows.zero_()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-3
        p.rows.copy_(rows)
        p.call()
    side.synchronize()
    p.check(p.record(drop, new))
    p.enc.close()


def test_a_step_that_cannot_be_made_writes_no_row(K):
    """The whole run behind a refused step: the caches and the streams are as they were."""
    import torch
    p = Program(K, 256, 8, 3, 16, 6, 5, 400)
    p.feed(1, [0] * 3, [20, 5, 30])
    p.call()
    p.record([0] * 3, [20, 5, 30])
    want = {k: t.clone() for k, t in p.m.items()}
    p.feed(2, [20, 0, 0], [60, 60, 60])
    p.call()
    with pytest.raises(K.CfdetrError) as e:
        p.enc.sync_status()
    assert e.value.status == K.CFDETR_ECAPACITY
    for k, t in want.items():
        assert torch.equal(p.m[k], t), k
    p.check([])
    p.enc.close()


def test_tokens_of_the_selection(K):
    """The new tokens' number comes from the encoder's own selection, without the host: its cu_seqlens are the step's offsets,
    its encoded rows (as they are, d wide) the keys and values, its capacity the padding; and the encoder is undisturbed."""
    import torch
    cfg = synth.Config("memory", 3, 64, 96, (16, 8), 64, 2, 1, 128, "bf16", box_rule="poisson", box_lambda=2.0, side_lo=8, side_hi=40)
    wl = synth.make_workload(cfg, seed=3)
    enc = K.Encoder(cfg, synth.make_weights(cfg, 4))
    enc.attach_memory(16, 100, 30, 3)
    m, out = enc.alloc_memory(3), enc.alloc_outputs(3)
    slots = torch.empty(enc.max_tokens, dtype=torch.int32, device="cuda")
    images, boxes = enc.upload_images(wl["images"]), enc.upload_boxes(wl["boxes"], wl["tier"], wl["box_offsets"])
    kept, before, given = [[] for _ in range(3)], None, 0
    q, row = T.normal(1, 3, 64).bfloat16(), torch.empty(3, 64, device="cuda", dtype=torch.bfloat16)
    for step in range(3):
        enc.multilevel_batch(images, 3, *boxes, out)
        rows = out["y_mixed"].bfloat16()
        # the last frame's tokens replace those of the frame before the last
        drop = torch.tensor([len(k[0]) if len(k) > 1 else 0 for k in kept], dtype=torch.int32, device="cuda")
        enc.memory_advance(out["cu_seqlens"], m["span"], m["table"], m["pool"], m["free_pages"], slots, drop=drop)
        enc.memory_append(rows, rows, slots, m["k_cache"], m["v_cache"])
        enc.memory_attention(q, m["k_cache"], m["v_cache"], m["span"], m["table"], row)
        enc.sync_status()
        cu = out["cu_seqlens"].tolist()
        for b, k in enumerate(kept):
            k.append(slots[cu[b]:cu[b + 1]].tolist())
            del k[:-2]
            assert m["span"][b, 1] == sum(len(x) for x in k)
            want = rows[cu[b]:cu[b + 1]]
            assert torch.equal(m["k_cache"][slots[cu[b]:cu[b + 1]].long()], want)
        assert (slots[cu[3]:] == -1).all()
        want, bound = R.attention(q, m["k_cache"], m["v_cache"], [sum(k, []) for k in kept], 2, 2, "bf16")
        T.within(row, want, bound)
        if before is not None:
            assert all(torch.equal(before[k], out[k]) for k in ("y_mixed", "y_coarse", "tok_desc", "cu_seqlens"))
        before = {k: t.clone() for k, t in out.items()}
    enc.close()


def test_profile_and_tensors_of_another_gpu(K):
    p = Program(K, 64, 2, 2, 8, 10, 4, 20)
    p.feed(1, [0, 0], [3, 4])
    K.cfdetr_profile_begin(p.enc.ctx)
    p.call()
    got = K.cfdetr_profile_end(p.enc.ctx)
    assert [got[k]["launches"] for k in ("plan", "gather", "qkv", "attention")] == [1, 1, 1, 1]
    p.enc.gpu += 1
    with pytest.raises(ValueError):
        p.call()
    p.enc.gpu -= 1
    p.enc.close()
