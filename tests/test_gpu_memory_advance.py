"""Steps of a memory of streams against pages taken and given back one by one: in place and apart, one workgroup and many, padded
slots, steps that cannot be made; and the refusals."""
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


def _up(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _device(s):
    return {"span": _up(s.span), "table": _up(s.table), "pool": _up(s.pool), "free_pages": _up(s.free)}


def _cu(new):
    return _up(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))


def _advance(enc, dev, drop, new, padding, apart, no_drop=False):
    """Takes the step on the device; returns the new state's tensors and the slots, whose surroundings are checked."""
    import torch
    n = int(np.sum(new)) + padding
    room = torch.full((n + 2,), 12345, dtype=torch.int32, device="cuda")
    to = dict(dev)
    outs = {}
    if apart:
        outs = {"span_out": torch.full_like(dev["span"], 77), "table_out": torch.full_like(dev["table"], -9), "pool_out": torch.full_like(dev["pool"], 77)}
        to.update(span=outs["span_out"], table=outs["table_out"], pool=outs["pool_out"])
    enc.memory_advance(_cu(new), dev["span"], dev["table"], dev["pool"], dev["free_pages"], room[1:-1], drop=None if no_drop else _up(np.asarray(drop, dtype=np.int32)), **outs)
    assert room[0] == 12345 and room[-1] == 12345
    return to, room[1:-1]


@pytest.mark.parametrize("streams,page,n_pages,cols,most,padding", [
    (1, 8, 3, 2, 20, 0), (3, 8, 20, 4, 20, 1), (7, 16, 40, 6, 30, 0), (64, 8, 500, 17, 60, 5), (300, 16, 20_000, 40, 600, 0), (1000, 32, 9000, 8, 200, 3),
    (5, 1024, 12, 3, 3000, 0), (2, 256, 300, 200, 40_000, 700), (4096, 8, 9000, 2, 16, 0),
])
def test_steps_in_a_row(K, streams, page, n_pages, cols, most, padding):
    import torch
    enc = T.encoder(64, 8)
    enc.attach_memory(page, n_pages, cols, streams)
    rng = np.random.default_rng(streams + page)
    s = R.State(streams, page, n_pages, cols)
    dev, made = _device(s), 0
    for i in range(14):
        drop, new = R.random_step(rng, s, most)
        if i == 0:
            drop = [0] * streams   # (none given)
        want = R.step(s, drop, new)
        if want is None:
            # a share of it, so that most steps are made
            new = [n // 8 for n in new]
            want = R.step(s, drop, new)
        if want is None:
            continue
        made += 1
        old_table = dev["table"].clone()
        dev, slots = _advance(enc, dev, drop, new, padding, i % 2, i == 0)
        after, want_slots = want
        n = len(want_slots)
        assert slots[:n].tolist() == want_slots and (slots[n:] == -1).all()
        assert (dev["span"].cpu().numpy() == after.span).all() and (dev["pool"].cpu().numpy() == after.pool).all()
        assert (dev["free_pages"].cpu().numpy() == after.free).all()
        table = dev["table"].cpu().numpy()
        held = np.zeros_like(table, dtype=bool)
        for b in range(streams):
            held[b, [j % cols for j in after.pages(b)]] = True
        assert (table[held] == after.table[held]).all()
        # other entries are as they were
        rest = np.full_like(table, -9) if i % 2 else np.where(after.table != s.table, after.table, old_table.cpu().numpy())
        assert (table[~held] == rest[~held]).all()
        after.table[~held] = table[~held]
        s = after
        s.check()
    enc.sync_status()
    assert made >= 6
    enc.close()


def _refused(K, enc, s, drop, cu, n_new, apart=False, **given):
    """The step is not made: state as it was, slots -1, and the status says so."""
    import torch
    dev = dict(_device(s), **given)
    before = {k: t.clone() for k, t in dev.items()}
    slots = torch.full((n_new,), 5, dtype=torch.int32, device="cuda")
    outs = {k + "_out": torch.full_like(dev[k], 77) for k in ("span", "table", "pool")} if apart else {}
    enc.memory_advance(_up(np.asarray(cu, dtype=np.int32)), dev["span"], dev["table"], dev["pool"], dev["free_pages"], slots,
                       drop=None if drop is None else _up(np.asarray(drop, dtype=np.int32)), **outs)
    with pytest.raises(K.CfdetrError) as e:
        enc.sync_status()
    assert e.value.status == K.CFDETR_ECAPACITY
    for k, t in before.items():
        assert torch.equal(dev[k], t), k
    for k in ("span", "table", "pool") if apart else ():
        assert torch.equal(outs[k + "_out"], before[k]), k
    assert (slots == -1).all()
    enc.sync_status()


@pytest.mark.parametrize("streams,n_new", [(3, 40), (700, 3000)])
@pytest.mark.parametrize("apart", (False, True))
def test_steps_that_cannot_be_made(K, streams, n_new, apart):
    """With one workgroup and with many."""
    import torch
    page, cols, n_pages = 8, 3, 2 * streams
    enc = T.encoder(64, 8)
    enc.attach_memory(page, n_pages, cols, streams)
    s, _ = R.step(R.State(streams, page, n_pages, cols), [0] * streams, [9] + [3] * (streams - 1))
    even = np.arange(streams + 1)
    zero = np.zeros(streams + 1, dtype=np.int32)
    enough = np.minimum(1, even)
    wanted = [0, 6, 6] if streams == 3 else [14] + [4] * (streams - 1)     # a page or more, and none is free
    _refused(K, enc, s, None, np.concatenate([[0], np.cumsum(wanted)]), n_new, apart, pool=torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
    _refused(K, enc, s, None, enough * 16, n_new, apart)                   # a fourth page of a ring of three
    _refused(K, enc, s, None, enough * (n_new + 1), n_new, apart)          # beyond the slots
    _refused(K, enc, s, None, zero + 1, n_new, apart)                      # not from 0
    _refused(K, enc, s, None, np.concatenate([[0, 4], 3 + zero[2:]]), n_new, apart)   # descending
    _refused(K, enc, s, None, np.concatenate([[0, -1], zero[2:]]), n_new, apart)
    _refused(K, enc, s, np.concatenate([[-1], zero[2:]]), zero, n_new, apart)
    for span in ([-1, 4], [24, 1], [3, -2], [0, 25], [1, 24], [2 ** 31 - 1, 2 ** 31 - 1]):
        bad = _up(s.span)
        bad[-1] = torch.tensor(span, dtype=torch.int32)
        _refused(K, enc, s, None, enough, n_new, apart, span=bad)
    for pool in ([-1, 4], [n_pages, 4], [0, -1], [0, n_pages + 1]):
        _refused(K, enc, s, None, zero, n_new, apart, pool=torch.tensor(pool, dtype=torch.int32, device="cuda"))
    # (all pages free and some given back)
    _refused(K, enc, s, np.full(streams, 2 ** 31 - 1), zero, n_new, apart, pool=torch.tensor([1, n_pages], dtype=torch.int32, device="cuda"))
    enc.close()


def test_page_numbers_that_are_none(K):
    """A list that no step has left: no slot comes of it, and the status says so."""
    import torch
    enc = T.encoder(64, 8)
    enc.attach_memory(8, 10, 4, 2)
    s = R.State(2, 8, 10, 4)
    s.free[:4] = 3, -1, 10, 2 ** 31 - 1
    dev, slots = _advance(enc, _device(s), None, [16, 16], 0, False, True)
    assert slots.tolist() == list(range(24, 32)) + [-1] * 24
    with pytest.raises(K.CfdetrError):
        enc.sync_status()
    enc.close()


def test_no_new_tokens(K):
    """No slots, no tensor for them; streams without tokens keep nothing."""
    import torch
    enc = T.encoder(64, 8)
    enc.attach_memory(8, 10, 4, 3)
    s, _ = R.step(R.State(3, 8, 10, 4), [0] * 3, [9, 0, 8])
    dev, slots = _advance(enc, _device(s), [4, 0, 8], [0, 0, 0], 0, False)
    after, _ = R.step(s, [4, 0, 8], [0, 0, 0])
    assert slots.numel() == 0 and dev["span"].tolist() == after.span.tolist() == [[4, 5], [0, 0], [0, 0]]
    assert dev["pool"].tolist() == after.pool.tolist() and dev["free_pages"].tolist() == after.free.tolist()
    enc.sync_status()
    enc.close()


def test_refusals(K):
    import torch
    enc = T.encoder(64, 8)
    lib = K.load_library()
    i = torch.zeros(64, dtype=torch.int32, device="cuda")
    p, q = i.data_ptr(), i.data_ptr() + 64

    def call(B=2, drop=p, cu=p, n_new=4, span=p, span_out=p, table=p, table_out=p, pool=p, pool_out=p, free=p, slots=p):
        K.cfdetr_memory_advance(enc.ctx, B, drop, cu, n_new, span, span_out, table, table_out, pool, pool_out, free, slots, enc._stream())

    with pytest.raises(K.CfdetrError) as e:
        call()
    assert e.value.status == K.CFDETR_EINVAL
    for bad in (dict(page_size=12), dict(n_pages=0), dict(max_pages=0), dict(max_streams=5000), dict(n_kv_heads=3), dict(page_size=1024, n_pages=1 << 22)):
        with pytest.raises(K.CfdetrError) as e:
            enc.attach_memory(**dict(dict(page_size=8, n_pages=10, max_pages=4, max_streams=2), **bad))
        assert e.value.status == K.CFDETR_ESHAPE and K.cfdetr_last_error(enc.ctx)
    assert lib.cfdetr_memory_attach(enc.ctx, None) == K.CFDETR_EINVAL
    enc.attach_memory(8, 10, 4, 2)
    with pytest.raises(K.CfdetrError) as e:
        enc.attach_memory(8, 10, 4, 2)
    assert e.value.status == K.CFDETR_EINVAL
    for bad, status in ((dict(B=0), K.CFDETR_EINVAL), (dict(B=3), K.CFDETR_ECAPACITY), (dict(n_new=-1), K.CFDETR_EINVAL), (dict(n_new=(1 << 30) + 1), K.CFDETR_EINVAL),
                        *((dict([(name, value)]), K.CFDETR_EINVAL) for name in ("cu", "span", "span_out", "table", "table_out", "pool", "pool_out", "free", "slots")
                          for value in (None, p + 2)), (dict(drop=p + 1), K.CFDETR_EINVAL), (dict(span=p + 4), K.CFDETR_EINVAL), (dict(span_out=p + 4), K.CFDETR_EINVAL)):
        with pytest.raises(K.CfdetrError) as e:
            call(**bad)
        assert e.value.status == status and K.cfdetr_last_error(enc.ctx), bad
    enc.sync_status()
    enc.close()
