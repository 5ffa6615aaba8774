"""Steps of a memory of streams with more new tokens than one a thread of the chip (four consecutive slots a thread), and steps in
place that give many pages back."""
import numpy as np
import pytest

import differential_reference as T
import stream_memory_reference as R
from test_gpu_memory_advance import _advance, _device, _refused

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _most_of_one_slot():
    """Slots up to which a thread has one."""
    import torch
    return 512 * torch.cuda.get_device_properties(0).multi_processor_count


def _check(s, after, want_slots, dev, slots, old, apart):
    """Slots, state, and every entry of the table: those that are held, and the others as they were."""
    n = len(want_slots)
    assert np.array_equal(slots[:n].cpu().numpy(), want_slots) and (slots[n:] == -1).all()
    assert (dev["span"].cpu().numpy() == after.span).all() and (dev["pool"].cpu().numpy() == after.pool).all()
    assert (dev["free_pages"].cpu().numpy() == after.free).all()
    table = dev["table"].cpu().numpy()
    held = np.zeros_like(table, dtype=bool)
    for b in range(len(after.span)):
        held[b, [j % s.cols for j in after.pages(b)]] = True
    assert (table[held] == after.table[held]).all()
    rest = np.full_like(table, -9) if apart else np.where(after.table != s.table, after.table, old)
    assert (table[~held] == rest[~held]).all()


def _step(enc, s, drop, new, padding, apart):
    dev = _device(s)
    want = R.step(s, drop, new)
    assert want is not None
    dev, slots = _advance(enc, dev, drop, new, padding, apart)
    _check(s, *want, dev, slots, s.table, apart)
    enc.sync_status()
    want[0].check()
    return want[0]


@pytest.mark.parametrize("apart", (False, True))
@pytest.mark.parametrize("padding", (0, 1, 2, 5, 1023))
def test_many_streams_with_runs_of_empty_ones(K, apart, padding):
    """Ends of streams and pages inside a thread's four slots, streams without tokens between, the last tokens and the padding too."""
    most = _most_of_one_slot()
    rng = np.random.default_rng(padding + apart)
    streams, page, cols = 1000, 8, 400
    new = rng.integers(0, 4 * most // streams, streams)
    new[rng.random(streams) < 0.4] = 0      # (runs of several)
    small = rng.random(streams) < 0.3
    new[small] = rng.integers(0, 6, int(small.sum()))
    new[:3], new[-4:] = 0, 0
    while new.sum() <= most or new.sum() % 4 == 0:
        new[rng.integers(3, streams - 4)] += 101
    before = rng.integers(0, 40, streams)
    enc = T.encoder(64, 8)
    n_pages = int((before // page + new // page + 3).sum())
    enc.attach_memory(page, n_pages, cols, streams)
    assert new.max() + 60 < page * cols and new.sum() > most
    s, _ = R.step(R.State(streams, page, n_pages, cols), [0] * streams, before)
    _step(enc, s, [int(rng.choice([0, 1, h, rng.integers(0, h + 1)])) for h in before], new, padding, apart)
    enc.close()


@pytest.mark.parametrize("apart", (False, True))
@pytest.mark.parametrize("page", (8, 1024))
def test_few_long_streams(K, apart, page):
    """A step of few streams with very many tokens, then one that forgets most of them and adds as many: rings go round."""
    most = _most_of_one_slot()
    lengths = [most // 2 + 3, 0, most // 2 + 1001, 1]
    enc = T.encoder(64, 8)
    cols = max(lengths) // page + 9
    n_pages = 2 * sum(n // page + 3 for n in lengths)
    enc.attach_memory(page, n_pages, cols, 4)
    s = _step(enc, R.State(4, page, n_pages, cols), [0] * 4, lengths, 3, apart)
    s = _step(enc, s, [lengths[0] - 17, 0, lengths[2], 0], lengths, 0, apart)
    _step(enc, s, [lengths[0], 0, 5, 1], [lengths[0] - 30, lengths[2], 4, 0], 2, not apart)
    enc.close()


@pytest.mark.parametrize("apart", (False, True))
def test_steps_that_cannot_be_made_with_many_slots(K, apart):
    import torch
    n_new = _most_of_one_slot() + 1001
    streams, page, cols = 5, 8, n_new // 8 + 2
    n_pages = cols + 40
    enc = T.encoder(64, 8)
    enc.attach_memory(page, n_pages, cols, streams)
    s, _ = R.step(R.State(streams, page, n_pages, cols), [0] * streams, [9, 0, 33, 8, 1])
    _refused(K, enc, s, None, [0, n_new, n_new, n_new, n_new, n_new], n_new, apart, pool=torch.tensor([0, n_pages // 2], dtype=torch.int32, device="cuda"))
    _refused(K, enc, s, None, [0, n_new + 1] + [n_new + 1] * 4, n_new, apart)
    _refused(K, enc, s, None, [0, 5, 4, 5, 5, 5], n_new, apart)
    _refused(K, enc, s, [0, 0, -1, 0, 0], [0, 1, 2, 3, 4, n_new], n_new, apart)
    _step(enc, s, [9, 0, 1, 0, 0], [3, n_new - 50, 0, 1, 0], 46, apart)
    enc.close()


@pytest.mark.parametrize("streams,page,held,new", [(1, 8, 200_003, 1), (1, 8, 200_003, 0), (40, 8, 5_001, 3), (3000, 16, 100, 1), (6, 1024, 100_000, 1500)])
@pytest.mark.parametrize("window", (False, True))
def test_many_pages_given_back_in_place(K, streams, page, held, new, window):
    """Few tokens come, whole streams or most of them go, and the table stays: page numbers of many workgroups, state over the old one."""
    cols = held // page + 4
    enc = T.encoder(64, 8)
    n_pages = streams * (held // page + 3)
    enc.attach_memory(page, n_pages, cols, streams)
    rng = np.random.default_rng(held)
    s = R.State(streams, page, n_pages, cols)
    s.free[:] = rng.permutation(n_pages)
    s.pool[0] = n_pages // 3
    s, _ = R.step(s, [0] * streams, [held - b % 5 for b in range(streams)])
    drop = [(held * 9 // 10 if b % 3 else 1) if window else (2 ** 31 - 1 if b % 3 < 2 else 0) for b in range(streams)]
    if window and streams == 1:
        drop = [held - 20]
    s = _step(enc, s, drop, [new] * streams, 2, False)
    _step(enc, s, [2 ** 31 - 1] * streams, [new] * streams, 0, False)
    enc.close()
