"""Which rows count as the newest ones of a sequence."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_kv_evict import marked, row_numbers

pytestmark = pytest.mark.gpu


def test_the_newest_of_none_at_the_end_of_the_positions():
    """`recent` = 0 protects nothing, also where a position is the largest that there is."""
    s = R.Setup([60], 1, 16, 16, 16, seed=1)
    cache = s.cache()
    marks, row = B.KVMarks(cache), row_numbers(s, 0, 0, 60).cuda()
    marks.pos.view(-1)[row] = 2 ** 31 - 1
    marks.mass.view(-1)[row] = torch.arange(60, dtype=torch.float32, device="cuda")
    source, _ = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 20, 0)
    cache.check()
    assert source[0, 0].tolist() == list(range(40, 60))


def newest_stay(s, marks, keep, recent):
    """The definition, row by row: the rows whose position is above the largest one - recent, then those of the largest weight."""
    mass, pos = marks.mass.flatten().cpu(), marks.pos.flatten().cpu().long()
    source = torch.full((len(s.lens), s.kv_heads, keep), -1, dtype=torch.int32)
    for b, n in enumerate(s.lens):
        for h in range(s.kv_heads):
            if n <= keep:
                source[b, h, :n] = torch.arange(n)
                continue
            row = row_numbers(s, b, h, n)
            worth = torch.where(mass[row] > 0, mass[row], torch.zeros(n)).double()
            worth[pos[row] > pos[row].max() - recent] = float("inf")
            stays = torch.zeros(n, dtype=torch.bool)
            stays[torch.sort(worth, descending=True, stable=True).indices[:keep]] = True
            source[b, h] = torch.arange(keep)
            source[b, h][~stays[:keep]] = (stays[keep:].nonzero()[:, 0] + keep).to(torch.int32)
    return source.cuda(), torch.tensor([min(n, keep) for n in s.lens], dtype=torch.int32).cuda()


@pytest.mark.parametrize("kv_heads,page,lens,keep,recent", [
    (1, 16, [1, 2, 3], 1, 0),
    (1, 16, [1, 2, 3], 2, 2),
    (3, 16, [0, 33, 32, 31, 64, 65, 97], 32, 5),
    (8, 16, [2064, 2049, 2048, 2047], 2048, 256),
    (1, 256, [5000, 4999], 4998, 10),
    (4, 128, [700] * 90, 333, 100),
    (8, 16, [200, 201, 333] * 25, 100, 50),
    (1, 64, [70001], 4096, 1024),
    (2, 64, [40000, 20000], 39999, 0),
    (2, 64, [40000, 100, 17000], 16385, 7),
    (1, 64, [131000, 130999], 1000, 999),
    (3, 64, [9000, 8000, 13000], 777, 776),
])
def test_rows_in_any_order(kv_heads, page, lens, keep, recent):
    s = R.Setup(lens, kv_heads, 16, page, 16, seed=keep)
    cache, marks = marked(s, 1)
    want, new_lens = newest_stay(s, marks, keep, recent)
    source, got_lens = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, keep, recent, any_order=True)
    cache.check()
    assert torch.equal(source, want) and torch.equal(got_lens, new_lens)


def test_both_forms_agree_behind_an_append():
    s = R.Setup([500, 70, 333], 2, 16, 16, 16, seed=2)
    cache, marks = marked(s, 3)
    for b, n in enumerate(s.lens):
        for h in range(2):
            marks.pos.view(-1)[row_numbers(s, b, h, n)[-1].item()] = 20000  # the newest
    batch = B.KVBatch(s.table, s.kv_lens)
    want, _ = newest_stay(s, marks, 64, 20)
    for any_order in (False, True):
        source, _ = B.kv_select(cache, batch, marks, 64, 20, any_order=any_order)
        assert torch.equal(source, want), any_order
    cache.check()


def test_a_second_cut_before_the_next_append():
    """64 rows cut to 32 with the 8 newest protected, then to 16: they stay.  (The first cut keeps positions 0 to 9, 31, 40 to 52 and 56 to 63
    and leaves position 31 in the last row: above 31 - 8 there are 22, of which the first 16 do not reach beyond position 58.)"""
    s = R.Setup([64], 2, 16, 16, 16, seed=4)
    cache = s.cache()
    marks = B.KVMarks(cache)
    heavy = torch.zeros(64, device="cuda")
    heavy[:10] = heavy[31] = heavy[40:53] = 1.0
    for h in range(2):
        row = row_numbers(s, 0, h, 64).cuda()
        marks.pos.view(-1)[row] = torch.arange(64, dtype=torch.int32, device="cuda")
        marks.mass.view(-1)[row] = heavy
    batch = B.KVBatch(s.table, s.kv_lens)
    graph, held = torch.cuda.CUDAGraph(), {}
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):  # (the second cut, as a server captures it)
        held[0] = B.kv_select(cache, batch, marks, 16, 8, any_order=True)
        B.kv_compact(cache, batch, held[0][0], marks)
    source, new_lens = B.kv_select(cache, batch, marks, 32, 8)
    B.kv_compact(cache, batch, source, marks)
    s.kv_lens.copy_(new_lens)
    last = row_numbers(s, 0, 0, 32)[-1].item()
    assert marks.pos.view(-1)[last].item() == 31, "the last row is not the newest"
    graph.replay()
    cache.check()
    for h in range(2):
        stayed = set(marks.pos.view(-1)[row_numbers(s, 0, h, 16).cuda()].tolist())
        assert len(stayed) == 16 and set(range(56, 64)) <= stayed


def test_bad_pages_and_positions_at_both_ends():
    s = R.Setup([100], 1, 16, 16, 16, seed=6, table_extra=0)
    cache = s.cache()
    marks, row = B.KVMarks(cache), row_numbers(s, 0, 0, 100).cuda()
    marks.mass.view(-1)[row] = torch.arange(100, dtype=torch.float32, device="cuda")
    marks.pos.view(-1)[row] = -2 ** 31
    marks.pos.view(-1)[row[3]] = 2 ** 31 - 1
    batch = B.KVBatch(s.table, s.kv_lens)
    for recent, want in ((0, list(range(80, 100))), (1, [3] + list(range(81, 100))), (20, [3] + list(range(81, 100)))):
        source, _ = B.kv_select(cache, batch, marks, 20, recent, any_order=True)
        assert sorted(source[0, 0].tolist()) == want
    cache.check()
    marks.pos.view(-1)[row[40]] = 7  # the newest where the page of row 3 is no page
    s.table[0, 0] = -1
    source, _ = B.kv_select(cache, batch, marks, 20, 1, any_order=True)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE and sorted(source[0, 0].tolist()) == [40] + list(range(81, 100))


def test_on_a_side_stream_and_without_sequences():
    s = R.Setup([300, 64, 500], 2, 64, 16, 16, seed=12)
    cache, marks = marked(s, 13)
    batch, side = B.KVBatch(s.table, s.kv_lens), torch.cuda.Stream()
    want, new_lens = newest_stay(s, marks, 128, 10)
    torch.cuda.synchronize()
    source, lens = B.kv_select(cache, batch, marks, 128, 10, stream=side, any_order=True)
    torch.cuda.synchronize()
    assert torch.equal(source, want) and torch.equal(lens, new_lens)
    source, lens = B.kv_select(cache, B.KVBatch(s.table[:0], s.kv_lens[:0]), marks, 5, any_order=True)
    assert source.shape == (0, 2, 5) and lens.shape == (0,)
