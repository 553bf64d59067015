"""Choosing the rows of a cache that stay, and moving them, against a plain restatement on the CPU."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B

pytestmark = pytest.mark.gpu


def marked(s, seed, ties=True):
    """Marks with weights of all sizes (many of them equal where `ties`) and positions in any order."""
    cache = s.cache()
    marks = B.KVMarks(cache)
    g = torch.Generator().manual_seed(seed)
    mass = torch.exp(3 * torch.randn(marks.mass.shape, generator=g))
    if ties:
        few = torch.tensor([0.0, 1.0, 2.0 ** -126, 1.0000001, 5.0])
        mass = torch.where(torch.rand(mass.shape, generator=g) < 0.7, few[torch.randint(0, 5, mass.shape, generator=g)], mass)
    marks.mass.copy_(mass)
    marks.pos.copy_(torch.randint(0, 10000, marks.pos.shape, generator=g, dtype=torch.int32))
    return cache, marks


def row_numbers(s, b, h, n):
    i = torch.arange(n)
    page = s.table[b].cpu().long()[i // s.page_size]
    return (page * s.kv_heads + h) * s.page_size + i % s.page_size


def select(s, marks, keep, recent):
    """The definition, row by row."""
    mass, pos = marks.mass.flatten().cpu(), marks.pos.flatten().cpu().long()
    source = torch.full((len(s.lens), s.kv_heads, keep), -1, dtype=torch.int32)
    for b, n in enumerate(s.lens):
        for h in range(s.kv_heads):
            if n <= keep:
                source[b, h, :n] = torch.arange(n)
                continue
            row = row_numbers(s, b, h, n)
            worth = torch.where(mass[row] > 0, mass[row], torch.zeros(n)).double()
            worth[pos[row] > pos[row][-1] - recent] = float("inf")
            stays = torch.zeros(n, dtype=torch.bool)
            stays[torch.sort(worth, descending=True, stable=True).indices[:keep]] = True
            source[b, h] = torch.arange(keep)
            source[b, h][~stays[:keep]] = (stays[keep:].nonzero()[:, 0] + keep).to(torch.int32)
    return source.cuda(), torch.tensor([min(n, keep) for n in s.lens], dtype=torch.int32).cuda()


SELECT = [
    # kv_heads, page, lens, keep, recent
    (1, 16, [1, 2, 3], 1, 0),
    (1, 16, [1, 2, 3], 2, 2),
    (3, 16, [0, 33, 32, 31, 64, 65, 97], 32, 5),
    (2, 64, [500, 1000, 63, 65], 64, 64),
    (8, 16, [2064, 2049, 2048, 2047], 2048, 256),
    (1, 256, [5000, 4999], 4998, 10),
    (2, 32, [3001], 1, 1),
    (2, 32, [3001], 1000, 0),
    (4, 128, [700] * 90, 333, 100),
    (1, 64, [70001], 4096, 1024),
    (2, 64, [40000, 20000], 39999, 0),
    (2, 64, [40000, 100, 17000], 16385, 7),
]


@pytest.mark.parametrize("kv_heads,page,lens,keep,recent", SELECT)
@pytest.mark.parametrize("ties", [True, False])
def test_select_against_the_definition(kv_heads, page, lens, keep, recent, ties):
    s = R.Setup(lens, kv_heads, 16, page, 16, seed=keep)
    cache, marks = marked(s, 1, ties)
    batch = B.KVBatch(s.table, s.kv_lens)
    want, new_lens = select(s, marks, keep, recent)
    source, got_lens = B.kv_select(cache, batch, marks, keep, recent)
    cache.check()
    assert torch.equal(source, want) and torch.equal(got_lens, new_lens)
    source.fill_(-9)
    B.kv_select(cache, batch, marks, keep, recent, source=source, new_lens=got_lens)
    assert torch.equal(source, want)


@pytest.mark.parametrize("extra", [0, 2000, 16300])
def test_select_with_a_long_page_table(extra):
    """What the page table could hold decides how many CTAs share a sequence, not what the sequences are."""
    s = R.Setup([900, 37, 1025], 2, 16, 16, 16, seed=2, table_extra=extra)
    cache, marks = marked(s, 3)
    want, new_lens = select(s, marks, 100, 20)
    source, got = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 100, 20)
    cache.check()
    assert torch.equal(source, want) and torch.equal(got, new_lens)


def test_select_of_weights_that_are_no_weights():
    """Negative ones and NaN count as nothing, infinities as the most but for the newest; all equal: the first stay."""
    s = R.Setup([200], 1, 16, 16, 16, seed=4)
    cache, marks = marked(s, 5)
    batch, row = B.KVBatch(s.table, s.kv_lens), row_numbers(s, 0, 0, 200).cuda()
    mass, pos = marks.mass.view(-1), marks.pos.view(-1)
    pos[row] = torch.arange(200, dtype=torch.int32, device="cuda")
    mass[row[:50]], mass[row[50:60]], mass[row[60:70]] = float("nan"), -1.0, float("inf")
    mass[row[70:]] = 0.0
    source, _ = B.kv_select(cache, batch, marks, 30, 15)
    # ten infinities, fifteen newest, and five of the equal ones, the first
    assert source[0, 0].tolist() == [0, 1, 2, 3, 4] + list(range(60, 70)) + list(range(185, 200))
    for value in (0.0, float("nan"), 7.0, float("inf")):
        mass[row] = value
        source, _ = B.kv_select(cache, batch, marks, 30, 0)
        assert source[0, 0].tolist() == list(range(30))
    pos[row] = 5  # positions that say all rows are new
    source, _ = B.kv_select(cache, batch, marks, 30, 1)
    assert source[0, 0].tolist() == list(range(30))
    pos[row], pos[row[-1]] = -2 ** 31, 2 ** 31 - 1
    source, _ = B.kv_select(cache, batch, marks, 30, 30)
    assert source[0, 0].tolist() == list(range(29)) + [199] or source[0, 0].tolist()[29] == 199
    cache.check()


def test_select_with_bad_pages_and_lengths():
    s = R.Setup([100, 60], 2, 16, 16, 16, seed=6, table_extra=0)
    cache, marks = marked(s, 7, ties=False)
    marks.pos.zero_()
    page = s.table[0, 2].item()
    s.table[0, 2] = -1
    source, lens = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 50, 0)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE and lens.tolist() == [50, 50]
    s.table[0, 2] = page
    marks.mass[page] = 0.0
    want, _ = select(s, marks, 50, 0)
    assert torch.equal(source, want), "rows on a bad page are worth nothing"
    s.kv_lens[1] = 1000  # beyond the page table: cut to it
    s.lens[1] = s.table.shape[1] * 16
    s.table[1] = s.table[0]
    source, lens = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 50, 0)
    with pytest.raises(B.BitLinearError):
        cache.check()
    want, new_lens = select(s, marks, 50, 0)
    assert torch.equal(source, want) and torch.equal(lens, new_lens)


def everything(s, marks):
    kind = torch.int16 if s.bits == 16 else torch.int8
    got = [p.view(kind) for p in s.pools] + [z.view(torch.int32) for z in s.scales if z is not None]
    return got + ([] if marks is None else [marks.mass.view(torch.int32), marks.pos])


@pytest.mark.parametrize("heads_dim_page", [(1, 4, 16), (3, 100, 16), (8, 128, 64), (2, 64, 256), (5, 20, 32)])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("with_marks", [True, False])
def test_compact_moves_what_select_says(heads_dim_page, bits, with_marks):
    kv_heads, head_dim, page = heads_dim_page
    lens, keep = [333, 0, 100, 101, 1500, 40], 100
    s = R.Setup(lens, kv_heads, head_dim, page, bits, seed=8)
    cache, marks = marked(s, 9)
    batch = B.KVBatch(s.table, s.kv_lens)
    source, _ = B.kv_select(cache, batch, marks, keep, 30)
    given = marks if with_marks else None
    want = [x.clone() for x in everything(s, marks)]
    for i, x in enumerate(want):
        if not with_marks and i >= len(want) - 2:
            continue
        flat = x.view(-1, x.shape[-1]) if x.dim() == 4 else x.view(-1)
        for b, n in enumerate(lens):
            for h in range(kv_heads):
                src = source[b, h].long()
                src = src[src >= 0]
                row = row_numbers(s, b, h, n).cuda()
                flat[row[:len(src)]] = flat[row[src]]
    B.kv_compact(cache, batch, source, given)
    cache.check()
    for x, y in zip(everything(s, marks), want):
        assert torch.equal(x, y)
    B.kv_compact(cache, batch, source, given)  # nothing is read and written: the same again
    for x, y in zip(everything(s, marks), want):
        assert torch.equal(x, y)


def test_compact_leaves_out_what_it_cannot_move():
    """Sources that are destinations, behind the end or negative, and rows on bad pages."""
    s = R.Setup([60, 45], 1, 32, 16, 16, seed=10)
    cache, marks = marked(s, 11)
    batch = B.KVBatch(s.table, s.kv_lens)
    before = [x.clone() for x in everything(s, marks)]
    source = torch.arange(32, dtype=torch.int32, device="cuda").expand(2, 1, 32).contiguous()
    for bad in (3, 60, -2, 2 ** 31 - 1, -2 ** 31):
        source[0, 0, 7] = bad
        B.kv_compact(cache, batch, source, marks)
        with pytest.raises(B.BitLinearError) as e:
            cache.check()
        assert e.value.status == B.ERR_PAGE
        assert all(torch.equal(x, y) for x, y in zip(everything(s, marks), before))
    source[0, 0, 7] = -1
    source[1, 0, 3], source[1, 0, 4] = 44, 44  # (twice the same source is fine)
    s.table[0, 3] = s.n_pages
    source[0, 0, 8], source[0, 0, 9] = 50, 47  # 50 lies on the bad page
    B.kv_compact(cache, batch, source, marks)
    with pytest.raises(B.BitLinearError):
        cache.check()
    row0, row1 = row_numbers(s, 0, 0, 48).cuda(), row_numbers(s, 1, 0, 45).cuda()
    for x, y in zip(everything(s, marks), before):
        y = y.clone()
        flat = y.view(-1, y.shape[-1]) if y.dim() == 4 else y.view(-1)
        flat[row1[3]], flat[row1[4]], flat[row0[9]] = flat[row1[44]].clone(), flat[row1[44]].clone(), flat[row0[47]].clone()
        assert torch.equal(x, y)


def test_on_a_side_stream_and_in_a_graph():
    s = R.Setup([300, 64, 500], 2, 64, 16, 16, seed=12)
    cache, marks = marked(s, 13)
    batch, side = B.KVBatch(s.table, s.kv_lens), torch.cuda.Stream()
    want, new_lens = select(s, marks, 128, 10)
    torch.cuda.synchronize()
    source, lens = B.kv_select(cache, batch, marks, 128, 10, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(source, want) and torch.equal(lens, new_lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_select(cache, batch, marks, 128, 10, source=source, new_lens=lens)
        B.kv_compact(cache, batch, source, marks)
    s.kv_lens.copy_(torch.tensor([129, 500, 64], dtype=torch.int32))
    s.table[1:] = s.table[1:].flip(0)
    s.lens = [129, 500, 64]
    want, new_lens = select(s, marks, 128, 10)
    mass = marks.mass.clone()
    graph.replay()
    cache.check()
    assert torch.equal(source, want) and torch.equal(lens, new_lens)
    row = row_numbers(s, 1, 1, 500).cuda()
    assert torch.equal(marks.mass.view(-1)[row[:128]], mass.view(-1)[row[source[1, 1].long()]])


def test_without_sequences():
    s = R.Setup([10], 2, 64, 16, 16, seed=14)
    cache, marks = marked(s, 15)
    batch = B.KVBatch(s.table[:0], s.kv_lens[:0])
    source, lens = B.kv_select(cache, batch, marks, 5)
    B.kv_compact(cache, batch, source, marks)
    assert source.shape == (0, 2, 5) and lens.shape == (0,)


@pytest.mark.parametrize("bits", [16, 8])
def test_caches_beyond_32_bit_offsets(bits):
    """Keys (and values) of more than 4 GB, the sequences in the last pages: appended, weighed, chosen and moved there."""
    page, kv_heads, head_dim = 64, 8, 128
    n_pages = 2 ** 32 // (kv_heads * page * head_dim * bits // 8) + 40
    dtype = torch.bfloat16 if bits == 16 else torch.int8
    pools = [torch.zeros(n_pages, kv_heads, page, head_dim, dtype=dtype, device="cuda") for _ in range(2)]
    scales = [None if bits == 16 else torch.zeros(n_pages, kv_heads, page, device="cuda") for _ in range(2)]
    cache = B.KVCache.from_tensors(*pools, head_dim, *scales)
    marks = B.KVMarks(cache)
    lens, keep = [300, 129], 128
    s = R.Setup.__new__(R.Setup)
    s.lens, s.kv_heads, s.head_dim, s.page_size, s.bits, s.pools, s.scales = lens, kv_heads, head_dim, page, bits, pools, scales
    s.table = torch.arange(n_pages - 10, n_pages, dtype=torch.int32, device="cuda").flip(0).view(2, 5).contiguous()
    kv_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(16)
    k, v = (torch.randn(sum(lens), kv_heads, head_dim, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    cu = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
    B.kv_append_rmsnorm(cache, B.KVBatch(s.table, kv_lens, cu), k, v, marks=marks)
    want = [torch.cat([s.rows(which, b, n).transpose(0, 1) for b, n in enumerate(lens)]) for which in (0, 1)]
    for got, x in zip(want, (k, v)):
        size = x.double().abs().amax(-1, keepdim=True)
        assert torch.all((got - x.double()).abs() <= (0.0 if bits == 16 else (0.5 / 127 + 2.0 ** -20) * size))
    batch = B.KVBatch(s.table, kv_lens)
    q = torch.randn(2, 16, head_dim, generator=g).to(torch.bfloat16).cuda()
    B.attend_decode_weigh(cache, batch, marks, q, workspace=B.alloc_attend_weigh_workspace(16, kv_heads, head_dim, bits, 2, sum(lens)))
    assert abs(marks.mass.sum(dtype=torch.float64).item() - 32) < 1e-4
    source, _ = B.kv_select(cache, batch, marks, keep, 20)
    assert torch.equal(source, select(s, marks, keep, 20)[0])
    B.kv_compact(cache, batch, source, marks)
    cache.check()
    for b, n in enumerate(lens):
        at = sum(lens[:b])
        for which in (0, 1):
            now = s.rows(which, b, keep)
            for h in range(kv_heads):
                assert torch.equal(now[h], want[which][at + source[b, h].long(), h])


def test_small_launches_behind_each_other_with_nothing_to_weigh():
    """All slots empty: the attention's zeros are there when the next launch of the stream reads them."""
    s = R.Setup([40] * 300, 4, 64, 16, 16, seed=17)
    cache, marks = marked(s, 18)
    s.kv_lens.zero_()
    batch, q = B.KVBatch(s.table, s.kv_lens), torch.ones(300, 32, 64, dtype=torch.bfloat16, device="cuda")
    ws, mass = B.alloc_attend_weigh_workspace(32, 4, 64, 16, 300, 0), marks.mass.clone()
    out, seen = torch.empty_like(q), torch.empty_like(q)
    cu, empty = torch.arange(301, dtype=torch.int32, device="cuda"), torch.empty(300, 4, 64, dtype=torch.bfloat16, device="cuda")
    later = B.KVBatch(s.table, torch.ones(300, dtype=torch.int32, device="cuda"), cu)
    other = R.Setup([40] * 300, 4, 64, 16, 16, seed=17).cache()
    for _ in range(20):
        out.fill_(3.0)
        B.attend_decode_weigh(cache, batch, marks, q, out=out, workspace=ws)
        B.kv_append(other, later, empty, empty, q=out, q_out=seen)  # (a dependent launch that copies what it finds)
        assert torch.all(seen == 0)
    assert torch.equal(marks.mass, mass)
    cache.check()


@pytest.mark.parametrize("kv_heads,page,seqs,longest,keep,extra", [
    (8, 16, 30, 400, 100, 0), (2, 16, 128, 300, 64, 0), (2, 16, 129, 300, 64, 0), (8, 64, 10, 2000, 500, 700), (5, 32, 32, 64, 1, 0),
    (2, 16, 4, 900, 100, 850), (2, 16, 4, 900, 100, 1200), (1, 16, 4, 20000, 3000, 0), (3, 64, 4, 14000, 7001, 0), (8, 16, 19, 700, 90, 3000),
])
def test_select_from_sequences_of_many_lengths(kv_heads, page, seqs, longest, keep, extra):
    """A few waves of CTAs take the longest sequences first, and the page table's size decides how many share one; what they find does
    not depend on it.  Some are equally long, one is empty, one of the length that stays."""
    g = torch.Generator().manual_seed(seqs)
    lens = torch.randint(1, longest + 1, (seqs,), generator=g).tolist()
    lens[1], lens[2], lens[-1], lens[seqs // 2] = 0, keep, longest, longest
    s = R.Setup(lens, kv_heads, 16, page, 16, seed=seqs, table_extra=extra)
    cache, marks = marked(s, 21)
    want, new_lens = select(s, marks, keep, keep // 3)
    source, got = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, keep, keep // 3)
    cache.check()
    assert torch.equal(source, want) and torch.equal(got, new_lens)
