"""Attention of single tokens that adds every row's weight to its mark, against a 64-bit restatement."""
import math

import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import DECODE, QUERY_FIXED, check, decode_error, rows

pytestmark = pytest.mark.gpu


def weights(setup, q, scale=None):
    """[(row numbers [kv_heads, n], sum of the weights [kv_heads, n], how far it may be off)] of every sequence.

    A weight is off by the relative error that kv_reference.attend derives for the weights and the denominator together, 2 (d + (n + 64)
    2^-24), without a rounding to fewer bits; the sum over the group's G weights adds G 2^-24; weights below 2^-126 of the
    largest count as zero."""
    H, D = q.shape[1:]
    G, got = H // setup.kv_heads, []
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    for b, n in enumerate(setup.lens):
        if n == 0:
            continue
        x, k = q[b].double().view(setup.kv_heads, G, D), setup.rows(0, b, n)
        p = torch.softmax(scale * torch.einsum("hgd,hld->hgl", x, k), -1)
        worst = scale * torch.einsum("hgd,hld->hgl", x.abs(), k.abs()).amax(-1, keepdim=True) * (D + 4) * 2.0 ** -24
        if setup.bits == 8:
            worst = worst + QUERY_FIXED * scale * (x.abs().amax(-1)[..., None] * k.abs().sum(-1)[:, None]).amax(-1, keepdim=True)
        off = 2 * (2 * worst + 2.0 ** -21 + (n + 64) * 2.0 ** -24)
        i = torch.arange(n, device="cuda")
        number = setup.table[b].long()[i // setup.page_size] * setup.kv_heads * setup.page_size + i % setup.page_size
        number = number + torch.arange(setup.kv_heads, device="cuda")[:, None] * setup.page_size
        got.append((number, p.sum(1), 1.01 * (off * p).sum(1) + G * 2.0 ** -24 * p.sum(1) + G * 2.0 ** -125))
    return got


def check_mass(mass, before, expected, times=1):
    """Every addition to a mark rounds once more."""
    want, bound = before.double().flatten().clone(), torch.zeros(before.numel(), dtype=torch.float64, device="cuda")
    for number, p, off in expected:
        want.index_add_(0, number.flatten(), times * p.flatten())
        bound.index_add_(0, number.flatten(), times * off.flatten())
    bound += times * 2.0 ** -24 * want.abs() * (bound > 0)
    d = (mass.double().flatten() - want).abs()
    assert torch.all(d <= bound), f"off by {(d / bound.clamp(min=1e-300)).max().item():.2f} of the bound"


def marks_of(cache, seed):
    marks = B.KVMarks(cache)
    marks.mass.copy_(torch.rand(marks.mass.shape, generator=torch.Generator().manual_seed(seed)))
    marks.pos.fill_(-5)
    return marks


@pytest.mark.parametrize("heads,kv_heads,head_dim,page,lens", DECODE)
@pytest.mark.parametrize("bits", [16, 8])
def test_weights_against_64_bits(heads, kv_heads, head_dim, page, lens, bits):
    s = R.Setup(lens, kv_heads, head_dim, page, bits, seed=heads)
    q = rows(len(lens), heads, head_dim, 1, extra=16)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    marks = marks_of(cache, 2)
    before = marks.mass.clone()
    ws = B.alloc_attend_weigh_workspace(heads, kv_heads, head_dim, bits, len(lens), sum(lens))
    # (the scores' part need not be clear)
    ws[B.attend_weigh_workspace_bytes(heads, kv_heads, head_dim, bits, len(lens), 0) // 2:].fill_(255)
    out = B.attend_decode_weigh(cache, batch, marks, q, workspace=ws)
    cache.check()
    want, bound = R.attend(s, q, [1] * len(lens), **decode_error(bits))
    check(out, want, bound)
    expected = weights(s, q)
    check_mass(marks.mass, before, expected)
    assert torch.equal(out, B.attend_decode(cache, batch, q)), "the attention itself is attend_decode's"
    # again on the same workspace: the same bits are added
    once = marks.mass.clone()
    marks.mass.copy_(before)
    assert torch.equal(B.attend_decode_weigh(cache, batch, marks, q, workspace=ws), out)
    assert torch.equal(marks.mass, once)
    B.attend_decode_weigh(cache, batch, marks, q, workspace=ws)
    check_mass(marks.mass, before, expected, times=2)
    assert torch.all(marks.pos == -5)


@pytest.mark.parametrize("bits", [16, 8])
def test_long_and_many_sequences(bits):
    lens = [70001, 3, 1, 500, 0, 33000]
    s = R.Setup(lens, 2, 128, 64, bits, seed=3)
    q = rows(len(lens), 16, 128, 4)
    cache = s.cache()
    marks = marks_of(cache, 5)
    before = marks.mass.clone()
    ws = B.alloc_attend_weigh_workspace(16, 2, 128, bits, len(lens), sum(lens))
    B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=ws)
    check_mass(marks.mass, before, weights(s, q))
    lens = torch.randint(0, 90, (1500,), generator=torch.Generator().manual_seed(6)).tolist()  # more than a CTA has threads
    s = R.Setup(lens, 1, 16, 16, bits, seed=7)
    q = rows(len(lens), 2, 16, 8)
    cache = s.cache()
    marks = marks_of(cache, 9)
    before = marks.mass.clone()
    ws = B.alloc_attend_weigh_workspace(2, 1, 16, bits, len(lens), sum(lens))
    B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=ws)
    cache.check()
    check_mass(marks.mass, before, weights(s, q))


@pytest.mark.parametrize("bits", [16, 8])
def test_bad_pages_missing_room_and_long_lengths(bits):
    s = R.Setup([200, 40, 100], 2, 64, 16, bits, seed=10)
    q = rows(3, 8, 64, 11)
    cache = s.cache()
    ws = B.alloc_attend_weigh_workspace(8, 2, 64, bits, 3, 340)
    # a page that does not exist: its rows get nothing, the others the weights of a sequence without it
    page = s.table[0, 3].item()
    s.table[0, 3] = s.n_pages
    marks = marks_of(cache, 12)
    before = marks.mass.clone()
    B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=ws)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    gone = marks.mass - before
    assert torch.all(gone[page] == 0)
    for b in range(3):
        got = sum(gone[p, :, :].sum(-1).double() for p in s.table[b, :-(-s.lens[b] // 16)].tolist() if p != s.n_pages)
        assert torch.all((got - 4).abs() < 1e-4), "four query heads give a weight of one each"
    s.table[0, 3] = page
    # a workspace with less room: right results, and the status says that weights are missing
    small = B.alloc_attend_weigh_workspace(8, 2, 64, bits, 3, 0)
    marks.mass.copy_(before)
    long = R.Setup([3000, 40, 100], 2, 64, 16, bits, seed=10)
    cache = long.cache()
    marks = marks_of(cache, 12)
    before = marks.mass.clone()
    out = B.attend_decode_weigh(cache, B.KVBatch(long.table, long.kv_lens), marks, q, workspace=small)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    want, bound = R.attend(long, q, [1] * 3, **decode_error(bits))
    check(out, want, bound)
    given = marks.mass - before
    number, p, off = weights(long, q)[0]
    d = (given.flatten()[number].double() - p).abs()
    assert torch.all((d <= off + 2.0 ** -23) | (given.flatten()[number] == 0)), "whole weights, or none"
    # a length beyond the page table is cut to it
    cut = R.Setup([64, 20], 1, 64, 16, bits, seed=13, table_extra=0)
    cache = cut.cache()
    marks = marks_of(cache, 14)
    before = marks.mass.clone()
    cut.kv_lens[0] = 1000
    B.attend_decode_weigh(cache, B.KVBatch(cut.table, cut.kv_lens), marks, q[:2, :4], workspace=B.alloc_attend_weigh_workspace(4, 1, 64, bits, 2, 84))
    with pytest.raises(B.BitLinearError):
        cache.check()
    check_mass(marks.mass, before, weights(cut, q[:2, :4]))


def test_rows_that_two_sequences_share_get_both_weights():
    s = R.Setup([80, 80], 2, 64, 16, 16, seed=15)
    s.table[1] = s.table[0]
    q = rows(2, 4, 64, 16)
    cache = s.cache()
    marks = marks_of(cache, 17)
    before = marks.mass.clone()
    B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=B.alloc_attend_weigh_workspace(4, 2, 64, 16, 2, 160))
    cache.check()
    check_mass(marks.mass, before, weights(s, q))


def test_scores_that_are_not_finite():
    """All scores -infinity: zeros and no weight; one NaN: that head's result is NaN, and so is what its kv head's rows get."""
    s = R.Setup([40, 40, 40], 1, 64, 16, 16, seed=18)
    q = rows(3, 1, 64, 19)
    key = s.pools[0].view(-1, 64)
    first = s.table[:, 0].long() * 16
    for p in range(3):
        at = s.table[0, p].long() * 16
        key[at:at + 16] = 1.0
        key[at:at + 16, 0] = float("inf")
    q[0] = 1.0
    q[0, 0, 0] = -1.0
    key[first[1] + 3, 5] = float("nan")
    cache = s.cache()
    marks = marks_of(cache, 20)
    before = marks.mass.clone()
    out = B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=B.alloc_attend_weigh_workspace(1, 1, 64, 16, 3, 120))
    mass = marks.mass.view(-1)
    i = torch.arange(40, device="cuda")
    row = lambda b: s.table[b].long()[i // 16] * 16 + i % 16  # noqa: E731
    assert torch.all(out[0] == 0) and torch.equal(mass[row(0)], before.view(-1)[row(0)])
    assert torch.all(torch.isnan(out[1])) and torch.all(torch.isnan(mass[row(1)]))
    assert torch.all(torch.isfinite(out[2])) and abs((mass - before.view(-1))[row(2)].sum().item() - 1) < 1e-4


def test_on_a_side_stream_and_in_a_graph():
    s = R.Setup([300, 64], 2, 128, 64, 8, seed=21)
    q = rows(2, 8, 128, 22)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    marks = marks_of(cache, 23)
    before = marks.mass.clone()
    ws = B.alloc_attend_weigh_workspace(8, 2, 128, 8, 2, 364)
    out = B.attend_decode_weigh(cache, batch, marks, q, workspace=ws)
    once = marks.mass.clone()
    side = torch.cuda.Stream()
    marks.mass.copy_(before)
    torch.cuda.synchronize()
    got = B.attend_decode_weigh(cache, batch, marks, q, workspace=ws, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, out) and torch.equal(marks.mass, once)
    graph = torch.cuda.CUDAGraph()
    held = torch.empty_like(out)
    with torch.cuda.graph(graph):
        B.attend_decode_weigh(cache, batch, marks, q, out=held, workspace=ws)
    s.kv_lens.copy_(torch.tensor([130, 0], dtype=torch.int32))
    s.lens = [130, 0]
    marks.mass.copy_(before)
    graph.replay()
    cache.check()
    want, bound = R.attend(s, q, [1, 1], **decode_error(8))
    check(held, want, bound)
    check_mass(marks.mass, before, weights(s, q))


@pytest.mark.parametrize("bits", [16, 8])
def test_the_last_tokens_of_a_prompt_as_sequences_of_their_own(bits):
    """A window of 16 tokens at the end of one sequence of 300: every row gets what those of the tokens that see it give."""
    n, window = 300, 16
    one = R.Setup([n], 2, 128, 32, bits, seed=24)
    q = rows(window, 8, 128, 25)
    cache = one.cache()
    marks = marks_of(cache, 26)
    before = marks.mass.clone()
    s = R.Setup.__new__(R.Setup)
    s.__dict__.update(one.__dict__)
    s.lens = list(range(n - window + 1, n + 1))
    s.table, s.kv_lens = one.table.expand(window, -1).contiguous(), torch.tensor(s.lens, dtype=torch.int32, device="cuda")
    out = B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=B.alloc_attend_weigh_workspace(8, 2, 128, bits, window, sum(s.lens)))
    cache.check()
    cu = torch.tensor([0, window], dtype=torch.int32, device="cuda")
    want, bound = R.attend(one, q, [window], **decode_error(bits))
    check(out, want, bound)
    check(B.attend_prompt(cache, B.KVBatch(one.table, one.kv_lens, cu), q), *R.attend(one, q, [window], weight_rounding=2.0 ** -8))
    expected = weights(s, q)
    want, bound = before.double().flatten(), torch.zeros(before.numel(), dtype=torch.float64, device="cuda")
    for number, p, off in expected:
        want.index_add_(0, number.flatten(), p.flatten())
        bound.index_add_(0, number.flatten(), off.flatten())
    bound += window * 2.0 ** -24 * want.abs() * (bound > 0)  # (one rounding for each addition)
    assert torch.all((marks.mass.double().flatten() - want).abs() <= bound)


def test_a_page_table_cut_to_its_first_columns():
    """The rows of the table keep their distance; selection takes the narrow one, whatever the wide one could hold."""
    s = R.Setup([200, 150], 1, 64, 16, 16, seed=27, table_extra=20000)
    cache = s.cache()
    marks = marks_of(cache, 28)
    with pytest.raises(B.BitLinearError) as e:
        B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 64)
    assert e.value.status == B.ERR_SHAPE
    narrow = B.KVBatch(s.table[:, :13], s.kv_lens)
    source, lens = B.kv_select(cache, narrow, marks, 64)
    B.kv_compact(cache, narrow, source, marks)
    cache.check()
    assert lens.tolist() == [64, 64] and torch.all(source.sort(-1).values.diff() > 0)
