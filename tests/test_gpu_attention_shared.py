"""Attention of single tokens for sequences that begin with the same rows, against a 64-bit restatement."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import QUERY_FIXED, WEIGHT_BF16, check, rows

pytestmark = pytest.mark.gpu


def error_of(bits):
    """Weights rounded to bf16 in the shared part; over an 8-bit cache the queries to fixed point in the rest."""
    return dict(weight_rounding=WEIGHT_BF16, query_rounding=QUERY_FIXED if bits == 8 else 0.0)


def shared(groups, kv_heads, head_dim, page, bits, seed, alone=()):
    """(setup, groups' batch) of groups (rows shared, lengths); `alone`: lengths of sequences in front of them that share nothing."""
    lens = list(alone) + [n for _, own in groups for n in own]
    s = R.Setup(lens, kv_heads, head_dim, page, bits, seed=seed)
    bounds, spans = [len(alone)], []
    table = torch.full((len(groups), max(s.table.shape[1], max(span // page for span, _ in groups))), -3, dtype=torch.int32, device="cuda")
    for g, (span, own) in enumerate(groups):
        first = bounds[-1]
        longest = first + max(range(len(own)), key=lambda i: own[i])
        assert lens[longest] >= span
        w = span // page
        s.table[first:first + len(own), :w] = s.table[longest, :w].clone()
        table[g, :w] = s.table[longest, :w]
        bounds.append(first + len(own))
        spans.append(span)
    cu = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    return s, B.KVBatch(table, torch.tensor(spans, dtype=torch.int32, device="cuda"), cu)


CASES = [
    # heads, kv_heads, head_dim, page, groups, alone
    (1, 1, 4, 16, [(32, [33, 40])], []),
    (32, 32, 100, 16, [(1000, [1001, 1040, 1000, 1060])], []),
    (64, 8, 128, 64, [(640, [700, 641, 0, 300] * 8)], [5, 0]),
    (28, 4, 128, 32, [(333, [400, 350, 380]), (0, [5, 6]), (64, [70]), (1500, [1600] * 41 + [1499])], [900]),
    (8, 8, 64, 256, [(512, [513] * 130)], []),
    (71, 1, 64, 64, [(4096, [4100, 5000])], []),
    (12, 2, 80, 128, [(3000, [3001] * 5), (129, [200] * 3)], []),
    (16, 16, 64, 16, [(48, [50, 49])] * 20, [1]),
    (6, 2, 20, 32, [(100, [100, 101, 102]), (5, [9, 9])], [3]),
    (5, 1, 112, 16, [(10000, [10000, 10001, 16, 0])], []),
    (64, 8, 128, 64, [(8192, [8193 + 7 * i for i in range(20)])], []),
    (4, 4, 128, 16, [(160, [170, 160, 161, 159] * 30), (64, [64] * 3)], [2]),
    (32, 2, 64, 32, [(96, [97, 200, 96]), (320, [330, 319])], []),
    (6, 6, 100, 16, [(640, [700] * 16 + [641])], []),
    (20, 4, 128, 64, [(1280, [1300, 1290, 1281, 1280, 2000, 1, 0])] * 2, []),
]


@pytest.mark.parametrize("heads,kv_heads,head_dim,page,groups,alone", CASES)
@pytest.mark.parametrize("bits", [16, 8])
def test_shared_against_64_bits(heads, kv_heads, head_dim, page, groups, alone, bits):
    s, of = shared(groups, kv_heads, head_dim, page, bits, heads, alone)
    n = len(s.lens)
    q, out = rows(n, heads, head_dim, 1, extra=16), rows(n, heads, head_dim, 2, extra=8)
    guard = out.as_strided((n, out.stride(0)), (out.stride(0), 1))
    edge = guard[:, heads * head_dim:].clone()
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    ws = B.alloc_attend_shared_workspace(heads, kv_heads, head_dim, n)
    B.attend_decode_shared(cache, batch, of, q, out=out, workspace=ws, share_from=0)
    cache.check()
    want, bound = R.attend(s, q, [1] * n, **error_of(bits))
    check(out, want, bound)
    assert torch.equal(guard[:, heads * head_dim:], edge)
    first = out.clone()
    out.fill_(0.5)
    B.attend_decode_shared(cache, batch, of, q, out=out, workspace=ws, share_from=0)  # on the workspace as the first call left it
    assert torch.equal(out, first)
    assert torch.equal(B.attend_decode_shared(cache, batch, of, q, share_from=0), first)


def test_without_groups_it_is_the_plain_attention():
    s, of = shared([(64, [100, 90])], 2, 64, 16, 16, 3, alone=[50])
    q = rows(3, 8, 64, 4)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    want = B.attend_decode(cache, batch, q)
    none = B.KVBatch(of.page_table[:0], of.kv_lens[:0], of.cu_tokens[:1])
    assert torch.equal(B.attend_decode_shared(cache, batch, none, q, share_from=0), want)
    of.kv_lens.zero_()
    assert torch.equal(B.attend_decode_shared(cache, batch, of, q, share_from=0), want)
    of.kv_lens.fill_(15)  # less than a page
    assert torch.equal(B.attend_decode_shared(cache, batch, of, q, share_from=0), want)
    of.kv_lens.fill_(64)
    of.cu_tokens.copy_(torch.tensor([1, 2], dtype=torch.int32))  # a group of one
    assert torch.equal(B.attend_decode_shared(cache, batch, of, q, share_from=0), want)
    cache.check()


@pytest.mark.parametrize("bounds", [[0, 3, 2, 4], [-1, 2, 3, 4], [0, 2, 3, 5], [0, 2 ** 31 - 1, -2 ** 31, 4], [4, 3, 2, 1]])
def test_bounds_that_make_no_sense(bounds):
    s, of = shared([(32, [60, 50]), (0, [20]), (0, [33])], 2, 64, 16, 16, 5)
    of.kv_lens.fill_(32)
    of.cu_tokens.copy_(torch.tensor(bounds, dtype=torch.int64).to(torch.int32))
    q = rows(4, 8, 64, 6)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    want = B.attend_decode(cache, batch, q)
    got = B.attend_decode_shared(cache, batch, of, q, share_from=0)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE and torch.equal(got, want)


@pytest.mark.parametrize("bits", [16, 8])
def test_bad_pages_and_lengths(bits):
    """A shared page that does not exist takes no part for any sequence of the group, and the status is set; a shared length beyond the
    groups' page table is cut to it."""
    s, of = shared([(160, [200, 180, 170])], 2, 64, 16, bits, 7)
    q = rows(3, 8, 64, 8)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    of.page_table[0, 2] = s.n_pages
    got = B.attend_decode_shared(cache, batch, of, q, share_from=0)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    without = R.Setup([1], 2, 64, 16, bits)
    without.__dict__.update(s.__dict__)
    without.table = torch.cat([s.table[:, :2], s.table[:, 3:]], 1)
    without.lens = [n - 16 for n in s.lens]
    want, bound = R.attend(without, q, [1] * 3, **error_of(bits))
    check(got, want, bound)
    of.page_table[0, 2] = s.table[0, 2]
    cut = B.KVBatch(of.page_table[:, :4].contiguous(), torch.tensor([1000], dtype=torch.int32, device="cuda"), of.cu_tokens)
    got = B.attend_decode_shared(cache, batch, cut, q, share_from=0)
    with pytest.raises(B.BitLinearError):
        cache.check()
    want, bound = R.attend(s, q, [1] * 3, **error_of(bits))
    check(got, want, bound)


def test_values_that_are_not_finite_reach_those_that_see_them():
    """A NaN and an infinity in shared rows that one of the sequences is too short to see."""
    s, of = shared([(256, [300, 290, 100, 256])], 1, 64, 16, 16, 9)
    v = s.pools[1].view(-1, 64)
    i = torch.tensor([130, 200], device="cuda")
    row = s.table[0].long()[i // 16] * 16 + i % 16
    v[row[0], 7], v[row[1], 9] = float("nan"), float("inf")
    q = rows(4, 4, 64, 10, size=0.3)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    got = B.attend_decode_shared(cache, batch, of, q, share_from=0)
    cache.check()
    see = torch.tensor([0, 1, 3], device="cuda")
    assert torch.all(torch.isnan(got[see][..., 7])) and torch.all(got[see][..., 9] == float("inf"))
    clean = torch.ones(64, dtype=torch.bool, device="cuda")
    clean[[7, 9]] = False
    v[row[0], 7], v[row[1], 9] = 0.0, 0.0
    want, bound = R.attend(s, q, [1] * 4, **error_of(16))
    check(got[..., clean], want[..., clean], bound[..., clean])
    check(got[2], want[2], bound[2])


@pytest.mark.parametrize("bits", [16, 8])
def test_scores_of_any_size(bits):
    """Shared scores far above or below the others, and beyond 2^24."""
    for size in (30.0, 1e4, 1e8):
        s, of = shared([(320, [400, 390, 330])], 2, 64, 16, bits, 11)
        if bits == 8:
            for z in s.scales:
                z *= 4.0
        q = rows(3, 4, 64, 12, size=size)
        cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
        got = B.attend_decode_shared(cache, batch, of, q, share_from=0)
        cache.check()
        want, bound = R.attend(s, q, [1] * 3, **error_of(bits))
        check(got, want, bound)


def test_on_a_side_stream_and_in_a_graph():
    s, of = shared([(256, [300, 290, 280]), (64, [100, 90])], 2, 128, 16, 16, 13)
    q = rows(5, 8, 128, 14)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    ws = B.alloc_attend_shared_workspace(8, 2, 128, 5)
    want = B.attend_decode_shared(cache, batch, of, q, workspace=ws, share_from=0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = B.attend_decode_shared(cache, batch, of, q, stream=side, share_from=0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.graph(graph):
        B.attend_decode_shared(cache, batch, of, q, out=out, workspace=ws, share_from=0)
    s.kv_lens.copy_(torch.tensor([257, 0, 256, 91, 66], dtype=torch.int32))
    s.lens = [257, 0, 256, 91, 66]
    of.kv_lens.copy_(torch.tensor([128, 48], dtype=torch.int32))
    for _ in range(3):
        graph.replay()
    cache.check()
    want, bound = R.attend(s, q, [1] * 5, **error_of(16))
    check(out, want, bound)


@pytest.mark.parametrize("bits", [16, 8])
def test_an_expired_wait_is_reported(bits):
    s, of = shared([(256, [300, 290] * 20)], 1, 64, 16, bits, 15)
    q = rows(40, 8, 64, 16)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    ws = B.alloc_attend_shared_workspace(8, 1, 64, 40)
    want = B.attend_decode_shared(cache, batch, of, q, workspace=ws, share_from=0)
    cache.check()
    B.test_expire_next_wait(2000, True)
    B.attend_decode_shared(cache, batch, of, q, workspace=ws, share_from=0)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_TIMEOUT
    assert torch.equal(B.attend_decode_shared(cache, batch, of, q, workspace=ws, share_from=0), want)
    cache.check()


def test_a_workspace_serves_calls_of_different_sizes():
    """Calls of more and fewer sequences, share one workspace."""
    ws = B.alloc_attend_shared_workspace(16, 2, 64, 60)
    cases = []
    for n, groups in ((60, [(64, [70 + i for i in range(60)])]), (3, [(64, [100, 64, 90])]), (20, [(48, [50, 49, 60, 70])] * 5)):
        s, of = shared(groups, 2, 64, 16, 16, 30 + n)
        q = rows(n, 16, 64, n)
        cases.append((s, of, q, *R.attend(s, q, [1] * n, **error_of(16))))
    for _ in range(3):
        for s, of, q, want, bound in cases:
            cache = s.cache()
            check(B.attend_decode_shared(cache, B.KVBatch(s.table, s.kv_lens), of, q, workspace=ws, share_from=0), want, bound)
            cache.check()


def test_sharing_that_is_not_worth_its_cost():
    """Below the bound the call is the plain attention, whether the page table alone says so or the lengths; above it rows are shared."""
    s, of = shared([(256, [300, 290, 280]), (64, [100, 90])], 2, 128, 16, 16, 40)
    q = rows(5, 8, 128, 41)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    plain, split = B.attend_decode(cache, batch, q), B.attend_decode_shared(cache, batch, of, q, share_from=0)
    assert not torch.equal(plain, split)
    elements = (3 * 256 + 2 * 64) * 2 * 128
    room = 5 * of.page_table.shape[1] * 16 * 2 * 128
    assert elements + 1 < room
    for share_from, want in ((-1, plain), (room + 1, plain), (elements + 1, plain), (elements, split), (1, split)):
        assert torch.equal(B.attend_decode_shared(cache, batch, of, q, share_from=share_from), want), share_from
    cache.check()


def test_the_measured_bound():
    """130 sequences of 320 shared rows at 8 heads of 128: 42.6 M elements, above the bound."""
    s, of = shared([(320, [321 + i % 5 for i in range(130)])], 8, 128, 64, 16, 42)
    q = rows(130, 16, 128, 43)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    got = B.attend_decode_shared(cache, batch, of, q)
    assert torch.equal(got, B.attend_decode_shared(cache, batch, of, q, share_from=0)) and not torch.equal(got, B.attend_decode(cache, batch, q))
    want, bound = R.attend(s, q, [1] * 130, **error_of(16))
    check(got, want, bound)
    cache.check()
