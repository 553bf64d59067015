"""Appending to the paged key-value cache: stored rows, rotated queries and 8-bit codes against a 64-bit restatement."""
import math

import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B

pytestmark = pytest.mark.gpu

HEADS = [(32, 32, 100), (64, 8, 128), (3, 1, 64), (4, 2, 4), (6, 3, 20), (5, 5, 48), (2, 1, 80), (7, 7, 124)]


def tokens(counts, past, heads, kv_heads, head_dim, seed, extra_rows=0, stride_extra=8):
    """Slices of one fused projection output [T + extra_rows, ...] whose rows start on 16-byte boundaries."""
    g = torch.Generator().manual_seed(seed)
    T = sum(counts) + extra_rows
    widths = [(n * head_dim + 7) // 8 * 8 for n in (heads, kv_heads, kv_heads)]
    x = torch.randn(T, sum(widths) + stride_extra, generator=g).to(torch.bfloat16).cuda()
    parts, at = [], 0
    for n, w in zip((heads, kv_heads, kv_heads), widths):
        parts.append(x[:, at:at + n * head_dim].unflatten(1, (n, head_dim)))
        at += w
    return parts


def place(table, counts, lens, page_size):
    """(sequence, position) of every stored token and the rows it comes from."""
    rows, seqs, pos = [], [], []
    at = 0
    for b, n in enumerate(counts):
        for i in range(n):
            p = lens[b] - n + i
            if p >= 0:
                rows.append(at + i), seqs.append(b), pos.append(p)
        at += n
    return torch.tensor(rows, device="cuda"), torch.tensor(seqs, device="cuda"), torch.tensor(pos, device="cuda")


@pytest.mark.parametrize("heads,kv_heads,head_dim", HEADS)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_against_64_bits(heads, kv_heads, head_dim, bits, interleaved):
    page_size = {100: 16, 128: 64, 64: 32, 4: 16, 20: 256, 48: 128, 80: 16, 124: 32}[head_dim]
    counts, past = [1, 0, 37, 16, 5, 3], [0, 9, 250, 15, 16, 0]
    lens = [n + p for n, p in zip(counts, past)]
    lens[5] = 1  # three rows, length one: two of them lie in front of the sequence and are not stored
    s = R.Setup(lens, kv_heads, head_dim, page_size, bits, seed=head_dim + bits)
    q, k, v = tokens(counts, past, heads, kv_heads, head_dim, seed=1, extra_rows=2)
    rope = R.angles(max(lens), head_dim)
    cu = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)
    before = [(p.clone(), None if z is None else z.clone()) for p, z in zip(s.pools, s.scales)]
    q_out = torch.full((q.shape[0], heads * head_dim + 24 + (-heads * head_dim) % 8), 7.0, dtype=torch.bfloat16, device="cuda")
    view = q_out[:, :heads * head_dim].unflatten(1, (heads, head_dim))
    source = [x.clone() for x in (q, k, v)]
    B.kv_append(cache, batch, k, v, q=q, rope=rope, interleaved=interleaved, q_out=view)
    cache.check()
    for x, y in zip((q, k, v), source):
        assert torch.equal(x, y), "an input was modified"
    rows, seqs, pos = place(s.table, counts, lens, page_size)
    page, slot = s.table[seqs, pos // page_size].long(), pos % page_size

    # queries: two products and a sum in fp32 (3 roundings of at most |a c| + |b s|), then one rounding to bf16
    want, size = R.rotate(q[rows], rope, pos, interleaved)
    got = view[rows].double()
    assert torch.all((got - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * 3 * 2.0 ** -24 * size)
    kept = torch.ones(q_out.shape[0], dtype=torch.bool, device="cuda")
    kept[rows] = False
    assert torch.all(q_out[kept] == 7.0) and torch.all(q_out[:, heads * head_dim:] == 7.0), "rows or columns written that are not the call's"

    for which, x in ((0, k), (1, v)):
        z, size = R.rotate(x[rows], rope, pos, interleaved) if which == 0 else (x[rows].double(), None)
        stored = s.pools[which][page, :, slot]
        if bits == 16:
            if which == 0:
                assert torch.all((stored[..., :head_dim].double() - z).abs() <= 2.0 ** -8 * z.abs() + 1.01 * 3 * 2.0 ** -24 * size)
            else:
                assert torch.equal(stored[..., :head_dim], x[rows])
        else:
            c, scale = R.codes(z)
            assert torch.equal(stored[..., :head_dim], c)
            assert torch.equal(s.scales[which][page, :, slot], scale)
        assert torch.all(stored[..., head_dim:] == 0)
        # everything else as it was
        mask = torch.ones(s.n_pages, page_size, dtype=torch.bool, device="cuda")
        mask[page, slot] = False
        now, then = s.pools[which].transpose(1, 2)[mask], before[which][0].transpose(1, 2)[mask]
        view_as = torch.int16 if bits == 16 else torch.int8
        assert torch.equal(now.view(view_as), then.view(view_as))
        if bits == 8:
            assert torch.equal(s.scales[which].transpose(1, 2)[mask].view(torch.int32), before[which][1].transpose(1, 2)[mask].view(torch.int32))


@pytest.mark.parametrize("bits", [16, 8])
def test_append_one_token_per_sequence_in_place_and_without_rotation(bits):
    lens = [1, 0, 16, 17, 300]  # the second slot of the batch is empty
    s = R.Setup(lens, 2, 64, 16, bits, seed=5)
    q, k, v = tokens([1] * 5, None, 4, 2, 64, seed=2)
    rope = R.angles(300, 64)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    apart = torch.full((5, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    B.kv_append(cache, batch, k, v, q=q, rope=rope, q_out=apart)
    same = q.clone()
    same_before = same.clone()
    B.kv_append(cache, batch, k, v, q=same, rope=rope, q_out=same)
    cache.check()
    assert torch.all(apart[1] == 3.0) and torch.equal(same[1], same_before[1])
    live = [0, 2, 3, 4]
    assert torch.equal(apart[live], same[live])
    # without a table nothing is rotated, and q may be left out
    before = [p.clone() for p in s.pools]
    assert B.kv_append(cache, batch, k, v) is None
    cache.check()
    for b in live:
        page, slot = s.table[b, (lens[b] - 1) // 16].item(), (lens[b] - 1) % 16
        for which, x in ((0, k), (1, v)):
            got = s.pools[which][page, :, slot]
            if bits == 16:
                assert torch.equal(got, x[b])
            else:
                c, scale = R.codes(x[b].double())
                assert torch.equal(got, c) and torch.equal(s.scales[which][page, :, slot], scale)
            before[which][page, :, slot] = got
    for which in (0, 1):
        kind = torch.int16 if bits == 16 else torch.int8
        assert torch.equal(s.pools[which].view(kind), before[which].view(kind))
    plain = B.kv_append(cache, batch, k, v, q=q)
    assert torch.equal(plain[live], q[live])


@pytest.mark.parametrize("head_dim", [64, 100])
def test_codes_of_values_between_two_codes_and_of_rows_that_are_not_finite(head_dim):
    """bf16 quotients often lie exactly half way between two codes; zeros, subnormals, huge and non-finite rows."""
    T = 256
    g = torch.Generator().manual_seed(3)
    x = (torch.randint(-254, 255, (T, 1, head_dim), generator=g).float() / 2.0)
    x[:, 0, 0] = 127.0  # scale one: every second value is half way
    x[1] = 0.0
    x[2] = 1e-39
    x[3] *= 2.0 ** 120
    x[4] *= 2.0 ** -100
    x[5, 0, 7] = math.inf
    x[6, 0, 9] = math.nan
    x[7, 0, 1] = -math.inf
    x = x.to(torch.bfloat16).cuda()
    lens = [T]
    s = R.Setup(lens, 1, head_dim, 16, 8, seed=6)
    cache = s.cache()
    wide = torch.zeros(T, (head_dim + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")
    wide[:, :head_dim] = x[:, 0]
    view = wide[:, :head_dim].unflatten(1, (1, head_dim))
    batch = B.KVBatch(s.table, s.kv_lens, torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    B.kv_append(cache, batch, view, view)
    cache.check()
    for which in (0, 1):
        got = torch.cat([s.pools[which][p, 0] for p in s.table[0, :T // 16].tolist()])[:, :head_dim]
        scale = torch.cat([s.scales[which][p, 0] for p in s.table[0, :T // 16].tolist()])
        bad = torch.tensor([5, 6, 7], device="cuda")
        fine = torch.ones(T, dtype=torch.bool, device="cuda")
        fine[bad] = False
        c, z = R.codes(x[fine, 0].double())
        assert torch.equal(got[fine], c) and torch.equal(scale[fine], z)
        assert torch.all(got[bad] == 0) and torch.all(scale[bad].isnan())


def test_codes_of_rotated_rows_at_the_ends_of_the_range():
    """Rotated pairs whose length is beyond fp32's (and bf16's) largest value, subnormal ones, and the floor of beta."""
    T, D = 64, 64
    g = torch.Generator().manual_seed(4)
    x = torch.randn(T, 1, D, generator=g)
    x[0:8] = torch.sign(x[0:8]) * 3.3e38
    x[8:16] *= 2.0 ** 125
    x[16:24] *= 1e-39
    x[24:32] *= 1e-6
    x = x.to(torch.bfloat16).cuda()
    s = R.Setup([T], 1, D, 16, 8, seed=10)
    rope = R.angles(T, D)
    cache = s.cache()
    B.kv_append(cache, B.KVBatch(s.table, s.kv_lens, torch.tensor([0, T], dtype=torch.int32, device="cuda")), x, x, rope=rope)
    cache.check()
    got = torch.cat([s.pools[0][p, 0] for p in s.table[0, :T // 16].tolist()])
    scale = torch.cat([s.scales[0][p, 0] for p in s.table[0, :T // 16].tolist()])
    z, _ = R.rotate(x, rope, torch.arange(T, device="cuda"), False)
    c, want = R.codes(z)
    assert torch.equal(got, c[:, 0]) and torch.equal(scale, want[:, 0])


def test_rotary_table():
    for n, d, base in ((1, 4, 10000.0), (5000, 100, 10000.0), (70001, 128, 500000.0)):
        got = B.rope_table(n, d, base).double()
        a = torch.arange(n, dtype=torch.float64)[:, None] * base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
        want = torch.stack([a.cos(), a.sin()], -1).cuda()
        # the angle is off by a few 2^-53 of itself (pow and the product: 4 ulp), the result rounded to fp32
        assert torch.all((got - want).abs() <= 2.0 ** -24 * want.abs() + 8 * 2.0 ** -53 * n + 1e-12 + 2.0 ** -149)


def test_bad_pages_lengths_and_positions_are_reported_and_nothing_is_written():
    lens = [20, 40, 33]
    for what in ("page", "negative page", "length", "rope"):
        s = R.Setup(lens, 2, 64, 16, 16, seed=8, table_extra=0)
        q, k, v = tokens([2, 2, 2], None, 4, 2, 64, seed=4)
        rope = R.angles(40 if what != "rope" else 39, 64)
        cu = torch.tensor([0, 2, 4, 6], dtype=torch.int32, device="cuda")
        cache = s.cache()
        if what == "page":
            s.table[1, 2] = s.n_pages
        if what == "negative page":
            s.table[1, 2] = -1
        if what == "length":
            s.kv_lens[1] = 16 * s.table.shape[1] + 2  # both new tokens lie behind the table
        before = [p.clone() for p in s.pools]
        out = torch.zeros(6, 4, 64, dtype=torch.bfloat16, device="cuda")
        B.kv_append(cache, B.KVBatch(s.table, s.kv_lens, cu), k, v, q=q, rope=rope, q_out=out)
        with pytest.raises(B.BitLinearError) as e:
            cache.check()
        assert e.value.status == B.ERR_PAGE
        cache.check()  # cleared
        changed = (s.pools[1].view(torch.int16) != before[1].view(torch.int16)).any(-1).any(1).sum().item()
        assert changed == {"page": 4, "negative page": 4, "length": 4, "rope": 5}[what]
        assert torch.all(out[[0, 1, 4, 5]].abs().amax(-1) > 0)


def test_append_on_a_side_stream_and_in_a_captured_graph():
    lens = [5, 64, 100]
    s = R.Setup([n + 3 for n in lens], 2, 128, 32, 16, seed=9)
    q, k, v = tokens([1, 1, 1], None, 4, 2, 128, seed=5)
    rope = R.angles(128, 128)
    kv_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache, batch = s.cache(), B.KVBatch(s.table, kv_lens)
    out = torch.empty(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.kv_append(cache, batch, k, v, q=q, rope=rope, q_out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_append(cache, batch, k, v, q=q, rope=rope, q_out=out)
    for step in range(3):
        kv_lens.copy_(torch.tensor([n + step for n in lens], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(lens):
            pos = torch.tensor([n + step - 1], device="cuda")
            page, slot = s.table[b, pos // 32].long(), pos % 32
            want, _ = R.rotate(k[b:b + 1], rope, pos, False)
            assert torch.allclose(s.pools[0][page, :, slot].double(), want, rtol=2.0 ** -8, atol=1e-6)
            assert torch.equal(s.pools[1][page, :, slot], v[b:b + 1])
    cache.check()


def test_nothing_to_append():
    s = R.Setup([4], 2, 64, 16, 16)
    cache = s.cache()
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    B.kv_append(cache, B.KVBatch(s.table[:0], s.kv_lens[:0]), none, none)
    B.kv_append(cache, B.KVBatch(s.table, s.kv_lens, torch.zeros(2, dtype=torch.int32, device="cuda")), none, none)
    cache.check()
