"""Attention over the paged cache, of single tokens and of prompts, against a 64-bit restatement (kv_reference.py derives
the bounds)."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B

pytestmark = pytest.mark.gpu

WEIGHT_BF16 = 2.0 ** -8  # the prompt kernel rounds its weights to bf16
WEIGHT_TWO_BF16 = 2.0 ** -16  # the decode kernel splits them into two bf16 parts
# Over an int8 cache the decode kernel takes a query's elements to integers, the largest of which is 2^21 or more: each is off by at
# most half, 2^-22 of the largest.
QUERY_FIXED = 2.0 ** -22


def decode_error(bits):
    return dict(weight_rounding=WEIGHT_TWO_BF16, query_rounding=QUERY_FIXED if bits == 8 else 0.0)


def error_of(prompt, bits):
    return dict(weight_rounding=WEIGHT_BF16) if prompt else decode_error(bits)


def rows(T, heads, head_dim, seed, extra=0, size=1.5):
    """bf16 [T, heads, head_dim] inside wider rows."""
    g = torch.Generator().manual_seed(seed)
    n = heads * head_dim
    x = (size * torch.randn(T, (n + 7) // 8 * 8 + extra, generator=g)).to(torch.bfloat16).cuda()
    return x[:, :n].unflatten(1, (heads, head_dim))


def check(got, want, bound):
    d = (got.double() - want).abs()
    assert torch.all(d <= bound), f"off by {(d / bound).max().item():.2f} of the bound"


DECODE = [
    # heads, kv_heads, head_dim, page, lens
    (1, 1, 4, 16, [1, 16, 17]),
    (32, 32, 100, 16, [1, 0, 777, 15, 16, 17]),
    (64, 8, 128, 64, [2000, 1, 63, 64, 65, 0, 129]),
    (28, 4, 128, 32, [300, 31, 5000]),
    (8, 8, 64, 256, [255, 256, 257, 1025]),
    (12, 2, 80, 128, [700, 3]),
    (16, 1, 96, 16, [1, 40, 513]),
    (71, 1, 64, 64, [333, 64]),
    (24, 8, 20, 32, [90, 2049]),
    (9, 1, 128, 16, [48, 4097]),
    (34, 2, 112, 64, [100] * 40),
    (4, 2, 8, 16, list(range(0, 70))),
]


@pytest.mark.parametrize("heads,kv_heads,head_dim,page,lens", DECODE)
@pytest.mark.parametrize("bits", [16, 8])
def test_decode_against_64_bits(heads, kv_heads, head_dim, page, lens, bits):
    s = R.Setup(lens, kv_heads, head_dim, page, bits, seed=heads)
    q = rows(len(lens), heads, head_dim, 1, extra=16)
    out = rows(len(lens), heads, head_dim, 2, extra=8)
    guard = out.as_strided((len(lens), out.stride(0)), (out.stride(0), 1)) if len(lens) > 1 else None
    edge = guard[:, heads * head_dim:].clone() if guard is not None else None
    cache = s.cache()
    ws = B.alloc_attend_workspace(heads, kv_heads, head_dim, prompt=False)
    B.attend_decode(cache, B.KVBatch(s.table, s.kv_lens), q, out=out, workspace=ws)
    cache.check()
    want, bound = R.attend(s, q, [1] * len(lens), **decode_error(s.bits))
    check(out, want, bound)
    if guard is not None:
        assert torch.equal(guard[:, heads * head_dim:], edge)
    # the same call again, on the workspace as the first one left it: the same bits
    first = out.clone()
    out.fill_(0.5)
    B.attend_decode(cache, B.KVBatch(s.table, s.kv_lens), q, out=out, workspace=ws)
    assert torch.equal(out, first)


@pytest.mark.parametrize("bits", [16, 8])
def test_decode_of_a_long_and_a_short_context_together(bits):
    lens = [70001, 3, 1, 500, 0, 33000]
    s = R.Setup(lens, 2, 128, 64, bits, seed=3)
    q = rows(len(lens), 16, 128, 4)
    got = B.attend_decode(s.cache(), B.KVBatch(s.table, s.kv_lens), q)
    want, bound = R.attend(s, q, [1] * len(lens), **decode_error(s.bits))
    check(got, want, bound)


def test_decode_of_a_large_batch():
    """More sequences than the kernel has threads to look at their lengths at once."""
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 90, (1500,), generator=g).tolist()
    s = R.Setup(lens, 1, 16, 16, 16, seed=4)
    q = rows(len(lens), 2, 16, 5)
    got = B.attend_decode(s.cache(), B.KVBatch(s.table, s.kv_lens), q)
    want, bound = R.attend(s, q, [1] * len(lens), **decode_error(s.bits))
    check(got, want, bound)


PROMPT = [
    # heads, kv_heads, head_dim, page, new, past
    (1, 1, 4, 16, [1, 5, 0, 17], [0, 0, 4, 3]),
    (32, 32, 100, 16, [37], [411]),
    (8, 1, 128, 64, [129, 1, 64], [0, 1000, 63]),
    (28, 4, 128, 32, [40, 300], [100, 0]),
    (4, 4, 64, 256, [257, 256, 255, 1], [0, 1, 255, 256]),
    (12, 2, 80, 128, [130], [7]),
    (16, 1, 96, 16, [3, 61], [500, 2]),
    (71, 1, 64, 64, [9], [333]),
    (6, 2, 20, 32, [700], [0]),
    (5, 1, 112, 16, [90, 33, 2], [0, 15, 16]),
    (2, 2, 128, 64, [1500, 700], [0, 900]),
    (8, 8, 128, 16, list(range(0, 40)), list(range(40, 0, -1))),
]


@pytest.mark.parametrize("heads,kv_heads,head_dim,page,new,past", PROMPT)
@pytest.mark.parametrize("bits", [16, 8])
def test_prompt_against_64_bits(heads, kv_heads, head_dim, page, new, past, bits):
    lens = [n + p for n, p in zip(new, past)]
    T = sum(new)
    s = R.Setup(lens, kv_heads, head_dim, page, bits, seed=heads)
    q = rows(T + 3, heads, head_dim, 1, extra=16)
    out = rows(T + 3, heads, head_dim, 2, extra=8)
    guard = out.as_strided((T + 3, out.stride(0)), (out.stride(0), 1))
    edge, behind = guard[:, heads * head_dim:].clone(), out[T:].clone()
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)
    ws = B.alloc_attend_workspace(heads, kv_heads, head_dim, prompt=True)
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    cache.check()
    want, bound = R.attend(s, q[:T], new, weight_rounding=WEIGHT_BF16)
    check(out[:T], want, bound)
    assert torch.equal(out[T:], behind), "rows behind the last sequence were written"
    assert torch.equal(guard[:, heads * head_dim:], edge)
    first = out.clone()
    out[:T].fill_(0.5)
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    assert torch.equal(out, first)


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_that_see_nothing_are_zero(bits):
    """More rows than the sequence is long: the first ones lie in front of it."""
    s = R.Setup([3, 0, 2], 2, 64, 16, bits, seed=7)
    new = [5, 4, 2]
    q = rows(11, 4, 64, 3)
    cu = torch.tensor([0, 5, 9, 11], dtype=torch.int32, device="cuda")
    got = B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), q)
    want, bound = R.attend(s, q, new, weight_rounding=WEIGHT_BF16)
    assert torch.all(want[[0, 1, 5, 6, 7, 8]] == 0) and torch.all(got[[0, 1, 5, 6, 7, 8]] == 0)
    check(got, want, bound)


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_sharp_and_flat_softmax(prompt, bits):
    """Scores of several hundreds (one key takes all), all scores equal, and a caller's own scale."""
    lens, new = [700, 300], [1, 1] if not prompt else [200, 300]
    s = R.Setup(lens, 2, 128, 16, bits, seed=11)
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
    batch = B.KVBatch(s.table, s.kv_lens, cu if prompt else None)
    attend = B.attend_prompt if prompt else B.attend_decode
    for size, scale in ((30.0, None), (0.0, None), (1.5, 0.7), (1.5, 1e-6)):
        q = rows(sum(new), 16, 128, 3, size=size)
        got = attend(s.cache(), batch, q, scale=scale)
        want, bound = R.attend(s, q, new, scale=scale, **error_of(prompt, bits))
        check(got, want, bound)


@pytest.mark.parametrize("prompt", [False, True])
def test_rising_scores_move_the_running_maximum(prompt):
    """Keys that grow along the sequence raise the maximum in every tile, by small and by large steps."""
    n = 900
    s = R.Setup([n], 1, 64, 16, 16, seed=12)
    direction = torch.randn(64, generator=torch.Generator().manual_seed(2)).cuda()
    direction = direction / direction.norm()
    for top in (3.0, 40.0, 2000.0):
        for j in range(n):
            s.pools[0][s.table[0, j // 16].item(), 0, j % 16] = (direction * (top * j / n)).to(torch.bfloat16)
        new = [260 if prompt else 1]
        T = new[0]
        q = (direction * 8.0).to(torch.bfloat16).expand(T, 2, 64).contiguous()
        cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        got = (B.attend_prompt if prompt else B.attend_decode)(s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None), q)
        want, bound = R.attend(s, q, new, **error_of(prompt, s.bits))
        check(got, want, bound)


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_bad_pages_are_left_out_and_reported(prompt, bits):
    lens, new = [100, 130, 90], [1, 1, 1] if not prompt else [20, 30, 90]
    attend = B.attend_prompt if prompt else B.attend_decode
    for bad in (-1, 1 << 30, None):
        s = R.Setup(lens, 2, 64, 16, bits, seed=13, table_extra=0)
        q = rows(sum(new), 4, 64, 3)
        cu = torch.tensor([0, new[0], new[0] + new[1], sum(new)], dtype=torch.int32, device="cuda")
        want, bound = R.attend(s, q, new, **error_of(prompt, s.bits))
        if bad is None:  # a length beyond the table: the keys in it count, the rest does not exist
            s.kv_lens[1] = 16 * s.table.shape[1] + 1000
        else:
            s.table[1, 3] = bad
        cache = s.cache()
        got = attend(cache, B.KVBatch(s.table, s.kv_lens, cu if prompt else None), q)
        with pytest.raises(B.BitLinearError) as e:
            cache.check()
        assert e.value.status == B.ERR_PAGE
        other = [0] + [2] if not prompt else list(range(20)) + list(range(50, 140))
        check(got[other], want[other], bound[other])
        assert torch.all(torch.isfinite(got[[1]] if not prompt else got[20:50])) or bad is None
        if bad is not None and not prompt:
            # sequence 1 without the 16 keys of the bad page: the same as a sequence of the other keys
            left = [j for j in range(130) if j // 16 != 3]
            k, v = s_rows(s, 0, 1, 130, bad_page=3)[:, left], s_rows(s, 1, 1, 130, bad_page=3)[:, left]
            x = q[1].double().view(2, 2, 64)
            w = torch.softmax(torch.einsum("hgd,hld->hgl", x, k) / 8.0, -1)
            y = torch.einsum("hgl,hld->hgd", w, v).reshape(4, 64)
            assert torch.allclose(got[1].double(), y, rtol=2.0 ** -7, atol=1e-3)


def s_rows(s, which, b, n, bad_page):
    keep = s.table[b, bad_page].item()
    s.table[b, bad_page] = 0
    x = s.rows(which, b, n)
    s.table[b, bad_page] = keep
    return x


@pytest.mark.parametrize("prompt", [False, True])
def test_a_page_shared_by_two_sequences(prompt):
    s = R.Setup([64, 80], 2, 64, 32, 16, seed=14)
    s.table[1, :2] = s.table[0, :2]  # a common prefix of two pages
    new = [1, 1] if not prompt else [10, 16]
    q = rows(sum(new), 4, 64, 3)
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
    got = (B.attend_prompt if prompt else B.attend_decode)(s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None), q)
    want, bound = R.attend(s, q, new, **error_of(prompt, s.bits))
    check(got, want, bound)


@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("past", [50, 2850])
def test_a_poisoned_row_reaches_only_the_tokens_that_see_it(where, poison, past):
    """The 50th of 150 new tokens is poisoned: the 49 in front of it do not see it.  With the longer past several CTAs share
    the keys of a tile of rows."""
    lens, new, at = [past + 150, past + 150], [150, 150], past + 49
    s = R.Setup(lens, 1, 64, 16, 16, seed=15)
    clean = [p.clone() for p in s.pools]
    q = rows(300, 2, 64, 3)
    cu = torch.tensor([0, 150, 300], dtype=torch.int32, device="cuda")
    want, bound = R.attend(s, q, new, weight_rounding=WEIGHT_BF16)
    s.pools[0 if where == "key" else 1][s.table[0, at // 16].item(), 0, at % 16, 5] = poison
    got = B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), q)
    free = list(range(49)) + list(range(150, 300))
    check(got[free], want[free], bound[free])
    if where == "value":
        assert not torch.any(torch.isfinite(got[49:150, :, 5]))
        other = [d for d in range(64) if d != 5]
        check(got[..., other], want[..., other], bound[..., other])
    elif poison != poison:
        assert torch.all(got[49:150].isnan())
    # single tokens: in front of the poisoned position and behind it
    s.kv_lens.copy_(torch.tensor([at, at + 1], dtype=torch.int32))
    s.table[1] = s.table[0]
    s.lens = [at, at]
    got = B.attend_decode(s.cache(), B.KVBatch(s.table, s.kv_lens), q[:2])
    s.pools = clean
    want, bound = R.attend(s, q[:2], [1, 1], **decode_error(s.bits))
    check(got[0], want[0], bound[0])
    if where == "value" or poison != poison:
        assert not torch.any(torch.isfinite(got[1, :, 5]))


@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("past", [50, 2850])
def test_an_int8_row_that_is_not_finite_reaches_only_the_tokens_that_see_it(where, past):
    """Such a row has codes 0 and a scale of NaN."""
    lens, new, at = [past + 150, past + 150], [150, 150], past + 49
    s = R.Setup(lens, 1, 64, 16, 8, seed=18)
    q = rows(300, 2, 64, 3)
    cu = torch.tensor([0, 150, 300], dtype=torch.int32, device="cuda")
    want, bound = R.attend(s, q, new, weight_rounding=WEIGHT_BF16)
    which, page = 0 if where == "key" else 1, s.table[0, at // 16].item()
    s.pools[which][page, 0, at % 16] = 0
    s.scales[which][page, 0, at % 16] = float("nan")
    got = B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), q)
    free = list(range(49)) + list(range(150, 300))
    check(got[free], want[free], bound[free])
    assert torch.all(got[49:150].isnan())
    s.kv_lens.copy_(torch.tensor([at, at + 1], dtype=torch.int32))
    s.table[1] = s.table[0]
    got = B.attend_decode(s.cache(), B.KVBatch(s.table, s.kv_lens), q[:2])
    s.lens = [at, at]
    want, bound = R.attend(s, q[:1], [1, 0], **decode_error(s.bits))
    check(got[:1], want, bound)
    assert torch.all(got[1].isnan())


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_queries_of_any_size(prompt, bits):
    """Rows of zeros, of subnormal, tiny and huge elements, and of elements 30 binary orders apart; a NaN and an infinity stay in
    their own row and head."""
    lens, new = [100] * 8, [1] * 8
    s = R.Setup(lens, 2, 64, 16, bits, seed=19)
    q = rows(8, 4, 64, 5)
    q[0] = 0.0
    q[1] *= 1e-39
    q[2] *= 1e-30
    q[3] *= 1e4
    q[4, :, ::2] *= 2.0 ** -30
    cu = torch.arange(9, dtype=torch.int32, device="cuda")
    attend = B.attend_prompt if prompt else B.attend_decode
    batch = B.KVBatch(s.table, s.kv_lens, cu if prompt else None)
    got = attend(s.cache(), batch, q)
    want, bound = R.attend(s, q, new, **error_of(prompt, bits))
    check(got, want, bound)
    sick = q.clone()
    sick[5, 1, 7] = float("nan")
    sick[6, 2, 9] = float("inf")
    got = attend(s.cache(), batch, sick)
    well = torch.ones(8, 4, dtype=torch.bool, device="cuda")
    well[5, 1] = well[6, 2] = False
    check(got[well], want[well], bound[well])
    assert torch.all(got[5, 1].isnan()) and not torch.any(torch.isfinite(got[6, 2]))


def test_prompts_of_more_sequences_than_are_put_in_order():
    g = torch.Generator().manual_seed(2)
    new = torch.randint(0, 6, (700,), generator=g).tolist()
    lens = [n + p for n, p in zip(new, torch.randint(0, 60, (700,), generator=g).tolist())]
    s = R.Setup(lens, 1, 16, 16, 16, seed=20)
    q = rows(sum(new), 2, 16, 5)
    cu = torch.tensor([sum(new[:i]) for i in range(701)], dtype=torch.int32, device="cuda")
    got = B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), q)
    want, bound = R.attend(s, q, new, weight_rounding=WEIGHT_BF16)
    check(got, want, bound)


def test_one_workspace_serves_both_kernels_in_turn():
    s = R.Setup([3000, 200], 2, 128, 16, 16, seed=23)
    ws = torch.zeros(max(B.attend_workspace_bytes(8, 2, 128, p) for p in (False, True)), dtype=torch.uint8, device="cuda")
    cu = torch.tensor([0, 20, 30], dtype=torch.int32, device="cuda")
    q, single = rows(30, 8, 128, 1), rows(2, 8, 128, 2)
    for _ in range(3):
        got = B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), q, workspace=ws)
        want, bound = R.attend(s, q, [20, 10], weight_rounding=WEIGHT_BF16)
        check(got, want, bound)
        got = B.attend_decode(s.cache(), B.KVBatch(s.table, s.kv_lens), single, workspace=ws)
        want, bound = R.attend(s, single, [1, 1], **decode_error(16))
        check(got, want, bound)


def test_a_cache_beyond_32_bit_offsets():
    """Pages at the end of a pool of more than 2^32 bytes: appended to, and read by both kernels."""
    pages, page_size, kv_heads, D = 33000, 64, 8, 128
    shape = (pages, kv_heads, page_size, D)
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("not enough free memory")
    k, v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() * 2 > 1 << 32
    s = R.Setup([130], kv_heads, D, page_size, 16, seed=24, spare=0, table_extra=0)
    small = s.pools
    s.table = torch.tensor([[pages - 1, 32800, pages - 2]], dtype=torch.int32, device="cuda")
    s.pools = [k, v]
    n = 130
    new_k, new_v = rows(n, kv_heads, D, 1, size=1.0), rows(n, kv_heads, D, 2, size=1.0)
    cache, cu = s.cache(), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    B.kv_append(cache, B.KVBatch(s.table, s.kv_lens, cu), new_k, new_v)
    assert torch.equal(k[pages - 1, :, 0], new_k[0]) and torch.equal(v[32800, :, 63], new_v[127])
    q = rows(n, 16, D, 3)
    got = B.attend_prompt(cache, B.KVBatch(s.table, s.kv_lens, cu), q)
    want, bound = R.attend(s, q, [n], weight_rounding=WEIGHT_BF16)
    check(got, want, bound)
    got = B.attend_decode(cache, B.KVBatch(s.table, s.kv_lens), q[:1])
    want, bound = R.attend(s, q[:1], [1], **decode_error(16))
    check(got, want, bound)
    cache.check()
    del k, v, small


@pytest.mark.parametrize("bits", [16, 8])
def test_an_expired_wait_of_the_prompt_kernel_ends_it_with_a_status(bits):
    """One CTA, whose first copy and its announcement are left out, with a limit of 2 ms: the call returns, the cache's
    status says so, and the next call on the same workspace is right."""
    s = R.Setup([200], 1, 64, 16, bits, seed=25)
    q = rows(60, 2, 64, 1)
    cu = torch.tensor([0, 60], dtype=torch.int32, device="cuda")
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)
    ws, out = B.alloc_attend_workspace(2, 1, 64, prompt=True), torch.empty(60, 2, 64, dtype=torch.bfloat16, device="cuda")
    want, bound = R.attend(s, q, [60], weight_rounding=WEIGHT_BF16)
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    check(out, want, bound)
    B.test_expire_next_wait(2000, True)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    end.record()
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_TIMEOUT
    assert 1.5 < start.elapsed_time(end) < 500.0
    for _ in range(2):
        out.fill_(0.5)
        B.attend_prompt(cache, batch, q, out=out, workspace=ws)
        cache.check()
        check(out, want, bound)


@pytest.mark.parametrize("prompt", [False, True])
def test_a_captured_graph_follows_lengths_pages_and_queries(prompt):
    """Two graphs over one workspace, replayed in turn, while lengths and pages change."""
    lens = [300, 40, 129]
    new = [1, 1, 1] if not prompt else [60, 7, 129]
    T = sum(new)
    attend = B.attend_prompt if prompt else B.attend_decode
    cu = torch.tensor([0, new[0], new[0] + new[1], T], dtype=torch.int32, device="cuda")
    one, two = R.Setup(lens, 2, 128, 16, 16, seed=16), R.Setup(lens, 2, 128, 16, 8, seed=17)
    q, out = rows(T, 8, 128, 3), [torch.empty(T, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ws = B.alloc_attend_workspace(8, 2, 128, prompt=prompt)
    graphs = []
    for s, o in zip((one, two), out):
        cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None)
        attend(cache, batch, q, out=o, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attend(cache, batch, q, out=o, workspace=ws)
        graphs.append((g, cache, batch))
    for step, change in enumerate(([300, 40, 129], [299, 39, 129], [60, 7, 129], [200, 8, 129])):
        for i, s in enumerate((one, two)):
            s.lens = change
            s.kv_lens.copy_(torch.tensor(change, dtype=torch.int32))
        q.copy_(rows(T, 8, 128, 20 + step))
        for _ in range(2):
            for g, _, _ in graphs:
                g.replay()
        for s, o in zip((one, two), out):
            want, bound = R.attend(s, q, new, **error_of(prompt, s.bits))
            check(o, want, bound)


@pytest.mark.parametrize("prompt", [False, True])
def test_two_streams_with_workspaces_of_their_own(prompt):
    new = [1, 1] if not prompt else [100, 33]
    attend = B.attend_prompt if prompt else B.attend_decode
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
    cases = []
    for seed in (21, 22):
        s = R.Setup([4000, 600], 2, 128, 16, 16, seed=seed)
        cases.append((s, s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None), rows(sum(new), 8, 128, seed),
                      B.alloc_attend_workspace(8, 2, 128, prompt=prompt), torch.cuda.Stream(),
                      torch.empty(sum(new), 8, 128, dtype=torch.bfloat16, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for _, cache, batch, q, ws, stream, out in cases:
            attend(cache, batch, q, out=out, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for s, _, _, q, _, _, out in cases:
        want, bound = R.attend(s, q, new, **error_of(prompt, s.bits))
        check(out, want, bound)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads,kv_heads,head_dim", [(24, 8, 64), (4, 4, 100), (8, 1, 128)])
def test_chunks_whose_keys_are_split_among_as_many_ctas_as_their_number_allows(heads, kv_heads, head_dim, bits):
    # one workspace, one captured call: how the rows belong to sequences, and with that the splits, changes between replays
    s = R.Setup([2100, 1300, 900, 5], kv_heads, head_dim, 32, bits, seed=51)
    T, q = 60, rows(60, heads, head_dim, 51)
    cu = torch.tensor([0, 15, 30, 45, 60], dtype=torch.int32, device="cuda")
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)
    ws = B.alloc_attend_workspace(heads, kv_heads, head_dim, prompt=True)
    out = torch.empty(T, heads, head_dim, dtype=torch.bfloat16, device="cuda")
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    for new in ([15, 15, 15, 15], [60, 0, 0, 0], [0, 59, 0, 1], [1, 2, 55, 2], [20, 20, 20, 0]):
        cu.copy_(torch.tensor([sum(new[:i]) for i in range(5)], dtype=torch.int32))
        out.fill_(0.5)
        graph.replay()
        want, bound = R.attend(s, q, new, weight_rounding=WEIGHT_BF16)
        check(out, want, bound)
        first = out.clone()
        graph.replay()
        assert torch.equal(out, first)
    cache.check()
    assert not ws[:2048].any(), "the counters are left at zero"


@pytest.mark.parametrize("heads,kv_heads", [(4096, 1024), (4096, 1)])
@pytest.mark.parametrize("bits", [16, 8])
def test_the_most_heads(heads, kv_heads, bits):
    s = R.Setup([70, 3], kv_heads, 32, 16, bits, seed=41)
    q = rows(2, heads, 32, 41)
    out = B.attend_decode(s.cache(), B.KVBatch(s.table, s.kv_lens), q)
    want, bound = R.attend(s, q, [1, 1], **decode_error(bits))
    check(out, want, bound)
    q = rows(5, heads, 32, 42)
    cu = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    out = B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), q)
    want, bound = R.attend(s, q, [3, 2], weight_rounding=WEIGHT_BF16)
    check(out, want, bound)


@pytest.mark.parametrize("cu", [[0, 4, 9], [0, 4, 2], [0, 4, 2 ** 31 - 1], [-3, 4, 4], [-2 ** 31, 4, 5]])
def test_token_rows_that_do_not_exist_are_neither_read_nor_written(cu):
    # five rows were handed over; the first sequence's four are computed where its rows are in order
    s = R.Setup([30, 21], 2, 64, 16, 16, seed=43)
    q = rows(5, 4, 64, 43)
    wide = torch.full((15, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    out = wide[5:10]
    bounds = torch.tensor(cu, dtype=torch.int32, device="cuda")
    B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, bounds), q, out=out)
    assert torch.all(wide[:5] == 3.0) and torch.all(wide[10:] == 3.0)
    if cu[0] == 0:
        want, bound = R.attend(s, q[:4], [4], weight_rounding=WEIGHT_BF16)
        check(out[:4], want, bound)


@pytest.mark.parametrize("prompt", [False, True])
def test_what_a_call_allocates_belongs_to_its_stream(prompt):
    # the current stream is busy, and its free memory holds ones: a workspace that it filled would not be zero in time
    new = [1, 1] if not prompt else [100, 33]
    attend = B.attend_prompt if prompt else B.attend_decode
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
    s = R.Setup([4000, 600], 2, 128, 16, 16, seed=31)
    cache, batch, q = s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None), rows(sum(new), 8, 128, 31)
    stale = torch.full((B.attend_workspace_bytes(8, 2, 128, prompt),), 255, dtype=torch.uint8, device="cuda")
    side, by_number = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    del stale
    torch.cuda._sleep(100_000_000)
    outs = []
    for stream in (side, by_number.cuda_stream):
        q_rotated = B.kv_append(s.cache(), B.KVBatch(s.table[:0], s.kv_lens[:0]), q[:0, :2], q[:0, :2], q=q[:0], stream=stream)
        assert q_rotated.shape == (0, 8, 128)
        table = B.rope_table(64, 128, stream=stream)
        outs.append((attend(cache, batch, q, stream=stream), table))
    torch.cuda.synchronize()
    want, bound = R.attend(s, q, new, **error_of(prompt, s.bits))
    for out, table in outs:
        check(out, want, bound)
        assert torch.equal(table, B.rope_table(64, 128))


def test_nothing_to_attend():
    s = R.Setup([4], 2, 64, 16, 16)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert B.attend_decode(s.cache(), B.KVBatch(s.table[:0], s.kv_lens[:0]), none).shape == (0, 4, 64)
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert B.attend_prompt(s.cache(), B.KVBatch(s.table, s.kv_lens, zero), none).shape == (0, 4, 64)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("hidden,heads,kv_heads", [(3200, 32, 32), (1024, 8, 2)])
def test_a_prompt_and_then_single_tokens_through_the_projections(hidden, heads, kv_heads, bits):
    """One attention block as a decoder layer runs it: BitLinear q/k/v (one fused weight, RMSNorm in front), append, attend,
    BitLinear o; first a prompt of two sequences, then three tokens each from a captured graph.  Every operator is held to its
    64-bit restatement on the inputs it was given."""
    from paper_2402_17764_b200 import synthetic as S
    D = hidden // heads
    width = (heads + 2 * kv_heads) * D
    w_qkv, g_qkv = B.quantize_weights(S.latent_weights(width, hidden, 1).cuda())
    w_o, g_o = B.quantize_weights(S.latent_weights(hidden, hidden, 2).cuda())
    gain = torch.ones(hidden, device="cuda")
    new, steps = [45, 130], 3
    cache = B.KVCache(40, kv_heads, D, page_size=16, bits=bits)
    table = torch.randperm(40, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda().view(2, 20)
    kv_lens = torch.tensor(new, dtype=torch.int32, device="cuda")
    rope = B.rope_table(200, D)

    class Held(R.Setup):
        def __init__(self, lens):
            self.lens, self.kv_heads, self.head_dim, self.page_size, self.bits = lens, kv_heads, D, 16, bits
            self.pools, self.scales, self.table = [cache.k, cache.v], [cache.k_scale, cache.v_scale], table

    def block(h, batch, attend, ws, fws, q_out, a, y):
        T = h.shape[0]
        qkv = B.forward_rmsnorm(w_qkv, g_qkv, h, gain, 1e-5, width, workspace=fws[0])
        q = qkv[:, :heads * D].unflatten(1, (heads, D))
        k = qkv[:, heads * D:(heads + kv_heads) * D].unflatten(1, (kv_heads, D))
        v = qkv[:, (heads + kv_heads) * D:].unflatten(1, (kv_heads, D))
        B.kv_append(cache, batch, k, v, q=q, rope=rope, q_out=q_out)
        attend(cache, batch, q_out, out=a, workspace=ws)
        B.forward(w_o, g_o, a.view(T, hidden), hidden, Y=y, workspace=fws[1])
        return qkv, k, v

    def held(qkv, k, q_out, a, y, lens, counts):
        pos = torch.cat([torch.arange(n - c, n) for n, c in zip(lens, counts)]).cuda()
        seq = torch.cat([torch.full((c,), i) for i, c in enumerate(counts)]).cuda()
        z, size = R.rotate(k, rope, pos, False)
        stored = cache.k[table[seq, pos // 16].long(), :, pos % 16][..., :D]
        if bits == 16:
            assert torch.all((stored.double() - z).abs() <= 2.0 ** -8 * z.abs() + 1.01 * 3 * 2.0 ** -24 * size)
        else:
            assert torch.equal(stored, R.codes(z)[0])
        want, bound = R.attend(Held(lens), q_out, counts, weight_rounding=WEIGHT_BF16)
        check(a, want, bound)
        assert torch.equal(y, B.forward(w_o, g_o, a.view(-1, hidden), hidden))

    def buffers(T):
        return [torch.empty(T, heads, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, heads, D, dtype=torch.bfloat16, device="cuda"),
                torch.empty(T, hidden, dtype=torch.bfloat16, device="cuda")]

    T = sum(new)
    cu = torch.tensor([0, new[0], T], dtype=torch.int32, device="cuda")
    q_out, a, y = buffers(T)
    fws = [B.alloc_workspace(T, width, hidden), B.alloc_workspace(T, hidden, hidden)]
    h = S.activations(T, hidden, 5).cuda()
    qkv, k, v = block(h, B.KVBatch(table, kv_lens, cu), B.attend_prompt, B.alloc_attend_workspace(heads, kv_heads, D, prompt=True), fws, q_out, a, y)
    cache.check()
    held(qkv, k, q_out, a, y, new, new)

    q_out, a, y = buffers(2)
    fws = [B.alloc_workspace(2, width, hidden), B.alloc_workspace(2, hidden, hidden)]
    ws = B.alloc_attend_workspace(heads, kv_heads, D, prompt=False)
    batch = B.KVBatch(table, kv_lens)
    h = S.activations(2, hidden, 6).cuda()
    kv_lens.add_(1)
    block(h, batch, B.attend_decode, ws, fws, q_out, a, y)  # the first run sets kernel attributes
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qkv, k, v = block(h, batch, B.attend_decode, ws, fws, q_out, a, y)
    for step in range(steps):
        h.copy_(S.activations(2, hidden, 7 + step))
        graph.replay()
        torch.cuda.synchronize()
        cache.check()
        held(qkv, k, q_out, a, y, [n + 1 + step for n in new], [1, 1])
        kv_lens.add_(1)
