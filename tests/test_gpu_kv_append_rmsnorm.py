"""Appending with normalised queries and keys, at positions of the caller's, with marks, against a 64-bit restatement."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_kv_append import HEADS, place, tokens

pytestmark = pytest.mark.gpu

# 1 / rms in fp32: a lane's squares and their sum over the lanes (at most 16 + 5 roundings of positive terms), the mean and its epsilon
# (2), half of that by the root, then root and quotient (2): 14 2^-24.  Two products with it make 16, the rotation's
# products and sum 19; 20 with what is of second order.
OVER_RMS = 14 * 2.0 ** -24
ROTATED = 20 * 2.0 ** -24


def gains(head_dim, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.3 * torch.randn(2, head_dim, generator=g)).cuda().unbind(0)


def over_rms(x, eps):
    x = x.double()
    return 1 / torch.sqrt(((x * x).mean(-1, keepdim=True) + eps).clamp(min=2.0 ** -126))


def marks_of(cache):
    marks = B.KVMarks(cache)
    marks.mass.fill_(3.0)
    marks.pos.fill_(-5)
    return marks


@pytest.mark.parametrize("heads,kv_heads,head_dim", HEADS)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_against_64_bits(heads, kv_heads, head_dim, bits, interleaved):
    page_size = {100: 16, 128: 64, 64: 32, 4: 16, 20: 256, 48: 128, 80: 16, 124: 32}[head_dim]
    counts, past = [1, 0, 37, 16, 5, 3], [0, 9, 250, 15, 16, 0]
    lens = [n + p for n, p in zip(counts, past)]
    lens[5] = 1  # two of the three rows lie in front of the sequence
    s = R.Setup(lens, kv_heads, head_dim, page_size, bits, seed=head_dim + bits)
    q, k, v = tokens(counts, past, heads, kv_heads, head_dim, seed=1, extra_rows=2)
    rope, eps = R.angles(2000, head_dim), 1e-5
    q_gain, k_gain = gains(head_dim, 2)
    cu = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)
    marks = marks_of(cache)
    positions = torch.randint(0, 2000, (q.shape[0],), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    before = [p.clone() for p in s.pools]
    q_out = torch.full((q.shape[0], heads * head_dim + 24 + (-heads * head_dim) % 8), 7.0, dtype=torch.bfloat16, device="cuda")
    view = q_out[:, :heads * head_dim].unflatten(1, (heads, head_dim))
    B.kv_append_rmsnorm(cache, batch, k, v, q=q, q_gain=q_gain, k_gain=k_gain, norm_eps=eps, rope=rope, interleaved=interleaved,
                        positions=positions, marks=marks, q_out=view)
    cache.check()
    rows, seqs, slot = place(s.table, counts, lens, page_size)
    page, at, angle = s.table[seqs, slot // page_size].long(), slot % page_size, positions[rows].long()

    def normed(x, gain):
        return x[rows].double() * over_rms(x[rows], eps) * gain.double()

    want, size = R.rotate(normed(q, q_gain), rope, angle, interleaved)
    assert torch.all((view[rows].double() - want).abs() <= 2.0 ** -8 * want.abs() + ROTATED * size)
    kept = torch.ones(q_out.shape[0], dtype=torch.bool, device="cuda")
    kept[rows] = False
    assert torch.all(q_out[kept] == 7.0) and torch.all(q_out[:, heads * head_dim:] == 7.0)
    for which in (0, 1):
        stored = s.pools[which][page, :, at]
        if bits == 16:
            if which == 0:
                want, size = R.rotate(normed(k, k_gain), rope, angle, interleaved)
                assert torch.all((stored[..., :head_dim].double() - want).abs() <= 2.0 ** -8 * want.abs() + ROTATED * size)
            else:
                assert torch.equal(stored[..., :head_dim], v[rows])
        else:
            factor = over_rms(k[rows], eps)[..., 0] if which == 0 else 1.0
            z = R.rotate(k[rows].double() * k_gain.double(), rope, angle, interleaved)[0] if which == 0 else v[rows].double()
            beta = z.abs().amax(-1)
            assert torch.all(beta * factor > 1e-5), "the floor is another test's"
            assert torch.equal(stored[..., :head_dim], torch.round(z * 127 / beta[..., None]).to(torch.int8))
            scale = beta * factor / 127
            got = s.scales[which][page, :, at].double()
            assert torch.all((got - scale).abs() <= (OVER_RMS + 2 * 2.0 ** -24) * scale)
        assert torch.all(stored[..., head_dim:] == 0)
        mask = torch.ones(s.n_pages, page_size, dtype=torch.bool, device="cuda")
        mask[page, at] = False
        now, then = s.pools[which].transpose(1, 2)[mask], before[which].transpose(1, 2)[mask]
        kind = torch.int16 if bits == 16 else torch.int8
        assert torch.equal(now.contiguous().view(kind), then.contiguous().view(kind)), "rows written that are not the call's"
    mass, pos = torch.full_like(marks.mass, 3.0), torch.full_like(marks.pos, -5)
    mass[page, :, at] = 0.0
    pos[page, :, at] = positions[rows][:, None]
    assert torch.equal(marks.mass, mass) and torch.equal(marks.pos, pos)


@pytest.mark.parametrize("head_dim", [128, 100])
@pytest.mark.parametrize("bits", [16, 8])
def test_what_is_not_given_is_not_done(head_dim, bits):
    """Without gains, positions and marks the call is kv_append; with one gain only the queries, or the keys, change."""
    counts = [5, 1, 0, 9]
    s, t = (R.Setup([5, 8, 3, 40], 2, head_dim, 16, bits, seed=4) for _ in range(2))
    q, k, v = tokens(counts, None, 6, 2, head_dim, seed=5)
    rope, cu = R.angles(64, head_dim), torch.tensor([0, 5, 6, 6, 15], dtype=torch.int32, device="cuda")
    kind = torch.int16 if bits == 16 else torch.int8

    def contents(x):
        return [p.view(kind) for p in x.pools] + [z.view(torch.int32) for z in x.scales if z is not None]

    want = B.kv_append(t.cache(), B.KVBatch(t.table, t.kv_lens, cu), k, v, q=q, rope=rope)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)
    got = B.kv_append_rmsnorm(cache, batch, k, v, q=q, rope=rope)
    assert torch.equal(got, want) and all(torch.equal(x, y) for x, y in zip(contents(s), contents(t)))
    q_gain, k_gain = gains(head_dim, 6)
    got = B.kv_append_rmsnorm(cache, batch, k, v, q=q, q_gain=q_gain, rope=rope)
    assert not torch.equal(got, want) and all(torch.equal(x, y) for x, y in zip(contents(s), contents(t)))
    got = B.kv_append_rmsnorm(cache, batch, k, v, q=q, k_gain=k_gain, rope=rope)
    assert torch.equal(got, want) and not torch.equal(s.pools[0].view(kind), t.pools[0].view(kind))
    assert torch.equal(s.pools[1].view(kind), t.pools[1].view(kind))
    assert B.kv_append_rmsnorm(cache, batch, k, v, k_gain=k_gain, rope=rope) is None
    cache.check()


@pytest.mark.parametrize("head_dim", [64, 100])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_rows_of_every_size(head_dim, eps):
    """Rows whose squares leave fp32's range, rows of zeros and rows that are not finite."""
    sizes = [0.0, 1e-38, 1e-30, 1e-20, 1e-8, 1.0, 1e15, 1e19, 1e30, 3e38]
    T = len(sizes) + 2
    g = torch.Generator().manual_seed(7)
    x = (2 * torch.rand(T, 2, head_dim, generator=g) - 1).double()
    x[:len(sizes)] *= torch.tensor(sizes).double()[:, None, None]
    x[-2, 0, 3], x[-1, 1, 5] = float("inf"), float("nan")
    x = x.to(torch.bfloat16).cuda()
    width = (2 * head_dim + 7) // 8 * 8
    padded = torch.zeros(T, width, dtype=torch.bfloat16, device="cuda")
    padded[:, :2 * head_dim] = x.flatten(1)
    x = padded[:, :2 * head_dim].unflatten(1, (2, head_dim))
    gain = gains(head_dim, 8)[0]
    s = R.Setup([T], 2, head_dim, 16, 16, seed=9)
    cache = s.cache()
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    out = B.kv_append_rmsnorm(cache, B.KVBatch(s.table, s.kv_lens, cu), x, x, q=x, q_gain=gain, k_gain=gain, norm_eps=eps)
    cache.check()
    r = over_rms(x, eps)
    want = x.double() * r * gain.double()
    # (1 / rms itself may be subnormal for the largest rows: half a step of 2^-149; an element below 2^-126 keeps fewer bits)
    tolerance = 2.0 ** -8 * want.abs() + OVER_RMS * 2 * want.abs() + x.double().abs() * 2.0 ** -150 * 2 + 2.0 ** -133
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(want), torch.isnan(out))
    assert torch.all((out.double() - want).abs()[finite] <= tolerance[finite])
    assert torch.equal(torch.isfinite(out), finite)
    stored = s.pools[0][s.table[0, 0].long()].transpose(0, 1)[:T, :, :head_dim]
    assert torch.equal(stored.contiguous().view(torch.int16), out.contiguous().view(torch.int16))


@pytest.mark.parametrize("head_dim", [64, 100])
def test_8_bit_rows_at_the_floor_and_not_finite(head_dim):
    """Rows whose largest normalised element is below the floor of beta, all-zero rows, infinities, NaN and a gain that is not
    finite."""
    T = 7
    g = torch.Generator().manual_seed(10)
    x = torch.randn(T, 1, head_dim, generator=g)
    x[1] *= 0
    x[2] *= 1e-10
    x[3] *= 1e-11
    x[4, 0, 0], x[5, 0, 1] = float("inf"), float("nan")
    x[6] *= 2.0 ** 126 / x[6].abs().max()
    padded = torch.zeros(T, (head_dim + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")
    padded[:, :head_dim] = x.flatten(1).to(torch.bfloat16).cuda()
    x = padded[:, :head_dim].unflatten(1, (1, head_dim))
    gain = gains(head_dim, 11)[0]
    s = R.Setup([T], 1, head_dim, 16, 8, seed=12)
    cache = s.cache()
    batch = B.KVBatch(s.table, s.kv_lens, torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    B.kv_append_rmsnorm(cache, batch, x, x, k_gain=gain, norm_eps=1e-5)
    cache.check()
    page = s.table[0, 0].long()
    codes, scale = s.pools[0][page, 0, :T, :head_dim], s.scales[0][page, 0, :T]
    z, r = x[:, 0].double() * gain.double(), over_rms(x[:, 0], 1e-5)
    floor = 1e-5 / r
    beta = torch.maximum(z.abs().amax(-1, keepdim=True), floor)
    want = z * 127 / beta
    for t in (0, 1, 2, 3, 6):
        # at the floor the factor, off by OVER_RMS, does not cancel out
        slack = 127 * 2 * OVER_RMS if t in (1, 2, 3) else 0.0
        assert torch.all((codes[t].double() - want[t]).abs() <= 0.5 + slack + 1e-12)
        assert abs(scale[t].item() - (beta * r / 127)[t].item()) <= (OVER_RMS + 2.0 ** -23) * (beta * r / 127)[t].item()
    assert torch.all(codes[4:6] == 0) and torch.all(torch.isnan(scale[4:6]))
    bad = gain.clone()
    bad[2] = float("nan")
    B.kv_append_rmsnorm(cache, batch, x, x, k_gain=bad, norm_eps=1e-5)
    assert torch.all(torch.isnan(s.scales[0][page, 0, :T])) and torch.all(s.pools[0][page, 0, :T] == 0)


@pytest.mark.parametrize("bits", [16, 8])
def test_bad_positions_pages_and_rows(bits):
    """Positions outside the rotary table: the token is left out and the status set; a bad page: rotated, not stored, not marked."""
    s = R.Setup([20, 20, 20], 2, 64, 16, bits, seed=13)
    s.table[1, 1] = s.n_pages
    q, k, v = tokens([1, 1, 1], None, 4, 2, 64, seed=14)
    gain, rope = gains(64, 15)[0], R.angles(50, 64)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    for bad in ([49, 3, 50], [0, 7, -1], [5, 2, 2 ** 31 - 1]):
        before = [p.clone() for p in s.pools]
        marks, out = marks_of(cache), torch.full((3, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        B.kv_append_rmsnorm(cache, batch, k, v, q=q, q_gain=gain, k_gain=gain, rope=rope, marks=marks, q_out=out,
                            positions=torch.tensor(bad, dtype=torch.int32, device="cuda"))
        with pytest.raises(B.BitLinearError) as e:
            cache.check()
        assert e.value.status == B.ERR_PAGE
        assert torch.all(out[2] == 7.0) and not torch.any(out[:2] == 7.0)
        row = s.table[0, 1].long(), slice(None), 3
        assert torch.all(marks.mass[row] == 0) and torch.all(marks.pos[row] == bad[0])
        changed = [(p.view(torch.int16 if bits == 16 else torch.int8) != b.view(torch.int16 if bits == 16 else torch.int8)).any(-1) for p, b in zip(s.pools, before)]
        for c in changed + [marks.mass != 3.0, marks.pos != -5]:
            c[row] = False
            assert not c.any()
        # without a rotary table any position is kept
        B.kv_append_rmsnorm(cache, B.KVBatch(s.table[2:], s.kv_lens[2:]), k[2:], v[2:], k_gain=gain, marks=marks,
                            positions=torch.tensor(bad[2:], dtype=torch.int32, device="cuda"))
        cache.check()
        assert torch.all(marks.pos[s.table[2, 1].long(), :, 3] == bad[2])


def test_in_place_on_a_side_stream_and_in_a_graph():
    s = R.Setup([17, 4], 2, 128, 16, 8, seed=16)
    q, k, v = tokens([1, 1], None, 8, 2, 128, seed=17)
    q_gain, k_gain = gains(128, 18)
    rope, cache, batch = R.angles(100, 128), s.cache(), B.KVBatch(s.table, s.kv_lens)
    marks, positions = marks_of(cache), torch.tensor([90, 3], dtype=torch.int32, device="cuda")
    args = dict(q_gain=q_gain, k_gain=k_gain, rope=rope, positions=positions, marks=marks)
    want = B.kv_append_rmsnorm(cache, batch, k, v, q=q, **args)
    codes = s.pools[0].clone()
    side = torch.cuda.Stream()
    own = q.clone()
    torch.cuda.synchronize()
    assert B.kv_append_rmsnorm(cache, batch, k, v, q=own, q_out=own, stream=side, **args) is own
    got = B.kv_append_rmsnorm(cache, batch, k, v, q=q, stream=side, **args)
    torch.cuda.synchronize()
    assert torch.equal(own, want) and torch.equal(got, want) and torch.equal(s.pools[0], codes)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.graph(graph):
        B.kv_append_rmsnorm(cache, batch, k, v, q=q, q_out=out, **args)
    positions.copy_(torch.tensor([1, 99], dtype=torch.int32))
    graph.replay()
    fresh = B.kv_append_rmsnorm(cache, batch, k, v, q=q, **args)
    assert torch.equal(out, fresh) and not torch.equal(out, want)
    cache.check()


def test_nothing_to_append():
    s = R.Setup([3], 2, 64, 16, 16, seed=19)
    empty = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cu = torch.zeros(2, dtype=torch.int32, device="cuda")
    out = B.kv_append_rmsnorm(s.cache(), B.KVBatch(s.table, s.kv_lens, cu), empty, empty, q=empty, q_gain=gains(64, 1)[0])
    assert out.shape == (0, 2, 64)
