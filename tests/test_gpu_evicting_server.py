"""The operators of a server that evicts rows and shares beginnings, one after the other as such a server calls them."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import decode_error, error_of, check, rows

pytestmark = pytest.mark.gpu


def normed(x, gain, eps):
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()


@pytest.mark.parametrize("heads,kv_heads,head_dim,bits", [(8, 2, 128, 16), (6, 6, 100, 16), (8, 2, 64, 8), (4, 4, 100, 8)])
def test_prompts_steps_and_evictions(heads, kv_heads, head_dim, bits):
    """Two prompts, then single tokens; whenever a sequence is a page over its budget, rows are evicted.  What the cache holds is
    followed row by row from what was appended (to within the rounding of a row: a normalised key, rotated at its own position),
    and every attention is held to 64 bits over the rows that the cache then holds."""
    page, keep, recent, eps = 16, 48, 16, 1e-5
    counts, steps = [70, 41], 40
    n_pages, table_pages = 16, 8
    cache = B.KVCache(n_pages, kv_heads, head_dim, page_size=page, bits=bits)
    marks = B.KVMarks(cache)
    g = torch.Generator().manual_seed(1)
    table = torch.randperm(n_pages, generator=g).to(torch.int32).view(2, table_pages).cuda()
    gains = (1 + 0.2 * torch.randn(2, head_dim, generator=g)).cuda()
    rope = R.angles(200, head_dim)
    lens = torch.tensor(counts, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device="cuda")
    seen = [sum(counts[:1]), counts[1]]                 # tokens of each sequence so far
    held = [[list(range(n)) for _ in range(kv_heads)] for n in counts]  # positions of the rows, by kv head
    said = [{}, {}]                                     # position -> (key, value) in 64 bits, of all kv heads

    def setup():
        s = R.Setup.__new__(R.Setup)
        s.lens, s.kv_heads, s.head_dim, s.page_size, s.bits = lens.tolist(), kv_heads, head_dim, page, bits
        s.table, s.pools, s.scales = table, [cache.k, cache.v], [cache.k_scale, cache.v_scale]
        return s

    def append(tokens, batch, positions):
        q, k, v = (rows(len(tokens), n, head_dim, 100 * seen[0] + i, size=2.0) for i, n in enumerate((heads, kv_heads, kv_heads)))
        where = torch.tensor(positions, dtype=torch.int32, device="cuda")
        out = B.kv_append_rmsnorm(cache, batch, k, v, q=q, q_gain=gains[0], k_gain=gains[1], norm_eps=eps, rope=rope, positions=where, marks=marks)
        want, _ = R.rotate(normed(q, gains[0], eps), rope, where.long(), False)
        assert torch.all((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * want.abs().max())
        keys = R.rotate(normed(k, gains[1], eps), rope, where.long(), False)[0]
        for t, b in enumerate(tokens):
            said[b][positions[t]] = keys[t], v[t].double()
        return out

    def check_cache():
        s = setup()
        for b in range(2):
            n = s.lens[b]
            for h in range(kv_heads):
                assert len(held[b][h]) == n
                for which in (0, 1):
                    want = torch.stack([said[b][p][which][h] for p in held[b][h]])
                    largest = want.abs().amax(-1, keepdim=True)
                    # bf16: half a step of each value; codes: half a code, and the scale's rounding
                    tolerance = 2.0 ** -8 * want.abs() + 2.0 ** -18 * largest if bits == 16 else (0.5 / 127 + 2.0 ** -18) * largest
                    assert torch.all((s.rows(which, b, n)[h] - want).abs() <= tolerance)
                pos = marks.pos[table[b].long()[torch.arange(n, device="cuda") // page], h, torch.arange(n, device="cuda") % page]
                assert pos.tolist() == held[b][h]
        return s

    batch = B.KVBatch(table, lens, cu)
    q = append([0] * counts[0] + [1] * counts[1], batch, list(range(counts[0])) + list(range(counts[1])))
    out = B.attend_prompt(cache, batch, q)
    s = check_cache()
    want, bound = R.attend(s, q, counts, **error_of(True, bits))
    check(out, want, bound)
    single = B.KVBatch(table, lens)
    ws = B.alloc_attend_weigh_workspace(heads, kv_heads, head_dim, bits, 2, 2 * table_pages * page)
    evictions = 0
    for step in range(steps):
        lens += 1
        for b in range(2):
            for h in range(kv_heads):
                held[b][h].append(seen[b])
        q = append([0, 1], single, list(seen))
        seen = [n + 1 for n in seen]
        total = marks.mass.double().sum().item()
        out = B.attend_decode_weigh(cache, single, marks, q, workspace=ws)
        s = check_cache()
        want, bound = R.attend(s, q, [1, 1], **decode_error(bits))
        check(out, want, bound)
        assert abs(marks.mass.double().sum().item() - total - 2 * heads) < 1e-3, "every query head hands out a weight of one"
        if max(lens.tolist()) < keep + page:
            continue
        before = setup()
        mass = marks.mass.clone()
        source, new_lens = B.kv_select(cache, single, marks, keep, recent)
        B.kv_compact(cache, single, source, marks)
        for b in range(2):
            for h in range(kv_heads):
                n = before.lens[b]
                at = lambda x: x[table[b].long()[torch.arange(n, device="cuda") // page], h, torch.arange(n, device="cuda") % page]  # noqa: E731
                got = [i for i in source[b, h].tolist() if i >= 0]
                if n > keep:
                    newest = [i for i in range(n) if held[b][h][i] > seen[b] - 1 - recent]
                    assert set(newest) <= set(got) and len(set(got)) == keep
                    worth = at(mass)
                    gone = sorted(set(range(n)) - set(got))
                    assert worth[gone].max() <= worth[sorted(set(got) - set(newest))].min()
                held[b][h] = [held[b][h][i] for i in got]
        lens.copy_(new_lens)
        evictions += 1
        check_cache()
    assert evictions >= 2
    cache.check()


@pytest.mark.parametrize("bits", [16, 8])
def test_users_of_one_instruction(bits):
    """One prompt into pages that all users' tables begin with; each user's own tokens behind it, step by step: the attention
    that reads the shared rows once gives what the plain one does."""
    heads, kv_heads, head_dim, page, users, span, steps = 16, 4, 128, 32, 9, 200, 6
    own = 1
    table_pages = span // page + own + 1
    cache = B.KVCache(table_pages * users + 8, kv_heads, head_dim, page_size=page, bits=bits)
    pages = torch.arange(users * table_pages, dtype=torch.int32).view(users, table_pages).flip(1).contiguous().cuda()
    shared_pages = pages[0, :span // page].clone()
    pages[:, :span // page] = shared_pages
    rope, gain = R.angles(span + steps + 1, head_dim), torch.ones(head_dim, device="cuda")
    # the whole pages of the instruction once, its rest (a part of a page) for every user
    whole, rest = span // page * page, span % page
    k, v = rows(span, kv_heads, head_dim, 1), rows(span, kv_heads, head_dim, 2)
    B.kv_append_rmsnorm(cache, B.KVBatch(pages[:1], torch.tensor([whole], dtype=torch.int32, device="cuda"),
                                         torch.tensor([0, whole], dtype=torch.int32, device="cuda")), k[:whole], v[:whole], k_gain=gain, rope=rope)
    lens = torch.full((users,), span, dtype=torch.int32, device="cuda")
    every = torch.arange(users + 1, dtype=torch.int32, device="cuda")
    B.kv_append_rmsnorm(cache, B.KVBatch(pages, lens, every * rest), k[whole:].repeat(users, 1, 1), v[whole:].repeat(users, 1, 1), k_gain=gain, rope=rope)
    batch = B.KVBatch(pages, lens)
    groups = B.KVBatch(shared_pages[None].contiguous(), torch.tensor([span], dtype=torch.int32, device="cuda"),
                       torch.tensor([0, users], dtype=torch.int32, device="cuda"))
    ws = B.alloc_attend_shared_workspace(heads, kv_heads, head_dim, users)
    s = R.Setup.__new__(R.Setup)
    s.kv_heads, s.head_dim, s.page_size, s.bits, s.table = kv_heads, head_dim, page, bits, pages
    s.pools, s.scales = [cache.k, cache.v], [cache.k_scale, cache.v_scale]
    for step in range(steps):
        lens += 1
        q, k, v = (rows(users, n, head_dim, 10 * step + i + 5, size=2.0) for i, n in enumerate((heads, kv_heads, kv_heads)))
        q = B.kv_append_rmsnorm(cache, batch, k, v, q=q, q_gain=gain, k_gain=gain, rope=rope)
        out = B.attend_decode_shared(cache, batch, groups, q, workspace=ws, share_from=0)
        s.lens = lens.tolist()
        want, bound = R.attend(s, q, [1] * users, weight_rounding=2.0 ** -8, query_rounding=2.0 ** -22)
        check(out, want, bound)
        check(B.attend_decode(cache, batch, q), want, bound)
    cache.check()
