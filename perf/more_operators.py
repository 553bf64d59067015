"""Further operators around the paged key-value cache, as they are measured:

  append   appending to the cache with the RMS norm of every query and key head and the rotary embedding in the same pass, at
           positions of the caller's (a sequence that rows were evicted from holds fewer rows than it has tokens);
  weigh    attention of one new token per sequence that also adds every row's weight to what the row has received so far;
  select   which rows of a sequence and kv head stay in the cache, by the weight they have received and by their age;
  compact  moving the rows that stay to the front;
  shared   attention of one new token per sequence for sequences that begin with the same tokens, whose rows are read once.

A case names one operator ("op"), the heads, the cache's page size and element (16: bf16, 8: int8 codes with one fp32 scale per
token and head) and the lengths of its sequences: every sequence has `past` rows in the cache (shared: behind the shared ones)
and receives `new` ones, both spread over the logarithm of their range by the case's own `mix`.  Heads and widths are those of
the 3B-, 7B-, 13B- and 70B-shaped layers (hidden 3200, 4096, 5120 and 8192), or generic ones of width 64.

`run` computes an operator in its plain form, in 32 bits with elementary torch operations, or, where `own` is true, through
the package's own entry points.
"""
import math
import random

import torch

own = False

EPS = 1e-5  # of the norms


def _case(name, op, heads, kv_heads, head_dim, page, bits, seqs, new, past, mix, interleaved=False, keep=0, recent=0, groups=0, shared=0):
    return {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "bits": bits,
            "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "mix": mix,
            "interleaved": interleaved, "keep": keep, "recent": recent, "groups": groups, "shared": shared}


def listed():
    return [
        # one generated token of a 3B-shaped model with normalised queries and keys: nothing but latency
        _case("append 1 token 3B", "append", 32, 32, 100, 16, 16, 1, (1, 1), (500, 500), 1),
        # a whole prompt of a 70B-shaped model
        _case("append prompt 70B", "append", 64, 8, 128, 64, 16, 1, (4096, 4096), (0, 0), 2),
        # a step of 64 users whose 8-bit caches hold a small part of their conversations
        _case("append step of 64 int8 70B", "append", 64, 8, 128, 32, 8, 64, (1, 1), (8, 60), 3, True),
        # one user, a short context: latency
        _case("weigh 1 user 3B", "weigh", 32, 32, 100, 16, 16, 1, (1, 1), (776, 776), 4),
        # one user, a very long context
        _case("weigh 128k context 70B", "weigh", 64, 8, 128, 64, 16, 1, (1, 1), (131071, 131071), 5),
        # a ragged batch over an 8-bit cache without shared heads
        _case("weigh ragged int8 13B", "weigh", 40, 40, 128, 32, 8, 24, (1, 1), (100, 4095), 6),
        # a user's cache has grown by one page over its budget
        _case("select page over 7B", "select", 32, 32, 128, 16, 16, 1, (1, 1), (2063, 2063), 7, keep=2048, recent=256),
        # long conversations of a batch are cut down
        _case("select long 70B", "select", 64, 8, 128, 64, 16, 16, (1, 1), (6000, 65535), 8, keep=4096, recent=1024),
        # the rows of that one page
        _case("compact page over 7B", "compact", 32, 32, 128, 16, 16, 1, (1, 1), (2063, 2063), 9, keep=2048, recent=256),
        # a batch of prompts is cut down to its budget
        _case("compact batch 70B", "compact", 64, 8, 128, 64, 16, 64, (1, 1), (1500, 8191), 10, keep=1024, recent=128),
        # four samples of one prompt
        _case("shared 4 samples 7B", "shared", 32, 32, 128, 16, 16, 4, (1, 1), (0, 60), 11, groups=1, shared=1000),
        # 64 users of one long instruction
        _case("shared 64 users 70B", "shared", 64, 8, 128, 64, 16, 64, (1, 1), (0, 800), 12, groups=1, shared=16384),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1))


def draw(rng):
    op = rng.choice(["append", "weigh", "select", "compact", "shared"])
    heads, kv_heads, head_dim = rng.choice([(32, 32, 100), (32, 32, 128), (40, 40, 128), (64, 8, 128), (24, 8, 64), (16, 16, 64), (28, 4, 128)])
    page, bits = rng.choice([16, 32, 64, 128]), rng.choice([16, 16, 8])
    kind = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, bits=bits, mix=rng.randrange(1, 1 << 30),
                interleaved=rng.random() < 0.5)
    seqs = _log(rng, 1, 64)
    row = kv_heads * head_dim * bits // 4  # bytes of the keys and values of one token
    if op == "append":
        hi = max(1, _log(rng, 1, 4096) // seqs) if rng.random() < 0.6 else 1
        return _drawn(op, kind, seqs, (max(1, hi // 9), hi), (0, _log(rng, 0, 64 if bits == 8 else 1000)))
    if op == "weigh":
        hi = _log(rng, 1, max(16, min(100000 if seqs < 3 else 8000, 400_000_000 // (row * seqs))))
        return _drawn(op, kind, seqs, (1, 1), (_log(rng, 0, hi), hi))
    if op == "shared":
        groups = min(max(1, seqs // 2), rng.choice([1, 1, 2, 3, 7]))
        shared = _log(rng, 64, min(16384, 120_000_000 // (row * groups)))
        return _drawn(op, kind, seqs, (1, 1), (0, _log(rng, 1, 1000)), groups=groups, shared=shared)
    hi = _log(rng, 40, min(60000, (800_000_000 if op == "compact" else 1_200_000_000) // (row * seqs)))
    keep = _log(rng, 20, min(8192, hi))
    return _drawn(op, kind, seqs, (1, 1), (_log(rng, 1, hi), hi), keep=keep, recent=_log(rng, 0, keep))


def _drawn(op, kind, seqs, new, past, **more):
    case = _case("", op, new=new, past=past, seqs=seqs, **kind, **more)
    del case["name"]
    return case


def _lengths(case):
    """(new, past) of every sequence; the first one has the largest of both, so that a case's size does not hang on `mix`."""
    rng = random.Random(case["mix"])
    new = [_log(rng, case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    past = [_log(rng, case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])]
    new[0], past[0] = case["new_hi"], case["past_hi"]
    return new, past


def _groups(case):
    """Bounds of the groups' sequences, and how many positions each group shares: half to all of `shared`."""
    n, rng = case["groups"], random.Random(case["mix"] + 1)
    return [i * case["seqs"] // n for i in range(n + 1)], [case["shared"] if i == 0 else rng.randint(case["shared"] // 2, case["shared"]) for i in range(n)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, H, Hk, D, ps, B = case["op"], case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["seqs"]
    new, past = _lengths(case)
    whole = [0] * B  # pages that a sequence shares with the others of its group
    if op == "shared":
        bounds, spans = _groups(case)
        for i, span in enumerate(spans):
            for b in range(bounds[i], bounds[i + 1]):
                whole[b] = span // ps
                past[b] += span
    lens = [n + p for n, p in zip(new, past)]
    T, W = sum(new), -(-D // 16) * 16
    own_pages = [-(-n // ps) - w for n, w in zip(lens, whole)]
    n_pages = sum(own_pages) + (sum(span // ps for span in spans) if op == "shared" else 0) + 3  # a pool in use has free pages
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(B, max(n + w for n, w in zip(own_pages, whole)), dtype=torch.int32, device="cuda")
    at = 0
    if op == "shared":
        for i, span in enumerate(spans):
            table[bounds[i]:bounds[i + 1], :span // ps] = order[at:at + span // ps]
            at += span // ps
    for b, n in enumerate(own_pages):
        table[b, whole[b]:whole[b] + n] = order[at:at + n]
        at += n
    shape = (n_pages, Hk, ps, W)

    def tensor(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    s = {"case": case, "table": table, "T": T, "max_len": max(lens), "lens": tensor(lens),
         "cu": tensor([sum(new[:i]) for i in range(B + 1)])}

    def pool():
        if op == "select":  # (looks at no key or value)
            return torch.empty(shape, dtype=torch.bfloat16 if case["bits"] == 16 else torch.int8, device="cuda"), \
                None if case["bits"] == 16 else torch.empty(shape[:3], device="cuda")
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
        x[..., D:] = 0
        if case["bits"] == 16:
            return x, None
        big = x.abs().amax(-1).float().clamp(min=1e-5)
        codes = torch.empty(shape, dtype=torch.int8, device="cuda")
        codes.copy_((x.float() * (127.0 / big)[..., None]).round_())
        return codes, big / 127.0

    s["k"], s["k_scale"] = pool()
    s["v"], s["v_scale"] = pool()
    if op != "shared":
        # what rows have received: of all sizes, some of them nothing at all
        s["mass"] = torch.exp(2.0 * torch.randn(shape[:3], generator=g, device="cuda"))
        s["mass"].mul_(torch.rand(shape[:3], generator=g, device="cuda") > 0.05)
        if op == "weigh":
            s["mass"] /= max(lens)  # (of the size of what one token gives)
        s["pos"] = torch.zeros(shape[:3], dtype=torch.int32, device="cuda")
    if op in ("select", "compact"):
        # positions with gaps (of rows evicted earlier); behind an earlier eviction the rows up to the budget stand in any order
        L = s["max_len"]
        i, last = torch.arange(L, device="cuda"), s["lens"].long()[:, None, None] - 1
        pos = 2 * i + torch.randint(0, 2, (B, Hk, L), generator=g, device="cuda")
        mixed = torch.rand(B, Hk, L, generator=g, device="cuda").masked_fill_(i >= torch.clamp(last, max=case["keep"]), 2.0) + (i >= case["keep"])
        pos = pos.gather(-1, torch.sort(mixed, dim=-1, stable=True).indices)
        s["pos"].view(-1)[_row_numbers(s)[i.expand(B, Hk, L) <= last]] = pos[i.expand(B, Hk, L) <= last].to(torch.int32)
        if op == "compact":
            s["source"] = _plain_select(s)[0]
        else:
            s["source"] = torch.empty(B, Hk, case["keep"], dtype=torch.int32, device="cuda")
            s["new_lens"] = torch.empty(B, dtype=torch.int32, device="cuda")
    if op == "append":
        # what the fused q/k/v projection of a layer wrote: one row per token
        qkv = 3.0 * torch.randn(T, (H + 2 * Hk) * D, generator=g, device="cuda", dtype=torch.bfloat16)
        s["q"] = qkv[:, :H * D].unflatten(1, (H, D))
        s["new_k"] = qkv[:, H * D:(H + Hk) * D].unflatten(1, (Hk, D))
        s["new_v"] = qkv[:, (H + Hk) * D:].unflatten(1, (Hk, D))
        s["q_gain"], s["k_gain"] = 1.0 + 0.2 * torch.randn(2, D, generator=g, device="cuda")
        evicted = torch.randint(0, 1000, (B,), generator=g, device="cuda")
        b, _, slot = _places(s)
        s["positions"] = (slot + evicted[b]).to(torch.int32)
        angle = torch.arange(max(lens) + 1000, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        s["q_out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
    if op in ("weigh", "shared"):
        s["q"] = (1.5 * torch.randn(T, H, D, generator=g, device="cuda")).to(torch.bfloat16)
    if op == "shared":
        s["bounds"], s["spans"] = tensor(bounds), tensor(spans)
        s["most"], s["span"] = max(y - x for x, y in zip(bounds, bounds[1:])), max(x // ps * ps for x in spans)
        s["own_len"] = max(n - w * ps for n, w in zip(lens, whole))
    if own:
        from paper_2402_17764_b200 import binding
        s["cache"] = binding.KVCache.from_tensors(s["k"], s["v"], D, k_scale=s["k_scale"], v_scale=s["v_scale"])
        s["batch"] = binding.KVBatch(table, s["lens"], cu_tokens=s["cu"] if op == "append" else None)
        if op != "shared":
            s["marks"] = binding.KVMarks.from_tensors(s["cache"], s["mass"], s["pos"])
        if op == "weigh":
            s["out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
            s["workspace"] = binding.alloc_attend_weigh_workspace(H, Hk, D, case["bits"], B, sum(lens))
        if op == "shared":
            s["groups"] = binding.KVBatch(table[s["bounds"][:-1].long()], s["spans"], cu_tokens=s["bounds"])
            s["out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
            s["workspace"] = binding.alloc_attend_shared_workspace(H, Hk, D, B)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------


def _places(s):
    """Of every new token: its sequence, its number in it and the row of the sequence that it is stored at."""
    t = torch.arange(s["T"], device="cuda")
    cu = s["cu"].long()
    b = torch.searchsorted(cu[1:], t, right=True)
    i = t - cu[b]
    return b, i, s["lens"].long()[b] - (cu[b + 1] - cu[b]) + i


def _row_numbers(s):
    """Of every sequence, kv head and row of it: the row's number in the pools, [sequences, heads, longest length]."""
    ps, Hk = s["case"]["page"], s["case"]["kv_heads"]
    i = torch.arange(s["max_len"], device="cuda")
    page = s["table"].long()[:, i // ps]
    return (page[:, None] * Hk + torch.arange(Hk, device="cuda")[:, None]) * ps + i % ps


def _rotate(x, cs, interleaved):
    cs = cs.to(x.dtype)
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    half = x.shape[-1] // 2
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    lo, hi = a * c - b * n, b * c + a * n
    return torch.stack([lo, hi], -1).flatten(-2) if interleaved else torch.cat([lo, hi], -1)


def _over_rms(x):
    """1 / root mean square of every head of every token."""
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _codes(x, factor):
    """8-bit codes of the rows of factor x, and their scales: symmetric, by the largest magnitude of a token's head.  The factor
    of a row cancels out of its codes.  In 64 bits, with one division: values may lie right between two codes."""
    big = torch.maximum(x.abs().amax(-1, keepdim=True), 1e-5 / factor)
    return torch.round(x * 127 / big).clamp(-127, 127).to(torch.int8), (factor * big / 127)[..., 0].float()


def _plain_append(s):
    case, D = s["case"], s["case"]["head_dim"]
    b, _, slot = _places(s)
    page, at = s["table"].long()[b, slot // case["page"]], slot % case["page"]
    cs = s["rope"][s["positions"].long()]
    q = s["q"].float()
    s["q_out"].copy_(_rotate(q * _over_rms(q) * s["q_gain"], cs, case["interleaved"]))
    if case["bits"] == 8:
        k, v = s["new_k"].double(), s["new_v"].double()
        k, s["k_scale"][page, :, at] = _codes(_rotate(k * s["k_gain"].double(), cs, case["interleaved"]), _over_rms(k))
        v, s["v_scale"][page, :, at] = _codes(v, torch.ones_like(v[..., :1]))
    else:
        k, v = s["new_k"].float(), s["new_v"]
        k = _rotate(k * _over_rms(k) * s["k_gain"], cs, case["interleaved"])
    s["k"][page, :, at, :D] = k.to(s["k"].dtype)
    s["v"][page, :, at, :D] = v.to(s["v"].dtype)
    s["mass"][page, :, at] = 0
    s["pos"][page, :, at] = s["positions"][:, None]


def _rows(pool, scale, s, table, first, count):
    """Rows first .. first + count of every row of the page table in 32 bits: [sequences, heads, count, head width]."""
    ps = s["case"]["page"]
    i = first[:, None] + torch.arange(count, device="cuda")
    page = table.long().gather(1, (i // ps).clamp(max=table.shape[1] - 1))
    x = pool.transpose(1, 2)[page, i % ps][..., :s["case"]["head_dim"]].float()  # [sequences, count, heads, width]
    if scale is not None:
        x *= scale.transpose(1, 2)[page, i % ps][..., None]
    return x.transpose(1, 2)


def _scores(q, k, hidden, D):
    """Scores of queries [sequences, heads, queries, width]; -infinity where hidden, [sequences, heads or 1, queries or 1, keys]."""
    return torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).masked_fill_(hidden, -math.inf)


def _plain_weigh(s):
    case = s["case"]
    B, H, Hk, D = case["seqs"], case["heads"], case["kv_heads"], case["head_dim"]
    lens, start = s["lens"].long(), torch.zeros(B, dtype=torch.int64, device="cuda")
    hidden = torch.arange(s["max_len"], device="cuda") >= lens[:, None]
    x = _scores(s["q"].float().view(B, Hk, H // Hk, D), _rows(s["k"], s["k_scale"], s, s["table"], start, s["max_len"]), hidden[:, None, None], D)
    p = torch.softmax(x, -1)
    y = torch.matmul(p, _rows(s["v"], s["v_scale"], s, s["table"], start, s["max_len"]))
    seen = (~hidden)[:, None].expand(B, Hk, -1)
    s["mass"].view(-1).index_add_(0, _row_numbers(s)[seen], p.sum(2)[seen])
    return {"out": y.reshape(B, H, D).to(torch.bfloat16), "mass": s["mass"]}


def _plain_select(s):
    case, keep = s["case"], s["case"]["keep"]
    rows, lens = _row_numbers(s), s["lens"].long()[:, None, None]
    i = torch.arange(s["max_len"], device="cuda")
    pos = s["pos"].view(-1)[rows]
    newest = pos.gather(-1, (lens - 1).expand(*pos.shape[:2], 1))
    worth = s["mass"].view(-1)[rows].masked_fill(pos > newest - case["recent"], math.inf).masked_fill(i >= lens, -1.0)
    best = torch.sort(worth, dim=-1, descending=True, stable=True).indices[..., :keep]
    stays = torch.zeros_like(worth, dtype=torch.bool).scatter_(-1, best, True) & (i < lens)
    if keep > s["max_len"]:
        i = torch.arange(keep, device="cuda")
        stays = torch.nn.functional.pad(stays, (0, keep - s["max_len"]))
    hole, mover = ~stays[..., :keep], stays[..., keep:]
    # the j-th row that moves goes to the j-th hole
    source = torch.where(hole, -1, i[:keep])
    from_b, from_h, from_i = mover.nonzero(as_tuple=True)
    rank = mover.cumsum(-1)[from_b, from_h, from_i]
    places = torch.full((*hole.shape[:2], keep + 1), -1, dtype=torch.int64, device="cuda")
    places[from_b, from_h, rank] = from_i + keep
    source = torch.where(hole, places.gather(-1, hole.cumsum(-1)), source)
    return source.to(torch.int32), torch.clamp(s["lens"], max=keep)


def _plain_compact(s):
    case, keep, rows = s["case"], s["case"]["keep"], _row_numbers(s)
    source = s["source"].long()
    to = torch.arange(keep, device="cuda").expand_as(source)
    moves = (source >= 0) & (source != to)
    b, h, _ = moves.nonzero(as_tuple=True)
    src, dst = rows[b, h, source[moves]], rows[b, h, to[moves]]
    for name in ("k", "v", "k_scale", "v_scale", "mass", "pos"):
        if s[name] is not None:
            x = s[name].view(-1, s[name].shape[-1]) if name in ("k", "v") else s[name].view(-1)
            x[dst] = x[src]


def _plain_shared(s):
    """The scores of the shared rows group by group, of the others sequence by sequence, and one softmax over both."""
    case = s["case"]
    B, H, Hk, D, ps, n = case["seqs"], case["heads"], case["kv_heads"], case["head_dim"], case["page"], s["most"]
    G, lens, bounds = H // Hk, s["lens"].long(), s["bounds"].long()
    whole = s["spans"].long() // ps * ps
    group = torch.searchsorted(bounds[1:], torch.arange(B, device="cuda"), right=True)
    place = torch.arange(B, device="cuda") - bounds[group]
    member = (bounds[:-1, None] + torch.arange(n, device="cuda")).clamp(max=B - 1)
    q = s["q"].float().view(B, Hk, G, D)
    zero = torch.zeros_like(whole)
    k, v = (_rows(s[x], s[x + "_scale"], s, s["table"][bounds[:-1]], zero, s["span"]) for x in "kv")
    hidden = torch.arange(s["span"], device="cuda") >= whole[:, None]
    x = _scores(q[member].transpose(1, 2).reshape(len(whole), Hk, n * G, D), k, hidden[:, None, None], D).view(len(whole), Hk, n, G, -1)
    own_k, own_v = (_rows(s[x], s[x + "_scale"], s, s["table"], whole[group], s["own_len"]) for x in "kv")
    hidden = torch.arange(s["own_len"], device="cuda") >= (lens - whole[group])[:, None]
    own_x = _scores(q, own_k, hidden[:, None, None], D)
    top = torch.maximum(x.amax(-1).transpose(1, 2)[group, place], own_x.amax(-1))  # [B, Hk, G]
    own_p = torch.exp(own_x - top[..., None])
    p = torch.exp(x.sub_(top[member].transpose(1, 2)[..., None]))
    total = p.sum(-1).transpose(1, 2)[group, place] + own_p.sum(-1)
    y = torch.matmul(p.view(len(whole), Hk, n * G, -1), v).view(len(whole), Hk, n, G, D).transpose(1, 2)[group, place]
    return ((y + torch.matmul(own_p, own_v)) / total[..., None]).reshape(B, H, D).to(torch.bfloat16)


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        from paper_2402_17764_b200 import binding
    if op == "weigh":
        if own:
            out = binding.attend_decode_weigh(s["cache"], s["batch"], s["marks"], s["q"], out=s["out"], workspace=s["workspace"])
            return {"out": out, "mass": s["mass"]}
        return _plain_weigh(s)
    if op == "shared":
        if own:
            return binding.attend_decode_shared(s["cache"], s["batch"], s["groups"], s["q"], out=s["out"], workspace=s["workspace"])
        return _plain_shared(s)
    if op == "select":
        if own:
            return binding.kv_select(s["cache"], s["batch"], s["marks"], case["keep"], case["recent"], source=s["source"], new_lens=s["new_lens"])
        return _plain_select(s)
    if op == "append":
        if own:
            binding.kv_append_rmsnorm(s["cache"], s["batch"], s["new_k"], s["new_v"], q=s["q"], q_gain=s["q_gain"], k_gain=s["k_gain"],
                                      norm_eps=EPS, rope=s["rope"], interleaved=case["interleaved"], positions=s["positions"],
                                      marks=s["marks"], q_out=s["q_out"])
        else:
            _plain_append(s)
    elif own:
        binding.kv_compact(s["cache"], s["batch"], s["source"], s["marks"])
    else:
        _plain_compact(s)
    k, v = s["k"], s["v"]
    if case["bits"] == 8:  # what the codes stand for
        k, v = k * s["k_scale"][..., None], v * s["v_scale"][..., None]
    out = {"k": k, "v": v, "mass": s["mass"], "pos": s["pos"]}
    return {**out, "q": s["q_out"]} if op == "append" else out


def work(case):
    op, B, H, Hk, D, keep = case["op"], case["seqs"], case["heads"], case["kv_heads"], case["head_dim"], case["keep"]
    new, past = _lengths(case)
    lens, T = [n + p for n, p in zip(new, past)], sum(new)
    kv = 2 * Hk * (D * case["bits"] // 8 + (4 if case["bits"] == 8 else 0))  # a token's keys and values in the cache
    if op == "append":
        return {"bytes": T * (4 * H * D + 4 * Hk * D + kv + 8 * Hk + 4) + min(T, max(lens) + 1000) * 4 * D, "flops": 7 * T * (H + Hk) * D}
    if op == "weigh":
        return {"bytes": T * 4 * H * D + sum(lens) * (kv + 8 * Hk), "flops": 4 * H * D * sum(lens)}
    if op == "select":  # mass and position of every row; the marks of rows of shorter sequences are not looked at
        return {"bytes": 8 * Hk * sum(n for n in lens if n > keep) + 4 * B * Hk * keep, "flops": 2 * Hk * sum(lens)}
    if op == "compact":  # about keep (n - keep) / n of a sequence's rows move
        return {"bytes": 4 * B * Hk * keep + 2 * (kv + 8 * Hk) * sum(keep * (n - keep) // n for n in lens if n > keep), "flops": 0}
    bounds, spans = _groups(case)
    many = sum((y - x) * w for x, y, w in zip(bounds, bounds[1:], spans))
    return {"bytes": T * 4 * H * D + (sum(spans) + sum(lens)) * kv, "flops": 4 * H * D * (many + sum(lens))}


# ---- 64 bits -------------------------------------------------------------------------------------------


def _history(s, b, h, n):
    """Keys and values of the first n rows of sequence b and kv head h."""
    case = s["case"]
    rows = s["table"][b, :-(-n // case["page"])].long()
    got = []
    for x in "kv":
        y = s[x][rows, h].flatten(0, 1)[:n, :case["head_dim"]].double()
        got.append(y if case["bits"] == 16 else y * s[x + "_scale"][rows, h].flatten()[:n, None].double())
    return rows, got


def exact(case, seed):
    s = prepare(case, seed)
    op, H, Hk, D, ps, B = case["op"], case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["seqs"]
    new, past = _lengths(case)
    lens = s["lens"].tolist()
    if op == "select":
        return None  # whole numbers
    if op in ("weigh", "shared"):
        y = torch.empty(B, H, D, dtype=torch.float64, device="cuda")
        mass = s["mass"].double() if op == "weigh" else None
        for b in range(B):
            for h in range(Hk):
                rows, (k, v) = _history(s, b, h, lens[b])
                q = s["q"][b, h * (H // Hk):(h + 1) * (H // Hk)].double()
                p = torch.softmax(q @ k.T / math.sqrt(D), -1)
                y[b, h * (H // Hk):(h + 1) * (H // Hk)] = p @ v
                if op == "weigh":
                    got = torch.nn.functional.pad(p.sum(0), (0, len(rows) * ps - lens[b])).view(len(rows), ps)
                    mass[rows, h] += got
        return y if op == "shared" else {"out": y, "mass": mass}
    scale = {n: s[n + "_scale"].double() if case["bits"] == 8 else None for n in "kv"}
    pools = {n: s[n].double() * (scale[n][..., None] if case["bits"] == 8 else 1.0) for n in "kv"}
    mass = s["mass"].double()
    if op == "compact":
        for b, n in enumerate(lens):
            table = s["table"][b].long()
            for h in range(Hk):
                to = torch.arange(case["keep"], device="cuda")
                go = (s["source"][b, h] >= 0) & (s["source"][b, h] != to)
                to, src = to[go], s["source"][b, h][go].long()
                for x in (pools["k"], pools["v"], mass):
                    x[table[to // ps], h, to % ps] = x[table[src // ps], h, src % ps]
        return {"k": pools["k"], "v": pools["v"], "mass": mass, "pos": None}
    half, q_out, at = D // 2, [], 0
    for b, (n, p) in enumerate(zip(new, past)):
        turn = torch.complex(*s["rope"][s["positions"][at:at + n].long()].double().unbind(-1))[:, None]

        def normed(x, gain):
            x = x[at:at + n].double()
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS) * gain.double()
            pairs = x.unflatten(-1, (half, 2)) if case["interleaved"] else x.unflatten(-1, (2, half)).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            return y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)

        q_out.append(normed(s["q"], s["q_gain"]))
        slot = torch.arange(p, p + n, device="cuda")
        page = s["table"][b].long()[slot // ps]
        for name, x in (("k", normed(s["new_k"], s["k_gain"])), ("v", s["new_v"][at:at + n].double())):
            if case["bits"] == 8:
                big = x.abs().amax(-1, keepdim=True).clamp(min=1e-5)
                x = torch.round(127 * x / big).clamp(-127, 127) * big / 127
            pools[name][page, :, slot % ps, :D] = x
        mass[page, :, slot % ps] = 0
        at += n
    return {"k": pools["k"], "v": pools["v"], "mass": mass, "pos": None, "q": torch.cat(q_out)}
