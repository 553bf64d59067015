"""The operators around the projections of a decoder layer, as they are measured: a paged key-value cache that is
appended to (with the rotary embedding applied on the way), the attention of one new token per sequence over it, and the
attention of the tokens of prompts or prompt chunks over it.

A case names one operator ("op"), the heads, the cache's page size and element (16: bf16, 8: int8 codes with one fp32
scale per token and head) and the lengths of its sequences: every sequence has `past` tokens in the cache and receives
`new` ones, both spread over the logarithm of their range by the case's own `mix`.  Heads and widths are those of the
3B-, 7B-, 13B- and 70B-shaped layers (hidden 3200, 4096, 5120 and 8192), or generic ones of width 64.

`run` computes an operator in its plain form, in 32 bits with elementary torch operations, or, where `own` is true, through
the package's own entry points.
"""
import math
import random

import torch

own = False

WIDTH = {100: 112, 128: 128, 64: 64, 80: 80, 96: 96}  # elements of a cache row: the head padded to 16 elements


def _case(name, op, heads, kv_heads, head_dim, page, bits, seqs, new, past, mix, interleaved=False):
    return {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "bits": bits,
            "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1], "mix": mix,
            "interleaved": interleaved}


def listed():
    return [
        # one generated token of a 3B-shaped model: nothing but latency
        _case("append 1 token 3B", "append", 32, 32, 100, 16, 16, 1, (1, 1), (500, 500), 1),
        # one generated token of each of 64 users of a 70B-shaped model
        _case("append step of 64 70B", "append", 64, 8, 128, 64, 16, 64, (1, 1), (100, 4000), 2),
        # a whole prompt of a 70B-shaped model
        _case("append prompt 70B", "append", 64, 8, 128, 64, 16, 1, (4096, 4096), (0, 0), 3),
        # several prompts of odd lengths into an 8-bit cache, pairs interleaved as in some checkpoints
        _case("append ragged int8 13B", "append", 40, 40, 128, 32, 8, 7, (1, 1500), (0, 0), 4, True),
        # one user, a short context: latency
        _case("decode 1 user 3B", "decode", 32, 32, 100, 16, 16, 1, (1, 1), (776, 776), 5),
        # one user, a very long context
        _case("decode 128k context 70B", "decode", 64, 8, 128, 64, 16, 1, (1, 1), (131071, 131071), 6),
        # a ragged batch without shared heads
        _case("decode ragged 7B", "decode", 32, 32, 128, 16, 16, 32, (1, 1), (0, 4095), 7),
        # a large batch over an 8-bit cache with shared heads
        _case("decode batch int8 70B", "decode", 64, 8, 128, 32, 8, 128, (1, 1), (256, 8191), 8),
        # a short chunk behind a short context: latency
        _case("prompt chunk 3B", "prompt", 32, 32, 100, 16, 16, 1, (37, 37), (411, 411), 9),
        # one long prompt
        _case("prompt 8k 7B", "prompt", 32, 32, 128, 64, 16, 1, (8192, 8192), (0, 0), 10),
        # prompts of odd lengths, batched
        _case("prompt ragged 13B", "prompt", 40, 40, 128, 16, 16, 6, (1, 2047), (0, 0), 11),
        # turns of long conversations over an 8-bit cache
        _case("prompt extend int8 70B", "prompt", 64, 8, 128, 64, 8, 4, (64, 512), (2000, 12000), 12),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1))


def draw(rng):
    op = rng.choice(["append", "decode", "prompt"])
    heads, kv_heads, head_dim = rng.choice([(32, 32, 100), (32, 32, 128), (40, 40, 128), (64, 8, 128), (24, 8, 64), (16, 16, 64), (28, 4, 128)])
    page, bits = rng.choice([16, 32, 64, 128]), rng.choice([16, 16, 8])
    mix, interleaved = rng.randrange(1, 1 << 30), rng.random() < 0.5
    if op == "append":
        seqs = _log(rng, 1, 128)
        hi = max(1, _log(rng, 1, 4096) // seqs) if rng.random() < 0.6 else 1
        past = (0, _log(rng, 0, 64 if bits == 8 else 2000))
        return _without_name(op, heads, kv_heads, head_dim, page, bits, seqs, (max(1, hi // 9), hi), past, mix, interleaved)
    row = kv_heads * head_dim * bits // 4  # bytes of the keys and values of one token
    if op == "decode":
        seqs = _log(rng, 1, 128)
        longest = max(16, min(100000 if seqs < 3 else 8000, 400_000_000 // (row * seqs)))
        hi = _log(rng, 1, longest)
        return _without_name(op, heads, kv_heads, head_dim, page, bits, seqs, (1, 1), (_log(rng, 0, hi), hi), mix, interleaved)
    seqs = _log(rng, 1, 8)
    hi = _log(rng, 1, 4000 // seqs)
    past = _log(rng, 0, 12000)
    most = 60_000_000 // (heads * seqs)  # scores of one head and sequence
    past = min(past, max(0, most // hi - hi))
    return _without_name(op, heads, kv_heads, head_dim, page, bits, seqs, (max(1, hi // 7), hi), (past // 2, past), mix, interleaved)


def _without_name(*args):
    case = _case("", *args)
    del case["name"]
    return case


def _lengths(case):
    """(new, past) of every sequence; the first one has the largest of both, so that a case's size does not hang on `mix`."""
    rng = random.Random(case["mix"])
    new = [_log(rng, case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    past = [_log(rng, case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])]
    new[0], past[0] = case["new_hi"], case["past_hi"]
    return new, past


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, Hk, D, ps, B = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["seqs"]
    new, past = _lengths(case)
    lens = [n + p for n, p in zip(new, past)]
    T, W = sum(new), WIDTH[D]
    pages = [-(-n // ps) for n in lens]
    n_pages = sum(pages) + 3  # a pool in use has pages of others, and free ones
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(B, max(pages), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, Hk, ps, W)
    s = {"case": case, "table": table, "T": T, "max_new": max(new), "max_len": max(lens),
         "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "cu": torch.tensor([sum(new[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")}

    def pool():
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
    if case["op"] == "append":
        # what the fused q/k/v projection of a layer wrote: one row per token
        qkv = torch.randn(T, (H + 2 * Hk) * D, generator=g, device="cuda", dtype=torch.bfloat16)
        s["q"] = qkv[:, :H * D].unflatten(1, (H, D))
        s["new_k"] = qkv[:, H * D:(H + Hk) * D].unflatten(1, (Hk, D))
        s["new_v"] = qkv[:, (H + Hk) * D:].unflatten(1, (Hk, D))
        angle = torch.arange(max(lens), device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        s["q_out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
    else:
        s["q"] = (1.5 * torch.randn(T, H, D, generator=g, device="cuda")).to(torch.bfloat16)
    if own:
        from paper_2402_17764_b200 import binding
        s["cache"] = binding.KVCache.from_tensors(s["k"], s["v"], D, k_scale=s["k_scale"], v_scale=s["v_scale"])
        s["batch"] = binding.KVBatch(table, s["lens"], cu_tokens=None if case["op"] == "decode" else s["cu"])
        if case["op"] != "append":
            s["out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda")
            s["workspace"] = binding.alloc_attend_workspace(H, Hk, D, prompt=case["op"] == "prompt")
    return s


# ---- the plain forms -----------------------------------------------------------------------------------


def _places(s):
    """Of every new token: its sequence, its number in it and its position."""
    t = torch.arange(s["T"], device="cuda")
    cu = s["cu"].long()
    b = torch.searchsorted(cu[1:], t, right=True)
    i = t - cu[b]
    return b, i, s["lens"].long()[b] - (cu[b + 1] - cu[b]) + i


def _rotate(x, cs, interleaved, dtype=torch.float32):
    x, cs = x.to(dtype), cs.to(dtype)
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    half = x.shape[-1] // 2
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    lo, hi = a * c - b * n, b * c + a * n
    return torch.stack([lo, hi], -1).flatten(-2) if interleaved else torch.cat([lo, hi], -1)


def _codes(x):
    """8-bit codes of the rows of x, and their scales: symmetric, by the largest magnitude of a token's head.  In 64 bits,
    with one division: bf16 values often lie right between two codes, and 32 bits would send them either way."""
    big = x.abs().amax(-1).clamp(min=1e-5)
    return torch.round(x * 127 / big[..., None]).clamp(-127, 127).to(torch.int8), (big / 127).float()


def _plain_append(s):
    case, D = s["case"], s["case"]["head_dim"]
    b, _, pos = _places(s)
    page = s["table"].long()[b, pos // case["page"]]
    slot = pos % case["page"]
    cs = s["rope"][pos]
    s["q_out"].copy_(_rotate(s["q"], cs, case["interleaved"]))
    wide = torch.float64 if case["bits"] == 8 else torch.float32
    k, v = _rotate(s["new_k"], cs, case["interleaved"], wide), s["new_v"].to(wide)
    if case["bits"] == 8:
        k, s["k_scale"][page, :, slot] = _codes(k)
        v, s["v_scale"][page, :, slot] = _codes(v)
    s["k"][page, :, slot, :D] = k.to(s["k"].dtype)
    s["v"][page, :, slot, :D] = v.to(s["v"].dtype)


def _rows(pool, scale, s):
    """The cache rows of every sequence in order, in 32 bits: [sequences, heads, length, head width]."""
    table, D = s["table"].long(), s["case"]["head_dim"]
    x = pool[table][..., :D].float()
    if scale is not None:
        x *= scale[table][..., None]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :s["max_len"]]


def _plain_attend(s):
    """Softmax attention over the cached keys at or before each token's own position."""
    case, N = s["case"], s["max_new"]
    H, Hk, D = case["heads"], case["kv_heads"], case["head_dim"]
    B, G = case["seqs"], H // Hk
    cu, lens = s["cu"].long(), s["lens"].long()
    i = torch.arange(N, device="cuda")
    q = s["q"][(cu[:-1, None] + i).clamp(max=s["T"] - 1)].float()  # [B, N, H, D], rows past a sequence's own are unused
    q = q.view(B, N, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * N, D)
    x = torch.matmul(q, _rows(s["k"], s["k_scale"], s).transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(B, Hk, G, N, -1)
    last = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + i
    seen = torch.arange(x.shape[-1], device="cuda") <= torch.minimum(last, lens[:, None] - 1)[..., None]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True)).exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x.view(B, Hk, G * N, -1), _rows(s["v"], s["v_scale"], s)).view(B, Hk, G, N, D).div_(total)
    b, n, _ = _places(s)
    return y.permute(0, 3, 1, 2, 4).reshape(B, N, H, D)[b, n].to(torch.bfloat16)


def run(state):
    s, case = state, state["case"]
    if case["op"] == "append":
        if own:
            from paper_2402_17764_b200 import binding
            binding.kv_append(s["cache"], s["batch"], s["new_k"], s["new_v"], q=s["q"], rope=s["rope"], q_out=s["q_out"],
                              interleaved=case["interleaved"])
        else:
            _plain_append(s)
        k, v = s["k"], s["v"]
        if case["bits"] == 8:  # what the codes stand for
            k, v = k * s["k_scale"][..., None], v * s["v_scale"][..., None]
        return {"q": s["q_out"], "k": k, "v": v}
    if own:
        from paper_2402_17764_b200 import binding
        attend = binding.attend_decode if case["op"] == "decode" else binding.attend_prompt
        return attend(s["cache"], s["batch"], s["q"], out=s["out"], workspace=s["workspace"])
    return _plain_attend(s)


def work(case):
    H, Hk, D = case["heads"], case["kv_heads"], case["head_dim"]
    new, past = _lengths(case)
    T, total = sum(new), sum(new) + sum(past)
    kv = 2 * Hk * (D * case["bits"] // 8 + (4 if case["bits"] == 8 else 0))  # a token's keys and values in the cache
    if case["op"] == "append":
        positions = max(n + p for n, p in zip(new, past)) - min(past)
        return {"bytes": T * (4 * H * D + 4 * Hk * D + kv) + min(T, positions) * 4 * D, "flops": 3 * T * (H + Hk) * D}
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(new, past))
    return {"bytes": T * 4 * H * D + total * kv, "flops": 4 * H * D * pairs}


# ---- 64 bits -------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    H, Hk, D, ps = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    new, past = _lengths(case)
    scale = {n: s[n + "_scale"].double() if case["bits"] == 8 else None for n in "kv"}
    if case["op"] == "append":
        half, q_out, at = D // 2, [], 0
        pools = {n: s[n].double() * (scale[n][..., None] if case["bits"] == 8 else 1.0) for n in "kv"}
        for b, (n, p) in enumerate(zip(new, past)):
            pos = torch.arange(p, p + n, device="cuda")
            turn = torch.complex(*s["rope"][pos].double().unbind(-1))[:, None]

            def rotated(x):
                x = x[at:at + n].double()
                pairs = x.unflatten(-1, (half, 2)) if case["interleaved"] else x.unflatten(-1, (2, half)).transpose(-1, -2)
                y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
                return y.flatten(-2) if case["interleaved"] else y.transpose(-1, -2).flatten(-2)

            q_out.append(rotated(s["q"]))
            for name, x in (("k", rotated(s["new_k"])), ("v", s["new_v"][at:at + n].double())):
                if case["bits"] == 8:
                    big = x.abs().amax(-1, keepdim=True).clamp(min=1e-5)
                    x = torch.round(127 * x / big).clamp(-127, 127) * big / 127
                pools[name][s["table"][b].long()[pos // ps], :, pos % ps, :D] = x
            at += n
        return {"q": torch.cat(q_out), "k": pools["k"], "v": pools["v"]}
    y, at = torch.empty(s["T"], H, D, dtype=torch.float64, device="cuda"), 0
    for b, (n, p) in enumerate(zip(new, past)):
        rows = s["table"][b, :-(-(n + p) // ps)].long()
        for h in range(Hk):
            k, v = (s[x][rows, h, :, :D].double() * (scale[x][rows, h][..., None] if case["bits"] == 8 else 1.0) for x in "kv")
            k, v = k.flatten(0, 1)[:n + p], v.flatten(0, 1)[:n + p]
            for first in range(0, n, 1024):
                rest = min(1024, n - first)
                reach = p + first + rest
                for j in range(h * (H // Hk), (h + 1) * (H // Hk)):
                    x = s["q"][at + first:at + first + rest, j].double() @ k[:reach].T / math.sqrt(D)
                    later = torch.arange(reach, device="cuda") > torch.arange(p + first, reach, device="cuda")[:, None]
                    y[at + first:at + first + rest, j] = torch.softmax(x.masked_fill(later, -math.inf), -1) @ v[:reach]
        at += n
    return y
