"""Plain 64-bit restatement of the cache and attention operators, and the error bounds their results are held to."""
import math

import torch

NAN = float("nan")


def padded(head_dim):
    return (head_dim + 15) // 16 * 16


class Setup:
    """A paged cache with random contents for sequences of the given total lengths, and its 64-bit contents.

    Slots and pages that no sequence uses hold NaN (bf16) or NaN scales (int8): nothing may be read from them into a result.
    `spare`: pages nobody uses.  Page numbers are shuffled.
    """

    def __init__(self, lens, kv_heads, head_dim, page_size, bits, seed=0, spare=3, table_extra=2, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.kv_heads, self.head_dim, self.page_size, self.bits = list(lens), kv_heads, head_dim, page_size, bits
        W = padded(head_dim)
        need = [-(-n // page_size) for n in lens]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        table = torch.full((len(lens), max([1] + need) + table_extra), -7, dtype=torch.int32)  # unused entries: no page
        shape = (self.n_pages, kv_heads, page_size, W)
        used = torch.zeros(self.n_pages, page_size, dtype=torch.bool)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            for p in range(n):
                used[order[at + p].item(), :min(page_size, lens[b] - p * page_size)] = True
            at += n
        self.used = used
        self.pools, self.scales = [], []
        for _ in range(2):
            x = torch.randn(shape, generator=g)
            if bits == 16:
                x[..., head_dim:] = 0
                x[~used[:, None].expand(shape[:3])] = NAN
                self.pools.append(x.to(torch.bfloat16))
                self.scales.append(None)
            else:
                codes = torch.randint(-127, 128, shape, generator=g, dtype=torch.int8)
                codes[..., head_dim:] = 0
                scale = torch.rand(shape[:3], generator=g) * 0.02 + 0.004
                scale[~used[:, None].expand(shape[:3])] = NAN
                self.pools.append(codes)
                self.scales.append(scale)
        self.table = table.to(device)
        self.pools = [p.to(device) for p in self.pools]
        self.scales = [s if s is None else s.to(device) for s in self.scales]
        self.kv_lens = torch.tensor(self.lens, dtype=torch.int32, device=device)

    def cache(self):
        from paper_2402_17764_b200 import binding as B
        return B.KVCache.from_tensors(self.pools[0], self.pools[1], self.head_dim, self.scales[0], self.scales[1])

    def rows(self, which, b, n):
        """The first n keys (0) or values (1) of sequence b in 64 bits: [kv_heads, n, head_dim]."""
        ids = self.table[b, :-(-n // self.page_size)].long()
        x = self.pools[which][ids][..., :self.head_dim].double()
        if self.bits == 8:
            x = x * self.scales[which][ids].double()[..., None]
        return x.transpose(0, 1).reshape(self.kv_heads, -1, self.head_dim)[:, :n]


def attend(setup, q, counts, scale=None, weight_rounding=0.0, query_rounding=0.0):
    """(out, bound): the attention of the new tokens (counts[b] rows of q [T, heads, D] belong to sequence b, at its last
    positions) and how far a result may be from it.

    The bound, per output element, with w_j the weights and A = sum_j w_j |v_j|:
      a score is a dot product of D fp32 terms, scaled: |ds| <= (D + 4) 2^-24 scale sum_i |q_i k_i| (+ an int8 row's scale,
        one more rounding, within the + 4);  exp2 and its argument reduction add 2^-21 relative;
      a kernel that rounds the queries to fixed point, each element by at most query_rounding max_i |q_i|, adds
        scale query_rounding max_i |q_i| sum_i |k_i|;
      every weight is then off by a factor within 1 +- d, d = 2 max_j |ds_j| + 2^-21 + weight_rounding (one rounding of the
        weight to fewer bits, for a kernel that does that), the sums of n terms and the joins by (n + 64) 2^-24 more;
      numerator and denominator together: 2 (d + (n + 64) 2^-24) A, to first order; 1 % on top covers the second;
      the result is rounded to bf16: 2^-8 |out|, and half the smallest subnormal step;
      weights below 2^-126 (the smallest normal number of fp32 and bf16) may count as zero, and so may a weight times an
      int8 row's scale: the largest weight is at least 1 (the reference is never above the maximum), so what is lost is at
      most L 2^-126 max |v| for weights and L 2^-126 127 for weights times scales, together at most L 2^-119 max(1, max |v|).
    """
    T, H, D = q.shape
    G = H // setup.kv_heads
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = torch.zeros(T, H, D, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    at = 0
    for b, n in enumerate(counts):
        L = setup.lens[b]
        if n == 0:
            continue
        x = q[at:at + n].double().reshape(n, setup.kv_heads, G, D).permute(1, 2, 0, 3)  # [kv, G, n, D]
        k, v = setup.rows(0, b, L), setup.rows(1, b, L)
        if L > 0:
            s = scale * torch.einsum("hgnd,hld->hgnl", x, k)
            size = scale * torch.einsum("hgnd,hld->hgnl", x.abs(), k.abs())
            pos = L - n + torch.arange(n, device=q.device)
            hidden = torch.arange(L, device=q.device)[None] > pos[:, None]
            s = s.masked_fill(hidden, -math.inf)
            w = torch.softmax(s, -1).nan_to_num(0.0)  # a row that sees nothing has no weights
            y = torch.einsum("hgnl,hld->hgnd", w, v)
            A = torch.einsum("hgnl,hld->hgnd", w, v.abs())
            worst = size.masked_fill(hidden, 0.0).amax(-1, keepdim=True) * (D + 4) * 2.0 ** -24
            if query_rounding:
                fixed = scale * x.abs().amax(-1)[..., None] * k.abs().sum(-1)[:, None, None]
                worst = worst + query_rounding * fixed.masked_fill(hidden, 0.0).amax(-1, keepdim=True)
            d = 2 * worst + 2.0 ** -21 + weight_rounding + (L + 64) * 2.0 ** -24
            e = 1.01 * 2 * d * A + 2.0 ** -8 * y.abs() + 2.0 ** -134 + L * 2.0 ** -119 * max(1.0, v.abs().nan_to_num(0.0, 0.0).max().item())
            out[at:at + n] = y.permute(2, 0, 1, 3).reshape(n, H, D)
            bound[at:at + n] = e.permute(2, 0, 1, 3).reshape(n, H, D)
        at += n
    return out, bound


def angles(n_pos, head_dim, base=10000.0, device="cuda"):
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * base ** (-2.0 * torch.arange(head_dim // 2, dtype=torch.float64) / head_dim)
    return torch.stack([a.cos(), a.sin()], -1).float().to(device)


def rotate(x, rope, pos, interleaved):
    """(rotated, size) in 64 bits; size = |a c| + |b s| of every element, for the bound."""
    x = x.double()
    c, s = rope[pos].double().unbind(-1)
    c, s = c[:, None], s[:, None]
    half = x.shape[-1] // 2
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    lo, hi = a * c - b * s, b * c + a * s
    zlo, zhi = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    join = (lambda u, w: torch.stack([u, w], -1).flatten(-2)) if interleaved else (lambda u, w: torch.cat([u, w], -1))
    return join(lo, hi), join(zlo, zhi)


def codes(x):
    """(codes, scale) of rows x in 64 bits."""
    beta = x.abs().amax(-1, keepdim=True).clamp(min=1e-5)
    return torch.round(x * 127.0 / beta).clamp(-127, 127).to(torch.int8), (beta[..., 0] / 127.0).float()
