"""Plain 64-bit forms of the head norms and of the 8-bit rows, and a paged 8-bit cache with its host copy, for the tests."""
import random

import torch

import _paged_reference as R
from paper_2512_04857_b200 import lar

DEV = "cuda:0"


def norm(x, kind, w, b, eps):
    """x [T, H, d], w and b [d] or [H, d] or None -> fp64."""
    x = x.double()
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    y = y if w is None else y * w.double()
    return y if b is None else y + b.double()


def norm_tolerance(x, kind, w, b, eps):
    """|fp32 norm - norm| before the last rounding.  Sums of d terms: d 2^-24 of their magnitudes.  The mean is off by d 2^-24 mean|x|; the squares'
    sum by d 2^-24 of itself (and through the mean by less), its root by half of that, rsqrtf by 2 units in the last place (2^-22);
    subtraction, three products and the bias round once each."""
    d = x.shape[-1]
    x = x.double()
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    f = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    off = d * 2.0 ** -24 * x.abs().mean(-1, keepdim=True) if kind == "layer" else 0.0
    y = ((x - mean) * f).abs()
    e = y * (d * 2.0 ** -24 + 2.0 ** -22 + 5 * 2.0 ** -24) + off * f * (1 + y)
    if w is not None:
        e, y = e * w.double().abs(), y * w.double().abs()
    if b is not None:
        e = e + 2.0 ** -24 * (y + b.double().abs())
    return e


def rotated(y, tol, pos, axes, theta, interleaved, restart):
    """The rotation of y (fp64, known to tol) and the tolerance of the fp32 one."""
    ref = R.rotate(y, pos, axes, theta, interleaved, restart)
    return ref, R.partner_sum(tol, interleaved) + R.rotation_tolerance(torch.float32, ref, y, interleaved)


def rounded(ref, tol, dtype):
    return tol + (ref.abs() + tol) * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)


def quantise(x):
    """Codes (float8_e4m3fn) and scale bytes of rows [..., d] of bf16 / fp32 values: by the definition, in fp64."""
    x = x.double()
    big = x.abs().amax(-1)
    k = torch.full(big.shape, -117, dtype=torch.int64)
    for step in range(120 + 117):                   # the smallest power for which no element exceeds 448 times it
        k += (big > 448 * 2.0 ** k.double()).long()
    y = x * 2.0 ** -k.double()[..., None]
    grid = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    y = torch.round(y / grid) * grid                # (to even)
    y = torch.where(k[..., None] == 120, y.clamp(-240, 240), y)
    byte = torch.where(big == 0, 127, k + 127)
    bad = ~torch.isfinite(big)
    return torch.where(bad[..., None], 0.0, y).float().to(torch.float8_e4m3fn), torch.where(bad, 255, byte).to(torch.uint8)


def values(codes, byte):
    """fp64 values of rows; byte 255: NaN."""
    v = codes.double() * torch.exp2(byte.double() - 127)[..., None]
    return torch.where((byte == 255)[..., None], float("nan"), v)


class Cache8:
    """A paged 8-bit cache on the GPU; memory of slots that are not live is NaN codes and bytes of 255."""

    def __init__(self, d, hkv, page, layout, n, lens, seed=0, extra_cols=0):
        rng = random.Random(seed)
        self.d, self.hkv, self.page, self.layout, self.n, self.lens = d, hkv, page, layout, n, lens
        S, self.per_head = len(n), layout == "heads"
        tables = hkv if self.per_head else 1
        cols = -(-max(max(lens), 1) // page) + extra_cols
        need = [-(-x // page) for x in lens]
        n_pages = sum(need) * tables + 3
        ids = rng.sample(range(n_pages), sum(need) * tables)
        self.table = torch.full((S, tables, cols), 1 << 30, dtype=torch.int32)
        for s in range(S):
            for h in range(tables):
                for c in range(need[s]):
                    self.table[s, h, c] = ids.pop()
        heads = 1 if self.per_head else hkv
        shape = (n_pages, heads, page, d) if layout == "hnd" else (n_pages, page, heads, d)
        pool = lambda: torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV)
        self.pools = [p.transpose(1, 2) if layout == "hnd" else p for p in (pool(), pool())]
        self.scales = [torch.full((n_pages, heads, page), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.table_dev = (self.table if self.per_head else self.table[:, 0]).contiguous().to(DEV)
        self.lens_dev = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.kv = lar.PagedKV8(self.pools[0].view(torch.float8_e4m3fn), self.pools[1], self.scales[0], self.scales[1], self.table_dev,
                               self.lens_dev, hkv, status=self.status)
        self.cu = torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32, device=DEV)

    def at(self, s, j0, j1):
        """Index tensors (page, row, head) [hkv, j1 - j0] of slots j0 .. j1 - 1 of sequence s, on the host."""
        j = torch.arange(j0, j1)
        h = torch.arange(self.hkv)[:, None]
        page = self.table[s][h if self.per_head else torch.zeros_like(h), j // self.page].long()
        return page, (j % self.page).expand(self.hkv, -1), torch.zeros_like(page) if self.per_head else h.expand_as(page)

    def put(self, s, which, j0, codes, byte):
        """codes [hkv, n, d], byte [hkv, n] into slots j0 on."""
        if codes.shape[1] == 0:
            return
        p, r, h = (x.to(DEV) for x in self.at(s, j0, j0 + codes.shape[1]))
        self.pools[which][p, r, h] = codes.view(torch.uint8).to(DEV)
        self.scales[which][p, h, r] = byte.to(DEV)

    def get(self, s, which, j0, j1):
        p, r, h = (x.to(DEV) for x in self.at(s, j0, j1))
        return self.pools[which][p, r, h].cpu().view(torch.float8_e4m3fn), self.scales[which][p, h, r].cpu()

    def fill(self, seed, start=None, spread=0.0):
        """Random live rows; spread: their sizes vary by that many powers of two."""
        self.vals = [[], []]
        g = torch.Generator().manual_seed(seed)
        for i in range(2):
            for s, L in enumerate(self.lens):
                x = torch.randn(self.hkv, L, self.d, generator=g) * torch.exp2((torch.rand(self.hkv, L, 1, generator=g) * spread).round())
                codes, byte = quantise(x)
                lo = max(0, start[s]) if start is not None else 0
                self.put(s, i, min(lo, L), codes[:, lo:], byte[:, lo:])
                self.vals[i].append(values(codes, byte))

    def rows(self, which):
        return lambda s, h, j0, j1: self.vals[which][s][h, j0:j1]


def attention_tolerance(dtype, ref, mag, big, d, longest, vmax):
    """As R.attention_tolerance; what is computed from the codes takes weights in fp16 (2^-11 of each; fp32 rows two of them: 2^-22), which below
    2^-28 of the largest is off by 2^-39 of it; q in two fp16 numbers is off by 2^-22.  Longer chunks are the kernels of bf16 and fp32 caches."""
    rel = 2 * (big * (d * 2.0 ** -24 + 2.0 ** -21) + longest * 2.0 ** -24 + 2.0 ** -20)[..., None]
    tol = mag * rel + longest * 2.0 ** -39 * 2 * vmax + 1e-30
    tol = tol + mag * (2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -22)
    return tol + (ref.abs() + tol) * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)
