"""Rotary positions with several axes, the append to a paged cache and the chunk attention over it, against plain 64-bit
forms on the sizes and masks where they can go wrong; refusals run without a GPU."""
import ctypes as C
import math
import random
import threading

import pytest
import torch

import _paged_reference as R
from paper_2512_04857_b200 import lar

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------------- refusals (no GPU)
def _kv(**kw):
    base = dict(struct_size=C.sizeof(lar.lar_paged_kv_t), dtype=lar.LAR_BF16, n_seqs=2, n_kv_heads=2, head_dim=64,
                page_tokens=32, n_pages=8, table_cols=4, page_stride=2 * 32 * 64, row_stride=2 * 64, head_stride=64,
                k_pool=4096, v_pool=8192, page_table=256, table_seq_stride=4, table_head_stride=0, lens=512, lens_stride=1,
                status=None)
    base.update(kw)
    return lar.lar_paged_kv_t(**base)


def _r(data=4096, token_stride=256, head_stride=64):
    return lar.lar_rows_t(data, token_stride, head_stride)


def _attn(kv, q=None, out=None, hq=4, n=6, cu=None, start=None, causal=1, scale=0.0, mc=0, ml=0, ws=None, nb=0):
    return lar.lib().lar_paged_attn(kv, q or _r(), out or _r(1 << 20), hq, n, cu, start, causal, scale, mc, ml, ws, nb, None)


INVALID = lar.LAR_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(struct_size=8), dict(dtype=2), dict(n_seqs=0), dict(n_kv_heads=0), dict(head_dim=96), dict(page_tokens=48),
    dict(page_tokens=8), dict(page_tokens=256), dict(n_pages=0), dict(table_cols=0), dict(table_cols=1 << 26),
    dict(page_stride=2 * 32 * 64 + 4), dict(row_stride=32), dict(row_stride=-128), dict(head_stride=0), dict(head_stride=4),
    dict(k_pool=4098), dict(v_pool=None), dict(k_pool=None), dict(page_table=None), dict(page_table=258), dict(lens=None),
    dict(lens=514), dict(lens_stride=-1), dict(table_seq_stride=-1), dict(status=6),
])
def test_paged_cache_refusals(bad):
    assert _attn(_kv(**bad)) == INVALID
    rows = _r(4096, 128, 64)
    assert lar.lib().lar_paged_append_rope(_kv(**bad), None, None, 0, rows, rows, None, None, 0, 6, None, None) == INVALID
    assert lar.lib().lar_paged_attn_workspace_bytes(_kv(**bad), 4, 6, 3, 128) == 0


def test_attention_refusals():
    kv = _kv()
    assert _attn(kv, hq=3) == INVALID                       # not a multiple of the KV heads
    assert _attn(kv, hq=34) == INVALID                      # 17 heads per KV head
    assert _attn(kv, n=5) == INVALID                        # equal chunks: not divisible
    assert _attn(kv, n=-1) == INVALID
    assert _attn(kv, scale=-1.0) == INVALID and _attn(kv, scale=float("nan")) == INVALID
    assert _attn(kv, scale=float("inf")) == INVALID
    assert _attn(kv, mc=-1) == INVALID and _attn(kv, ml=-1) == INVALID
    assert _attn(kv, cu=258) == INVALID and _attn(kv, start=258) == INVALID
    assert _attn(kv, q=_r(4104)) == INVALID and _attn(kv, q=_r(None)) == INVALID
    assert _attn(kv, q=_r(4096, 260)) == INVALID and _attn(kv, q=_r(4096, 256, 32)) == INVALID
    assert _attn(kv, out=_r(1 << 20, 64, 64)) == INVALID    # output rows on top of one another
    assert _attn(kv, n=0) == lar.LAR_OK                     # nothing to do
    assert lar.lib().lar_paged_attn(None, _r(), _r(), 4, 6, None, None, 1, 0.0, 0, 0, None, 0, None) == INVALID
    big = _kv(n_seqs=1, n_pages=4096, table_cols=4096)      # one token over 131072 slots: the workspace is wanted
    need = lar.lib().lar_paged_attn_workspace_bytes(big, 4, 1, 1, 0)
    assert need > 0
    assert _attn(big, n=1, ws=4096, nb=need - 1) == lar.LAR_ERR_NOMEM
    assert _attn(big, n=1, ws=4100, nb=need) == INVALID
    many = _kv(n_seqs=1025, dtype=lar.LAR_BF16)             # bf16: the lengths of at most 1024 sequences are kept on chip
    assert _attn(many, n=1025) == lar.LAR_ERR_CAPACITY
    huge = _kv(n_seqs=1024, n_pages=1 << 30, table_cols=1 << 23, page_tokens=128)
    assert _attn(huge, hq=2, n=1 << 20, q=_r(4096, 128), out=_r(1 << 20, 128)) == lar.LAR_ERR_CAPACITY   # 2^31 slot tiles or more


def test_append_refusals():
    L, kv, rows = lar.lib(), _kv(), _r(4096, 128, 64)
    rope = lar.make_rope(64, (8, 12, 12))

    def call(kv=kv, rope=rope, pos=256, ps=6, k=rows, v=rows, q=None, qo=None, hq=0, n=6, cu=None):
        return L.lar_paged_append_rope(kv, rope, pos, ps, k, v, q, qo, hq, n, cu, None)
    assert call(pos=None) == INVALID and call(rope=None) == INVALID and call(ps=5) == INVALID and call(pos=258) == INVALID
    assert call(k=None) == INVALID and call(v=_r(None)) == INVALID and call(k=_r(4097, 128, 64)) == INVALID
    assert call(q=rows) == INVALID and call(q=rows, qo=rows) == INVALID and call(hq=2) == INVALID and call(hq=-1) == INVALID
    assert call(rope=lar.make_rope(128, (64,))) == INVALID  # another head_dim
    assert call(n=7) == INVALID and call(cu=255) == INVALID
    assert call(n=0) == lar.LAR_OK and call(n=0, pos=None, k=None) == lar.LAR_OK
    assert call(kv=_kv(n_kv_heads=4097, table_head_stride=4, head_stride=0)) == INVALID and call(q=rows, qo=rows, hq=4097) == INVALID


def test_rope_refusals():
    L, rows = lar.lib(), _r(4096, 128, 64)

    def rot(rope, dtype=lar.LAR_BF16, pos=256, ps=6, n=6, q=rows, qo=rows, hq=2, k=None, ko=None, hk=0):
        return L.lar_rope_rotate(rope, dtype, pos, ps, n, q, qo, hq, k, ko, hk, 0, None)
    good = lar.make_rope(64, (8, 12, 12))
    for bad in (lar.make_rope(64, (8, 12)), lar.make_rope(64, (8, 12, 13)), lar.make_rope(64, (32, 0)), lar.make_rope(96, (48,)),
                lar.make_rope(64, (33, -1)), lar.make_rope(64, (32,), theta=0.0), lar.make_rope(64, (32,), theta=float("nan")),
                lar.make_rope(64, (1 << 30, 1 << 30, 32))):
        assert rot(bad) == INVALID
        assert L.lar_rope_table(bad, 256, 6, 6, 4096, None) == INVALID
    with pytest.raises(lar.LarError):
        lar.make_rope(64, (8, 8, 8, 4, 4))
    assert rot(good, dtype=3) == INVALID and rot(good, pos=None) == INVALID and rot(good, ps=5) == INVALID
    assert rot(good, hq=0) == INVALID and rot(good, k=rows) == INVALID and rot(good, hk=1) == INVALID
    assert rot(good, n=-1) == INVALID and rot(good, n=0) == lar.LAR_OK and rot(None) == INVALID
    assert rot(good, qo=_r(4096, 64, 64)) == INVALID and rot(good, q=_r(4100, 128, 64)) == INVALID
    assert L.lar_rope_table(good, 256, 6, -1, 4096, None) == INVALID and L.lar_rope_table(good, 256, 6, 0, 4096, None) == lar.LAR_OK
    assert L.lar_rope_table(good, 256, 5, 6, 4096, None) == INVALID and L.lar_rope_table(good, 256, 6, 6, 4098, None) == INVALID


def test_binding_refuses_tensors_that_do_not_fit():
    x, pos = torch.zeros(4, 2, 64), torch.zeros(1, 4, dtype=torch.int32)
    rope = lar.make_rope(64, (32,))
    with pytest.raises(lar.LarError):
        lar.rope_rotate(rope, pos, x, x)                                       # not on a GPU
    with pytest.raises(lar.LarError):
        lar.rope_rotate(rope, pos, x.double(), x.double())
    with pytest.raises(lar.LarError):
        lar.rope_rotate(rope, pos.long(), x, x)
    with pytest.raises(lar.LarError):
        lar.rope_rotate(rope, pos[:, :3], x, x)
    pool, table, lens = torch.zeros(4, 32, 2, 64), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    lar.PagedKV(pool, pool, table, lens, 2)
    for a in ((pool, pool.bfloat16(), table, lens, 2), (pool, pool, table.long(), lens, 2), (pool, pool, table, lens, 4),
              (pool, pool, table[:, None], lens, 2), (pool, pool, table, lens[:0], 2)):
        with pytest.raises(lar.LarError):
            lar.PagedKV(*a)


# ---------------------------------------------------------------------------------------------------------- rotary
def _randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float32) * scale).to(dtype)


def _pos(axes, n, seed, far=100000):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-20, far, (axes, n), generator=g, dtype=torch.int32)
    if axes > 1:
        p[1:] %= 128
    return p


def _assert_close(got, ref, tol, what=""):
    err = (got.double().cpu() - ref).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).nan_to_num(9e9).max()):.3g} x the bound"


ROPES = [((32,), 64), ((16, 16), 64), ((8, 12, 12), 64), ((11, 5, 9, 7), 64), ((64,), 128), ((16, 24, 24), 128), ((1, 62, 1), 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("restart", [False, True])
@pytest.mark.parametrize("axes,d", ROPES)
def test_rotary_rows(dtype, interleaved, restart, axes, d):
    for n, hq, hk in ((1, 1, 0), (5, 3, 1), (130, 20, 20), (2400, 5, 2)):
        x = _randn((n, hq + hk + 1, d), dtype, n + d)                    # views of one projection's output
        pos = _pos(len(axes), n, n)
        rope = lar.make_rope(d, axes, theta=10000.0, interleaved=interleaved, restart=restart)
        xd, pd = x.to(DEV), pos.to(DEV)
        q, k = xd[:, :hq], xd[:, hq:hq + hk] if hk else None
        qo = torch.full((hq, n, d), 7.0, dtype=dtype, device=DEV).transpose(0, 1)    # head-major output
        ko = torch.empty(n, hk, d, dtype=dtype, device=DEV) if hk else None
        lar.rope_rotate(rope, pd, q, qo, k, ko)
        ref = R.rotate(x, pos, axes, 10000.0, interleaved, restart)
        tol = R.rotation_tolerance(dtype, ref, x, interleaved)
        _assert_close(qo, ref[:, :hq], tol[:, :hq], "q")
        if hk:
            _assert_close(ko, ref[:, hq:hq + hk], tol[:, hq:hq + hk], "k")
        # in place and back: two rotations' roundings, the first's scaled by |cos| + |sin| <= sqrt 2
        lar.rope_rotate(rope, pd, q, q)
        assert torch.equal(q, qo)
        assert torch.equal(xd[:, hq + hk:].cpu(), x[:, hq + hk:])        # neighbours untouched
        lar.rope_rotate(rope, pd, q, q, inverse=True)
        xq = x[:, :hq]
        first = R.rotation_tolerance(dtype, ref[:, :hq], xq, interleaved)
        back = R.partner_sum(first, interleaved) + R.rotation_tolerance(dtype, xq.double(), ref[:, :hq].abs() + first, interleaved)
        _assert_close(q, xq.double(), back, "back")


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hk", [(1, 0), (1, 1), (2, 0), (9, 8), (300, 7)])
def test_rotary_rows_of_large_batches(hq, hk):
    """Two tokens per CTA, with every count of rows that its division has to get right at the edges (one row among them)."""
    n, d = 2401, 64
    x, pos = _randn((n, hq + hk, d), F32, hq), _pos(1, n, hk)
    rope, xd = lar.make_rope(d, (32,)), x.to(DEV)
    q, k = xd[:, :hq], xd[:, hq:] if hk else None
    qo, ko = torch.full_like(q, 9.0, memory_format=torch.contiguous_format), torch.full((n, hk, d), 9.0, device=DEV) if hk else None
    lar.rope_rotate(rope, pos.to(DEV), q, qo, k, ko)
    ref = R.rotate(x, pos, (32,), 10000.0, False, False)
    tol = R.rotation_tolerance(F32, ref, x, False)
    _assert_close(qo, ref[:, :hq], tol[:, :hq], "q")
    if hk:
        _assert_close(ko, ref[:, hq:], tol[:, hq:], "k")


@pytest.mark.gpu
def test_rotary_gradient_is_the_inverse_rotation():
    """d/dx of <g, rotate(x)> against differences of the 64-bit form, and against the kernel's inverse rotation of g."""
    axes, d, n, h = (8, 12, 12), 64, 3, 2
    x, g, pos = _randn((n, h, d), F32, 1), _randn((n, h, d), F32, 2), _pos(3, n, 3)
    rope = lar.make_rope(d, axes)
    gx = torch.empty(n, h, d, device=DEV)
    lar.rope_rotate(rope, pos.to(DEV), g.to(DEV), gx, inverse=True)
    f = lambda y: (g.double() * R.rotate(y, pos, axes, 10000.0, False, False)).sum()
    ref = torch.zeros(n, h, d, dtype=torch.float64)
    for i in range(n * h * d):
        e = torch.zeros(n * h * d, dtype=torch.float64)
        e[i] = 0.5                                             # the form is linear: any step gives the exact quotient
        e = e.view(n, h, d)
        ref.view(-1)[i] = f(x.double() + e) - f(x.double() - e)
    _assert_close(gx, ref, R.rotation_tolerance(F32, ref, g, False) + 1e-12, "gradient")


@pytest.mark.gpu
def test_table_feeds_the_decode_step():
    """lar_rope_table -> lar_decode_step_rope equals lar_rope_rotate -> lar_decode_step, bit for bit."""
    for interleaved in (False, True):
        w = dict(n_layers=1, batch=3, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", cond_len=5, line_width=8, n_lines=4,
                 anchor_len=8, recent_lines=1, budget_lines=4)
        caches = [lar.Cache(lar.make_config(**w)) for _ in range(2)]
        rope = lar.make_rope(64, (10, 11, 11), interleaved=interleaved)
        kc, vc = _randn((3, 2, 5, 64), BF, 1).to(DEV), _randn((3, 2, 5, 64), BF, 2).to(DEV)
        for c in caches:
            c.append_kv(0, kc, vc, 5)
        for step in range(4):
            q, k, v = (_randn((3, h, 64), BF, 10 * step + i).to(DEV) for i, h in enumerate((4, 2, 2)))
            pos = _pos(3, 3, step).to(DEV)
            cs = torch.empty(3, 64, device=DEV)
            lar.rope_table(rope, pos, cs)
            outs = [torch.empty_like(q) for _ in range(2)]
            caches[0].decode_step_rope(0, q, k, v, outs[0], 256, 128, 128, 256, cs, interleaved)
            qr, kr = torch.empty_like(q), torch.empty_like(k)
            lar.rope_rotate(rope, pos, q, qr, k, kr)
            caches[1].decode_step(0, qr, kr, v, outs[1])
            assert torch.equal(outs[0], outs[1])
        for c in caches:
            assert c.poll_device_status() == 0
            c.close()


# ------------------------------------------------------------------------------------------------- a cache for the tests
class PagedCase:
    """Pools with shuffled pages, NaN wherever no live row lies, and a table whose unused entries are out of range."""

    def __init__(self, dtype, d, hkv, page, layout, n, lens, seed=0, extra_cols=1):
        rng = random.Random(seed)
        self.dtype, self.d, self.hkv, self.page, self.layout, self.n, self.lens = dtype, d, hkv, page, layout, n, lens
        S, per_head = len(n), layout == "heads"
        tables = hkv if per_head else 1
        cols = -(-max(max(lens), 1) // page) + extra_cols
        need = [-(-x // page) for x in lens]
        n_pages = sum(need) * tables + 3
        ids = rng.sample(range(n_pages), sum(need) * tables)
        self.table = torch.full((S, tables, cols), 1 << 30, dtype=torch.int32)
        for s in range(S):
            for h in range(tables):
                for c in range(need[s]):
                    self.table[s, h, c] = ids.pop()
                if cols - need[s] > 1:
                    self.table[s, h, need[s] + 1:] = -7
        heads = 1 if per_head else hkv
        shape = (n_pages, heads, page, d) if layout == "hnd" else (n_pages, page, heads, d)
        self.pools = [torch.full(shape, float("nan"), dtype=dtype) for _ in range(2)]
        if layout == "hnd":
            self.pools = [p.transpose(1, 2) for p in self.pools]
        self.dev = [self._to_dev(p) for p in self.pools]
        tab = (self.table if per_head else self.table[:, 0]).contiguous().to(DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.lens_dev = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.kv = lar.PagedKV(self.dev[0], self.dev[1], tab, self.lens_dev, hkv, status=self.status)
        self.cu = torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32, device=DEV)

    def _to_dev(self, p):
        return p.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) if self.layout == "hnd" else p.to(DEV)

    def place(self, s, h, j):
        per_head = self.layout == "heads"
        return int(self.table[s, h if per_head else 0, j // self.page]), j % self.page, 0 if per_head else h

    def fill(self, start, seed):
        """Random live rows (slots before start stay NaN)."""
        for i, p in enumerate(self.pools):
            for s, L in enumerate(self.lens):
                x = _randn((self.hkv, L, self.d), self.dtype, seed * 1000 + 2 * s + i)
                for h in range(self.hkv):
                    for j in range(start[s] if start else 0, L):
                        a, b, c = self.place(s, h, j)
                        p[a, b, c] = x[h, j]
            self.dev[i].copy_(p.to(DEV))

    def rows(self, which):
        def get(s, h, j0, j1):
            return torch.stack([self.pools[which][self.place(s, h, j)] for j in range(j0, j1)])
        return get


# ---------------------------------------------------------------------------------------------------------- append
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", [("heads", 32, 128, 3, 6), ("nhd", 16, 64, 5, 0), ("hnd", 64, 128, 2, 8),
                                                  ("nhd", 128, 64, 1, 4), ("heads", 16, 64, 20, 20)])
@pytest.mark.parametrize("n,lens", [([1], [1]), ([1, 0, 1, 1], [64, 9, 65, 1]), ([0, 33, 7, 0, 130], [3, 33, 70, 0, 257])])
def test_append(dtype, layout, page, d, hkv, hq, n, lens):
    for rotated in (True, False):
        c = PagedCase(dtype, d, hkv, page, layout, n, lens, seed=page + d)
        T = sum(n)
        pad = 2                                                # a padded batch: tokens that belong to no sequence
        x = _randn((T + pad, hq + 2 * hkv, d), dtype, 5)
        xd = x.to(DEV)
        axes = (8, 12, 12) if d == 64 else (16, 24, 24)
        pos = _pos(3, T + pad, 6)
        rope = lar.make_rope(d, axes, interleaved=page == 16)
        qo = torch.full((T + pad, hq, d), 7.0, dtype=dtype, device=DEV) if hq else None
        c.kv.append_rope(xd[:, hq:hq + hkv], xd[:, hq + hkv:], c.cu, rope if rotated else None, pos.to(DEV) if rotated else None,
                         xd[:, :hq] if hq else None, qo)
        ref = R.rotate(x, pos, axes, 10000.0, page == 16, False) if rotated else x.double()
        tol = R.rotation_tolerance(dtype, ref, x, page == 16) if rotated else torch.zeros_like(ref)
        want = [p.double().clone() for p in c.pools]
        tols = torch.zeros_like(want[0])
        t = 0
        for s, a in enumerate(n):
            for i in range(a):
                for h in range(hkv):
                    at = c.place(s, h, lens[s] - a + i)
                    want[0][at], want[1][at] = ref[t, hq + h], x[t, hq + hkv + h].double()
                    tols[at] = tol[t, hq + h]
                t += 1
        for i in range(2):
            got, nan = c.dev[i].double().cpu(), want[i].isnan()
            assert torch.equal(got.isnan(), nan)               # every other row as it was
            _assert_close(got[~nan], want[i][~nan], (tols if i == 0 else tols * 0)[~nan], f"pool {i}")
        if hq:
            _assert_close(qo[:T], ref[:T, :hq], tol[:T, :hq], "q")
            assert (qo[T:] == 7.0).all()
        assert int(c.status) == 0


@pytest.mark.gpu
def test_append_follows_no_bad_page_or_slot():
    c = PagedCase(BF, 64, 2, 32, "nhd", [40, 3], [40, 10])
    table = c.kv._keep[2]
    table[0, 1] = 10 ** 6                                     # the second page of sequence 0
    c.lens_dev[1] = 2                                          # fewer entries than the chunk has tokens
    before = [x.clone() for x in c.dev]
    x = _randn((43, 4, 64), BF, 1).to(DEV)
    c.kv.append_rope(x[:, :2], x[:, 2:], c.cu)
    assert int(c.status) == 64
    for which, pool in enumerate(c.dev):
        want = before[which].clone()
        want[int(c.table[0, 0, 0])] = x[:32, 2 * which:2 * which + 2]
        page = int(c.table[1, 0, 0])
        want[page, 0:2] = x[41:43, 2 * which:2 * which + 2]    # tokens 1 and 2 of the chunk have slots 0 and 1
        assert torch.equal(pool.nan_to_num(9.0), want.nan_to_num(9.0))


# ------------------------------------------------------------------------------------------------------- attention
LENGTHS = [
    ([1], [1]),
    ([1, 1, 0, 1], [63, 64, 9, 65]),
    ([1, 1], [700, 129]),
    ([3, 0, 17, 2], [3, 0, 130, 257]),
    ([40, 1, 130], [40, 300, 200]),
    ([300, 5], [310, 5]),
]
SHAPES = [("heads", 32, 128, 2, 4), ("nhd", 64, 64, 2, 2), ("hnd", 16, 128, 1, 8), ("nhd", 128, 128, 3, 3), ("heads", 64, 64, 1, 3),
          ("hnd", 32, 64, 1, 16)]


def _check_attention(c, hq, causal, start, workspace, seed, out_pad=2, hints=True, q=None, scale=0.0):
    T, d, dtype = sum(c.n), c.d, c.dtype
    q = _randn((T + out_pad, hq, d), dtype, seed) if q is None else q
    buf = torch.full((T + out_pad, hq + 1, d), 5.0, dtype=dtype, device=DEV)     # out is a view with a gap behind each token
    out = buf[:, :hq]
    mc, ml = hints if isinstance(hints, tuple) else (max(c.n), max(c.lens)) if hints else (0, 0)
    ws = c.kv.attn_workspace(hq, T + out_pad, mc, ml) if workspace else None
    if ws is not None:
        ws.fill_(255)
    sd = torch.tensor(start, dtype=torch.int32, device=DEV) if start is not None else None
    c.kv.attn(q.to(DEV), out, c.cu, causal=causal, kv_start=sd, softmax_scale=scale, max_chunk=mc, max_len=ml, workspace=ws)
    ref, mag, big = R.attention(q[:T], c.rows(0), c.rows(1), c.n, c.lens, start, causal, hq // c.hkv, scale or d ** -0.5)
    tol = R.attention_tolerance(dtype, ref, mag, big, d, max(c.lens))
    _assert_close(out[:T], ref, tol, f"causal {causal} start {start} workspace {ws is not None}")
    assert (out[T:] == 5.0).all() and (buf[:, hq:] == 5.0).all()
    assert int(c.status) == 0
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", SHAPES)
@pytest.mark.parametrize("n,lens", LENGTHS)
def test_attention(dtype, layout, page, d, hkv, hq, n, lens):
    c = PagedCase(dtype, d, hkv, page, layout, n, lens, seed=d + page)
    c.fill(None, 3)
    for causal in (True, False):
        for workspace in (False, True):
            _check_attention(c, hq, causal, None, workspace, 11)
    _check_attention(c, hq, True, None, True, 12, hints=False)
    for hints in ((1, 1), (10 ** 6, 10 ** 6)):            # bounds that do not hold choose another launch shape, no other result
        _check_attention(c, hq, True, None, True, 12, hints=hints)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,lens,start", [
    ([20, 5, 1], [20, 70, 66], [7, 69, 65]),          # the first tokens of a chunk are padding: they see nothing
    ([40, 1, 9], [40, 64, 9], [200, 64, 9]),          # nothing is live: every row is zero
    ([150, 3], [400, 140], [129, 128]),               # the padding ends inside, and at the end of, a step of slots
    ([2, 2], [90, 90], [-5, 33]),                     # negative: no padding
])
def test_attention_with_left_padding(dtype, n, lens, start):
    c = PagedCase(dtype, 64, 2, 32, "heads", n, lens)
    c.fill([max(s, 0) for s in start], 4)
    for causal in (True, False):
        for workspace in (False, True):
            out = _check_attention(c, 4, causal, start, workspace, 21)
            if start[0] == 200:
                assert (out[:sum(n)] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", SHAPES)
@pytest.mark.parametrize("n,lens,start", [(n, lens, None) for n, lens in LENGTHS] + [
    ([20, 5, 1], [20, 70, 66], [7, 69, 65]),
    ([40, 1, 9], [40, 64, 9], [200, 64, 9]),
    ([2, 1, 3], [1300, 900, 40], [700, 0, 33]),
])
def test_attention_of_short_caches_in_long_tables(dtype, layout, page, d, hkv, hq, n, lens, start):
    """Lengths that only the GPU knows: tables and bounds that allow long caches make the kernels cut the few slots there are."""
    c = PagedCase(dtype, d, hkv, page, layout, n, lens, seed=d + page, extra_cols=1 + 8192 // page)
    c.fill(start, 3)
    for causal in (True, False):
        _check_attention(c, hq, causal, start, True, 13, hints=(max(n), 10 ** 6))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,d", [([70, 1], 64), ([40, 9], 64), ([33, 1], 128), ([3, 1], 64), ([2, 8], 128)])
def test_attention_of_extreme_logits(dtype, n, d):
    """Logits of several hundred either way: the running maximum has to be taken off, and to grow along the cache."""
    c = PagedCase(dtype, d, 1, 32, "nhd", n, [300, 513])
    c.fill(None, 5)
    for i, s in enumerate(c.lens):                    # keys that grow with the slot
        for j in range(s):
            c.pools[0][c.place(i, 0, j)] *= 1.0 + j / 16
    c.dev[0].copy_(c.pools[0].to(DEV))
    for workspace in (False, True):
        _check_attention(c, 2, True, None, workspace, 31)
        _check_attention(c, 2, True, None, workspace, 32, scale=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_many_ragged_prompts(d, causal):
    """More row tiles than SMs, of very different lengths: CTAs take them on demand."""
    rng = random.Random(d)
    n = [rng.choice([1, 33, 64, 65, 90]) for _ in range(48)]
    lens = [a + rng.choice([0, 0, 100]) for a in n]
    c = PagedCase(BF, d, 2, 32, "nhd", n, lens, seed=d)
    start = [rng.choice([0, 0, 7, 40]) for _ in n]
    c.fill(start, 3)
    _check_attention(c, 8, causal, start, True, 5)
    _check_attention(c, 8, causal, start, False, 6)


@pytest.mark.gpu
def test_attention_of_as_many_sequences_as_there_may_be():
    n = [1] * 1024
    c = PagedCase(BF, 64, 1, 16, "nhd", n, [1 + i % 40 for i in range(1024)], seed=1)
    c.fill(None, 2)
    for hints in ((1, 40), (40, 40), (300, 40)):          # the kernels for few rows, for one row tile and for two
        _check_attention(c, 4, True, None, True, 3, hints=hints)


@pytest.mark.gpu
def test_attention_of_long_chunks_in_whole_and_cut_rounds():
    """One full round of row tiles over the SMs, and a rest whose slots are cut into equal ranges."""
    c = PagedCase(BF, 64, 4, 64, "hnd", [1280, 1216], [2900, 2850])
    for p, x in zip(c.pools, c.dev):
        x.normal_()
        p.copy_(x.cpu())
    _check_attention(c, 16, True, None, True, 7)


@pytest.mark.gpu
@pytest.mark.parametrize("n,lens", [([1] * 40, [700] * 40), ([1, 1, 1], [5000, 70, 3000]), ([20] * 6, [1200] * 6), ([90] * 6, [1200] * 6), ([100] * 40, [150] * 40),
                                    ([300], [4000])])
def test_attention_repeats_itself(n, lens):
    """Many runs of the same call, next to work on another stream, give the same bits and never run into a wait limit."""
    c = PagedCase(BF, 128, 2, 64, "nhd", [0] * len(n), lens)
    c.n = n
    c.cu = torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32, device=DEV)
    for p in c.dev:
        p.normal_()
    T = sum(n)
    q = _randn((T, 8, 128), BF, 1).to(DEV) * 3
    outs = [torch.empty_like(q) for _ in range(2)]
    ws = c.kv.attn_workspace(8, T, max(n), max(lens))
    side, big = torch.cuda.Stream(), torch.randn(1 << 24, device=DEV)
    for rep in range(60):
        out = outs[min(rep, 1)]
        out.fill_(7.0)
        with torch.cuda.stream(side):
            big.mul_(1.0001)
        c.kv.attn(q, out, c.cu, max_chunk=max(n), max_len=max(lens), workspace=ws)
        if rep:
            assert torch.equal(outs[0], outs[1]), rep
    assert int(c.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_reads_a_bad_page_as_zeros(dtype):
    c = PagedCase(dtype, 128, 2, 32, "nhd", [3, 2], [100, 40])
    c.fill(None, 6)
    table = c.kv._keep[2]
    for bad in (10 ** 6, -1, -2 ** 31, 2 ** 31 - 1):
        table[0, 1] = bad
        q = _randn((5, 4, 128), dtype, 7)
        out = torch.empty(5, 4, 128, dtype=dtype, device=DEV)
        c.kv.attn(q.to(DEV), out, c.cu)
        assert int(c.status) == 64
        c.status.zero_()
        zeroed = lambda which: (lambda s, h, j0, j1: torch.stack([
            torch.zeros(128, dtype=dtype) if s == 0 and 32 <= j < 64 else c.pools[which][c.place(s, h, j)] for j in range(j0, j1)]))
        ref, mag, big = R.attention(q, zeroed(0), zeroed(1), c.n, c.lens, None, True, 2, 128 ** -0.5)
        _assert_close(out, ref, R.attention_tolerance(dtype, ref, mag, big, 128, 100))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_of_lengths_the_table_cannot_hold(dtype):
    """A length beyond the table is cut to what the table holds; a chunk longer than its cache sees what there is."""
    c = PagedCase(dtype, 64, 1, 32, "heads", [2, 9], [64, 4], extra_cols=0)
    c.fill(None, 8)
    q = _randn((11, 1, 64), dtype, 9)
    out = torch.empty(11, 1, 64, dtype=dtype, device=DEV)
    c.lens_dev[0] = 10 ** 6
    c.kv.attn(q.to(DEV), out, c.cu)
    ref, mag, big = R.attention(q[:2], c.rows(0), c.rows(1), [2, 0], [64, 4], None, True, 1, 0.125)
    _assert_close(out[:2], ref, R.attention_tolerance(dtype, ref, mag, big, 64, 64))
    assert (out[2:7] == 0).all()                       # slots before the cache's first
    ref, mag, big = R.attention(q[7:], c.rows(0), c.rows(1), [0, 4], [64, 4], None, True, 1, 0.125)
    _assert_close(out[7:], ref, R.attention_tolerance(dtype, ref, mag, big, 64, 64))


# ------------------------------------------------------------------------------------------------- used together
@pytest.mark.gpu
def test_prefill_of_the_librarys_cache_then_decode_steps():
    """A conditional prefix enters the cache with rotated keys, its attention runs over the cache, and decode steps with
    the table of the same rotary embedding follow: everything against the 64-bit forms."""
    S, Hq, Hkv, d, Cn = 3, 4, 2, 128, 37
    for flags, dtype in ((0, "bf16"), (lar.LAR_FLAG_SHUFFLE_PAGES | lar.LAR_FLAG_PDL, "bf16"), (lar.LAR_FLAG_SHUFFLE_PAGES, "fp32")):
        td = BF if dtype == "bf16" else F32
        cfg = lar.make_config(n_layers=2, batch=S, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, dtype=dtype, cond_len=Cn,
                              line_width=8, n_lines=4, anchor_len=8, recent_lines=1, budget_lines=4, flags=flags, page_seed=3)
        cache = lar.Cache(cfg)
        axes = (16, 24, 24)
        rope = lar.make_rope(d, axes)
        start = [0, 5, 36]
        sd = torch.tensor(start, dtype=torch.int32, device=DEV)
        for layer in range(2):
            x = _randn((S * Cn, Hq + 2 * Hkv, d), td, layer)
            pos = _pos(3, S * Cn, layer)
            xd, qo = x.to(DEV), torch.empty(S * Cn, Hq, d, dtype=td, device=DEV)
            cache.append_kv_rope(layer, xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], Cn, rope, pos.to(DEV), xd[:, :Hq], qo)
            with pytest.raises(lar.LarError) as e:
                cache.append_kv_rope(layer, xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], Cn)
            assert e.value.status == lar.LAR_ERR_BAD_STATE
            out = torch.empty_like(qo)
            view = cache.paged_view(layer)
            view.attn(qo, out, kv_start=sd, max_chunk=Cn, max_len=Cn, workspace=view.attn_workspace(Hq, S * Cn, Cn, Cn))
            turned = R.rotate(x[:, :Hq + Hkv], pos, axes, 10000.0, False, False).to(td)
            k, v = turned[:, Hq:].view(S, Cn, Hkv, d), x[:, Hq + Hkv:].view(S, Cn, Hkv, d)
            ref, mag, big = R.attention(qo.cpu(), lambda s, h, a, b: k[s, a:b, h], lambda s, h, a, b: v[s, a:b, h], [Cn] * S, [Cn] * S,
                                        start, True, Hq // Hkv, d ** -0.5)
            # the reference's keys may round to the other neighbour: one step of bf16 (2^-7) or fp32 (2^-23) of each product
            step = (2.0 ** -7 if td == BF else 2.0 ** -23) * 2 * big[..., None] * mag
            _assert_close(out, ref, R.attention_tolerance(td, ref, mag, big, d, Cn) + step, f"{dtype} layer {layer}")
            lens, imap = cache.get_state(layer)
            assert (lens == Cn).all() and (imap[:, :Cn] == torch.arange(Cn).numpy()).all()
            # a decode step behind it: compared with the plain attention over the same rows (no padding mask there)
            q1, k1, v1 = (_randn((S, h, d), td, 50 + layer + i) for i, h in enumerate((Hq, Hkv, Hkv)))
            o1 = torch.empty(S, Hq, d, dtype=td, device=DEV)
            cache.decode_step(layer, q1.to(DEV), k1.to(DEV), v1.to(DEV), o1)
            view.attn(q1.to(DEV), out[:S], max_chunk=1, max_len=Cn + 1)       # the same token as a chunk of one
            ka, va = torch.cat([k, k1[:, None]], 1), torch.cat([v, v1[:, None]], 1)
            ref, mag, big = R.attention(q1, lambda s, h, a, b: ka[s, a:b, h], lambda s, h, a, b: va[s, a:b, h], [1] * S, [Cn + 1] * S,
                                        None, True, Hq // Hkv, d ** -0.5)
            step = (2.0 ** -7 if td == BF else 2.0 ** -23) * 2 * big[..., None] * mag
            for o in (o1, out[:S]):
                _assert_close(o, ref, R.attention_tolerance(td, ref, mag, big, d, Cn + 1) + step, f"{dtype} step {layer}")
        assert cache.poll_device_status() == 0
        cache.close()


@pytest.mark.gpu
@pytest.mark.parametrize("extra_cols,max_len", [(0, 310), (256, 8192)])     # units stay whole, and are cut and joined
def test_chunks_of_a_growing_cache_in_a_graph(extra_cols, max_len):
    """Append and attention of chunks captured once and replayed with other lengths, positions and pages: the graph reads
    them on the device.  Two replays share the workspace, one behind the other; they run on a side stream."""
    hq, hkv, d, page, S = 4, 2, 64, 32, 3
    n, T = [4, 1, 7], 12
    c = PagedCase(BF, d, hkv, page, "nhd", n, [300, 290, 310], extra_cols=extra_cols)
    c.fill(None, 1)
    rope, axes = lar.make_rope(d, (32,)), (32,)
    x, pos = torch.empty(T, hq + 2 * hkv, d, dtype=BF, device=DEV), torch.zeros(1, T, dtype=torch.int32, device=DEV)
    qo, out = torch.empty(T, hq, d, dtype=BF, device=DEV), torch.empty(T, hq, d, dtype=BF, device=DEV)
    ws = c.kv.attn_workspace(hq, T, 7, max_len)
    side = torch.cuda.Stream()

    def step():
        c.kv.append_rope(x[:, hq:hq + hkv], x[:, hq + hkv:], c.cu, rope, pos, x[:, :hq], qo)
        c.kv.attn(qo, out, c.cu, max_chunk=7, max_len=max_len, workspace=ws)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    c.fill(None, 1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for rep, lens in enumerate(([300, 290, 310], [4, 1, 30], [257, 64, 128])):
        xs, ps = _randn((T, hq + 2 * hkv, d), BF, 60 + rep), _pos(1, T, rep)
        x.copy_(xs.to(DEV))
        pos.copy_(ps.to(DEV))
        c.lens_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        c.lens = lens
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i in range(2):                              # the rows the append has just written
            c.pools[i].copy_(c.dev[i].cpu())
        ref, mag, big = R.attention(qo.cpu(), c.rows(0), c.rows(1), n, lens, None, True, hq // hkv, d ** -0.5)
        _assert_close(out, ref, R.attention_tolerance(BF, ref, mag, big, d, 310), f"replay {rep}")
        turned = R.rotate(xs[:, :hq], ps, axes, 10000.0, False, False)
        _assert_close(qo, turned, R.rotation_tolerance(BF, turned, xs[:, :hq], False), "q")
    assert int(c.status) == 0


# --------------------------------------------------------------------------------------- one workspace for many calls
WS_HEADS = [(1, 1), (2, 8), (4, 8), (8, 1), (3, 20), (16, 2)]        # (heads of a group, KV heads)


@pytest.mark.parametrize("dtype", [lar.LAR_BF16, lar.LAR_FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,hkv", WS_HEADS)
def test_a_workspace_holds_for_smaller_calls(dtype, d, group, hkv):
    """What is asked for a call covers every call with fewer sequences, tokens, tokens of a chunk and entries."""
    def need(seqs, tokens, chunk, length):
        kv = _kv(dtype=dtype, head_dim=d, n_seqs=seqs, n_kv_heads=hkv, n_pages=1 << 16, table_cols=1 << 11, row_stride=hkv * d,
                 head_stride=d, page_stride=hkv * d * 32)
        return lar.lib().lar_paged_attn_workspace_bytes(kv, group * hkv, tokens, chunk, length)
    rng = random.Random(d + hkv)
    pick = lambda hi: max(1, min(hi, int(hi ** rng.random() + 0.5)))
    for _ in range(300):
        seqs, chunk, length = pick(1024), pick(8192), pick(65536)
        tokens = pick(seqs * chunk)
        if rng.random() < 0.5:                                          # bounds that are not known: no chunk is longer than the batch
            chunk, large = tokens, need(seqs, tokens, 0, 0)
        else:
            large = need(seqs, tokens, chunk, length)
        for _ in range(4):
            s, t, c, n = pick(seqs), pick(tokens), rng.choice([0, pick(chunk)]), pick(length)
            if c == 0 and t > chunk:
                continue
            assert need(s, t, c, n) <= large, (seqs, tokens, chunk, length, s, t, c, n)
    # 32 sequences of single tokens and 24 of them; a prompt and one token
    assert need(24, 24, 1, 4288) <= need(32, 32, 1, 4288) <= need(222, 222, 1, 4288)
    assert need(1, 1, 1, 4096) <= need(1, 4096, 4096, 4096) and need(1, 2048, 2048, 4096) <= need(1, 4096, 4096, 4096)
    assert need(1, 1, -1, 0) == 0 and need(1, 1, 1, -1) == 0            # attn refuses these


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hkv,hq", [(128, 2, 8), (64, 3, 3)])
def test_one_workspace_for_a_prompt_and_what_follows(dtype, d, hkv, hq):
    """Sized once for the largest call, then used for smaller ones of every launch shape (the fence behind it stays)."""
    lens = [2600, 700, 130, 2100]
    c = PagedCase(dtype, d, hkv, 64, "nhd", [600, 3, 0, 40], lens, seed=d)
    for p, x in zip(c.pools, c.dev):
        x.normal_()
        p.copy_(x.cpu())
    n_bytes = lar.lib().lar_paged_attn_workspace_bytes(c.kv.desc, hq, 643, 600, 2600)
    buf = torch.full((n_bytes + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    ws = buf[:n_bytes]
    for seqs, n in ((4, [600, 3, 0, 40]), (4, [1, 1, 1, 1]), (4, [300, 0, 0, 0]), (2, [40, 2]), (1, [1]), (1, [9]), (1, [200]), (4, [2, 0, 1, 2])):
        part = lar.PagedKV(c.dev[0], c.dev[1], c.kv._keep[2][:seqs], c.lens_dev[:seqs], hkv, status=c.status)
        cu = torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32, device=DEV)
        q = _randn((sum(n), hq, d), dtype, sum(n))
        out = torch.full((sum(n), hq, d), 5.0, dtype=dtype, device=DEV)
        part.attn(q.to(DEV), out, cu, max_chunk=max(n), max_len=2600, workspace=ws)
        ref, mag, big = R.attention(q, c.rows(0), c.rows(1), n, lens[:seqs], None, True, hq // hkv, d ** -0.5)
        _assert_close(out, ref, R.attention_tolerance(dtype, ref, mag, big, d, 2600), f"{n}")
    assert int(c.status) == 0 and (buf[n_bytes:] == 0xA5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 0, 2], [40, 0, 9], [200, 0, 33]])     # few rows, one and two row tiles
def test_attention_reports_slots_that_the_table_does_not_hold(dtype, n):
    """A length beyond the table, below zero, or of fewer entries than the chunk has tokens leaves bit 64 in the status word."""
    c = PagedCase(dtype, 64, 2, 32, "nhd", n, [256, 256, 256], extra_cols=0)
    c.fill(None, 8)
    q = _randn((sum(n), 2, 64), dtype, 9).to(DEV)
    out = torch.empty_like(q)
    ws = c.kv.attn_workspace(2, sum(n), max(n), 256)
    for lens, want in (([256, 256, 256], 0), (n, 0), ([256, 10 ** 6, 256], 0), ([256, -3, 256], 0),    # (no tokens: nothing is looked up)
                       ([257, 256, 256], 64), ([256, 0, n[2] - 1], 64), ([-1, 0, 256], 64), ([256, 0, -2 ** 31], 64), ([256, 0, 2 ** 31 - 1], 64)):
        for causal in (True, False):
            c.lens_dev.copy_(torch.tensor(lens))
            c.kv.attn(q, out, c.cu, causal=causal, max_chunk=max(n), max_len=256, workspace=ws)
            assert int(c.status) == want, (lens, causal)
            c.status.zero_()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,n", [(1, [1, 3]), (2, [2, 7]), (4, [40, 9])])        # the kernels of 8, 16 and 64 rows
def test_fp32_attention_of_the_largest_numbers(d, hq, n):
    """Finite values next to fp32's largest stay finite: in V, and in q or K where the other factor is zero."""
    c = PagedCase(F32, d, 1, 32, "nhd", n, [70, 129])
    c.fill(None, 5)
    top = torch.tensor([0x7f7fffff, 0x7f7fff8b, 0x7f7ff000, 0x7f7fefff], dtype=torch.int32).view(torch.float32)
    for s, length in enumerate(c.lens):
        for e in range(d):                            # one slot of each column, either sign
            c.pools[1][c.place(s, 0, (7 * e) % (length - max(n)))][e] = top[e % 4] * (1 if e & 4 else -1)
        for j in range(length):
            c.pools[0][c.place(s, 0, j)][:4] = top * (1 if j & 1 else -1)
            c.pools[0][c.place(s, 0, j)][4:8] = 0.0
    for p, x in zip(c.pools, c.dev):
        x.copy_(p.to(DEV))
    q = _randn((sum(n), hq, d), F32, 4)
    q[..., :4] = 0.0
    q[..., 4:8] = top
    for workspace in (False, True):
        _check_attention(c, hq, True, None, workspace, 0, out_pad=0, q=q)


# ------------------------------------------------------------------------------------------------------ status word
def test_a_paged_cache_has_a_status_word_of_its_own():
    """Where the caller gives none, the binding keeps one: a wait that ran out or a bad page is not lost."""
    pool, table, lens = torch.zeros(4, 32, 2, 64), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    kv = lar.PagedKV(pool, pool, table, lens, 2)
    assert kv.desc.status and kv.poll_device_status() == 0
    word = torch.zeros(1, dtype=torch.int32)
    kv = lar.PagedKV(pool, pool, table, lens, 2, status=word)
    assert kv.desc.status == word.data_ptr()
    word.fill_(68)
    assert kv.poll_device_status() == 68 and kv.poll_device_status() == 0 and int(word) == 0


@pytest.mark.gpu
def test_status_of_a_paged_cache_and_of_a_layer():
    c = PagedCase(BF, 64, 2, 32, "nhd", [3], [40])
    c.fill(None, 1)
    kv = lar.PagedKV(c.dev[0], c.dev[1], c.kv._keep[2], c.lens_dev, 2)
    q = _randn((3, 2, 64), BF, 1).to(DEV)
    out = torch.empty_like(q)
    kv.attn(q, out, c.cu)
    assert kv.poll_device_status() == 0
    kv._keep[2][0, 1] = -1
    kv.attn(q, out, c.cu)
    assert kv.poll_device_status() == 64 and kv.poll_device_status() == 0
    cache = lar.Cache(lar.make_config(n_layers=1, batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, dtype="bf16", cond_len=3, line_width=8, n_lines=4,
                                      anchor_len=8, recent_lines=1, budget_lines=4))
    assert cache.paged_view(0).poll_device_status() == 0
    view = cache.paged_view(0)
    view.attn(q, out, c.cu)                                # an empty cache: the chunk is longer than it
    assert view.poll_device_status() == 64 and cache.poll_device_status() == 0
    cache.close()


# ------------------------------------------------------------------------------------ views, and calls behind each other
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout", ["interleaved", "heads outermost", "one head's pages"])
@pytest.mark.parametrize("d,hkv,hq,n", [(64, 2, 4, [1, 3]), (128, 2, 8, [1, 2]), (64, 3, 3, [40, 9]), (128, 2, 4, [150, 7]), (128, 1, 1, [1, 1])])
def test_attention_of_views(dtype, layout, d, hkv, hq, n):
    """q in a fused projection or head-major, out head-major, pools in one tensor or heads outermost, the table and the lengths
    parts of larger tensors: strides of the tensor maps on the bf16 path."""
    page, lens = 32, [300, 170]
    T, cols = sum(n), 10
    heads, per_head = (1, True) if layout == "one head's pages" else (hkv, False)
    pages = 2 * cols * (hkv if per_head else 1)
    base = _randn({"interleaved": (pages, 2, page, heads, d), "heads outermost": (2, heads, pages, page, d),
                   "one head's pages": (pages, page, 2, 1, d)}[layout], dtype, 1)
    dev = base.to(DEV)

    def pools(x):
        if layout == "interleaved":
            return x[:, 0], x[:, 1]
        if layout == "heads outermost":
            return x[0].permute(1, 2, 0, 3), x[1].permute(1, 2, 0, 3)
        return x[:, :, 0], x[:, :, 1]
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).int()
    table = ids.view(2, hkv, cols) if per_head else ids.view(2, cols)
    wide = torch.full((4, *table.shape[1:-1], cols + 3), -1, dtype=torch.int32)
    wide[::2, ..., 1:cols + 1] = table
    lens3 = torch.tensor([lens[0], -1, -1, lens[1]], dtype=torch.int32, device=DEV)
    kv = lar.PagedKV(*pools(dev), wide.to(DEV)[::2, ..., 1:cols + 1], lens3[::3], hkv)
    cu = torch.tensor([0, n[0], T], dtype=torch.int32, device=DEV)
    kc, vc = pools(base)
    at = lambda s, h, j: (int(table[s, h, j // page] if per_head else table[s, j // page]), j % page, 0 if per_head else h)
    rows = lambda pool: (lambda s, h, a, b: torch.stack([pool[at(s, h, j)] for j in range(a, b)]))
    fused, major = _randn((T, hq + 2 * hkv, d), dtype, 3), _randn((hq, T, d), dtype, 4)
    for q, qd in ((fused[:, :hq], fused.to(DEV)[:, :hq]), (major.transpose(0, 1), major.to(DEV).transpose(0, 1))):
        for workspace in (False, True):
            out = torch.full((hq, T + 1, d), 5.0, dtype=dtype, device=DEV)
            ws = kv.attn_workspace(hq, T, max(n), 300) if workspace else None
            kv.attn(qd, out[:, :T].transpose(0, 1), cu, max_chunk=max(n), max_len=300, workspace=ws)
            ref, mag, big = R.attention(q, rows(kc), rows(vc), n, lens, None, True, hq // hkv, d ** -0.5)
            _assert_close(out[:, :T].transpose(0, 1), ref, R.attention_tolerance(dtype, ref, mag, big, d, 300), f"workspace {workspace}")
            assert (out[:, T:] == 5.0).all()
    assert kv.poll_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 1, 1], [5, 0, 20], [160, 1, 90]])
def test_unlike_calls_share_a_workspace_one_behind_the_other(dtype, n):
    """Calls with other queries, lengths, caches and outputs queued on one workspace without a wait between them, eagerly and as
    graphs on a side stream: parts left by the call before must not be met."""
    hq, hkv, d = 8, 2, 64
    T, ws = sum(n), None
    calls = []
    for i, lens in enumerate(([3000, 2500, 2900], [160, 1, 700], [2049, 2900, 90], [3000, 3000, 3000])):
        c = PagedCase(dtype, d, hkv, 64, "nhd", n, lens, seed=i, extra_cols=50)
        for p, x in zip(c.pools, c.dev):
            x.normal_()
            p.copy_(x.cpu())
        q = _randn((T, hq, d), dtype, 70 + i)
        ref, mag, big = R.attention(q, c.rows(0), c.rows(1), n, lens, None, True, hq // hkv, d ** -0.5)
        calls.append((c, q.to(DEV), ref, R.attention_tolerance(dtype, ref, mag, big, d, 3000)))
        ws = ws if ws is not None else c.kv.attn_workspace(hq, T, max(n), 3000)

    def run(i, out):
        c, q = calls[i][:2]
        c.kv.attn(q, out, c.cu, max_chunk=max(n), max_len=3000, workspace=ws)
    order = [0, 1, 2, 3, 1, 0, 3, 2, 2, 0]
    outs = [torch.full((T, hq, d), 5.0, dtype=dtype, device=DEV) for _ in order]
    ws.fill_(255)
    for i, out in zip(order, outs):
        run(i, out)
    torch.cuda.synchronize()
    check = lambda: [_assert_close(out, calls[i][2], calls[i][3], f"call {i}") for i, out in zip(order, outs)]
    check()
    side, graphs = torch.cuda.Stream(), []
    for i, out in zip(order, outs):
        out.fill_(5.0)
    torch.cuda.synchronize()
    for i, out in zip(order, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            run(i, out)
        graphs.append(g)
    with torch.cuda.stream(side):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    check()
    assert all(int(c.status) == 0 for c, *_ in calls)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,lens", [([1, 3], [700, 90]), ([1, 1], [3000, 2100]), ([12, 1], [700, 1500]), ([40, 2], [700, 1500]), ([150, 1], [2500, 700])])
def test_attention_of_enormous_logits(dtype, d, n, lens):
    """Logits of 10^9 to 10^30: the products are exact (one element of q is not zero) and lie so far apart that each row is the value
    row of its largest logit -- and of the slots that share it, half and half."""
    page, hq = 32, 2
    for power in (0, 20, 70):                            # the largest logits: about 2^30, 2^50, 2^100
        c = PagedCase(dtype, d, 1, page, "nhd", n, lens, seed=power)
        c.fill(None, 5)
        g = torch.Generator().manual_seed(power)
        best = []
        for s, length in enumerate(lens):
            keys = torch.randperm(length, generator=g).float().bfloat16().float() + 4096.0      # (some are equal once rounded)
            keys = keys.bfloat16().float()
            best.append(keys)
            for j in range(length):
                row = c.pools[0][c.place(s, 0, j)]
                row.zero_()
                row[3] = keys[j] * 2.0 ** (17 + power // 2)
        for p, x in zip(c.pools, c.dev):
            x.copy_(p.to(DEV))
        T = sum(n)
        q = torch.zeros(T, hq, d, dtype=dtype)
        q[:, 0, 3], q[:, 1, 3] = 2.0 ** (power - power // 2 + 3), -(2.0 ** (power - power // 2 + 3))
        for workspace in (False, True):
            out = torch.full((T, hq, d), 5.0, dtype=dtype, device=DEV)
            ws = c.kv.attn_workspace(hq, T, max(n), max(lens)) if workspace else None
            c.kv.attn(q.to(DEV), out, c.cu, max_chunk=max(n), max_len=max(lens), workspace=ws)
            t = 0
            for s, a in enumerate(n):
                V = c.rows(1)(s, 0, 0, lens[s]).double()
                for i in range(a):
                    seen = best[s][:lens[s] - a + i + 1]
                    for h, top in ((0, seen.max()), (1, seen.min())):
                        at = (seen == top).nonzero()[:, 0]
                        ref = V[at].mean(0)
                        # weights are 1 each: the sum of the value rows (fp32, in 22 bits each) and its quotient, rounded to the storage type
                        tol = V[at].abs().mean(0) * (2.0 ** -20) + (ref.abs() * 2.0 ** -8 if dtype == BF else 0) + 1e-12
                        _assert_close(out[t + i, h], ref, tol, f"2^{power} seq {s} token {i} head {h} workspace {workspace}")
                t += a
    assert int(c.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 1], [9, 1], [40, 5]])
def test_offsets_beyond_32_bits(dtype, n):
    """Pages, tokens and heads that lie 2^30 and 2^31 elements apart: appended to and attended over."""
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 35 GB")
    d, hkv, hq, page, far = 64, 2, 4, 64, 1 << 30
    T, lens = sum(n), [300, 3 * page]
    buf = torch.empty(4 * far + (1 << 23), dtype=dtype, device=DEV)
    pool = lambda at: buf.as_strided((5, page, hkv, d), (far, hkv * d, d, 1), at)
    rows = lambda heads, at: buf.as_strided((T, heads, d), (heads * d, far, 1) if heads == 4 else (heads * d, d, 1), at)
    table = torch.tensor([[4, 1, 3, 0, 2], [-1] * 5], dtype=torch.int32)
    table[1, :3] = torch.tensor([2, 4, 3])                # (pages of their own and pages shared with the first sequence)
    kp, vp = pool(0), pool(1 << 20)
    q, qo, out = rows(hq, 2 << 20), rows(hq, 3 << 20), rows(hq, 4 << 20)
    k, v = rows(hkv, 5 << 20), rows(hkv, (5 << 20) + (4 * far))
    host = {}
    for name, x in (("kp", kp), ("vp", vp), ("q", q), ("k", k), ("v", v)):
        host[name] = _randn(tuple(x.shape), dtype, len(host))
        x.copy_(host[name].to(DEV))
    start = [0, 128]                                      # (what the second sequence sees lies in its own rows)
    c = torch.tensor([0, n[0], T], dtype=torch.int32, device=DEV)
    kv = lar.PagedKV(kp, vp, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), hkv)
    rope, pos = lar.make_rope(d, (32,)), _pos(1, T, 5)
    kv.append_rope(k, v, c, rope, pos.to(DEV), q, qo)
    turned = {x: R.rotate(host[x], pos, (32,), 10000.0, False, False) for x in ("q", "k")}
    _assert_close(qo, turned["q"], R.rotation_tolerance(dtype, turned["q"], host["q"], False), "q")
    t = 0
    tol = torch.zeros(5, page, hkv, d, dtype=torch.float64)
    for s, a in enumerate(n):
        for i in range(a):
            j = lens[s] - a + i
            at = int(table[s, j // page]), j % page
            host["kp"][at], host["vp"][at] = turned["k"][t].to(dtype), host["v"][t]
            tol[at] = R.rotation_tolerance(dtype, turned["k"][t:t + 1], host["k"][t:t + 1], False)[0] + turned["k"][t].abs() * 2.0 ** -8 * (dtype == BF)
            t += 1
    assert torch.equal(vp.cpu(), host["vp"])
    _assert_close(kp, host["kp"].double(), tol + 1e-12 * (tol > 0), "keys")
    seen = [kp.cpu(), vp.cpu()]
    get = lambda which: (lambda s, h, a, b: torch.stack([seen[which][int(table[s, j // page]), j % page, h] for j in range(a, b)]))
    ref, mag, big = R.attention(qo.cpu(), get(0), get(1), n, lens, start, True, hq // hkv, d ** -0.5)
    for workspace in (False, True):
        ws = kv.attn_workspace(hq, T, max(n), 300) if workspace else None
        kv.attn(qo, out, c, kv_start=torch.tensor(start, dtype=torch.int32, device=DEV), max_chunk=max(n), max_len=300, workspace=ws)
        _assert_close(out, ref, R.attention_tolerance(dtype, ref, mag, big, d, 300), "out")
    assert kv.poll_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,length", [(1, 3000), (9, 700), (12, 1500), (40, 1500), (150, 2500)])
@pytest.mark.parametrize("base,step", [(2.0 ** 20, 1.0), (2.0 ** 26, 8.0), (2.0 ** 29, 64.0), (-(2.0 ** 29), 64.0)])
def test_attention_of_large_logits_that_lie_close(dtype, d, n, length, base, step):
    """Logits base + step k (exact in fp32) with k growing along the cache, and values that shrink as the weights grow: slots of
    every level count, so the references of all tiles, parts and splits have to agree far below the logits' own rounding."""
    c = PagedCase(dtype, d, 1, 64, "nhd", [n], [length], seed=n)
    c.fill(None, 6)
    scale = 0.125
    levels = 6
    level = torch.arange(length) * levels // length                       # 0 .. levels - 1
    for j in range(length):
        at = c.place(0, 0, j)
        c.pools[0][at] = 0.0
        c.pools[0][at][0], c.pools[0][at][1] = base / 1024, step / 8 * float(level[j])
        c.pools[1][at] *= math.exp(-step * scale * float(level[j]))
    for p, x in zip(c.pools, c.dev):
        x.copy_(p.to(DEV))
    q = torch.zeros(n, 2, d, dtype=dtype)
    q[..., 0], q[..., 1] = 1024.0, 8.0
    V = c.rows(1)(0, 0, 0, length).double()
    weight = torch.exp(step * scale * (level - (levels - 1)).double())
    # A weight's argument is at most step scale levels, rounded a few times; sums of 3000 terms and the tensor core's cut-off sums
    # (2^-21 each); bf16: weights rounded once, and the result.
    rel = step * scale * levels * 2.0 ** -21 + 3000 * 2.0 ** -24 + 2.0 ** -16
    for workspace in (False, True):
        out = torch.full((n, 2, d), 5.0, dtype=dtype, device=DEV)
        ws = c.kv.attn_workspace(2, n, n, length) if workspace else None
        c.kv.attn(q.to(DEV), out, c.cu, softmax_scale=scale, max_chunk=n, max_len=length, workspace=ws)
        for i in range(n):
            hi = length - n + i + 1
            w = weight[:hi] / weight[:hi].sum()
            ref, mag = w @ V[:hi], w @ V[:hi].abs()
            tol = mag * rel + (mag * 2.0 ** -8 + ref.abs() * 2.0 ** -8 if dtype == BF else 0)
            _assert_close(out[i, 0], ref, tol, f"token {i} workspace {workspace}")
            assert torch.equal(out[i, 0], out[i, 1])
    assert int(c.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [(BF, 1), (BF, 40), (BF, 160), (F32, 1)])
def test_first_call_of_a_thread(dtype, n):
    """A thread that has made no CUDA call yet: attention (a tensor map is encoded), append and rotation."""
    c = PagedCase(dtype, 64, 1, 64, "nhd", [n], [300])
    c.fill(None, 1)
    q, pos, rope = _randn((n, 2, 64), dtype, 1).to(DEV), torch.zeros(1, n, dtype=torch.int32, device=DEV), lar.make_rope(64, (32,))
    want, out, k = torch.empty_like(q), torch.empty_like(q), c.dev[0].new_zeros(n, 1, 64)
    c.kv.attn(q, want, c.cu)
    errors = []

    def call(what):
        try:
            what()
        except Exception as e:                                        # noqa: BLE001 -- shown by the test
            errors.append(e)
    for what in (lambda: c.kv.attn(q, out, c.cu), lambda: lar.rope_rotate(rope, pos, q, q), lambda: c.kv.append_rope(k, k, c.cu, rope, pos)):
        t = threading.Thread(target=call, args=(what,))
        t.start()
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 20, 160])                              # few rows, one and two row tiles
def test_attention_from_two_threads(n):
    """Calls of one kernel with different amounts of shared memory from two threads at once, on streams and outputs of their own."""
    d, hkv, hq = 64, 1, 4
    work, fn = [], lar._fast().lar_paged_attn
    for seqs, length in ((1, 300), (900, 200)):
        pools = [torch.randn(seqs * 5, 64, hkv, d, device=DEV, generator=torch.Generator(DEV).manual_seed(seqs + i)).to(BF) for i in range(2)]
        table = torch.arange(seqs * 5, dtype=torch.int32, device=DEV).view(seqs, 5)
        kv = lar.PagedKV(*pools, table, torch.full((seqs,), length, dtype=torch.int32, device=DEV), hkv)
        T = 900                                                          # (the few tokens of one of the calls keep the GPU's queue short)
        cu = (torch.arange(seqs + 1, device=DEV) * n).clamp(max=T).int()
        q = torch.randn(T, hq, d, device=DEV).to(BF)
        outs = [torch.zeros_like(q) for _ in range(2)]
        kv.attn(q, outs[0], cu, max_chunk=n, max_len=length)
        work.append((kv, q, cu, outs, length, torch.cuda.Stream()))
    torch.cuda.synchronize()
    errors = []

    def loop(kv, q, cu, outs, length, stream):
        try:
            with torch.cuda.stream(stream):
                kv.attn(q, outs[1], cu, max_chunk=n, max_len=length)
            rows = [lar.lar_rows_t(x.data_ptr(), x.stride(0), x.stride(1)) for x in (q, outs[1])]
            args = (kv._at, C.addressof(rows[0]), C.addressof(rows[1]), hq, q.shape[0], cu.data_ptr(), None, 1, 0.0, n, length, None, 0, stream.cuda_stream)
            errors.extend(s for s in (fn(*args) for _ in range(4000)) if s)
        except Exception as e:                                        # noqa: BLE001 -- shown by the test
            errors.append(e)
    threads = [threading.Thread(target=loop, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, (len(errors), errors[:4])
    for kv, q, cu, outs, length, stream in work:
        assert torch.equal(outs[0], outs[1]) and kv.poll_device_status() == 0


@pytest.mark.gpu
def test_rotated_prefill_refuses_a_layer_that_is_not_empty():
    """With the call-order checks off a step may come before the prefix: the prefill would take its rows for its own."""
    cfg = lar.make_config(n_layers=2, batch=1, n_q_heads=2, n_kv_heads=2, head_dim=64, dtype="bf16", cond_len=3, line_width=8, n_lines=4, anchor_len=8,
                          recent_lines=1, budget_lines=4, flags=lar.LAR_FLAG_NO_HOST_CHECKS)
    cache = lar.Cache(cfg)
    x = torch.zeros(1, 2, 64, dtype=BF, device=DEV)
    rows = torch.zeros(3, 2, 64, dtype=BF, device=DEV)
    cache.decode_step(0, x, x, x, torch.empty_like(x))
    with pytest.raises(lar.LarError) as e:
        cache.append_kv_rope(0, rows, rows, 3)
    assert e.value.status == lar.LAR_ERR_BAD_STATE
    assert (cache.get_state(0)[0] == 1).all()
    cache.append_kv_rope(1, rows, rows, 3)
    assert (cache.get_state(1)[0] == 3).all()
    cache.close()
