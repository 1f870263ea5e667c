"""Head norms with the rotation, the 8-bit paged cache (append, read back) and the attention over it, against plain 64-bit forms on the
sizes and masks where they can go wrong; refusals run without a GPU."""
import ctypes as C

import pytest
import torch

import _paged_reference as R
import _q8_reference as Q
from _q8_reference import Cache8
from paper_2512_04857_b200 import lar

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INVALID, OK = lar.LAR_ERR_INVALID_ARG, lar.LAR_OK


# ------------------------------------------------------------------------------------------------- refusals (no GPU)
def _norm(**kw):
    return lar.lar_head_norm_t(**{**dict(struct_size=C.sizeof(lar.lar_head_norm_t), kind=0, weight_dtype=0, eps=1e-6, weight=4096, bias=None,
                                         head_stride=0), **kw})


def _r(data=4096, token_stride=128, head_stride=64):
    return lar.lar_rows_t(data, token_stride, head_stride)


def _q8(k_scale=4096, v_scale=8192, sp=64, sh=32, struct_size=C.sizeof(lar.lar_paged_q8_t), reserved=0, **kw):
    kv = dict(struct_size=C.sizeof(lar.lar_paged_kv_t), dtype=lar.LAR_E4M3, n_seqs=2, n_kv_heads=2, head_dim=64, page_tokens=32, n_pages=8,
              table_cols=4, page_stride=2 * 32 * 64, row_stride=2 * 64, head_stride=64, k_pool=4096, v_pool=8192, page_table=256,
              table_seq_stride=4, table_head_stride=0, lens=512, lens_stride=1, status=None)
    kv.update(kw)
    return lar.lar_paged_q8_t(struct_size, reserved, lar.lar_paged_kv_t(**kv), k_scale, v_scale, sp, sh)


BAD_NORMS = [dict(struct_size=8), dict(kind=2), dict(kind=-1), dict(weight_dtype=2), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
             dict(eps=float("inf")), dict(weight=4104), dict(bias=4097), dict(head_stride=-64), dict(head_stride=4), dict(head_stride=32)]


@pytest.mark.parametrize("bad", BAD_NORMS)
def test_norm_refusals(bad):
    L, rope, rows = lar.lib(), lar.make_rope(64, (32,)), _r()
    for qn, kn in ((_norm(**bad), None), (None, _norm(**bad))):
        assert L.lar_norm_rope_rotate(qn, kn, rope, 0, 64, 256, 6, 6, rows, rows, 2, rows, rows, 2, None) == INVALID
        assert L.lar_paged_append_norm_rope(_q8(dtype=0).kv, qn, kn, rope, 256, 6, rows, rows, rows, rows, 2, 6, None, None) == INVALID
        assert L.lar_paged_q8_append(_q8(), 0, qn, kn, rope, 256, 6, rows, rows, rows, rows, 2, 6, None, None) == INVALID


def test_norm_rope_refusals():
    L, rope, rows, n = lar.lib(), lar.make_rope(64, (8, 12, 12)), _r(), _norm()

    def call(qn=n, kn=n, rope=rope, dtype=0, d=64, pos=256, ps=6, t=6, q=rows, qo=rows, hq=2, k=rows, ko=rows, hk=2):
        return L.lar_norm_rope_rotate(qn, kn, rope, dtype, d, pos, ps, t, q, qo, hq, k, ko, hk, None)
    assert call(dtype=2) == INVALID and call(d=96) == INVALID and call(d=128) == INVALID and call(t=-1) == INVALID
    assert call(pos=None) == INVALID and call(rope=None) == INVALID and call(ps=5) == INVALID and call(pos=258) == INVALID
    assert call(hq=0) == INVALID and call(hq=4097) == INVALID and call(hk=0) == INVALID and call(k=None) == INVALID
    assert call(k=None, ko=None, hk=0) == INVALID                     # a norm of keys that are not there
    assert call(q=_r(4100)) == INVALID and call(qo=_r(4096, 64, 64)) == INVALID and call(ko=None) == INVALID
    assert call(t=0) == OK and call(t=0, rope=None, pos=None) == OK
    kv = _q8(dtype=0).kv
    assert L.lar_paged_append_norm_rope(kv, n, None, None, None, 0, rows, rows, None, None, 0, 6, None, None) == INVALID   # a norm of no q
    assert L.lar_paged_append_norm_rope(None, n, None, None, None, 0, rows, rows, rows, rows, 2, 6, None, None) == INVALID
    assert L.lar_paged_append_norm_rope(kv, None, n, None, None, 0, rows, rows, None, None, 0, 7, None, None) == INVALID
    assert L.lar_paged_append_norm_rope(kv, None, n, None, None, 0, rows, rows, None, None, 0, 0, None, None) == OK
    assert L.lar_append_kv_norm_rope(None, 0, n, n, None, None, 0, rows, rows, rows, rows, 1, None) == INVALID


@pytest.mark.parametrize("bad", [
    dict(struct_size=8), dict(reserved=1), dict(dtype=0), dict(dtype=1), dict(dtype=3), dict(n_seqs=0), dict(head_dim=96), dict(page_tokens=48), dict(row_stride=72),
    dict(row_stride=48), dict(page_stride=2 * 32 * 64 + 8), dict(head_stride=0), dict(k_pool=4104), dict(v_pool=None), dict(lens=None),
    dict(k_scale=None), dict(v_scale=None), dict(k_scale=4104), dict(v_scale=8196), dict(sp=40), dict(sp=16), dict(sp=-64), dict(sh=0), dict(sh=16),
    dict(sh=40), dict(sh=-32), dict(head_stride=0, table_head_stride=8, sh=32),
])
def test_8bit_cache_refusals(bad):
    L, rows, c = lar.lib(), _r(), _q8(**bad)
    assert L.lar_paged_q8_append(c, 0, None, None, None, None, 0, rows, rows, None, None, 0, 6, None, None) == INVALID
    assert L.lar_paged_q8_read(c, 0, rows, rows, 6, None, None) == INVALID
    assert L.lar_paged_q8_attn(c, 0, rows, rows, 2, 6, None, None, 1, 0.0, 0, 0, None, 0, None) == INVALID
    assert L.lar_paged_q8_attn_workspace_bytes(c, 0, 2, 6, 0, 0) == 0


def test_8bit_call_refusals():
    L, rows, c = lar.lib(), _r(), _q8()
    assert L.lar_paged_q8_append(None, 0, None, None, None, None, 0, rows, rows, None, None, 0, 6, None, None) == INVALID
    assert L.lar_paged_q8_append(c, 2, None, None, None, None, 0, rows, rows, None, None, 0, 6, None, None) == INVALID
    assert L.lar_paged_q8_append(c, 0, None, None, None, None, 0, rows, rows, None, None, 0, 5, None, None) == INVALID
    assert L.lar_paged_q8_append(c, 0, None, None, None, None, 0, rows, rows, None, None, 0, 0, None, None) == OK
    assert L.lar_paged_q8_read(None, 0, rows, rows, 6, None, None) == INVALID and L.lar_paged_q8_read(c, 2, rows, rows, 6, None, None) == INVALID
    assert L.lar_paged_q8_read(c, 0, None, rows, 6, None, None) == INVALID and L.lar_paged_q8_read(c, 0, rows, _r(4096, 64, 64), 6, None, None) == INVALID
    assert L.lar_paged_q8_read(c, 0, rows, rows, 5, None, None) == INVALID and L.lar_paged_q8_read(c, 0, rows, rows, 6, 258, None) == INVALID
    assert L.lar_paged_q8_read(c, 0, rows, rows, 0, None, None) == OK

    def attn(c=c, dt=0, q=rows, o=rows, hq=2, n=6, cu=None, st=None, sc=0.0, mc=0, ml=0, ws=None, nb=0):
        return L.lar_paged_q8_attn(c, dt, q, o, hq, n, cu, st, 1, sc, mc, ml, ws, nb, None)
    assert attn(c=None) == INVALID and attn(dt=2) == INVALID and attn(hq=3) == INVALID and attn(hq=34) == INVALID and attn(n=5) == INVALID
    assert attn(sc=-1.0) == INVALID and attn(sc=float("nan")) == INVALID and attn(mc=-1) == INVALID and attn(ml=-1) == INVALID
    assert attn(cu=258) == INVALID and attn(st=258) == INVALID and attn(q=_r(4104)) == INVALID and attn(o=_r(None)) == INVALID
    assert attn(n=0) == OK
    assert attn(n=200, q=_r(), o=_r()) == lar.LAR_ERR_NOMEM                    # a long chunk without its workspace
    need = L.lar_paged_q8_attn_workspace_bytes(c, 0, 2, 200, 100, 0)
    assert need > 0 and attn(n=200, ws=4096, nb=16) == lar.LAR_ERR_NOMEM and attn(n=200, ws=4100, nb=need) == INVALID
    assert attn(c=_q8(n_seqs=1025), n=1025) == lar.LAR_ERR_CAPACITY
    assert L.lar_paged_q8_attn_workspace_bytes(c, 2, 2, 6, 0, 0) == 0 and L.lar_paged_q8_attn_workspace_bytes(None, 0, 2, 6, 0, 0) == 0


def test_binding_refuses_what_does_not_fit():
    x, w = torch.zeros(4, 2, 64), torch.zeros(64)
    with pytest.raises(lar.LarError):
        lar.HeadNorm("batch")
    with pytest.raises(lar.LarError):
        lar.HeadNorm("rms", w)                                             # not on a GPU
    with pytest.raises(lar.LarError):
        lar.norm_rope_rotate(None, None, x, x, q_norm=lar.HeadNorm("rms"))
    table, lens, pool = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(3, 16, 2, 64, dtype=torch.uint8)
    for k_scale in (torch.zeros(3, 16, 2, dtype=torch.uint8), torch.zeros(3, 2, 16), torch.zeros(3, 2, 32, dtype=torch.uint8)[..., ::2]):
        with pytest.raises(lar.LarError):
            lar.PagedKV8(pool, pool, k_scale, k_scale, table, lens, 2)
    with pytest.raises(lar.LarError):
        lar.PagedKV8(pool.float(), pool.float(), torch.zeros(3, 2, 16, dtype=torch.uint8), torch.zeros(3, 2, 16, dtype=torch.uint8), table, lens, 2)


@pytest.mark.parametrize("dtype", [lar.LAR_BF16, lar.LAR_FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,hkv", [(1, 2), (4, 8), (16, 1)])
def test_an_8bit_workspace_holds_for_smaller_calls(dtype, d, group, hkv):
    """Random pairs of calls: what the larger one asks for suffices for the smaller one (an OK launch shape is refused with NOMEM first)."""
    import random
    rng, L = random.Random(d + group + dtype), lar.lib()

    def cache(seqs, cols):
        return _q8(n_seqs=seqs, n_kv_heads=hkv, head_dim=d, page_tokens=64, n_pages=4096, table_cols=cols, page_stride=hkv * 64 * d,
                   row_stride=hkv * d, head_stride=d, sp=hkv * 64, sh=64, table_seq_stride=cols)
    for _ in range(400):
        big = [rng.randint(1, 40), rng.randint(1, 200), rng.choice([1, 2, 5, 16, 40, 200, 1000])]       # sequences, table entries, chunk
        small = [rng.randint(1, x) for x in big]
        need = [L.lar_paged_q8_attn_workspace_bytes(cache(s, c), dtype, group * hkv, s * t, t, 0) for s, c, t in (big, small)]
        assert need[1] <= need[0]


# ------------------------------------------------------------------------------------------------------------ norms
def _randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def _pos(axes, n, seed):
    return torch.randint(-100, 40000, (axes, n), generator=torch.Generator().manual_seed(seed)).to(torch.int32)


def _close(got, ref, tol, what=""):
    diff = (got.double().cpu() - ref).abs()
    bad = ~(diff <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((diff / tol)[bad].max()):.3g} bounds"


def _params(kind, heads, d, per_head, dtype, seed, bias):
    shape = (heads, d) if per_head else (d,)
    w = _randn(shape, F32, seed, 0.3).add_(1).to(dtype)
    b = _randn(shape, dtype, seed + 1, 0.2) if bias else None
    return w, b, lar.HeadNorm(kind, w.to(DEV), None if b is None else b.to(DEV), eps=1e-5)


AXES = {64: (8, 12, 12), 128: (16, 24, 24)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("wtype", [BF, F32])
@pytest.mark.parametrize("kind,bias,per_head", [("rms", False, False), ("layer", True, True), ("rms", True, True), ("layer", False, False)])
@pytest.mark.parametrize("d,hq,hk,n", [(64, 3, 1, 1), (128, 8, 2, 37), (64, 20, 20, 70), (128, 1, 0, 5), (128, 5, 3, 2500)])
def test_norm_and_rotation_of_rows(dtype, wtype, kind, bias, per_head, d, hq, hk, n):
    inter, restart = n % 2 == 1, n > 40
    x = _randn((n, hq + hk + 1, d), dtype, n + d)                       # rows with a gap behind each token
    x[0, 0] = 0                                                        # a row of zeros
    xd = x.to(DEV)
    pos, rope = _pos(3, n, 3), lar.make_rope(d, AXES[d], interleaved=inter, restart=restart)
    qw, qb, qn = _params(kind, hq, d, per_head, wtype, 5, bias)
    qo = torch.full((n, hq + 1, d), 7.0, dtype=dtype, device=DEV)
    args, kwargs = (xd[:, :hq], qo[:, :hq]), dict(q_norm=qn)
    if hk:
        kw, kb, kn = _params(kind, hk, d, per_head, wtype, 8, bias)
        ko = torch.empty(hk, n, d, dtype=dtype, device=DEV).transpose(0, 1)   # heads outermost
        args, kwargs = args + (xd[:, hq:hq + hk], ko), dict(q_norm=qn, k_norm=kn)
    for rotate in (True, False):
        lar.norm_rope_rotate(rope if rotate else None, pos.to(DEV) if rotate else None, *args, **kwargs)
        for got, rows, w, b in [(qo[:, :hq], x[:, :hq], qw, qb)] + ([(ko, x[:, hq:hq + hk], kw, kb)] if hk else []):
            ref, tol = Q.norm(rows, kind, w, b, 1e-5), Q.norm_tolerance(rows, kind, w, b, 1e-5)
            if rotate:
                ref, tol = Q.rotated(ref, tol, pos, AXES[d], 10000.0, inter, restart)
            _close(got, ref, Q.rounded(ref, tol, dtype), f"rotate {rotate}")
        assert (qo[:, hq] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_of_one_of_q_and_k_in_place(dtype):
    """No norm of q, one of k without weights; outputs on top of the inputs; another kind for each."""
    n, d = 19, 128
    x = _randn((n, 7, d), dtype, 1)
    pos, rope = _pos(1, n, 2), lar.make_rope(d, (64,))
    for kinds in ((None, "layer"), ("layer", None), ("rms", "layer")):
        xd = x.to(DEV)
        norms = [None if k is None else lar.HeadNorm(k) for k in kinds]
        lar.norm_rope_rotate(rope, pos.to(DEV)[0], xd[:, :4], xd[:, :4], xd[:, 4:], xd[:, 4:], q_norm=norms[0], k_norm=norms[1])
        for kind, rows in zip(kinds, (slice(0, 4), slice(4, 7))):
            ref, tol = x[:, rows].double(), torch.zeros(n, rows.stop - rows.start, d, dtype=torch.float64)
            if kind:
                ref, tol = Q.norm(x[:, rows], kind, None, None, 1e-6), Q.norm_tolerance(x[:, rows], kind, None, None, 1e-6)
            ref, tol = Q.rotated(ref, tol, pos, (64,), 10000.0, False, False)
            _close(xd[:, rows], ref, Q.rounded(ref, tol, dtype), str(kinds))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm_of_extreme_rows(kind):
    """Squares beyond fp32, rows far smaller than eps, rows with an infinity or a NaN next to ordinary ones."""
    x = _randn((1, 9, 128), F32, 4)
    for h, s in enumerate((1e30, 2e37, 1e19, 1e-25, 1e-3)):
        x[0, h] *= s
    x[0, 5, 17], x[0, 6, 3] = float("inf"), float("nan")
    x[0, 7] = 3.0e38
    out = torch.empty(1, 9, 128, device=DEV)
    lar.norm_rope_rotate(None, None, x.to(DEV), out, q_norm=lar.HeadNorm(kind))
    ref = Q.norm(x, kind, None, None, 1e-6)
    tol = Q.norm_tolerance(x, kind, None, None, 1e-6)
    fine = [0, 1, 2, 3, 4, 8] + ([7] if kind == "rms" else [])          # (a row of equal elements has nothing but rounding left after its mean)
    _close(out[:, fine], ref[:, fine], (tol + ref.abs() * 2.0 ** -24 + 1e-37)[:, fine])
    assert out[0, 6].isnan().all() and out[0, 5].isnan().any()


# ---------------------------------------------------------------------------------------------------- append, read
def _check_read(c, n, dtype, expect):
    """read(): the newest n[s] entries; expect(s) -> (K, V) values [hkv, n, d]."""
    T = sum(n)
    cu = torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=torch.int32, device=DEV)
    out = torch.full((T + 2, 2 * c.hkv + 1, c.d), 3.0, dtype=dtype, device=DEV)
    c.kv.read(out[:, :c.hkv], out[:, c.hkv:2 * c.hkv], cu)
    t = 0
    for s, a in enumerate(n):
        for i, want in enumerate(expect(s)):
            got = out[t:t + a, i * c.hkv:(i + 1) * c.hkv].transpose(0, 1).double().cpu()
            assert torch.equal(got.nan_to_num(9.0), want.nan_to_num(9.0)) and torch.equal(got.isnan(), want.isnan())
        t += a
    assert (out[T:] == 3.0).all() and (out[:, -1] == 3.0).all()


STORES = [("heads", 32, 128, 3, 6), ("nhd", 16, 64, 5, 0), ("hnd", 64, 128, 2, 8), ("nhd", 128, 64, 1, 4), ("heads", 16, 64, 20, 20)]
CHUNKS = [([1], [1]), ([1, 0, 1, 1], [64, 9, 65, 1]), ([0, 33, 7, 0, 130], [3, 33, 70, 0, 257])]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", STORES)
@pytest.mark.parametrize("n,lens", CHUNKS)
def test_8bit_append_and_read(dtype, layout, page, d, hkv, hq, n, lens):
    T, inter = sum(n), page == 16
    x = _randn((T + 2, hq + 2 * hkv, d), dtype, 5, 3.0)
    x[0, hq] = 0
    pos, rope = _pos(3, T + 2, 6), lar.make_rope(d, AXES[d], interleaved=inter)
    for kind in (None, "rms", "layer"):
        c = Cache8(d, hkv, page, layout, n, lens, seed=page + d)
        before = [y.clone() for y in c.pools + c.scales]
        xd = x.to(DEV)
        qn = kn = None
        qo = torch.full((T + 2, hq, d), 7.0, dtype=dtype, device=DEV) if hq else None
        if kind:
            kw, kb, kn = _params(kind, hkv, d, True, F32, 9, True)
            if hq:
                qw, qb, qn = _params(kind, hq, d, False, BF, 11, False)
        c.kv.append_norm_rope(xd[:, hq:hq + hkv], xd[:, hq + hkv:], c.cu, rope if kind else None, pos.to(DEV) if kind else None,
                              xd[:, :hq] if hq else None, qo, q_norm=qn, k_norm=kn)
        stored, t = {}, 0
        for s, a in enumerate(n):
            keys, vals = (x[t:t + a, hq + i * hkv:hq + (i + 1) * hkv].transpose(0, 1) for i in range(2))
            got_k, got_v = (c.get(s, i, lens[s] - a, lens[s]) for i in range(2))
            want = Q.quantise(vals)
            assert torch.equal(got_v[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got_v[1], want[1])
            if kind is None:
                want = Q.quantise(keys)
                assert torch.equal(got_k[0].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got_k[1], want[1])
            elif a:
                rows = x[t:t + a, hq:hq + hkv]
                ref, tol = Q.rotated(Q.norm(rows, kind, kw, kb, 1e-5), Q.norm_tolerance(rows, kind, kw, kb, 1e-5), pos[:, t:t + a], AXES[d], 10000.0, inter, False)
                # half a step: 2^-4 of a value, or 2^-10 of the scale below 2^-6 of it; a row whose largest element lies within tol of a border may have either scale
                exp = Q.quantise(ref + 0.0)[1].double() - 127
                step = torch.maximum((ref.abs() + tol) * 2.0 ** -4, 2.0 ** (exp + 1 - 10)[..., None])
                _close(Q.values(*got_k).transpose(0, 1), ref, tol + step, f"keys {kind}")
                border = Q.quantise(ref * (1 + 2.0 ** -18))[1] != Q.quantise(ref * (1 - 2.0 ** -18))[1]
                assert torch.equal(got_k[1].transpose(0, 1)[~border].double() - 127, exp[~border])
            stored[s] = (Q.values(*got_k), Q.values(*got_v))
            c.put(s, 0, lens[s] - a, before[0].new_full((hkv, a, d), 0x7f), before[2].new_full((hkv, a), 255))
            c.put(s, 1, lens[s] - a, before[0].new_full((hkv, a, d), 0x7f), before[2].new_full((hkv, a), 255))
            t += a
        assert all(torch.equal(a, b) for a, b in zip(before, c.pools + c.scales))     # every other row as it was
        if hq:
            ref, tol = x[:T, :hq].double(), torch.zeros(T, hq, d, dtype=torch.float64)
            if kind:
                ref, tol = Q.rotated(Q.norm(x[:T, :hq], kind, qw, qb, 1e-5), Q.norm_tolerance(x[:T, :hq], kind, qw, qb, 1e-5), pos[:, :T], AXES[d], 10000.0, inter, False)
            _close(qo[:T], ref, Q.rounded(ref, tol, dtype), "q")
            assert (qo[T:] == 7.0).all()
        # read back, into both types
        c.kv.append_norm_rope(xd[:, hq:hq + hkv], xd[:, hq + hkv:], c.cu, rope if kind else None, pos.to(DEV) if kind else None, k_norm=kn)
        for out_type in (BF, F32):
            _check_read(c, n, out_type, lambda s: stored[s])
        assert int(c.status) == 0


@pytest.mark.gpu
def test_8bit_rows_of_all_sizes():
    """Scales at both ends and at their borders, ties, infinities and NaN, through equal chunks without cu_tokens."""
    rows = [torch.full((64,), s) for s in (0.0, 448.0, 448.25, 449.0, 2.0 ** -126, 2.0 ** -149, 3.4028234663852886e38, 2.0 ** -109 * 1.75, 224.0, 1.0)]
    rows += [_randn((64,), F32, i, 2.0 ** e) for i, e in enumerate((-140, -120, -100, -20, 0, 60, 120))]
    rows.append(torch.linspace(-449, 449, 64))
    rows.append(torch.tensor([448.0] + [2.0 ** -9 * (i + 0.5) for i in range(31)] + [17.0 + 0.5 * i for i in range(32)]))   # ties
    bad = [_randn((64,), F32, 50 + i) for i in range(3)]
    bad[0][5], bad[1][63], bad[2][0] = float("inf"), float("nan"), -float("inf")
    x = torch.stack(rows + bad)
    x = torch.cat([x, x.flip(0)[:len(x) % 2]])                           # two sequences
    half = len(x) // 2
    c = Cache8(64, 1, 16, "nhd", [half, half], [half + 5, half])
    k, v = x[:, None].to(DEV), x[:, None].flip(0).contiguous().to(DEV)
    c.kv.append_rope(k, v)
    for s in range(2):
        for i, y in enumerate((x, x.flip(0))):
            want, got = Q.quantise(y[s * half:(s + 1) * half]), c.get(s, i, c.lens[s] - half, c.lens[s])
            assert torch.equal(got[1][0], want[1]) and torch.equal(got[0][0].view(torch.uint8), want[0].view(torch.uint8))
    ko, vo = torch.empty(2 * half, 1, 64, device=DEV), torch.empty(2 * half, 1, 64, device=DEV)
    c.kv.read(ko, vo)
    want = Q.values(*Q.quantise(x))
    assert torch.equal(ko[:, 0].double().cpu().nan_to_num(7.0), want.nan_to_num(7.0)) and ko[:, 0].isnan().any(1).sum() == want.isnan().all(1).sum()
    fine = torch.isfinite(x).all(1) & (x.abs().amax(1) > 2.0 ** -108)
    assert ((ko[:, 0].cpu().double() - x.double()).abs() <= torch.maximum(x.double().abs() * 2.0 ** -4, x.double().abs().amax(1, keepdim=True) * 2.0 ** -18))[fine].all()


@pytest.mark.gpu
def test_8bit_append_and_read_follow_no_bad_page_or_slot():
    c = Cache8(64, 2, 32, "nhd", [40, 3], [40, 10])
    c.table_dev[0, 1] = 10 ** 6                               # the second page of sequence 0
    c.lens_dev[1] = 2                                          # fewer entries than the chunk has tokens
    before = [y.clone() for y in c.pools + c.scales]
    x = _randn((43, 4, 64), BF, 1).to(DEV)
    c.kv.append_rope(x[:, :2], x[:, 2:], c.cu)
    assert int(c.status) == 64
    want = [Q.quantise(x[:, 2 * i:2 * i + 2].cpu()) for i in range(2)]
    for i in range(2):
        pool, scale = before[i], before[2 + i]
        for rows, page in ((slice(0, 32), int(c.table[0, 0, 0])), (slice(41, 43), int(c.table[1, 0, 0]))):
            m = rows.stop - rows.start                         # tokens 1 and 2 of the second chunk have slots 0 and 1
            pool[page, :m] = want[i][0][rows].view(torch.uint8).to(DEV)
            scale[page, :, :m] = want[i][1][rows].T.to(DEV)
        assert torch.equal(pool, c.pools[i]) and torch.equal(scale, c.scales[i])
    c.status.zero_()
    out = torch.full((43, 4, 64), 5.0, device=DEV)
    c.kv.read(out[:, :2], out[:, 2:], c.cu)
    assert int(c.status) == 64 and (out[32:41] == 0).all()     # a page outside the pool, a slot before the first: zeros
    for i in range(2):
        v = Q.values(*want[i]).float().to(DEV)
        assert torch.equal(out[:32, 2 * i:2 * i + 2], v[:32]) and torch.equal(out[41:, 2 * i:2 * i + 2], v[41:])


# ------------------------------------------------------------------------------------------------------- attention
LENGTHS = [([1], [1]), ([1, 1, 0, 1], [63, 64, 9, 65]), ([1, 1], [700, 129]), ([3, 0, 17, 2], [3, 0, 130, 257]), ([40, 1, 130], [40, 300, 200]),
           ([300, 5], [310, 5])]
SHAPES = [("heads", 32, 128, 2, 4), ("nhd", 64, 64, 2, 2), ("hnd", 16, 128, 1, 8), ("nhd", 128, 128, 3, 3), ("heads", 64, 64, 1, 3), ("hnd", 32, 64, 1, 16),
          ("heads", 16, 64, 2, 4)]


def _check_attention(c, hq, dtype, causal, start, workspace, seed, hints=True, q=None, scale=0.0, equal_chunks=False):
    T, d, group = sum(c.n), c.d, hq // c.hkv
    q = _randn((T + 2 * (not equal_chunks), hq, d), dtype, seed) if q is None else q
    buf = torch.full((q.shape[0], hq + 1, d), 5.0, dtype=dtype, device=DEV)     # out is a view with a gap behind each token
    out = buf[:, :hq]
    mc, ml = hints if isinstance(hints, tuple) else (max(c.n), max(c.lens)) if hints else (0, 0)
    # The bound of the chunks decides which kernels a call takes: above 64 bf16 rows per KV head those of bf16 caches, which round a weight to bf16
    # (2^-8 of it, and the sum over the weights' magnitudes 2^-8 of mag), the others to fp16 (2^-11; two of them for fp32 rows).
    few = dtype == F32 or (mc or -(-q.shape[0] // len(c.n))) * group <= 64
    ws = c.kv.attn_workspace(hq, q.shape[0], mc, ml, dtype=dtype) if workspace or not few else None
    if ws is not None:
        ws.fill_(255)
    sd = torch.tensor(start, dtype=torch.int32, device=DEV) if start is not None else None
    c.kv.attn(q.to(DEV), out, None if equal_chunks else c.cu, causal=causal, kv_start=sd, softmax_scale=scale, max_chunk=mc, max_len=ml, workspace=ws)
    ref, mag, big = R.attention(q[:T], c.rows(0), c.rows(1), c.n, c.lens, start, causal, group, scale or d ** -0.5)
    vmax = max([float(v.abs().nan_to_num().max()) for v in c.vals[1] if v.numel()] + [0.0])
    tol = torch.maximum(Q.attention_tolerance(dtype, ref, mag, big, d, max(c.lens), vmax),
                        R.attention_tolerance(dtype, ref, mag, big, d, max(c.lens)) if not few else torch.zeros(()))
    _close(out[:T], ref, tol, f"causal {causal} start {start} workspace {ws is not None}")
    assert (out[T:] == 5.0).all() and (buf[:, hq:] == 5.0).all()
    assert int(c.status) == 0
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", SHAPES)
@pytest.mark.parametrize("n,lens", LENGTHS)
def test_8bit_attention(dtype, layout, page, d, hkv, hq, n, lens):
    c = Cache8(d, hkv, page, layout, n, lens, seed=d + page)
    c.fill(3)
    for causal in (True, False):
        for workspace in (False, True):
            _check_attention(c, hq, dtype, causal, None, workspace, 11)
    _check_attention(c, hq, dtype, True, None, True, 12, hints=False)
    _check_attention(c, hq, dtype, True, None, True, 12, hints=(1, 0))       # a bound of the chunks that does not hold chooses another launch shape
    _check_attention(c, hq, dtype, True, None, True, 12, hints=(10 ** 6, 10 ** 6))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,lens,start", [([2, 1, 4], [40, 70, 4], [7, 64, 4]), ([1, 1], [1300, 900], [40, 899]), ([40, 9, 20], [60, 90, 20], [20, 90, 0]),
                                          ([3, 3], [5, 5], [100, -3])])
def test_8bit_attention_with_left_padding(dtype, n, lens, start):
    """Rows whose mask leaves nothing are zero; what lies before the start is NaN."""
    for d, hkv, hq, layout in ((128, 2, 4, "nhd"), (64, 1, 2, "heads")):
        c = Cache8(d, hkv, 32, layout, n, lens, seed=1)
        c.fill(5, start=start)
        for causal in (True, False):
            out = _check_attention(c, hq, dtype, causal, start, True, 21)
            for s, (a, b) in enumerate(zip(n, lens)):
                if start[s] >= b:
                    assert (out[sum(n[:s]):sum(n[:s + 1])] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,lens", [([1, 1], [2500, 800]), ([2, 5, 3], [1500, 3000, 40]), ([40, 1], [1200, 700])])
def test_8bit_attention_of_values_of_unlike_sizes(dtype, d, n, lens):
    """Rows of K up to 2^6 apart, rows of V up to 2^40 apart: what counts is the row's largest weight times value."""
    c = Cache8(d, 2, 32, "nhd", n, lens, seed=2)
    c.fill(7, spread=6.0)
    small = [c.vals[0], None]
    c.fill(8, spread=40.0)
    for s in range(len(n)):                          # keys of the first filling, values of the second
        codes, byte = Q.quantise(small[0][s].float())
        c.put(s, 0, 0, codes, byte)
    c.vals[0] = small[0]
    _check_attention(c, 4, dtype, True, None, True, 3)
    # a slot with enormous values that the softmax leaves out: its weight is 2^-90, the others' values have all their bits
    g = torch.Generator().manual_seed(3)
    for s, L in enumerate(lens):
        keys, vals = torch.randn(2, L, d, generator=g) * 0.05, torch.randn(2, L, d, generator=g)
        keys[:, 0, 0], vals[:, 0] = -120.0, vals[:, 0] * 2.0 ** 45
        for i, y in enumerate((keys, vals)):
            codes, byte = Q.quantise(y)
            c.put(s, i, 0, codes, byte)
            c.vals[i][s] = Q.values(codes, byte)
    q = _randn((sum(n) + 2, 4, d), dtype, 4, 0.1)
    q[:, :, 0] = 8.0
    got = _check_attention(c, 4, dtype, False, None, True, 3, q=q, scale=0.1)
    assert float(got[:sum(n)].abs().max()) < 10


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("base,step", [(2.0 ** 20, 1.0), (2.0 ** 26, 8.0), (-(2.0 ** 29), 64.0), (2.0 ** 31, 256.0)])
def test_8bit_attention_of_large_logits_that_lie_close(dtype, d, base, step):
    """Logits base + i step, exact in fp32: weights 2^-(i step scale log2 e), whatever base is."""
    L, n = 700, 3
    c = Cache8(d, 1, 32, "nhd", [n], [L])
    c.fill(1)
    keys = torch.zeros(1, L, d)
    i = torch.arange(L) % 13
    sign = 1.0 if base > 0 else -1.0
    keys[0, :, 0], keys[0, :, 1] = sign * 256.0, (i + 1).float()
    codes, byte = Q.quantise(keys)
    c.put(0, 0, 0, codes, byte)
    c.vals[0][0] = Q.values(codes, byte)
    assert torch.equal(c.vals[0][0].float(), keys)
    q = torch.zeros(n, 2, d)
    q[:, :, 0], q[:, :, 1] = abs(base) / 256.0, step
    q = q.to(dtype)
    ws = c.kv.attn_workspace(2, n, n, L, dtype=dtype)
    out = torch.empty(n, 2, d, dtype=dtype, device=DEV)
    scale = 1.0 / step
    c.kv.attn(q.to(DEV), out, softmax_scale=scale, max_chunk=n, max_len=L, workspace=ws)
    x = (i.double() * scale * step)
    for t in range(n):
        p = torch.softmax(x[:L - n + t + 1], 0)
        V = c.vals[1][0][0, :L - n + t + 1]
        ref, mag = p @ V, p @ V.abs()
        tol = mag * (2.0 ** -8 + 2.0 ** -14) + ref.abs() * 2.0 ** -7 if dtype == BF else mag * 2.0 ** -14
        _close(out[t], ref.expand(2, d), tol.expand(2, d), f"token {t}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 1], [3, 2], [30, 2]])
def test_8bit_attention_over_rows_that_are_not_finite(dtype, n):
    """A row stored from NaN or infinity makes the sequence's rows that see it NaN; other sequences, and rows of zeros, are as they should be."""
    lens = [300, 200]
    for which in range(2):
        c = Cache8(64, 2, 32, "hnd", n, lens, seed=3)
        c.fill(4)
        zero = Q.quantise(torch.zeros(2, 20, 64))
        c.put(1, which, 50, *zero)
        c.vals[which][1][:, 50:70] = 0
        bad = torch.randn(2, 1, 64)
        bad[:, 0, 3] = float("nan")
        c.put(0, which, 100, *Q.quantise(bad))
        c.vals[which][0][:, 100] = float("nan")
        q = _randn((sum(n), 4, 64), dtype, 5)
        out = torch.empty(sum(n), 4, 64, dtype=dtype, device=DEV)
        c.kv.attn(q.to(DEV), out, c.cu, max_chunk=max(n), max_len=300, workspace=c.kv.attn_workspace(4, sum(n), max(n), 300, dtype=dtype))
        assert out[:n[0]].isnan().all() and int(c.status) == 0
        ref, mag, big = R.attention(q, c.rows(0), c.rows(1), n, lens, None, True, 2, 0.125)
        tol = torch.maximum(Q.attention_tolerance(dtype, ref, mag, big, 64, 300, 10.0), R.attention_tolerance(dtype, ref, mag, big, 64, 300))
        _close(out[n[0]:], ref[n[0]:], tol[n[0]:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 1], [8, 3], [40, 20]])
def test_8bit_attention_reads_a_bad_page_as_zeros(dtype, n):
    lens = [100, 70]
    c = Cache8(64, 1, 16, "nhd", n, lens, seed=3)
    c.fill(4)
    c.table_dev[0, 2], c.table_dev[1, 0] = -1, c.kv.desc.kv.n_pages
    for i in range(2):
        c.vals[i][0][:, 32:48] = 0
        c.vals[i][1][:, :16] = 0
    q = _randn((sum(n), 2, 64), dtype, 5)
    out = torch.empty(sum(n), 2, 64, dtype=dtype, device=DEV)
    c.kv.attn(q.to(DEV), out, c.cu, max_chunk=max(n), max_len=100, workspace=c.kv.attn_workspace(2, sum(n), max(n), 100, dtype=dtype))
    ref, mag, big = R.attention(q, c.rows(0), c.rows(1), n, lens, None, True, 2, 0.125)
    _close(out, ref, torch.maximum(Q.attention_tolerance(dtype, ref, mag, big, 64, 100, 10.0), R.attention_tolerance(dtype, ref, mag, big, 64, 100)))
    assert c.kv.poll_device_status() == 64 and c.kv.poll_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 4, 50])
def test_8bit_attention_of_equal_chunks_in_batches(dtype, n):
    """No cu_tokens; long chunks over more sequences than are unpacked at a time."""
    S, L = (9, 700) if n < 50 else (5, 9000)
    c = Cache8(128, 2, 128, "nhd", [n] * S, [L - 3 * s for s in range(S)], extra_cols=0 if n < 50 else 240)
    c.fill(6)
    _check_attention(c, 4, dtype, True, None, True, 7, hints=(n, 0), equal_chunks=True)


@pytest.mark.gpu
def test_8bit_attention_repeats_itself():
    c = Cache8(128, 2, 32, "nhd", [1, 2, 1], [5000, 70, 3000])
    c.fill(6)
    q = _randn((4, 8, 128), BF, 1).to(DEV)
    ws = c.kv.attn_workspace(8, 4, 2, 5000)
    outs = []
    for i in range(4):
        ws.random_(0, 255)
        outs.append(torch.empty_like(q))
        c.kv.attn(q, outs[-1], c.cu, max_chunk=2, max_len=5000, workspace=ws)
    assert all(torch.equal(o, outs[0]) for o in outs)
