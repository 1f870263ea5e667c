"""Norms with the rotation on the way into caches of bf16 and fp32 rows, the caller's and the library's own, against plain 64-bit forms."""
import pytest
import torch

import _paged_reference as R
import _q8_reference as Q
from paper_2512_04857_b200 import lar
from test_norm_q8_ops import AXES, CHUNKS, STORES, _close, _params, _pos, _randn
from test_paged_ops import PagedCase

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _expected(rows, norm, pos, d, inter, restart=False):
    """fp64 rows and the tolerance of the fp32 ones before the last rounding.  norm: (kind, w, b), or None: rotation alone (2^-24 of a row of the storage type)."""
    y, tol = (rows.double(), torch.zeros(rows.shape, dtype=torch.float64)) if norm is None else (Q.norm(rows, *norm, 1e-5), Q.norm_tolerance(rows, *norm, 1e-5))
    return (y, tol) if pos is None else Q.rotated(y, tol, pos, AXES[d], 10000.0, inter, restart)


def _put(c, want, tols, which, s, ref, tol):
    """The tokens of sequence s (ref [n, hkv, d]) at their slots of what is expected of pool `which`."""
    a = ref.shape[0]
    for i in range(a):
        for h in range(c.hkv):
            at = c.place(s, h, c.lens[s] - a + i)
            want[which][at], tols[which][at] = ref[i, h], tol[i, h]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", STORES)
@pytest.mark.parametrize("n,lens", CHUNKS)
def test_norm_append_into_pages(dtype, layout, page, d, hkv, hq, n, lens):
    """Ragged chunks of a padded batch, rows of zeros, every kind and placing of norms; other rows of the cache stay as they were."""
    T, inter = sum(n), page == 16
    x = _randn((T + 2, hq + 2 * hkv, d), dtype, 5, 3.0)
    x[0, hq] = 0
    xd, pos = x.to(DEV), _pos(3, T + 2, 6)
    v = x[:, hq + hkv:].double()
    for q_kind, k_kind, rotated in (("rms", "rms", True), ("layer", "layer", True), (None, "rms", True), ("layer", None, True), ("rms", "layer", False)):
        if q_kind and not hq:
            q_kind, k_kind = None, k_kind or "layer"
        c = PagedCase(dtype, d, hkv, page, layout, n, lens, seed=page + d)
        qn = kn = q_norm = k_norm = None
        if q_kind:
            w, b, qn = _params(q_kind, hq, d, False, BF, 11, False)
            q_norm = (q_kind, w, b)
        if k_kind:
            w, b, kn = _params(k_kind, hkv, d, True, F32, 9, True)
            k_norm = (k_kind, w, b)
        qo = torch.full((T + 2, hq, d), 7.0, dtype=dtype, device=DEV) if hq else None
        rope = lar.make_rope(d, AXES[d], interleaved=inter) if rotated else None
        c.kv.append_norm_rope(xd[:, hq:hq + hkv], xd[:, hq + hkv:], c.cu, rope, pos.to(DEV) if rotated else None, xd[:, :hq] if hq else None, qo, q_norm=qn, k_norm=kn)
        ref, tol = _expected(x[:, hq:hq + hkv], k_norm, pos if rotated else None, d, inter)
        want = [p.double().clone() for p in c.pools]
        tols = [torch.zeros_like(p) for p in want]
        t = 0
        for s, a in enumerate(n):
            _put(c, want, tols, 0, s, ref[t:t + a], tol[t:t + a])
            _put(c, want, tols, 1, s, v[t:t + a], torch.zeros_like(v[t:t + a]))
            t += a
        for i in range(2):
            got, nan = c.dev[i].double().cpu(), want[i].isnan()
            assert torch.equal(got.isnan(), nan)
            if i == 0:
                _close(got[~nan], want[i][~nan], Q.rounded(want[i], tols[i], dtype)[~nan], f"keys {k_kind} {rotated}")
            else:
                assert torch.equal(got[~nan], want[i][~nan])
        if hq:
            ref, tol = _expected(x[:T, :hq], q_norm, pos[:, :T] if rotated else None, d, inter)
            _close(qo[:T], ref, Q.rounded(ref, tol, dtype), f"q {q_kind}")
            assert (qo[T:] == 7.0).all()
        assert int(c.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_norm_append_of_equal_chunks_from_and_to_views(dtype, d):
    """No cu_tokens; heads outermost in what goes in and comes out; q on top of itself; enough tokens for several of them a CTA."""
    n, S, hkv, hq, L = 900, 3, 1, 3, 950
    for inter in (False, True):
        c = PagedCase(dtype, d, hkv, 64, "nhd", [n] * S, [L - 7 * s for s in range(S)])
        x = _randn((hq + 2 * hkv, S * n, d), dtype, 3)
        xd, pos = x.to(DEV).transpose(0, 1), _pos(3, S * n, 4)
        norms = [("layer",) + _params("layer", h, d, False, F32, 2 + h, True) for h in (hq, hkv)]
        q = xd[:, :hq]
        c.kv.append_norm_rope(xd[:, hq:hq + hkv], xd[:, hq + hkv:], None, lar.make_rope(d, AXES[d], interleaved=inter, restart=True), pos.to(DEV), q, q,
                              q_norm=norms[0][3], k_norm=norms[1][3])
        y = x.transpose(0, 1)
        ref, tol = _expected(y[:, :hq], norms[0][:3], pos, d, inter, True)
        _close(q, ref, Q.rounded(ref, tol, dtype), "q")
        ref, tol = _expected(y[:, hq:hq + hkv], norms[1][:3], pos, d, inter, True)
        tol = Q.rounded(ref, tol, dtype)
        pools = [p.cpu() for p in c.dev]
        for s in range(S):
            j = torch.arange(L - 7 * s - n, L - 7 * s)
            at = c.table[s, 0][j // 64].long(), j % 64
            _close(pools[0][at], ref[s * n:(s + 1) * n], tol[s * n:(s + 1) * n], f"keys {s}")
            assert torch.equal(pools[1][at], y[s * n:(s + 1) * n, hq + hkv:])
        assert int(c.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_append_follows_no_bad_page_or_slot(dtype):
    c = PagedCase(dtype, 128, 2, 32, "nhd", [40, 3], [40, 10])
    c.kv._keep[2][0, 1] = 10 ** 6                              # the second page of sequence 0
    c.lens_dev[1] = 2                                          # fewer entries than the chunk has tokens
    before = [x.clone() for x in c.dev]
    x = _randn((43, 4, 128), dtype, 1)
    norm = lar.HeadNorm("rms", eps=1e-5)
    xd = x.to(DEV)
    c.kv.append_norm_rope(xd[:, :2], xd[:, 2:], c.cu, k_norm=norm)
    assert int(c.status) == 64
    ref, tol = _expected(x[:, :2], ("rms", None, None), None, 128, False)
    tol = Q.rounded(ref, tol, dtype)
    for rows, page in ((slice(0, 32), int(c.table[0, 0, 0])), (slice(41, 43), int(c.table[1, 0, 0]))):
        m = rows.stop - rows.start                             # tokens 1 and 2 of the second chunk have slots 0 and 1
        _close(c.dev[0][page, :m], ref[rows], tol[rows])
        for pool, old in zip(c.dev, before):
            old[page, :m] = pool[page, :m]
        assert torch.equal(c.dev[1][page, :m].cpu(), x[rows, 2:])
    for pool, old in zip(c.dev, before):                        # every other row as it was
        assert torch.equal(pool.nan_to_num(9.0), old.nan_to_num(9.0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_append_into_pages_far_apart(dtype):
    """Pages, tokens and heads 2^30 elements and more apart."""
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 18 GB")
    d, hkv, hq, page, far, T = 64, 2, 2, 64, 1 << 30, 5
    buf = torch.empty(4 * far + (1 << 23), dtype=dtype, device=DEV)
    pools = [buf.as_strided((5, page, hkv, d), (far, hkv * d, d, 1), at) for at in (0, 1 << 20)]
    for p in pools:
        p.fill_(7.0)
    x = [_randn((T, 2, d), dtype, i) for i in range(3)]
    at = [buf.as_strided((T, 2, d), (2 * d, 2 * far, 1), (2 + i) << 20) for i in range(3)]
    for a, b in zip(at, x):
        a.copy_(b.to(DEV))
    qo = buf.as_strided((T, 2, d), (far // 2, d, 1), 6 << 20)
    table = torch.tensor([[2, 4]], dtype=torch.int32)
    kv = lar.PagedKV(*pools, table.to(DEV), torch.tensor([page + 3], dtype=torch.int32, device=DEV), hkv)
    pos, norm = _pos(3, T, 2), lar.HeadNorm("rms", eps=1e-5)
    kv.append_norm_rope(at[1], at[2], None, lar.make_rope(d, AXES[d]), pos.to(DEV), at[0], qo, q_norm=norm, k_norm=norm)
    for got, rows in ((qo, x[0]), (torch.cat([pools[0][2, page - 2:], pools[0][4, :3]]), x[1])):
        ref, tol = _expected(rows, ("rms", None, None), pos, d, False)
        _close(got, ref, Q.rounded(ref, tol, dtype))
    assert torch.equal(torch.cat([pools[1][2, page - 2:], pools[1][4, :3]]).cpu(), x[2])
    for p in pools:
        assert (p[:2] == 7.0).all() and (p[2, :page - 2] == 7.0).all() and (p[4, 3:] == 7.0).all()
    assert kv.poll_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,inter", [(128, True), (128, False), (64, True)])
def test_norm_prefill_of_the_librarys_cache(dtype, d, inter):
    """Keys and values of the prefix where the layer's description says they are, from a prefix longer than a CTA's tokens."""
    S, Hq, Hkv, Cn, td = 2, 4, 2, 301, BF if dtype == "bf16" else F32
    cache = lar.Cache(lar.make_config(n_layers=1, batch=S, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, dtype=dtype, cond_len=Cn, line_width=8, n_lines=4,
                                      anchor_len=8, recent_lines=1, budget_lines=4, flags=lar.LAR_FLAG_SHUFFLE_PAGES, page_seed=3))
    x, pos = _randn((S * Cn, Hq + 2 * Hkv, d), td, 1), _pos(3, S * Cn, 2)
    xd, qo = x.to(DEV), torch.empty(S * Cn, Hq, d, dtype=td, device=DEV)
    kw, kb, kn = _params("layer", Hkv, d, True, BF, 9, True)
    cache.append_kv_rope(0, xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], Cn, lar.make_rope(d, AXES[d], interleaved=inter), pos.to(DEV), xd[:, :Hq], qo, k_norm=kn)
    lens, imap = cache.get_state(0)
    assert (lens == Cn).all() and (torch.from_numpy(imap[:, :Cn]) == torch.arange(Cn)).all()
    ref, tol = _expected(x[:, :Hq], None, pos, d, inter)
    _close(qo, ref, Q.rounded(ref, tol, td), "q")
    ref, tol = _expected(x[:, Hq:Hq + Hkv], ("layer", kw, kb), pos, d, inter)
    # queries that are each token's own key: a slot that held another key or value would weigh, or be weighed, otherwise
    k, v, off = ref.view(S, Cn, Hkv, d), x[:, Hq + Hkv:].view(S, Cn, Hkv, d), Q.rounded(ref, tol, td).view(S, Cn, Hkv, d)
    q = ref.repeat_interleave(Hq // Hkv, 1).to(td)
    out = torch.empty(S * Cn, Hq, d, dtype=td, device=DEV)
    cache.paged_view(0).attn(q.to(DEV), out, softmax_scale=0.25, max_chunk=Cn, max_len=Cn)
    get = lambda y: (lambda s, h, a, b: y[s, a:b, h])
    want, mag, big = R.attention(q, get(k), get(v), [Cn] * S, [Cn] * S, None, True, Hq // Hkv, 0.25)
    # keys are off by what the norm, the rotation and the last rounding are: a logit by the sum of |q| times that, a weight by e to twice as much
    _, _, less = R.attention(q, get(off), get(v), [Cn] * S, [Cn] * S, None, True, Hq // Hkv, 0.25)
    _close(out, want, R.attention_tolerance(td, want, mag, big, d, Cn) + torch.expm1(2 * less)[..., None] * 2 * mag, "attention")
    assert cache.poll_device_status() == 0
    cache.close()
