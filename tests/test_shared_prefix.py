"""Attention of sequences that have their first slots in common, against the plain 64-bit attention of each; refusals run without a GPU."""
import ctypes as C
import random

import pytest
import torch

import _paged_reference as R
from paper_2512_04857_b200 import lar
from test_paged_ops import PagedCase, _assert_close, _kv, _r, _randn

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INVALID, OK = lar.LAR_ERR_INVALID_ARG, lar.LAR_OK


# ------------------------------------------------------------------------------------------------- refusals (no GPU)
def _call(kv, q=None, out=None, hq=4, n=6, cu=None, groups=1, cug=256, sh=512, scale=0.0, mc=0, ml=0, ms=0, ws=None, nb=0):
    return lar.lib().lar_paged_attn_shared(kv, q or _r(), out or _r(1 << 20), hq, n, cu, groups, cug, sh, 1, scale, mc, ml, ms, ws, nb, None)


def test_shared_refusals():
    kv = _kv()
    for bad in (dict(struct_size=8), dict(dtype=2), dict(n_seqs=0), dict(head_dim=96), dict(page_tokens=48), dict(row_stride=32), dict(lens=None)):
        assert _call(_kv(**bad)) == INVALID
        assert lar.lib().lar_paged_attn_shared_workspace_bytes(_kv(**bad), 4, 6, 1, 0, 0, 0) == 0
    assert _call(None) == INVALID and _call(kv, hq=3) == INVALID and _call(kv, hq=34) == INVALID and _call(kv, n=5) == INVALID
    assert _call(kv, groups=0) == INVALID and _call(kv, groups=-1) == INVALID and _call(kv, cug=None) == INVALID and _call(kv, sh=None) == INVALID
    assert _call(kv, cug=258) == INVALID and _call(kv, sh=514) == INVALID and _call(kv, cu=258) == INVALID
    assert _call(kv, scale=-1.0) == INVALID and _call(kv, scale=float("inf")) == INVALID
    assert _call(kv, mc=-1) == INVALID and _call(kv, ml=-1) == INVALID and _call(kv, ms=-1) == INVALID
    assert _call(kv, q=_r(4104)) == INVALID and _call(kv, out=_r(1 << 20, 64, 64)) == INVALID
    assert _call(kv, n=0) == OK
    need = lar.lib().lar_paged_attn_shared_workspace_bytes(kv, 4, 6, 1, 0, 0, 0)
    assert need > 0 and _call(kv, ws=4096, nb=1024) == lar.LAR_ERR_NOMEM and _call(kv, ws=4100, nb=need) == INVALID
    assert _call(_kv(n_seqs=1025), n=1025) == lar.LAR_ERR_CAPACITY and _call(kv, groups=1025) == lar.LAR_ERR_CAPACITY
    with pytest.raises(lar.LarError):
        lar.PagedKV8.attn_shared(None)


@pytest.mark.parametrize("dtype", [lar.LAR_BF16, lar.LAR_FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,hkv", [(1, 2), (4, 8), (16, 1)])
def test_a_shared_workspace_holds_for_smaller_calls(dtype, d, group, hkv):
    """What a call needs is at most what lar_paged_attn_shared_workspace_bytes says of it, and that is at most what it says of a larger one.  Its
    own need: the smallest size that is not refused with NOMEM would launch a kernel, so only sizes one below the bound of the smaller are looked at."""
    rng, L = random.Random(d + group + dtype), lar.lib()

    def bytes_of(seqs, cols, chunk, groups, shared):
        kv = _kv(dtype=dtype, n_seqs=seqs, n_kv_heads=hkv, head_dim=d, page_tokens=64, n_pages=4096, table_cols=cols, page_stride=hkv * 64 * d,
                 row_stride=hkv * d, head_stride=d, table_seq_stride=cols)
        return L.lar_paged_attn_shared_workspace_bytes(kv, group * hkv, seqs * chunk, groups, chunk, 64 * cols, shared)
    for _ in range(400):
        big = [rng.randint(1, 60), rng.randint(1, 200), rng.choice([1, 2, 5, 16, 40, 200, 1000]), rng.randint(1, 8), rng.randint(1, 4000)]
        small = [rng.randint(1, x) for x in big]
        assert bytes_of(*small) <= bytes_of(*big)


# ------------------------------------------------------------------------------------------------------- attention
def _share(c, groups, shared, pages=True):
    """The first shared[g] slots of group g's sequences hold what those of its first one do: whole pages by the table, the rest as copies."""
    for (a, b), L in zip(groups, shared):
        for s in range(a + 1, b):
            if pages:
                c.table[s, :, :L // c.page] = c.table[a, :, :L // c.page]
            for j in range(L // c.page * c.page if pages else 0, L):
                for h in range(c.hkv):
                    for p in c.pools:
                        p[c.place(s, h, j)] = p[c.place(a, h, j)]
    tab = c.kv._keep[2]
    tab.copy_((c.table if c.layout == "heads" else c.table[:, 0]).to(DEV))
    for p, x in zip(c.pools, c.dev):
        x.copy_(p.to(DEV))


def _case(dtype, d, hkv, page, layout, n, lens, groups, shared, pages=True):
    c = PagedCase(dtype, d, hkv, page, layout, n, lens, seed=d + page)
    c.fill(None, 3)
    _share(c, groups, shared, pages)
    return c


def _check(c, hq, groups, said, causal=True, workspace=True, hints=True, seed=11, equal=False, q=None):
    T, d, dtype, pad = sum(c.n), c.d, c.dtype, 0 if equal else 2
    q = _randn((T + pad, hq, d), dtype, seed) if q is None else q
    buf = torch.full((T + pad, hq + 1, d), 5.0, dtype=dtype, device=DEV)     # out is a view with a gap behind each token
    out = buf[:, :hq]
    mc, ml, ms = hints if isinstance(hints, tuple) else (max(c.n), max(c.lens), max(0, *said)) if hints else (0, 0, 0)
    ws = c.kv.attn_shared_workspace(hq, T + pad, len(groups), mc, ml, ms) if workspace else None
    if ws is not None:
        ws.fill_(255)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    c.kv.attn_shared(q.to(DEV), out, dev([a for a, _ in groups] + [groups[-1][1]]), dev(said), None if equal else c.cu, causal, max_chunk=mc, max_len=ml,
                     max_shared=ms, workspace=ws)
    ref, mag, big = R.attention(q[:T], c.rows(0), c.rows(1), c.n, c.lens, None, causal, hq // c.hkv, d ** -0.5)
    # two sums joined: two exponentials (2^-22 each) and a rounding of each more than one sum
    tol = R.attention_tolerance(dtype, ref, mag, big, d, max(c.lens)) + mag * 2.0 ** -20
    _assert_close(out[:T], ref, tol, f"causal {causal} workspace {ws is not None} hints {hints}")
    assert (out[T:] == 5.0).all() and (buf[:, hq:] == 5.0).all()
    assert int(c.status) == 0
    return out


GROUPS = [
    # tokens, entries, groups, slots in common
    ([1], [1], [(0, 1)], [0]),
    ([1] * 5, [80, 65, 66, 90, 70], [(0, 5)], [64]),
    ([1, 2, 0, 3, 1], [140, 150, 9, 141, 137], [(0, 2), (2, 2), (2, 5)], [130, 77, 0]),
    ([2, 1, 1, 1, 1, 2], [40, 700, 650, 641, 300, 280], [(1, 4), (4, 6)], [640, 257]),        # the first sequence is of no group
    ([1, 1, 1], [300, 300, 40], [(0, 2)], [299]),                                              # nor is the last; nothing of their own but the chunk
    ([17, 9, 1, 20], [200, 190, 185, 210], [(0, 4)], [170]),
    ([40, 33, 70], [400, 390, 420], [(0, 3)], [320]),
]
SHAPES = [("heads", 32, 128, 2, 4), ("nhd", 64, 64, 2, 2), ("hnd", 16, 128, 1, 8), ("nhd", 128, 128, 3, 3), ("heads", 64, 64, 1, 3), ("hnd", 32, 64, 1, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,page,d,hkv,hq", SHAPES)
@pytest.mark.parametrize("n,lens,groups,shared", GROUPS)
def test_shared_attention(dtype, layout, page, d, hkv, hq, n, lens, groups, shared):
    c = _case(dtype, d, hkv, page, layout, n, lens, groups, shared, pages=d == 128)
    for causal in (True, False):
        _check(c, hq, groups, shared, causal)
    _check(c, hq, groups, shared, workspace=False)
    _check(c, hq, groups, shared, hints=False)
    for hints in ((1, 1, 1), (1, 0, 0), (10 ** 6, 10 ** 6, 10 ** 6)):       # bounds that do not hold choose another launch shape, no other result
        _check(c, hq, groups, shared, hints=hints)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_lengths_that_the_caches_do_not_hold(dtype):
    """More than the shortest cache held before its chunk: only that much is taken as common.  Negative: nothing."""
    n, lens, groups = [1, 3, 1, 2], [100, 90, 200, 120], [(0, 2), (2, 4)]
    c = _case(dtype, 64, 2, 16, "nhd", n, lens, groups, [87, 118])
    for said in ([87, 118], [88, 10 ** 6], [2 ** 31 - 1, 119], [-5, -1], [50, 2]):
        for causal in (True, False):
            _check(c, 4, groups, said, causal)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hkv,hq", [(128, 2, 8), (64, 2, 2)])
@pytest.mark.parametrize("seqs,tokens,common,own", [(40, 1, 2100, 300), (24, 3, 1500, 20), (70, 2, 700, 60), (9, 16, 3000, 40)])
def test_shared_attention_of_many_sequences(dtype, d, hkv, hq, seqs, tokens, common, own):
    """Row tiles of several sequences, slots in common that are spread over many CTAs."""
    rng = random.Random(seqs)
    n = [rng.randint(1, tokens) for _ in range(seqs)]
    lens = [common + max(a, rng.randint(1, own)) for a in n]
    groups = [(0, seqs // 3), (seqs // 3, seqs)]
    c = PagedCase(dtype, d, hkv, 64, "nhd", n, lens, seed=seqs)
    whole = common // 64
    for a, b in groups:                                                      # (before the filling, so that it fills one copy)
        c.table[a:b, :, :whole] = c.table[a:a + 1, :, :whole]
    g = torch.Generator().manual_seed(1)
    rows = [[torch.randn(hkv, L, d, generator=g).to(dtype) for L in lens] for _ in range(2)]
    for i in range(2):
        for a, b in groups:
            for s in range(a, b):
                rows[i][s][:, :whole * 64] = rows[i][a][:, :whole * 64]
        for s, L in enumerate(lens):
            j = torch.arange(L)
            page = c.table[s, 0][j // 64].long()
            c.pools[i][page, j % 64] = rows[i][s].transpose(0, 1)
        c.dev[i].copy_(c.pools[i].to(DEV))
    c.kv._keep[2].copy_(c.table[:, 0].to(DEV))
    c.rows = lambda i: (lambda s, h, j0, j1: rows[i][s][h, j0:j1])
    _check(c, hq, groups, [whole * 64, whole * 64 - 5])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_attention_of_equal_chunks(dtype):
    c = _case(dtype, 128, 1, 32, "hnd", [2] * 6, [70, 72, 80, 69, 100, 90], [(0, 3), (3, 6)], [64, 66])
    _check(c, 4, [(0, 3), (3, 6)], [64, 66], equal=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 1, 1], [9, 3, 20]])
def test_shared_attention_in_a_graph_of_a_growing_cache(dtype, n):
    """Captured once, replayed with other lengths, groups and slots in common; what an earlier replay left in the workspace does not matter."""
    lens = [200, 190, 230]
    c = _case(dtype, 64, 2, 16, "nhd", n, lens, [(0, 3)], [150])
    q = _randn((sum(n), 4, 64), dtype, 3)
    qd, out = q.to(DEV), torch.empty(sum(n), 4, 64, dtype=dtype, device=DEV)
    groups, shared = torch.tensor([0, 3], dtype=torch.int32, device=DEV), torch.tensor([150], dtype=torch.int32, device=DEV)
    ws = c.kv.attn_shared_workspace(4, sum(n), 1, max(n), 256, 200)
    run = lambda: c.kv.attn_shared(qd, out, groups, shared, c.cu, max_chunk=max(n), max_len=256, max_shared=200, workspace=ws)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for new_lens, cut, slots in ((lens, 3, 150), ([160, 170, 152 + 20], 3, 140), ([100, 110, 90], 2, 70), (lens, 1, 33)):
        c.lens = new_lens
        c.lens_dev.copy_(torch.tensor(new_lens, dtype=torch.int32))
        groups.copy_(torch.tensor([0, cut], dtype=torch.int32))
        shared.fill_(slots)
        graph.replay()
        ref, mag, big = R.attention(q, c.rows(0), c.rows(1), n, new_lens, None, True, 2, 0.125)
        _assert_close(out, ref, R.attention_tolerance(dtype, ref, mag, big, 64, 256) + mag * 2.0 ** -20, f"{new_lens}")
    assert int(c.status) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hints", [True, False])
def test_shared_attention_of_groups_whose_first_sequences_are_done(dtype, hints):
    """Sequences without tokens, whose pages and lengths are gone, in every place of a group."""
    n, lens, groups, said = [0, 0, 1, 2, 0, 1, 0, 0, 3, 0], [0, 0, 300, 290, 0, 310, 0, 0, 205, 0], [(0, 5), (5, 7), (7, 10)], [270, 300, 200]
    c = _case(dtype, 64, 2, 16, "nhd", n, lens, [(2, 4)], [270])
    for s, m in enumerate(n):
        if m == 0:
            c.kv._keep[2][s] = -1
    for causal in (True, False):
        _check(c, 4, groups, said, causal, hints=hints)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_attention_reports_bad_pages(dtype):
    c = _case(dtype, 64, 1, 16, "nhd", [1, 1], [100, 90], [(0, 2)], [80])
    c.kv._keep[2][0, 2] = -1                                                 # read for both sequences: zeros
    for p in c.pools:
        for s in range(2):
            for j in range(32, 48):
                p[c.place(s, 0, j)] = 0
    q = _randn((2, 2, 64), dtype, 5)
    out = torch.empty(2, 2, 64, dtype=dtype, device=DEV)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    c.kv.attn_shared(q.to(DEV), out, dev([0, 2]), dev([80]), c.cu, workspace=c.kv.attn_shared_workspace(2, 2, 1))
    ref, mag, big = R.attention(q, c.rows(0), c.rows(1), c.n, c.lens, None, True, 2, 0.125)
    _assert_close(out, ref, R.attention_tolerance(dtype, ref, mag, big, 64, 100) + mag * 2.0 ** -20, "")
    assert int(c.status) == 64


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_attention_repeats_itself(dtype):
    n, lens = [1] * 12, [1700 + 13 * i for i in range(12)]
    c = PagedCase(dtype, 128, 2, 64, "nhd", n, lens, seed=5)
    for x in c.dev:
        x.normal_()
    q = _randn((12, 8, 128), dtype, 1).to(DEV)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    ws, outs = c.kv.attn_shared_workspace(8, 12, 1, 1, 1900, 1600), []
    for _ in range(4):
        ws.random_(0, 255)
        outs.append(torch.empty_like(q))
        c.kv.attn_shared(q, outs[-1], dev([0, 12]), dev([1600]), c.cu, max_chunk=1, max_len=1900, max_shared=1600, workspace=ws)
    assert all(torch.equal(o, outs[0]) for o in outs)
