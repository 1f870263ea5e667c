"""Head norms, 8-bit caches and slots in common as a program uses them: one behind the other, in graphs, on views, from threads and streams, with one
workspace for many calls, far apart in memory."""
import ctypes as C
import random
import threading

import pytest
import torch

import _paged_reference as R
import _q8_reference as Q
from _q8_reference import Cache8
from paper_2512_04857_b200 import lar
from test_norm_q8_ops import AXES, _close, _params, _pos, _randn
from test_paged_ops import PagedCase
from test_shared_prefix import _share

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------------------------------------- workspaces
@pytest.mark.parametrize("seed", range(3))
def test_what_a_workspace_is_asked_for_suffices(seed):
    """Calls of all sizes up to those a workspace was sized for, bounds that hold and that do not: none is refused for its workspace.  What is not refused
    would be launched, so this runs where there is no GPU (the launch is what fails then)."""
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    L, rng = lar.lib(), random.Random(seed)
    pick = lambda hi: max(1, min(hi, int(hi ** rng.random() + 0.5)))
    for _ in range(400):
        d, (group, hkv), dt = rng.choice([64, 128]), rng.choice([(1, 1), (2, 8), (4, 8), (8, 1), (3, 20), (16, 2), (1, 32)]), rng.choice([0, 1])
        hq, rows = group * hkv, lar.lar_rows_t(4096, group * hkv * d, d)

        def kv(code, seqs, cols):
            return lar.lar_paged_kv_t(C.sizeof(lar.lar_paged_kv_t), code, seqs, hkv, d, 64, 1 << 16, cols, hkv * 64 * d, hkv * d, d, 4096, 1 << 30, 256, cols, 0,
                                      512, 1, None)

        def q8(seqs, cols):
            return lar.lar_paged_q8_t(C.sizeof(lar.lar_paged_q8_t), 0, kv(lar.LAR_E4M3, seqs, cols), 4096, 1 << 20, hkv * 64, 64)
        seqs, cols, chunk, groups = pick(1024), pick(2000), pick(4000), pick(1024)
        tokens, length, shared, known = pick(seqs * chunk), pick(64 * cols), pick(64 * cols), rng.random() < 0.6
        hints = (chunk, length) if known else (0, 0)
        bytes8 = L.lar_paged_q8_attn_workspace_bytes(q8(seqs, cols), dt, hq, tokens, *hints)
        bytes_s = L.lar_paged_attn_shared_workspace_bytes(kv(dt, seqs, cols), hq, tokens, groups, *hints, shared if known else 0)
        longest = chunk if known else tokens
        for _ in range(6):
            s, c, t, g, m = pick(seqs), pick(cols), pick(tokens), pick(groups), rng.choice([0, pick(longest), longest])
            n, sh = pick(length if known else 64 * c), pick(shared if known else 64 * c)
            if m == 0 and t > longest:
                continue
            assert L.lar_paged_q8_attn(q8(s, c), dt, rows, rows, hq, t, 256, None, 1, 0.0, m, n, 4096, bytes8, None) != lar.LAR_ERR_NOMEM
            assert L.lar_paged_attn_shared(kv(dt, s, c), rows, rows, hq, t, 256, g, 256, 256, 1, 0.0, m, n, sh, 4096, bytes_s, None) != lar.LAR_ERR_NOMEM


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hkv,hq", [(128, 2, 8), (64, 3, 3)])
def test_one_workspace_for_calls_of_all_kinds(dtype, d, hkv, hq):
    """Sized once for the largest call of the 8-bit cache and of slots in common, used by both in turn (the fence behind it stays)."""
    lens = [2600, 700, 130, 2100]
    c8 = Cache8(d, hkv, 64, "nhd", [600, 3, 0, 40], lens, seed=d)
    c8.fill(3)
    c = PagedCase(dtype, d, hkv, 64, "nhd", [600, 3, 0, 40], lens, seed=d)
    for p, x in zip(c.pools, c.dev):
        x.normal_()
        p.copy_(x.cpu())
    _share(c, [(0, 4)], [120])
    n_bytes = max(lar.lib().lar_paged_q8_attn_workspace_bytes(c8.kv.desc, 0 if dtype == BF else 1, hq, 643, 600, 2600),
                  lar.lib().lar_paged_attn_shared_workspace_bytes(c.kv.desc, hq, 643, 2, 600, 2600, 120))
    buf = torch.full((n_bytes + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    ws = buf[:n_bytes]
    for seqs, n in ((4, [600, 3, 0, 40]), (4, [1, 1, 1, 1]), (2, [40, 2]), (1, [1]), (4, [2, 0, 1, 2]), (4, [30, 1, 9, 25])):
        cu, T = dev([0] + torch.tensor(n).cumsum(0).tolist()), sum(n)
        q = _randn((T, hq, d), dtype, T)
        out = torch.full((T, hq, d), 5.0, dtype=dtype, device=DEV)
        part8 = lar.PagedKV8(c8.pools[0], c8.pools[1], *c8.scales, c8.table_dev[:seqs], c8.lens_dev[:seqs], hkv, status=c8.status)
        part8.attn(q.to(DEV), out, cu, max_chunk=max(n), max_len=2600, workspace=ws)
        ref, mag, big = R.attention(q, c8.rows(0), c8.rows(1), n, lens[:seqs], None, True, hq // hkv, d ** -0.5)
        _close(out, ref, torch.maximum(R.attention_tolerance(dtype, ref, mag, big, d, 2600), Q.attention_tolerance(dtype, ref, mag, big, d, 2600, 6.0)), f"8 bit {n}")
        part = lar.PagedKV(c.dev[0], c.dev[1], c.kv._keep[2][:seqs], c.lens_dev[:seqs], hkv, status=c.status)
        said = min([120] + [b - a for a, b in zip(n, lens) if a])
        part.attn_shared(q.to(DEV), out, dev([0, seqs // 2, seqs]), dev([said, said]), cu, max_chunk=max(n), max_len=2600, max_shared=120, workspace=ws)
        ref, mag, big = R.attention(q, c.rows(0), c.rows(1), n, lens[:seqs], None, True, hq // hkv, d ** -0.5)
        _close(out, ref, R.attention_tolerance(dtype, ref, mag, big, d, 2600) + mag * 2.0 ** -20, f"shared {n}")
    assert (buf[n_bytes:] == 0xA5).all() and int(c.status) == 0 and int(c8.status) == 0


# -------------------------------------------------------------------------------------------------------- used together
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("layout,kind", [("nhd", "rms"), ("heads", "layer")])
def test_a_generation_over_an_8bit_cache(dtype, layout, kind):
    """Prompts of unlike lengths, then tokens one by one: norm, rotation and quantisation, attention over what is stored, everything as it was stored."""
    S, hq, hkv, d, page = 3, 4, 2, 128, 16
    n0, steps = [37, 5, 70], 4
    c = Cache8(d, hkv, page, layout, n0, [a + steps for a in n0], seed=1)
    rope = lar.make_rope(d, AXES[d])
    kw, kb, kn = _params(kind, hkv, d, True, dtype, 9, kind == "layer")
    qw, qb, qn = _params(kind, hq, d, False, dtype, 11, kind == "layer")
    ws = c.kv.attn_workspace(hq, sum(n0), max(n0), 96, dtype=dtype)
    lens = [0] * S
    for step in range(steps + 1):
        n = n0 if step == 0 else [1] * S
        lens = [a + b for a, b in zip(lens, n)]
        c.lens_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        cu, T = dev([0] + torch.tensor(n).cumsum(0).tolist()), sum(n)
        x, pos = _randn((T, hq + 2 * hkv, d), dtype, 20 + step), _pos(3, T, 30 + step)
        xd, qo = x.to(DEV), torch.empty(T, hq, d, dtype=dtype, device=DEV)
        c.kv.append_norm_rope(xd[:, hq:hq + hkv], xd[:, hq + hkv:], cu, rope, pos.to(DEV), xd[:, :hq], qo, q_norm=qn, k_norm=kn)
        out = torch.empty_like(qo)
        c.kv.attn(qo, out, cu, max_chunk=max(n), max_len=96, workspace=ws)
        ref, tol = Q.rotated(Q.norm(x[:, :hq], kind, qw, qb, 1e-5), Q.norm_tolerance(x[:, :hq], kind, qw, qb, 1e-5), pos, AXES[d], 10000.0, False, False)
        _close(qo, ref, Q.rounded(ref, tol, dtype), f"q {step}")
        stored = [[Q.values(*c.get(s, i, 0, lens[s])) for s in range(S)] for i in range(2)]
        get = lambda i: (lambda s, h, a, b: stored[i][s][h, a:b])
        ref, mag, big = R.attention(qo.cpu(), get(0), get(1), n, lens, None, True, hq // hkv, d ** -0.5)
        tol = torch.maximum(R.attention_tolerance(dtype, ref, mag, big, d, 96), Q.attention_tolerance(dtype, ref, mag, big, d, 96, 6.0))
        _close(out, ref, tol, f"attention {step}")
        # read back whole: into a cache in bf16 / fp32, over which the attention is the same up to its rounding
        total = sum(lens)
        rows = torch.empty(2, total, hkv, d, dtype=dtype, device=DEV)
        c.kv.read(rows[0], rows[1], dev([0] + torch.tensor(lens).cumsum(0).tolist()))
        for i in range(2):
            assert torch.equal(rows[i].double().cpu(), torch.cat([stored[i][s].transpose(0, 1) for s in range(S)]))
    assert c.kv.poll_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prefill_of_the_librarys_cache_with_norms(dtype):
    """The prefix through norms and rotation, its attention, and a decode step behind it."""
    S, Hq, Hkv, d, Cn, td = 3, 4, 2, 64, 21, BF if dtype == "bf16" else F32
    for kind in ("rms", "layer"):
        cache = lar.Cache(lar.make_config(n_layers=2, batch=S, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, dtype=dtype, cond_len=Cn, line_width=8, n_lines=4,
                                          anchor_len=8, recent_lines=1, budget_lines=4, flags=lar.LAR_FLAG_SHUFFLE_PAGES, page_seed=3))
        rope = lar.make_rope(d, AXES[d])
        kw, kb, kn = _params(kind, Hkv, d, True, BF, 9, True)
        qw, qb, qn = _params(kind, Hq, d, True, F32, 11, False)
        for layer in range(2):
            x, pos = _randn((S * Cn, Hq + 2 * Hkv, d), td, layer), _pos(3, S * Cn, layer)
            xd, qo = x.to(DEV), torch.empty(S * Cn, Hq, d, dtype=td, device=DEV)
            args = (layer, xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:], Cn, rope, pos.to(DEV), xd[:, :Hq], qo)
            cache.append_kv_rope(*args, q_norm=qn, k_norm=kn)
            with pytest.raises(lar.LarError) as e:
                cache.append_kv_rope(*args, q_norm=qn, k_norm=kn)
            assert e.value.status == lar.LAR_ERR_BAD_STATE
            lens, imap = cache.get_state(layer)
            assert (lens == Cn).all() and (torch.from_numpy(imap[:, :Cn]) == torch.arange(Cn)).all()
            turned = {}
            for name, rows, w, b in (("q", x[:, :Hq], qw, qb), ("k", x[:, Hq:Hq + Hkv], kw, kb)):
                turned[name] = Q.rotated(Q.norm(rows, kind, w, b, 1e-5), Q.norm_tolerance(rows, kind, w, b, 1e-5), pos, AXES[d], 10000.0, False, False)
            _close(qo, turned["q"][0], Q.rounded(*turned["q"], td), "q")
            view, out = cache.paged_view(layer), torch.empty_like(qo)
            view.attn(qo, out, max_chunk=Cn, max_len=Cn)
            k, v = turned["k"][0].to(td).view(S, Cn, Hkv, d), x[:, Hq + Hkv:].view(S, Cn, Hkv, d)
            q1, k1, v1 = (_randn((S, h, d), td, 50 + layer + i) for i, h in enumerate((Hq, Hkv, Hkv)))
            o1 = torch.empty(S, Hq, d, dtype=td, device=DEV)
            cache.decode_step(layer, q1.to(DEV), k1.to(DEV), v1.to(DEV), o1)
            ka, va = torch.cat([k, k1[:, None]], 1), torch.cat([v, v1[:, None]], 1)
            for got, q, n, L in ((out, qo.cpu(), [Cn] * S, Cn), (o1, q1, [1] * S, Cn + 1)):
                ref, mag, big = R.attention(q, lambda s, h, a, b: ka[s, a:b, h], lambda s, h, a, b: va[s, a:b, h], n, [L] * S, None, True, Hq // Hkv, d ** -0.5)
                # the reference's keys may round to the other neighbour: one step of bf16 (2^-7); in fp32 a key is off by what the norm and the rotation are
                # (64 elements: 64 + 40 roundings of 2^-24 in all, twice for the exponent's two keys)
                step = (2.0 ** -7 if td == BF else 208 * 2.0 ** -24) * 2 * big[..., None] * mag
                _close(got, ref, R.attention_tolerance(td, ref, mag, big, d, L) + step, f"{kind} {layer}")
        assert cache.poll_device_status() == 0
        cache.close()


# --------------------------------------------------------------------------------------------------------------- graphs
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 1, 1], [4, 2, 3], [40, 9, 20]])
def test_a_layer_step_over_an_8bit_cache_in_a_graph(dtype, n):
    """Append and attention captured once, replayed with other tokens, lengths and positions, with a second graph of the same workspace in between."""
    hq, hkv, d, page = 4, 2, 64, 16
    longest = [210, 230, 190]
    c = Cache8(d, hkv, page, "hnd", n, longest, seed=2)
    c.fill(3)
    T = sum(n)
    x, pos = torch.empty(T, hq + 2 * hkv, d, dtype=dtype, device=DEV), torch.empty(3, T, dtype=torch.int32, device=DEV)
    qo, out = torch.empty(T, hq, d, dtype=dtype, device=DEV), torch.empty(T, hq, d, dtype=dtype, device=DEV)
    rope, norm = lar.make_rope(d, AXES[d]), lar.HeadNorm("rms")
    ws = c.kv.attn_workspace(hq, T, max(n), 240, dtype=dtype)

    def step():
        c.kv.append_norm_rope(x[:, hq:hq + hkv], x[:, hq + hkv:], c.cu, rope, pos, x[:, :hq], qo, q_norm=norm, k_norm=norm)
        c.kv.attn(qo, out, c.cu, max_chunk=max(n), max_len=240, workspace=ws)
    x.normal_(), pos.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            step()
    for rep, lens in enumerate((longest, [60, 41, 95], [190, 230, 20], [longest[0], 100, 64])):
        xs, ps = _randn((T, hq + 2 * hkv, d), dtype, 40 + rep), _pos(3, T, 50 + rep)
        x.copy_(xs.to(DEV)), pos.copy_(ps.to(DEV)), c.lens_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(9.0)
        graphs[rep % 2].replay()
        stored = [[Q.values(*c.get(k, i, 0, lens[k])) for k in range(3)] for i in range(2)]
        get = lambda i: (lambda k, h, a, b: stored[i][k][h, a:b])
        ref, mag, big = R.attention(qo.cpu(), get(0), get(1), n, lens, None, True, hq // hkv, d ** -0.5)
        _close(out, ref, torch.maximum(R.attention_tolerance(dtype, ref, mag, big, d, 240), Q.attention_tolerance(dtype, ref, mag, big, d, 240, 8.0)), f"replay {rep}")
    assert int(c.status) == 0


# ------------------------------------------------------------------------------------------------------- memory layouts
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [[1, 3], [40, 9]])
@pytest.mark.parametrize("swap", [False, True])
def test_8bit_cache_of_views(dtype, n, swap):
    """K and V in one tensor, either first, rows with gaps, scales in one tensor; q and out with heads outermost."""
    hq, hkv, d, page, pages = 4, 2, 64, 32, 9
    lens = [130, 90]
    both = torch.full((pages, page, hkv, 2, 2 * d), 0x7f, dtype=torch.uint8, device=DEV)
    scales = torch.full((2, pages, 2 * hkv, page), 255, dtype=torch.uint8, device=DEV)
    pools = [both[..., 0, :d], both[..., 1, :d]]
    bytes_ = [scales[0][:, :hkv], scales[1][:, :hkv]]
    if swap:
        pools, bytes_ = pools[::-1], bytes_[::-1]
    table = torch.tensor([[3, 1, 4, 0, 8], [5, 2, 6, 7, 7]], dtype=torch.int32)
    kv = lar.PagedKV8(*pools, *bytes_, table.to(DEV), dev(lens), hkv)
    T, cu = sum(n), dev([0, n[0], sum(n)])
    all_n, all_cu = lens, dev([0, lens[0], sum(lens)])
    x = _randn((2, sum(lens), hkv, d), dtype, 3)
    gap = torch.empty(2, hkv, sum(lens) + 3, d, dtype=dtype, device=DEV)[:, :, :-3].transpose(1, 2)
    gap.copy_(x.to(DEV))
    kv.append_rope(gap[0], gap[1], all_cu)
    vals = [Q.values(*Q.quantise(x[i])) for i in range(2)]
    get = lambda i: (lambda s, h, a, b: vals[i][sum(lens[:s]):sum(lens[:s + 1])][a:b, h])
    q = _randn((T, hq, d), dtype, 4)
    qd = torch.empty(hq, T, d, dtype=dtype, device=DEV).transpose(0, 1)
    qd.copy_(q.to(DEV))
    out = torch.full((hq, T + 2, d), 5.0, dtype=dtype, device=DEV)
    kv.attn(qd, out[:, :T].transpose(0, 1), cu, max_chunk=max(n), max_len=130, workspace=kv.attn_workspace(hq, T, max(n), 130, dtype=dtype))
    ref, mag, big = R.attention(q, get(0), get(1), n, lens, None, True, hq // hkv, d ** -0.5)
    _close(out[:, :T].transpose(0, 1), ref, torch.maximum(R.attention_tolerance(dtype, ref, mag, big, d, 130), Q.attention_tolerance(dtype, ref, mag, big, d, 130, 6.0)))
    assert (out[:, T:] == 5.0).all() and (both[..., d:] == 0x7f).all() and (scales[:, :, hkv:] == 255).all()
    back = torch.empty(2, hkv, sum(lens) + 1, d, dtype=dtype, device=DEV)[:, :, 1:].transpose(1, 2)
    kv.read(back[0], back[1], all_cu)
    for i in range(2):
        assert torch.equal(back[i].double().cpu(), vals[i])
    assert kv.poll_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [[1, 1], [40, 5]])
def test_8bit_offsets_beyond_32_bits(n):
    """Pages and tokens 2^31 bytes and more apart: appended to, attended over, read back."""
    if torch.cuda.get_device_properties(0).total_memory < 60 << 30:
        pytest.skip("needs 20 GB")
    d, hkv, hq, page, far, T, lens = 64, 2, 4, 64, 1 << 31, sum(n), [300, 192]
    buf = torch.zeros(4 * far + (1 << 24), dtype=torch.uint8, device=DEV)
    pool = lambda at: buf.as_strided((5, page, hkv, d), (far, hkv * d, d, 1), at)
    scale = lambda at: buf.as_strided((5, hkv, page), (far, page, 1), at)
    rows = torch.empty(4 * (1 << 29) + (1 << 22), dtype=BF, device=DEV)
    view = lambda heads, at: rows.as_strided((T, heads, d), (d, 1 << 29, 1), at)        # heads 2^30 bytes apart
    table = torch.tensor([[4, 1, 3, 0, 2], [2, 4, 3, -1, -1]], dtype=torch.int32)
    kv = lar.PagedKV8(pool(0), pool(1 << 20), scale(2 << 20), scale(3 << 20), table.to(DEV), dev(lens), hkv)
    vals = []
    for i in range(2):
        codes, byte = Q.quantise(torch.randn(5, page, hkv, d, generator=torch.Generator().manual_seed(i)))
        pool(i << 20).copy_(codes.view(torch.uint8).to(DEV))
        scale((2 + i) << 20).copy_(byte.transpose(1, 2).to(DEV))
        vals.append(Q.values(codes, byte))
    q, qo, out, k, v = view(hq, 0), view(hq, 1 << 18), view(hq, 2 << 18), view(hkv, 3 << 18), view(hkv, 4 << 18)
    host = {}
    for name, x in (("q", q), ("k", k), ("v", v)):
        host[name] = _randn(tuple(x.shape), BF, len(host))
        x.copy_(host[name].to(DEV))
    cu = dev([0, n[0], T])
    start = [0, 128]                                       # (what the second sequence sees lies in its own rows)
    kv.append_norm_rope(k, v, cu, None, None, q, qo, q_norm=lar.HeadNorm("rms"))
    ref, tol = Q.norm(host["q"], "rms", None, None, 1e-6), Q.norm_tolerance(host["q"], "rms", None, None, 1e-6)
    _close(qo, ref, Q.rounded(ref, tol, BF), "q")
    t = 0
    for s, a in enumerate(n):
        for i in range(a):
            j = lens[s] - a + i
            for w, x in enumerate(("k", "v")):
                vals[w][int(table[s, j // page]), j % page] = Q.values(*Q.quantise(host[x][t]))
            t += 1
    get = lambda w: (lambda s, h, a, b: torch.stack([vals[w][int(table[s, j // page]), j % page, h] for j in range(a, b)]))
    back = torch.empty(2, T, hkv, d, device=DEV)
    kv.read(back[0], back[1], cu)
    for w in range(2):
        want = torch.cat([torch.stack([get(w)(s, h, lens[s] - a, lens[s]) for h in range(hkv)], 1) for s, a in enumerate(n)])
        assert torch.equal(back[w].double().cpu(), want)
    kv.attn(qo, out, cu, kv_start=dev(start), max_chunk=max(n), max_len=300, workspace=kv.attn_workspace(hq, T, max(n), 300))
    ref, mag, big = R.attention(qo.cpu(), get(0), get(1), n, lens, start, True, 2, d ** -0.5)
    _close(out, ref, torch.maximum(R.attention_tolerance(BF, ref, mag, big, d, 300), Q.attention_tolerance(BF, ref, mag, big, d, 300, 6.0)))
    assert kv.poll_device_status() == 0


@pytest.mark.gpu
def test_as_many_sequences_as_there_may_be():
    S, d = 1024, 64
    n, lens = [(s % 3) for s in range(S)], [2 + s % 40 for s in range(S)]
    c8 = Cache8(d, 1, 16, "nhd", n, lens, seed=1)
    c8.fill(1)
    q = _randn((sum(n), 2, d), BF, 1)
    out = torch.empty(sum(n), 2, d, dtype=BF, device=DEV)
    c8.kv.attn(q.to(DEV), out, c8.cu, max_chunk=2, max_len=41, workspace=c8.kv.attn_workspace(2, sum(n), 2, 41))
    ref, mag, big = R.attention(q, c8.rows(0), c8.rows(1), n, lens, None, True, 2, d ** -0.5)
    _close(out, ref, Q.attention_tolerance(BF, ref, mag, big, d, 41, 6.0))
    # every sequence a group of its own, and all of them one group that has nothing in common
    kv = lar.PagedKV(*(torch.randn(c8.pools[0].shape, device=DEV).to(BF) for _ in range(2)), c8.table_dev, c8.lens_dev, 1)
    a, b = torch.empty_like(out), torch.empty_like(out)
    kv.attn(q.to(DEV), a, c8.cu, max_chunk=2, max_len=41)
    ws = kv.attn_shared_workspace(2, sum(n), S, 2, 41, 30)
    for groups, slots in ((list(range(S + 1)), 30), ([0, S], 0)):
        kv.attn_shared(q.to(DEV), b, dev(groups), dev([slots] * (len(groups) - 1)), c8.cu, max_chunk=2, max_len=41, max_shared=30, workspace=ws)
        assert ((a.float() - b.float()).abs() <= 2 * 2.0 ** -8 * a.float().abs() + 2.0 ** -7).all()      # each off by its weights' and its own rounding
    assert c8.kv.poll_device_status() == 0 and kv.poll_device_status() == 0


# ---------------------------------------------------------------------------------------------------- threads and streams
def _calls(dtype, n, hq=4, hkv=2, d=64):
    """An 8-bit cache and one with slots in common, and what the calls over them give."""
    lens = [300 + 7 * i for i in range(4)]
    c8 = Cache8(d, hkv, 16, "nhd", [n] * 4, lens, seed=n)
    c8.fill(n)
    c = PagedCase(dtype, d, hkv, 16, "nhd", [n] * 4, lens, seed=n)
    for x in c.dev:
        x.normal_()
    q = _randn((4 * n, hq, d), dtype, n).to(DEV)
    w8, ws = c8.kv.attn_workspace(hq, 4 * n, n, 330, dtype=dtype), c.kv.attn_shared_workspace(hq, 4 * n, 1, n, 330, 200)
    groups, shared, norm, rows = dev([0, 4]), dev([200]), lar.HeadNorm("layer"), torch.empty(4 * n, hkv, d, dtype=dtype, device=DEV)

    def run(outs):
        lar.norm_rope_rotate(None, None, q, outs[0], q_norm=norm)
        c8.kv.attn(q, outs[1], c8.cu, max_chunk=n, max_len=330, workspace=w8)
        c.kv.attn_shared(q, outs[2], groups, shared, c.cu, max_chunk=n, max_len=330, max_shared=200, workspace=ws)
        c8.kv.read(rows, rows.clone(), c8.cu)
    return run, lambda: [torch.empty_like(q) for _ in range(3)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [(BF, 1), (BF, 40), (F32, 3)])
def test_calls_from_two_threads_and_streams(dtype, n):
    """Each thread with caches, workspaces and a stream of its own (its first CUDA calls): what one thread alone gives."""
    work = []
    for k in range(2):
        run, outs = _calls(dtype, n + 2 * k)
        want = outs()
        run(want)
        work.append((run, want, [outs() for _ in range(20)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    errors = []

    def loop(run, want, many, stream):
        try:
            with torch.cuda.stream(stream):
                for outs in many:
                    run(outs)
        except Exception as e:                                        # noqa: BLE001 -- shown by the test
            errors.append(e)
    threads = [threading.Thread(target=loop, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for _, want, many, _ in work:
        assert all(torch.equal(a, b) for outs in many for a, b in zip(want, outs))
