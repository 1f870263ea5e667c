"""Head norms, 8-bit caches and slots in common where numbers, lengths and addresses come to their ends, against plain 64-bit forms."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

import _paged_reference as R
import _q8_reference as Q
import test_shared_prefix
from _q8_reference import Cache8
from paper_2512_04857_b200 import lar
from test_norm_q8_ops import _check_attention, _close, _q8, _r, _randn

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INVALID = lar.LAR_ERR_INVALID_ARG
dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)


def _store(c, which, s, rows):
    """rows [hkv, n, d] into the slots of sequence s from 0 on, as the cache holds them."""
    codes, byte = Q.quantise(rows)
    c.put(s, which, 0, codes, byte)
    c.vals[which][s] = Q.values(codes, byte)


# ------------------------------------------------------------------------------------------------- logits of all sizes
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("a,b", [(0, 0), (0, 114), (0, 118), (8, 110), (-60, 118), (-100, 112), (-118, 117), (-124, 118), (60, -60), (100, -110), (119, -117), (115, -20)])
def test_8bit_attention_of_queries_and_keys_of_any_size(dtype, d, n, a, b):
    """q of 2^a and keys of up to 2^(b + 8), whose logits 2^(a + b) (257 + i) are exact in fp32: the softmax is that of i, whatever a and b are.  Some slots'
    keys are as large as keys can be where q is zero: their logits are 0, as those of a row of zeros are."""
    L = 300
    c = Cache8(d, 1, 32, "nhd", [n], [L])
    c.fill(1)
    i = torch.arange(L) % 13
    keys = torch.zeros(1, L, d, dtype=torch.float64)
    keys[0, :, 0], keys[0, :, 1] = 2.0 ** (b + 8), (i + 1) * 2.0 ** b
    keys[0, ::50] = 0
    keys[0, 7::50] = 0
    keys[0, 7::50, 5] = 2.0 ** 127
    _store(c, 0, 0, keys.float())
    assert torch.equal(c.vals[0][0], keys)
    q = torch.zeros(n, 2, d, dtype=torch.float64)
    q[:, :, :2] = 2.0 ** a
    q = q.to(dtype)
    out = torch.empty(n, 2, d, dtype=dtype, device=DEV)
    c.kv.attn(q.to(DEV), out, softmax_scale=2.0 ** -(a + b), max_chunk=n, max_len=L, workspace=c.kv.attn_workspace(2, n, n, L, dtype=dtype))
    x = keys[0, :, :2].sum(-1) * 2.0 ** -b
    for t in range(n):
        p = torch.softmax(x[:L - n + t + 1], 0)
        V = c.vals[1][0][0, :L - n + t + 1]
        ref, mag = p @ V, p @ V.abs()
        # A logit times the scale: 12 below the largest at most where the weight counts, off by three roundings (2^-22 of 18, in powers of two); exponential
        # 2^-21, sums of 300 terms: below 2^-15 of mag, in numerator and denominator.  Weights of bf16 rows: rounded to fp16 or bf16 (2^-8).
        tol = mag * 2.0 ** -14
        if dtype == BF:
            tol = tol + mag * (2.0 ** -8 if 2 * n > 64 else 2.0 ** -11)
            tol = tol + (ref.abs() + tol) * 2.0 ** -8
        else:
            tol = tol + ref.abs() * 2.0 ** -24
        _close(out[t], ref.expand(2, d), tol.expand(2, d), f"token {t}")


# ---------------------------------------------------------------------------------------------------- constant rows
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_layer_norm_of_large_rows_of_one_value(dtype, d):
    """A row of equal elements has nothing left after its mean: what comes out is the bias, also where the row's sum lies beyond fp32.  Rows of +x and -x in
    turn come out as +-1 times the weight and the bias."""
    sizes = [0.0, 1.0, 3333.333, -0.7e-3, -2.0 ** 40, 2.0 ** 100, 2.0 ** 119, 2.0 ** 121, -2.0 ** 122, 1.9e36, 2.0 ** 126, 2.0 ** 127, -2.0 ** 127, 3.3e38]
    x = torch.tensor(sizes)[None, :, None].expand(2, -1, d).clone()
    x[1, :, ::2] *= -1
    x = x.to(dtype)
    w, b = _randn((d,), F32, 1, 0.3) + 1, _randn((d,), F32, 2)
    out = torch.empty(2, len(sizes), d, dtype=dtype, device=DEV)
    norm = lar.HeadNorm("layer", w.to(DEV), b.to(DEV))
    lar.norm_rope_rotate(None, None, x.to(DEV), out, q_norm=norm)
    assert torch.equal(out[0].cpu(), b.to(dtype).expand(len(sizes), d))
    _close(out[1], Q.norm(x[1:], "layer", w, b, 1e-6)[0], Q.rounded(Q.norm(x[1:], "layer", w, b, 1e-6), Q.norm_tolerance(x[1:], "layer", w, b, 1e-6), dtype)[0])
    # the same rows as keys on the way into an 8-bit cache
    S = len(sizes)
    c = Cache8(d, S, 16, "nhd", [2], [2])
    c.kv.append_norm_rope(x.to(DEV), x.to(DEV), k_norm=norm)
    codes, byte = c.get(0, 0, 0, 1)
    want = Q.quantise(b.expand(S, 1, d))
    assert torch.equal(codes.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(byte, want[1])


# ------------------------------------------------------------------------------------------------- values of all sizes
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hkv,hq", [(64, 2, 4), (128, 1, 8)])
@pytest.mark.parametrize("n,lens", [([1], [300]), ([3, 1], [700, 90]), ([40, 9], [400, 1200])])
@pytest.mark.parametrize("power", [-10, -30, -45, -70])
def test_8bit_attention_of_small_values_beside_rows_of_zeros(dtype, d, hkv, hq, n, lens, power):
    """A row of zeros adds nothing, whatever its byte (127) says: small values beside it keep all their bits."""
    c = Cache8(d, hkv, 32, "nhd", n, lens, seed=1)
    c.fill(2)
    g = torch.Generator().manual_seed(3)
    for s, L in enumerate(lens):
        v = torch.randn(hkv, L, d, generator=g) * 2.0 ** power
        v[:, ::5] = 0
        v[:, 3:90] = 0                                           # whole tiles of them
        _store(c, 1, s, v)
    for causal in (True, False):
        _check_attention(c, hq, dtype, causal, None, True, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 50])
def test_8bit_attention_of_the_smallest_values(dtype, d, n):
    """Values of 2^-98 to 2^-114: the result is as small, but far from what fp32 cannot hold."""
    L = 200
    for power in (-98, -104, -108, -114):
        c = Cache8(d, 1, 16, "nhd", [n], [L])
        c.fill(1)
        g = torch.Generator().manual_seed(3)
        _store(c, 1, 0, torch.randn(1, L, d, generator=g).clamp(-4, 4) * 2.0 ** power)
        q = _randn((n, 2, d), dtype, 5)
        out = torch.empty(n, 2, d, dtype=dtype, device=DEV)
        c.kv.attn(q.to(DEV), out, max_chunk=n, max_len=L, workspace=c.kv.attn_workspace(2, n, n, L, dtype=dtype))
        up = 2.0 ** -power
        big_v = c.vals[1][0] * up
        ref, mag, big = R.attention(q, c.rows(0), lambda s, h, j0, j1: big_v[h, j0:j1], [n], [L], None, True, 2, d ** -0.5)
        tol = torch.maximum(Q.attention_tolerance(dtype, ref, mag, big, d, L, 4.0), R.attention_tolerance(dtype, ref, mag, big, d, L) if 2 * n > 64 else torch.zeros(()))
        _close(out.double() * up, ref, tol + 2.0 ** -149 * up * 2 * L, f"2^{power}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_8bit_rows_are_as_near_as_the_format_says(dtype):
    """Rows whose largest element is anything from just above 224 to 448 times the power, the others down to 2^-12 of the power: off by half a step, 2^-4 of an element or 2^-10 of the
    power (for the first of these rows 2^-17.8 of the largest element)."""
    g = torch.Generator().manual_seed(1)
    tops = [225.0, 226.0, 256.0, 300.0, 446.0, 448.0]
    rows = torch.exp2(torch.rand(len(tops) * 40, 64, generator=g) * 14 - 12) * torch.where(torch.rand(len(tops) * 40, 64, generator=g) < 0.5, -1.0, 1.0)
    rows[:, 0] = torch.tensor(tops).repeat(40)
    rows[:, 1] = 2.0 ** -9 * 1.5 - 2.0 ** -16                      # just below the middle of two steps
    x = (rows * torch.exp2(torch.arange(len(rows)) % 50 - 25.0)[:, None]).to(dtype)[:, None]
    n = len(x)
    c = Cache8(64, 1, 16, "nhd", [n], [n])
    c.kv.append_rope(x.to(DEV), x.to(DEV))
    ko, vo = torch.empty_like(x, device=DEV), torch.empty_like(x, device=DEV)
    c.kv.read(ko, vo)
    assert torch.equal(ko, vo)
    power = torch.exp2(c.get(0, 0, 0, n)[1][0].double() - 127)[:, None]
    x, diff = x[:, 0].double(), (ko[:, 0].cpu().double() - x[:, 0].double()).abs()
    largest = x.abs().amax(1, keepdim=True)
    assert (largest > 224 * power).all() and (largest <= 448 * power).all()
    assert (diff <= torch.maximum(x.abs() * 2.0 ** -4, power * 2.0 ** -10)).all()
    assert (diff <= torch.maximum(x.abs() * 2.0 ** -4, largest * 2.0 ** -17.8)).all() and (diff > torch.maximum(x.abs() * 2.0 ** -4, largest * 2.0 ** -18)).any()


# ---------------------------------------------------------------------------------------- slots in common, row tiles
@pytest.mark.gpu
@pytest.mark.parametrize("d,hkv,hq", [(128, 2, 8), (64, 1, 8)])
@pytest.mark.parametrize("seqs,tokens,common,own", [(90, 1, 700, 20), (100, 1, 1100, 64), (60, 3, 1536, 200), (400, 1, 1990, 30)])
def test_shared_attention_of_row_tiles_that_leave_sms_idle(d, hkv, hq, seqs, tokens, common, own):
    """More than 128 rows per KV head and group over fewer than 2048 slots in common: few units, which are cut as a join follows anyway."""
    test_shared_prefix.test_shared_attention_of_many_sequences(BF, d, hkv, hq, seqs, tokens, common, own)


# ------------------------------------------------------------------------------------- what a pass that gave up leaves
def test_parts_of_a_row_lie_inside_the_workspace(tmp_path):
    """The join of slots in common reads a row's parts where the row's pass says; a pass whose wait ran out leaves whatever the workspace held.  For any words there the ranges
    and the row stay inside what the pass has, and what a pass does write is taken as it is."""
    src = tmp_path / "t.cpp"
    src.write_text('''#include "part_range.h"
        extern "C" void f(int x, int y, int ranges, int rows, int* out) {
            lar::PartRange p = lar::part_range(x, y, ranges, rows);
            out[0] = p.first; out[1] = p.last; out[2] = p.row;
        }''')
    so = tmp_path / "t.so"
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I", os.path.join(os.path.dirname(lar.LIB_PATH), "csrc"), "-o", str(so), str(src)], check=True)
    f, out, rng = C.CDLL(str(so)).f, (C.c_int * 3)(), random.Random(1)
    word = lambda: rng.choice([0, -1, 255, 2 ** 31 - 1, -2 ** 31, rng.getrandbits(32) - 2 ** 31, rng.getrandbits(24), rng.getrandbits(9)])
    for _ in range(20000):
        ranges, rows = rng.choice([1, 8, 148, 296, 444]), rng.choice([1, 8, 64, 256])
        x, y = word(), word()
        f(x, y, ranges, rows, out)
        if x < 0:
            assert out[0] == -1
            continue
        assert 0 <= out[0] < ranges and out[1] < ranges and 0 <= out[2] < rows
        a, b, r = rng.randrange(ranges), rng.randrange(ranges), rng.randrange(rows)
        f(a + 65536 * b, r, ranges, rows, out)
        assert list(out) == [a, b, r]


# ------------------------------------------------------------------------------------------------- idle sequences
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,lens", [([0, 1, 0, 1], [90, 70, 0, 300]), ([0, 6, 1, 0], [700, 70, 130, 40]), ([0, 150, 0, 1, 0], [500, 300, 0, 200, 260]),
                                    ([70, 0, 33], [2500, 90, 2100])])
def test_8bit_attention_beside_sequences_without_tokens(dtype, n, lens):
    """Sequences without tokens may have given up their pages, whatever their lengths still say: nothing of them is looked at and nothing recorded."""
    for layout, d, hkv, hq in (("nhd", 128, 2, 4), ("heads", 64, 2, 2)):
        c = Cache8(d, hkv, 32, layout, n, lens, seed=4)
        c.fill(5)
        for s, m in enumerate(n):
            if m == 0:
                c.table_dev[s] = -1
        for causal in (True, False):
            for hints in (True, False):
                _check_attention(c, hq, dtype, causal, None, True, 6, hints=hints)


# ------------------------------------------------------------------------------------------------ addresses, refusals
def test_pools_too_far_apart_are_refused_by_every_call():
    """K and V are one tensor to the copies, the distance of their pools one of its strides: below 2^40 bytes, and that of the scales too."""
    L, rows = lar.lib(), _r()
    for far, near in ((1 << 40, (1 << 40) - 16), ((1 << 46) + 4096, 1 << 20)):
        for where in ("pool", "scale"):
            for first, second in ((4096, 4096 + far), (4096 + far, 4096)):
                c = _q8(k_pool=first, v_pool=second) if where == "pool" else _q8(k_scale=first, v_scale=second)
                assert L.lar_paged_q8_append(c, 0, None, None, None, None, 0, rows, rows, None, None, 0, 6, None, None) == INVALID
                assert L.lar_paged_q8_append(c, 0, None, None, None, None, 0, rows, rows, None, None, 0, 0, None, None) == INVALID
                assert L.lar_paged_q8_read(c, 0, rows, rows, 0, None, None) == INVALID
                for n in (0, 6, 200):
                    assert L.lar_paged_q8_attn(c, 0, rows, rows, 2, n, None, None, 1, 0.0, 0, 0, None, 0, None) == INVALID
                assert L.lar_paged_q8_attn_workspace_bytes(c, 0, 2, 200, 100, 0) == 0
            ok = _q8(k_pool=4096, v_pool=4096 + near) if where == "pool" else _q8(k_scale=4096 + near, v_scale=4096)
            assert L.lar_paged_q8_read(ok, 0, rows, rows, 0, None, None) == lar.LAR_OK
            assert L.lar_paged_q8_attn(ok, 0, rows, rows, 2, 0, None, None, 1, 0.0, 0, 0, None, 0, None) == lar.LAR_OK
            assert L.lar_paged_q8_attn_workspace_bytes(ok, 0, 2, 200, 100, 0) > 0


def test_a_long_8bit_call_is_refused_before_anything_is_launched():
    """A workspace that holds the unpacked rows but not what the attention over them wants, and caches whose tiles that attention cannot count: refused by the checks, not behind the
    first kernels (without a GPU a launch would fail in another way)."""
    L = lar.lib()
    c, n = _q8(n_seqs=2, n_pages=4096, table_cols=200, table_seq_stride=200), 400     # 2 x 6400 slots, 2 heads of 64
    need = L.lar_paged_q8_attn_workspace_bytes(c, 0, 2, n, 200, 0)
    slots = 200 * 32
    unpacked = 2 * 2 * slots * 2 * 64 * 2 + -(-2 * slots // 128 * 4 // 256) * 256       # K and V of both sequences as bf16 rows, their page table
    assert unpacked + 4096 < need
    call = lambda c, n, nb: L.lar_paged_q8_attn(c, 0, _r(), _r(1 << 20), 2, n, None, None, 1, 0.0, 200, 0, 4096, nb, None)
    assert call(c, n, unpacked - 1) == lar.LAR_ERR_NOMEM and call(c, n, unpacked) == lar.LAR_ERR_NOMEM
    huge = _q8(n_seqs=8, n_pages=1 << 24, table_cols=1 << 23, page_tokens=128, sp=256, sh=128, page_stride=2 * 128 * 64)
    assert call(huge, 8 * 20000, 1 << 62) == lar.LAR_ERR_CAPACITY
