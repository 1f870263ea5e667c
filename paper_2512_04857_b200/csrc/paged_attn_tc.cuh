// Chunk attention for bf16 storage on the 5th-generation tensor cores (tcgen05, accumulators in TMEM), one persistent kernel
// for everything but a few rows per KV head: candidate chunks over long caches (bound by the cache's bytes) and prompts (bound by the
// chain logits -> exponentials -> P -> product).
//
// A row tile is up to 128 (token, head of the group) rows of one KV head.  A CTA works on NT of them at a time:
//   NT = 2  chunks of more than 128 rows, of 128-element rows over long caches more than 32: up to 256 rows share every K/V tile of 128 slots; while the softmax of one row tile runs on its warps, the
//           tensor cores work for the other.  4096 tokens of 32 / 8 heads of 128 over 32768 slots: 1.69 ms, 1.2 PFLOP/s.
//   NT = 1  fewer rows: K/V tiles of 64 slots, two logit buffers (the logits of the next tile are formed while the softmax of this
//           one runs) and two CTAs per SM, since what counts is that the cache streams without a pause.
// Roles (coupled by mbarriers only, every wait bounded):
//   NT * 4 softmax warps  one thread per row: logits from TMEM, mask, running maximum and sum (fp32), P (bf16) into TMEM (NT = 1: over the
//                         logits it came from); output rows at the end.
//   NT MMA warps          one thread per row tile: S = Q K^T (both from shared memory), O += P V (P from TMEM, V from shared memory with the
//                         slots as its K dimension).
//   NT producer warps     rings of K and V tiles: one TMA box per page (or part of one) and 64 columns, the lanes issuing them side by
//                         side; the first also works out what comes next.
// The output accumulator is rescaled only where a row's maximum has grown by more than 2^8 since its last rescaling (P then
// reaches 2^8 at most, far inside the range of bf16 and fp32; the factor cancels in the final division), so the
// accumulator hardly ever leaves TMEM.
//
// P is rounded to bf16 for the product with V (both operands of a product have one type; the library's decode kernel does the same), the row sum is
// of the weights before that rounding, in fp32.  Relative error against 64 bits, all of a result: 1.9e-3 to 2.4e-3, where rounding the result
// alone gives 1.6e-3 to 1.7e-3 (paged_attn_few.cuh alike).  Logits, maximum, sum and accumulator are fp32.
//
// Slots outside [start, len) of a tile hold memory that may be anything: keys are masked by selection, and the value rows
// are cleared in shared memory before the product (0 * NaN would reach the output).
//
// Work.  A unit is one (sequence, KV head, NT row tiles), heads outermost (the CTAs of a moment share K/V in L2), the longest tiles of
// a sequence first.
//   Many units, or units of unlike length (prompts): whole units, each CTA takes the next one when it is free (a counter in the workspace).
//   Fewer, long units: NT = 2 whole units round-robin, as many full rounds as there are; what is left, and with NT = 1 all units,
//   is one list of slot tiles that is cut into equal ranges, one per CTA; a unit cut by a range boundary leaves (O, m, l) per
//   CTA in the workspace and join_ranges_kernel adds them up in the order of the CTAs.
//   Without a workspace: whole units round-robin.
#pragma once
#include <cuda.h>

#include "decode_stream.cuh"  // wait_or_abort, mbar_arrive, ex2_approx, proxy fences
#include "paged_attn.cuh"

namespace lar {

constexpr int kTcMaxSeqs = 1024;  // sequences of a call (their lengths are kept in shared memory)
constexpr int kTcMaxStages = 4;
constexpr int kCutTiles = 8, kCutTilesJoined = 4;  // slot tiles that idle CTAs have to gain for units to be cut: a join of its own, or one that follows anyway

template <int D, int NT>
struct TcShape {
    static constexpr int BN = NT == 2 ? 128 : 64;            // slots of a K/V tile
    static constexpr int HALVES = D / 64;                    // 128-byte column blocks
    static constexpr int TILE_BYTES = BN * D * 2;            // K or V tile
    static constexpr int STAGE_BYTES = 2 * TILE_BYTES;
    static constexpr int SM_WARPS = NT * 4;
    // NT = 2: three warpgroups, the third (two MMA warps, two producers) gives registers to the softmax warps: 2 * 216 + 72 =
    // 3 * 168, what the block was launched with
    static constexpr int THREADS = NT == 2 ? 384 : SM_WARPS * 32 + 64;
    static constexpr int SM_REGS = 216, OTHER_REGS = 504 - 2 * SM_REGS;
    static constexpr int P_PARTS = NT == 2 ? 2 : 1;          // P is handed over in parts of 64 slots: the product starts on the first
    // TMEM columns.  NT = 2: one logit buffer for both row tiles (a softmax warp takes its logits into registers at once, so the buffer is
    // free for the other row tile's), P of each row tile (64 columns), two accumulators.  (D = 64 has room for a buffer each: measured slower,
    // 416 instead of 381 us for 2048 tokens over 16384 slots; taking turns keeps the row tiles' exponentials apart.)  NT = 1: two logit buffers that P overlays,
    // one accumulator.
    static constexpr int P_COL = NT == 2 ? BN : 0, P_COLS = BN / (NT == 2 ? 2 : 1), O_COL = 2 * BN;
    static constexpr int TMEM_COLS = NT == 2 ? 512 : 256;
    static_assert(O_COL + NT * D <= TMEM_COLS, "TMEM");
    static __host__ __device__ constexpr int s_col(int buf) { return NT == 1 ? buf * BN : 0; }
    static __host__ __device__ constexpr int p_col(int buf) { return P_COL + buf * P_COLS; }
};

struct TcMaps {
    CUtensorMap q;     // {d, heads of a group, KV heads, tokens}, box 64 x group x 1 x tq
    CUtensorMap k, v;  // {d, rows of a page, heads, pages}, box 64 x min(page, BN) x 1 x 1
};

struct TcArgs {
    PagedAttnArgs a;
    int stages;
    int rows_cap;      // rows of a row tile in shared memory: tq * group rounded up to 8
    int box_rows;      // slots of one K/V box
    int split;         // ranges may cut units
    int min_items;     // slot tiles that a range has at least
    int* counter;      // whole units are handed out as CTAs ask for them (zero before the launch); null: round-robin
    int4* records;     // split: per CTA the unit that begins in its range and goes on in the next CTAs
};

// per sequence, in shared memory
struct SeqInfo {
    int t0, n, len, lo;
};

// ---------------------------------------------------------------------------------- tcgen05
__device__ __forceinline__ void tc_alloc(uint32_t smem_dst, int cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_dealloc(uint32_t tmem, int cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D += A B over 16 elements of the contracted dimension.  a_lo, b_lo: low words of the descriptors, to which the immediate offsets are
// added here, so that a loop keeps two registers and not one descriptor per step.
template <uint32_t HIGH, uint32_t A_OFF, uint32_t B_OFF>
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b32 x, y;\n .reg .b64 a, b;\n setp.ne.u32 p, %4, 0;\n add.u32 x, %1, %5;\n add.u32 y, %2, %6;\n"
        " mov.b64 a, {x, %7};\n mov.b64 b, {y, %7};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"((uint32_t)acc), "n"(A_OFF), "n"(B_OFF), "r"(HIGH)
        : "memory");
}
// the same with A in TMEM
template <uint32_t HIGH, uint32_t A_OFF, uint32_t B_OFF>
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b32 x, y;\n .reg .b64 b;\n setp.ne.u32 p, %4, 0;\n add.u32 x, %1, %5;\n add.u32 y, %2, %6;\n"
        " mov.b64 b, {y, %7};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, p;\n}\n" ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"((uint32_t)acc), "n"(A_OFF), "n"(B_OFF), "r"(HIGH)
        : "memory");
}
#define LAR_R4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define LAR_I4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
// 32 columns of the warp's 32 lanes, one lane per thread
__device__ __forceinline__ void tc_ld32(uint32_t tmem, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : LAR_R4(r, 0), LAR_R4(r, 4), LAR_R4(r, 8), LAR_R4(r, 12), LAR_R4(r, 16), LAR_R4(r, 20), LAR_R4(r, 24), LAR_R4(r, 28)
        : "r"(tmem));
}
__device__ __forceinline__ void tc_st32(uint32_t tmem, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(tmem), LAR_I4(r, 0), LAR_I4(r, 4),
        LAR_I4(r, 8), LAR_I4(r, 12), LAR_I4(r, 16), LAR_I4(r, 20), LAR_I4(r, 24), LAR_I4(r, 28)
        : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Position in the ring of stages: which stage, and the parity of this use of it.
struct RingPos {
    int st = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void next(int n) {
        if (++st == n) {
            st = 0;
            ph ^= 1;
        }
    }
    __device__ __forceinline__ void skip(int k, int n) {
        const int to = st + k, turns = to / n;
        st = to - turns * n;
        ph ^= turns & 1;
    }
};
// fp32 accumulator, bf16 operands, M = 128
__host__ __device__ constexpr uint32_t tc_idesc(int n, bool b_transposed) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_transposed ? 1u : 0u) << 16) | ((uint32_t)(n / 8) << 17) | ((128u / 16u) << 24);
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}

// ---------------------------------------------------------------------------------- work list
// One step of a CTA's work: some slot tiles of one unit.
struct alignas(16) TcSeg {
    int seq, head, tok0, n_tok;  // tokens of the unit
    int slot0;                   // slot of its first token
    int lo, len;                 // live slots of the sequence
    int jb;                      // first slot tile
    int nb;                      // slot tiles (-1: no more work)
    int whole;                   // nothing of the unit lies in other CTAs
    int b0;                      // tiles of the unit before this step's
    int unit_end;                // end of the unit in the list of slot tiles; in the ring, the CTA that holds its last one
};
constexpr int kTcSegs = 4;  // steps that are known ahead of the warps that work on them

// ---------------------------------------------------------------------------------- shared memory
template <int D, int NT>
struct TcSmem {
    using S = TcShape<D, NT>;
    static __host__ __device__ int q_bytes(int rows_cap) { return NT * S::HALVES * ((rows_cap * 128 + 1023) / 1024 * 1024); }
    // the MMA reads 128 rows whatever rows_cap is: behind the last Q tile there is always a K/V stage or more
    static __host__ __device__ int tail(int n_seqs) { return 44 * 8 + kTcSegs * (int)sizeof(TcSeg) + n_seqs * 16 + 2 * (n_seqs + 1) * 4 + 16 * 4; }
    static __host__ __device__ int bytes(int rows_cap, int stages, int n_seqs) {
        return 1024 + q_bytes(rows_cap) + stages * S::STAGE_BYTES + tail(n_seqs);
    }
};

// A CTA's work: first whole units, every step-th one, then an equal range of the slot tiles of the units that are left.
template <int NT, int BN, int D>
struct TcWork {
    static constexpr int kUnitCost = NT == 2 ? 2 : BN == 64 ? (D == 64 ? 3 : 2) : (D == 64 ? 8 : 4);
    const SeqInfo* info;
    const int* pre;    // units before each sequence
    const int* items;  // slot tiles before each sequence, of the units from first_cut on
    int n_seqs, tq, causal;
    int x, end, step;  // whole units
    int y, y_end;      // range of slot tiles
    int first_cut;     // the first unit that may be cut

    // Items of a unit in the list that is cut into ranges: its slot tiles, and kUnitCost more for taking up and finishing a
    // unit (queries, last product, output rows: measured 2.3 us against 0.75 us for a tile with D = 64).
    static __device__ __forceinline__ int tiles_of_unit(const SeqInfo& s) { return s.len > s.lo ? (s.len + BN - 1) / BN - s.lo / BN : 0; }
    static __device__ __forceinline__ int items_of_unit(const SeqInfo& s) { return tiles_of_unit(s) + kUnitCost; }

    __device__ __forceinline__ bool next(TcSeg& g) {
        for (;;) {
            const bool cut = x >= end;
            if (cut && y >= y_end) return false;
            const int at = cut ? y : x;
            const int* before = cut ? items : pre;
            int a = 0, b = n_seqs;  // before[a] <= at < before[b]
            while (b - a > 1) {
                const int m = (a + b) >> 1;
                if (before[m] <= at) a = m; else b = m;
            }
            const SeqInfo s = info[a];
            const int ut = NT * tq, tiles = (s.n + ut - 1) / ut;
            const int r = at - before[a];
            int unit = r, take = 1 << 30;
            g.b0 = 0;
            g.whole = 1;
            if (cut) {
                const int full = tiles_of_unit(s), w = full + kUnitCost;
                const int q = r / w;
                unit = NT == 2 ? q + max(first_cut - pre[a], 0) : q;
                g.b0 = r - q * w;
                g.unit_end = y - g.b0 + max(full, 1);  // (the items behind the slot tiles belong to the range with the last tile)
                take = min(w - g.b0, y_end - y);
                y += take;
                if (g.b0 > 0 && g.b0 >= full) continue;
                g.whole = g.b0 == 0 && take >= full;
            } else {
                x += step;
            }
            g.head = unit / tiles;
            const int tile = tiles - 1 - (unit - g.head * tiles);  // the tiles that see most first
            g.seq = a;
            g.tok0 = s.t0 + tile * ut;
            g.n_tok = min(ut, s.n - tile * ut);
            g.slot0 = s.len - s.n + tile * ut;
            g.lo = s.lo;
            g.len = s.len;
            g.jb = s.lo / BN + g.b0;
            // (NT = 2: both row tiles take the same steps, the first one's last may be masked whole)
            const int hi = causal ? min(s.len, g.slot0 + g.n_tok) : s.len;
            g.nb = hi > s.lo ? max(min((hi + BN - 1) / BN - g.jb, take), 0) : 0;
            return true;
        }
    }
};

// Transposes a 4 x 4 matrix of 16-byte pieces held a row per lane by four neighbouring lanes.
__device__ __forceinline__ void quad_transpose(uint4 (&c)[4], int lane) {
    auto swap = [&](uint4& a, uint4& b, int mask) {  // the lower lane gives b and keeps a, the upper one gives a and keeps b
        const bool upper = (lane & mask) != 0;
        uint4 s = upper ? a : b;
        s.x = __shfl_xor_sync(0xffffffffu, s.x, mask);
        s.y = __shfl_xor_sync(0xffffffffu, s.y, mask);
        s.z = __shfl_xor_sync(0xffffffffu, s.z, mask);
        s.w = __shfl_xor_sync(0xffffffffu, s.w, mask);
        if (upper) a = s; else b = s;
    };
    swap(c[0], c[1], 1);
    swap(c[2], c[3], 1);
    swap(c[0], c[2], 2);
    swap(c[1], c[3], 2);
}

// The whole warp waits, and gives up together (what follows are warp-wide instructions).
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, wait_or_abort(bar, parity, abort_flag));
}

// The reference of a row, scaled before it is subtracted, so that a weight is one multiply-add.  Its rounding is a factor common to all weights that were
// formed with it: it cancels in a row that keeps its reference; a change of reference takes the ratio of the scaled ones, and what leaves the CTA as a part
// is freed of it.  From 2^31 on the factor itself leaves fp32's range.  Logits that differ at all then differ by 2^7 scaled, so that only those equal to
// the reference count whatever the scale, and a power of two for it makes the scaled reference exact.  (12 prompts of 340 to 4160 tokens 466 us, 466 with
// the scaled reference alone, 471 with a branch that subtracts first where it matters.)
struct ScaledRef {
    float m, sc, scale, scaled;
    __device__ __forceinline__ ScaledRef(float largest, float sc_) : m(softmax_ref(largest)), sc(sc_) {
        scale = fabsf(m * sc) < 2147483648.f ? sc : __uint_as_float(__float_as_uint(sc) & 0x7f800000u);
        scaled = __fmul_rn(m, scale);
    }
    // what weights formed with this reference are to be multiplied by for a larger one
    __device__ __forceinline__ float ratio_to(float larger) const {
        const ScaledRef to(larger, sc);
        return ex2_approx(scale == sc && to.scale == sc ? scaled - to.scaled : (m - larger) * sc);
    }
    __device__ __forceinline__ float rounding() const { return ex2_approx(-fmaf(m, scale, -scaled)); }
};

// PART: the rows of all units, cut or not, are left as (O, m, l) for a kernel that joins them with those over other slots.
template <int D, int NT, bool PART = false>
__global__ void __launch_bounds__(TcShape<D, NT>::THREADS, NT == 2 ? 1 : 2) paged_attn_tc_kernel(const __grid_constant__ TcArgs ta, const __grid_constant__ TcMaps maps) {
    using S = TcShape<D, NT>;
    constexpr int BN = S::BN, HALVES = S::HALVES;
    using Work = TcWork<NT, BN, D>;
    const PagedAttnArgs& a = ta.a;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* gbase = smem_raw + (base - smem_u32(smem_raw));
    const int NS = ta.stages;
    const uint32_t q_half = (uint32_t)((ta.rows_cap * 128 + 1023) / 1024 * 1024);  // bytes of 64 columns of a Q tile
    const uint32_t q_tile = q_half * HALVES;
    const uint32_t ring = base + NT * q_tile;
    unsigned char* tail = gbase + NT * q_tile + NS * S::STAGE_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(tail);
    const uint32_t bar0 = smem_u32(bars);
    auto q_full = [&](int i) { return bar0 + 8u * i; };
    auto q_empty = [&](int i) { return bar0 + 8u * (2 + i); };
    auto s_full = [&](int i) { return bar0 + 8u * (4 + i); };
    auto p_full = [&](int i) { return bar0 + 8u * (6 + i); };
    auto pv_done = [&](int i) { return bar0 + 8u * (8 + i); };
    auto o_free = [&](int i) { return bar0 + 8u * (10 + i); };
    const uint32_t bar_drain = bar0 + 8u * 12;
    auto k_full = [&](int st) { return bar0 + 8u * (13 + st); };
    auto v_full = [&](int st) { return bar0 + 8u * (17 + st); };
    auto k_empty = [&](int st) { return bar0 + 8u * (21 + st); };
    auto v_empty = [&](int st) { return bar0 + 8u * (25 + st); };  // NT = 1: not used, k_empty is both
    auto p2_full = [&](int i) { return bar0 + 8u * (29 + i); };
    auto s_free = [&](int i) { return bar0 + 8u * (31 + i); };
    auto seg_full = [&](int i) { return bar0 + 8u * (34 + i); };
    auto seg_empty = [&](int i) { return bar0 + 8u * (38 + i); };
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + 42);
    uint32_t* tmem_ptr = reinterpret_cast<uint32_t*>(bars + 42) + 1;
    TcSeg* seg_ring = reinterpret_cast<TcSeg*>(bars + 44);
    SeqInfo* info = reinterpret_cast<SeqInfo*>(seg_ring + kTcSegs);
    int* pre = reinterpret_cast<int*>(info + a.kv.n_seqs);
    int* items = pre + a.kv.n_seqs + 1;
    int* wsum = items + a.kv.n_seqs + 1;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (warp == S::SM_WARPS) {
        if (lane == 0) {
            for (int i = 0; i < 2; ++i) {
                mbar_init(q_full(i), 1);
                mbar_init(q_empty(i), 1);
                mbar_init(s_full(i), 1);
                mbar_init(p_full(i), 4);
                mbar_init(p2_full(i), 4);
                mbar_init(pv_done(i), 1);
                mbar_init(o_free(i), 4);
                mbar_init(s_free(i), 4);
            }
            mbar_init(bar_drain, NT);
            for (int i = 0; i < kTcMaxStages; ++i) {
                mbar_init(k_full(i), 1);
                mbar_init(v_full(i), 1);
                mbar_init(k_empty(i), NT);  // (each row tile's MMA warp)
                mbar_init(v_empty(i), NT);
            }
            for (int i = 0; i < kTcSegs; ++i) {
                mbar_init(seg_full(i), 1);
                mbar_init(seg_empty(i), S::SM_WARPS + 2 * NT - 1);  // softmax, MMA and (NT = 2) V warps
            }
            mbar_fence_init_smem();
            *abort_flag = 0;
        }
        __syncwarp();
        tc_alloc(smem_u32(tmem_ptr), S::TMEM_COLS);
    }
    // units and slot tiles before each sequence: every thread takes a run of sequences.  (The host makes sure that the sums fit
    // 31 bits.)
    const int per = (a.kv.n_seqs + S::THREADS - 1) / S::THREADS, s0 = tid * per, s1 = min(s0 + per, a.kv.n_seqs);
    auto scan = [&](int sum, int* out) {  // out[s + 1] holds the sums within this thread's run
        int inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += up;
        }
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        int before = inc - sum;
        for (int w = 0; w < warp; ++w) before += wsum[w];
        for (int s = s0; s < s1; ++s) out[s + 1] += before;
        if (tid == 0) out[0] = 0;
        __syncthreads();
    };
    if (PART) {  // (slots in common: behind the kernel that makes the groups; own slots: beside this one, see the end)
        if (a.kv.row_of) grid_dep_wait();
        grid_dep_launch();
    }
    if (!PART && ta.split) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (the joining kernel waits for this one's end)
    const bool by_tiles = NT == 1 && ta.split;  // every unit may be cut: its slot tiles are all that is counted
    {
        int sum = 0;
        for (int s = s0; s < s1; ++s) {
            SeqInfo v;
            int t1;
            chunk_of(a.kv, s, v.t0, t1);
            v.n = t1 - v.t0;
            v.len = live_len(a.kv, s, v.n, blockIdx.x == 0 && !(PART && a.kv.row_of));
            v.lo = a.start ? max(__ldcg(a.start + s), 0) : 0;  // (from L2: with PART written by a kernel before the last)
            info[s] = v;
            sum += (v.n + NT * a.tq - 1) / (NT * a.tq) * a.kv.n_kv_heads * (by_tiles ? Work::items_of_unit(v) : 1);
            (by_tiles ? items : pre)[s + 1] = sum;
        }
        scan(sum, by_tiles ? items : pre);
    }
    Work work;
    work.info = info;
    work.pre = pre;
    work.items = items;
    work.n_seqs = a.kv.n_seqs;
    work.tq = a.tq;
    work.causal = a.causal;
    work.x = blockIdx.x;
    work.step = gridDim.x;
    work.end = by_tiles ? 0 : pre[a.kv.n_seqs];
    work.y = work.y_end = 0;
    work.first_cut = work.end;
    int total = 0, n_ranges = 0;  // slot tiles that are dealt out in ranges, and the CTAs that get one
    if (ta.split) {
        if (NT == 2) {
            const int first = work.end / gridDim.x * gridDim.x, left = work.end - first;
            int sum = 0;
            for (int s = s0; s < s1; ++s) {
                const int n = pre[s + 1] - max(first, pre[s]);
                if (n > 0) sum += n * Work::items_of_unit(info[s]);
                items[s + 1] = sum;
            }
            scan(sum, items);
            total = items[a.kv.n_seqs];
            // a last round that fills most of the CTAs, or whose idle ones would wait for a few slot tiles only, stays whole
            if ((long long)total * (gridDim.x - left) >= (long long)(PART ? kCutTilesJoined : kCutTiles) * left * gridDim.x) work.end = work.first_cut = first;
            else total = 0;
        } else {
            total = items[a.kv.n_seqs];
        }
        n_ranges = min((total + ta.min_items - 1) / ta.min_items, (int)gridDim.x);
        if ((int)blockIdx.x < n_ranges) {
            work.y = (int)((long long)total * blockIdx.x / n_ranges);
            work.y_end = (int)((long long)total * (blockIdx.x + 1) / n_ranges);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_ptr;

    // The K producer works out the steps and leaves them in a ring; the other warps (MMA: one thread) read them from there.
    int seg_no = 0;
    auto next_seg = [&](TcSeg& g, bool one_thread) {
        const int r = seg_no % kTcSegs;
        const uint32_t turn = (seg_no / kTcSegs) & 1;
        ++seg_no;
        if (!(one_thread ? wait_or_abort(seg_full(r), turn, abort_flag) : warp_wait(seg_full(r), turn, abort_flag))) return false;
        g = seg_ring[r];
        if (!one_thread) __syncwarp();
        if (one_thread || lane == 0) mbar_arrive(seg_empty(r));
        return g.nb >= 0;
    };
    if (NT == 2) {
        if (warp < S::SM_WARPS)
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::SM_REGS));
        else
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::OTHER_REGS));
    }
    if (warp < S::SM_WARPS) {
        // ------------------------------------------------------------------ softmax: one thread per row
        const int tile = warp >> 2, w4 = warp & 3;
        const uint32_t lane_base = (uint32_t)(w4 * 32) << 16;
        const uint32_t tm_o = tmem + lane_base + S::O_COL + tile * D;
        const int row = w4 * 32 + lane;
        const int G = a.group;
        const float sc = a.scale_log2;
        int steps = 0;     // softmax steps of this row tile so far
        RingPos ring0;     // stage of the segment's first slot tile
        bool ok = true, recorded = false;
        // The product of a step is over.  A parity wait is safe only for the newest phase a barrier can be in, with the phase before it known
        // to be over.  NT = 2: every step waits for the one before.  NT = 1 waits now and then, so each logit buffer has a
        // barrier of its own: the logits of step s show that the product of s - 2 (same buffer) is over, and that of s + 1 needs P
        // which has not been handed over yet.
        auto product_wait = [&](int s) {
            const bool done = NT == 2 ? warp_wait(pv_done(tile), s & 1, abort_flag) : warp_wait(pv_done(s & 1), (s >> 1) & 1, abort_flag);
            tc_fence_after();
            return done;
        };
        TcSeg g;
        while (ok && next_seg(g, false)) {
            const int n = g.nb;
            const int nt = min(a.tq, g.n_tok - tile * a.tq);  // tokens of this row tile
            const int rows = nt > 0 ? nt * G : 0;
            const int t = row / G, head_g = row - t * G;
            const int slot_first = g.slot0 + tile * a.tq;
            const int last = row >= rows ? -1 : a.causal ? min(slot_first + t, g.len - 1) : g.len - 1;
            const int min_last = a.causal ? min(slot_first, g.len - 1) : g.len - 1;
            const bool active = w4 * 32 < rows;
            float m_used = -INFINITY, l = 0.f;
            for (int j = 0; j < n; ++j) {
                const int buf = NT == 2 ? tile : (steps & 1);
                const int sp = NT == 2 ? (steps & 1) : ((steps >> 1) & 1);
                if (!(ok = warp_wait(s_full(buf), sp, abort_flag))) break;
                tc_fence_after();
                const int base_slot = (g.jb + j) * BN;
                if (base_slot < g.lo || base_slot + BN > g.len) {
                    // value rows of slots that are not live: cleared (by each row tile's warps for their own product: both write zeros)
                    RingPos rp = ring0;
                    rp.skip(j, NS);
                    if (!(ok = warp_wait(v_full(rp.st), rp.ph, abort_flag))) break;
                    const int slot = base_slot + row;
                    if (row < BN && (slot < g.lo || slot >= g.len)) {
                        const uint32_t at = ring + rp.st * S::STAGE_BYTES + S::TILE_BYTES + row * 128;
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at + h * BN * 128 + c * 16), "r"(0) : "memory");
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                uint32_t s[BN];
                if (active) {
                    const uint32_t tm_s = tmem + lane_base + S::s_col(buf);
#pragma unroll
                    for (int c = 0; c < BN; c += 32) tc_ld32(tm_s + c, s + c);
                    tc_wait_ld();
                }
                if (NT == 2) {  // the logit buffer goes to the other row tile
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_free(tile));
                }
                // NT = 2: before P is stored, P of the step before has been read (NT = 1 has two buffers); before the accumulator is
                // rescaled, the products of all steps before are in it
                bool product_over = j == 0;
                if (active) {
                    const uint32_t tm_p = tmem + lane_base + S::p_col(buf);
                    if (base_slot < g.lo || base_slot + BN - 1 > min_last) {
                        const int c_lo = g.lo - base_slot, c_hi = last - base_slot;
#pragma unroll
                        for (int c = 0; c < BN; ++c)
                            if (c > c_hi) s[c] = 0xff800000u;
                        if (c_lo > 0) {
#pragma unroll
                            for (int c = 0; c < BN; ++c)
                                if (c < c_lo) s[c] = 0xff800000u;
                        }
                    }
                    float mx[4] = {m_used, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < BN; c += 8)
#pragma unroll
                        for (int i = 0; i < 4; ++i) mx[i] = fmaxf(fmaxf(mx[i], __uint_as_float(s[c + i])), __uint_as_float(s[c + 4 + i]));
                    const float m_new = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    const bool grow = row < rows && m_new > m_used && (m_new - m_used) * sc > 8.f;
                    if (j == 0) {
                        m_used = m_new;
                    } else if (__any_sync(0xffffffffu, grow)) {
                        if (!(ok = product_wait(steps - 1))) break;
                        product_over = true;
                        const float f = !grow ? 1.f : m_used == -INFINITY ? 0.f : ScaledRef(m_used, sc).ratio_to(m_new);
                        l *= f;
                        if (grow) m_used = m_new;
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t o[32];
                            tc_ld32(tm_o + c, o);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tc_st32(tm_o + c, o);
                        }
                    }
                    const ScaledRef ref(m_used, sc);
                    const uint64_t sc2 = pack_f32x2(ref.scale, ref.scale), mr2 = pack_f32x2(-ref.scaled, -ref.scaled);
                    uint64_t sum2[2] = {0, 0};
#pragma unroll
                    for (int c = 0; c < BN; c += 64) {
                        uint32_t p[32];
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            float x, y;
                            const uint64_t v = fma_f32x2(pack_f32x2(__uint_as_float(s[c + 2 * i]), __uint_as_float(s[c + 2 * i + 1])), sc2, mr2);
                            unpack_f32x2(v, x, y);
                            x = ex2_approx(x);
                            y = ex2_approx(y);
                            sum2[i & 1] = add_f32x2(sum2[i & 1], pack_f32x2(x, y));
                            p[i] = pack_bf16(x, y);
                        }
                        if (NT == 2 && c == 0 && !product_over) {
                            if (!(ok = product_wait(steps - 1))) break;
                        }
                        tc_st32(tm_p + c / 2, p);
                        if (c + 64 < BN) {  // the first part goes ahead
                            tc_wait_st();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(p_full(buf));
                        }
                    }
                    if (!ok) break;
                    float s0, s1, s2, s3;
                    unpack_f32x2(sum2[0], s0, s1);
                    unpack_f32x2(sum2[1], s2, s3);
                    l += (s0 + s1) + (s2 + s3);
                    tc_wait_st();
                } else if (NT == 2) {
                    // (a warp without rows keeps step with the products too: it waits for every phase in turn)
                    if (!product_over && !(ok = product_wait(steps - 1))) break;
                    if (lane == 0) mbar_arrive(p_full(buf));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(S::P_PARTS == 2 ? p2_full(buf) : p_full(buf));
                ++steps;
            }
            if (!ok) break;
            // the output rows, or this CTA's part of them
            if (n > 0 && !(ok = product_wait(steps - 1))) break;
            const bool mine = row < rows;
            const int slotp = blockIdx.x * 2 + (g.b0 > 0 ? 0 : 1);
            if (active) {
                // nothing seen: 0; NaN stays NaN.  Parts are joined by their references as they are.
                const bool done = g.whole && !PART;
                const float inv = done ? (l > 0.f ? 1.0f / l : l) : ScaledRef(m_used, sc).rounding();
                const size_t part = ((size_t)slotp * NT + tile) * ta.rows_cap + row;
                // a thread has a row, but four neighbours write 64 bytes of one row together
                unsigned long long own_row = 0;
                const size_t all = (size_t)(g.tok0 + tile * a.tq + t) * (a.kv.n_kv_heads * G) + g.head * G + head_g;  // (PART)
                if (PART && mine && g.whole)
                    own_row = reinterpret_cast<unsigned long long>(a.row_o + all * D);
                else if (mine)
                    own_row = g.whole ? reinterpret_cast<unsigned long long>(a.out.p) + 2 * ((long long)(g.tok0 + tile * a.tq + t) * a.out.token_stride + (long long)(g.head * G + head_g) * a.out.head_stride)
                                      : reinterpret_cast<unsigned long long>(a.part_o + part * D);
                char* rows4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) rows4[i] = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, own_row, (lane & 28) + i));
                auto put = [&](uint4 (&c)[4], int offset) {
                    quad_transpose(c, lane);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (rows4[i]) *reinterpret_cast<uint4*>(rows4[i] + offset + (lane & 3) * 16) = c[i];
                };
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    if (n > 0) {
                        tc_ld32(tm_o + c, o);
                        tc_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0;
                    }
                    uint4 u[4];
                    if (done) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            u[i].x = pack_bf16(__uint_as_float(o[8 * i]) * inv, __uint_as_float(o[8 * i + 1]) * inv);
                            u[i].y = pack_bf16(__uint_as_float(o[8 * i + 2]) * inv, __uint_as_float(o[8 * i + 3]) * inv);
                            u[i].z = pack_bf16(__uint_as_float(o[8 * i + 4]) * inv, __uint_as_float(o[8 * i + 5]) * inv);
                            u[i].w = pack_bf16(__uint_as_float(o[8 * i + 6]) * inv, __uint_as_float(o[8 * i + 7]) * inv);
                        }
                        put(u, c * 2);
                    } else {
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[h + i] = __float_as_uint(__uint_as_float(o[h + i]) * inv);
#pragma unroll
                            for (int i = 0; i < 4; ++i) u[i] = make_uint4(o[h + 4 * i], o[h + 4 * i + 1], o[h + 4 * i + 2], o[h + 4 * i + 3]);
                            put(u, (c + h) * 4);
                        }
                    }
                    __syncwarp();  // (tcgen05.ld is a warp-wide instruction: all lanes together again)
                }
                if (PART && mine && g.b0 == 0) a.row_ref[all] = make_int2(g.whole ? -1 : (int)blockIdx.x + 65536 * g.unit_end, tile * ta.rows_cap + row);
                if (mine && !done) {
                    float* ml = PART && g.whole ? a.row_ml + all * 2 : a.part_ml + part * 2;
                    ml[0] = m_used;  // (-inf: nothing seen)
                    ml[1] = l * inv;
                }
            }
            if (!g.whole && g.b0 == 0) {
                // the unit goes on in the next CTAs: up to the one that holds its last item
                if (tid == 0) ta.records[blockIdx.x] = make_int4(g.tok0, g.n_tok, g.head, g.unit_end);
                recorded = true;
            }
            if (n > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(o_free(tile));
            }
            ring0.skip(n, NS);
        }
        if (ta.split && !recorded && tid == 0) ta.records[blockIdx.x] = make_int4(0, 0, 0, 0);
    } else if (warp == S::SM_WARPS || (NT == 2 && warp == S::SM_WARPS + 3)) {
        // ------------------------------------------------------------------ MMA: one thread per row tile, so that a wait for one row tile
        // holds up nothing of the other
        if (lane == 0) {
            constexpr uint32_t id_s = tc_idesc(BN, false), id_o = tc_idesc(D, true);
            // Shared-memory matrix descriptors, 128-byte swizzle.  K-major rows of 128 bytes (64 elements of the contracted dimension): groups of
            // 8 rows lie 1024 bytes apart.  Slots-as-K (V): 64 columns per 128-byte row, column blocks BN * 128 bytes apart, groups of 8 slots
            // 1024 apart.  Low word: address / 16 | column-block distance / 16 << 16; high word: group distance / 16 | version 1 << 14 |
            // 128-byte swizzle << 29.
            constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
            constexpr uint32_t kStage = S::STAGE_BYTES >> 4;
            const int tile = warp == S::SM_WARPS ? 0 : 1;
            const uint32_t qa = ((base + tile * q_tile) >> 4) | (1u << 16), qb = qa + (q_half >> 4), k_lo = (ring >> 4) | (1u << 16);
            const uint32_t v_lo = ((ring + S::TILE_BYTES) >> 4) | ((uint32_t)(BN * 128 >> 4) << 16);
            const uint32_t tm_o = tmem + S::O_COL + tile * D;
            RingPos kp, vp;     // next K tile to form logits with, V tile of the current step
            int formed = 0;     // logit tiles formed so far
            int steps = 0;      // products issued so far
            int segs = 0;       // segments with steps so far
            bool ok = true;
            // S = Q K^T with the K tile at kp.  NT = 2: the two row tiles use the logit buffer in turn, and each use waits until
            // the one before it has been taken into registers.
            auto form_logits = [&](bool last) {
                if (!wait_or_abort(k_full(kp.st), kp.ph, abort_flag)) return false;
                if (NT == 2 && tile + formed > 0 && !wait_or_abort(s_free(1 - tile), (formed - 1 + tile) & 1, abort_flag)) return false;
                tc_fence_after();
                const int buf = NT == 2 ? tile : formed & 1;
                const uint32_t ka = k_lo + kp.st * kStage, d = tmem + S::s_col(buf);
                tc_mma_ss<kDescHigh, 0, 0>(d, qa, ka, id_s, false);
                tc_mma_ss<kDescHigh, 2, 2>(d, qa, ka, id_s, true);
                tc_mma_ss<kDescHigh, 4, 4>(d, qa, ka, id_s, true);
                tc_mma_ss<kDescHigh, 6, 6>(d, qa, ka, id_s, true);
                if (HALVES == 2) {
                    const uint32_t kb = ka + BN * 128 / 16;
                    tc_mma_ss<kDescHigh, 0, 0>(d, qb, kb, id_s, true);
                    tc_mma_ss<kDescHigh, 2, 2>(d, qb, kb, id_s, true);
                    tc_mma_ss<kDescHigh, 4, 4>(d, qb, kb, id_s, true);
                    tc_mma_ss<kDescHigh, 6, 6>(d, qb, kb, id_s, true);
                }
                tc_commit(s_full(buf));
                if (NT == 2) tc_commit(k_empty(kp.st));
                if (last) tc_commit(q_empty(tile));
                kp.next(NS);
                ++formed;
                return true;
            };
            auto add_values = [&](int buf, bool acc, int k0) {  // O += P V, slots k0 * 16 .. + 63 of the V tile at vp
                const uint32_t va = v_lo + vp.st * kStage + k0 * 128, pa = tmem + S::p_col(buf) + k0 * 8;
                tc_mma_ts<kDescHigh, 0, 0>(tm_o, pa, va, id_o, acc);
                tc_mma_ts<kDescHigh, 8, 128>(tm_o, pa, va, id_o, true);
                tc_mma_ts<kDescHigh, 16, 256>(tm_o, pa, va, id_o, true);
                tc_mma_ts<kDescHigh, 24, 384>(tm_o, pa, va, id_o, true);
            };
            TcSeg g;
            while (ok && next_seg(g, true)) {
                const int n = g.nb;
                if (n == 0) continue;
                if (!(ok = wait_or_abort(q_full(tile), segs & 1, abort_flag))) break;
                ok = form_logits(n == 1);
                for (int j = 0; ok && j < n; ++j) {
                    // the logits of the next step come first, so that they are there when the softmax of this step is done
                    if (j + 1 < n) {
                        ok = form_logits(j + 2 == n);
                        if (!ok) break;
                    }
                    const int buf = NT == 2 ? tile : steps & 1, pp = NT == 2 ? steps & 1 : (steps >> 1) & 1;
                    if (!(ok = wait_or_abort(v_full(vp.st), vp.ph, abort_flag))) break;
                    if (j == 0 && segs > 0 && !(ok = wait_or_abort(o_free(tile), (segs - 1) & 1, abort_flag))) break;
                    if (!(ok = wait_or_abort(p_full(buf), pp, abort_flag))) break;
                    tc_fence_after();
                    add_values(buf, j > 0, 0);
                    if (S::P_PARTS == 2) {
                        if (!(ok = wait_or_abort(p2_full(buf), pp, abort_flag))) break;
                        tc_fence_after();
                        add_values(buf, true, 4);
                    }
                    tc_commit(pv_done(buf));
                    tc_commit(NT == 2 ? v_empty(vp.st) : k_empty(vp.st));
                    ++steps;
                    vp.next(NS);
                }
                ++segs;
            }
            // everything issued has completed before TMEM is given back
            tc_commit(bar_drain);
            mbar_wait_bounded(bar_drain, 0);
        }
        __syncwarp();
    } else if (warp <= S::SM_WARPS + NT) {
        // ------------------------------------------------------------------ producers: NT = 2 one warp for Q and K and one for V (a K tile's
        // place is free as soon as its logits are formed, a V tile's a step later); NT = 1 one warp, lanes 0-15 K and 16-31 V
        const bool k_warp = warp == S::SM_WARPS + 1;
        int issued = 0, segs[2] = {0, 0};
        RingPos kv;
        bool ok = true;
        const int nbox = BN / ta.box_rows;  // boxes of 64 columns of a tile (at most 8)
        const int is_v = NT == 2 ? !k_warp : lane >> 4, idx = NT == 2 ? lane : lane & 15, box = idx & (nbox - 1), half = idx / nbox;
        const bool boxes = half < HALVES;
        const int box_slot = box * ta.box_rows, row_mask = a.kv.page_tokens - 1;
        const int cap = a.kv.table_cols << a.kv.page_shift;
        const uint32_t dst0 = ring + is_v * S::TILE_BYTES + half * (BN * 128) + box_slot * 128;
        const CUtensorMap* map = is_v ? &maps.v : &maps.k;
        const uint32_t full0 = is_v ? v_full(0) : k_full(0), empty0 = NT == 2 && is_v ? v_empty(0) : k_empty(0);
        TcSeg g;
        int unit = blockIdx.x, asked = 0;  // whole units handed out on demand: this one, and what the counter gave for the next
        for (;;) {
            if (k_warp) {
                bool more = true;
                if (ta.counter) {
                    if (seg_no > 0) unit = gridDim.x + __shfl_sync(0xffffffffu, asked, 0);
                    work.x = unit;
                    if (lane == 0 && unit < work.end) asked = atomicAdd(ta.counter, 1);  // (used a unit later)
                }
                more = work.next(g);
                if (!more) g.nb = -1;
                else if (!g.whole) g.unit_end = (int)(((long long)g.unit_end * n_ranges + total - 1) / total - 1);  // the CTA with its last item
                const int r = seg_no % kTcSegs;
                if (seg_no >= kTcSegs && !(ok = warp_wait(seg_empty(r), (seg_no / kTcSegs - 1) & 1, abort_flag))) break;
                ++seg_no;
                if (lane == 0) {
                    seg_ring[r] = g;
                    mbar_arrive(seg_full(r));
                }
                if (!more) break;
            } else if (!next_seg(g, false)) {
                break;
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if (g.nb == 0 || !k_warp) continue;
                if (segs[i] > 0 && !(ok = warp_wait(q_empty(i), (segs[i] - 1) & 1, abort_flag))) break;
                ++segs[i];
                if (lane == 0) {
                    mbar_expect_tx(q_full(i), (uint32_t)(a.tq * a.group * 128 * HALVES));
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) tma_load_4d(base + i * q_tile + h * q_half, &maps.q, h * 64, 0, g.head, g.tok0 + i * a.tq, q_full(i));
                }
            }
            if (!ok) break;
            const int* table = a.kv.table + (PART && a.kv.row_of ? a.kv.row_of[g.seq] : g.seq) * a.kv.table_seq_stride + g.head * a.kv.table_head_stride;
            const int head_c = a.kv.head_stride > 0 ? g.head : 0;
            const int nmax = g.nb, len = min(g.len, cap), lo = g.lo;
            int slot = g.jb * BN + box_slot;  // first slot of this lane's box
            auto page_of = [&](int slot) {
                int page = a.kv.n_pages;  // outside the tensor: the box is filled with zeros
                if (boxes && slot < len && slot + ta.box_rows > lo) {
                    const int p = table[slot >> a.kv.page_shift];
                    if (p >= 0 && p < a.kv.n_pages) page = p;
                    else paged_report(a.kv, kStPage);
                }
                return page;
            };
            int page = nmax > 0 ? page_of(slot) : 0;
            for (int j = 0; j < nmax; ++j) {
                const int page_next = j + 1 < nmax ? page_of(slot + BN) : 0;
                if (issued >= NS && !(ok = warp_wait(empty0 + 8u * kv.st, kv.ph ^ 1, abort_flag))) break;
                if (NT == 2 ? lane == 0 : idx == 0) mbar_expect_tx(full0 + 8u * kv.st, S::TILE_BYTES);
                __syncwarp();
                if (boxes) tma_load_4d(dst0 + kv.st * S::STAGE_BYTES, map, half * 64, slot & row_mask, head_c, page, full0 + 8u * kv.st);
                ++issued;
                kv.next(NS);
                slot += BN;
                page = page_next;
            }
            if (!ok) break;
        }
        if (!ok && (NT == 2 ? lane == 0 : idx == 0)) {
            // given up: the copies in flight land before the CTA's shared memory goes to somebody else
            for (int i = 0; i < NT; ++i)
                if (segs[i] > 0) mbar_wait_bounded(q_full(i), (segs[i] - 1) & 1);
            for (int n = issued > NS ? issued - NS : 0; n < issued; ++n) mbar_wait_bounded(full0 + 8u * (n % NS), (n / NS) & 1);
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == S::SM_WARPS) tc_dealloc(tmem, S::TMEM_COLS);
    if (tid == 0 && *abort_flag) paged_report(a.kv, kStWaitLimit);
    if (PART && !a.kv.row_of) grid_dep_wait();  // (who waits for this kernel's end has waited for the other's)
}

// Adds up the parts of the units that range boundaries cut, in the order of the CTAs that left them.
template <int D, int NT>
__global__ void __launch_bounds__(128) join_ranges_kernel(const __grid_constant__ TcArgs ta) {
    grid_dep_wait();
    const PagedAttnArgs& a = ta.a;
    const int4 rec = ta.records[blockIdx.x];  // first token, tokens, head, last CTA
    const int c0 = blockIdx.x, c1 = min(rec.w, (int)gridDim.x - 1);
    // four columns of a row per thread
    for (int i = blockIdx.y * blockDim.x + threadIdx.x; i < rec.y * a.group * (D / 4); i += gridDim.y * blockDim.x) {
        const int unit_row = i / (D / 4), e = (i - unit_row * (D / 4)) * 4;  // (token, head of the group) of the unit
        const int t = unit_row / a.group, tile = NT == 2 && t >= a.tq ? 1 : 0, row = unit_row - tile * a.tq * a.group;
        auto at = [&](int c) { return ((size_t)(c * 2 + (c == c0 ? 1 : 0)) * NT + tile) * ta.rows_cap + row; };
        float M = -INFINITY, L = 0.f;  // (one pass with a running maximum: the loads of all parts are under way at once)
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int c = c0; c <= c1; ++c) {
            const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + at(c) * 2);
            const float4 p = *reinterpret_cast<const float4*>(a.part_o + at(c) * D + e);
            const float mn = fmaxf(M, ml.x), ref = softmax_ref(mn);
            const float f0 = ex2_approx((M - ref) * a.scale_log2), f = ex2_approx((ml.x - ref) * a.scale_log2);
            M = mn;
            L = fmaf(ml.y, f, L * f0);
            o.x = fmaf(p.x, f, o.x * f0);
            o.y = fmaf(p.y, f, o.y * f0);
            o.z = fmaf(p.z, f, o.z * f0);
            o.w = fmaf(p.w, f, o.w * f0);
        }
        const float inv = L > 0.f ? 1.0f / L : L;
        const int h = rec.z * a.group + unit_row - t * a.group;
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(a.out.p) + (long long)(rec.x + t) * a.out.token_stride + (long long)h * a.out.head_stride + e;
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    }
}

}  // namespace lar
