// Attention over the 8-bit paged cache for many query rows per key head: prompts and chunks of them (d = 64 and 128).
//
// The rows of a sequence and key head are its queries times the G query heads of the group; an item is a slab of 256 of them, two tiles
// of 128, against the keys that they see, in steps of 64.  Logits and outputs are tcgen05 products in half precision with fp32
// accumulators in TMEM.  e4m3 numbers are exact in half precision: one warp looks the pages up and copies them (bulk copies of sixteen
// tokens), four warps turn them into half-precision tiles in the 128-byte swizzle and take the page's scale into them, relative to the
// largest of the part's pages: k 2^(ek - EK + 6), exact in pages whose scale is within 2^-21 of it.  So the softmax sees one scale.
// Queries are scaled by a power of two a row into half precision (it goes into the row's softmax constant); weights are 2^9 w, rounded
// to half precision.
//
// CTA = 512 threads: warps 0-3 / 4-7 softmax of tile A / B (thread = row = TMEM lane), warps 8 / 9 MMA issuers of tile A / B (one
// elected lane), warp 10 look-ups and copies, warp 11 idle (it completes a warpgroup for the register hand-over), warps 12-15 convert.
// TMEM columns: S(t, b) 128 t + 64 b (b = step parity), P over the first 32 of them, O_t 256 + 128 t.
// The softmax takes no row maximum after the first step: any reference gives the exact softmax; a step whose row sum passes 60,000
// (a weight could pass the largest half-precision number) is redone with a fresh maximum.  One exponential in eight goes through a
// polynomial on the FMA pipe.  Every wait is bounded (tc_common.cuh); on expiry the CTA aborts cleanly and reports a code.
//
// What bounds it, d = 128: shared memory's port and the softmax warps together.  A step of both tiles moves 1,024 cycles of operands
// for the tensor pipe (A of the logits alone 512) and 512 of conversions; its exponentials take 1,010 cycles of the exponent unit;
// measured 1,750 cycles (of 1,920 in an earlier form the softmax took 1,270 to work and 330 to wait for logits).  4,096 queries behind
// 28,672 tokens, 32 heads on 8: 1,580 us in the first 20 ms of launches (1,305 TFLOP/s), 1,830 at the power cap (1,120; a cuBLAS GEMM
// 1,639 and 1,396).  d = 64: 580 TFLOP/s, by the softmax warps, a thread a row, two warps a scheduler, which load, compute, store and wait in turn: 1,250 of
// 1,700 cycles a step at work (the exponent unit 900).  How long a step takes also depends on the code around it: with masked steps in a
// loop instead of unrolled 128 items of d = 128 take 480 us against 488.  Tried, on 128 items: the converters' own cp.async (their addresses
// were half of a step: 587 us against 522), logits of two steps in one product (N = 128, one buffer a tile: 567 against 522; d = 64 494
// against 466), no polynomial 524 and one in sixteen 524 against 512, one in four 513 (d = 64 456 against 459).
// Where there are few steps: 200 queries of 32 heads on 8 13.8 us, of which the launch 2.5, the deal 1.6, queries and exponents 2, the first
// step 1.6, the output 2.
// Items: those of the last round, or all if they are fewer than the SMs, are split along the keys (128 queries, 32 heads on 8, over
// 32,768 keys: 537 -> 99 us).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cache_common.cuh"
#include "flat_internal.cuh"
#include "ptx_sm100.cuh"
#include "tc_common.cuh"

namespace flat {

using namespace cache;
using namespace ptx;
using namespace tc;

namespace {

constexpr int BM = 128, BN = 64, THREADS = 512;
constexpr int KS = 3, VS = 3;                            // stages of half-precision keys and values
constexpr int POLY_LANE = 3;                             // element index mod 8 that takes the polynomial
// Weights at the reference maximum are 2^9: 64 of them add up to half of MOST_SUM, so that a step passes it only where the reference is
// exceeded, and what half precision rounds away lies 2^34 below the reference.
constexpr float SHIFT = 9.f, MOST_SUM = 60000.f;
constexpr int LIFT = 6;                                  // log2: the largest e4m3 number times 2^6 is 28,672

__host__ __device__ constexpr uint32_t S_COL(int t, int b) { return 128u * t + 64u * b; }
__host__ __device__ constexpr uint32_t O_COL(int t) { return 256u + 128u * t; }

template <int D> struct Layout {
    static constexpr int LS = D == 128 ? 4 : 6;          // steps of pages on their way
    static constexpr int Q_BYTES = BM * D * 2, KV_BYTES = BN * D * 2, RAW_BYTES = BN * D;
    static constexpr int K_AT = 2 * Q_BYTES, V_AT = K_AT + KS * KV_BYTES, RAW_AT = V_AT + VS * KV_BYTES, BARS_AT = RAW_AT + LS * 2 * RAW_BYTES;
    static constexpr int Q_FULL = 0, K_FULL = 2, K_EMPTY = K_FULL + KS, V_FULL = K_EMPTY + KS, V_EMPTY = V_FULL + VS, S_FULL = V_EMPTY + VS,
                         P_FULL = S_FULL + 4, PV_DONE = P_FULL + 4,
                         EXPS_READY = PV_DONE + 4, SCALE_FULL = EXPS_READY + 1, RAW_FULL = SCALE_FULL + 2, SCALE_EMPTY = RAW_FULL + LS,
                         RAW_EMPTY = SCALE_EMPTY + 2, NUM_BARS = RAW_EMPTY + LS;
    static constexpr int SMEM_BYTES = BARS_AT + NUM_BARS * 8 + 32 + 1024;
    static_assert(SMEM_BYTES <= 232448, "shared memory");
};

// Instruction descriptor of kind::f16 with half-precision A and B, fp32 accumulator.
__host__ __device__ constexpr uint32_t idesc_half(int M, int N, int b_mn_major) {
    return (1u << 4) | (static_cast<uint32_t>(b_mn_major) << 16) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float two_to(int e) {         // 2^e for any e: 0 below, the largest power above
    e = e < -127 ? -127 : e > 127 ? 127 : e;
    return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// Of sixteen logits p_i = 2^(s_i * unit + neg_m), rounded to half precision into eight TMEM columns at `p_addr`; the fp32 sums of the
// unrounded p go to sum0 and sum1 (a NaN logit makes them NaN or, through the polynomial, 2^126: the step is redone then).  TAIL: only the first `nvalid` take part.
template <bool TAIL>
__device__ __forceinline__ void exp16(const uint32_t* s, uint64_t unit2, uint64_t neg_m2, uint32_t p_addr, int nvalid, uint64_t& sum0, uint64_t& sum1) {
    uint32_t pk[8];
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; i += 2) unpack2(fma2(pack2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), unit2, neg_m2), p[i], p[i + 1]);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        p[i] = !TAIL && (i & 7) == POLY_LANE ? ex2_poly<true>(p[i]) : ex2_approx(p[i]);
        if (TAIL && i >= nvalid) p[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        sum0 = add2(sum0, pack2(p[i], p[i + 1]));
        sum1 = add2(sum1, pack2(p[i + 2], p[i + 3]));
        pk[i / 2] = pack_half2(p[i], p[i + 1]);
        pk[i / 2 + 1] = pack_half2(p[i + 2], p[i + 3]);
    }
    tmem_st_x8(p_addr, pk);
}
__device__ __forceinline__ float total(uint64_t sum0, uint64_t sum1) {
    float a, b, c, d;
    unpack2(sum0, a, b);
    unpack2(sum1, c, d);
    return (a + b) + (c + d);
}
// The weights of a step's 64 logits over the first half of their columns (sixteen at a time: 128 items of d = 128 518 us against 530 by
// the 32, d = 64 453 against 465); returns their sum.
__device__ __forceinline__ float exp_store(const uint32_t (&s)[BN], float unit, float neg_m, uint32_t s_addr) {
    uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll
    for (int c = 0; c < BN / 16; ++c) exp16<false>(s + c * 16, pack2(unit, unit), pack2(neg_m, neg_m), s_addr + c * 8, 16, sum0, sum1);
    return total(sum0, sum1);
}
// The same out of TMEM, for the first `nvalid` keys, of those not the groups of sixteen in `out` (a loop: this is rare, and the shorter the
// kernel's code the better its common steps run).  A group's weights go over logits that have been read.
__device__ __forceinline__ float exp_store_tail(float unit, float neg_m, uint32_t s_addr, int nvalid, int out) {
    uint64_t sum0 = 0ull, sum1 = 0ull;
#pragma unroll 1
    for (int c = 0; c < BN / 16; ++c) {
        uint32_t s[16];
        tmem_ld_x16(s_addr + c * 16, s);
        tc_wait_ld();
        exp16<true>(s, pack2(unit, unit), pack2(neg_m, neg_m), s_addr + c * 8, out >> c & 1 ? 0 : nvalid - c * 16, sum0, sum1);
    }
    return total(sum0, sum1);
}
// The largest unit * s of the keys that take part.
__device__ __forceinline__ float row_max(const uint32_t (&s)[BN], float unit, int nvalid, int out) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < BN; ++i)
        if (i < nvalid && !(out >> (i / 16) & 1)) m = fmaxf(m, __uint_as_float(s[i]) * unit);
    return m;
}

// Sixteen e4m3 (a piece) times a half-precision pair `by`.
__device__ __forceinline__ void widen16(const uint32_t (&w)[4], __half2 by, uint32_t (&h)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t lo, hi;
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w[i]));
        const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&lo), by), y = __hmul2(*reinterpret_cast<const __half2*>(&hi), by);
        h[2 * i] = *reinterpret_cast<const uint32_t*>(&x);
        h[2 * i + 1] = *reinterpret_cast<const uint32_t*>(&y);
    }
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void lds16(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// `bytes` (a multiple of 16, like both addresses) to shared memory of this CTA; they count on the mbarrier.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

template <int N> struct Const { static constexpr int value = N; };
struct PrefillArgs {
    CacheView c;
    const __nv_bfloat16* Q;
    __nv_bfloat16* O;
    float* lse;
    long long q_st, q_sh, o_st, o_sh, total;
    int Hq, G, max_new, least_rows, causal;              // sequences of at most least_rows rows are not this kernel's
    float scale_log2e;
    int sms, most_items;                                 // CTAs that run at a time; items that the grid was made for
    int* counters;                                       // [sms][8], 0 between launches
    float* part_lse;                                     // [sms][2 BM], base 2
    float* part_o;                                       // [sms][D / 4][2 BM][4]
};

// One row of an item (place `in` of its 256) from its parts: their normalised outputs and log-sums.
template <int D>
__device__ __forceinline__ void join_rows(const PrefillArgs& p, int slot0, int parts, int in, bool there, int token, int head) {
    const float* lse = p.part_lse + slot0 * 2 * BM + in;
    float top = -INFINITY, sum = 0.f;
    for (int i = 0; i < parts; ++i) top = fmaxf(top, __ldcg(lse + i * 2 * BM));
    const float ref = top == -INFINITY ? 0.f : top;
    for (int i = 0; i < parts; ++i) sum += ex2_approx(__ldcg(lse + i * 2 * BM) - ref);
    const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
    if (p.lse && there) p.lse[static_cast<int64_t>(token) * p.Hq + head] = (sum > 0.f ? ref + log2f(sum) : sum == sum ? -INFINITY : sum) * 0.6931471805599453f;
    __nv_bfloat16* out = p.O + token * p.o_st + head * p.o_sh;
    const float4* from = reinterpret_cast<const float4*>(p.part_o) + static_cast<int64_t>(slot0) * (D / 4) * 2 * BM + in;
#pragma unroll 2
    for (int c = 0; c < D / 8; ++c) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
#pragma unroll 4
        for (int i = 0; i < parts; ++i) {
            const float w = ex2_approx(__ldcg(lse + i * 2 * BM) - ref) * inv;
            const float4 x = __ldcg(from + (static_cast<int64_t>(i) * (D / 4) + 2 * c) * 2 * BM), y = __ldcg(from + (static_cast<int64_t>(i) * (D / 4) + 2 * c + 1) * 2 * BM);
            a.x += w * x.x; a.y += w * x.y; a.z += w * x.z; a.w += w * x.w;
            b.x += w * y.x; b.y += w * y.y; b.z += w * y.z; b.w += w * y.w;
        }
        if (there) *reinterpret_cast<uint4*>(out + 8 * c) = make_uint4(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y), pack_bf16x2(b.z, b.w));
    }
}

// What a CTA works on: sequence, its first query, length, tokens before the new ones; head; rows of the sequence and the slab's first;
// keys that the slab sees, and those that all of its rows see; the part's steps; whether the second tile has rows.
struct Work {
    int s, q0, len, before, h, rows, row0, n, n_all, j0, nsteps, two;
};
constexpr int GROUPS = 32;                               // groups of sixteen tokens that are looked up at a time: eight steps

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
cache_prefill_kernel(const __grid_constant__ PrefillArgs p) {
    using LY = Layout<D>;
    constexpr int Q_BYTES = LY::Q_BYTES, KV_BYTES = LY::KV_BYTES, RAW_BYTES = LY::RAW_BYTES, LS = LY::LS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + LY::BARS_AT);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + LY::NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    __shared__ int top_exp[2], any_bad;
    __shared__ volatile int cleaned;                     // values that are NaN and not for every row have been taken out
    // an item in parts: the part's place in the workspace (-1: the item is in one part), its index among them, their number, the item's place
    __shared__ int part_slot, part_index, part_count, part_item;
    __shared__ Work work;                                // (what the roles need of the mapping below: read again, not kept in registers)
    __shared__ int scales[2 * GROUPS];                   // of sixteen tokens: the exponents of the keys and values, a byte each; -1: no page there
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const CacheView& cv = p.c;
    if (threadIdx.x == 32) {
        for (int i = 0; i < LY::NUM_BARS; ++i)
            mbar_init(&bars[i], i == LY::EXPS_READY ? 8
                                : i < LY::K_EMPTY || (i >= LY::V_FULL && i < LY::V_EMPTY) || (i >= LY::P_FULL && i < LY::PV_DONE) || i >= LY::SCALE_EMPTY ? 4
                                : (i >= LY::K_EMPTY && i < LY::V_FULL) || (i >= LY::V_EMPTY && i < LY::S_FULL) ? 2 : 1);
        *abort_flag = 0;
        top_exp[0] = top_exp[1] = any_bad = cleaned = 0;
        fence_mbar_init();
    }
    if (warp == 2) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    // (the previous kernels of the stream have finished before the next one may start: a decode launch behind this one relies on it)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---------------------------------------------------------------- the CTA's work, by one warp (by every warp for itself: 200 queries, 32 heads, 17.7 us against 17.3,
    // 1,024 over 8,192 keys 143 against 139)
    // Items: sequence after sequence, their last slabs (under the causal mask the longest) first, the heads side by side.  Those of the last
    // round, fewer than there are SMs, are split along the keys into as many parts as find an SM.
    auto slabs_of = [&](int s, Span& sp) {
        if (!read_span(cv, s, p.total, p.max_new, sp)) return 0;
        const int rows = sp.n * p.G;
        return rows <= p.least_rows ? 0 : (rows + 2 * BM - 1) / (2 * BM);
    };
    auto deal = [&] {
    if (lane == 0) work.nsteps = 0;                      // (nothing to do)
    const int per = (cv.num_seqs + 31) / 32, s_end = min(lane * per + per, cv.num_seqs);
    auto before = [&](int v) {                           // of the lanes below and this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        return v;
    };
    Span sp{0, 0, 0};
    int mine_all = 0, slabs = 0;                         // of this lane's sequences: items, and then units
    unsigned steps_all = 0;                              // (used where there are fewer items than SMs: it fits then)
    for (int s = lane * per; s < s_end; ++s) {
        slabs = slabs_of(s, sp);
        mine_all = min(mine_all + slabs * cv.Hkv, 0x3ffffff);          // (with offsets that go back and forth it could pass 31 bits)
        steps_all += static_cast<unsigned>(slabs * cv.Hkv) * ((sp.len + BN - 1) / BN);
    }
    // (up to 32 sequences: a lane keeps its one, and what the warp needs of any of them comes by shuffle)
    const Span own = sp;
    const int own_slabs = slabs;
    auto fetch = [&](int s) {
        if (per > 1) return slabs_of(s, sp);
        sp = Span{__shfl_sync(0xffffffffu, own.q0, s), __shfl_sync(0xffffffffu, own.n, s), __shfl_sync(0xffffffffu, own.len, s)};
        return __shfl_sync(0xffffffffu, own_slabs, s);
    };
    const int items = __reduce_add_sync(0xffffffffu, mine_all);
    if (items > p.most_items) {                          // (offsets that go back and forth: more rows than the tensors have)
        if (cv.status && lane == 0) atomicExch(cv.status, FLAT_CACHE_BAD_LENGTH);
        return;
    }
    // All items in one round: parts of `each` steps, as many as there are SMs.  Several rounds: the last one's items in `split` parts each.
    // Joining costs about a step a part, so n steps take n / P + P in P parts: no more than sqrt(n) of them, of four steps at least.
    int each = 0;
    if (items < p.sms) {
        steps_all = __reduce_add_sync(0xffffffffu, steps_all);
        each = (steps_all + p.sms - items - 1) / static_cast<unsigned>(p.sms - items);
    }
    auto most_parts = [&](int steps, int wanted) { return max(1, min(min(wanted, 16), min(steps / 4, static_cast<int>(sqrtf(static_cast<float>(steps)))))); };
    auto parts_of = [&](int steps) { return each ? most_parts(steps, (steps + each - 1) / each) : 1; };       // (by the sequence's length)
    if (each) {
        if (per == 1) mine_all = slabs * cv.Hkv * parts_of((sp.len + BN - 1) / BN);          // (the lane's own)
        else {
            mine_all = 0;
            for (int s = lane * per; s < s_end; ++s) mine_all += slabs_of(s, sp) * cv.Hkv * parts_of((sp.len + BN - 1) / BN);
        }
    }
    const int upto = before(mine_all), units = __shfl_sync(0xffffffffu, upto, 31);
    const int rest = each ? 0 : units % p.sms, whole = units - rest, split = rest ? min(p.sms / rest, 16) : 1, unit = blockIdx.x;
    if (unit >= whole + rest * split) return;
    const int entry = unit < whole ? unit : whole + (unit - whole) / split;      // among the units before the split
    const int from = __ffs(__ballot_sync(0xffffffffu, upto > entry)) - 1;
    int s = from * per, first = __shfl_sync(0xffffffffu, upto - mine_all, from);
    slabs = fetch(s);
    int of = parts_of((sp.len + BN - 1) / BN);
    while (entry >= first + slabs * cv.Hkv * of) {
        first += slabs * cv.Hkv * of;
        ++s;
        slabs = fetch(s);
        of = parts_of((sp.len + BN - 1) / BN);
    }
    const int item = (entry - first) / of, h = item % cv.Hkv, row0 = (slabs - 1 - item / cv.Hkv) * 2 * BM, rows = sp.n * p.G;
    // keys that any row of the slab sees; the part's steps j0 .. j0 + nsteps - 1
    const int last_tok = (row0 + 2 * BM < rows ? row0 + 2 * BM - 1 : rows - 1) / p.G;
    const int n = p.causal ? last_tok + 1 + sp.len - sp.n : sp.len;
    const int all_steps = (n + BN - 1) / BN;
    // (an early slab may have fewer steps than its sequence has parts)
    const int parts = each ? min(of, all_steps) : unit < whole ? 1 : most_parts(all_steps, split);
    const int part = each ? (entry - first) % of : unit < whole ? 0 : (unit - whole) % split;
    if (part >= parts) return;
    if (lane == 0) {
        const int j0 = all_steps * part / parts;
        const int n_all = p.causal ? min(row0 / p.G + 1 + sp.len - sp.n, n) : n;
        work = Work{s, sp.q0, sp.len, sp.len - sp.n, h, rows, row0, n, n_all, j0, all_steps * (part + 1) / parts - j0, rows - row0 > BM};
        part_slot = parts == 1 ? -1 : each ? unit : unit - whole;
        part_index = part;
        part_count = parts;
        part_item = each ? unit - part : (unit - whole) / split;
    }
    };
    if (warp == 0) deal();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t bars_s = smem_u32(bars), abort_s = smem_u32(const_cast<int*>(abort_flag)), base_s = smem_u32(base);
    const int nsteps = work.nsteps;
    if (nsteps == 0) {                                   // (the whole CTA)
        if (warp == 2) tmem_dealloc(tmem, 512);
        return;
    }

    if (warp >= 12) {
        // ------------------------------------------------------------ keys and values: e4m3 pages -> half-precision tiles
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        const int tid = threadIdx.x - 384, u = tid >> 2, q = tid & 3, len = work.len, key0 = work.j0 * BN + u;
        constexpr int PIECES = BN * D / 16 / 128;        // of 16 bytes, a thread and tile: 4 (d = 128) or 2
        // Piece i: sixteen features from 16 q on, of panel (i / 2) ^ (u % 2) (of 64 features; d = 64: the only one), of the row u + 32 (i % 2):
        // eight lanes then read two rows in eight different banks, and write eight.
        auto panel = [&](int i) { return D == 128 ? (i >> 1) ^ (u & 1) : 0; };
        const uint32_t chunk0 = ((2 * q) ^ (u & 7)) << 4, chunk1 = ((2 * q + 1) ^ (u & 7)) << 4;
        bool ok = true;
        auto wait = [&](int bar, uint32_t parity, int code) {
            if (ok) ok = warp_wait(bars_s + 8 * bar, parity, abort_s, cv.status, code);
        };
        auto convert = [&](uint32_t (&v)[PIECES][4], uint32_t to, int e0, int e1, int top) {
            // (tokens that no row of the slab sees may lie in pages that the largest was not taken over: they must stay finite)
            const __half2 by[2] = {__float2half2_rn(two_to(min(e0 - top, 0) + LIFT)), __float2half2_rn(two_to(min(e1 - top, 0) + LIFT))};
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                uint32_t x[8];
                widen16(v[i], by[i & 1], x);
                const uint32_t at = to + panel(i) * (BN * 128) + (u + 32 * (i & 1)) * 128;
                sts16(at + chunk0, x[0], x[1], x[2], x[3]);
                sts16(at + chunk1, x[4], x[5], x[6], x[7]);
            }
            fence_proxy_async_smem();
            __syncwarp();
        };
        wait(LY::EXPS_READY, 0, 0xb13);
        const int EK = top_exp[0], EV = top_exp[1];
        for (int j = 0; j < nsteps && ok; ++j) {
            if (j % 8 == 0) wait(LY::SCALE_FULL + ((j >> 3) & 1), (j >> 4) & 1, 0xb14);
            wait(LY::RAW_FULL + j % LS, (j / LS) & 1, 0xb12);
            if (!ok) break;
            const uint32_t from = base_s + LY::RAW_AT + (j % LS) * 2 * RAW_BYTES + u * D + q * 16;
            uint32_t k[PIECES][4], v[PIECES][4];
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                lds16(from + 32 * (i & 1) * D + panel(i) * 64, k[i]);
                lds16(from + RAW_BYTES + 32 * (i & 1) * D + panel(i) * 64, v[i]);
            }
            const int g0 = (j * 4 + (u >> 4)) & (2 * GROUPS - 1), e0 = scales[g0], e1 = scales[g0 + 2];
            // (rows without a token hold anything: zeros)
            const bool none0 = e0 < 0 || key0 + j * BN >= len, none1 = e1 < 0 || key0 + j * BN + 32 >= len;
            if (__any_sync(0xffffffffu, none0 || none1)) {
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
                    if (i & 1 ? none1 : none0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) k[i][e] = v[i][e] = 0u;
                    }
            }
            wait(LY::K_EMPTY + j % KS, ((j / KS) & 1) ^ 1, 0xb10);
            if (!ok) break;
            convert(k, base_s + LY::K_AT + (j % KS) * KV_BYTES, e0 & 255, e1 & 255, EK);
            if (lane == 0) {
                mbar_arrive(&bars[LY::K_FULL + j % KS]);
                mbar_arrive(&bars[LY::RAW_EMPTY + j % LS]);      // (all of it is in registers)
            }
            // (a weight of 0 would not keep a NaN from the rows that do not see its key: the rows that do get it at the end)
            const int n_all = work.n_all;
            if ((work.j0 + j + 1) * BN > n_all) {
                uint32_t any = 0;
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t gone = key0 + j * BN + 32 * (i & 1) >= n_all ? nan_bytes(v[i][e]) : 0u;
                        any |= gone;
                        v[i][e] &= ~gone;
                    }
                if (any) cleaned = 1;
            }
            wait(LY::V_EMPTY + j % VS, ((j / VS) & 1) ^ 1, 0xb11);
            if (!ok) break;
            convert(v, base_s + LY::V_AT + (j % VS) * KV_BYTES, e0 >> 8 & 255, e1 >> 8 & 255, EV);
            if (lane == 0) {
                mbar_arrive(&bars[LY::V_FULL + j % VS]);
                if (j % 8 == 7) mbar_arrive(&bars[LY::SCALE_EMPTY + ((j >> 3) & 1)]);
            }
        }
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 10) {
            // -------------------------------------------------------- page table, exponents and copies, eight steps at a time (a lane sixteen tokens)
            const int32_t* table = cv.table + static_cast<int64_t>(work.s) * cv.max_pages;
            const int end = min(work.len, (work.j0 + nsteps) * BN);
            constexpr uint32_t BYTES = 16 * D;           // of sixteen tokens: they lie in one page, one after the other
            bool ok = true;
            int issued = 0;
            auto wait = [&](int bar, uint32_t parity, int code) {
                if (ok) ok = warp_wait(bars_s + 8 * bar, parity, abort_s, cv.status, code);
            };
            auto look = [&](int b) {                     // the lane's sixteen tokens of batch b: page * heads + head; -1: no page there
                const int key = work.j0 * BN + (b * GROUPS + lane) * 16;
                if (b * 8 >= nsteps || key >= end) return -1;
                const int id = table[key >> cv.page_shift];
                return id >= 0 && id < cv.num_pages ? id * cv.Hkv + work.h : -1;
            };
            int next = look(0);
            for (int b = 0; b * 8 < nsteps && ok; ++b) {
                const int place = next, key = work.j0 * BN + (b * GROUPS + lane) * 16;
                const int64_t src = ((static_cast<int64_t>(place < 0 ? 0 : place) << cv.page_shift) + (key & (cv.page - 1))) * D;
                int scale = -1;
                if (place >= 0) scale = cv.k_exp[place] | cv.v_exp[place] << 8;
                next = look(b + 1);
                for (int i = 0; i < 8 && b * 8 + i < nsteps && ok; ++i) {
                    const int j = b * 8 + i, st = j % LS;
                    wait(LY::RAW_EMPTY + st, ((j / LS) & 1) ^ 1, 0xb16);
                    if (!ok) break;
                    const unsigned have = __ballot_sync(0xffffffffu, place >= 0) >> (4 * i) & 15;
                    if (lane == 0) mbar_arrive_expect_tx(&bars[LY::RAW_FULL + st], 2 * BYTES * __popc(have));
                    __syncwarp();
                    if (place >= 0 && lane >> 2 == i) {
                        const uint32_t dst = base_s + LY::RAW_AT + st * 2 * RAW_BYTES + (lane & 3) * BYTES;
                        bulk_load(dst, cv.k + src, BYTES, bars_s + 8 * (LY::RAW_FULL + st));
                        bulk_load(dst + RAW_BYTES, cv.v + src, BYTES, bars_s + 8 * (LY::RAW_FULL + st));
                    }
                    __syncwarp();
                    issued = j + 1;
                    if (i == 0) {                        // (behind the first copies: the exponents have arrived by now)
                        wait(LY::SCALE_EMPTY + (b & 1), ((b >> 1) & 1) ^ 1, 0xb15);
                        if (!ok) break;
                        scales[(b & 1) * GROUPS + lane] = scale;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bars[LY::SCALE_FULL + (b & 1)]);
                    }
                }
            }
            // (copies in flight end before the CTA does, whoever gave up waiting for them)
            for (int j = issued > LS ? issued - LS : 0; j < issued; ++j) drain_wait(&bars[LY::RAW_FULL + j % LS], (j / LS) & 1);
        } else if (warp <= 9) {
            // -------------------------------------------------------- MMA issuer of tile t (whole warp walks, one lane issues)
            const int t = warp - 8;
            constexpr uint32_t IDESC_S = idesc_half(BM, BN, 0), IDESC_PV = idesc_half(BM, D, 1);
            const uint64_t q_desc = make_smem_desc_sw128(base_s + t * Q_BYTES, 16, 1024);
            const uint64_t k_desc = make_smem_desc_sw128(base_s + LY::K_AT, 16, 1024);
            const uint64_t v_desc = make_smem_desc_sw128(base_s + LY::V_AT, BN * 128, 1024);
            bool ok = true;
            auto wait = [&](int bar, uint32_t parity, int code) {
                if (ok) ok = warp_wait(bars_s + 8 * bar, parity, abort_s, cv.status, code);
            };
            if (t == 1 && !work.two)                          // (no rows in this tile: only let the stages go)
                for (int j = 0; j < nsteps && ok; ++j) {
                    wait(LY::K_FULL + j % KS, (j / KS) & 1, 0xb25);
                    if (ok && lane == 0) mbar_arrive(&bars[LY::K_EMPTY + j % KS]);
                    wait(LY::V_FULL + j % VS, (j / VS) & 1, 0xb26);
                    if (ok && lane == 0) mbar_arrive(&bars[LY::V_EMPTY + j % VS]);
                    __syncwarp();
                }
            else {
            auto issue_s = [&](int j) {                  // S_t(j) = Q_t K_j^T, then release the K stage
                const uint64_t kd = k_desc + static_cast<uint64_t>(((j % KS) * KV_BYTES) >> 4);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_ss(tmem + S_COL(t, j & 1), q_desc + static_cast<uint64_t>(((k / 4) * (BM * 128) + (k % 4) * 32) >> 4),
                           kd + static_cast<uint64_t>(((k / 4) * (BN * 128) + (k % 4) * 32) >> 4), IDESC_S, k > 0);
                tc_commit(&bars[LY::S_FULL + 2 * t + (j & 1)]);
                tc_commit(&bars[LY::K_EMPTY + j % KS]);
            };
            auto issue_pv = [&](int j) {                 // O_t += P_t(j) V_j, then release the V stage
                const uint64_t vd = v_desc + static_cast<uint64_t>(((j % VS) * KV_BYTES) >> 4);
#pragma unroll
                for (int k = 0; k < BN / 16; ++k)
                    mma_ts(tmem + O_COL(t), tmem + S_COL(t, j & 1) + k * 8, vd + static_cast<uint64_t>((k * 2048) >> 4), IDESC_PV, (j > 0 || k > 0));
                tc_commit(&bars[LY::PV_DONE + 2 * t + (j & 1)]);
                tc_commit(&bars[LY::V_EMPTY + j % VS]);
            };
            wait(LY::Q_FULL + t, 0, 0xb20);
            for (int j = 0; j < 2 && j < nsteps; ++j) {
                wait(LY::K_FULL + j % KS, (j / KS) & 1, 0xb21);
                tc_fence_after();
                if (ok && elect_one()) issue_s(j);
                __syncwarp();
            }
            for (int j = 0; j < nsteps && ok; ++j) {
                const bool more = j + 2 < nsteps;
                wait(LY::V_FULL + j % VS, (j / VS) & 1, 0xb22);
                if (more) wait(LY::K_FULL + (j + 2) % KS, ((j + 2) / KS) & 1, 0xb23);
                wait(LY::P_FULL + 2 * t + (j & 1), (j >> 1) & 1, 0xb24);
                if (!ok) break;
                tc_fence_after();
                // (S(j + 2) overwrites P(j): it goes behind the MMAs that read it)
                if (elect_one()) { issue_pv(j); if (more) issue_s(j + 2); }
                __syncwarp();
            }
            }
        }
    } else {
        // ------------------------------------------------------------ softmax + epilogue (warps 0-7)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int n = work.n, j0 = work.j0, rows = work.rows;
        const int32_t* table = cv.table + static_cast<int64_t>(work.s) * cv.max_pages;
        const int last_page = (min(n, (j0 + nsteps) * BN) - 1) >> cv.page_shift;      // of the part
        const bool active = warp < 4 || work.two;
        const int t = warp >> 2, mine = (warp & 3) * 32 + lane, row = work.row0 + t * BM + mine;
        const uint32_t tl = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t my_bars = bars_s + 8 * (LY::S_FULL + 2 * t);       // S_FULL of the tile; P_FULL and PV_DONE 32 and 64 bytes on
        const int tok = (row < rows ? row : rows - 1) / p.G, head = work.h * p.G + (row < rows ? row - tok * p.G : 0), token = work.q0 + tok;
        float unit = 0.f;
        // The warp's rows, RPI at a time, LPR lanes a row (queries in, outputs out; a lane a row asks for every sector twice: 200 queries, 32
        // heads, 17.3 us against 13.8): f(i, row, the piece's place).
        constexpr int LPR = D / 8, RPI = 32 / LPR;
        const int piece = lane % LPR;
        auto walk = [&](long long stride_t, long long stride_h, auto unrolled, auto f) {
            int r = work.row0 + t * BM + (warp & 3) * 32 + lane / LPR, tk = r / p.G, g = r - tk * p.G;
            const int tokens = RPI / p.G, heads = RPI - tokens * p.G;     // from one row to the next of the walk
            const long long step = tokens * stride_t + heads * stride_h, over = stride_t - p.G * stride_h;
            long long at = (static_cast<long long>(work.q0) + tk) * stride_t + (static_cast<long long>(work.h) * p.G + g) * stride_h + piece * 8;
#pragma unroll (decltype(unrolled)::value)
            for (int i = 0; i < D / 8; ++i) {
                f(i, r, at);
                r += RPI;
                g += heads;
                at += step;
                if (g >= p.G) { g -= p.G; at += over; }
            }
        };
        // Of the walk's i-th row, the lane's piece: its place in the tile (128-byte swizzle).
        auto spot = [&](int i) {
            const int in = (warp & 3) * 32 + i * RPI + lane / LPR;
            return base_s + t * Q_BYTES + (piece >> 3) * (BM * 128) + in * 128 + (((piece & 7) ^ (in & 7)) << 4);
        };
        {
            // (eight features a lane, LPR lanes a row: sectors of 32 bytes are asked for once)
            uint4 v[D / 8];
            walk(p.q_st, p.q_sh, Const<D / 8>{}, [&](int i, int r, long long at) {
                v[i] = make_uint4(0, 0, 0, 0);
                if (r < rows) v[i] = *reinterpret_cast<const uint4*>(p.Q + at);
            });
            // the part's largest exponents of the keys and values, and whether a page is missing
            int ke = 0, ve = 0, bad = 0;
            for (int i = (j0 * BN >> cv.page_shift) + threadIdx.x; i <= last_page; i += 4 * 256) {
                int place[4];                            // (four on their way: a place waits for its page)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    int id;
                    place[u] = -1;
                    if (i + 256 * u > last_page) continue;
                    if (read_page(cv, work.s, i + 256 * u, id)) place[u] = id * cv.Hkv + work.h;
                    else bad = 1;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    ke = max(ke, place[u] >= 0 ? static_cast<int>(cv.k_exp[place[u]]) : 0);
                    ve = max(ve, place[u] >= 0 ? static_cast<int>(cv.v_exp[place[u]]) : 0);
                }
            }
            ke = __reduce_max_sync(0xffffffffu, ke);
            ve = __reduce_max_sync(0xffffffffu, ve);
            bad = __any_sync(0xffffffffu, bad);
            if (lane == 0) {
                atomicMax(&top_exp[0], ke);
                atomicMax(&top_exp[1], ve);
                if (bad) any_bad = 1;
                mbar_arrive(&bars[LY::EXPS_READY]);
            }
            // the query rows into half precision, a power of two taken out of each
            int my_e = 0;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                uint32_t m = w[0] & 0x7fff7fffu;         // magnitudes of two features: their bits are in their order
#pragma unroll
                for (int k = 1; k < 4; ++k) m = __vmaxu2(m, w[k] & 0x7fff7fffu);
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
                int e = static_cast<int>(max(m & 0xffffu, m >> 16) >> 7) - 127;     // the row's largest: 2^e to 2^(e + 1)
                e = e < -100 ? -100 : e;
                const int theirs = __shfl_sync(0xffffffffu, e, (lane % RPI) * LPR);
                if (lane / RPI == i) my_e = theirs;
                const float up = two_to(14 - e);
                uint32_t x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = pack_half2(__uint_as_float(w[k] << 16) * up, __uint_as_float(w[k] & 0xffff0000u) * up);
                sts16(spot(i), x[0], x[1], x[2], x[3]);
            }
            unit = p.scale_log2e * two_to(my_e - 14);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars[LY::Q_FULL + t]);
        }
        bool ok = warp_wait(bars_s + 8 * LY::EXPS_READY, 0, abort_s, cv.status, 0xb35);
        unit *= two_to(top_exp[0] - 127 - LIFT);
        if (active) {
        const bool missing = any_bad != 0;
        float m_ref = -INFINITY, l = 0.f;
        const int nrow = p.causal ? min(tok + 1 + work.before, n) : n;
        const int nrow_min = __shfl_sync(0xffffffffu, nrow, 0);
        for (int j = 0; j < nsteps && ok; ++j) {
            const uint32_t s_addr = tl + S_COL(t, j & 1);
            ok = warp_wait(my_bars + 8 * (j & 1), (j >> 1) & 1, abort_s, cv.status, 0xb30 + t);
            if (!ok) break;
            tc_fence_after();
            uint32_t x[BN];
            tmem_ld_x32(s_addr, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
            tmem_ld_x32(s_addr + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
            tc_wait_ld();
            const int col0 = (j0 + j) * BN;
            int out = 0;                                 // (rare) groups of sixteen keys whose page is missing
            if (missing)
                for (int i = 0; i < BN / 16; ++i) {
                    const int index = (col0 + 16 * i) >> cv.page_shift;
                    int id = 0;
                    if (index <= last_page) id = table[index];
                    if (id < 0 || id >= cv.num_pages) out |= 1 << i;
                }
            const bool tail = col0 + BN > nrow_min || out != 0;          // (warp-uniform) some row has masked keys in this step
            const int nvalid = nrow > col0 ? (nrow - col0 < BN ? nrow - col0 : BN) : 0;
            bool careful = j == 0 || tail;
            float lt = 0.f;
            if (!careful) {
                lt = exp_store(x, unit, SHIFT - m_ref, s_addr);
                careful = __any_sync(0xffffffffu, !(lt <= MOST_SUM));
                if (careful) {           // (the weights went over the first half of the logits: they go back)
                    tmem_st_x32(s_addr, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
                    tmem_ld_x32(s_addr + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
                    tc_wait_ld();
                    tc_wait_st();
                }
            }
            if (careful) {
                const float mx = row_max(x, unit, nvalid, out);
                if (__any_sync(0xffffffffu, mx > m_ref)) {
                    const float m_new = fmaxf(m_ref, mx);
                    const float alpha = m_new == -INFINITY ? 1.f : ex2_approx(m_ref - m_new);   // 0 on the row's first keys
                    l *= alpha;
                    if (j > 0) {
                        ok = warp_wait(my_bars + 64 + 8 * ((j - 1) & 1), ((j - 1) >> 1) & 1, abort_s, cv.status, 0xb32 + t);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t r[16];
                            tmem_ld_x16(tl + O_COL(t) + c * 16, r);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
                            tmem_st_x16(tl + O_COL(t) + c * 16, r);
                        }
                    }
                    m_ref = m_new;
                }
                lt = exp_store_tail(unit, m_ref == -INFINITY ? 0.f : SHIFT - m_ref, s_addr, nvalid, out);
            }
            l += lt;
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_s(my_bars + 32 + 8 * (j & 1));
        }
        if (ok) ok = warp_wait(my_bars + 64 + 8 * ((nsteps - 1) & 1), ((nsteps - 1) >> 1) & 1, abort_s, cv.status, 0xb34 + t);
        if (ok) {
            // (the scale by itself: over the sum it could lie below the least normal number)
            const float inv = l > 0.f ? 1.f / l : l == l ? 0.f : l, scale = two_to(top_exp[1] - 127 - LIFT);
            const float lse2 = l > 0.f ? m_ref - SHIFT + log2f(l) : l == l ? -INFINITY : l;
            const int slot = part_slot;
            if (slot >= 0) p.part_lse[(slot * 2 + t) * BM + mine] = lse2;
            else if (p.lse && row < rows) p.lse[static_cast<int64_t>(token) * p.Hq + head] = lse2 * 0.6931471805599453f;
            tc_fence_after();
            float4* prow = reinterpret_cast<float4*>(p.part_o) + (static_cast<int64_t>(slot) * (D / 4) * 2 + t) * BM + mine;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t r[32];
                tmem_ld_x32(tl + O_COL(t) + c * 32, r);
                tc_wait_ld();
                float f[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(r[i]) * inv * scale;
                if (slot >= 0) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) prow[(c * 8 + v) * 2 * BM] = make_float4(f[4 * v], f[4 * v + 1], f[4 * v + 2], f[4 * v + 3]);
                } else {                                 // into the queries' memory (their products are done), from where whole rows go out
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int at = c * 4 + v;        // (the piece of the row)
                        sts16(base_s + t * Q_BYTES + (at >> 3) * (BM * 128) + mine * 128 + (((at & 7) ^ (mine & 7)) << 4), pack_bf16x2(f[8 * v], f[8 * v + 1]),
                              pack_bf16x2(f[8 * v + 2], f[8 * v + 3]), pack_bf16x2(f[8 * v + 4], f[8 * v + 5]), pack_bf16x2(f[8 * v + 6], f[8 * v + 7]));
                    }
                }
            }
            if (cleaned) {                               // the values that were taken out, into the row's own place of what was just written
                const volatile Work& w = work;           // (read again: nothing of this is kept in registers through the steps)
                const int r = w.row0 + t * BM + mine, key1 = r < w.rows ? min(p.causal ? r / p.G + 1 + w.before : w.n, (w.j0 + w.nsteps) * BN) : 0;
#pragma unroll 1
                for (int key = max(w.n_all, w.j0 * BN); key < key1; ++key) {
                    const int id = cv.table[static_cast<int64_t>(w.s) * cv.max_pages + (key >> cv.page_shift)];
                    if (id < 0 || id >= cv.num_pages) continue;
                    const uint8_t* v = cv.v + (((static_cast<int64_t>(id) * cv.Hkv + w.h) << cv.page_shift) + (key & (cv.page - 1))) * D;
#pragma unroll 1
                    for (int f = 0; f < D; ++f) {
                        if ((v[f] & 0x7f) != 0x7f) continue;
                        if (slot >= 0) reinterpret_cast<float*>(prow + (f >> 2) * 2 * BM)[f & 3] = __int_as_float(0x7fffffff);
                        else asm volatile("st.shared.u16 [%0], %1;" ::"r"(base_s + t * Q_BYTES + (f >> 6) * (BM * 128) + mine * 128 + (((f >> 3 & 7) ^ (mine & 7)) << 4) + (f & 7) * 2),
                                          "h"(static_cast<uint16_t>(0x7fff)) : "memory");
                    }
                }
            }
            if (slot < 0) {
                __syncwarp();
                walk(p.o_st, p.o_sh, Const<4>{}, [&](int i, int r, long long at) {
                    uint32_t x[4];
                    lds16(spot(i), x);
                    if (r < rows) *reinterpret_cast<uint4*>(p.O + at) = make_uint4(x[0], x[1], x[2], x[3]);
                });
            }
        }
        if (part_slot >= 0) {
            // -------------------------------------------------------- an item in parts: the warp that comes last with its 32 rows joins them
            // (in the order of the keys; a part whose waits gave up counts too, so that the counter ends at 0: what it left is not valid, as
            // `status` says.  Here, in the branch of these warps: the others have given up the registers.)
            __threadfence();
            __syncwarp();
            int* counter = p.counters + part_item * 8 + warp;
            int last = 0;
            if (lane == 0) last = atomicAdd(counter, 1) == part_count - 1;
            if (__shfl_sync(0xffffffffu, last, 0)) {
                __threadfence();
                if (lane == 0) *counter = 0;
                join_rows<D>(p, part_slot - part_index, part_count, t * BM + mine, row < rows, token, head);
            }
        }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) tmem_dealloc(tmem, 512);
}

template <int D>
int launch_d(const flat_attn_cache_t& c, const PrefillArgs& p, cudaStream_t st) {
    PrefillArgs args = p;
    if (!ensure_dynamic_smem<cache_prefill_kernel<D>>(Layout<D>::SMEM_BYTES)) return FLAT_ERR_CUDA;
    // No more items than this: a sequence has a slab for every 256 rows and one for the rest, and only those with more than least_rows
    // rows count.  (CTAs without work leave at once, but one after the other.)
    const int64_t rows = p.total * p.G, slabs = (static_cast<int64_t>(p.max_new) * p.G + 2 * BM - 1) / (2 * BM);
    const int64_t last = rows / (p.least_rows + 1) < c.num_seqs ? rows / (p.least_rows + 1) : c.num_seqs;
    const int64_t bound = rows / (2 * BM) + last, most = slabs * c.num_seqs < bound ? slabs * c.num_seqs : bound;
    args.most_items = static_cast<int>(most * c.Hkv < 0x7fffffff ? most * c.Hkv : 0x7fffffff);
    const int64_t items = most * c.Hkv + p.sms;          // (parts beyond whole items: fewer than there are SMs)
    if (items > 0x7fffffff) return FLAT_ERR_SHAPE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(items));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = Layout<D>::SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cache_prefill_kernel<D>, args) == cudaSuccess ? FLAT_OK : FLAT_ERR_CUDA;
}

}  // namespace

size_t cache_prefill_counter_bytes() { return (device_sm_count() * 8 * sizeof(int) + 255) & ~size_t(255); }
size_t cache_prefill_part_bytes(int d) { return static_cast<size_t>(device_sm_count()) * 2 * BM * (d + 1) * sizeof(float); }

int launch_cache_prefill(const flat_attn_cache_t& c, const flat_attn_cache_fwd_params_t& q, int least_rows, int* counters, float* parts, cudaStream_t st) {
    PrefillArgs p{};
    p.c = cache_view(c);
    p.Q = static_cast<const __nv_bfloat16*>(q.Q);
    p.O = static_cast<__nv_bfloat16*>(q.O);
    p.lse = q.lse;
    p.q_st = q.q_stride_t; p.q_sh = q.q_stride_h; p.o_st = q.o_stride_t; p.o_sh = q.o_stride_h;
    p.total = q.total;
    p.Hq = q.Hq; p.G = q.Hq / c.Hkv; p.max_new = q.max_new; p.least_rows = least_rows; p.causal = q.causal;
    p.sms = device_sm_count();
    p.counters = counters;
    p.part_lse = parts;
    p.part_o = p.part_lse + static_cast<size_t>(p.sms) * 2 * BM;
    p.scale_log2e = q.scale * 1.4426950408889634f;
    return c.d == 64 ? launch_d<64>(c, p, st) : launch_d<128>(c, p, st);
}

}  // namespace flat
