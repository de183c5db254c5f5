// Attention over the 8-bit paged cache for many query rows per key head: prompts and chunks of them (d = 64 and 128).
//
// The rows of a sequence and key head are its queries times the G query heads of the group; an item is a slab of 256 of them, two tiles
// of 128, against the keys that they see, in steps of 64.  Logits and outputs are tcgen05 products in half precision with fp32
// accumulators in TMEM.  e4m3 numbers are exact in half precision; four warps bring the pages (cp.async into memory of their own,
// no barrier), turn them into half-precision tiles in the 128-byte swizzle and take the page's scale into them, relative to the largest
// of the sequence and head: k 2^(ek - EK + 6), exact until 2^-30 of the largest value becomes subnormal.  So the softmax sees one
// scale.  Queries are scaled by a power of two a row into half precision (it goes into the row's softmax constant); weights are 2^9 w,
// rounded to half precision.
//
// CTA = 512 threads: warps 0-3 / 4-7 softmax of tile A / B (thread = row = TMEM lane), warps 8 / 9 MMA issuers of tile A / B (one
// elected lane), warps 10, 11 idle (they complete a warpgroup for the register hand-over), warps 12-15 bring and convert keys and values.
// TMEM columns: S(t, b) 128 t + 64 b (b = step parity), P over the first 32 of them, O_t 256 + 128 t.
// The softmax takes no row maximum after the first step: any reference gives the exact softmax; a step whose row sum passes 60,000
// (a weight could pass the largest half-precision number) is redone with a fresh maximum.  One exponential in four goes through a
// polynomial on the FMA pipe.  Every wait is bounded (tc_common.cuh); on expiry the CTA aborts cleanly and reports a code.
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
constexpr int KS = 3, VS = 3, LS = 3;                    // stages: half-precision keys, values; pages as they come
constexpr int POLY_LANE = 3;                             // element index mod 8 that takes the polynomial
// Weights at the reference maximum are 2^9: 64 of them add up to half of MOST_SUM, so that a step passes it only where the reference is
// exceeded, and what half precision rounds away lies 2^34 below the reference.
constexpr float SHIFT = 9.f, MOST_SUM = 60000.f;
constexpr int LIFT = 6;                                  // log2: the largest e4m3 number times 2^6 is 28,672

__host__ __device__ constexpr uint32_t S_COL(int t, int b) { return 128u * t + 64u * b; }
__host__ __device__ constexpr uint32_t O_COL(int t) { return 256u + 128u * t; }

template <int D> struct Layout {
    static constexpr int Q_BYTES = BM * D * 2, KV_BYTES = BN * D * 2, RAW_BYTES = BN * D;
    static constexpr int K_AT = 2 * Q_BYTES, V_AT = K_AT + KS * KV_BYTES, RAW_AT = V_AT + VS * KV_BYTES, BARS_AT = RAW_AT + LS * 2 * RAW_BYTES;
    static constexpr int Q_FULL = 0, K_FULL = 2, K_EMPTY = K_FULL + KS, V_FULL = K_EMPTY + KS, V_EMPTY = V_FULL + VS, S_FULL = V_EMPTY + VS,
                         P_FULL = S_FULL + 4, PV_DONE = P_FULL + 4, NUM_BARS = PV_DONE + 4;
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

// p_i = 2^(s_i * unit + neg_m) of 64 logits, rounded to half precision into 32 TMEM columns at `p_addr`; returns the fp32 sum of the
// unrounded p.  TAIL: only the first `nvalid` take part, and of those not the groups of sixteen in `out`.
template <bool TAIL>
__device__ __forceinline__ float exp_store(const uint32_t (&s)[BN], float unit, float neg_m, uint32_t p_addr, int nvalid, int out) {
    uint64_t sum0 = 0ull, sum1 = 0ull;
    const uint64_t unit2 = pack2(unit, unit), neg_m2 = pack2(neg_m, neg_m);
#pragma unroll
    for (int c = 0; c < BN / 32; ++c) {
        uint32_t pk[16];
        float p[32];
#pragma unroll
        for (int i = 0; i < 32; i += 2)
            unpack2(fma2(pack2(__uint_as_float(s[c * 32 + i]), __uint_as_float(s[c * 32 + i + 1])), unit2, neg_m2), p[i], p[i + 1]);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            p[i] = !TAIL && (i & 7) == POLY_LANE ? ex2_poly(p[i]) : ex2_approx(p[i]);
            if (TAIL && (c * 32 + i >= nvalid || (out >> (2 * c + i / 16) & 1))) p[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            sum0 = add2(sum0, pack2(p[i], p[i + 1]));
            sum1 = add2(sum1, pack2(p[i + 2], p[i + 3]));
            pk[i / 2] = pack_half2(p[i], p[i + 1]);
            pk[i / 2 + 1] = pack_half2(p[i + 2], p[i + 3]);
        }
        tmem_st_x16(p_addr + c * 16, pk);
    }
    float a, b, cc, d;
    unpack2(sum0, a, b);
    unpack2(sum1, cc, d);
    return (a + b) + (cc + d);
}
// The largest unit * s of the keys that take part.
__device__ __forceinline__ float row_max(const uint32_t (&s)[BN], float unit, int nvalid, int out) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < BN; ++i)
        if (i < nvalid && !(out >> (i / 16) & 1)) m = fmaxf(m, __uint_as_float(s[i]) * unit);
    return m;
}

// Sixteen e4m3 (a piece) times a half-precision pair `by`, as two 16-byte chunks.
__device__ __forceinline__ void widen16(const uint4& v, __half2 by, uint32_t (&h)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
        const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&r), by);
        h[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

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

template <int D>
__global__ void __launch_bounds__(THREADS, 1)
cache_prefill_kernel(const __grid_constant__ PrefillArgs p) {
    using LY = Layout<D>;
    constexpr int Q_BYTES = LY::Q_BYTES, KV_BYTES = LY::KV_BYTES, RAW_BYTES = LY::RAW_BYTES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(base + LY::BARS_AT);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + LY::NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    __shared__ int top_exp[2], any_bad;
    // an item in parts: the part's place in the workspace (-1: the item is in one part), its index among them, their number, the item's place
    __shared__ int part_slot, part_index, part_count, part_item;
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const CacheView& cv = p.c;
    // (the previous kernels of the stream have finished before the next one may start: a decode launch behind this one relies on it)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---------------------------------------------------------------- the CTA's work (every warp for itself)
    // Items: sequence after sequence, their last slabs (under the causal mask the longest) first, the heads side by side.  Those of the last
    // round, fewer than there are SMs, are split along the keys into as many parts as find an SM.
    auto slabs_of = [&](int s, Span& sp) {
        if (!read_span(cv, s, p.total, p.max_new, sp)) return 0;
        const int rows = sp.n * p.G;
        return rows <= p.least_rows ? 0 : (rows + 2 * BM - 1) / (2 * BM);
    };
    const int per = (cv.num_seqs + 31) / 32, s_end = min(lane * per + per, cv.num_seqs);
    Span sp;
    int upto = 0;                                        // items of this lane's sequences and those before
    for (int s = lane * per; s < s_end; ++s) upto += slabs_of(s, sp) * cv.Hkv;
    const int mine_all = upto;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    const int items = __shfl_sync(0xffffffffu, upto, 31), rest = items % p.sms, whole = items - rest;
    const int split = rest ? min(p.sms / rest, 16) : 1, unit = blockIdx.x;
    if (unit >= whole + rest * split) return;            // (the whole CTA)
    if (items > p.most_items) {                          // (offsets that go back and forth: more rows than the tensors have)
        if (cv.status && threadIdx.x == 0) atomicExch(cv.status, FLAT_CACHE_BAD_LENGTH);
        return;
    }
    const int item = unit < whole ? unit : whole + (unit - whole) / split, part = unit < whole ? 0 : (unit - whole) % split;
    const int from = __ffs(__ballot_sync(0xffffffffu, upto > item)) - 1;
    int s = from * per, first = __shfl_sync(0xffffffffu, upto - mine_all, from);
    int slabs = slabs_of(s, sp);
    while (item >= first + slabs * cv.Hkv) { first += slabs * cv.Hkv; ++s; slabs = slabs_of(s, sp); }
    const int h = (item - first) % cv.Hkv, row0 = (slabs - 1 - (item - first) / cv.Hkv) * 2 * BM, rows = sp.n * p.G;
    // keys that any row of the slab sees; the part's steps j0 .. j0 + nsteps - 1
    const int last_tok = (row0 + 2 * BM < rows ? row0 + 2 * BM - 1 : rows - 1) / p.G;
    const int n = p.causal ? last_tok + 1 + sp.len - sp.n : sp.len;
    const int all_steps = (n + BN - 1) / BN, pages = (n + cv.page - 1) >> cv.page_shift;
    // (joining costs about a step a part, so n steps take n / P + P in P parts: no more than sqrt(n) of them, of four steps at least)
    const int parts = unit < whole ? 1 : max(1, min(min(split, all_steps / 4), static_cast<int>(sqrtf(static_cast<float>(all_steps)))));
    if (part >= parts) return;
    const int j0 = all_steps * part / parts, nsteps = all_steps * (part + 1) / parts - j0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < LY::NUM_BARS; ++i)
            mbar_init(&bars[i], i < LY::K_EMPTY || (i >= LY::V_FULL && i < LY::V_EMPTY) || (i >= LY::P_FULL && i < LY::PV_DONE) ? 4
                                : (i >= LY::K_EMPTY && i < LY::V_FULL) || (i >= LY::V_EMPTY && i < LY::S_FULL) ? 2 : 1);
        *abort_flag = 0;
        top_exp[0] = top_exp[1] = any_bad = 0;
        part_slot = parts > 1 ? unit - whole : -1;
        part_index = part;
        part_count = parts;
        part_item = (unit - whole) / split;
        fence_mbar_init();
    }
    if (warp == 0) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    {   // the largest exponents of the keys and values, and whether a page is missing
        int ke = 0, ve = 0, bad = 0;
        for (int i = threadIdx.x; i < pages; i += THREADS) {
            int id;
            if (read_page(cv, s, i, id)) {
                const int64_t at = static_cast<int64_t>(id) * cv.Hkv + h;
                ke = max(ke, static_cast<int>(cv.k_exp[at]));
                ve = max(ve, static_cast<int>(cv.v_exp[at]));
            } else {
                bad = 1;
            }
        }
        ke = __reduce_max_sync(0xffffffffu, ke);
        ve = __reduce_max_sync(0xffffffffu, ve);
        bad = __reduce_max_sync(0xffffffffu, bad);
        if (lane == 0) { atomicMax(&top_exp[0], ke); atomicMax(&top_exp[1], ve); if (bad) any_bad = 1; }
        __syncthreads();
    }
    const int EK = top_exp[0], EV = top_exp[1];
    const uint32_t tmem = *tmem_slot;
    const uint32_t bars_s = smem_u32(bars), abort_s = smem_u32(const_cast<int*>(abort_flag)), base_s = smem_u32(base);

    if (warp >= 12) {
        // ------------------------------------------------------------ keys and values: pages -> half-precision tiles
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        const int tid = threadIdx.x - 384;
        constexpr int PIECES = BN * D / 16 / 128;        // of 16 bytes, a thread and tile: 4 (d = 128) or 2
        // piece i: sixteen features from 64 (i / 2) + 16 (tid % 4) of the row tid / 4 + 32 (i % 2): eight lanes write to eight banks
        const uint32_t raw = base_s + LY::RAW_AT + tid * 16;
        const int r0 = tid >> 2, part = tid & 3;
        auto load_ids = [&](int j, int (&id)[2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int key = (j0 + j) * BN + r0 + 32 * i;
                id[i] = -1;
                if (j < nsteps && key < sp.len) {
                    id[i] = cv.table[static_cast<int64_t>(s) * cv.max_pages + (key >> cv.page_shift)];
                    if (id[i] < 0 || id[i] >= cv.num_pages) id[i] = -1;
                }
            }
        };
        auto issue = [&](int j, const int (&id)[2]) {
            if (j < nsteps) {
                const uint32_t dst = raw + (j % LS) * 2 * RAW_BYTES;
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    const int key = (j0 + j) * BN + r0 + 32 * (i & 1);
                    const int64_t src = ((((static_cast<int64_t>(id[i & 1] < 0 ? 0 : id[i & 1]) * cv.Hkv + h) << cv.page_shift) + (key & (cv.page - 1))) * D)
                                        + 64 * (i >> 1) + 16 * part;
                    const int bytes = id[i & 1] >= 0 ? 16 : 0;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + i * 2048), "l"(cv.k + src), "r"(bytes) : "memory");
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + RAW_BYTES + i * 2048), "l"(cv.v + src), "r"(bytes) : "memory");
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        auto load_exps = [&](const int (&id)[2], int (&e)[4]) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e[i] = e[2 + i] = 0;
                if (id[i] >= 0) {
                    const int64_t at = static_cast<int64_t>(id[i]) * cv.Hkv + h;
                    e[i] = cv.k_exp[at];
                    e[2 + i] = cv.v_exp[at];
                }
            }
        };
        auto convert = [&](uint32_t from, uint32_t to, int e0, int e1, int top) {
            // (tokens that no row of the slab sees may lie in pages that the largest was not taken over: they must stay finite)
            const __half2 by[2] = {__float2half2_rn(two_to(min(e0 - top, 0) + LIFT)), __float2half2_rn(two_to(min(e1 - top, 0) + LIFT))};
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                uint4 v;
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from + i * 2048) : "memory");
                uint32_t x[8];
                widen16(v, by[i & 1], x);
                const int row = r0 + 32 * (i & 1);
                const uint32_t at = to + (i >> 1) * (BN * 128) + row * 128;
                sts16(at + (((2 * part) ^ (row & 7)) << 4), x[0], x[1], x[2], x[3]);
                sts16(at + (((2 * part + 1) ^ (row & 7)) << 4), x[4], x[5], x[6], x[7]);
            }
            fence_proxy_async_smem();
            __syncwarp();
        };
        // ids of the steps j + 1, j + 2 and exponents of step j are at hand when step j begins
        int id1[2], id2[2], e[4];
        bool ok = true;
        {
            int id0[2];
            load_ids(0, id0);
            load_ids(1, id1);
            load_ids(2, id2);
            issue(0, id0);
            issue(1, id1);
            load_exps(id0, e);
        }
        for (int j = 0; j < nsteps && ok; ++j) {
            int id3[2], next[4];
            load_ids(j + 3, id3);
            load_exps(id1, next);
            asm volatile("cp.async.wait_group %0;" ::"n"(LS - 2) : "memory");
            issue(j + 2, id2);
            const uint32_t from = raw + (j % LS) * 2 * RAW_BYTES;
            ok = warp_wait(bars_s + 8 * (LY::K_EMPTY + j % KS), ((j / KS) & 1) ^ 1, abort_s, cv.status, 0xb10);
            if (!ok) break;
            convert(from, base_s + LY::K_AT + (j % KS) * KV_BYTES, e[0], e[1], EK);
            if (lane == 0) mbar_arrive(&bars[LY::K_FULL + j % KS]);
            ok = warp_wait(bars_s + 8 * (LY::V_EMPTY + j % VS), ((j / VS) & 1) ^ 1, abort_s, cv.status, 0xb11);
            if (!ok) break;
            convert(from + RAW_BYTES, base_s + LY::V_AT + (j % VS) * KV_BYTES, e[2], e[3], EV);
            if (lane == 0) mbar_arrive(&bars[LY::V_FULL + j % VS]);
#pragma unroll
            for (int i = 0; i < 2; ++i) { id1[i] = id2[i]; id2[i] = id3[i]; e[i] = next[i]; e[2 + i] = next[2 + i]; }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    } else if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
        if (warp <= 9) {
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
    } else {
        // ------------------------------------------------------------ softmax + epilogue (warps 0-7)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int t = warp >> 2, mine = (warp & 3) * 32 + lane, row = row0 + t * BM + mine;
        const uint32_t tl = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t my_bars = bars_s + 8 * (LY::S_FULL + 2 * t);       // S_FULL of the tile; P_FULL and PV_DONE 32 and 64 bytes on
        const int tok = (row < rows ? row : rows - 1) / p.G, head = h * p.G + (row < rows ? row - tok * p.G : 0);
        float unit;
        {   // the query row into half precision
            const uint4* q = reinterpret_cast<const uint4*>(p.Q + (sp.q0 + tok) * p.q_st + head * p.q_sh);
            uint4 v[D / 8];
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                v[i] = row < rows ? q[i] : make_uint4(0, 0, 0, 0);
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[e] << 16)), fabsf(__uint_as_float(w[e] & 0xffff0000u))));
            }
            int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;  // the row's largest: 2^e to 2^(e + 1)
            e = e < -100 ? -100 : e;
            const float up = two_to(14 - e);
            unit = p.scale_log2e * two_to(e - 14) * two_to(EK - 127 - LIFT);
            const uint32_t at = base_s + t * Q_BYTES + mine * 128;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                uint32_t x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = pack_half2(__uint_as_float(w[k] << 16) * up, __uint_as_float(w[k] & 0xffff0000u) * up);
                sts16(at + (i >> 3) * (BM * 128) + (((i & 7) ^ (mine & 7)) << 4), x[0], x[1], x[2], x[3]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars[LY::Q_FULL + t]);
        }
        const bool missing = any_bad != 0;
        float m_ref = -INFINITY, l = 0.f;
        const int nrow = p.causal && tok + 1 + sp.len - sp.n < n ? tok + 1 + sp.len - sp.n : n;
        const int nrow_min = __shfl_sync(0xffffffffu, nrow, 0);
        bool ok = true;
        for (int j = 0; j < nsteps; ++j) {
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
                    if (index < pages) id = cv.table[static_cast<int64_t>(s) * cv.max_pages + index];
                    if (id < 0 || id >= cv.num_pages) out |= 1 << i;
                }
            const bool tail = col0 + BN > nrow_min || out != 0;          // (warp-uniform) some row has masked keys in this step
            const int nvalid = nrow > col0 ? (nrow - col0 < BN ? nrow - col0 : BN) : 0;
            bool careful = j == 0 || tail;
            float lt = 0.f;
            if (!careful) {
                lt = exp_store<false>(x, unit, SHIFT - m_ref, s_addr, BN, 0);
                careful = __any_sync(0xffffffffu, !(lt <= MOST_SUM));
                if (careful) {           // (the weights went over the first half of the logits only)
                    tmem_ld_x32(s_addr + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
                    tc_wait_ld();
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
                lt = exp_store<true>(x, unit, m_ref == -INFINITY ? 0.f : SHIFT - m_ref, s_addr, nvalid, out);
            }
            l += lt;
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_s(my_bars + 32 + 8 * (j & 1));
        }
        if (ok) ok = warp_wait(my_bars + 64 + 8 * ((nsteps - 1) & 1), ((nsteps - 1) >> 1) & 1, abort_s, cv.status, 0xb34 + t);
        if (ok) {
            const float inv = l > 0.f ? two_to(EV - 127 - LIFT) / l : l == l ? 0.f : l;
            const float lse2 = l > 0.f ? m_ref - SHIFT + log2f(l) : l == l ? -INFINITY : l;
            const int slot = part_slot;
            if (slot >= 0) p.part_lse[(slot * 2 + t) * BM + mine] = lse2;
            else if (p.lse && row < rows) p.lse[static_cast<int64_t>(sp.q0 + tok) * p.Hq + head] = lse2 * 0.6931471805599453f;
            tc_fence_after();
            __nv_bfloat16* orow = p.O + (sp.q0 + tok) * p.o_st + head * p.o_sh;
            float4* prow = reinterpret_cast<float4*>(p.part_o) + (static_cast<int64_t>(slot) * (D / 4) * 2 + t) * BM + mine;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t r[32];
                tmem_ld_x32(tl + O_COL(t) + c * 32, r);
                tc_wait_ld();
                float f[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(r[i]) * inv;
                if (slot >= 0) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) prow[(c * 8 + v) * 2 * BM] = make_float4(f[4 * v], f[4 * v + 1], f[4 * v + 2], f[4 * v + 3]);
                } else if (row < rows) {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        *reinterpret_cast<uint4*>(orow + c * 32 + v * 8) = make_uint4(pack_bf16x2(f[8 * v], f[8 * v + 1]), pack_bf16x2(f[8 * v + 2], f[8 * v + 3]),
                                                                                      pack_bf16x2(f[8 * v + 4], f[8 * v + 5]), pack_bf16x2(f[8 * v + 6], f[8 * v + 7]));
                }
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
                join_rows<D>(p, part_slot - part_index, part_count, t * BM + mine, row < rows, sp.q0 + tok, head);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, 512);
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

static size_t prefill_counter_bytes() { return (device_sm_count() * 8 * sizeof(int) + 255) & ~size_t(255); }
size_t cache_prefill_workspace_bytes(int d) { return prefill_counter_bytes() + static_cast<size_t>(device_sm_count()) * 2 * BM * (d + 1) * sizeof(float); }

int launch_cache_prefill(const flat_attn_cache_t& c, const flat_attn_cache_fwd_params_t& q, int least_rows, void* workspace, cudaStream_t st) {
    PrefillArgs p{};
    p.c = cache_view(c);
    p.Q = static_cast<const __nv_bfloat16*>(q.Q);
    p.O = static_cast<__nv_bfloat16*>(q.O);
    p.lse = q.lse;
    p.q_st = q.q_stride_t; p.q_sh = q.q_stride_h; p.o_st = q.o_stride_t; p.o_sh = q.o_stride_h;
    p.total = q.total;
    p.Hq = q.Hq; p.G = q.Hq / c.Hkv; p.max_new = q.max_new; p.least_rows = least_rows; p.causal = q.causal;
    p.sms = device_sm_count();
    char* w = static_cast<char*>(workspace);
    p.counters = reinterpret_cast<int*>(w);
    p.part_lse = reinterpret_cast<float*>(w + prefill_counter_bytes());
    p.part_o = p.part_lse + static_cast<size_t>(p.sms) * 2 * BM;
    p.scale_log2e = q.scale * 1.4426950408889634f;
    return c.d == 64 ? launch_d<64>(c, p, st) : launch_d<128>(c, p, st);
}

}  // namespace flat
