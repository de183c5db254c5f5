// New tokens' keys and values into the pages of the 8-bit cache: e4m3 values with a power-of-two scale for each page and head.
//
// With top = max |x| over the page's new tokens, e = the least integer >= -117 with top <= 448 * 2^e (448 is the largest e4m3
// number), not below the page's exponent where earlier tokens share it; q = e4m3(x * 2^-e), a product that is exact and one
// rounding.  A scale that is a power of two costs a floating-point format nothing (its relative precision is the same
// everywhere), and lets a page whose scale grows be requantised without a second rounding, subnormal numbers aside.
//
// Bound: device memory, 2 bytes read and 1 written per feature.  The keys (or the values) of a page and head are a unit: a warp
// reads its new tokens once into registers (32 bytes a lane and pass, up to four passes in flight; two to eight warps for larger pages),
// reduces, scales and writes them; what a unit waits for is its chain of loads (offsets, table entry, tokens), so that many
// small units an SM are better than few large ones (24 prompts of 1-4K tokens, pages of 64, d = 128: four CTAs an SM 62.9 us, eight
// passes in two CTAs 71.6, two passes 89).  The largest magnitude is taken from the bits, two values at a time, the check for infinities
// only where there is one (with plain comparisons twice the time).  Measured: 6 prompts, 11,700 tokens, 8 heads, d = 128 in pages of
// 16 (72 MB) 14.8 us out of memory, 11 out of L2.  A call's grid goes by its tokens, not by its longest sequence: 254 sequences with one and two with 5,596
// new tokens together 13 us in pages of 16 and 21 of 64 (a place for as many pages as the longest has, for every sequence: 367 and 392).
// With one new token a sequence a warp takes the token's keys or values of a head: 64 sequences, 8 heads 3.1 us, which is the launch
// and the chain.  The page that is requantised when its scale grows has eight rows in flight a lane.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cache_common.cuh"
#include "flat_internal.cuh"

namespace flat {

namespace {

using namespace cache;

// The exponent for a largest magnitude (finite).
__device__ __forceinline__ int exponent_for(float top) {
    if (!(top > 0.f)) return MIN_EXP;
    // top = m 2^x, 1 <= m < 2; 448 = 1.75 * 2^8.  (Subnormal numbers of bf16 lie far below the least exponent.)
    const int x = static_cast<int>(__float_as_uint(top) >> 23) - 127;
    const int e = x - 8 + ((__float_as_uint(top) & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < MIN_EXP ? MIN_EXP : e;
}
__device__ __forceinline__ float power_of_two(int e) {   // -126 <= e <= 127
    return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
// Two bf16 (one word) to two e4m3, times s.  CHECK: infinities (which the conversion would make the largest number) become NaN.
template <bool CHECK>
__device__ __forceinline__ uint32_t quantise2(uint32_t w, float s) {
    float a = __uint_as_float(w << 16) * s, b = __uint_as_float(w & 0xffff0000u) * s;
    if (CHECK) {
        if (isinf(a)) a = __int_as_float(0x7fc00000);
        if (isinf(b)) b = __int_as_float(0x7fc00000);
    }
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
template <bool CHECK>
__device__ __forceinline__ uint4 quantise16(const uint4& a, const uint4& b, float s) {
    uint4 q;
    q.x = quantise2<CHECK>(a.x, s) | quantise2<CHECK>(a.y, s) << 16;
    q.y = quantise2<CHECK>(a.z, s) | quantise2<CHECK>(a.w, s) << 16;
    q.z = quantise2<CHECK>(b.x, s) | quantise2<CHECK>(b.y, s) << 16;
    q.w = quantise2<CHECK>(b.z, s) | quantise2<CHECK>(b.w, s) << 16;
    return q;
}
// The largest finite magnitude of bf16 values, two at a time: magnitude bits plus 0x80 are a positive 16-bit number for finite values
// and a negative one for infinities and NaN.  `top`: the largest so far of each half; `all`: bit 15 or 31 once one is not finite.
__device__ __forceinline__ void largest(uint32_t w, uint32_t& top, uint32_t& all) {
    const uint32_t h = (w & 0x7fff7fffu) + 0x00800080u;
    all |= h;
    asm("max.s16x2 %0, %0, %1;" : "+r"(top) : "r"(h));
}
__device__ __forceinline__ void largest16(const uint4& a, const uint4& b, uint32_t& top, uint32_t& all) {
    largest(a.x, top, all); largest(a.y, top, all); largest(a.z, top, all); largest(a.w, top, all);
    largest(b.x, top, all); largest(b.y, top, all); largest(b.z, top, all); largest(b.w, top, all);
}
// Over the warp: that magnitude's bits plus 0x80, and 2^30 if a value was not finite (one number for the warps of a unit to compare).
__device__ __forceinline__ int warp_largest(uint32_t top, uint32_t all) {
    const int lo = static_cast<int16_t>(top & 0xffffu), hi = static_cast<int>(top) >> 16;
    return __reduce_max_sync(0xffffffffu, max(lo, hi)) | (__any_sync(0xffffffffu, (all & 0x80008000u) != 0) ? 1 << 30 : 0);
}
constexpr uint32_t NOTHING = 0x00800080u;                // (two zeros)
__device__ __forceinline__ float magnitude(int largest) { return __uint_as_float(static_cast<uint32_t>((largest & 0xffff) - 0x80) << 16); }

// The rows row, row + step, ... below `rows` (sixteen of their values, from `at` on) rounded again to a scale `down` powers of two above
// theirs.  Eight rows in flight: what this waits for is latency.  (Not
// inlined: it is rare, and its registers would cost every call half the warps of an SM.)
__device__ __noinline__ void requantise_rows(uint8_t* at, int row, int rows, int step, int width, int down) {
    const float s = power_of_two(down > 40 ? -40 : -down);       // (448 * 2^-40 is 0 in e4m3, like everything below)
    constexpr int FLIGHT = 8;
    for (; row < rows; row += step * FLIGHT) {
        uint4 v[FLIGHT];
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i)
            if (row + i * step < rows) v[i] = *reinterpret_cast<const uint4*>(at + (row + i * step) * width);
#pragma unroll
        for (int i = 0; i < FLIGHT; ++i) {
            if (row + i * step >= rows) continue;
            uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t out = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const __half2_raw f = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[j] >> (16 * h)), __NV_E4M3);
                    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&f));
                    out |= static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(x.x * s, x.y * s), __NV_SATFINITE, __NV_E4M3)) << (16 * h);
                }
                w[j] = out;
            }
            *reinterpret_cast<uint4*>(at + (row + i * step) * width) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}
// The exponent of a page and head, from that of its new tokens and, where earlier ones share the page, theirs (the byte `was`).
// (Bytes above the largest exponent that this file writes are not valid; they must not lead outside the range of powers.)
__device__ __forceinline__ int joint_exponent(float top, bool shared, int was) {
    const int e = exponent_for(top), old = (was > 247 ? 247 : was) - 127;
    return shared && old > e ? old : e;
}

struct AppendArgs {
    CacheView c;
    const __nv_bfloat16* x[2];                           // K, V
    long long st[2], sh[2];
    long long total;
    int max_new;
    unsigned most_pages;                                 // that the grid was made for (append_kernel)
};

// ---------------------------------------------------------------- one new token a sequence: a warp per (sequence, head, K or V)
template <int D>
__global__ void __launch_bounds__(128)
append_one_kernel(const __grid_constant__ AppendArgs p) {
    constexpr int LANES = D / 16;                        // the lanes that hold the token, sixteen features each
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned unit = blockIdx.x * 4 + threadIdx.x / 32;
    const int lane = threadIdx.x & 31, which = unit & 1;
    const unsigned s = (unit >> 1) / p.c.Hkv, h = (unit >> 1) % p.c.Hkv;
    Span sp;
    if (s >= static_cast<unsigned>(p.c.num_seqs) || !read_span(p.c, s, p.total, p.max_new, sp) || sp.n != 1) return;
    const int pos = sp.len - 1, row = pos & (p.c.page - 1);
    int page_id;
    if (!read_page(p.c, s, pos >> p.c.page_shift, page_id)) return;
    uint4 a = make_uint4(0, 0, 0, 0), b = a;
    if (lane < LANES) {
        const uint4* x = reinterpret_cast<const uint4*>(p.x[which] + sp.q0 * p.st[which] + h * p.sh[which]) + 2 * lane;
        a = x[0];
        b = x[1];
    }
    const int64_t place = static_cast<int64_t>(page_id) * p.c.Hkv + h;
    uint8_t* exp = (which ? p.c.v_exp : p.c.k_exp) + place;
    const int was = row > 0 ? *exp : 0;
    uint32_t top = NOTHING, all = 0;
    largest16(a, b, top, all);
    const int most = warp_largest(top, all);
    const int e = joint_exponent(magnitude(most), row > 0, was);
    uint8_t* at = (which ? p.c.v : p.c.k) + place * p.c.page * D + 16 * (lane % LANES);
    if (lane < LANES)
        *reinterpret_cast<uint4*>(at + row * D) = most >> 30 ? quantise16<true>(a, b, power_of_two(-e)) : quantise16<false>(a, b, power_of_two(-e));
    if (row > 0 && e + 127 > was) requantise_rows(at, lane / LANES, row, 32 / LANES, D, e + 127 - was);
    if (lane == 0 && (row == 0 || e + 127 != was)) *exp = static_cast<uint8_t>(e + 127);
}

// ---------------------------------------------------------------- a page and head, keys or values: a unit of one to eight warps
template <int D, int PAGE> struct Unit {
    static constexpr int PASSES = PAGE * D / 512 < 4 ? PAGE * D / 512 : 4;        // of a warp: sixteen features a lane
    static constexpr int WARPS = PAGE * D / 512 / PASSES, PER_CTA = 8 / WARPS;     // (at most 16,384 features: eight warps)
};
template <int D, int PAGE>
__global__ void __launch_bounds__(256, 4)
append_kernel(const __grid_constant__ AppendArgs p) {
    using U = Unit<D, PAGE>;
    constexpr int ROWS = U::WARPS * 32 / (D / 16);       // of a pass
    __shared__ int tops[8], found[U::PER_CTA][5];        // found: sequence, its span, the page's place among those of its new tokens
    __shared__ unsigned sums[8];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x % (32 * U::WARPS);
    const unsigned heads = p.c.Hkv;
    // The pages that new tokens go to, sequence after sequence, are counted; unit / 2 / heads is a page's place among them.  (No more than
    // num_seqs * max_pages: with their heads, keys and values they fit 32 bits.)
    auto pages_of = [&](int s, Span& sp) {
        if (!read_span(p.c, s, p.total, p.max_new, sp) || sp.n == 0) return 0u;
        return static_cast<unsigned>((sp.len - 1) / PAGE - (sp.len - sp.n) / PAGE + 1);
    };
    auto before_and_this = [&](unsigned v) {             // of the lanes below and this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        return v;
    };
    const unsigned first_unit = blockIdx.x * U::PER_CTA, unit = first_unit + warp / U::WARPS;
    const int which = unit & 1, h = (unit >> 1) % heads;
    int s, slot;
    Span sp{0, 0, 0};
    unsigned all_pages;
    if (p.c.num_seqs <= 32) {                            // every warp for itself, a lane a sequence
        const unsigned pages = lane < p.c.num_seqs ? pages_of(lane, sp) : 0, upto = before_and_this(pages), at = (unit >> 1) / heads;
        all_pages = __shfl_sync(0xffffffffu, upto, 31);
        s = __ffs(__ballot_sync(0xffffffffu, upto > at)) - 1;              // (-1: no such unit)
        slot = at - __shfl_sync(0xffffffffu, upto - pages, s);
        sp = Span{__shfl_sync(0xffffffffu, sp.q0, s), __shfl_sync(0xffffffffu, sp.n, s), __shfl_sync(0xffffffffu, sp.len, s)};
    } else {
        // the CTA together, a thread a few sequences (by every warp for itself: 256 sequences, two of them with 5,600 tokens, 19.6 us against 12.0;
        // this for six sequences: 13.3 against 11.0)
        const int per = (p.c.num_seqs + 255) / 256, s_begin = threadIdx.x * per, s_end = min(s_begin + per, p.c.num_seqs);
        unsigned pages = 0;
#pragma unroll 4
        for (int i = s_begin; i < s_end; ++i) pages += pages_of(i, sp);
        unsigned upto = before_and_this(pages);
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        all_pages = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (w < warp) upto += sums[w];
            all_pages += sums[w];
        }
        // the thread whose sequences have the page of a unit says which one it is
#pragma unroll 1
        for (int i = 0; i < U::PER_CTA; ++i) {
            const unsigned at = ((first_unit + i) >> 1) / heads;
            unsigned before = upto - pages;
            if (at < before || at >= upto) continue;
            int whose = s_begin;
            if (per > 1)                                 // (one sequence a thread: it has been read)
                for (unsigned n = pages_of(whose, sp); at >= before + n; n = pages_of(++whose, sp)) before += n;
            found[i][0] = whose; found[i][1] = sp.q0; found[i][2] = sp.n; found[i][3] = sp.len; found[i][4] = at - before;
        }
        __syncthreads();
        const int mine = warp / U::WARPS;
        s = found[mine][0];
        slot = found[mine][4];
        sp = Span{found[mine][1], found[mine][2], found[mine][3]};
    }
    const unsigned units = 2 * heads * all_pages;
    if (first_unit >= units) return;                     // (the whole CTA)
    if (all_pages > p.most_pages) {                      // (offsets that go back and forth: more tokens than there are)
        if (p.c.status && threadIdx.x == 0) atomicExch(p.c.status, FLAT_CACHE_BAD_LENGTH);
        return;
    }
    bool work = unit < units;
    const int start = sp.len - sp.n, first_page = start / PAGE, index = first_page + slot;
    int page_id = 0;
    work = work && read_page(p.c, s, index, page_id);
    const int r0 = slot == 0 ? start - first_page * PAGE : 0;
    const int r1 = !work ? 0 : sp.len - index * PAGE < PAGE ? sp.len - index * PAGE : PAGE;
    const int row = tid / (D / 16), col = tid % (D / 16) * 16;
    const __nv_bfloat16* x = p.x[which] + h * p.sh[which] + col;
    const int64_t token0 = sp.q0 + (index * PAGE - start);      // the token of row 0 (if it were new)
    const int64_t place = static_cast<int64_t>(page_id) * p.c.Hkv + h;
    uint8_t* exp = (which ? p.c.v_exp : p.c.k_exp) + place;
    uint4 a[U::PASSES], b[U::PASSES];
#pragma unroll
    for (int i = 0; i < U::PASSES; ++i) {
        const int r = row + i * ROWS;
        a[i] = b[i] = make_uint4(0, 0, 0, 0);
        if (r >= r0 && r < r1) {
            const uint4* v = reinterpret_cast<const uint4*>(x + (token0 + r) * p.st[which]);
            a[i] = v[0];
            b[i] = v[1];
        }
    }
    const int was = work && r0 > 0 ? *exp : 0;
    uint32_t top = NOTHING, all = 0;
#pragma unroll
    for (int i = 0; i < U::PASSES; ++i) largest16(a[i], b[i], top, all);
    int most = warp_largest(top, all);
    if (U::WARPS > 1) {
        if (lane == 0) tops[warp] = most;
        __syncthreads();                                 // (and every thread has read the exponent)
#pragma unroll
        for (int w = 0; w < U::WARPS; ++w) {
            const int other = tops[warp / U::WARPS * U::WARPS + w];
            most = max(most & 0xffff, other & 0xffff) | ((most | other) & 1 << 30);
        }
    }
    if (!work) return;
    const int e = joint_exponent(magnitude(most), r0 > 0, was);
    uint8_t* at = (which ? p.c.v : p.c.k) + place * (PAGE * D) + col;
    const float scale = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < U::PASSES; ++i) {
        const int r = row + i * ROWS;
        if (r >= r0 && r < r1) *reinterpret_cast<uint4*>(at + r * D) = most >> 30 ? quantise16<true>(a[i], b[i], scale) : quantise16<false>(a[i], b[i], scale);
    }
    // (the new tokens are out of the registers)
    if (r0 > 0 && e + 127 > was) requantise_rows(at, row, r0, ROWS, D, e + 127 - was);
    if (tid == 0) *exp = static_cast<uint8_t>(e + 127);
}

template <int D>
int launch_d(const AppendArgs& args, cudaStream_t st) {
    AppendArgs p = args;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void (*kern)(AppendArgs) = append_one_kernel<D>;
    int64_t blocks;
    if (p.max_new == 1) {
        blocks = (static_cast<int64_t>(p.c.num_seqs) * p.c.Hkv * 2 + 3) / 4;
        cfg.blockDim = dim3(128);
    } else {
        const int per_cta = p.c.page == 16 ? Unit<D, 16>::PER_CTA : p.c.page == 32 ? Unit<D, 32>::PER_CTA : p.c.page == 64 ? Unit<D, 64>::PER_CTA : Unit<D, 128>::PER_CTA;
        // Pages that new tokens may go to: those of the longest for every sequence, or as many as all tokens fill and two more a sequence
        const int64_t longest = (p.max_new + static_cast<int64_t>(p.c.page) - 2) / p.c.page + 1;
        const int64_t most = p.total / p.c.page + 2 * static_cast<int64_t>(p.c.num_seqs), pages = longest < most / p.c.num_seqs ? longest * p.c.num_seqs : most;
        p.most_pages = static_cast<unsigned>(pages < 0xffffffffll ? pages : 0xffffffffll);
        blocks = (pages * p.c.Hkv * 2 + per_cta - 1) / per_cta;
        cfg.blockDim = dim3(256);
        kern = p.c.page == 16 ? append_kernel<D, 16> : p.c.page == 32 ? append_kernel<D, 32> : p.c.page == 64 ? append_kernel<D, 64> : append_kernel<D, 128>;
    }
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));  // (2^34 tokens and heads of a cache are at most 2^30 CTAs)
    return cudaLaunchKernelEx(&cfg, kern, p) == cudaSuccess ? FLAT_OK : FLAT_ERR_CUDA;
}

}  // namespace

int launch_cache_append(const flat_attn_cache_t& c, const void* K, const void* V, int64_t total, long long k_st, long long k_sh,
                        long long v_st, long long v_sh, int max_new, cudaStream_t st) {
    AppendArgs p{cache_view(c), {static_cast<const __nv_bfloat16*>(K), static_cast<const __nv_bfloat16*>(V)}, {k_st, v_st}, {k_sh, v_sh},
                 total, max_new, 0};
    return c.d == 64 ? launch_d<64>(p, st) : launch_d<128>(p, st);
}

}  // namespace flat
