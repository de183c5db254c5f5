// New tokens' keys and values into the pages of the 8-bit cache: e4m3 values with a power-of-two scale for each page and head.
//
// With top = max |x| over the page's new tokens, e = the least integer >= -117 with top <= 448 * 2^e (448 is the largest e4m3
// number), not below the page's exponent where earlier tokens share it; q = e4m3(x * 2^-e), a product that is exact and one
// rounding.  A scale that is a power of two costs a floating-point format nothing (its relative precision is the same
// everywhere), and lets a page whose scale grows be requantised without a second rounding, subnormal numbers aside.
//
// Bound: device memory, 2 bytes read and 1 written per feature.  A page and head of a sequence is a unit: its new tokens are
// read once into registers, 32 bytes a thread and pass, reduced, scaled and written.  With one new token a sequence a warp takes the
// token's keys or values of a head: there the launch and the chain of dependent loads count (offsets, table entry, exponent), and
// the page that is requantised when its scale grows, eight rows in flight a lane.
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
// Two bf16 (one word) to two e4m3, times s.  Infinities become NaN.
__device__ __forceinline__ uint32_t quantise2(uint32_t w, float s) {
    float a = __uint_as_float(w << 16) * s, b = __uint_as_float(w & 0xffff0000u) * s;
    if (isinf(a)) a = __int_as_float(0x7fc00000);
    if (isinf(b)) b = __int_as_float(0x7fc00000);
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float finite_top2(uint32_t w, float top) {
    const float a = fabsf(__uint_as_float(w << 16)), b = fabsf(__uint_as_float(w & 0xffff0000u));
    if (a < INFINITY) top = fmaxf(top, a);               // (false for NaN)
    if (b < INFINITY) top = fmaxf(top, b);
    return top;
}
__device__ __forceinline__ uint4 quantise16(const uint4& a, const uint4& b, float s) {
    uint4 q;
    q.x = quantise2(a.x, s) | quantise2(a.y, s) << 16;
    q.y = quantise2(a.z, s) | quantise2(a.w, s) << 16;
    q.z = quantise2(b.x, s) | quantise2(b.y, s) << 16;
    q.w = quantise2(b.z, s) | quantise2(b.w, s) << 16;
    return q;
}
__device__ __forceinline__ float finite_top16(const uint4& a, const uint4& b) {
    float t = finite_top2(a.x, 0.f);
    t = finite_top2(a.y, t); t = finite_top2(a.z, t); t = finite_top2(a.w, t);
    t = finite_top2(b.x, t); t = finite_top2(b.y, t); t = finite_top2(b.z, t); t = finite_top2(b.w, t);
    return t;
}
// The rows row, row + step, ... below `rows` (sixteen of their values, from `at` on) rounded again to a scale `down` powers of two above
// theirs.  Eight rows in flight: what this waits for is latency.
__device__ __forceinline__ void requantise_rows(uint8_t* at, int row, int rows, int step, int width, int down) {
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
    int max_new, slots;                                  // slots: pages that a sequence's new tokens may touch
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
    float top = finite_top16(a, b);
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int e = joint_exponent(top, row > 0, was);
    uint8_t* at = (which ? p.c.v : p.c.k) + place * p.c.page * D + 16 * (lane % LANES);
    if (row > 0 && e + 127 > was) requantise_rows(at, lane / LANES, row, 32 / LANES, D, e + 127 - was);
    if (lane < LANES) *reinterpret_cast<uint4*>(at + row * D) = quantise16(a, b, power_of_two(-e));
    if (lane == 0 && (row == 0 || e + 127 != was)) *exp = static_cast<uint8_t>(e + 127);
}

// ---------------------------------------------------------------- a page and head a CTA: the first half of its warps takes K, the second V
template <int D, int PAGE>
__global__ void __launch_bounds__(256)
append_kernel(const __grid_constant__ AppendArgs p) {
    constexpr int WARPS = PAGE * D / 16 / 32 >= 4 ? 4 : PAGE * D / 16 / 32, SIDE = 32 * WARPS;   // per side
    constexpr int PASSES = PAGE * D / 16 / SIDE, ROWS = SIDE / (D / 16);
    __shared__ float tops[2][WARPS];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int which = threadIdx.x / SIDE, tid = threadIdx.x % SIDE;
    const unsigned heads = p.c.Hkv, slots = p.slots;
    const int h = blockIdx.x % heads, slot = blockIdx.x / heads % slots, s = blockIdx.x / heads / slots;
    Span sp{};
    if (!read_span(p.c, s, p.total, p.max_new, sp)) return;
    const int start = sp.len - sp.n, first_page = start / PAGE, index = first_page + slot;
    if (sp.n == 0 || index * PAGE >= sp.len) return;
    int page_id;
    if (!read_page(p.c, s, index, page_id)) return;
    const int r0 = slot == 0 ? start - first_page * PAGE : 0, r1 = sp.len - index * PAGE < PAGE ? sp.len - index * PAGE : PAGE;
    const int row = tid / (D / 16), col = tid % (D / 16) * 16;
    const __nv_bfloat16* x = p.x[which] + h * p.sh[which] + col;
    const int64_t token0 = sp.q0 + (index * PAGE - start);      // the token of row 0 (if it were new)
    uint4 a[PASSES], b[PASSES];
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int r = row + i * ROWS;
        a[i] = b[i] = make_uint4(0, 0, 0, 0);
        if (r >= r0 && r < r1) {
            const uint4* v = reinterpret_cast<const uint4*>(x + (token0 + r) * p.st[which]);
            a[i] = v[0];
            b[i] = v[1];
        }
    }
    uint8_t* exp = (which ? p.c.v_exp : p.c.k_exp) + static_cast<int64_t>(page_id) * p.c.Hkv + h;
    const int was = r0 > 0 ? *exp : 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) top = fmaxf(top, finite_top16(a[i], b[i]));
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if ((threadIdx.x & 31) == 0) tops[which][tid >> 5] = top;
    __syncthreads();                                     // (and every thread has read the exponent)
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, tops[which][w]);
    const int e = joint_exponent(top, r0 > 0, was);
    uint8_t* at = (which ? p.c.v : p.c.k) + (static_cast<int64_t>(page_id) * p.c.Hkv + h) * PAGE * D + col;
    if (r0 > 0 && e + 127 > was) requantise_rows(at, row, r0, ROWS, D, e + 127 - was);
    const float scale = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int r = row + i * ROWS;
        if (r >= r0 && r < r1) *reinterpret_cast<uint4*>(at + r * D) = quantise16(a[i], b[i], scale);
    }
    if (tid == 0) *exp = static_cast<uint8_t>(e + 127);
}

template <int D>
int launch_d(const AppendArgs& p, cudaStream_t st) {
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
        blocks = static_cast<int64_t>(p.c.num_seqs) * p.c.Hkv * p.slots;
        const int warps = p.c.page * D / 16 / 32;
        cfg.blockDim = dim3(64 * (warps < 4 ? warps : 4));
        kern = p.c.page == 16 ? append_kernel<D, 16> : p.c.page == 32 ? append_kernel<D, 32> : p.c.page == 64 ? append_kernel<D, 64> : append_kernel<D, 128>;
    }
    if (blocks > 0x1fffffff) return FLAT_ERR_SHAPE;      // (units, four to a CTA, are counted in 32 bits)
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    return cudaLaunchKernelEx(&cfg, kern, p) == cudaSuccess ? FLAT_OK : FLAT_ERR_CUDA;
}

}  // namespace

int launch_cache_append(const flat_attn_cache_t& c, const void* K, const void* V, int64_t total, long long k_st, long long k_sh,
                        long long v_st, long long v_sh, int max_new, cudaStream_t st) {
    AppendArgs p{cache_view(c), {static_cast<const __nv_bfloat16*>(K), static_cast<const __nv_bfloat16*>(V)}, {k_st, v_st}, {k_sh, v_sh},
                 total, max_new, static_cast<int>((max_new + static_cast<int64_t>(c.page) - 2) / c.page + 1)};
    return c.d == 64 ? launch_d<64>(p, st) : launch_d<128>(p, st);
}

}  // namespace flat
