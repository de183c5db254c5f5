// Rotary positions: the first r features of every query and key head, taken in pairs (x1, x2), are rotated by an angle that
// grows with the token's position,
//     y = a (x1 cos t - x2 sin t, x2 cos t + x1 sin t),      t = position * f_i   for pair i,
// so that a logit depends on the distance of its two tokens.  The gradient is the rotation the other way: dx = a R(-t) dy.
// (The paper's decoder workloads encode positions in some way; it does not model how.)
//
// Angles.  In radians and fp32 a position of 10^6 loses what the angle is made of (2^-24 * 10^6 = 0.06 rad).  The table
// holds every frequency in turns per token as a 64-bit fraction, f = F 2^-64; position * F in wrapping 64-bit arithmetic is the
// angle's fraction of a turn, reduced exactly, off by at most |position| 2^-65 turns.  Its upper 32 bits lose another 2^-32 turns (1.5e-9
// rad), and after taking off the nearest quarter turn what is left has 29 bits, rounded to fp32: 2.4e-8 rad.
//
// Bound: device memory, every feature read once and written once.  A CTA takes a few tokens and all their heads, computes the
// tokens' cosines and sines once (shared memory); a thread keeps its token and its place in the row, so those it needs stay in
// registers while it goes from head to head with 16-byte loads and stores.  Measured: 8 x 16 heads of 128 x 2,048 tokens, queries and keys
// (269 MB) 44 us, 6.1 TB/s, 0.93 of a copy; 4 x 16 heads of 64 x 4,096, half of each in neighbouring pairs (134 MB) 23.6 us (51
// with the angles read from shared memory for every vector).  An odd number of pairs, or one that no vector divides, in the half layout: partners one by
// one, 43 us where 22 would be the rate of the others.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "flat_internal.cuh"

namespace flat {

namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_FLIGHT = 2;                           // units in flight per thread (four, and three CTAs an SM: the same; four in two CTAs: 26 us against 22)

// How a row's units (two 16-byte vectors, or one: ROPE_ODD) lie.
enum {
    ROPE_HALF = 0,         // pairs (i, i + r / 2), r / 2 a multiple of the vector: a unit is two vectors r / 2 apart, or (d - r) / 2 where they pass
    ROPE_NEIGHBOURS = 1,   // pairs (2 i, 2 i + 1): a unit is two vectors d / 2 apart (next to each other they would share sectors: 30 us against 24)
    ROPE_ODD = 2           // pairs (i, i + r / 2) at any even r: a unit is one vector, its partners are read one by one
};

__device__ __forceinline__ void unpack(const uint4& v, float (&f)[8], const __nv_bfloat16*) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(w[e] << 16); f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
}
__device__ __forceinline__ void unpack(const uint4& v, float (&f)[4], const float*) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack(const float (&f)[8], const __nv_bfloat16*) {
    return make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
}
__device__ __forceinline__ uint4 pack(const float (&f)[4], const float*) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// One of the two tensors (queries, keys): strides of batch, head and token in elements.
struct RopeSide {
    const void* x;
    void* y;
    long long xs[3], ys[3];
};
struct RopeArgs {
    RopeSide q, k;
    int B, N, Hq, heads, d, r;
    const int32_t* positions;
    long long positions_stride_b;
    const uint64_t* table;
    float amplitude, sign;
    int tile_shift;                                      // log2 of the tokens a CTA takes
};

// Floats from one token's angles to the next: cosines, as many sines; not a multiple of 32, so that tokens lie in different banks.
__host__ __device__ inline int angle_stride(int r) { return 2 * ((r / 2 + 3) & ~3) + 2; }

template <typename T, int MODE>
__global__ void __launch_bounds__(ROPE_THREADS, 4)
rope_kernel(const __grid_constant__ RopeArgs p) {
    constexpr int V = 16 / sizeof(T), UNIT = MODE == ROPE_ODD ? V : 2 * V;
    extern __shared__ float angles[];                    // [token][cosines | sines]
    const int half = p.r / 2, tile = 1 << p.tile_shift, n0 = blockIdx.x << p.tile_shift, b = blockIdx.y;
    const int stride = angle_stride(p.r);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = threadIdx.x; i < half << p.tile_shift; i += ROPE_THREADS) {
        const int t = i / half, c = i - t * half, n = n0 + t;
        if (n >= p.N) break;
        const int64_t position = p.positions ? p.positions[b * p.positions_stride_b + n] : n;
        const uint32_t turns = static_cast<uint32_t>((static_cast<uint64_t>(position) * p.table[c]) >> 32);
        const uint32_t quarter = (turns + 0x20000000u) >> 30;
        float s, co;
        sincospif(static_cast<float>(static_cast<int32_t>(turns - (quarter << 30))) * 4.656612873077393e-10f, &s, &co);   // 2^-31
        const float cq = quarter & 1 ? -s : co, sq = quarter & 1 ? co : s;
        const float flip = quarter & 2 ? -p.amplitude : p.amplitude;
        angles[t * stride + c] = cq * flip;
        angles[t * stride + stride / 2 + c] = sq * flip * p.sign;
    }
    __syncthreads();
    // Units: those of a row side by side, then the tile's tokens, then the heads: as 256 is a multiple of a head's units, a thread
    // keeps its token and its place in the row, and with them its cosines and sines.
    const int per_row = p.d / UNIT, row_shift = 31 - __clz(per_row), head_shift = row_shift + p.tile_shift;
    const int e = threadIdx.x & (per_row - 1), token = threadIdx.x >> row_shift & (tile - 1), n = n0 + token;
    // the unit's (first) vector, its pairs' place among the angles; where it is not rotated: `at` behind r
    const bool turned = MODE != ROPE_HALF || e * UNIT < p.r;
    const int at = MODE == ROPE_HALF && !turned ? p.r + e * V - half : e * V;
    const int mate = MODE == ROPE_NEIGHBOURS ? p.d / 2 : turned ? half : (p.d - p.r) / 2;         // from the first vector to the second
    float cs[V], sn[V];                                  // HALF, ODD: of feature at + j; NEIGHBOURS: of the pairs of both vectors
    {
        const float *co = angles + token * stride, *si = co + stride / 2;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int f = MODE == ROPE_NEIGHBOURS ? (2 * j < V ? at + 2 * j : at + mate + 2 * j - V) / 2 : MODE == ROPE_ODD && at + j >= half ? at + j - half : at + j;
            const bool there = f < half;                 // (beyond: never used)
            cs[j] = there ? co[f] : 0.f;
            sn[j] = there ? (MODE == ROPE_ODD && at + j < half ? -si[f] : si[f]) : 0.f;
        }
    }
    const int head_step = ROPE_THREADS >> head_shift;
    for (int h0 = threadIdx.x >> head_shift; h0 - static_cast<int>(threadIdx.x >> head_shift) < p.heads; h0 += head_step * ROPE_FLIGHT) {
        uint4 a[ROPE_FLIGHT], c[ROPE_FLIGHT];
        float partner[MODE == ROPE_ODD ? ROPE_FLIGHT : 1][V];
        T* out[ROPE_FLIGHT];
#pragma unroll
        for (int i = 0; i < ROPE_FLIGHT; ++i) {
            int h = h0 + i * head_step;
            out[i] = nullptr;
            if (h < p.heads && n < p.N) {
                const bool key = h >= p.Hq;
                if (key) h -= p.Hq;
                const RopeSide& side = key ? p.k : p.q;
                const T* x = static_cast<const T*>(side.x) + b * side.xs[0] + h * side.xs[1] + n * side.xs[2];
                out[i] = static_cast<T*>(side.y) + b * side.ys[0] + h * side.ys[1] + n * side.ys[2];
                a[i] = *reinterpret_cast<const uint4*>(x + at);
                if (MODE != ROPE_ODD) c[i] = *reinterpret_cast<const uint4*>(x + at + mate);
                if (MODE == ROPE_ODD) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int f = at + j;
                        partner[i][j] = f < p.r ? static_cast<float>(x[f < half ? f + half : f - half]) : 0.f;
                    }
                }
            }
        }
        // (a row's units are lanes of one warp: where Y is X, every partner has been read before any is written)
        if (MODE == ROPE_ODD) __syncwarp();
#pragma unroll
        for (int i = 0; i < ROPE_FLIGHT; ++i) {
            if (!out[i]) continue;
            float x1[V], x2[V];
            unpack(a[i], x1, static_cast<const T*>(nullptr));
            if (MODE == ROPE_ODD) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (at + j < p.r) x1[j] = x1[j] * cs[j] + partner[i][j] * sn[j];
                *reinterpret_cast<uint4*>(out[i] + at) = pack(x1, static_cast<const T*>(nullptr));
                continue;
            }
            if (MODE == ROPE_HALF && !turned) {
                *reinterpret_cast<uint4*>(out[i] + at) = a[i];
                *reinterpret_cast<uint4*>(out[i] + at + mate) = c[i];
                continue;
            }
            unpack(c[i], x2, static_cast<const T*>(nullptr));
            if (MODE == ROPE_HALF) {
                float y1[V], y2[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    y1[j] = x1[j] * cs[j] - x2[j] * sn[j];
                    y2[j] = x2[j] * cs[j] + x1[j] * sn[j];
                }
                *reinterpret_cast<uint4*>(out[i] + at) = pack(y1, static_cast<const T*>(nullptr));
                *reinterpret_cast<uint4*>(out[i] + at + half) = pack(y2, static_cast<const T*>(nullptr));
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {            // pairs j of the 2 V features of both vectors
                    float &u = 2 * j < V ? x1[2 * j % V] : x2[2 * j % V], &v = 2 * j < V ? x1[2 * j % V + 1] : x2[2 * j % V + 1];
                    if ((2 * j < V ? at + 2 * j : at + mate + 2 * j - V) < p.r) {
                        const float w = u * cs[j] - v * sn[j];
                        v = v * cs[j] + u * sn[j];
                        u = w;
                    }
                }
                *reinterpret_cast<uint4*>(out[i] + at) = pack(x1, static_cast<const T*>(nullptr));
                *reinterpret_cast<uint4*>(out[i] + at + mate) = pack(x2, static_cast<const T*>(nullptr));
            }
        }
    }
}

template <typename T>
int launch_typed(const RopeArgs& args, bool neighbours, cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    RopeArgs p = args;
    const int mode = neighbours ? ROPE_NEIGHBOURS : (p.r / 2) % V == 0 && (p.d - p.r) % (2 * V) == 0 ? ROPE_HALF : ROPE_ODD;
    // Tokens per CTA: eight, or fewer while that leaves SMs without a CTA
    p.tile_shift = 3;
    const int64_t sms = device_sm_count();
    while (p.tile_shift > 0 && (((p.N - 1) >> p.tile_shift) + 1) * static_cast<int64_t>(p.B) < 2 * sms) --p.tile_shift;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(((p.N - 1) >> p.tile_shift) + 1, p.B);
    cfg.blockDim = dim3(ROPE_THREADS);
    cfg.dynamicSmemBytes = static_cast<size_t>(angle_stride(p.r)) * sizeof(float) << p.tile_shift;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    auto kern = mode == ROPE_HALF ? rope_kernel<T, ROPE_HALF> : mode == ROPE_NEIGHBOURS ? rope_kernel<T, ROPE_NEIGHBOURS> : rope_kernel<T, ROPE_ODD>;
    return cudaLaunchKernelEx(&cfg, kern, p) == cudaSuccess ? FLAT_OK : FLAT_ERR_CUDA;
}

}  // namespace

int launch_rope(const flat_attn_rope_params_t& p, bool back, cudaStream_t st) {
    RopeArgs a{};
    auto side = [](const void* x, void* y, const long long (&xs)[3], const long long (&ys)[3]) {
        return RopeSide{x, y, {xs[0], xs[1], xs[2]}, {ys[0], ys[1], ys[2]}};
    };
    a.q = side(p.Q, p.Qr, p.q_stride, p.qr_stride);
    if (p.K) a.k = side(p.K, p.Kr, p.k_stride, p.kr_stride);
    a.B = p.B; a.N = p.N; a.Hq = p.Hq; a.heads = p.Hq + (p.K ? p.Hk : 0); a.d = p.d; a.r = p.rotary_dim;
    a.positions = p.positions;
    a.positions_stride_b = p.positions_stride_b;
    a.table = p.table;
    a.amplitude = p.amplitude;
    a.sign = back ? -1.f : 1.f;
    return p.dtype == FLAT_DTYPE_F32 ? launch_typed<float>(a, p.interleaved, st) : launch_typed<__nv_bfloat16>(a, p.interleaved, st);
}

}  // namespace flat
