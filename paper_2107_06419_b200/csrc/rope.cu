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
// tokens' cosines and sines once (shared memory) and rotates with 16-byte loads and stores, four pairs of them in flight a thread.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "flat_internal.cuh"

namespace flat {

namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_FLIGHT = 4;                           // units in flight per thread

// How a row's units (two 16-byte vectors, or one: ROPE_ODD) lie.
enum {
    ROPE_HALF = 0,         // pairs (i, i + r / 2), r / 2 a multiple of the vector: a unit is two vectors r / 2 apart, the rest pass in pairs of vectors
    ROPE_NEIGHBOURS = 1,   // pairs (2 i, 2 i + 1): a unit is 32 contiguous bytes
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

template <typename T, int MODE>
__global__ void __launch_bounds__(ROPE_THREADS)
rope_kernel(const __grid_constant__ RopeArgs p) {
    constexpr int V = 16 / sizeof(T), UNIT = MODE == ROPE_ODD ? V : 2 * V;
    extern __shared__ float angles[];                    // [token][cos: r / 2 | sin: r / 2], as read in vectors
    const int half = p.r / 2, tile = 1 << p.tile_shift, n0 = blockIdx.x << p.tile_shift, b = blockIdx.y;
    const int pad = (half + 3) & ~3;                     // (16-byte rows)
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
        angles[t * 2 * pad + c] = cq * flip;
        angles[t * 2 * pad + pad + c] = sq * flip * p.sign;
    }
    __syncthreads();
    // Units: consecutive ones of a row side by side, then the rows of the tile's tokens, head after head.
    const int per_row = p.d / UNIT, row_shift = 31 - __clz(per_row), units = (p.heads << p.tile_shift) << row_shift;
    for (int u0 = threadIdx.x; u0 - static_cast<int>(threadIdx.x) < units; u0 += ROPE_THREADS * ROPE_FLIGHT) {
        uint4 a[ROPE_FLIGHT], c[ROPE_FLIGHT];
        float partner[MODE == ROPE_ODD ? ROPE_FLIGHT : 1][V];
        T* out[ROPE_FLIGHT];
        int at[ROPE_FLIGHT], token[ROPE_FLIGHT];
#pragma unroll
        for (int i = 0; i < ROPE_FLIGHT; ++i) {
            const int u = u0 + i * ROPE_THREADS, row = u >> row_shift, e = u & (per_row - 1);
            token[i] = row & (tile - 1);
            int h = row >> p.tile_shift;
            out[i] = nullptr;
            if (u < units && n0 + token[i] < p.N) {
                const bool key = h >= p.Hq;
                if (key) h -= p.Hq;
                const RopeSide& side = key ? p.k : p.q;
                const T* x = static_cast<const T*>(side.x) + b * side.xs[0] + h * side.xs[1] + (n0 + token[i]) * side.xs[2];
                out[i] = static_cast<T*>(side.y) + b * side.ys[0] + h * side.ys[1] + (n0 + token[i]) * side.ys[2];
                if (MODE == ROPE_HALF) {
                    at[i] = e * UNIT < p.r ? e * V : e * UNIT;
                    a[i] = *reinterpret_cast<const uint4*>(x + at[i]);
                    c[i] = *reinterpret_cast<const uint4*>(x + at[i] + (at[i] < half ? half : V));
                } else {
                    at[i] = e * UNIT;
                    a[i] = *reinterpret_cast<const uint4*>(x + at[i]);
                    if (MODE == ROPE_NEIGHBOURS) c[i] = *reinterpret_cast<const uint4*>(x + at[i] + V);
                    if (MODE == ROPE_ODD) {
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const int f = at[i] + j;
                            partner[i][j] = f < p.r ? static_cast<float>(x[f < half ? f + half : f - half]) : 0.f;
                        }
                    }
                }
            }
        }
        // (a row's units are lanes of one warp: where Y is X, every partner has been read before any is written)
        if (MODE == ROPE_ODD) __syncwarp();
#pragma unroll
        for (int i = 0; i < ROPE_FLIGHT; ++i) {
            if (!out[i]) continue;
            const float *co = angles + token[i] * 2 * pad, *si = co + pad;
            float x1[V];
            unpack(a[i], x1, static_cast<const T*>(nullptr));
            if (MODE == ROPE_ODD) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int f = at[i] + j;
                    if (f < half) x1[j] = x1[j] * co[f] - partner[i][j] * si[f];
                    else if (f < p.r) x1[j] = x1[j] * co[f - half] + partner[i][j] * si[f - half];
                }
                *reinterpret_cast<uint4*>(out[i] + at[i]) = pack(x1, static_cast<const T*>(nullptr));
                continue;
            }
            float x2[V];
            unpack(c[i], x2, static_cast<const T*>(nullptr));
            if (MODE == ROPE_HALF) {
                if (at[i] < half) {
                    float y1[V], y2[V];
#pragma unroll
                    for (int j = 0; j < V; j += 4) {
                        const float4 cc = *reinterpret_cast<const float4*>(co + at[i] + j), ss = *reinterpret_cast<const float4*>(si + at[i] + j);
                        const float cv[4] = {cc.x, cc.y, cc.z, cc.w}, sv[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            y1[j + k] = x1[j + k] * cv[k] - x2[j + k] * sv[k];
                            y2[j + k] = x2[j + k] * cv[k] + x1[j + k] * sv[k];
                        }
                    }
                    *reinterpret_cast<uint4*>(out[i] + at[i]) = pack(y1, static_cast<const T*>(nullptr));
                    *reinterpret_cast<uint4*>(out[i] + at[i] + half) = pack(y2, static_cast<const T*>(nullptr));
                } else {
                    *reinterpret_cast<uint4*>(out[i] + at[i]) = a[i];
                    *reinterpret_cast<uint4*>(out[i] + at[i] + V) = c[i];
                }
            } else {
                auto rotate = [&](float& u, float& v, int pair) {
                    if (pair >= half) return;
                    const float cv = co[pair], sv = si[pair], w = u * cv - v * sv;
                    v = v * cv + u * sv;
                    u = w;
                };
#pragma unroll
                for (int j = 0; j < V; j += 2) {
                    rotate(x1[j], x1[j + 1], (at[i] + j) / 2);
                    rotate(x2[j], x2[j + 1], (at[i] + V + j) / 2);
                }
                *reinterpret_cast<uint4*>(out[i] + at[i]) = pack(x1, static_cast<const T*>(nullptr));
                *reinterpret_cast<uint4*>(out[i] + at[i] + V) = pack(x2, static_cast<const T*>(nullptr));
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
    const int pad = (p.r / 2 + 3) & ~3;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(((p.N - 1) >> p.tile_shift) + 1, p.B);
    cfg.blockDim = dim3(ROPE_THREADS);
    cfg.dynamicSmemBytes = static_cast<size_t>(2 * pad) * sizeof(float) << p.tile_shift;
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
