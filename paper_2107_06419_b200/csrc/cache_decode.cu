// Attention over the 8-bit paged cache, for few query rows per key head: decode steps and drafts (d = 64 and 128).
//
// With K = 2^ek k and V = 2^ev v (k, v: e4m3; one ek, ev a page and head), a row's output is sum_j w_j 2^ev_j v_j / sum_j w_j,
// w_j = 2^(x_j - m), x_j = (q . k_j) scale log2(e) 2^ek_j.  e4m3 numbers are exact in half precision, so they go into the warp-level
// m16n8k16 products (half in, fp32 out) as they are; the scale of the keys is one multiplication per sixteen logits' constant,
// the scale of the values is taken relative to the largest one so far and multiplied to the weights before they are rounded.
// Weights are kept as 2^15 w, which uses half precision's range: what is rounded away lies 2^39 below a row's largest weight.
//
// What bounds it: device memory, 2 d bytes a token and key head against 4 d FLOP a query row.  The rows of a unit are the queries
// of one sequence times the G query heads that share a key head, sixteen to a tile, so the cache is read once for up to sixteen rows.
// Keys (and, in the second product, features) are the rows of the products and queries their columns, so that eight rows are one
// column block; ldmatrix transposes the values' bytes.  64 sequences of 8,192 tokens, 32 query heads on 8, d = 128 (1.07 GB): 164 us,
// 6.56 TB/s, the rate of a copy; of 1,000 to 16,384 tokens (852 MB) 141 us, 6.05 TB/s, with queries as rows (twice the products for eight
// rows) 176, with conversions through the header's structures (two more instructions for two values) 215.  What is left where an
// item is short is the chain of a part -- table entry, tokens, products, join, about 3 us -- and 2 us of deal: one sequence of 2,000 tokens
// 8.8 us, 16 sequences of 2-8K with 16 heads of 64 in pages of sixteen 31.8 (4.0 TB/s).  With two row groups twelve warps an SM do not cover
// the chain of a chunk (750 instructions): 12 sequences of 4-32K, 4 key heads, 28 rows in two tiles 92 us (2.5 TB/s of the cache read
// once); those forms spill 24 to 88 bytes.
//
// Work is dealt by chunks of 8 KB (keys and values of 32 tokens, d = 128): all chunks of all (sequence, key head, row tile) in one
// row, an equal share of neighbouring chunks to each team, or, where there are few items, a part of one item each.  A team is a
// CTA (four warps, which take a part's chunks in turn and join through shared memory), or one warp where there are more items than
// warps.  An item that ends up in several teams is joined by whichever of them comes last, from their normalised outputs and
// log-sums, in the order of the keys.  Every warp keeps its own ring of chunks (cp.async, 16 bytes a lane and instruction: any page size and order, tokens
// behind the length filled with zeros), so no barrier is in the loop.
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

namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int HALF_BYTES = 4096, CHUNK_BYTES = 2 * HALF_BYTES;            // a chunk's keys, then its values
// RG: row groups of eight in a tile.  Three CTAs an SM and two chunks a warp in the ring; with two row groups that takes the queries
// out of the registers into memory that the team shares, and a team of one warp, which would need its own, has two CTAs and three chunks.
// (Four row groups: 48 items of 28 rows 98 us, in two tiles of sixteen 100; 1,100 instructions a chunk are too long a chain for
// eight warps an SM.)
constexpr int TILE = 16;
__host__ __device__ constexpr bool SHARED_Q(int RG, int TEAM) { return RG == 2 && TEAM > 1; }
__host__ __device__ constexpr int CTAS(int RG, int TEAM) { return RG == 1 || SHARED_Q(RG, TEAM) ? 3 : 2; }
__host__ __device__ constexpr int STAGES(int RG, int TEAM) { return CTAS(RG, TEAM) == 3 ? 2 : 3; }
__host__ __device__ constexpr int SMEM_BYTES(int D, int RG, int TEAM) { return WARPS * STAGES(RG, TEAM) * CHUNK_BYTES + (SHARED_Q(RG, TEAM) ? RG * D * 16 : 0); }
constexpr int ALIGN_COST = 5;                                             // chunks
// Aligned parts have at least this many chunks, one a warp; of a long item more: its parts are joined one after the other, sixteen in
// flight (0.03 us each), a warp's chunk takes 0.6 us, so P parts of n chunks take about n / (4 P) 0.6 + 0.03 P us, least at P = sqrt(5 n).
__device__ __forceinline__ unsigned least_part(unsigned n) { return max(WARPS, static_cast<int>(sqrtf(0.2f * n)) + 1); }
constexpr float WEIGHT_SHIFT = 15.f;                                      // weights are kept as 2^15 w

struct DecodeArgs {
    CacheView c;
    const __nv_bfloat16* Q;
    __nv_bfloat16* O;
    float* lse;
    long long q_st, q_sh, o_st, o_sh, total;
    int Hq, G, max_new, most_rows, causal;               // sequences with more than most_rows rows are not this kernel's
    int beside;                                          // launched behind the other kernel of the same call
    float scale_log2e;
    int* counters;                                       // [teams], 0 between launches
    float* part_lse;                                     // [2 teams][16], base 2
    float* part_o;                                       // [2 teams][16][D]
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool take) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_groups() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void lds16(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Two 16 x 16 matrices of bytes (lane i: the address of row i % 16 of matrix i / 16), transposed: r[2 y] holds column g, rows 4 t .. + 3
// of matrix y, r[2 y + 1] column g + 8 (g = lane / 4, t = lane % 4).
__device__ __forceinline__ void ldsm_bytes(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// c (16 x 8) += a (16 x 16) b (16 x 8), half precision in
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four e4m3 as two pairs of half-precision numbers.
__device__ __forceinline__ void halves(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void sts16(uint32_t addr, const uint32_t (&r)[4]) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
// The 8 x 8 matrix of half-precision pairs (lane: row lane / 4, columns 2 (lane % 4), + 1), transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// Over the lanes of the same lane % 4.
__device__ __forceinline__ float column_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
}
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 4);
    v += __shfl_xor_sync(0xffffffffu, v, 8);
    return v + __shfl_xor_sync(0xffffffffu, v, 16);
}
__device__ __forceinline__ float two_to(int e) {         // 2^e for any e: 0 below, the largest power above
    e = e < -127 ? -127 : e > 127 ? 127 : e;
    return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// The values of the keys key0 .. key1 - 1 that are NaN, for each row (of `rows`, from row0 of the sequence's on) that sees the key, by a warp: store(row,
// feature).  Key j is seen from token j - before on.
template <int D, typename Store>
__device__ __noinline__ void put_nan(const CacheView& cv, const int32_t* table, int h, int key0, int key1, int before, int row0, int rows, int G, Store store) {
    const int at = (threadIdx.x & 31) * 4;               // the lane's four features
    for (int key = key0; key < key1 && at < D; ++key) {
        const int id = table[key >> cv.page_shift];
        if (id < 0 || id >= cv.num_pages) continue;
        const int64_t token = ((static_cast<int64_t>(id) * cv.Hkv + h) << cv.page_shift) + (key & (cv.page - 1));
        const uint32_t gone = nan_bytes(*reinterpret_cast<const uint32_t*>(cv.v + token * D + at));
        if (!gone) continue;
        for (int row = 0; row < rows; ++row)
            if ((row0 + row) / G >= key - before)
                for (int e = 0; e < 4; ++e)
                    if (gone >> (8 * e) & 1) store(row, at + e);
    }
}

// TEAM: warps of a team (4 or 1).  RG: row groups of eight in a tile (1: no sequence has more than eight rows).  SMALL: pages of less
// than a chunk.  DRAFTS: rows may see fewer keys than their sequence has (without what that takes, one sequence of 2,000 tokens 8.8 us, with it
// 9.1; only one row group has both forms).
template <int D, int RG, int TEAM, bool SMALL, bool DRAFTS>
__global__ void __launch_bounds__(THREADS, CTAS(RG, TEAM))
cache_decode_kernel(const __grid_constant__ DecodeArgs p) {
    constexpr int CH = HALF_BYTES / D;                   // tokens of a chunk: 32 (d = 128) or 64
    constexpr int PIECES = D / 16, RPI = 32 / PIECES;    // 16-byte pieces of a row; rows that a copy instruction brings
    constexpr int NT = CH / 16;                          // logit blocks of sixteen keys
    constexpr int STAGES = flat::STAGES(RG, TEAM);
    constexpr bool SHARED_Q = flat::SHARED_Q(RG, TEAM);
    constexpr int JOIN = D + 4;                          // floats from row to row where the warps join: eight lanes' rows in eight banks' distance
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ float warp_lse[WARPS][TILE];
    __shared__ int last_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int member = TEAM == 1 ? 0 : warp;             // the warp's place in its team
    const unsigned team = TEAM == 1 ? blockIdx.x * WARPS + warp : blockIdx.x, teams = TEAM == 1 ? gridDim.x * WARPS : gridDim.x;
    const CacheView& cv = p.c;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // Behind the call's other kernel (cache_prefill.cu), which starts this one after it has waited for what was before and works on other rows:
    // the two run side by side, and this one waits for it at its end, so that what comes behind this one comes behind both.
    if (!p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");

    // ---------------------------------------------------------------- the deal: by every warp for itself, a lane a few sequences
    // (counts of chunks fit 32 bits: the host sees to it)
    auto shape = [&](int s, Span& sp, int& nch, int& tiles) {             // chunks of all items of a sequence
        nch = tiles = 0;
        if (!read_span(cv, s, p.total, p.max_new, sp) || sp.n == 0) return 0u;
        const int64_t rows = static_cast<int64_t>(sp.n) * p.G;
        if (rows > p.most_rows) return 0u;
        tiles = (static_cast<int>(rows) + TILE - 1) / TILE;
        nch = (sp.len + CH - 1) / CH;
        return static_cast<unsigned>(nch) * tiles * cv.Hkv;
    };
    const int per = (cv.num_seqs + 31) / 32, s_begin = lane * per, s_end = min(s_begin + per, cv.num_seqs);
    int nch = 0, tiles = 0;
    Span sp{0, 0, 0};
    unsigned units = 0, items = 0;
#pragma unroll 4
    for (int s = s_begin; s < s_end; ++s) {
        units += shape(s, sp, nch, tiles);
        items += tiles * cv.Hkv;
    }
    // (up to 32 sequences: a lane keeps its one, and what the warp needs of any of them comes by shuffle)
    const Span own = sp;
    const int own_nch = nch, own_tiles = tiles;
    auto fetch = [&](int s) {                            // chunks of all items of sequence s; sp, nch, tiles
        if (per > 1) return shape(s, sp, nch, tiles);
        sp = Span{__shfl_sync(0xffffffffu, own.q0, s), __shfl_sync(0xffffffffu, own.n, s), __shfl_sync(0xffffffffu, own.len, s)};
        nch = __shfl_sync(0xffffffffu, own_nch, s);
        tiles = __shfl_sync(0xffffffffu, own_tiles, s);
        return static_cast<unsigned>(nch) * tiles * cv.Hkv;
    };
    const unsigned chunks_all = __reduce_add_sync(0xffffffffu, units);
    // An equal share of the chunks each.  Where there are less than half as many items as teams, and it costs no team more than ALIGN_COST
    // chunks, every team has a part of one item instead, and an item's parts are alike: a team that goes from one item to the next
    // pays for two (about as long as ALIGN_COST chunks).
    unsigned share = (chunks_all + teams - 1) / teams;
    unsigned aligned = 0;                                // chunks of a part, at least
    auto pieces = [&](unsigned n) {                      // parts of an item of n chunks
        const unsigned c = max(aligned, least_part(n));
        return (n + c - 1) / c;
    };
    auto units_of = [&](unsigned chunks) { return TEAM > 1 && aligned ? tiles * cv.Hkv * pieces(nch) : chunks; };
    if (TEAM > 1) {
        const unsigned items_all = __reduce_add_sync(0xffffffffu, items);
        if (2 * items_all <= teams) {
            const unsigned c = (chunks_all + teams - items_all - 1) / (teams - items_all);
            if (c <= share + ALIGN_COST) aligned = c;
        }
        if (aligned) {
            share = 1;
            units = 0;
            if (per == 1) units = units_of(0);           // (the lane's own)
            else for (int s = s_begin; s < s_end; ++s) units += units_of(shape(s, sp, nch, tiles));
        }
    }
    unsigned upto = units;                               // units of this lane's sequences and those before
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    const unsigned all = __shfl_sync(0xffffffffu, upto, 31);
    unsigned pos = team * share;
    const unsigned begin = pos, end = min(pos + share, all);
    if (TEAM > 1 && pos >= end) {                        // (the whole CTA)
        if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
        return;
    }
    // the sequence of the first unit: the first lane whose sequences reach beyond it has it
    const int from = __ffs(__ballot_sync(0xffffffffu, upto > pos)) - 1;
    int s = from * per;
    unsigned base = __shfl_sync(0xffffffffu, upto - units, from < 0 ? 0 : from);
    if (pos < end) units = units_of(fetch(s));            // from here on: of sequence s, which begins with unit `base`

    const uint32_t ring = ptx::smem_u32(smem) + warp * STAGES * CHUNK_BYTES;
    const int page_mask = cv.page - 1, slots = SMALL ? CH >> cv.page_shift : 1;
    // ldmatrix row of the lane: sixteen keys of piece x, of piece x + 1
    const int vrow = lane & 15, vpiece = lane >> 4;
    // copies: the lane's place in 512 bytes (RPI rows), keys' pieces of odd rows changed by four, values' by the row
    const int crow = lane / PIECES, piece = lane % PIECES;
    // logits: rows g and g + 8 of a block of sixteen keys are the keys krow and krow + 2, so that the weights that a lane holds as
    // the right operand (rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9) are those of the keys 4 t .. 4 t + 3
    const int krow = 4 * (g >> 1) + (g & 1);

    while (pos < end) {
        while (pos >= base + units) { base += units; ++s; units = units_of(fetch(s)); }
        const unsigned rel = pos - base;
        // the item, its chunks a0 .. a1 - 1 that are this part, its parts and the team that has the first of them
        const unsigned of = TEAM > 1 && aligned ? pieces(nch) : nch;      // units of an item
        const unsigned item = of == 1 ? rel : rel / of, item_begin = base + item * of, at = rel - item * of;
        int a0 = at, a1 = min(at + end - pos, static_cast<unsigned>(nch));
        if (TEAM > 1 && aligned) {
            const int each = (nch + of - 1) / of;
            a0 = min(static_cast<int>(at) * each, nch);
            a1 = min(a0 + each, nch);
        }
        const unsigned first_team = share == 1 ? item_begin : item_begin / share;
        const int parts = share == 1 ? of : (item_begin + of - 1) / share - first_team + 1;
        const int64_t slot = 2 * team + (pos == begin ? 0 : 1);
        const int h = tiles == 1 ? item : item / tiles, tile = item - h * tiles;
        const int rows = min(sp.n * p.G - tile * TILE, TILE);
        // of the item's row: its token and its head of the group
        auto place_of = [&](int row, int& tok, int& gh) {
            const int flat = tile * TILE + row;
            tok = sp.n == 1 ? 0 : flat / p.G;
            gh = flat - tok * p.G;
        };

        // ------------------------------------------------------------ copies
        const int count = a1 - a0 - member <= 0 ? 0 : (a1 - a0 - member + TEAM - 1) / TEAM;     // this warp's chunks
        const int pages = (sp.len + page_mask) >> cv.page_shift;
        const int32_t* table = cv.table + static_cast<int64_t>(s) * cv.max_pages;
        // Of the k-th chunk: page * heads + head; -1: no page.  SMALL: lane j that of the j-th slot; otherwise every lane the same.
        auto load_place = [&](int k) {
            const int index = ((a0 + member + k * TEAM) * CH >> cv.page_shift) + (SMALL ? lane : 0);
            if (k >= count || index >= pages || (SMALL && lane >= slots)) return -1;
            const int id = table[index];
            if (id < 0 || id >= cv.num_pages) {
                if (cv.status) atomicExch(cv.status, FLAT_CACHE_BAD_PAGE);
                return -1;
            }
            return id * cv.Hkv + h;
        };
        auto issue = [&](int k, int place) {
            if (k < count) {
                const int st = k % STAGES, key0 = (a0 + member + k * TEAM) * CH;
                const int64_t off = (static_cast<int64_t>(place < 0 ? 0 : place) << cv.page_shift) * D + lane * 16;
                const uint32_t dst = ring + st * CHUNK_BYTES + crow * D;
                const bool full = key0 + CH <= sp.len && (SMALL ? __all_sync(0xffffffffu, place >= 0 || lane >= slots) : place >= 0);
                // sixteen tokens of a page and head are contiguous: a pointer for them, 512 bytes a copy instruction
#pragma unroll
                for (int u = 0; u < CH / 16; ++u) {
                    int64_t o = off;
                    bool there = place >= 0;
                    if (SMALL) {
                        const int slot = (u * 16) >> cv.page_shift;
                        o = __shfl_sync(0xffffffffu, off - lane * 16, slot) + lane * 16;
                        there = __shfl_sync(0xffffffffu, place, slot) >= 0;
                    }
                    o += ((key0 + 16 * u) & page_mask) * D;
                    const uint8_t *ks = cv.k + o, *vs = cv.v + o;
#pragma unroll
                    for (int i = 0; i < 16 / RPI; ++i) {
                        const int row = u * 16 + i * RPI;        // (of lane 0's piece)
                        const int kp = D == 128 ? piece ^ ((crow & 1) << 2) : piece, vp = D == 128 ? piece ^ ((row + crow) & 7) : piece ^ ((crow >> 1) & 3);
                        const uint32_t kd = dst + row * D + kp * 16, vd = dst + HALF_BYTES + row * D + vp * 16;
                        if (full) {
                            copy16(kd, ks + i * 512);
                            copy16(vd, vs + i * 512);
                        } else {
                            const bool take = there && key0 + row + crow < sp.len;
                            copy16(kd, ks + i * 512, take);
                            copy16(vd, vs + i * 512, take);
                        }
                    }
                }
            }
            commit();
        };
        auto load_exps = [&](int place, int& ek, int& ev) {
            ek = ev = 0;
            if (place >= 0) {
                ek = cv.k_exp[place];
                ev = cv.v_exp[place];
            }
        };
        int place[STAGES];                               // of the chunk at hand and those in the ring behind it
        place[0] = load_place(0);
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) {
            place[k + 1] = load_place(k + 1);
            issue(k, place[k]);
        }
        int ek_next, ev_next;
        load_exps(place[0], ek_next, ev_next);

        // ------------------------------------------------------------ queries: half precision, a power of two taken out of each row
        // Slice 4 x + w of the contraction: a lane's features 16 (t + 4 x) + 4 w .. + 3, the ones that it reads of a key
        uint32_t qb[SHARED_Q ? 1 : D / 16][RG][2];
        const uint32_t queries = ptx::smem_u32(smem) + WARPS * STAGES * CHUNK_BYTES + lane * 8;      // (SHARED_Q) [slice][row group][lane]
        float unit[RG][2];                               // of the rows 8 r + 2 t, + 1: logits' scale, keys that they see
        int nrow[RG][2];
#pragma unroll
        for (int r = 0; r < RG; ++r) {
            const int row = g + 8 * r;
            int tok, gh;
            place_of(row, tok, gh);
            uint4 raw[D / 64][2];
            float top = 0.f;
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    raw[x][e] = make_uint4(0, 0, 0, 0);
                    if (row < rows)
                        raw[x][e] = reinterpret_cast<const uint4*>(p.Q + (sp.q0 + tok) * p.q_st + (static_cast<long long>(h) * p.G + gh) * p.q_sh + 16 * (t + 4 * x))[e];
                    const uint32_t w[4] = {raw[x][e].x, raw[x][e].y, raw[x][e].z, raw[x][e].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
                }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;          // the row's largest: 2^e to 2^(e + 1)
            e = e < -100 ? -100 : e;
            const float up = two_to(14 - e), down = p.scale_log2e * two_to(e - 14);
            const long long lim = static_cast<long long>(tok) + 1 + sp.len - sp.n;
            const int seen = row < rows ? (p.causal && lim < sp.len ? static_cast<int>(lim) : sp.len) : 0;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                unit[r][y] = __shfl_sync(0xffffffffu, down, 4 * (2 * t + y));
                nrow[r][y] = __shfl_sync(0xffffffffu, seen, 4 * (2 * t + y));
            }
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint4& v = raw[x][w >> 1];
                    const uint32_t lo = w & 1 ? v.z : v.x, hi = w & 1 ? v.w : v.y;
                    const uint32_t q0 = pack_half2(__uint_as_float(lo << 16) * up, __uint_as_float(lo & 0xffff0000u) * up);
                    const uint32_t q1 = pack_half2(__uint_as_float(hi << 16) * up, __uint_as_float(hi & 0xffff0000u) * up);
                    if (!SHARED_Q) {
                        qb[SHARED_Q ? 0 : 4 * x + w][r][0] = q0;
                        qb[SHARED_Q ? 0 : 4 * x + w][r][1] = q1;
                    } else if (warp == w) {              // (every warp has them, each leaves a quarter)
                        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(queries + ((4 * x + w) * RG + r) * 256), "r"(q0), "r"(q1) : "memory");
                    }
                }
        }
        if (SHARED_Q) __syncthreads();
        int tok0, gh0;
        place_of(0, tok0, gh0);
        const long long lim0 = static_cast<long long>(tok0) + 1 + sp.len - sp.n;     // keys that every row sees
        const int nmin = p.causal && lim0 < sp.len ? static_cast<int>(lim0) : sp.len;

        // ------------------------------------------------------------ the chunks
        // o[x][r]: features 16 x + g (0, 1) and 16 x + g + 8 (2, 3) of the rows 8 r + 2 t and 8 r + 2 t + 1
        float o[PIECES][RG][4], m[RG][2], l[RG][2];
        int E = -1000;                                   // o is in units of 2^E
        bool cleaned = false;                            // values that are NaN and not for every row have been taken out (the same in all lanes)
#pragma unroll
        for (int r = 0; r < RG; ++r) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][r][e] = 0.f;
            m[r][0] = m[r][1] = -INFINITY;
            l[r][0] = l[r][1] = 0.f;
        }
        for (int k = 0; k < count; ++k) {
            const int st = k % STAGES, key0 = (a0 + member + k * TEAM) * CH;
            wait_groups<STAGES - 2>();
            __syncwarp();
            // bit j: slot j has no page
            const int bad = SMALL ? __ballot_sync(0xffffffffu, lane < slots && place[0] < 0) : place[0] < 0;
            const int ek = ek_next, ev = ev_next;
            issue(k + STAGES - 1, place[STAGES - 1]);    // (into the stage that every lane had read before this chunk's barrier)
            load_exps(place[1], ek_next, ev_next);
#pragma unroll
            for (int i = 0; i < STAGES - 1; ++i) place[i] = place[i + 1];
            place[STAGES - 1] = load_place(k + STAGES);
            const uint32_t ks = ring + st * CHUNK_BYTES, vs = ks + HALF_BYTES;
            // A weight of 0 would not keep the NaN of a value from a row that does not see it: out they go where some row does not, and
            // into the outputs of those that do at the end.  (Drafts, one or two chunks of an item.)
            if (DRAFTS && nmin < sp.len && key0 + CH > nmin) {
                bool found = false;
#pragma unroll 1
                for (int i = lane; i < HALF_BYTES / 16; i += 32) {
                    if (key0 + i / PIECES < nmin) continue;
                    uint32_t w[4], any = 0;
                    lds16(vs + i * 16, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t gone = nan_bytes(w[e]);
                        any |= gone;
                        w[e] &= ~gone;
                    }
                    if (any) {
                        sts16(vs + i * 16, w);
                        found = true;
                    }
                }
                if (__any_sync(0xffffffffu, found)) cleaned = true;
                __syncwarp();
            }
            // base-2 logits; keys that a row does not see take no part
            const bool masked = key0 + CH > nmin || bad != 0;
            float uk[NT], wv[NT];                        // of sixteen keys: their scale; what their weights are multiplied by for their values' scale
            int evs[NT], e_top = -1000;
            const float ek_scale = two_to(ek - 127);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                uk[i] = SMALL ? __shfl_sync(0xffffffffu, ek_scale, (i * 16) >> cv.page_shift) : ek_scale;
                evs[i] = SMALL ? __shfl_sync(0xffffffffu, ev, (i * 16) >> cv.page_shift) : ev;
                e_top = max(e_top, evs[i]);
            }
            if (e_top > E) {
                const float down = E < -500 ? 0.f : two_to(E - e_top);
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
#pragma unroll
                    for (int r = 0; r < RG; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[i][r][e] *= down;
                E = e_top;
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) wv[i] = two_to(evs[i] - E);
            // logits, keys as rows: c[i][r]: keys 16 i + krow (0, 1) and 16 i + krow + 2 (2, 3) of the rows 8 r + 2 t and 8 r + 2 t + 1
            float c[NT][RG][4];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int r = 0; r < RG; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[i][r][e] = 0.f;
            if (SHARED_Q) {                              // slice by slice: its queries serve all blocks
#pragma unroll
                for (int x = 0; x < D / 64; ++x) {
                    uint32_t w[NT][4], v[NT][4];
                    const int at = (D == 128 ? (t + 4 * x) ^ ((krow & 1) << 2) : t) * 16;
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        lds16(ks + (i * 16 + krow) * D + at, w[i]);
                        lds16(ks + (i * 16 + krow + 2) * D + at, v[i]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t q[RG][2];
#pragma unroll
                        for (int r = 0; r < RG; ++r)
                            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(q[r][0]), "=r"(q[r][1]) : "r"(queries + ((4 * x + e) * RG + r) * 256));
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            uint32_t a[4];
                            halves(w[i][e], a[0], a[2]);
                            halves(v[i][e], a[1], a[3]);
#pragma unroll
                            for (int r = 0; r < RG; ++r) mma16(c[i][r], a, q[r][0], q[r][1]);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const uint32_t row = ks + (i * 16 + krow) * D;
#pragma unroll
                    for (int x = 0; x < D / 64; ++x) {
                        uint32_t w[4], v[4];
                        const int at = (D == 128 ? (t + 4 * x) ^ ((krow & 1) << 2) : t) * 16;
                        lds16(row + at, w);
                        lds16(row + 2 * D + at, v);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t a[4];
                            halves(w[e], a[0], a[2]);
                            halves(v[e], a[1], a[3]);
#pragma unroll
                            for (int r = 0; r < RG; ++r) mma16(c[i][r], a, qb[SHARED_Q ? 0 : 4 * x + e][r][0], qb[SHARED_Q ? 0 : 4 * x + e][r][1]);
                        }
                    }
                }
            }
            bool grown = false;
            float mx[RG][2];
#pragma unroll
            for (int r = 0; r < RG; ++r) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const float u = unit[r][y] * uk[i];
                        c[i][r][y] *= u;
                        c[i][r][2 + y] *= u;
                    }
                if (masked) {
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const int key = key0 + i * 16 + krow;
                        const bool gone = bad >> (SMALL ? (i * 16) >> cv.page_shift : 0) & 1;
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            if (gone || key >= nrow[r][y]) c[i][r][y] = -INFINITY;
                            if (gone || key + 2 >= nrow[r][y]) c[i][r][2 + y] = -INFINITY;
                        }
                    }
                }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    mx[r][y] = fmaxf(c[0][r][y], c[0][r][2 + y]);
#pragma unroll
                    for (int i = 1; i < NT; ++i) mx[r][y] = tc::max3(mx[r][y], c[i][r][y], c[i][r][2 + y]);
                    grown = grown || mx[r][y] > m[r][y];
                }
            }
            // (the maximum is taken over the lanes only where one of them has met a larger logit)
            if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int r = 0; r < RG; ++r) {
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float mn = fmaxf(m[r][y], column_max(mx[r][y]));
                        const float a = mn == -INFINITY ? 1.f : tc::ex2_approx(m[r][y] - mn);
                        m[r][y] = mn;
                        l[r][y] *= a;
#pragma unroll
                        for (int i = 0; i < PIECES; ++i) { o[i][r][y] *= a; o[i][r][2 + y] *= a; }
                    }
                }
            }
            uint32_t pb[NT][RG][2];                 // weights as the right operand
#pragma unroll
            for (int r = 0; r < RG; ++r) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float ref = m[r][y] == -INFINITY ? 0.f : m[r][y] - WEIGHT_SHIFT;
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float w = tc::ex2_approx(c[i][r][2 * e + y] - ref);
                            l[r][y] += w;
                            c[i][r][2 * e + y] = w * wv[i];
                        }
                }
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    pb[i][r][0] = transpose8(pack_half2(c[i][r][0], c[i][r][1]));
                    pb[i][r][1] = transpose8(pack_half2(c[i][r][2], c[i][r][3]));
                }
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int row = i * 16 + vrow;
#pragma unroll
                for (int x = 0; x < PIECES; x += 2) {
                    const int piece = x + vpiece;
                    uint32_t b[4];
                    ldsm_bytes(vs + row * D + (D == 128 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3)) * 16, b);
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        uint32_t a[4];               // rows g, g + 8: features 16 (x + y) + g, + 8
                        halves(b[2 * y], a[0], a[2]);
                        halves(b[2 * y + 1], a[1], a[3]);
#pragma unroll
                        for (int r = 0; r < RG; ++r) {
                            mma16(o[x + y][r], a, pb[i][r][0], pb[i][r][1]);
                        }
                    }
                }
            }
        }
        wait_groups<0>();

        // ------------------------------------------------------------ normalised outputs and log-sums of this warp's keys
        float lg[RG][2];
        const float scale = two_to(E - 127);             // (multiplied by itself: over the sum it could lie below the least normal number)
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const float sum = column_sum(l[r][y]), inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
                lg[r][y] = sum > 0.f ? m[r][y] - WEIGHT_SHIFT + log2f(sum) : sum == sum ? -INFINITY : sum;
#pragma unroll
                for (int i = 0; i < PIECES; ++i) { o[i][r][y] = o[i][r][y] * inv * scale; o[i][r][2 + y] = o[i][r][2 + y] * inv * scale; }
            }
        const bool whole = parts == 1;
        auto finish = [&](int row, int col, float4 v, float lse2) {     // four features of the item's row
            int tok, gh;
            place_of(row, tok, gh);
            const int head = h * p.G + gh;
            uint2 w;
            w.x = tc::pack_bf16x2(v.x, v.y);
            w.y = tc::pack_bf16x2(v.z, v.w);
            *reinterpret_cast<uint2*>(p.O + (sp.q0 + tok) * p.o_st + head * p.o_sh + col) = w;
            if (p.lse && col == 0) p.lse[static_cast<long long>(sp.q0 + tok) * p.Hq + head] = lse2 * 0.6931471805599453f;
        };
        auto put_cleaned = [&](auto store) {             // the NaN that were taken out of this warp's chunks, into what it has written
            __syncwarp();
            for (int k = 0; k < count; ++k) {
                const int key0 = (a0 + member + k * TEAM) * CH;
                put_nan<D>(cv, table, h, max(key0, nmin), min(key0 + CH, sp.len), sp.len - sp.n, tile * TILE, rows, p.G, store);
            }
        };
        if (TEAM == 1) {
#pragma unroll
            for (int r = 0; r < RG; ++r)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int row = 8 * r + 2 * t + y;
                    if (row >= rows) continue;
                    int tok, gh;
                    place_of(row, tok, gh);
                    const int head = h * p.G + gh;
                    __nv_bfloat16* out = p.O + (sp.q0 + tok) * p.o_st + head * p.o_sh + g;
                    float* part = p.part_o + (slot * TILE + row) * D + g;
#pragma unroll
                    for (int x = 0; x < PIECES; ++x)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            if (whole) out[16 * x + 8 * e] = __float2bfloat16(o[x][r][2 * e + y]);
                            else part[16 * x + 8 * e] = o[x][r][2 * e + y];
                        }
                    if (g == 0 && !whole) p.part_lse[slot * TILE + row] = lg[r][y];
                    if (g == 0 && whole && p.lse) p.lse[static_cast<long long>(sp.q0 + tok) * p.Hq + head] = lg[r][y] * 0.6931471805599453f;
                }
            if (cleaned && whole)
                put_cleaned([out = p.O + sp.q0 * p.o_st + h * p.G * p.o_sh, o_st = p.o_st, o_sh = p.o_sh, G = p.G, row0 = tile * TILE](int row, int feature) {
                    const int tok = (row0 + row) / G;
                    out[tok * o_st + (row0 + row - tok * G) * o_sh + feature] = __ushort_as_bfloat16(0x7fff);
                });
            else if (cleaned) put_cleaned([out = p.part_o + slot * TILE * D](int row, int feature) { out[row * D + feature] = __int_as_float(0x7fffffff); });
        } else {
            // the team's warps join through the memory of their rings
            __syncthreads();
            float* joined = reinterpret_cast<float*>(smem);                // [warp][row][JOIN]
#pragma unroll
            for (int r = 0; r < RG; ++r)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int row = 8 * r + 2 * t + y;
#pragma unroll
                    for (int x = 0; x < PIECES; ++x) {
                        joined[(warp * 8 * RG + row) * JOIN + 16 * x + g] = o[x][r][y];
                        joined[(warp * 8 * RG + row) * JOIN + 16 * x + 8 + g] = o[x][r][2 + y];
                    }
                    if (g == 0) warp_lse[warp][row] = lg[r][y];
                }
            if (cleaned) put_cleaned([out = joined + warp * 8 * RG * JOIN](int row, int feature) { out[row * JOIN + feature] = __int_as_float(0x7fffffff); });
            __syncthreads();
            for (int i = threadIdx.x; i < rows * (D / 4); i += THREADS) {
                const int row = i / (D / 4), col = i % (D / 4) * 4;
                float top = -INFINITY, sum = 0.f;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < WARPS; ++w) top = fmaxf(top, warp_lse[w][row]);
                const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) {
                    const float a = tc::ex2_approx(warp_lse[w][row] - ref);
                    const float4 x = *reinterpret_cast<const float4*>(joined + (w * 8 * RG + row) * JOIN + col);
                    sum += a;
                    v.x += a * x.x; v.y += a * x.y; v.z += a * x.z; v.w += a * x.w;
                }
                const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum, lse2 = sum > 0.f ? ref + log2f(sum) : sum == sum ? -INFINITY : sum;
                v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
                if (whole) finish(row, col, v, lse2);
                else {
                    *reinterpret_cast<float4*>(p.part_o + (slot * TILE + row) * D + col) = v;
                    if (col == 0) p.part_lse[slot * TILE + row] = lse2;
                }
            }
        }
        // ------------------------------------------------------------ an item in several teams: the last one joins its parts
        if (!whole) {
            // (one thread's fences, with the barriers on either side, order what all of them have written and will read)
            bool mine;
            auto arrive = [&] {
                __threadfence();
                const bool last = atomicAdd(p.counters + first_team, 1) == parts - 1;
                __threadfence();
                return last;
            };
            if (TEAM == 1) {
                __syncwarp();
                int last = 0;
                if (lane == 0) last = arrive();
                mine = __shfl_sync(0xffffffffu, last, 0);
                __syncwarp();
            } else {
                __syncthreads();
                if (threadIdx.x == 0) last_word = arrive();
                __syncthreads();
                mine = last_word;
            }
            if (mine) {
                const int64_t slot0 = 2 * static_cast<int64_t>(first_team) + (item_begin == first_team * share ? 0 : 1);
                for (int i = TEAM == 1 ? lane : threadIdx.x; i < rows * (D / 4); i += 32 * TEAM) {
                    const int row = i / (D / 4), col = i % (D / 4) * 4;
                    float ref = -INFINITY, sum = 0.f;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    constexpr int BATCH = 16;            // (parts in flight: each costs a way to L2 and back)
                    for (int j0 = 0; j0 < parts; j0 += BATCH) {
                        float lj[BATCH];
                        float4 x[BATCH];
                        float top = ref;
#pragma unroll
                        for (int j = 0; j < BATCH; ++j) {
                            lj[j] = -INFINITY;
                            x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (j0 + j < parts) {
                                const int64_t q = j0 + j == 0 ? slot0 : 2 * static_cast<int64_t>(first_team + j0 + j);
                                lj[j] = __ldcg(p.part_lse + q * TILE + row);
                                x[j] = __ldcg(reinterpret_cast<const float4*>(p.part_o + (q * TILE + row) * D + col));
                            }
                        }
#pragma unroll
                        for (int j = 0; j < BATCH; ++j) top = fmaxf(top, lj[j]);
                        const float use = top == -INFINITY ? 0.f : top;
                        const float a0_ = tc::ex2_approx(ref - use);
                        ref = top;
                        sum *= a0_;
                        v.x *= a0_; v.y *= a0_; v.z *= a0_; v.w *= a0_;
#pragma unroll
                        for (int j = 0; j < BATCH; ++j) {
                            const float a = tc::ex2_approx(lj[j] - use);
                            sum += a;
                            v.x += a * x[j].x; v.y += a * x[j].y; v.z += a * x[j].z; v.w += a * x[j].w;
                        }
                    }
                    const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
                    v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
                    finish(row, col, v, sum > 0.f ? (ref == -INFINITY ? 0.f : ref) + log2f(sum) : sum == sum ? -INFINITY : sum);
                }
                if (TEAM == 1 ? lane == 0 : threadIdx.x == 0) p.counters[first_team] = 0;
            }
        }
        if (TEAM > 1) __syncthreads();                   // (the rings' memory is free again)
        pos += TEAM > 1 && aligned ? 1 : a1 - a0;
    }
    if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

}  // namespace

namespace {
size_t most_teams() { return static_cast<size_t>(device_sm_count()) * 3 * WARPS; }     // (three CTAs an SM, a team a warp)
size_t most_part_rows() { return static_cast<size_t>(device_sm_count()) * 3 * WARPS * 2 * TILE; }    // (two places a team)

template <int D, int RG, int TEAM, bool SMALL, bool DRAFTS>
int launch(const DecodeArgs& p, cudaStream_t st) {
    if (!ensure_dynamic_smem<cache_decode_kernel<D, RG, TEAM, SMALL, DRAFTS>>(SMEM_BYTES(D, RG, TEAM))) return FLAT_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(device_sm_count() * CTAS(RG, TEAM));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_BYTES(D, RG, TEAM);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cache_decode_kernel<D, RG, TEAM, SMALL, DRAFTS>, p) == cudaSuccess ? FLAT_OK : FLAT_ERR_CUDA;
}
template <int D, int RG, bool DRAFTS>
int launch_form(const DecodeArgs& p, bool by_warp, cudaStream_t st) {
    const bool small = p.c.page < HALF_BYTES / D;
    if (by_warp) return small ? launch<D, RG, 1, true, DRAFTS>(p, st) : launch<D, RG, 1, false, DRAFTS>(p, st);
    return small ? launch<D, RG, WARPS, true, DRAFTS>(p, st) : launch<D, RG, WARPS, false, DRAFTS>(p, st);
}
template <int D>
int launch_d(const DecodeArgs& p, int64_t most, bool by_warp, cudaStream_t st) {
    if (most > 8) return launch_form<D, 2, true>(p, by_warp, st);
    return p.causal && p.max_new > 1 ? launch_form<D, 1, true>(p, by_warp, st) : launch_form<D, 1, false>(p, by_warp, st);
}
}  // namespace

size_t cache_decode_counter_bytes() { return (most_teams() * sizeof(int) + 255) & ~size_t(255); }
size_t cache_decode_part_bytes(int d) { return (most_part_rows() * (d + 1) * sizeof(float) + 255) & ~size_t(255); }

int launch_cache_decode(const flat_attn_cache_t& c, const flat_attn_cache_fwd_params_t& q, int most_rows, bool beside, int* counters, float* parts, cudaStream_t st) {
    DecodeArgs p{};
    p.c = cache_view(c);
    p.Q = static_cast<const __nv_bfloat16*>(q.Q);
    p.O = static_cast<__nv_bfloat16*>(q.O);
    p.lse = q.lse;
    p.q_st = q.q_stride_t; p.q_sh = q.q_stride_h; p.o_st = q.o_stride_t; p.o_sh = q.o_stride_h;
    p.total = q.total;
    p.Hq = q.Hq; p.G = q.Hq / c.Hkv; p.max_new = q.max_new; p.most_rows = most_rows; p.causal = q.causal;
    p.beside = beside;
    p.scale_log2e = q.scale * 1.4426950408889634f;
    p.counters = counters;
    p.part_lse = parts;
    p.part_o = p.part_lse + most_part_rows();
    const int64_t rows = static_cast<int64_t>(q.max_new) * p.G, most = rows < most_rows ? rows : most_rows;
    const int64_t items = static_cast<int64_t>(c.num_seqs) * c.Hkv * ((most + TILE - 1) / TILE);
    const bool by_warp = items >= static_cast<int64_t>(most_teams());
    return c.d == 64 ? launch_d<64>(p, most, by_warp, st) : launch_d<128>(p, most, by_warp, st);
}

}  // namespace flat
