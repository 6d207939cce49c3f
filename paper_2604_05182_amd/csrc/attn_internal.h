// What the forward and the backward of dense attention over packed sequences share: the problem's description, where a workgroup's
// rows are, tiles in LDS and the MFMA operands read from them, the bias.  (gfx950)
#pragma once
#include "lsrm_internal.h"

#include <utility>

namespace lsrm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxBuckets = 64;
constexpr int kBiasPad = 64;             // entries on each side of a head's expanded bias that repeat its first and last one
constexpr int kMaxBiasEntries = 10240;   // of the expanded bias of a group of heads, with the repeated ones (in LDS: 40 KB)
constexpr int kMaxBiasSpan = 1022;       // last bound - first bound (the gradient's sums take up to 18 KB)

struct AttnArgs {
    const uint16_t *q, *k, *v, *bias, *dout, *o;
    uint16_t *out, *dq, *dk, *dv, *dbias;
    const float *lse_in;
    float *lse;
    const int32_t *q_off, *k_off, *q_len, *k_len;
    int64_t qs[2], ks[2], vs[2], os[2];  // {row, head} strides in elements
    int n_q, n_k, n_seq, h_q, h_kv, group, causal;
    int n_slots;           // backward: workgroups that leave sums of the bias' gradient
    int unit_cap;          // forward of few rows: units of all sequences at most
    int parts;             // parts that the walk of a workgroup is cut into
    float *part;           // forward: sums of the parts
    float2 *part_ml;       // forward of many rows: their maxima and sums of exponentials
    float2 *aux;           // backward: [h_q][n_q] {lse log2e (+inf for a query without keys), -D}, one such for each part of the dQ walks
    float *part_q, *part_k, *part_v, *part_bias;
    int n_buckets, b0, b_last;  // of the bias (0: none), first and last bound
    int tab;                    // entries of a head's expanded bias
    int32_t bounds[kMaxBuckets - 1];
    float scale, sl2;
};

// validates params; fills everything but the tensors
lsrm_status make_attn_args(const lsrm_attn_params *p, AttnArgs *a);
size_t attn_forward_ws_bytes(const AttnArgs &a, int d);
size_t attn_backward_ws_bytes(const AttnArgs &a, int d);
lsrm_status launch_attn_forward(AttnArgs a, int d, void *ws, hipStream_t st);
lsrm_status launch_attn_backward(AttnArgs a, int d, void *ws, hipStream_t st);

// A value that all lanes hold, as a scalar.  (Divisions are done by the vector unit, whose results the compiler takes for each lane's own: branches on
// them then mask lanes, and addresses for the copies to LDS must be scalars.)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// ---- where a workgroup's rows are ------------------------------------------------------------------------------------
// The query rows of a key/value head are numbered (query, head of its group), heads fastest: a tile of rows then reads a key or
// value once for all heads that share it, single queries fill a tile with their heads, and a causal tile's rows see almost
// the same keys.
struct Sequence {
    int q0, n_q, q_slot;  // first row, queries, rows of the slot
    int k0, n_k, k_slot;
    int shift;  // position of query 0
};
// (whatever the offsets and lengths hold, the rows lie in the tensors)
__device__ __forceinline__ Sequence load_sequence(const AttnArgs &a, int s) {
    const int q0 = a.q_off[s], q1 = a.q_off[s + 1], k0 = a.k_off[s], k1 = a.k_off[s + 1];
    const int q_len = a.q_len != nullptr ? a.q_len[s] : 0, k_len = a.k_len != nullptr ? a.k_len[s] : 0;
    Sequence r;
    r.q0 = min(max(q0, 0), a.n_q);
    r.q_slot = min(max(q1, r.q0), a.n_q) - r.q0;
    r.k0 = min(max(k0, 0), a.n_k);
    r.k_slot = min(max(k1, r.k0), a.n_k) - r.k0;
    r.n_q = a.q_len != nullptr ? min(max(q_len, 0), r.q_slot) : r.q_slot;
    r.n_k = a.k_len != nullptr ? min(max(k_len, 0), r.k_slot) : r.k_slot;
    r.shift = r.n_k - r.n_q;
    return r;
}

// Which tile of `bm` rows (of the keys: KEYS, else of the queries) is x?  Up to 64 sequences, a lane of the wavefront loads each and counts its
// tiles; those of the sequences that take longest come first, so that what runs last is short.  False if there are fewer tiles.
// Beyond, sequence s has the tiles from number floor(first row / bm) + s on -- room for all of its own, and nobody needs to count -- and is
// found by probing 64 places at a time; then some numbers are no tile.
__device__ __forceinline__ int tile_slot(int off, int n_rows, int mult, int bm, int s) { return min(max(off, 0), n_rows) * mult / bm + s; }
template <bool KEYS>
__device__ __forceinline__ bool find_tile(const AttnArgs &a, int mult, int bm, int x, Sequence &s, int &tile, int &seq) {
    const int lane = threadIdx.x & 63, n_rows = KEYS ? a.n_k : a.n_q;
    if (a.n_seq <= 64) {
        const Sequence mine = load_sequence(a, min(lane, a.n_seq - 1));
        const int rows = (KEYS ? mine.k_slot : mine.q_slot) * mult, tiles = lane < a.n_seq ? (rows + bm - 1) / bm : 0;
        const int work = KEYS ? mine.n_q : mine.n_k;
        int first = 0;
        for (int i = 0; i < a.n_seq; ++i) {
            const int w = __builtin_amdgcn_readlane(work, i), n = __builtin_amdgcn_readlane(tiles, i);
            first += w > work || (w == work && i < lane) ? n : 0;
        }
        const uint64_t found = __builtin_amdgcn_ballot_w64(first <= x && x < first + tiles);
        if (found == 0) return false;
        seq = __builtin_ctzll(found);
        tile = x - __builtin_amdgcn_readlane(first, seq);
        s.q0 = __builtin_amdgcn_readlane(mine.q0, seq);
        s.n_q = __builtin_amdgcn_readlane(mine.n_q, seq);
        s.q_slot = __builtin_amdgcn_readlane(mine.q_slot, seq);
        s.k0 = __builtin_amdgcn_readlane(mine.k0, seq);
        s.n_k = __builtin_amdgcn_readlane(mine.n_k, seq);
        s.k_slot = __builtin_amdgcn_readlane(mine.k_slot, seq);
        s.shift = s.n_k - s.n_q;
        return true;
    }
    const int32_t *off = KEYS ? a.k_off : a.q_off;
    int lo = 0, hi = a.n_seq;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step;
        const uint64_t below = __builtin_amdgcn_ballot_w64(i < hi && tile_slot(off[min(i, a.n_seq - 1)], n_rows, mult, bm, i) <= x);
        const int c = __builtin_ctzll(~below);  // (the last lane's place is never below hi)
        lo += c * step;
        hi = min(hi, lo + step);
    }
    seq = uniform(lo);
    tile = x - tile_slot(off[seq], n_rows, mult, bm, seq);
    s = load_sequence(a, seq);
    return tile >= 0 && (int64_t)tile * bm < (int64_t)(KEYS ? s.k_slot : s.q_slot) * mult;
}

// ---- tiles in LDS ----------------------------------------------------------------------------------------------------
// A tile is 32 rows of one head, row-major, as they are in memory; the 16-byte chunks of a row change places by a key of its row
// number, so that reads of one chunk of 16 rows (MFMA operands along the channels) and of four chunks of four rows
// (transposing reads), what the 64 banks serve at a time, have no bank twice.
template <int D>
struct AttnGeo {
    static constexpr int NS = D / 16, ND = D / 32;  // 16-channel slabs, 32-channel tiles
    static constexpr int ROW = 2 * D;               // bytes
    static constexpr int TILE = 32 * ROW;
    static constexpr int RPC = 1024 / ROW;          // rows per copy instruction
    static constexpr int COPIES = TILE / 1024;      // copy instructions per tile
    static constexpr int OUT_ROW = 2 * D + 16;      // padded row of the output staging (bytes)
};
template <int D>
__device__ __forceinline__ int row_key(int r) {
    const int low = (r >> 2) & 3;
    return D == 128 ? ((r & 3) << 2) | low : D == 64 ? (((r >> 1) & 1) << 2) | low : low;
}
// row permutation of the operand whose product becomes the next contraction's operand: bits 2 and 3 swapped
__device__ __forceinline__ int perm32(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Where this lane's 16 bytes of copy instruction i of a tile come from: row of the tile, byte in the row
template <int D>
struct CopyLane {
    int row, chunk;  // of instruction 0; the others add i * RPC rows and change two bits of the chunk (copy_flip)
    __device__ explicit CopyLane(int lane) {
        row = lane * 16 / AttnGeo<D>::ROW;
        chunk = (lane * 16 % AttnGeo<D>::ROW) / 16 ^ row_key<D>(row);
    }
};
template <int D>
__device__ __forceinline__ constexpr int copy_flip(int i) {
    return D == 128 ? i & 3 : D == 64 ? (i & 1) << 1 : 0;
}

// Copies the instructions first, first + step, ... of n rows (a multiple of 32, tiles behind each other) from src, rows stride_b bytes apart, to
// dst.  Rows from `avail` on (>= 1) are copies of row avail - 1: nothing behind a sequence's keys is ever read.
template <int D, int N, int STEP>
__device__ __forceinline__ void copy_rows(const char *src, uint32_t stride_b, int avail, const char *dst, int first, const CopyLane<D> &c) {
    using G = AttnGeo<D>;
    constexpr int N_COPY = N / G::RPC;
    avail = uniform(avail);
    if (avail >= N) {
#pragma unroll
        for (int n = 0; n < N_COPY / STEP; ++n) {
            const int i = first + n * STEP;
            copy_kb_to_lds(src + (uint64_t)(i * G::RPC) * stride_b, c.row * stride_b + ((c.chunk ^ copy_flip<D>(i)) << 4), dst + i * 1024);
        }
    } else {
#pragma unroll
        for (int n = 0; n < N_COPY / STEP; ++n) {
            const int i = first + n * STEP;
            copy_kb_to_lds(src, min(i * G::RPC + c.row, avail - 1) * stride_b + ((c.chunk ^ copy_flip<D>(i)) << 4), dst + i * 1024);
        }
    }
}

// Addresses of MFMA A operands in a tile (add the tile's own):
//   rows   fragment ks: lane (hh = lane / 32, r): row perm32(r), channels 16 ks + 8 hh + 0..7     at at[ks]
//   transp fragment (ks2, dt): lane (hh, r): channel 32 dt + r, rows 16 ks2 + 8 hh + 0..7: two transposing loads of four rows
//          (ds_read_b64_tr_b16: in each group of 16 lanes, lane j gets as element e the 16-bit element j % 4 of what lane
//          4 e + j / 4 addressed), at tr[half][dt] + 16 ks2 rows
template <int D>
struct TileLane {
    uint32_t at[AttnGeo<D>::NS], tr[2][AttnGeo<D>::ND];
    __device__ explicit TileLane(int lane) {
        using G = AttnGeo<D>;
        const int hh = lane >> 5, r = perm32(lane & 31);
#pragma unroll
        for (int x = 0; x < G::NS; ++x) at[x] = r * G::ROW + (((2 * x + hh) ^ row_key<D>(r)) << 4);
        const int s = lane & 15, half16 = (lane >> 4) & 1;
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
            for (int dt = 0; dt < G::ND; ++dt) {
                const int row = 8 * hh + 4 * h2 + (s >> 2);
                tr[h2][dt] = row * G::ROW + (((4 * dt + 2 * half16 + ((s & 3) >> 1)) ^ row_key<D>(row)) << 4) + ((s & 1) << 3);
            }
    }
};

union BFrag {
    bf16x8 v;
    uint32_t u[4];
    i32x2 h[2];
};

template <int D>
__device__ __forceinline__ bf16x8 read_row_frag(const char *tile, const TileLane<D> &t, int ks) {
    return *reinterpret_cast<const bf16x8 *>(tile + t.at[ks]);
}

// start + (rows of the tile) x b over all channels
template <int D>
__device__ __forceinline__ f32x16 mfma_rows(const f32x16 &start, const char *tile, const TileLane<D> &t, const bf16x8 (&b)[AttnGeo<D>::NS]) {
    f32x16 acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_row_frag<D>(tile, t, 0), b[0], start, 0, 0, 0);
#pragma unroll
    for (int ks = 1; ks < AttnGeo<D>::NS; ++ks)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_row_frag<D>(tile, t, ks), b[ks], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ f32x16 splat(float x) {
    f32x16 r;
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = x;
    return r;
}

// fragment (ks2, dt) of the transposed tile.  (The copies to LDS are inline assembly, so the compiler knows of none that this load would
// have to wait for.)
template <int D>
__device__ __forceinline__ bf16x8 read_tr_frag(const char *tile, const TileLane<D> &t, int ks2, int dt) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int at = ks2 * 16 * AttnGeo<D>::ROW;
    union {
        s16x4 h[2];
        bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + t.tr[0][dt] + at));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + t.tr[1][dt] + at));
    return u.v;
}
// acc[dt] += (transposed tile: channels x 32 rows) x b[ks2] for every dt and ks2
template <int D>
__device__ __forceinline__ void mfma_transposed(f32x16 (&acc)[AttnGeo<D>::ND], const char *tile, const TileLane<D> &t, const BFrag (&b)[2]) {
#pragma unroll
    for (int ks2 = 0; ks2 < 2; ++ks2)
#pragma unroll
        for (int dt = 0; dt < AttnGeo<D>::ND; ++dt)
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_tr_frag<D>(tile, t, ks2, dt), b[ks2].v, acc[dt], 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    bf16x2 p;
    p[0] = (__bf16)a;
    p[1] = (__bf16)b;
    return *reinterpret_cast<uint32_t *>(&p);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// accumulator tile -> the two B operands (16-row slabs) of the next contraction
__device__ __forceinline__ void to_b_operand(const f32x16 &x, BFrag (&b)[2]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) b[k / 4].u[k % 4] = pack_bf16(x[2 * k], x[2 * k + 1]);
}
// row of a tile that accumulator element i of a product with permuted rows belongs to
__device__ __forceinline__ int acc_row(int i, int hh) { return 16 * (i / 8) + 8 * hh + i % 8; }

// max / sum across the two lane halves (lanes i and i + 32 hold the same column)
__device__ __forceinline__ float half_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// s_waitcnt vmcnt <= n and lgkmcnt == 0; a bare barrier: who copied waits for the copies before it
constexpr int vm_lgkm_imm(int n) { return (n & 0xF) | ((n >> 4) << 14) | 0x0070; }
template <int N>
__device__ __forceinline__ void wait_copies() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(vm_lgkm_imm(N));
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wg_barrier() { asm volatile("s_barrier" ::: "memory"); }

// Results of an MFMA become readable by VALU instructions a fixed number of cycles after issue; the compiler pads, but not reliably where a
// branch lies between.  24 wait states cover the 8 passes.
__device__ __forceinline__ void mfma_settle() { asm volatile("s_nop 15\n\ts_nop 7" ::: "memory"); }

// x (transposed: channels x the 32 rows from v0 on, times mul; zeros in rows that are not live) -> bf16 rows of a tensor of query rows, through
// `stage` (32 OUT_ROW bytes of the wavefront's own), so that they are written in 16-byte pieces
template <int D>
__device__ __forceinline__ void store_query_rows(const AttnArgs &a, const Sequence &s, int head_kv, int v0, int slot_rows,
                                                 const f32x16 (&x)[AttnGeo<D>::ND], float mul, bool live, char *stage, uint16_t *dst,
                                                 const int64_t (&stride)[2], int lane) {
    using G = AttnGeo<D>;
#pragma unroll
    for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            uint2 w;
            w.x = live ? pack_bf16(x[dt][4 * gq] * mul, x[dt][4 * gq + 1] * mul) : 0;
            w.y = live ? pack_bf16(x[dt][4 * gq + 2] * mul, x[dt][4 * gq + 3] * mul) : 0;
            *reinterpret_cast<uint2 *>(stage + (lane & 31) * G::OUT_ROW + (32 * dt + 8 * gq + 4 * (lane >> 5)) * 2) = w;
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int CH = D / 8, RPP = 64 / CH;
#pragma unroll
    for (int it = 0; it < 32 / RPP; ++it) {
        const int rr = it * RPP + lane / CH, v = v0 + rr;
        if (v < slot_rows) {
            const int tok = (unsigned)v / (unsigned)a.group, g = v - tok * a.group;
            *reinterpret_cast<uint4 *>(dst + (s.q0 + tok) * stride[0] + (int64_t)(head_kv * a.group + g) * stride[1] + 8 * (lane % CH)) =
                *reinterpret_cast<const uint4 *>(stage + rr * G::OUT_ROW + (lane % CH) * 16);
        }
    }
}

// Where there are few workgroups, walks are cut into parts, of which fp32 sums are added up afterwards.  How many is a trade between walks
// that leave the chip empty and sums that are written and read; by what both take (one walk step of a wavefront: `cycles`, the chip
// full from `full` workgroups on; 3.5 bytes of sums a nanosecond, and 4 us for the launch):
//   T(parts) = steps / min(1, workgroups parts / full) + (parts > 1) (4 us + parts bytes / 3.5 TB/s)
// Always 512 workgroups instead: 32 heads of 32 on 2, 6372 tokens 450 -> 390 us a training step.
// walk: steps of an average walk (a part has four at least); grid: workgroups that are launched for each part; time: T, in us.
int best_parts(double steps, double cycles, double workgroups, double full, double bytes, int64_t walk, int64_t grid, double *time = nullptr);
// walk steps of single wavefronts (32 x 32): those of average sequences, half of them where causal
inline double walk_steps(const AttnArgs &a) {
    return (double)a.n_q * a.group * a.h_kv / 32 * a.n_k / a.n_seq / 32 * (a.causal && a.n_q == a.n_k ? 0.5 : 1.0);
}
// workgroups that fill the chip
inline int full_chip(int d) { return d == 32 ? 1024 : 512; }

template <typename F>
lsrm_status launch_attn(F kernel, int64_t grid, int threads, int lds, const AttnArgs &a, hipStream_t st) {
    // (set on every call: cheap, and right whichever device is current and whichever thread calls)
    if (lds > 64 * 1024)
        LSRM_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), lds, st, a);
    LSRM_HIP_CHECK(hipGetLastError());
    return LSRM_OK;
}

// ---- the bias --------------------------------------------------------------------------------------------------------
// The bias of one key/value head's query heads, expanded by distance, times log2e: entry x of a head is for the distance
// b0 - 1 - kBiasPad + x.  What a tile of 32 queries and 32 keys looks up lies within the entries unless all its distances are before the first or
// from the last bound on (then one bucket serves the tile): a lane's entries are at fixed places around one address, with no
// clamping of single distances.  -1e30 and below mask their bucket.
// In LDS behind the expanded entries: the bounds and the group's bias as it is.  Every thread of the workgroup takes part; nobody may read
// before the next barrier.
inline int bias_lds_floats(const AttnArgs &a) { return a.n_buckets > 0 ? a.group * a.tab + kMaxBuckets + a.group * a.n_buckets : 0; }
__device__ __forceinline__ void expand_bias(const AttnArgs &a, int head_kv, float *tab, int threads) {
    int *bounds = reinterpret_cast<int *>(tab + a.group * a.tab);
    float *bias = tab + a.group * a.tab + kMaxBuckets;
    const int tid = threadIdx.x, n = a.n_buckets;
    if (tid < kMaxBuckets) bounds[tid] = tid < n - 1 ? a.bounds[tid] : 0x7fffffff;
    for (int i = tid; i < a.group * n; i += threads) {
        const float y = __uint_as_float((uint32_t)a.bias[(int64_t)head_kv * a.group * n + i] << 16);
        bias[i] = y <= -1.0e30f ? -__builtin_inff() : y * kLog2e;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();
    for (int x = tid; x < a.tab; x += threads) {
        const int rel = a.b0 - 1 - kBiasPad + x;
        int b = 0;  // bounds that are <= rel
#pragma unroll
        for (int step = kMaxBuckets / 2; step > 0; step /= 2) b += bounds[b + step - 1] <= rel ? step : 0;
        for (int g = 0; g < a.group; ++g) tab[g * a.tab + x] = bias[g * n + b];
    }
}
// entry of distance rel
__device__ __forceinline__ int bias_entry(const AttnArgs &a, int rel) { return rel - a.b0 + 1 + kBiasPad; }

}  // namespace lsrm
