// Dense attention over packed sequences, forward, on gfx950.
//
// Per 32 keys and wavefront (32 query rows):  S^T = K Q^T (A = 32 key rows, B = Q^T), probabilities in registers (each lane owns one query
// row, so maxima and sums are in-lane), O^T += V^T P^T (A = the transposed tile, read out of the row-major one by the transposing LDS
// loads).  The running maximum is kept optimistically: the exponentials of a tile are taken against the present one and only their
// sum is examined; a tile whose sum exceeds 2^10 is redone after raising the maximum.  Probabilities are rounded to bf16, to nearest, as the
// operand of the second product (no other matrix instruction takes them beside bf16 values at that rate); scores, maxima, sums and
// outputs are fp32 up to the one rounding at the end.
// Bound: at d = 128 by the matrix pipe at the clock that it is given (16 heads, 16384 tokens, causal: 1025 us, 1.07 PFLOP/s; a library
// product of 8192 x 8192 reaches 1.24 on the same card); below by the exponentials and what goes with them, 16 cycles and about 10
// instructions of the vector pipe for 16 of them (d = 64, 6 sequences of 1006 .. 4096 tokens, 16 heads: 252 us, 0.82 PFLOP/s; 32 heads of 32
// on 2, 3 sequences of up to 8000, causal: 440 us, 0.67); for few queries by the reading of keys and values (428 K keys, 2 heads of 128: 78 us, 5.6 TB/s).
#include "attn_internal.h"

#include <algorithm>

namespace lsrm {

namespace {

constexpr float kMinusHuge = -3.2e38f;  // initial running maximum, in the exponent's unit: finite, so no inf - inf, and below any score
constexpr float kSumLimit = 1024.0f;
constexpr int kFewRows = 32;

// The rows of one wavefront: 32 from row v0 of the sequence on.
template <int D, bool BIAS>
struct Rows {
    bf16x8 q[AttnGeo<D>::NS];
    f32x16 o[AttnGeo<D>::ND];
    float m, l;
    int lim;                // keys that this lane's row sees
    int lim_min, lim_max;   // the fewest and most that a row of the wavefront sees
    int pos, pos_min, pos_max;
    const float *tab;       // expanded bias of this lane's head
};
template <int D, bool BIAS>
__device__ __forceinline__ void load_rows(const AttnArgs &a, const Sequence &s, int head_kv, int v0, int lane, const float *tab, Rows<D, BIAS> &r) {
    const int n_rows = s.n_q * a.group;
    r.m = BIAS ? kMinusHuge : kMinusHuge / fmaxf(a.sl2, 1.0f);
    r.l = 0.f;
#pragma unroll
    for (int dt = 0; dt < AttnGeo<D>::ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) r.o[dt][i] = 0.f;
    r.lim = r.lim_min = r.lim_max = r.pos = r.pos_min = r.pos_max = 0;
    r.tab = tab;
    if (v0 >= n_rows) {
#pragma unroll
        for (int ks = 0; ks < AttnGeo<D>::NS; ++ks) r.q[ks] = bf16x8{};
        return;
    }
    // rows behind the last one do its work again; what they get is not written
    const int last = min(v0 + 31, n_rows - 1), v = min(v0 + (lane & 31), last);
    const int tok = (unsigned)v / (unsigned)a.group, g = v - tok * a.group;
    r.pos = tok + s.shift;
    r.pos_min = uniform((unsigned)v0 / (unsigned)a.group) + s.shift;
    r.pos_max = uniform((unsigned)last / (unsigned)a.group) + s.shift;
    auto seen = [&](int pos) { return a.causal ? min(max(pos + 1, 0), s.n_k) : s.n_k; };
    r.lim = seen(r.pos);
    r.lim_min = seen(r.pos_min);
    r.lim_max = seen(r.pos_max);
    if (BIAS) r.tab = tab + g * a.tab;
    const uint16_t *q = a.q + (s.q0 + tok) * a.qs[0] + (int64_t)(head_kv * a.group + g) * a.qs[1] + 8 * (lane >> 5);
#pragma unroll
    for (int ks = 0; ks < AttnGeo<D>::NS; ++ks) r.q[ks] = *reinterpret_cast<const bf16x8 *>(q + 16 * ks);
}

// Scores, with a bias, are kept in the exponent's unit (times log2e); without one the factor goes into the exponential's argument.
template <int D, bool BIAS>
__device__ __forceinline__ void add_bias(const AttnArgs &a, const Rows<D, BIAS> &r, f32x16 &s, int j0, int hh) {
    const bool ahead = j0 - r.pos_max >= a.b_last;
    if (ahead || j0 + 31 - r.pos_min < a.b0) {  // one bucket for the whole tile
        const float c = r.tab[ahead ? a.tab - 1 : 0];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = s[i] * a.sl2 + c;
    } else {
        const float *at = r.tab + bias_entry(a, j0 - r.pos) + 8 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = s[i] * a.sl2 + at[acc_row(i, 0)];
    }
}

template <int D, bool BIAS>
__device__ __forceinline__ void mask_scores(const Rows<D, BIAS> &r, f32x16 &s, int j0, int hh) {
    if (j0 + 32 > r.lim_min) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (j0 + acc_row(i, hh) >= r.lim) s[i] = -__builtin_inff();
    }
}

// The exponentials of a tile's scores, as the next product's operand; returns their sum.
__device__ __forceinline__ float exponentials(const f32x16 &s, float sl, float mc, BFrag (&b)[2]) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float x = __builtin_amdgcn_exp2f(s[2 * k] * sl - mc), y = __builtin_amdgcn_exp2f(s[2 * k + 1] * sl - mc);
        b[k / 4].u[k % 4] = pack_bf16(x, y);
        sum += x;
        sum += y;
    }
    return sum;
}

// One tile of 32 keys from key j0 of the sequence on.  Where a sum exceeds the limit, the running maximum is raised, what was summed so
// far rescaled, and the tile's exponentials done again.
template <int D, bool BIAS>
__device__ __forceinline__ void attend(const AttnArgs &a, Rows<D, BIAS> &r, const char *kt, const char *vt, const TileLane<D> &t, int j0, int hh) {
    f32x16 s = mfma_rows<D>(splat(0.f), kt, t, r.q);
    const float sl = BIAS ? 1.0f : a.sl2;
    if (BIAS) add_bias<D, BIAS>(a, r, s, j0, hh);
    mask_scores<D, BIAS>(r, s, j0, hh);
    BFrag b[2];
    float sum = exponentials(s, sl, r.m * sl, b);
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(sum <= kSumLimit)) != 0, 0)) {
        mfma_settle();  // the accumulators of the tile before may be in flight
        float mx = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
        const float m_new = fmaxf(r.m, half_max(mx));
        const float alpha = __builtin_amdgcn_exp2f((r.m - m_new) * sl);
        r.m = m_new;
        r.l *= alpha;
        // (in place: as ordinary code it made the compiler copy all accumulators on the way that is nearly always taken)
#pragma unroll
        for (int dt = 0; dt < AttnGeo<D>::ND; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) asm volatile("v_mul_f32 %0, %1, %0" : "+v"(r.o[dt][i]) : "v"(alpha));
        sum = exponentials(s, sl, m_new * sl, b);
    }
    r.l += sum;
    mfma_transposed<D>(r.o, vt, t, b);
}

// ---- many rows: four wavefronts of 32 rows share the tiles ------------------------------------------------------------
// Two stages of 64 keys (128 at d = 32) in LDS, one copied while the other is used, one barrier a stage; two workgroups on a CU at d = 128, four below, which
// fill each other's waits.  Tried and slower: 64 rows to a wavefront (each tile read from LDS once for both halves; d = 64 263 -> 302 us, at
// d = 128 one wavefront per SIMD 1042 -> 2388 us); scores of the next tile dealt between the exponentials of this one (d = 64 263 -> 292 us: the
// registers cost a fourth wavefront); sums by the two-element dot product of the rounded probabilities (d = 64 252 -> 260 us, d = 32 446 -> 430).
template <int D>
constexpr int kStageOf = D == 32 ? 128 : 64;  // keys per stage
template <int D>
constexpr int kForwardLds = 2 * kStageOf<D> * 2 * AttnGeo<D>::ROW;

// SPLIT: the keys are cut into a.parts parts, of which sums are left for attn_join_rows.
template <int D, bool BIAS, bool SPLIT>
__global__ __launch_bounds__(256, 2) void attn_forward_kernel(AttnArgs a) {
    using G = AttnGeo<D>;
    constexpr int kStage = kStageOf<D>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5;
    const int head_kv = blockIdx.x % a.h_kv, place = blockIdx.x / a.h_kv;
    const int part = SPLIT ? uniform(place % a.parts) : 0;
    int tile, seq;
    Sequence s;
    if (!find_tile<false>(a, a.group, 128, SPLIT ? uniform(place / a.parts) : place, s, tile, seq)) return;
    const int slot_rows = s.q_slot * a.group;
    if (a.causal) tile = (slot_rows - 1) / 128 - tile;  // the last rows, which see most keys, first
    const int v0 = tile * 128;
    const int n_rows = s.n_q * a.group;
    int keys = 0;  // that the last live row sees, hence any
    if (v0 < n_rows) {
        const int last = uniform((unsigned)min(v0 + 127, n_rows - 1) / (unsigned)a.group);
        keys = a.causal ? min(max(last + s.shift + 1, 0), s.n_k) : s.n_k;
    }
    int n_st = (keys + kStage - 1) / kStage, st_begin = 0;
    if (SPLIT) {
        const int per = uniform((n_st + a.parts - 1) / a.parts);
        st_begin = part * per;
        n_st = min(st_begin + per, n_st);
    }
    const char *kb = reinterpret_cast<const char *>(a.k + s.k0 * a.ks[0] + head_kv * a.ks[1]);
    const char *vb = reinterpret_cast<const char *>(a.v + s.k0 * a.vs[0] + head_kv * a.vs[1]);
    const uint32_t k_row = (uint32_t)a.ks[0] * 2, v_row = (uint32_t)a.vs[0] * 2;
    const CopyLane<D> c(lane);
    auto copy_stage = [&](int st, char *at) {
        const int j0 = st * kStage;
        copy_rows<D, kStage, 4>(kb + (uint64_t)j0 * k_row, k_row, keys - j0, at, wave, c);
        copy_rows<D, kStage, 4>(vb + (uint64_t)j0 * v_row, v_row, keys - j0, at + kStage * G::ROW, wave, c);
    };
    if (st_begin < n_st) copy_stage(st_begin, lds);
    float *tab = reinterpret_cast<float *>(lds + kForwardLds<D>);
    if (BIAS) expand_bias(a, head_kv, tab, 256);
    Rows<D, BIAS> r;
    load_rows<D, BIAS>(a, s, head_kv, v0 + wave * 32, lane, tab, r);
    const TileLane<D> t(lane);
    // (two stages to a turn, so that places in LDS are constants and cost no arithmetic)
    auto stage = [&](int st, char *at, char *next) {
        wait_copies<0>();
        wg_barrier();
        if (st + 1 < n_st) copy_stage(st + 1, next);
#pragma unroll
        for (int h = 0; h < kStage / 32; ++h)
            if (st * kStage + 32 * h < r.lim_max)
                attend<D, BIAS>(a, r, at + h * G::TILE, at + (kStage + 32 * h) * G::ROW, t, st * kStage + 32 * h, hh);
    };
    constexpr int STAGE = 2 * kStage * G::ROW;
    for (int st = st_begin; st < n_st; st += 2) {
        stage(st, lds, lds + STAGE);
        if (st + 1 < n_st) stage(st + 1, lds + STAGE, lds);
    }
    wait_copies<0>();
    wg_barrier();
    mfma_settle();
    const float l = half_sum(r.l), inv = l > 0.f || l != l ? 1.0f / l : 0.f;
    const int row = v0 + wave * 32 + (lane & 31);
    const bool live = row < n_rows;
    if (SPLIT) {
        if (row >= slot_rows) return;
        const int tok = (unsigned)row / (unsigned)a.group;
        const int64_t at = ((int64_t)part * a.n_q + s.q0 + tok) * a.h_q + head_kv * a.group + row - tok * a.group;
        if (hh == 0) a.part_ml[at] = make_float2(r.m * (BIAS ? 1.0f : a.sl2), live ? l : 0.f);
        float *to = a.part + at * D + 4 * hh;
#pragma unroll
        for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq)
                *reinterpret_cast<f32x4 *>(to + 32 * dt + 8 * gq) =
                    f32x4{r.o[dt][4 * gq], r.o[dt][4 * gq + 1], r.o[dt][4 * gq + 2], r.o[dt][4 * gq + 3]};
        return;
    }
    store_query_rows<D>(a, s, head_kv, v0 + wave * 32, slot_rows, r.o, inv, live, lds + wave * 32 * G::OUT_ROW, a.out, a.os, lane);
    if (a.lse != nullptr && hh == 0 && row < slot_rows) {
        const int tok = (unsigned)row / (unsigned)a.group, g = row - tok * a.group;
        a.lse[(int64_t)(s.q0 + tok) * a.h_q + head_kv * a.group + g] =
            live && inv != 0.f ? (r.m * (BIAS ? 1.0f : a.sl2) + __builtin_amdgcn_logf(l)) * kLn2 : -__builtin_inff();
    }
}

// ---- few rows: the wavefronts of a workgroup take turns at the keys of one tile of rows -------------------------------
// Where there are too few tiles of rows to fill the chip, the keys are cut into parts too: a unit is (tile of 32 rows, part), a part
// the same number of keys in all sequences, so that sequences of different lengths cost what they hold.  Every workgroup works that
// number out from the lengths (there is no one to ask: offsets and lengths are in device memory and the host must not wait).
__device__ __forceinline__ int row_tiles(const AttnArgs &a, const Sequence &s) { return (s.q_slot * a.group + kFewRows - 1) / kFewRows; }
__device__ __forceinline__ int parts_of(const Sequence &s, int chunk) { return max(1, (s.n_k + chunk - 1) / chunk); }
// keys of a part, where the sequences have `tiles` tiles that attend `keys` keys in all:
// sum over tiles of ceil(keys / chunk) <= keys / chunk + tiles <= unit_cap
__device__ __forceinline__ int part_keys(const AttnArgs &a, int64_t keys, int tiles) {
    const int room = max(a.unit_cap - tiles, 1);
    return uniform(max(256, (int)((keys + room - 1) / room + 127) / 128 * 128));
}
// The sequence of number x -- of a unit (UNITS), or of a tile of rows -- what is left of x within it, and the units of the sequences before.
// False if there is none.  A lane holds one sequence; up to 64 of them are loaded once.
template <bool UNITS>
__device__ __forceinline__ bool find_unit(const AttnArgs &a, int x, Sequence &s, int &within, int &chunk, int &units_before) {
    const int lane = threadIdx.x & 63;
    Sequence mine = {};
    int64_t keys = 0;
    int tiles = 0;
    for (int i = lane; i < a.n_seq; i += 64) {
        mine = load_sequence(a, i);
        tiles += row_tiles(a, mine);
        keys += (int64_t)row_tiles(a, mine) * mine.n_k;
    }
    for (int y = 32; y > 0; y /= 2) {
        keys += __shfl_xor(keys, y);
        tiles += __shfl_xor(tiles, y);
    }
    chunk = part_keys(a, keys, tiles);
    int base = 0, units = 0;  // of the sequences before these 64: numbers, units
    for (int i0 = 0; i0 < a.n_seq; i0 += 64) {
        const bool any = i0 + lane < a.n_seq;
        if (a.n_seq > 64 && any) mine = load_sequence(a, i0 + lane);
        const int u = any ? row_tiles(a, mine) * parts_of(mine, chunk) : 0, n = UNITS ? u : any ? row_tiles(a, mine) : 0;
        int upto = n, u_upto = u;
        for (int y = 1; y < 64; y *= 2) {
            const int b = __shfl_up(upto, y), c = __shfl_up(u_upto, y);
            if (lane >= y) {
                upto += b;
                u_upto += c;
            }
        }
        const uint64_t found = __builtin_amdgcn_ballot_w64(n > 0 && x < base + upto);
        if (found != 0) {
            const int at = __builtin_ctzll(found);
            within = x - base - __builtin_amdgcn_readlane(upto - n, at);
            units_before = units + __builtin_amdgcn_readlane(u_upto - u, at);
            s.q0 = __builtin_amdgcn_readlane(mine.q0, at);
            s.n_q = __builtin_amdgcn_readlane(mine.n_q, at);
            s.q_slot = __builtin_amdgcn_readlane(mine.q_slot, at);
            s.k0 = __builtin_amdgcn_readlane(mine.k0, at);
            s.n_k = __builtin_amdgcn_readlane(mine.n_k, at);
            s.k_slot = __builtin_amdgcn_readlane(mine.k_slot, at);
            s.shift = s.n_k - s.n_q;
            return within >= 0;
        }
        base += __builtin_amdgcn_readlane(upto, 63);
        units += __builtin_amdgcn_readlane(u_upto, 63);
    }
    return false;
}

// Wavefronts of a workgroup.  Each has a ring of two slots (a K and a V tile) of its own.  Where the keys are cut, two workgroups share a CU, so
// that one streams while the other starts or ends; where they are not, a tile's keys are dealt to as many wavefronts as LDS has room for
// (beside the largest expanded bias: half as many).
template <int D, bool CROWDED>
constexpr int kFewWaves = (D == 128 ? 2 : 4) * (CROWDED ? 1 : 2);
template <int D>
constexpr int kFewRing = 2 * 2 * AttnGeo<D>::TILE;  // per wavefront
template <int D, bool CROWDED>
constexpr int kFewLds = kFewWaves<D, CROWDED> * (kFewRing<D> + 256);
template <int D>
constexpr int kPartFloats = kFewRows * (D + 2);

// Writes N channels of a row from channel c0 on.
template <int N>
__device__ __forceinline__ void store_channels(const AttnArgs &a, const Sequence &s, int head_kv, int v, int c0, const float (&x)[N], float m2,
                                               float l) {
    const bool live = v < s.n_q * a.group;
    const float inv = live && (l > 0.f || l != l) ? 1.0f / l : 0.f;
    const int tok = (unsigned)v / (unsigned)a.group, head = head_kv * a.group + v - tok * a.group;
    uint16_t *dst = a.out + (s.q0 + tok) * a.os[0] + (int64_t)head * a.os[1] + c0;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        uint2 w;
        w.x = inv != 0.f ? pack_bf16(x[i] * inv, x[i + 1] * inv) : 0;
        w.y = inv != 0.f ? pack_bf16(x[i + 2] * inv, x[i + 3] * inv) : 0;
        *reinterpret_cast<uint2 *>(dst + i) = w;
    }
    if (a.lse != nullptr && c0 == 0)
        a.lse[(int64_t)(s.q0 + tok) * a.h_q + head] = inv != 0.f ? (m2 + __builtin_amdgcn_logf(l)) * kLn2 : -__builtin_inff();
}

template <int D, bool BIAS, bool SPLIT>
__global__ __launch_bounds__((64 * kFewWaves<D, SPLIT || BIAS>), 1) void attn_few_kernel(AttnArgs a) {
    using G = AttnGeo<D>;
    constexpr int NW = kFewWaves<D, SPLIT || BIAS>, STEP = 32 * NW;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5;
    const int head_kv = blockIdx.x % a.h_kv, unit = blockIdx.x / a.h_kv;
    int tile, part = 0, n_parts = 1, chunk = 0, unused;
    Sequence s;
    if (SPLIT) {
        if (!find_unit<true>(a, unit, s, tile, chunk, unused)) return;
        n_parts = uniform(parts_of(s, chunk));
        part = uniform(tile % n_parts);
        tile = uniform(tile / n_parts);
    } else if (!find_tile<false>(a, a.group, kFewRows, unit, s, tile, unused)) {
        return;
    }
    const int v0 = tile * kFewRows, slot_rows = s.q_slot * a.group;
    if (v0 < 0 || v0 >= slot_rows) return;
    Rows<D, BIAS> r;
    float *tab = reinterpret_cast<float *>(lds + kFewLds<D, SPLIT || BIAS>);
    load_rows<D, BIAS>(a, s, head_kv, v0, lane, tab, r);
    const int j_begin = SPLIT ? part * chunk : 0, j_end = min(SPLIT ? j_begin + chunk : s.n_k, r.lim_max);
    const char *kb = reinterpret_cast<const char *>(a.k + s.k0 * a.ks[0] + head_kv * a.ks[1]);
    const char *vb = reinterpret_cast<const char *>(a.v + s.k0 * a.vs[0] + head_kv * a.vs[1]);
    const uint32_t k_row = (uint32_t)a.ks[0] * 2, v_row = (uint32_t)a.vs[0] * 2;
    const CopyLane<D> c(lane);
    const TileLane<D> t(lane);
    char *ring = lds + wave * kFewRing<D>;
    auto copy_tile = [&](int j0, int slot) {
        char *at = ring + slot * 2 * G::TILE;
        copy_rows<D, 32, 1>(kb + (uint64_t)j0 * k_row, k_row, j_end - j0, at, 0, c);
        copy_rows<D, 32, 1>(vb + (uint64_t)j0 * v_row, v_row, j_end - j0, at + G::TILE, 0, c);
    };
    int j0 = j_begin + wave * 32;
    if (j0 < j_end) copy_tile(j0, 0);
    if (BIAS) {
        expand_bias(a, head_kv, tab, 64 * NW);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
    }
    for (int slot = 0; j0 < j_end; j0 += STEP, slot ^= 1) {
        if (j0 + STEP < j_end) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // nobody waits for this slot's last reads but this wavefront
            copy_tile(j0 + STEP, slot ^ 1);
            wait_copies<2 * G::COPIES>();
        } else {
            wait_copies<0>();
        }
        const char *at = ring + slot * 2 * G::TILE;
        attend<D, BIAS>(a, r, at, at + G::TILE, t, j0, hh);
    }
    // the wavefronts' sums meet in LDS
    mfma_settle();
    constexpr int PITCH = D + 4;
    float *mine = reinterpret_cast<float *>(ring), *ml = reinterpret_cast<float *>(lds + NW * kFewRing<D>);
    const float l = half_sum(r.l);
#pragma unroll
    for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            f32x4 w = {r.o[dt][4 * gq], r.o[dt][4 * gq + 1], r.o[dt][4 * gq + 2], r.o[dt][4 * gq + 3]};
            *reinterpret_cast<f32x4 *>(mine + (lane & 31) * PITCH + 32 * dt + 8 * gq + 4 * hh) = w;
        }
    if (hh == 0) {
        ml[wave * 64 + lane] = r.m * (BIAS ? 1.0f : a.sl2);
        ml[wave * 64 + 32 + lane] = l;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();
    constexpr int TPR = 2 * NW < D / 4 ? 2 * NW : D / 4, CH = D / TPR;  // threads per row, channels per thread
    const int row = threadIdx.x / TPR, c0 = (threadIdx.x % TPR) * CH;
    if (row >= kFewRows || v0 + row >= slot_rows) return;
    float m2 = ml[row], sum = 0.f, x[CH] = {};
#pragma unroll
    for (int w = 1; w < NW; ++w) m2 = fmaxf(m2, ml[w * 64 + row]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[w * 64 + row] - m2);
        sum += f * ml[w * 64 + 32 + row];
        const float *from = reinterpret_cast<const float *>(lds + w * kFewRing<D>) + row * PITCH + c0;
#pragma unroll
        for (int i = 0; i < CH; ++i) x[i] += f * from[i];
    }
    if (SPLIT && n_parts > 1) {
        float *to = a.part + ((int64_t)unit * a.h_kv + head_kv) * kPartFloats<D>;
#pragma unroll
        for (int i = 0; i < CH; i += 4) *reinterpret_cast<f32x4 *>(to + row * D + c0 + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
        if (c0 == 0) {
            to[kFewRows * D + row] = m2;
            to[kFewRows * D + kFewRows + row] = sum;
        }
    } else {
        store_channels<CH>(a, s, head_kv, v0 + row, c0, x, m2, sum);
    }
}

// Joins the parts of a tile's rows: a workgroup takes every eighth row, one after the other, four channels to a lane and the parts dealt to
// 1024 / d groups of lanes.
constexpr int kJoinWays = 8;
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ f32x4 sums[GROUPS][LANES];
    __shared__ float part_max[4], part_sum[4];
    const int way = blockIdx.x % kJoinWays, head_kv = blockIdx.x / kJoinWays % a.h_kv, slot = blockIdx.x / kJoinWays / a.h_kv;
    int tile, chunk, unit;
    Sequence s;
    if (!find_unit<false>(a, slot, s, tile, chunk, unit)) return;
    const int slot_rows = s.q_slot * a.group, n_parts = parts_of(s, chunk);
    if (n_parts == 1 || tile * kFewRows + way >= slot_rows) return;
    unit += tile * n_parts;
    if (unit < 0 || n_parts > a.unit_cap - unit) return;  // (of offsets that do not ascend)
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, wave = threadIdx.x / 64;
    const float *from = a.part + ((int64_t)unit * a.h_kv + head_kv) * kPartFloats<D>;
    const int64_t step = (int64_t)a.h_kv * kPartFloats<D>;
    for (int row = way; row < kFewRows && tile * kFewRows + row < slot_rows; row += kJoinWays) {
        const float *ml = from + kFewRows * D + row;
        float m2 = kMinusHuge;
        for (int p = threadIdx.x; p < n_parts; p += 256) m2 = fmaxf(m2, ml[p * step]);
        for (int x = 32; x > 0; x /= 2) m2 = fmaxf(m2, __shfl_xor(m2, x));
        if (threadIdx.x % 64 == 0) part_max[wave] = m2;
        __syncthreads();
        m2 = fmaxf(fmaxf(part_max[0], part_max[1]), fmaxf(part_max[2], part_max[3]));
        float sum = 0.f;
        for (int p = threadIdx.x; p < n_parts; p += 256) sum += ml[p * step + kFewRows] * __builtin_amdgcn_exp2f(ml[p * step] - m2);
        for (int x = 32; x > 0; x /= 2) sum += __shfl_xor(sum, x);
        if (threadIdx.x % 64 == 0) part_sum[wave] = sum;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int p = group; p < n_parts; p += GROUPS)
            acc += __builtin_amdgcn_exp2f(ml[p * step] - m2) * *reinterpret_cast<const f32x4 *>(from + p * step + row * D + 4 * lane);
        sums[group][lane] = acc;
        __syncthreads();
        if (group == 0) {
            for (int i = 1; i < GROUPS; ++i) acc += sums[i][lane];
            const float x[4] = {acc[0], acc[1], acc[2], acc[3]};
            store_channels<4>(a, s, head_kv, tile * kFewRows + row, 4 * lane, x, m2, part_sum[0] + part_sum[1] + part_sum[2] + part_sum[3]);
        }
        __syncthreads();
    }
}

// Joins the parts of attn_forward_kernel: up to 2048 / d queries of a sequence's slot, one head to a workgroup, eight channels to a thread.
template <int D>
__global__ __launch_bounds__(256) void attn_join_rows(AttnArgs a) {
    constexpr int CH = D / 8, ROWS = 256 / CH;
    const int head = blockIdx.x % a.h_q;
    int tile, seq;
    Sequence s;
    if (!find_tile<false>(a, 1, ROWS, blockIdx.x / a.h_q, s, tile, seq)) return;
    const int r = tile * ROWS + threadIdx.x / CH, c0 = threadIdx.x % CH * 8;
    if (r >= s.q_slot) return;
    const int64_t at = (int64_t)(s.q0 + r) * a.h_q + head, step = (int64_t)a.n_q * a.h_q;
    float m2 = kMinusHuge, sum = 0.f, x[8] = {};
    for (int p = 0; p < a.parts; ++p) m2 = fmaxf(m2, a.part_ml[at + p * step].x);
#pragma unroll 4
    for (int p = 0; p < a.parts; ++p) {
        const float2 ml = a.part_ml[at + p * step];
        const float f = __builtin_amdgcn_exp2f(ml.x - m2);
        sum += f * ml.y;
        const f32x4 *from = reinterpret_cast<const f32x4 *>(a.part + (at + p * step) * D + c0);
        const f32x4 y = from[0], z = from[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] += f * y[i];
            x[4 + i] += f * z[i];
        }
    }
    const int head_kv = head / a.group;
    store_channels<8>(a, s, head_kv, r * a.group + head - head_kv * a.group, c0, x, m2, sum);
}

// How a forward call is worked on.  FEW: workgroups of 32 rows, whose wavefronts take turns at the keys: where these are all on the chip at
// the same time and the keys are short, a call takes as long as the fewest steps behind each other (5 sequences of up to 130 tokens, 4
// heads of 64 with a bias: 7.3 us, 9.4 in workgroups of 128 rows).  MANY: sequences of 64 and more rows (queries times heads of a group)
// in workgroups of 128, whose keys are cut into parts where there are few of them.  Others are cut for long keys, where the second launch
// does not cost more than it saves (4 streams of up to 513 keys: 11.1 us cut, 6.8 whole).
enum Way { MANY, FEW, FEW_SPLIT };
struct Plan {
    Way way;
    int64_t slots32;  // tiles of 32 rows at most
    int parts;        // MANY
    int unit_cap;     // FEW_SPLIT: units that the keys are cut into, per key/value head: two workgroups for every CU, or twice the tiles where
                      // there are many
    size_t part, part_ml, total;  // workspace
};
Plan forward_plan(const AttnArgs &a, int d) {
    Plan p{};
    const int64_t rows = (int64_t)a.n_q * a.group;
    p.slots32 = rows / kFewRows + a.n_seq;
    p.parts = 1;
    const bool small = p.slots32 * a.h_kv <= (d == 32 ? 512 : 256), short_keys = a.n_k / a.n_seq <= 1024;
    if (small && short_keys) {
        p.way = FEW;
    } else if (rows >= (int64_t)64 * a.n_seq) {
        p.way = MANY;
        p.parts = best_parts(walk_steps(a), d == 32 ? 380 : d == 64 ? 540 : 700, ((double)rows / 128 + 1) * a.h_kv, full_chip(d),
                             (double)a.n_q * a.h_q * (d + 2) * 8, (int64_t)a.n_k / a.n_seq / 32, (rows / 128 + a.n_seq) * a.h_kv);
        if (p.parts > 1) {
            p.part_ml = align_up((size_t)p.parts * a.n_q * a.h_q * d * 4, 256);
            p.total = p.part_ml + (size_t)p.parts * a.n_q * a.h_q * 8;
        }
    } else if (p.slots32 * a.h_kv >= 256 || short_keys) {
        p.way = FEW;
    } else {
        p.way = FEW_SPLIT;
        p.unit_cap = (int)std::max<int64_t>(2 * p.slots32, 512 / a.h_kv);
        p.total = (size_t)p.unit_cap * a.h_kv * kFewRows * (d + 2) * 4;
    }
    return p;
}

template <int D>
lsrm_status launch_forward_d(AttnArgs a, void *ws, hipStream_t st) {
    const Plan p = forward_plan(a, D);
    const int tab = bias_lds_floats(a) * 4;
    const bool bias = a.n_buckets > 0;
    if (p.way == MANY) {
        const int64_t grid = ((int64_t)a.n_q * a.group / 128 + a.n_seq) * a.h_kv * p.parts;
        a.parts = p.parts;
        if (p.parts == 1)
            return launch_attn(bias ? &attn_forward_kernel<D, true, false> : &attn_forward_kernel<D, false, false>, grid, 256,
                               kForwardLds<D> + tab, a, st);
        a.part = static_cast<float *>(ws);
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(ws) + p.part_ml);
        const lsrm_status rc = launch_attn(bias ? &attn_forward_kernel<D, true, true> : &attn_forward_kernel<D, false, true>, grid, 256,
                                           kForwardLds<D> + tab, a, st);
        if (rc != LSRM_OK) return rc;
        return launch_attn(&attn_join_rows<D>, ((int64_t)a.n_q / (2048 / D) + a.n_seq) * a.h_q, 256, 0, a, st);
    }
    const int64_t n_tiles = p.slots32 * a.h_kv;
    if (p.way == FEW)
        return bias ? launch_attn(&attn_few_kernel<D, true, false>, n_tiles, 64 * kFewWaves<D, true>, kFewLds<D, true> + tab, a, st)
                    : launch_attn(&attn_few_kernel<D, false, false>, n_tiles, 64 * kFewWaves<D, false>, kFewLds<D, false>, a, st);
    a.unit_cap = p.unit_cap;
    a.part = static_cast<float *>(ws);
    lsrm_status rc = launch_attn(bias ? &attn_few_kernel<D, true, true> : &attn_few_kernel<D, false, true>, (int64_t)a.unit_cap * a.h_kv,
                                 64 * kFewWaves<D, true>, kFewLds<D, true> + tab, a, st);
    if (rc != LSRM_OK) return rc;
    return launch_attn(&attn_join_kernel<D>, n_tiles * kJoinWays, 256, 0, a, st);
}

}  // namespace

int best_parts(double steps, double cycles, double workgroups, double full, double bytes, int64_t walk, int64_t grid, double *time) {
    const double work = steps * cycles / 4 / 256 / 2.1e3;  // us, with the chip full
    int best = 1;
    double least = 0;
    for (int p = 1; p <= 16 && (p == 1 || (p * 4 <= walk && p * grid <= 1 << 23)); ++p) {
        const double t = work / std::min(1.0, workgroups * p / full) + (p > 1 ? 4 + p * bytes / 3.5e6 : 0);
        if (p == 1 || t < least) {
            best = p;
            least = t;
        }
    }
    if (time != nullptr) *time = least;
    return best;
}

size_t attn_forward_ws_bytes(const AttnArgs &a, int d) { return a.n_seq == 0 || a.n_q == 0 ? 0 : forward_plan(a, d).total; }

lsrm_status launch_attn_forward(AttnArgs a, int d, void *ws, hipStream_t st) {
    switch (d) {
        case 32: return launch_forward_d<32>(a, ws, st);
        case 64: return launch_forward_d<64>(a, ws, st);
        default: return launch_forward_d<128>(a, ws, st);
    }
}

}  // namespace lsrm
