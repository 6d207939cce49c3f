// Dense attention over packed sequences, backward, on gfx950.
//
// With P = softmax probabilities recomputed from the saved log-sum-exp, D_i = dout_i . out_i, dP = dout V^T:
//     dV = P^T dout      dS = P o (dP - D)      dQ = scale dS K      dK = scale dS^T Q      dB[b] = sum of dS over bucket b
// Two passes that each own their output rows (no atomics between workgroups, one order of sums):
//   attn_dq_kernel   128 query rows to a workgroup (32 in small problems), one query row per lane (S^T = K Q^T), walks the keys; works out D for itself
//                    and leaves it, with the log-sum-exp, for the other pass.
//   attn_dkv_kernel  128 keys of a key/value head to a workgroup (32 in small problems), one key per lane (S = Q K^T), walks the queries of the heads that
//                    read them; sums dS by distance.
// Seven contractions where five are needed: the price of gradients that are the same in every run (one pass would have to add dQ from many
// workgroups).  P and dS are rounded to bf16, to nearest, as operands; D comes from the rounded outputs, which makes dQ's error 1.5 of that
// of a single rounding instead of 1.4 (dK, dV and the bias' gradient get the D that the first pass puts right).
// Bound: at d = 128 by the matrix pipe (8192 + 6782 tokens, 16 heads, causal: dQ 615 us and dK, dV 836 us, 1.13 and 1.11 PFLOP/s of the
// contractions done), below by the vector pipe beside it, of which each takes what the other leaves, and in small problems by the longest walk.
#include "attn_internal.h"

#include <algorithm>

namespace lsrm {

namespace {

template <int D>
constexpr int kStageOf = D == 32 ? 128 : 64;  // keys per stage of the dQ pass
template <int D>
constexpr int kDqLds = 2 * kStageOf<D> * 2 * AttnGeo<D>::ROW;
// FEW: the wavefronts take turns at the keys of the same 32 rows, each through a ring of two tiles of its own, and meet in LDS at the end.
// (Backward of 5 sequences of up to 257 tokens, 8 heads on 4: d = 32 14.9 -> 12.7 us, d = 64 18.6 -> 15.5, d = 128 29.7 -> 25.5.)
template <int D>
constexpr int kDqFewRing = 2 * 2 * AttnGeo<D>::TILE > 32 * (D + 4) * 4 ? 2 * 2 * AttnGeo<D>::TILE : 32 * (D + 4) * 4;
template <int D>
constexpr int kDqFewLds = 4 * (kDqFewRing<D> + 128);
template <int D>
constexpr int kDkvSlot = 2 * AttnGeo<D>::TILE + 256;  // 32 rows of q, of dout, and their entries of aux
// Slots of the dK/dV pass' ring, half of them used between two barriers and half under way: below d = 128 LDS has room for two tiles each.
template <int D>
constexpr int kDkvRing = D == 128 ? 2 : 4;
template <int D>
constexpr int kDkvLds = 4 * 32 * AttnGeo<D>::OUT_ROW > kDkvRing<D> * kDkvSlot<D> ? 4 * 32 * AttnGeo<D>::OUT_ROW : kDkvRing<D> * kDkvSlot<D>;

template <int D, bool BIAS, bool FEW>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(AttnArgs a) {
    using G = AttnGeo<D>;
    constexpr int kStage = FEW ? 32 : kStageOf<D>, ROWS = FEW ? 32 : 128, STRIDE = FEW ? 4 : 1;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5;
    const int head_kv = blockIdx.x % a.h_kv, place = blockIdx.x / a.h_kv;
    const int part = FEW ? 0 : place % a.parts;
    int tile, seq;
    Sequence s;
    if (!find_tile<false>(a, a.group, ROWS, FEW ? place : place / a.parts, s, tile, seq)) return;
    const int slot_rows = s.q_slot * a.group, n_rows = s.n_q * a.group;
    if (a.causal) tile = (slot_rows - 1) / ROWS - tile;  // the last rows, which see most keys, first
    const int v_wg = tile * ROWS;
    auto seen = [&](int pos) { return a.causal ? min(max(pos + 1, 0), s.n_k) : s.n_k; };
    const int keys = v_wg < n_rows ? seen(uniform((unsigned)min(v_wg + ROWS - 1, n_rows - 1) / (unsigned)a.group) + s.shift) : 0;
    const int st_all = (keys + kStage - 1) / kStage, st_per = FEW ? st_all : uniform((st_all + a.parts - 1) / a.parts);
    const int st_begin = part * st_per + (FEW ? wave : 0), st_end = FEW ? st_all : min(st_begin + st_per, st_all);
    const char *kb = reinterpret_cast<const char *>(a.k + s.k0 * a.ks[0] + head_kv * a.ks[1]);
    const char *vb = reinterpret_cast<const char *>(a.v + s.k0 * a.vs[0] + head_kv * a.vs[1]);
    const uint32_t k_row = (uint32_t)a.ks[0] * 2, v_row = (uint32_t)a.vs[0] * 2;
    const CopyLane<D> c(lane);
    char *ring = lds + (FEW ? wave * kDqFewRing<D> : 0);
    auto copy_stage = [&](int st) {
        char *at = ring + ((st - st_begin) / STRIDE & 1) * (2 * kStage * G::ROW);
        const int j0 = st * kStage;
        copy_rows<D, kStage, FEW ? 1 : 4>(kb + (uint64_t)j0 * k_row, k_row, keys - j0, at, FEW ? 0 : wave, c);
        copy_rows<D, kStage, FEW ? 1 : 4>(vb + (uint64_t)j0 * v_row, v_row, keys - j0, at + kStage * G::ROW, FEW ? 0 : wave, c);
    };
    if (st_begin < st_end) copy_stage(st_begin);
    float *tab = reinterpret_cast<float *>(lds + (FEW ? kDqFewLds<D> : kDqLds<D>));
    if (BIAS) expand_bias(a, head_kv, tab, 256);
    if (FEW && BIAS) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
    }

    const int v0 = v_wg + (FEW ? 0 : wave * 32), v = v0 + (lane & 31);
    const bool live = v < n_rows;
    const int last = max(min(v0 + 31, n_rows - 1), 0), vc = min(v, last);  // rows behind the last one do its work again, with P = 0
    const int tok = (unsigned)vc / (unsigned)a.group, g = vc - tok * a.group, head = head_kv * a.group + g;
    const int pos = tok + s.shift, pos_min = uniform((unsigned)v0 / (unsigned)a.group) + s.shift;
    const int pos_max = uniform((unsigned)last / (unsigned)a.group) + s.shift;
    const int lim = seen(pos), lim_min = seen(pos_min), lim_max = v0 < n_rows ? seen(pos_max) : 0;
    bf16x8 q[G::NS], dout[G::NS];
    float off = __builtin_inff(), delta = 0.f;
    if (v0 < n_rows) {
        const uint16_t *qp = a.q + (s.q0 + tok) * a.qs[0] + head * a.qs[1] + 8 * hh;
        const int64_t o_at = (s.q0 + tok) * a.os[0] + head * a.os[1] + 8 * hh;
#pragma unroll
        for (int ks = 0; ks < G::NS; ++ks) {
            q[ks] = *reinterpret_cast<const bf16x8 *>(qp + 16 * ks);
            dout[ks] = *reinterpret_cast<const bf16x8 *>(a.dout + o_at + 16 * ks);
            const bf16x8 o = *reinterpret_cast<const bf16x8 *>(a.o + o_at + 16 * ks);
#pragma unroll
            for (int i = 0; i < 8; ++i) delta += (float)dout[ks][i] * (float)o[i];
        }
        delta = half_sum(delta);
        const float lse = a.lse_in[(int64_t)(s.q0 + tok) * a.h_q + head];
        if (live && lse != -__builtin_inff()) off = lse * kLog2e;
    } else {
#pragma unroll
        for (int ks = 0; ks < G::NS; ++ks) q[ks] = dout[ks] = bf16x8{};
    }
    f32x16 dq[G::ND];
#pragma unroll
    for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[dt][i] = 0.f;
    const f32x16 minus_delta = splat(-delta);  // (what dP is added to: no instruction of its own takes D off)
    float miss = 0.f;  // sum of dS over this lane's keys
    const float *tab_g = tab + g * a.tab;
    const TileLane<D> t(lane);
    for (int st = st_begin; st < st_end; st += STRIDE) {
        if constexpr (FEW) {
            if (st + STRIDE < st_end) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // nobody waits for this slot's last reads but this wavefront
                copy_stage(st + STRIDE);
                wait_copies<2 * G::COPIES>();
            } else {
                wait_copies<0>();
            }
        } else {
            wait_copies<0>();
            wg_barrier();
            if (st + 1 < st_end) copy_stage(st + 1);
        }
        const char *at = ring + ((st - st_begin) / STRIDE & 1) * (2 * kStage * G::ROW);
#pragma unroll
        for (int h = 0; h < kStage / 32; ++h) {
            const int j0 = st * kStage + 32 * h;
            if (j0 >= lim_max) continue;
            const char *kt = at + h * G::TILE, *vt = at + (kStage + 32 * h) * G::ROW;
            f32x16 x = mfma_rows<D>(splat(0.f), kt, t, q), dp = mfma_rows<D>(minus_delta, vt, t, dout);
            const bool behind = BIAS && j0 + 31 - pos_min < a.b0, ahead = BIAS && j0 - pos_max >= a.b_last;
            if (BIAS) {
                if (behind || ahead) {
                    const float b = tab_g[ahead ? a.tab - 1 : 0];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = x[i] * a.sl2 + b;
                } else {
                    const float *entry = tab_g + bias_entry(a, j0 - pos) + 8 * hh;
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = x[i] * a.sl2 + entry[acc_row(i, 0)];
                }
            }
            if (j0 + 32 > lim_min) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (j0 + acc_row(i, hh) >= lim) x[i] = -__builtin_inff();
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                dp[i] = __builtin_amdgcn_exp2f(BIAS ? x[i] - off : x[i] * a.sl2 - off) * dp[i];
                miss += dp[i];
            }
            BFrag b[2];
            to_b_operand(dp, b);
            mfma_transposed<D>(dq, kt, t, b);
        }
    }
    wait_copies<0>();
    if (!FEW) wg_barrier();
    mfma_settle();
    if constexpr (FEW) {
        constexpr int PITCH = D + 4;
        float *mine = reinterpret_cast<float *>(ring) + (lane & 31) * PITCH + 4 * hh, *misses = reinterpret_cast<float *>(lds + 4 * kDqFewRing<D>);
#pragma unroll
        for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq)
                *reinterpret_cast<f32x4 *>(mine + 32 * dt + 8 * gq) = f32x4{dq[dt][4 * gq], dq[dt][4 * gq + 1], dq[dt][4 * gq + 2], dq[dt][4 * gq + 3]};
        miss = half_sum(miss);
        if (hh == 0) misses[wave * 32 + lane] = miss;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
        // (D put right, see below)
        if (wave == 0 && live && hh == 0)
            a.aux[(int64_t)head * a.n_q + s.q0 + tok] =
                make_float2(off, -((misses[lane] + misses[32 + lane]) + (misses[64 + lane] + misses[96 + lane])) - delta);
        const int row = threadIdx.x / 8, c0 = 4 * (threadIdx.x % 8), to_v = v0 + row;
        if (to_v >= slot_rows) return;
        const int to_tok = (unsigned)to_v / (unsigned)a.group, to_head = head_kv * a.group + to_v - to_tok * a.group;
        uint16_t *dst = a.dq + (s.q0 + to_tok) * a.qs[0] + to_head * a.qs[1] + c0;
#pragma unroll
        for (int ch = 0; ch < D; ch += 32) {
            f32x4 x[4];
#pragma unroll
            for (int w = 0; w < 4; ++w)
                x[w] = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds + w * kDqFewRing<D>) + row * PITCH + c0 + ch);
            const f32x4 y = ((x[0] + x[1]) + (x[2] + x[3])) * a.scale;
            *reinterpret_cast<uint2 *>(dst + ch) = to_v < n_rows ? make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])) : make_uint2(0, 0);
        }
        return;
    }
    if (a.parts == 1) {
        store_query_rows<D>(a, s, head_kv, v0, slot_rows, dq, a.scale, live, lds + wave * 32 * G::OUT_ROW, a.dq, a.qs, lane);
    } else if (v < slot_rows) {
        const int to_tok = (unsigned)v / (unsigned)a.group, to_head = head_kv * a.group + v - to_tok * a.group;
        float *to = a.part_q + (((int64_t)part * a.n_q + s.q0 + to_tok) * a.h_q + to_head) * D + 4 * hh;
#pragma unroll
        for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq) {
                const float z = live ? a.scale : 0.f;
                *reinterpret_cast<f32x4 *>(to + 32 * dt + 8 * gq) =
                    f32x4{dq[dt][4 * gq] * z, dq[dt][4 * gq + 1] * z, dq[dt][4 * gq + 2] * z, dq[dt][4 * gq + 3] * z};
            }
    }
    // D was taken from outputs that are rounded, as are the probabilities they were summed with; it is off by the sum of dS over
    // all keys, which belongs to be zero.  The other pass, and with it dK and the bias' gradient, get it put right.
    miss = half_sum(miss);
    if (live && hh == 0)
        a.aux[((int64_t)part * a.h_q + head) * a.n_q + s.q0 + tok] = make_float2(off, -miss - (part == 0 ? delta : 0.f));
}

// Sums of dS by distance, of a tile of 32 queries and 32 keys: a wavefront writes the tile skewed, so that a distance's elements lie in one
// row, each lane sums a row and adds it to the distance's place.  (Floating-point additions in LDS, one for each element, took 3.8 us
// a tile; this takes 0.3.)  Places of a row that no element has stay zero from the start.
// NE: elements of an accumulator at a time, 16 (the whole tile) or 4 (eight queries; at d = 128, where LDS is short).
template <int NE>
struct Skew {
    static constexpr int ROWS = 2 * NE, TOP = NE == 16 ? 31 : 11;      // queries; distance of row 0 below that of the first query and key
    static constexpr int N = 32 + TOP, PITCH = ROWS + 1;               // distances, floats from one to the next
    static constexpr int BYTES = (N * PITCH * 4 + 15) / 16 * 16;
};
template <int NE>
__device__ __forceinline__ void add_by_distance(const f32x16 &ds, bool live, float *skew, float *near, int lane) {
    using S = Skew<NE>;
    const int hh = lane >> 5, jl = lane & 31;
#pragma unroll
    for (int pass = 0; pass < 16 / NE; ++pass) {
        const int first = NE == 16 ? 0 : 16 * (pass / 2) + 4 * (pass % 2);  // query of the pass' first element
#pragma unroll
        for (int m = 0; m < NE; ++m) {
            const int e = pass * NE + m, row = acc_row(m, hh), place = NE == 16 ? row : m + 4 * hh;
            skew[(jl - row + S::TOP) * S::PITCH + place] = live ? ds[e] : 0.f;
        }
        // (lanes read what others wrote: the compiler, which sees one of them, must not move accesses across)
        asm volatile("" ::: "memory");
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        if (lane < S::N) {
#pragma unroll
            for (int r = 0; r < S::ROWS; ++r) sum[r % 4] += skew[lane * S::PITCH + r];
            near[lane - S::TOP - first] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        asm volatile("" ::: "memory");
    }
}

// What a workgroup has summed of the bias' gradient of one query head goes to its place, and the sums begin anew.
// near: [4 wavefronts][a.tab] by distance; lo, hi: of the lane, tiles before the first and from the last bound on.
__device__ __forceinline__ void flush_bias(const AttnArgs &a, float *near, float *far, float lo, float hi, float *dst) {
    for (int x = 32; x > 0; x /= 2) {
        lo += __shfl_xor(lo, x);
        hi += __shfl_xor(hi, x);
    }
    if (threadIdx.x % 64 == 0) {
        far[threadIdx.x / 64] = lo;
        far[4 + threadIdx.x / 64] = hi;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();
    for (int x = threadIdx.x; x < a.tab; x += 256) {
        near[x] = (near[x] + near[a.tab + x]) + (near[2 * a.tab + x] + near[3 * a.tab + x]);
        near[a.tab + x] = near[2 * a.tab + x] = near[3 * a.tab + x] = 0.f;
    }
    __syncthreads();
    // four threads to a bucket
    const int b = threadIdx.x / 4, n = a.n_buckets;
    float sum = 0.f;
    if (b < n) {
        const int from = b > 0 ? bias_entry(a, a.bounds[b - 1]) : 0, to = b < n - 1 ? bias_entry(a, a.bounds[b]) : a.tab;
        for (int x = from + threadIdx.x % 4; x < to; x += 4) sum += near[x];
    }
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if (b == 0) sum += (far[0] + far[1]) + (far[2] + far[3]);
    if (b == n - 1) sum += (far[4] + far[5]) + (far[6] + far[7]);
    if (b < n && threadIdx.x % 4 == 0) dst[b] = sum;
    __syncthreads();
    for (int x = threadIdx.x; x < a.tab; x += 256) near[x] = 0.f;
    __syncthreads();
}

// At d = 128 the value fragments of a wavefront's keys are read from LDS in every step, not held in 32 registers: with them two
// wavefronts do not fit a SIMD.
template <int D>
constexpr int kSkew = D == 128 ? 4 : 16;
template <int D>
constexpr int kDkvValues = D == 128 ? 4 * AttnGeo<D>::TILE : 0;

// FEW: where workgroups of 128 keys leave most of the chip empty, 32 keys to a workgroup: its four wavefronts hold the same keys, walk every fourth
// tile of queries each, through a ring of two slots of their own and with no barrier, and their sums meet in LDS once, at the end.  The longest
// walk, which is what small problems take, is a quarter as long, with nothing left to a launch behind.  (7 sequences of up to 257
// tokens, 8 heads of 32 on 4, bias: training step 53.6 -> 39.4 us; backward of 4 x 512 tokens, causal, 8 heads of 64 on 4: 41.8 -> 25.0 us.)
template <int D>
constexpr int kFewPitch = D + 4;  // floats of a row where the sums meet
template <int D>
constexpr int kFewRing = 2 * kDkvSlot<D> > 2 * 32 * kFewPitch<D> * 4 ? 2 * kDkvSlot<D> : 2 * 32 * kFewPitch<D> * 4;  // per wavefront

// What a wavefront has summed of the bias' gradient of one query head is added up by buckets into dst (LDS), and the sums begin anew.
__device__ __forceinline__ void flush_bias_wave(const AttnArgs &a, const int *bounds, float *near, float lo, float hi, float *dst, int lane) {
    for (int x = 32; x > 0; x /= 2) {
        lo += __shfl_xor(lo, x);
        hi += __shfl_xor(hi, x);
    }
    asm volatile("" ::: "memory");  // (lanes read what others wrote, in order)
    const int n = a.n_buckets;
    for (int b = lane / 4; b < (n + 15) / 16 * 16; b += 16) {  // four lanes to a bucket
        float sum = 0.f;
        if (b < n) {
            const int from = b > 0 ? bias_entry(a, bounds[b - 1]) : 0, to = b < n - 1 ? bias_entry(a, bounds[b]) : a.tab;
            for (int x = from + lane % 4; x < to; x += 4) sum += near[x];
        }
        sum += __shfl_xor(sum, 1);
        sum += __shfl_xor(sum, 2);
        if (b == 0) sum += lo;
        if (b == n - 1) sum += hi;
        if (b < n && lane % 4 == 0) dst[b] = sum;
    }
    asm volatile("" ::: "memory");
    for (int x = lane; x < a.tab; x += 64) near[x] = 0.f;
    asm volatile("" ::: "memory");
}

template <int D, bool BIAS, bool FEW>
__global__ __launch_bounds__(256, FEW && D == 128 ? 1 : 2) void attn_dkv_kernel(AttnArgs a) {
    using G = AttnGeo<D>;
    constexpr bool V_LDS = !FEW && kDkvValues<D> > 0;
    constexpr int KEYS = FEW ? 32 : 128;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5;
    const int head_kv = blockIdx.x % a.h_kv, place = blockIdx.x / a.h_kv;
    const int part = FEW ? 0 : place % a.parts;
    int tile = 0, seq;
    Sequence s = {};
    const bool none = !find_tile<true>(a, 1, KEYS, FEW ? place : place / a.parts, s, tile, seq);
    const int j_wg = tile * KEYS;
    const int j0 = j_wg + (FEW ? 0 : wave * 32), j = j0 + (lane & 31);
    const bool live = j < s.n_k;
    // query tiles of 32: those of a head from the first that sees a key of this workgroup on, head after head
    const int n_t = (s.n_q + 31) / 32, t0 = a.causal ? min(max(j_wg - s.shift, 0) / 32, n_t) : 0;
    const int n_all = !none && j_wg < s.n_k ? a.group * (n_t - t0) : 0, per = FEW ? n_all : uniform((n_all + a.parts - 1) / a.parts);
    const int i_begin = part * per, i_end = min(i_begin + per, n_all);
    float *sums = BIAS && a.part_bias != nullptr ? a.part_bias + ((int64_t)place * a.h_q + head_kv * a.group) * a.n_buckets : nullptr;
    if (BIAS && sums != nullptr && (!FEW || none)) {  // heads that this part does not walk
        const int g_first = i_begin < i_end ? i_begin / (n_t - t0) : a.group, g_last = i_begin < i_end ? (i_end - 1) / (n_t - t0) : -1;
        for (int i = threadIdx.x; i < a.group * a.n_buckets; i += 256) {
            const int g = i / a.n_buckets;
            if (g < g_first || g > g_last) sums[i] = 0.f;
        }
    }
    if (none) return;
    // in LDS behind the tiles: the bias; of its gradient: sums of the wavefronts' far tiles, sums by distance, skewed tiles (FEW: sums by distance,
    // skewed tiles, sums by head and bucket)
    char *ring = lds + (FEW ? wave * kFewRing<D> : 0);
    float *tab = reinterpret_cast<float *>(lds + (FEW ? 4 * kFewRing<D> : kDkvLds<D> + kDkvValues<D>));
    float *far = tab + a.group * (a.tab + a.n_buckets) + kMaxBuckets, *near = FEW ? far : far + 8;
    float *skew = near + 4 * a.tab + wave * (Skew<kSkew<D>>::BYTES / 4), *by_bucket = near + 4 * a.tab + Skew<kSkew<D>>::BYTES;
    if (FEW && BIAS && sums != nullptr) {  // (each wavefront its own)
        for (int x = lane; x < a.tab; x += 64) near[wave * a.tab + x] = 0.f;
        for (int x = lane; x < Skew<kSkew<D>>::BYTES / 4; x += 64) skew[x] = 0.f;
        for (int x = lane; x < a.group * a.n_buckets; x += 64) by_bucket[wave * a.group * a.n_buckets + x] = 0.f;
    }
    bf16x8 kf[G::NS], vf[V_LDS ? 1 : G::NS];
    f32x16 dk[G::ND], dv[G::ND];
#pragma unroll
    for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) dk[dt][i] = dv[dt][i] = 0.f;
    if (i_begin < i_end) {
        const uint32_t q_row = (uint32_t)a.qs[0] * 2, o_row = (uint32_t)a.os[0] * 2;
        const CopyLane<D> c(lane);
        constexpr int STEP = FEW ? 1 : G::COPIES < 4 ? G::COPIES : 4, RING = FEW ? 2 : kDkvRing<D>, STRIDE = FEW ? 4 : 1;
        // tile i of the walk goes to slot (i - i_begin) / STRIDE of the ring
        auto copy_tile = [&](int i, int g, int qt) {
            char *at = ring + ((i - i_begin) / STRIDE & (RING - 1)) * kDkvSlot<D>;
            const int head = head_kv * a.group + g, avail = s.n_q - 32 * qt;
            const int64_t row = s.q0 + 32 * qt;
            copy_rows<D, 32, STEP>(reinterpret_cast<const char *>(a.q + row * a.qs[0] + head * a.qs[1]), q_row, avail, at, wave % STEP, c);
            copy_rows<D, 32, STEP>(reinterpret_cast<const char *>(a.dout + row * a.os[0] + head * a.os[1]), o_row, avail, at + G::TILE,
                                   wave % STEP, c);
            if (FEW || wave == 0)
                copy_256_to_lds(a.aux + (int64_t)head * a.n_q + row, min(lane & 31, avail - 1) * 8 + hh * 4, at + 2 * G::TILE);
        };
        const int i_first = i_begin + (FEW ? wave : 0);
        int g = uniform(i_first / (n_t - t0)), qt = t0 + uniform(i_first % (n_t - t0)), g_copy = g, qt_copy = qt, i_copy = i_first;
        auto copy_next = [&] {
            copy_tile(i_copy, g_copy, qt_copy);
            i_copy += STRIDE;
            qt_copy += STRIDE;
            if constexpr (FEW) {
                while (qt_copy >= n_t) {
                    qt_copy -= n_t - t0;
                    ++g_copy;
                }
            } else if (qt_copy == n_t) {
                qt_copy = t0;
                ++g_copy;
            }
        };
        for (int n = 0; n < RING / 2 && i_copy < i_end; ++n) copy_next();
        char *values = lds + kDkvLds<D> + wave * G::TILE + lane * 16;  // of this lane: D / 16 pieces of 16 bytes, 1 KB apart
        float lo = 0.f, hi = 0.f;
        if (BIAS) {
            expand_bias(a, head_kv, tab, 256);
            if (!FEW && sums != nullptr)
                for (int i = threadIdx.x; i < 4 * a.tab + Skew<kSkew<D>>::BYTES; i += 256) near[i] = 0.f;  // (and the four wavefronts' skews)
        }
        const int jc = min(j, s.n_k - 1);
        const uint16_t *kp = a.k + (s.k0 + jc) * a.ks[0] + head_kv * a.ks[1] + 8 * hh;
        const uint16_t *vp = a.v + (s.k0 + jc) * a.vs[0] + head_kv * a.vs[1] + 8 * hh;
#pragma unroll
        for (int ks = 0; ks < G::NS; ++ks) {
            kf[ks] = *reinterpret_cast<const bf16x8 *>(kp + 16 * ks);
            if constexpr (V_LDS)
                *reinterpret_cast<bf16x8 *>(values + ks * 1024) = *reinterpret_cast<const bf16x8 *>(vp + 16 * ks);
            else
                vf[ks] = *reinterpret_cast<const bf16x8 *>(vp + 16 * ks);
        }
        const TileLane<D> t(lane);
        if (FEW && BIAS) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wg_barrier();
        }
        for (int i = i_first; i < i_end; i += STRIDE) {
            if constexpr (FEW) {
                if (i_copy < i_end) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // nobody waits for this slot's last reads but this wavefront
                    copy_next();
                    wait_copies<2 * G::COPIES + 1>();
                } else {
                    wait_copies<0>();
                }
            } else if (((i - i_begin) & (RING / 2 - 1)) == 0) {
                // (half the ring's tiles to a barrier, the other half under way)
                wait_copies<0>();
                wg_barrier();
                for (int n = 0; n < RING / 2 && i_copy < i_end; ++n) copy_next();
            }
            int g_next = g, qt_next = qt + STRIDE;
            if constexpr (FEW) {
                while (qt_next >= n_t) {
                    qt_next -= n_t - t0;
                    ++g_next;
                }
            } else if (qt_next == n_t) {
                qt_next = t0;
                ++g_next;
            }
            const int p0 = 32 * qt + s.shift;  // position of the tile's first query
            if (j0 < s.n_k && !(a.causal && p0 + 31 < j0)) {
                const char *at = ring + ((i - i_begin) / STRIDE & (RING - 1)) * kDkvSlot<D>;
                const float *aux = reinterpret_cast<const float *>(at + 2 * G::TILE) + 8 * hh;
                f32x16 p = mfma_rows<D>(splat(0.f), at, t, kf), dp;
                const bool behind = BIAS && j0 + 31 - p0 < a.b0, ahead = BIAS && j0 - p0 - 31 >= a.b_last;
                if (BIAS) {
                    const float *tab_g = tab + g * a.tab;
                    if (behind || ahead) {
                        const float b = tab_g[ahead ? a.tab - 1 : 0];
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[e] = p[e] * a.sl2 + b;
                    } else {
                        const float *entry = tab_g + bias_entry(a, j - p0) - 8 * hh;
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[e] = p[e] * a.sl2 + entry[-acc_row(e, 0)];
                    }
                }
                if (32 * qt + 32 > s.n_q || (a.causal && j0 + 31 > p0)) {
                    // rows of the tile that are queries and see this lane's key
                    const int from = a.causal ? j - p0 : 0, to = s.n_q - 32 * qt;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int row = acc_row(e, hh);
                        if (row < from || row >= to) p[e] = -__builtin_inff();
                    }
                }
                BFrag b[2];
                if constexpr (D == 64) {
                    // Matrix instructions of dP between the exponentials, those of dV between the products P o (dP - D): a wavefront
                    // issues in order, so the two overlap where they alternate (the barriers keep the compiler from regrouping).  3 % of a
                    // training step of 16 heads of 64, 10655 tokens.  Not at d = 32, where it takes the registers of a fourth wavefront on
                    // a SIMD (2 % slower), nor at d = 128, where there are none left (5 %).
                    f32x16 off;
                    bf16x8 f[G::NS];
#pragma unroll
                    for (int e4 = 0; e4 < 16; e4 += 4) {
                        const f32x4 o4 = *reinterpret_cast<const f32x4 *>(aux + 16 * (e4 / 8) + e4 % 8);
                        const f32x4 nd = *reinterpret_cast<const f32x4 *>(aux + 32 + 16 * (e4 / 8) + e4 % 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            off[e4 + e] = o4[e];
                            dp[e4 + e] = nd[e];  // (dP - D: the product is added to -D)
                        }
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n) f[n] = read_row_frag<D>(at + G::TILE, t, n);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n], vf[n], dp, 0, 0, 0);
                        asm volatile("" : "+v"(dp));
#pragma unroll
                        for (int e = 4 * n; e < 4 * n + 4; e += 2) {
                            p[e] = __builtin_amdgcn_exp2f(BIAS ? p[e] - off[e] : p[e] * a.sl2 - off[e]);
                            p[e + 1] = __builtin_amdgcn_exp2f(BIAS ? p[e + 1] - off[e + 1] : p[e + 1] * a.sl2 - off[e + 1]);
                            b[e / 8].u[e / 2 % 4] = pack_bf16(p[e], p[e + 1]);
                            asm volatile("" : "+v"(b[e / 8].u[e / 2 % 4]));
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n) f[n] = read_tr_frag<D>(at + G::TILE, t, n / G::ND, n % G::ND);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        dv[n % G::ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n], b[n / G::ND].v, dv[n % G::ND], 0, 0, 0);
                        asm volatile("" : "+v"(dv[n % G::ND]));
#pragma unroll
                        for (int e = 4 * n; e < 4 * n + 4; ++e) {
                            dp[e] *= p[e];
                            asm volatile("" : "+v"(dp[e]));
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                } else {
#pragma unroll
                    for (int e4 = 0; e4 < 16; e4 += 4) {
                        const f32x4 off = *reinterpret_cast<const f32x4 *>(aux + 16 * (e4 / 8) + e4 % 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e4 + e] = __builtin_amdgcn_exp2f(BIAS ? p[e4 + e] - off[e] : p[e4 + e] * a.sl2 - off[e]);
                    }
                    to_b_operand(p, b);
                    mfma_transposed<D>(dv, at + G::TILE, t, b);
                    // dP - D: the product is added to -D
#pragma unroll
                    for (int e4 = 0; e4 < 16; e4 += 4) {
                        const f32x4 nd = *reinterpret_cast<const f32x4 *>(aux + 32 + 16 * (e4 / 8) + e4 % 8);
#pragma unroll
                        for (int e = 0; e < 4; ++e) dp[e4 + e] = nd[e];
                    }
                    if constexpr (V_LDS) {
#pragma unroll
                        for (int ks = 0; ks < G::NS; ++ks)
                            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_row_frag<D>(at + G::TILE, t, ks),
                                                                         *reinterpret_cast<const bf16x8 *>(values + ks * 1024), dp, 0, 0, 0);
                    } else {
                        dp = mfma_rows<D>(dp, at + G::TILE, t, vf);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) dp[e] *= p[e];
                }
                if (BIAS && sums != nullptr) {
                    if (behind || ahead) {
                        float sum = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum += live ? dp[e] : 0.f;
                        if (behind) lo += sum; else hi += sum;
                    } else {
                        add_by_distance<kSkew<D>>(dp, live, skew, near + wave * a.tab + bias_entry(a, j0 - p0), lane);
                    }
                }
                to_b_operand(dp, b);
                mfma_transposed<D>(dk, at, t, b);
            }
            if (BIAS && sums != nullptr && (g_next != g || i + STRIDE >= i_end)) {
                if constexpr (FEW)
                    flush_bias_wave(a, reinterpret_cast<const int *>(tab + a.group * a.tab), near + wave * a.tab, lo, hi,
                                    by_bucket + (wave * a.group + g) * a.n_buckets, lane);
                else
                    flush_bias(a, near, far, lo, hi, sums + g * a.n_buckets);
                lo = hi = 0.f;
            }
            g = g_next;
            qt = qt_next;
        }
    }
    wait_copies<0>();
    if (!FEW) wg_barrier();
    mfma_settle();
    if constexpr (FEW) {
        // the wavefronts' sums meet
        float *mine = reinterpret_cast<float *>(ring) + (lane & 31) * kFewPitch<D> + 4 * hh;
#pragma unroll
        for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq) {
                *reinterpret_cast<f32x4 *>(mine + 32 * dt + 8 * gq) = f32x4{dk[dt][4 * gq], dk[dt][4 * gq + 1], dk[dt][4 * gq + 2], dk[dt][4 * gq + 3]};
                *reinterpret_cast<f32x4 *>(mine + 32 * kFewPitch<D> + 32 * dt + 8 * gq) =
                    f32x4{dv[dt][4 * gq], dv[dt][4 * gq + 1], dv[dt][4 * gq + 2], dv[dt][4 * gq + 3]};
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
        if (BIAS && sums != nullptr) {
            const int n = a.group * a.n_buckets;
            for (int i = threadIdx.x; i < n; i += 256) sums[i] = (by_bucket[i] + by_bucket[n + i]) + (by_bucket[2 * n + i] + by_bucket[3 * n + i]);
        }
        const int row = threadIdx.x / 8, c0 = 4 * (threadIdx.x % 8);
        if (j0 + row >= s.k_slot) return;
        const bool live = j0 + row < s.n_k;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const float mul = which == 0 ? a.scale : 1.0f;
            uint16_t *dst = (which == 0 ? a.dk + (s.k0 + j0 + row) * a.ks[0] + head_kv * a.ks[1] : a.dv + (s.k0 + j0 + row) * a.vs[0] + head_kv * a.vs[1]) + c0;
#pragma unroll
            for (int ch = 0; ch < D; ch += 32) {
                f32x4 x[4];
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    x[w] = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds + w * kFewRing<D>) + (which * 32 + row) * kFewPitch<D> + c0 + ch);
                const f32x4 y = ((x[0] + x[1]) + (x[2] + x[3])) * mul;
                *reinterpret_cast<uint2 *>(dst + ch) = live ? make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])) : make_uint2(0, 0);
            }
        }
        return;
    }
    if (a.parts == 1) {
        // (a key/value head's rows: the same as query rows of a group of one)
        char *stage = lds + wave * 32 * G::OUT_ROW;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const f32x16(&x)[G::ND] = which == 0 ? dk : dv;
            const float mul = which == 0 ? a.scale : 1.0f;
#pragma unroll
            for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
                for (int gq = 0; gq < 4; ++gq) {
                    uint2 w;
                    w.x = live ? pack_bf16(x[dt][4 * gq] * mul, x[dt][4 * gq + 1] * mul) : 0;
                    w.y = live ? pack_bf16(x[dt][4 * gq + 2] * mul, x[dt][4 * gq + 3] * mul) : 0;
                    *reinterpret_cast<uint2 *>(stage + (lane & 31) * G::OUT_ROW + (32 * dt + 8 * gq + 4 * hh) * 2) = w;
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            constexpr int CH = D / 8, RPP = 64 / CH;
            uint16_t *dst = which == 0 ? a.dk + s.k0 * a.ks[0] + head_kv * a.ks[1] : a.dv + s.k0 * a.vs[0] + head_kv * a.vs[1];
            const int64_t step = which == 0 ? a.ks[0] : a.vs[0];
#pragma unroll
            for (int it = 0; it < 32 / RPP; ++it) {
                const int rr = it * RPP + lane / CH;
                const uint4 w = *reinterpret_cast<const uint4 *>(stage + rr * G::OUT_ROW + (lane % CH) * 16);
                if (j0 + rr < s.k_slot) *reinterpret_cast<uint4 *>(dst + (j0 + rr) * step + 8 * (lane % CH)) = w;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    } else if (j < s.k_slot) {
        const int64_t at = (((int64_t)part * a.n_k + s.k0 + j) * a.h_kv + head_kv) * D + 4 * hh;
        const float z = live ? 1.0f : 0.f, zk = z * a.scale;
#pragma unroll
        for (int dt = 0; dt < G::ND; ++dt)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq) {
                *reinterpret_cast<f32x4 *>(a.part_k + at + 32 * dt + 8 * gq) =
                    f32x4{dk[dt][4 * gq] * zk, dk[dt][4 * gq + 1] * zk, dk[dt][4 * gq + 2] * zk, dk[dt][4 * gq + 3] * zk};
                *reinterpret_cast<f32x4 *>(a.part_v + at + 32 * dt + 8 * gq) =
                    f32x4{dv[dt][4 * gq] * z, dv[dt][4 * gq + 1] * z, dv[dt][4 * gq + 2] * z, dv[dt][4 * gq + 3] * z};
            }
    }
}

// Parts of dQ (Q) or of dK and dV, added in order.  A workgroup: up to 2048 / d rows of a sequence's slot, one head; eight channels to a thread.
template <int D, bool Q>
__global__ __launch_bounds__(256) void attn_sum_parts(AttnArgs a) {
    constexpr int CH = D / 8, ROWS = 256 / CH;
    const int heads = Q ? a.h_q : a.h_kv, n = Q ? a.n_q : a.n_k;
    const int which = Q ? 0 : blockIdx.x % 2, place = Q ? blockIdx.x : blockIdx.x / 2, head = place % heads;
    int tile, seq;
    Sequence s;
    if (!find_tile<!Q>(a, 1, ROWS, place / heads, s, tile, seq)) return;
    const int r = tile * ROWS + threadIdx.x / CH, ch = threadIdx.x % CH, row0 = Q ? s.q0 : s.k0;
    if (r >= (Q ? s.q_slot : s.k_slot)) return;
    if (Q && ch == 0 && r < s.n_q) {
        float2 *at = a.aux + (int64_t)head * n + row0 + r;
        float2 x = at[0];
        for (int p = 1; p < a.parts; ++p) x.y += at[(int64_t)p * heads * n].y;
        at[0] = x;
    }
    const int64_t step = (int64_t)n * heads * D;
    const float *at = (Q ? a.part_q : which == 0 ? a.part_k : a.part_v) + ((int64_t)(row0 + r) * heads + head) * D + 8 * ch;
    f32x4 x = *reinterpret_cast<const f32x4 *>(at), y = *reinterpret_cast<const f32x4 *>(at + 4);
#pragma unroll 4
    for (int p = 1; p < a.parts; ++p) {
        x += *reinterpret_cast<const f32x4 *>(at + p * step);
        y += *reinterpret_cast<const f32x4 *>(at + p * step + 4);
    }
    uint16_t *dst = Q ? a.dq : which == 0 ? a.dk : a.dv;
    const int64_t *stride = Q ? a.qs : which == 0 ? a.ks : a.vs;
    *reinterpret_cast<uint4 *>(dst + (int64_t)(row0 + r) * stride[0] + head * stride[1] + 8 * ch) =
        make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
}

// The bias' gradient: what the workgroups of a head left, added in order (in 64 bits).
__global__ __launch_bounds__(1024) void attn_sum_bias(AttnArgs a) {
    __shared__ double sums[16][kMaxBuckets];
    const int head = blockIdx.x, b = threadIdx.x % 64, way = threadIdx.x / 64;
    double x = 0.;
    if (b < a.n_buckets)
#pragma unroll 4
        for (int i = way; i < a.n_slots; i += 16) x += a.part_bias[((int64_t)i * a.h_q + head) * a.n_buckets + b];
    sums[way][b] = x;
    __syncthreads();
    if (way == 0 && b < a.n_buckets) {
        for (int i = 1; i < 16; ++i) x += sums[i][b];
        const __bf16 y = (__bf16)(float)x;
        a.dbias[head * a.n_buckets + b] = *reinterpret_cast<const uint16_t *>(&y);
    }
}

// bytes of LDS of a workgroup of few keys, few rows
template <int D>
int64_t few_keys_lds(const AttnArgs &a) {
    return 4 * kFewRing<D> + (a.n_buckets > 0 ? (bias_lds_floats(a) + 4 * (int64_t)a.tab + Skew<kSkew<D>>::BYTES + 4 * a.group * a.n_buckets) * 4 : 0);
}
template <int D>
int64_t few_rows_lds(const AttnArgs &a) {
    return kDqFewLds<D> + bias_lds_floats(a) * 4;
}
struct WsLayout {
    int q_slots, k_slots, q_parts, k_parts;
    bool few_rows, few_keys;
    size_t aux, part_q, part_k, part_v, part_bias, total;
};
WsLayout layout(const AttnArgs &a, int d) {
    WsLayout w;
    const int64_t rows = (int64_t)a.n_q * a.group;
    w.q_slots = (int)(rows / 128 + a.n_seq);
    w.k_slots = a.n_k / 128 + a.n_seq;
    const double steps = walk_steps(a), full = full_chip(d);
    // Tiles of 128 rows (keys), their walks cut into parts where there are few, or tiles of 32 with the walks dealt to four wavefronts: what promises to
    // be done first.  Neither takes less than the steps behind each other in its walks, at about twice the cycles of a step on a full chip; for tiles of
    // 32 two steps more, where the wavefronts' sums meet, and all of it as often as the chip has to be filled (with two workgroups to a CU), which they
    // are not for more than two times: each tile is copied for 32 rows instead of 128, at least a fifth of the time on a full chip.
    // Backward, with 128 keys and rows and with 32: 4 x 512 tokens, causal, 8 heads on 4, d = 64 41.8 and 21.8 us, d = 128 66.4 and 41.6; 32 x 64 tokens,
    // 8 heads of 64 (walks of two steps), 15.6 and 21.0; 8 x 900 tokens, 8 heads of 32 (four times the chip), 54 and 62.
    auto choose = [&](double cycles, int64_t n, double bytes, int64_t walk, int64_t grid, int64_t lds, int &parts) {
        const double wgs = ((double)n / 128 + 1) * a.h_kv, step = cycles * 2 / 2.1e3;
        double cut, few;
        parts = best_parts(steps, cycles, wgs, full, bytes, walk, grid, &cut);
        best_parts(steps, cycles, 4 * wgs, full, 0, 0, 0, &few);
        const int64_t at_once = 256 * std::min<int64_t>(2, 160 * 1024 / lds);
        const int64_t times = at_once > 0 ? (n / 32 * a.h_kv + at_once - 1) / at_once : 3;
        few = std::max(1.2 * few, step * ((walk + 3) / 4 + 2) * times);
        cut = std::max(cut, step * walk / parts + (parts > 1 ? 4 : 0));
        return times <= 2 && few <= cut;
    };
    const int64_t rows_lds = d == 32 ? few_rows_lds<32>(a) : d == 64 ? few_rows_lds<64>(a) : few_rows_lds<128>(a);
    const int64_t keys_lds = d == 32 ? few_keys_lds<32>(a) : d == 64 ? few_keys_lds<64>(a) : few_keys_lds<128>(a);
    w.few_rows = choose(d == 32 ? 450 : d == 64 ? 600 : 1050, rows, (double)a.n_q * a.h_q * d * 8, (int64_t)a.n_k / a.n_seq / 32,
                        (int64_t)w.q_slots * a.h_kv, rows_lds, w.q_parts);
    w.few_keys = choose(d == 32 ? 600 : d == 64 ? 800 : 1400, a.n_k, (double)a.n_k * a.h_kv * d * 16, rows / a.n_seq / 32,
                        (int64_t)w.k_slots * a.h_kv, keys_lds, w.k_parts);
    if (w.few_rows) {
        w.q_slots = (int)(rows / 32 + a.n_seq);
        w.q_parts = 1;
    }
    if (w.few_keys) {
        w.k_slots = a.n_k / 32 + a.n_seq;
        w.k_parts = 1;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 256);
        return here;
    };
    w.aux = take((size_t)w.q_parts * a.n_q * a.h_q * 8);
    w.part_q = take(w.q_parts > 1 ? (size_t)w.q_parts * a.n_q * a.h_q * d * 4 : 0);
    w.part_k = take(w.k_parts > 1 ? (size_t)w.k_parts * a.n_k * a.h_kv * d * 4 : 0);
    w.part_v = take(w.k_parts > 1 ? (size_t)w.k_parts * a.n_k * a.h_kv * d * 4 : 0);
    w.part_bias = take(a.n_buckets > 0 ? (size_t)w.k_slots * w.k_parts * a.h_q * a.n_buckets * 4 : 0);
    w.total = at;
    return w;
}

template <int D>
lsrm_status launch_backward_d(AttnArgs a, void *ws, hipStream_t st) {
    const bool bias = a.n_buckets > 0;
    if (a.n_seq > 0) {
        const WsLayout w = layout(a, D);
        char *base = static_cast<char *>(ws);
        a.aux = reinterpret_cast<float2 *>(base + w.aux);
        a.part_q = reinterpret_cast<float *>(base + w.part_q);
        a.part_k = reinterpret_cast<float *>(base + w.part_k);
        a.part_v = reinterpret_cast<float *>(base + w.part_v);
        a.part_bias = a.dbias != nullptr ? reinterpret_cast<float *>(base + w.part_bias) : nullptr;
        const int n_tab = bias_lds_floats(a) * 4;
        a.parts = w.q_parts;
        lsrm_status rc;
        if (w.few_rows)
            rc = launch_attn(bias ? &attn_dq_kernel<D, true, true> : &attn_dq_kernel<D, false, true>, (int64_t)w.q_slots * a.h_kv, 256,
                             (int)few_rows_lds<D>(a), a, st);
        else
            rc = launch_attn(bias ? &attn_dq_kernel<D, true, false> : &attn_dq_kernel<D, false, false>, (int64_t)w.q_slots * a.h_kv * w.q_parts, 256,
                             kDqLds<D> + n_tab, a, st);
        if (rc != LSRM_OK) return rc;
        if (w.q_parts > 1 && (rc = launch_attn(&attn_sum_parts<D, true>, ((int64_t)a.n_q / (2048 / D) + a.n_seq) * a.h_q, 256, 0, a, st)) != LSRM_OK) return rc;
        a.parts = w.k_parts;
        if (w.few_keys)
            rc = launch_attn(bias ? &attn_dkv_kernel<D, true, true> : &attn_dkv_kernel<D, false, true>, (int64_t)w.k_slots * a.h_kv, 256, (int)few_keys_lds<D>(a), a, st);
        else
            rc = launch_attn(bias ? &attn_dkv_kernel<D, true, false> : &attn_dkv_kernel<D, false, false>, (int64_t)w.k_slots * a.h_kv * w.k_parts, 256,
                             kDkvLds<D> + kDkvValues<D> + (bias ? n_tab + 32 + (a.dbias != nullptr ? 16 * a.tab + 4 * Skew<kSkew<D>>::BYTES : 0) : 0), a, st);
        if (rc != LSRM_OK) return rc;
        a.n_slots = w.k_slots * w.k_parts;  // (of the bias' sums)
        if (w.k_parts > 1 && (rc = launch_attn(&attn_sum_parts<D, false>, ((int64_t)a.n_k / (2048 / D) + a.n_seq) * a.h_kv * 2, 256, 0, a, st)) != LSRM_OK) return rc;
    } else {
        a.n_slots = 0;
    }
    if (bias && a.dbias != nullptr) return launch_attn(&attn_sum_bias, a.h_q, 1024, 0, a, st);
    return LSRM_OK;
}

}  // namespace

size_t attn_backward_ws_bytes(const AttnArgs &a, int d) { return a.n_seq > 0 ? layout(a, d).total : 0; }

lsrm_status launch_attn_backward(AttnArgs a, int d, void *ws, hipStream_t st) {
    switch (d) {
        case 32: return launch_backward_d<32>(a, ws, st);
        case 64: return launch_backward_d<64>(a, ws, st);
        default: return launch_backward_d<128>(a, ws, st);
    }
}

}  // namespace lsrm
