// C boundary of liblsrm: argument validation and dispatch.  See include/lsrm.h for the
// meaning, layout and ownership of every argument.
#include <vector>

#include <cmath>

#include "attn_internal.h"

namespace lsrm {

lsrm_status make_shape(const lsrm_nsa_params *p, Shape *s) {
    if (p == nullptr || s == nullptr) return LSRM_ERR_INVALID_ARG;
    if (p->n_obj < 0 || p->n_views < 0 || p->grid < 0 || p->h_q <= 0 || p->h_kv <= 0 || p->d <= 0 || p->topk < 0 ||
        p->window < 0 || p->n_seg < 0)
        return LSRM_ERR_INVALID_ARG;
    if (p->n_obj % kBlock != 0 || p->grid % 8 != 0 || (p->window & 1) != 0) return LSRM_ERR_INVALID_ARG;
    if (!(p->scale >= 0.0f) || __builtin_isinf(p->scale)) return LSRM_ERR_INVALID_ARG;
    if (p->h_q % p->h_kv != 0 || (p->gate_channels != 0 && p->gate_channels != 1)) return LSRM_ERR_INVALID_ARG;
    if (p->window_mode != 0 && p->window_mode != 1) return LSRM_ERR_INVALID_ARG;
    if (p->kv_packed != 0 && p->kv_packed != 1) return LSRM_ERR_INVALID_ARG;
    if (p->block != kBlock || (p->d != 32 && p->d != 64 && p->d != 128) || p->topk > 128) return LSRM_ERR_UNSUPPORTED;
    int64_t n_img = (int64_t)p->n_views * p->grid * p->grid;
    int64_t n = (int64_t)p->n_obj + n_img;
    if (n > (int64_t)1 << 30) return LSRM_ERR_UNSUPPORTED;
    s->n_obj = p->n_obj;
    s->n_views = p->n_views;
    s->grid = p->grid;
    s->h = p->h_q;
    s->h_kv = p->h_kv;
    s->gate_channels = p->gate_channels;
    s->d = p->d;
    s->topk = p->topk;
    s->own_block = p->window_mode == 1;
    s->window = s->own_block ? 128 : p->window;
    s->count = p->d_block_count;
    s->kv_packed = p->kv_packed;
    s->goff = p->d_group_offsets;
    s->ng = p->d_group_offsets != nullptr ? p->n_groups : 0;
    s->group_window = 0;
    if (s->ng > 0 && p->window_mode == 1) {
        // the window is the query's spatial block: a sliding window without reach limit inside per-block segments
        s->own_block = 0;
        s->group_window = 1;
        s->window = 1 << 30;
    }
    s->nb_obj = p->n_obj / kBlock;
    s->tiles_per_view = (p->grid / 8) * (p->grid / 8);
    s->n_tiles = p->n_views * s->tiles_per_view;
    s->nb = s->nb_obj + s->n_tiles;
    if (p->d_group_offsets != nullptr ? (p->n_groups < 1 || p->n_groups > s->nb) : p->n_groups != 0) return LSRM_ERR_INVALID_ARG;
    s->nbc = s->ng > 0 ? s->ng : s->nb;
    s->n = n;
    s->scale = p->scale > 0.0f ? p->scale : 1.0f / __builtin_sqrtf((float)p->d);
    return LSRM_OK;
}

// Segment offsets for the window: the caller's, validated, or the default split into
// [objects], [view 0], [view 1], ...
static lsrm_status make_segments(const lsrm_nsa_params *p, const Shape &s, std::vector<int32_t> *seg) {
    seg->clear();
    if (p->seg_offsets == nullptr) {
        seg->push_back(0);
        if (s.n_obj > 0) seg->push_back(s.n_obj);
        for (int m = 0; m < s.n_views; ++m)
            if (s.grid > 0) seg->push_back(s.n_obj + (m + 1) * s.grid * s.grid);
        return LSRM_OK;
    }
    if (p->n_seg < 1) return s.n == 0 ? LSRM_OK : LSRM_ERR_INVALID_ARG;
    for (int i = 0; i <= p->n_seg; ++i) {
        int32_t o = p->seg_offsets[i];
        if (o % kBlock != 0) return LSRM_ERR_INVALID_ARG;
        if (i == 0 ? o != 0 : o < seg->back()) return LSRM_ERR_INVALID_ARG;
        seg->push_back(o);
    }
    if (seg->back() != s.n) return LSRM_ERR_INVALID_ARG;
    return LSRM_OK;
}

// {0, 0} or multiples of 8, the rows' such that a 32-bit offset within a stage of 128 rows can hold it
static bool strides_of(const int64_t (&given)[2], int heads, int d, int64_t (&out)[2]) {
    if (given[0] == 0 && given[1] == 0) {
        out[0] = (int64_t)heads * d;
        out[1] = d;
    } else {
        out[0] = given[0];
        out[1] = given[1];
    }
    return out[0] > 0 && out[1] > 0 && out[0] % 8 == 0 && out[1] % 8 == 0 && out[0] <= (int64_t)1 << 24 && out[1] <= (int64_t)1 << 40;
}

lsrm_status make_attn_args(const lsrm_attn_params *p, AttnArgs *a) {
    if (p == nullptr) return LSRM_ERR_INVALID_ARG;
    *a = AttnArgs{};
    if (p->n_q < 0 || p->n_k < 0 || p->n_seq < 0 || p->h_q <= 0 || p->h_kv <= 0 || p->d <= 0) return LSRM_ERR_INVALID_ARG;
    if (p->h_q % p->h_kv != 0 || (p->causal != 0 && p->causal != 1)) return LSRM_ERR_INVALID_ARG;
    if (!(p->scale >= 0.0f) || __builtin_isinf(p->scale)) return LSRM_ERR_INVALID_ARG;
    if (p->n_seq > 0 && p->d_q_offsets == nullptr) return LSRM_ERR_INVALID_ARG;
    if (p->d_k_offsets == nullptr && p->n_k != p->n_q) return LSRM_ERR_INVALID_ARG;
    if (p->n_buckets < 0 || (p->n_buckets > 1 && p->bucket_bounds == nullptr)) return LSRM_ERR_INVALID_ARG;
    if (p->d != 32 && p->d != 64 && p->d != 128) return LSRM_ERR_UNSUPPORTED;
    const int64_t most = (int64_t)1 << 30;
    if (p->n_q > most || p->n_k > most || p->n_q * (p->h_q / p->h_kv) > most) return LSRM_ERR_UNSUPPORTED;
    a->group = p->h_q / p->h_kv;
    // workgroups of up to 512 threads that a launch can have, two for some of these
    const int64_t wgs = (int64_t)1 << 22, rows = p->n_q * a->group;
    if ((rows / 32 + p->n_seq) * p->h_kv > wgs || (p->n_q / 128 + p->n_seq) * p->h_q > wgs || (p->n_k / 128 + p->n_seq) * p->h_kv > wgs)
        return LSRM_ERR_UNSUPPORTED;
    if (!strides_of(p->q_stride, p->h_q, p->d, a->qs) || !strides_of(p->k_stride, p->h_kv, p->d, a->ks) ||
        !strides_of(p->v_stride, p->h_kv, p->d, a->vs) || !strides_of(p->o_stride, p->h_q, p->d, a->os))
        return LSRM_ERR_INVALID_ARG;
    a->n_q = (int)p->n_q;
    a->n_k = (int)p->n_k;
    a->n_seq = p->n_seq;
    a->h_q = p->h_q;
    a->h_kv = p->h_kv;
    a->causal = p->causal;
    a->q_off = p->d_q_offsets;
    a->q_len = p->d_q_lens;
    a->k_off = p->d_k_offsets != nullptr ? p->d_k_offsets : p->d_q_offsets;
    a->k_len = p->d_k_offsets == nullptr && p->d_k_lens == nullptr ? p->d_q_lens : p->d_k_lens;
    a->scale = p->scale > 0.0f ? p->scale : 1.0f / __builtin_sqrtf((float)p->d);
    a->sl2 = a->scale * kLog2e;
    if (__builtin_isinf(a->sl2)) return LSRM_ERR_INVALID_ARG;
    a->n_buckets = p->n_buckets;
    if (p->n_buckets > 0) {
        if (p->n_buckets > kMaxBuckets) return LSRM_ERR_UNSUPPORTED;
        for (int i = 0; i < p->n_buckets - 1; ++i) {
            a->bounds[i] = p->bucket_bounds[i];
            if (a->bounds[i] > 1 << 20 || a->bounds[i] < -(1 << 20)) return LSRM_ERR_UNSUPPORTED;
            if (i > 0 && a->bounds[i] <= a->bounds[i - 1]) return LSRM_ERR_INVALID_ARG;
        }
        a->b0 = p->n_buckets > 1 ? a->bounds[0] : 0;
        a->b_last = p->n_buckets > 1 ? a->bounds[p->n_buckets - 2] : 0;
        if (a->b_last - a->b0 > kMaxBiasSpan) return LSRM_ERR_UNSUPPORTED;
        a->tab = a->b_last - a->b0 + 2 + 2 * kBiasPad;
        if ((int64_t)a->group * a->tab > kMaxBiasEntries) return LSRM_ERR_UNSUPPORTED;
    }
    return LSRM_OK;
}

static bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

}  // namespace lsrm

using namespace lsrm;

extern "C" {

const char *lsrm_strerror(lsrm_status s) {
    switch (s) {
        case LSRM_OK: return "ok";
        case LSRM_ERR_INVALID_ARG: return "invalid argument";
        case LSRM_ERR_UNSUPPORTED: return "unsupported configuration";
        case LSRM_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case LSRM_ERR_HIP: return "HIP runtime error";
        case LSRM_ERR_TOO_LARGE: return "problem exceeds the fixed scratch of the allocation-free entry point";
        default: return "unknown status";
    }
}

size_t lsrm_workspace_bytes(const lsrm_nsa_params *p, int which_call) {
    Shape s;
    if (make_shape(p, &s) != LSRM_OK) return 0;
    switch (which_call) {
        case LSRM_WS_ROUTE: return route_ws_bytes(s);
        case LSRM_WS_FORWARD: return forward_ws_bytes(s);
        case LSRM_WS_BACKWARD: return backward_ws_bytes(s);
        case LSRM_WS_ROUTE_3D: return route3d_ws_bytes(s);
        default: return 0;
    }
}

lsrm_status lsrm_route_blocks(const lsrm_nsa_params *p, const float *d_pos, const lsrm_camera *d_cams, int32_t *d_idx,
                              float *d_dist2, void *d_ws, size_t ws_bytes, void *stream) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    if (s.nb == 0 || s.topk == 0) return LSRM_OK;
    if (d_idx == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.n_obj > 0 && d_pos == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.n_views > 0 && d_cams == nullptr) return LSRM_ERR_INVALID_ARG;
    if (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < route_ws_bytes(s)) return LSRM_ERR_WORKSPACE;
    return launch_route(s, d_pos, d_cams, d_idx, d_dist2, d_ws, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_route_blocks_static(const lsrm_nsa_params *p, const float *d_pos, const lsrm_camera *d_cams,
                                     int32_t *d_idx, float *d_dist2, void *stream) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    if (s.nb == 0 || s.topk == 0) return LSRM_OK;
    if (d_idx == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.n_obj > 0 && d_pos == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.n_views > 0 && d_cams == nullptr) return LSRM_ERR_INVALID_ARG;
    return launch_route_static(s, d_pos, d_cams, d_idx, d_dist2, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_route_blocks_3d(const lsrm_nsa_params *p, const lsrm_route3d_params *r, const float *d_pos,
                                 const float *d_pos_img, const lsrm_camera *d_cams, int32_t *d_idx, float *d_dist2,
                                 void *d_ws, size_t ws_bytes, void *stream) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    if (r == nullptr || r->prefilter < 1 || r->k_v2v < 0 || r->k_v2i < 0 || r->k_i2v < 0 || r->k_i2i < 0 ||
        (r->per_token != 0 && r->per_token != 1))
        return LSRM_ERR_INVALID_ARG;
    if ((int64_t)r->k_v2v + r->k_v2i > s.topk || (int64_t)r->k_i2v + r->k_i2i > s.topk) return LSRM_ERR_INVALID_ARG;
    if (s.nb == 0 || s.topk == 0) return LSRM_OK;
    if (d_idx == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.n_obj > 0 && d_pos == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.n_tiles > 0 && (d_cams == nullptr || d_pos_img == nullptr)) return LSRM_ERR_INVALID_ARG;
    const int pre = r->prefilter < s.tiles_per_view ? r->prefilter : s.tiles_per_view;
    if ((int64_t)s.n_views * pre > 4096) return LSRM_ERR_UNSUPPORTED;
    if (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < route3d_ws_bytes(s)) return LSRM_ERR_WORKSPACE;
    return launch_route_3d(s, *r, d_pos, d_pos_img, d_cams, d_idx, d_dist2, d_ws, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_nsa_compress(const lsrm_nsa_params *p, const uint16_t *d_k, const uint16_t *d_v, uint16_t *d_kc,
                              uint16_t *d_vc, void *stream) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    if (s.nb == 0) return LSRM_OK;
    if (d_k == nullptr || d_v == nullptr || d_kc == nullptr || d_vc == nullptr) return LSRM_ERR_INVALID_ARG;
    if (!aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_kc, 16) || !aligned(d_vc, 16)) return LSRM_ERR_INVALID_ARG;
    return launch_compress(s, d_k, d_v, d_kc, d_vc, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_nsa_compress_pack(const lsrm_nsa_params *p, const uint16_t *d_k, const uint16_t *d_v, uint16_t *d_kc,
                                   uint16_t *d_vc, void *d_ws, size_t ws_bytes, void *stream) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    if (s.nb == 0) return LSRM_OK;
    if (d_k == nullptr || d_v == nullptr || d_kc == nullptr || d_vc == nullptr) return LSRM_ERR_INVALID_ARG;
    if (!aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_kc, 16) || !aligned(d_vc, 16)) return LSRM_ERR_INVALID_ARG;
    if (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < forward_ws_bytes(s)) return LSRM_ERR_WORKSPACE;
    return launch_compress_pack(s, d_k, d_v, d_kc, d_vc, d_ws, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_nsa_forward(const lsrm_nsa_params *p, const uint16_t *d_q, const uint16_t *d_k, const uint16_t *d_v,
                             const uint16_t *d_kc, const uint16_t *d_vc, const int32_t *d_idx, const float *d_gates,
                             uint16_t *d_out, float *d_lse, uint16_t *d_out_branch, void *d_ws, size_t ws_bytes,
                             void *stream, void *ev_attn_start, void *ev_attn_stop) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    std::vector<int32_t> seg;
    rc = make_segments(p, s, &seg);
    if (rc != LSRM_OK) return rc;
    if (s.nb == 0) return LSRM_OK;
    if (d_q == nullptr || d_k == nullptr || d_v == nullptr || d_kc == nullptr || d_vc == nullptr ||
        d_gates == nullptr || d_out == nullptr)
        return LSRM_ERR_INVALID_ARG;
    if (s.topk > 0 && d_idx == nullptr) return LSRM_ERR_INVALID_ARG;
    if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_kc, 16) || !aligned(d_vc, 16) ||
        !aligned(d_out, 16) || (d_out_branch != nullptr && !aligned(d_out_branch, 16)))
        return LSRM_ERR_INVALID_ARG;
    if (s.gate_channels && !aligned(d_gates, 16)) return LSRM_ERR_INVALID_ARG;
    if (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < forward_ws_bytes(s)) return LSRM_ERR_WORKSPACE;
    return launch_forward(s, seg.data(), (int)seg.size() - 1, d_q, d_k, d_v, d_kc, d_vc, d_idx, d_gates, d_out, d_lse,
                          d_out_branch, d_ws, static_cast<hipStream_t>(stream), static_cast<hipEvent_t>(ev_attn_start),
                          static_cast<hipEvent_t>(ev_attn_stop));
}

lsrm_status lsrm_nsa_backward(const lsrm_nsa_params *p, const uint16_t *d_q, const uint16_t *d_k, const uint16_t *d_v,
                              const uint16_t *d_kc, const uint16_t *d_vc, const int32_t *d_idx, const float *d_gates,
                              const float *d_lse, const uint16_t *d_out_branch, const uint16_t *d_dout, uint16_t *d_dq,
                              uint16_t *d_dk, uint16_t *d_dv, void *d_ws, size_t ws_bytes, void *stream, void *ev_start,
                              void *ev_stop) {
    Shape s;
    lsrm_status rc = make_shape(p, &s);
    if (rc != LSRM_OK) return rc;
    std::vector<int32_t> seg;
    rc = make_segments(p, s, &seg);
    if (rc != LSRM_OK) return rc;
    if (s.nb == 0) return LSRM_OK;
    const void *in[] = {d_q, d_k, d_v, d_kc, d_vc, d_out_branch, d_dout, d_dq, d_dk, d_dv};
    for (const void *ptr : in)
        if (ptr == nullptr || !aligned(ptr, 16)) return LSRM_ERR_INVALID_ARG;
    if (d_gates == nullptr || d_lse == nullptr) return LSRM_ERR_INVALID_ARG;
    if (s.gate_channels && !aligned(d_gates, 16)) return LSRM_ERR_INVALID_ARG;
    if (s.topk > 0 && d_idx == nullptr) return LSRM_ERR_INVALID_ARG;
    if (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < backward_ws_bytes(s)) return LSRM_ERR_WORKSPACE;
    return launch_backward(s, seg.data(), (int)seg.size() - 1, d_q, d_k, d_v, d_kc, d_vc, d_idx, d_gates, d_lse,
                           d_out_branch, d_dout, d_dq, d_dk, d_dv, d_ws, static_cast<hipStream_t>(stream),
                           static_cast<hipEvent_t>(ev_start), static_cast<hipEvent_t>(ev_stop));
}

size_t lsrm_attn_workspace_bytes(const lsrm_attn_params *p, int which_call) {
    AttnArgs a;
    if (make_attn_args(p, &a) != LSRM_OK) return 0;
    switch (which_call) {
        case LSRM_WS_FORWARD: return attn_forward_ws_bytes(a, p->d);
        case LSRM_WS_BACKWARD: return attn_backward_ws_bytes(a, p->d);
        default: return 0;
    }
}

lsrm_status lsrm_attn_forward(const lsrm_attn_params *p, const uint16_t *d_q, const uint16_t *d_k, const uint16_t *d_v,
                              const uint16_t *d_bias, uint16_t *d_out, float *d_lse, void *d_ws, size_t ws_bytes, void *stream) {
    AttnArgs a;
    lsrm_status rc = make_attn_args(p, &a);
    if (rc != LSRM_OK) return rc;
    if ((a.n_buckets > 0) != (d_bias != nullptr)) return LSRM_ERR_INVALID_ARG;
    if (a.n_seq == 0 || a.n_q == 0) return LSRM_OK;
    if (d_q == nullptr || d_out == nullptr || (a.n_k > 0 && (d_k == nullptr || d_v == nullptr))) return LSRM_ERR_INVALID_ARG;
    if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_out, 16) || !aligned(d_bias, 2) || !aligned(d_lse, 4))
        return LSRM_ERR_INVALID_ARG;
    const size_t need = attn_forward_ws_bytes(a, p->d);
    if (need > 0 && (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < need)) return LSRM_ERR_WORKSPACE;
    a.q = d_q;
    a.k = d_k;
    a.v = d_v;
    a.bias = d_bias;
    a.out = d_out;
    a.lse = d_lse;
    return launch_attn_forward(a, p->d, d_ws, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_attn_backward(const lsrm_attn_params *p, const uint16_t *d_q, const uint16_t *d_k, const uint16_t *d_v,
                               const uint16_t *d_bias, const uint16_t *d_out, const float *d_lse, const uint16_t *d_dout, uint16_t *d_dq,
                               uint16_t *d_dk, uint16_t *d_dv, uint16_t *d_dbias, void *d_ws, size_t ws_bytes, void *stream) {
    AttnArgs a;
    lsrm_status rc = make_attn_args(p, &a);
    if (rc != LSRM_OK) return rc;
    if ((a.n_buckets > 0) != (d_bias != nullptr) || (d_dbias != nullptr && a.n_buckets == 0)) return LSRM_ERR_INVALID_ARG;
    if (a.n_seq > 0) {
        const void *of_q[] = {d_q, d_out, d_lse, d_dout, d_dq}, *of_k[] = {d_k, d_v, d_dk, d_dv};
        for (const void *x : of_q)
            if ((a.n_q > 0 && x == nullptr) || !aligned(x, x == d_lse ? 4 : 16)) return LSRM_ERR_INVALID_ARG;
        for (const void *x : of_k)
            if ((a.n_k > 0 && x == nullptr) || !aligned(x, 16)) return LSRM_ERR_INVALID_ARG;
    }
    if (!aligned(d_bias, 2) || !aligned(d_dbias, 2)) return LSRM_ERR_INVALID_ARG;
    const size_t need = attn_backward_ws_bytes(a, p->d);
    if (need > 0 && (d_ws == nullptr || !aligned(d_ws, 256) || ws_bytes < need)) return LSRM_ERR_WORKSPACE;
    a.q = d_q;
    a.k = d_k;
    a.v = d_v;
    a.bias = d_bias;
    a.o = d_out;
    a.lse_in = d_lse;
    a.dout = d_dout;
    a.dq = d_dq;
    a.dk = d_dk;
    a.dv = d_dv;
    a.dbias = d_dbias;
    return launch_attn_backward(a, p->d, d_ws, static_cast<hipStream_t>(stream));
}

lsrm_status lsrm_rel_bucket_bounds(int32_t n_side, int32_t max_distance, int32_t two_sided, int32_t *bounds, int32_t *n_bounds) {
    if (bounds == nullptr || n_bounds == nullptr || n_side < 2 || max_distance < 1 || (two_sided != 0 && two_sided != 1))
        return LSRM_ERR_INVALID_ARG;
    if (n_side > (two_sided ? kMaxBuckets / 2 : kMaxBuckets) || max_distance > 1 << 20) return LSRM_ERR_UNSUPPORTED;
    const int single = n_side / 2;  // distances 0 .. single - 1 have a bucket each
    int32_t start[kMaxBuckets];     // start[b]: smallest distance of bucket b
    for (int b = 0; b < n_side; ++b) {
        if (b <= single) {
            start[b] = b;
        } else {
            // the smallest distance with  ln(distance / single) / ln(max_distance / single) (n_side - single) >= b - single;  a distance
            // that the border meets exactly belongs to the higher bucket, whichever way the logarithms were rounded
            const double x = single * std::pow((double)max_distance / single, (double)(b - single) / (n_side - single));
            start[b] = (int32_t)std::ceil(x * (1.0 - 1e-9));
        }
        if (b > 0 && start[b] <= start[b - 1]) return LSRM_ERR_UNSUPPORTED;
    }
    // behind the query: j - position = -distance; a bucket of distances start[b] .. start[b + 1] - 1 begins at -(start[b + 1] - 1)
    int n = 0;
    for (int b = n_side - 2; b >= 0; --b) bounds[n++] = 1 - start[b + 1];
    if (two_sided)
        for (int b = 1; b < n_side; ++b) bounds[n++] = start[b];
    *n_bounds = n;
    return LSRM_OK;
}

}  // extern "C"
