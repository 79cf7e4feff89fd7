// Arguments of the fusion kernels (fuse.hip, and q4_rows.hip for a 4-bit cache).
#pragma once

#include "vz_internal.h"

namespace vz_fuse {

struct FuseArgs {
    const void* k_in;
    const void* v_in;
    const int32_t* off;
    const void* ak;
    const void* av;
    void* k_out;
    void* v_out;
    float* score_out;
    int32_t* pos_out;
    int32_t H;
    int32_t kinds;              // 2: K and V, 1: K only
    int32_t d;                  // row length (the wide-row kernel)
    int32_t T_in, n_spans;      // single sequence
    int64_t in_plane, out_plane;  // rows per (layer, head) plane of the input and of the output
    int32_t blocks_per_seq;     // ragged: span blocks per sequence in grid x
    // ragged batch (n_seqs > 0): sequence s reads input rows in_base[s] ..
    // + T_in[s] and offsets off[off_base[s] .. + n_spans[s]], writes output
    // slots base[s] .. + n_spans[s] (cap[s] slots are its own)
    int32_t n_seqs;
    const int64_t* in_base;
    const int32_t* T_in_s;
    const int64_t* off_base;
    const int32_t* n_spans_s;
    const int64_t* base;
    const int32_t* cap;
    int32_t* status;
    int64_t total_off;
    int32_t max_spans;
};

// Status of sequence s of a ragged fusion (VZ_OK when it can be served,
// VZ_IDLE for an idle slot).
__device__ __forceinline__ int ragged_fuse_status(const FuseArgs& a, int s) {
    const int64_t ib = a.in_base[s], ob = a.off_base[s], b = a.base[s];
    const int T = a.T_in_s[s], n = a.n_spans_s[s], c = a.cap[s];
    if (c == 0) return VZ_IDLE;
    if (T < 0 || n < 0 || c < 1 || ib < 0 || ib > a.in_plane - T || ob < 0 || ob > a.total_off - n - 1 || b < 0 ||
        b > a.out_plane - c)
        return VZ_ERR_INVALID;
    if (n > T) return VZ_ERR_SHAPE;
    if (n > c || n > a.max_spans) return VZ_ERR_CAPACITY;
    return VZ_OK;
}

// The arguments of a single sequence's and of a ragged batch's call, without the outputs.
inline FuseArgs fuse_args(const void* k_in, const void* v_in, int32_t T_in, const int32_t* off, int32_t n_spans,
                          const void* ak, const void* av, float* score_out, int32_t* pos_out, int32_t H, int32_t d,
                          int32_t cap_out) {
    FuseArgs a{};
    a.k_in = k_in;
    a.v_in = v_in;
    a.off = off;
    a.ak = ak;
    a.av = av;
    a.score_out = score_out;
    a.pos_out = pos_out;
    a.H = H;
    a.kinds = v_in ? 2 : 1;
    a.d = d;
    a.T_in = T_in;
    a.n_spans = n_spans;
    a.in_plane = T_in;
    a.out_plane = cap_out;
    return a;
}
inline FuseArgs fuse_args(const VzFuseRaggedArgs& g) {
    FuseArgs a = fuse_args(g.k_in, g.v_in, 0, g.span_off, 0, g.anchor_k, g.anchor_v, g.score_out, g.pos_out, g.Hkv, g.d,
                           0);
    a.in_plane = g.total_in;
    a.out_plane = g.total;
    a.n_seqs = g.n_seqs;
    a.in_base = g.in_base;
    a.T_in_s = g.T_in;
    a.off_base = g.off_base;
    a.n_spans_s = g.n_spans;
    a.base = g.seq_base;
    a.cap = g.cap;
    a.status = g.status;
    a.total_off = g.total_off;
    a.max_spans = g.max_spans;
    return a;
}

}  // namespace vz_fuse
