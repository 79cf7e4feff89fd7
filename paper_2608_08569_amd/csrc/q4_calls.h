// The launchers of the 4-bit caches (q4.h: the format).
#pragma once

#include "vz_internal.h"

// The planes: codes [L][Hkv][plane][d / 2], scales [L][Hkv][plane][d / 32].
struct VzQ4Cache {
    uint8_t* kc;
    uint8_t* ks;
    uint8_t* vc;
    uint8_t* vs;
};
hipError_t vz_launch_fuse_q4(const void* k_in, const void* v_in, int32_t T_in, const int32_t* off, int32_t n_spans,
                             const void* ak, const void* av, const VzQ4Cache& out, float* score_out, int32_t* pos_out,
                             int32_t L, int32_t H, int32_t d, int32_t cap_out, int32_t dtype, hipStream_t stream);
hipError_t vz_launch_fuse_q4_ragged(const VzFuseRaggedArgs& g, const VzQ4Cache& out, hipStream_t stream);
hipError_t vz_launch_unpack_q4(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t d, void* out,
                               int32_t dtype, hipStream_t stream);
// (k_cache and v_cache of the arguments are unused)
hipError_t vz_launch_decode_q4(const VzDecodeArgs& a, const VzQ4Cache& c, hipStream_t stream);
size_t vz_decode_q4_ws_bytes(int32_t L, int32_t Hq, int32_t Hkv, int32_t d, int64_t plane, int32_t n_seqs);
// Whether a single sequence's decode launches also run the eviction of the
// len + 1 slots they leave: one eviction, no kept positions asked for.
bool vz_decode_q4_evicts(const VzDecodeArgs& a, int32_t budget, bool kept);
hipError_t vz_launch_evict_q4(const VzEvictArgs& a, const VzQ4Cache& c, hipStream_t stream);
