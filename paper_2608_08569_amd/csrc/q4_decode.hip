// Decode step (Sec. 3.1 Eq. 1-2, Sec. 3.2.2 Eq. 6) over a 4-bit cache.
//
// Keys are split into chunks of 2^k keys; a workgroup takes one chunk of one
// layer, all KV heads, a wave per KV head (or per share of the chunk where
// there are fewer heads than waves), 32 keys at a time:
//
//   stats    S^T = K Q^T on the matrix cores, the running max and sum of exp2
//            per head, a pair per (chunk, head) to the workspace; the workgroup
//            whose chunk holds slot len quantises the new K and V rows, stores
//            them and takes them from LDS itself;
//   values   the sequence's max and sum from the pairs, the logits again, p,
//            out = P V on the matrix cores, each key's sum over the heads of p
//            and from it Eq. (6) for the chunk's keys;
//   finish   the output rows from the chunks' (not launched when there is one).
//
// The softmax's statistics come before any weight is formed, so the score of
// a key is the sum of its final probabilities in float32, with nothing kept per
// (key, head): forming the logits a second time reads 68 bytes of K again per
// key and KV head (d = 128), mostly from the memory-side cache, where keeping
// eight heads' float32 logits would write and read 64.
//
// K Q^T: v_mfma_scale_f32_16x16x128_f8f6f4 takes K's rows as they lie in the
// cache -- a lane the 16 bytes of a block's codes, its scale byte the
// instruction's scale operand -- so K is never converted.  The queries are its
// e2m3 operand (6 bits), in parts: q = sum over i of part_i 2^(s_i), each part
// the nearest to what the ones before leave, 4 or 5 bits further down.  Four
// parts (bfloat16 queries) leave less than 2^-18 of a block's largest channel
// and nothing of channels within 2^-12 of it; six (float32) less than 2^-28.
// Two parts ride in the head columns that a group of at most 8 heads leaves
// free, two in the contraction steps that a row of 64 channels leaves free.
// The instruction adds these products to float32 precision (errors at most
// 7e-8 of the sum of the products' magnitudes, none while the blocks' scales
// are within 2^6); with e4m3 queries it does not (up to 2e-4), and takes twice
// the time (15.9 against 8.8 ns a SIMD; four 16x16x32 bfloat16 ones and the
// sixteen conversions of K that they need: 65).
//
// P V: v_cvt_scalef32_pk_bf16_fp4 makes exact bfloat16 of V's codes, scale
// included (a lane: d / 16 channels of eight keys), and v_perm_b32 pairs the
// keys.  The accumulator layout of K Q^T (a lane: one head, keys 4 (lane / 16)
// + i of two 16-key tiles) is the operand layout of P V with its eight
// contraction steps taken in that key order, so p goes from one product into
// the other in registers; in a bfloat16 call rounded to bfloat16, of which its
// output has no more bits, in a float32 call as three bfloat16 parts (24 bits).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "q4.h"

namespace {

using vz::SeqItem;
using vz_q4::bf16x8_t;
using vz_q4::Rows;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x6 __attribute__((ext_vector_type(6)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / vz::kWave;
constexpr int kUnit = 32;                 // keys per wave and round
constexpr int kStatsDepth = 4, kValuesDepth = 1;  // units whose loads are in flight per wave
constexpr int kMinChunkLog2 = 5;          // chunks of 32 ..
constexpr int kMaxChunkLog2 = 10;         // .. 1024 keys
constexpr int kHeads = 16;                // head columns of a matrix instruction, and the largest group
constexpr int kBufferDword3 = 0x00020000;  // raw buffer descriptor word 3 (32-bit data format)
constexpr float kLog2e = 1.4426950408889634f;

struct Q4Args {
    const void* q;
    const void* k_new;
    const void* v_new;
    VzQ4Cache c;
    float* score;
    int32_t* pos;
    void* out;
    uint32_t* parts;  // the queries as operands, per (sequence, layer, KV head)
    float2* ml;   // max and sum of exp2 per (layer, head, chunk row, share) [L][Hq][nc_max][shares]
    float* part;  // the chunks' outputs [L][nc_max][shares][Hq][D], each over the sequence's sum of exp2
    int32_t len, next_pos, n_chunks;  // single sequence
    int32_t nc_max;                   // chunk rows per layer
    int32_t log2_chunk, shares;       // keys per chunk; waves that share a KV head's chunk
    int32_t Hq, Hkv, L;
    int64_t plane;
    float scale_log2, gamma;
    VzRagged rag;
};

// Waves that share the chunk of a KV head.
__host__ __device__ inline int shares_of(int Hkv) { return Hkv >= kWaves ? 1 : kWaves / Hkv; }

// ---- chunks of a ragged call (as the helpers of vz_internal.h, for any chunk size) ----
__device__ __forceinline__ int seq_chunks(const VzRagged& r, int s, int lg) {
    const int n = r.len[s];
    return vz::decode_served(r.base[s], r.cap[s], n, r.next_pos[s], r.total) ? (n >> lg) + 1 : 0;
}
// Flat chunk f of a layer, by a whole wave; false when it holds no work.
template <bool RAG>
__device__ __forceinline__ bool resolve_chunk(const Q4Args& a, int f, SeqItem& it, int& c) {
    if constexpr (!RAG) {
        it = SeqItem{0, a.len, a.next_pos, a.n_chunks, 0, 0};
        c = f;
        return f < a.n_chunks;
    } else {
        const VzRagged& r = a.rag;
        const int lane = threadIdx.x % vz::kWave;
        int run = 0;
        for (int s0 = 0; s0 < r.n && run <= a.nc_max; s0 += vz::kWave) {
            const int su = min(s0 + lane, r.n - 1);  // load for every lane, mask after
            const int64_t b = r.base[su];
            const int cp = r.cap[su], ln = r.len[su], np = r.next_pos[su];
            const bool ok = (s0 + lane < r.n) & vz::decode_served(b, cp, ln, np, r.total);
            const int n = ok ? (ln >> a.log2_chunk) + 1 : 0;
            const int incl = vz::wave_incl_scan(n);
            const unsigned long long hit = __ballot(run + incl > f);
            if (hit) {
                const int src = __builtin_ctzll(hit);
                it.n_chunks = __builtin_amdgcn_readlane(n, src);
                it.first = run + __builtin_amdgcn_readlane(incl, src) - it.n_chunks;
                it.s = s0 + src;
                it.len = __builtin_amdgcn_readlane(ln, src);
                it.next_pos = __builtin_amdgcn_readlane(np, src);
                const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(b), src);
                const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), src);
                it.base = static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
                c = f - it.first;
                return it.first + it.n_chunks <= a.nc_max;
            }
            run += __builtin_amdgcn_readlane(incl, vz::kWave - 1);
        }
        return false;
    }
}

// What exp2 is relative to: the max, or 0 where no key has a finite logit.
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

// Places in the workspace.
__device__ __forceinline__ float2* ml_of(const Q4Args& a, int l, int h, int chunk_row) {
    return a.ml + ((static_cast<size_t>(l) * a.Hq + h) * a.nc_max + chunk_row) * a.shares;
}
// Output row of a head of a chunk row's share (channel 0).
__device__ __forceinline__ float* part_of(const Q4Args& a, int l, int chunk_row, int share, int h, int d) {
    return a.part + (((static_cast<size_t>(l) * a.nc_max + chunk_row) * a.shares + share) * a.Hq + h) * d;
}

// A plane's bytes of the keys [k0, k0 + keys) that lie below n.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t keys_of(const uint8_t* plane, int k0, int n, int keys, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(plane) + static_cast<size_t>(k0) * bytes, 0,
                                             __builtin_amdgcn_readfirstlane(min(max(n - k0, 0), keys) * bytes),
                                             kBufferDword3);
}

// Eight floats as the NP bfloat16 parts of a matrix operand: their sum is the
// float to 8 NP bits.
template <int NP>
__device__ __forceinline__ void parts_of(const float (&x)[8], bf16x8_t (&p)[NP]) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __bf16 b = static_cast<__bf16>(r[i]);
            p[k][i] = b;
            r[i] -= static_cast<float>(b);
        }
}

struct KTile {  // a lane's part of 32 keys: key 16 t + lane % 16, its block of 32 channels (lane / 16) % (D / 32)
    uint32_t w[2][4];
    uint32_t s[2];  // the key's scale bytes
};
template <int D>
struct VTile {  // channels D / 16 (lane % 16) .. of keys 4 (lane / 16) + i and 16 further on
    uint32_t w[2][4];
    uint32_t s[2][4];
};

template <int D>
__device__ __forceinline__ int block_of_lane() {
    return (threadIdx.x % vz::kWave >> 4) % (D / vz_q4::kBlock);
}

template <int D>
__device__ __forceinline__ void load_k(KTile& k, const uint8_t* codes, const uint8_t* scales, int k0, int n) {
    using R = Rows<D>;
    const int r16 = threadIdx.x & 15;
    const __amdgpu_buffer_rsrc_t rc = keys_of(codes, k0, n, kUnit, R::kCodes);
    const __amdgpu_buffer_rsrc_t rs = keys_of(scales, k0, n, kUnit, R::kScales);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const auto y = __builtin_amdgcn_raw_buffer_load_b128(rc, (16 * t + r16) * R::kCodes + 16 * block_of_lane<D>(), 0, 0);
        __builtin_memcpy(k.w[t], &y, 16);
        if constexpr (D == 128) k.s[t] = __builtin_amdgcn_raw_buffer_load_b32(rs, (16 * t + r16) * 4, 0, 0);
        else k.s[t] = __builtin_amdgcn_raw_buffer_load_b16(rs, (16 * t + r16) * 2, 0, 0);
    }
}

template <int D>
__device__ __forceinline__ void load_v(VTile<D>& v, const uint8_t* codes, const uint8_t* scales, int k0, int n) {
    using R = Rows<D>;
    const int lane = threadIdx.x % vz::kWave, q4 = lane >> 4, r16 = lane & 15;
    const __amdgpu_buffer_rsrc_t rc = keys_of(codes, k0, n, kUnit, R::kCodes);
    const __amdgpu_buffer_rsrc_t rs = keys_of(scales, k0, n, kUnit, R::kScales);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = 16 * t + 4 * q4 + i, off = key * R::kCodes + D / 32 * r16;
            if constexpr (D == 128) v.w[t][i] = __builtin_amdgcn_raw_buffer_load_b32(rc, off, 0, 0);
            else v.w[t][i] = __builtin_amdgcn_raw_buffer_load_b16(rc, off, 0, 0);
        }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int key = 16 * t + 4 * q4;
        if constexpr (D == 128) {
            const auto y = __builtin_amdgcn_raw_buffer_load_b128(rs, 4 * key, 0, 0);
            __builtin_memcpy(v.s[t], &y, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v.s[t][i] = __builtin_amdgcn_raw_buffer_load_b16(rs, 2 * (key + i), 0, 0);
        }
    }
}

// The group's queries in parts, as operands of products with 16 rows of K:
// lane (q4, r16) holds its block's 32 channels of head r16 (PACK: r16 & 7; zero
// past the group), of product j the part in slot 2 j + (r16 >> 3) (PACK) or j;
// rows of 64 channels take twice as many parts a product, the second half of
// them in lanes q4 = 2, 3.
template <int DT, int D, bool PACK>
struct Queries {
    static constexpr int kParts = DT == VZ_F32 ? 6 : 4;
    static constexpr int kSlots = (PACK ? 2 : 1) * (128 / D);  // parts per product
    static constexpr int kProducts = (kParts + kSlots - 1) / kSlots;
    i32x8 q[kProducts];  // 6 words of 6-bit codes
    int s[kProducts];    // scale bytes
    __device__ __forceinline__ void load(const void* q0, int G) {
        using T = typename vz::Elem<DT>::T;
        const int lane = threadIdx.x % vz::kWave, q4 = lane >> 4, r16 = lane & 15;
        const int h = PACK ? r16 & 7 : r16, slot = (PACK ? r16 >> 3 : 0) + (D == 64 ? q4 >> 1 : 0) * (PACK ? 2 : 1);
        const T* const row = static_cast<const T*>(q0) + static_cast<size_t>(min(h, G - 1)) * D +
                             vz_q4::kBlock * block_of_lane<D>();
        f32x16 lo, hi;      // what is left of the even and odd channels (as the conversion takes them)
        uint32_t bits = 0;  // of the largest magnitude (a NaN's are above infinity's)
        constexpr int PER = vz::Elem<DT>::kPer16B;
#pragma unroll
        for (int i = 0; i < 32 / PER; ++i) {
            uint4 x;
            __builtin_memcpy(&x, row + PER * i, 16);  // any element alignment
            float f[PER];
            vz::unpack16<DT>(x, f);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                (e & 1 ? hi : lo)[(PER * i + e) / 2] = f[e];
                bits = max(bits, __float_as_uint(f[e]) & 0x7FFFFFFFu);
            }
        }
        const float top = __uint_as_float(bits);
        const bool bad = bits >= 0x7F800000u;
        // the first part's scale 2^e: top <= 7 2^e; its error is at most 2^(e - 2), the next one's (at 2^(e - 4))
        // 2^(e - 7), and 2^-5 of that after each further one
        int e = __builtin_amdgcn_frexp_expf(top) - (__builtin_amdgcn_frexp_mantf(top) > 0.875f ? 2 : 3);
        e = min(max(e, -96), 125);  // (every part's scale a normal float)
#pragma unroll
        for (int j = 0; j < kProducts; ++j) {
            q[j] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
            s[j] = 0;
        }
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int ep = e - (p == 0 ? 0 : 5 * p - 1) + 127;
            const float scale = __uint_as_float(static_cast<uint32_t>(ep) << 23);
            const u32x6 c = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(lo, hi, scale);
            if (p + 1 < kParts) {
                const f32x32 v = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(c, scale);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    lo[i] -= v[2 * i];
                    hi[i] -= v[2 * i + 1];
                }
            }
            const bool mine = (kSlots == 1 || p % kSlots == slot) && h < G;
#pragma unroll
            for (int i = 0; i < 6; ++i) q[p / kSlots][i] = mine ? static_cast<int>(c[i]) : q[p / kSlots][i];
            s[p / kSlots] = mine ? (bad ? vz_q4::kNoScale : ep) : s[p / kSlots];
        }
    }
    // to and from the workspace, a word per lane
    static constexpr int kWords = 7 * kProducts * vz::kWave;
    __device__ __forceinline__ void store(uint32_t* to) const {
        to += threadIdx.x % vz::kWave;
#pragma unroll
        for (int j = 0; j < kProducts; ++j)
#pragma unroll
            for (int i = 0; i < 7; ++i) to[(7 * j + i) * vz::kWave] = i < 6 ? q[j][i] : s[j];
    }
    __device__ __forceinline__ void reload(const uint32_t* from) {
        from += threadIdx.x % vz::kWave;
#pragma unroll
        for (int j = 0; j < kProducts; ++j) {
            q[j] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 6; ++i) q[j][i] = static_cast<int>(from[(7 * j + i) * vz::kWave]);
            s[j] = static_cast<int>(from[(7 * j + 6) * vz::kWave]);
        }
    }
};
// The parts of a KV head's queries in the workspace (row: (sequence, layer, KV head)).
template <int DT, int D, bool PACK>
__device__ __forceinline__ uint32_t* parts_of_query(const Q4Args& a, size_t row) {
    return a.parts + row * Queries<DT, D, PACK>::kWords;
}

// Q . K of 32 keys (not yet scaled), -inf for keys at or past n (MASK).  PACK
// (groups of at most 8 heads): set 0 holds head r16 & 7, keys 16 (r16 >> 3) +
// 4 q4 + i, so that every exp2 serves a key and a head that exist; else set t
// holds head r16, keys 16 t + 4 q4 + i.
template <int DT, int D, bool PACK>
__device__ __forceinline__ void dots_of(const KTile& k, const Queries<DT, D, PACK>& q, int k0, int n,
                                        float (&x)[PACK ? 1 : 2][4]) {
    const int lane = threadIdx.x % vz::kWave, q4 = lane >> 4, r16 = lane & 15;
    f32x4 acc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const i32x8 w = {static_cast<int>(k.w[t][0]), static_cast<int>(k.w[t][1]), static_cast<int>(k.w[t][2]),
                         static_cast<int>(k.w[t][3]), 0, 0, 0, 0};
        const int s = static_cast<int>(k.s[t] >> (8 * block_of_lane<D>()));  // (the low byte counts)
        acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = Queries<DT, D, PACK>::kProducts - 1; j >= 0; --j)  // formats: 4 e2m1, 2 e2m3
            acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, q.q[j], acc[t], 4, 2, 0, s, 0, q.s[j]);
    }
    const int half = PACK ? r16 >> 3 : 0;
#pragma unroll
    for (int t = 0; t < (PACK ? 1 : 2); ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (PACK) {
                const float y0 = acc[0][i] + vz::ror16<8>(acc[0][i]), y1 = acc[1][i] + vz::ror16<8>(acc[1][i]);
                x[t][i] = half ? y1 : y0;
            } else {
                x[t][i] = acc[t][i];
            }
        }
    if (k0 + kUnit > n) {
#pragma unroll
        for (int t = 0; t < (PACK ? 1 : 2); ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = k0 + 16 * (t + half) + 4 * q4 + i < n ? x[t][i] : -INFINITY;
    }
}

// Eq. (1) for one KV head, by one wave: the new K and V rows quantised and
// stored at their slot; K's codes and scales also to LDS (row: codes, then
// scales).  Lane: channels 2 lane and 2 lane + 1, a block per 16 lanes.
template <int DT, int D>
__device__ __forceinline__ void append(const Q4Args& a, size_t new_row, size_t slot, uint32_t* s_new) {
    using T = typename vz::Elem<DT>::T;
    using R = Rows<D>;
    const int lane = threadIdx.x % vz::kWave, ch = min(2 * lane, D - 2);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const T* const x = static_cast<const T*>(which ? a.v_new : a.k_new) + new_row * D + ch;
        const float x0 = vz::Elem<DT>::to_f32(x[0]), x1 = vz::Elem<DT>::to_f32(x[1]);
        const float a0 = fabsf(x0), a1 = fabsf(x1);
        float top = a0 < INFINITY && a1 < INFINITY ? fmaxf(a0, a1) : INFINITY;
        top = vz::row16_max(top);
        const vz_q4::Scale s = vz_q4::scale_for(top, 1.0);
        const uint32_t b = vz_q4::code_of(x0, s.unit) | (vz_q4::code_of(x1, s.unit) << 4);
        if (2 * lane < D) {
            uint8_t* const codes = (which ? a.c.vc : a.c.kc) + slot * R::kCodes;
            uint8_t* const scales = (which ? a.c.vs : a.c.ks) + slot * R::kScales;
            codes[lane] = static_cast<uint8_t>(b);
            if (lane % 16 == 0) scales[lane / 16] = static_cast<uint8_t>(s.byte);
            if (which == 0) {
                uint8_t* const s8 = reinterpret_cast<uint8_t*>(s_new);
                s8[lane] = static_cast<uint8_t>(b);
                if (lane % 16 == 0) s8[R::kCodes + lane / 16] = static_cast<uint8_t>(s.byte);
            }
        }
    }
    // the wave's own LDS writes before its reads
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

template <int DT, int D, bool RAG, bool PACK>
__global__ __launch_bounds__(kThreads, 4) void stats_kernel(const Q4Args a) {
    using R = Rows<D>;
    __shared__ __align__(16) uint32_t s_new[kWaves][(R::kCodes + 16) / 4];
    const int l = blockIdx.y;
    SeqItem it;
    int c;
    if (!resolve_chunk<RAG>(a, blockIdx.x, it, c)) return;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / vz::kWave), lane = threadIdx.x % vz::kWave;
    const int q4 = lane >> 4, r16 = lane & 15;
    const int G = a.Hq / a.Hkv, shares = a.shares;
    const int c0 = c << a.log2_chunk, c1 = min(c0 + (1 << a.log2_chunk), it.len + 1);  // the chunk's keys
    const size_t row_sl = static_cast<size_t>(it.s) * a.L + l;
    const bool newest = it.len < c1 && it.len >= c0;
    if (newest && threadIdx.x == 0 && blockIdx.z == 0) a.pos[static_cast<size_t>(l) * a.plane + it.base + it.len] = it.next_pos;
    const int item = blockIdx.z * kWaves + w;
    if (item < a.Hkv * shares) {
        const int g = item / shares, share = item - g * shares;
        const size_t head = (static_cast<size_t>(l) * a.Hkv + g) * a.plane + it.base;
        const uint8_t* const kc = a.c.kc + head * R::kCodes;
        const uint8_t* const ks = a.c.ks + head * R::kScales;
        const size_t row_g = row_sl * a.Hkv + g;
        // the wave's units: 32 keys from c0 + 32 (share + shares i) on
        const int n_units = ((c1 - c0 + kUnit - 1) / kUnit - share + shares - 1) / shares;
        auto unit_key = [&](int i) { return c0 + kUnit * (share + shares * i); };
        KTile kt[kStatsDepth];
        Queries<DT, D, PACK> q;
        q.load(static_cast<const typename vz::Elem<DT>::T*>(a.q) + row_g * G * D, G);
        if (c == 0 && share == 0) q.store(parts_of_query<DT, D, PACK>(a, row_g));
        asm volatile("" ::: "memory");  // (the registers of the parts' making are the loads' then)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < kStatsDepth; ++u) load_k<D>(kt[u], kc, ks, unit_key(u), it.len);
        // the unit that holds the new key, when it is this wave's
        const int u_new = (it.len - c0) / kUnit;
        const bool mine = newest && u_new % shares == share;
        if (mine) append<DT, D>(a, row_g, head + it.len, s_new[w]);
        float m = -INFINITY, ref = 0.f, z = 0.f;
        auto unit = [&](int i, KTile& k) {
            const int k0 = unit_key(i);
            if (mine && k0 + kUnit > it.len) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (k0 + 16 * t + r16 == it.len) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) k.w[t][j] = s_new[w][4 * block_of_lane<D>() + j];
                        k.s[t] = s_new[w][R::kCodes / 4];
                    }
            }
            float x[PACK ? 1 : 2][4];
            dots_of<DT, D, PACK>(k, q, k0, c1, x);
            load_k<D>(k, kc, ks, unit_key(i + kStatsDepth), it.len);  // (past the chunk: nothing)
            m = fmaxf(m, fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])));
            if constexpr (!PACK) m = fmaxf(m, fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
            const float last = ref;
            ref = finite_ref(m) * a.scale_log2;
            z *= __builtin_amdgcn_exp2f(last - ref);
#pragma unroll
            for (int t = 0; t < (PACK ? 1 : 2); ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) z += __builtin_amdgcn_exp2f(fmaf(x[t][e], a.scale_log2, -ref));
        };
        for (int i = 0; i < n_units; i += kStatsDepth) {
#pragma unroll
            for (int u = 0; u < kStatsDepth; ++u)
                if (i + u < n_units) unit(i + u, kt[u]);
        }
        // the lanes that hold a head: exp2 relative to the largest of their references
        m = m == -INFINITY ? -INFINITY : ref;
        float mw = vz::rows_max(m);
        if constexpr (PACK) mw = fmaxf(mw, vz::ror16<8>(mw));
        z *= __builtin_amdgcn_exp2f(m - finite_ref(mw));
        z = vz::rows_sum(z);
        if constexpr (PACK) z += vz::ror16<8>(z);
        if (q4 == 0 && r16 < G) ml_of(a, l, g * G + r16, it.first + c)[share] = make_float2(mw, z);
    }
}

// Sums over the lanes of a DPP row that hold a key's heads, in every lane: all
// 16, or (PACK) the 8 of each half row.
template <bool PACK>
__device__ __forceinline__ float heads_sum(float v) {
    if constexpr (!PACK) return vz::row16_sum(v);
    auto dpp = [](float x, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    v += dpp(v, std::integral_constant<int, 0xB1>{});         // quad_perm [1, 0, 3, 2]
    v += dpp(v, std::integral_constant<int, 0x4E>{});         // quad_perm [2, 3, 0, 1]
    return v + dpp(v, std::integral_constant<int, 0x141>{});  // row_half_mirror
}

// Max and sum of a head's n pairs, by the lanes (of lane number i of `step`)
// that hold the head, in each of them.
template <bool PACK>
__device__ __forceinline__ float2 merge_pairs(const float2* ml, int n) {
    const int lane = threadIdx.x % vz::kWave, q4 = lane >> 4, half = (lane >> 3) & 1;
    constexpr int STEP = PACK ? 8 : 4;
    const int i0 = PACK ? 2 * q4 + half : q4;
    float m = -INFINITY, z = 0.f;
    for (int i = i0; i < n; i += 4 * STEP) {
        float2 p[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            p[u] = ml[min(i + u * STEP, n - 1)];
            if (i + u * STEP >= n) p[u] = make_float2(-INFINITY, 0.f);
        }
        const float mn = fmaxf(fmaxf(fmaxf(p[0].x, p[1].x), fmaxf(p[2].x, p[3].x)), m);
        const float ref = finite_ref(mn);
        z *= __builtin_amdgcn_exp2f(m - ref);
#pragma unroll
        for (int u = 0; u < 4; ++u) z = fmaf(p[u].y, __builtin_amdgcn_exp2f(p[u].x - ref), z);
        m = mn;
    }
    float M = vz::rows_max(m);
    if constexpr (PACK) M = fmaxf(M, vz::ror16<8>(M));
    z *= __builtin_amdgcn_exp2f(m - finite_ref(M));
    z = vz::rows_sum(z);
    if constexpr (PACK) z += vz::ror16<8>(z);
    return make_float2(M, z);
}

template <int DT, int D, bool RAG, bool PACK>
__global__ __launch_bounds__(kThreads, 3) void values_kernel(const Q4Args a) {
    using R = Rows<D>;
    using E = vz::Elem<DT>;
    constexpr int NP = DT == VZ_F32 ? 3 : 1;                     // bfloat16 parts of p
    constexpr int NC = D / 16;                                   // channels per lane of V and of an output row
    constexpr int KEYS_PER_THREAD = (1 << kMaxChunkLog2) / kThreads;
    __shared__ float s_sum[kWaves][1 << kMaxChunkLog2];  // per key: the sum of p over a wave's heads
    const int l = blockIdx.y;
    SeqItem it;
    int c;
    if (!resolve_chunk<RAG>(a, blockIdx.x, it, c)) return;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / vz::kWave), lane = threadIdx.x % vz::kWave;
    const int q4 = lane >> 4, r16 = lane & 15;
    const int hc = PACK ? r16 & 7 : r16, half = PACK ? r16 >> 3 : 0;  // the lane's head, and 16 keys of a unit
    const int G = a.Hq / a.Hkv, shares = a.shares, items = a.Hkv * shares;
    const int c0 = c << a.log2_chunk, c1 = min(c0 + (1 << a.log2_chunk), it.len + 1);
    const size_t row_sl = static_cast<size_t>(it.s) * a.L + l;
    const int rows = it.n_chunks * shares;  // pairs and partial outputs of a head
    float total[KEYS_PER_THREAD];
#pragma unroll
    for (int i = 0; i < KEYS_PER_THREAD; ++i) total[i] = 0.f;
    for (int first = 0; first < items; first += kWaves) {
        const int item = first + w;
        if (item < items) {
            const int g = item / shares, share = item - g * shares;
            const size_t head = (static_cast<size_t>(l) * a.Hkv + g) * a.plane + it.base;
            const uint8_t* const kc = a.c.kc + head * R::kCodes;
            const uint8_t* const ks = a.c.ks + head * R::kScales;
            const uint8_t* const vc = a.c.vc + head * R::kCodes;
            const uint8_t* const vs = a.c.vs + head * R::kScales;
            const int n_units = ((c1 - c0 + kUnit - 1) / kUnit - share + shares - 1) / shares;
            auto unit_key = [&](int i) { return c0 + kUnit * (share + shares * i); };
            KTile kt[kValuesDepth];
            VTile<D> vt[kValuesDepth];
            Queries<DT, D, PACK> q;
            q.reload(parts_of_query<DT, D, PACK>(a, row_sl * a.Hkv + g));
#pragma unroll
            for (int u = 0; u < kValuesDepth; ++u) {
                load_k<D>(kt[u], kc, ks, unit_key(u), c1);
                load_v<D>(vt[u], vc, vs, unit_key(u), c1);
            }
            const float2 st = merge_pairs<PACK>(ml_of(a, l, g * G + min(hc, G - 1), it.first), rows);
            // (columns past the group: weights and sums of 0)
            const float ref = hc < G ? finite_ref(st.x) : INFINITY;
            const float inv_z = hc < G ? 1.0f / st.y : 0.f;
            f32x4 acc[NC];
#pragma unroll
            for (int t = 0; t < NC; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int rot = vz_q4::scale_rot(NC * r16 / vz_q4::kBlock);
            auto unit = [&](int u, KTile& k, VTile<D>& v) {
                const int k0 = unit_key(u);
                float x[PACK ? 1 : 2][4];
                dots_of<DT, D, PACK>(k, q, k0, c1, x);
                load_k<D>(k, kc, ks, unit_key(u + kValuesDepth), c1);  // (past the chunk: nothing)
                float p[8];
#pragma unroll
                for (int t = 0; t < (PACK ? 1 : 2); ++t) {
                    float ks4[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[4 * t + i] = __builtin_amdgcn_exp2f(fmaf(x[t][i], a.scale_log2, -ref));
                        ks4[i] = heads_sum<PACK>(p[4 * t + i] * inv_z);
                    }
                    const float sum = (r16 & 2) ? ((r16 & 1) ? ks4[3] : ks4[2]) : ((r16 & 1) ? ks4[1] : ks4[0]);
                    if ((r16 & 7) < 4 && (PACK || r16 < 4))
                        s_sum[w][k0 - c0 + 16 * (t + half) + 4 * q4 + (r16 & 3)] = sum;
                }
                if constexpr (PACK) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[4 + i] = vz::ror16<8>(p[i]);
                }
                bf16x8_t pp[NP];
                parts_of<NP>(p, pp);
                // channels 2 b and 2 b + 1 of the eight keys, then the keys of a channel side by side
                float vs8[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) vs8[e] = vz_q4::scale_of(v.s[e / 4][e % 4], rot);
                auto channels = [&](auto byte) {
                    constexpr int B = decltype(byte)::value;
                    uint32_t y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = vz_q4::pair_bf16<B>(v.w[e / 4][e % 4], vs8[e]);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const uint32_t sel = t ? 0x07060302u : 0x05040100u;  // the high or the low halves of two words
                        uint4 b;
                        b.x = __builtin_amdgcn_perm(y[1], y[0], sel);
                        b.y = __builtin_amdgcn_perm(y[3], y[2], sel);
                        b.z = __builtin_amdgcn_perm(y[5], y[4], sel);
                        b.w = __builtin_amdgcn_perm(y[7], y[6], sel);
                        bf16x8_t vb;
                        __builtin_memcpy(&vb, &b, 16);
#pragma unroll
                        for (int n = NP - 1; n >= 0; --n)
                            acc[2 * B + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pp[n], vb, acc[2 * B + t], 0, 0, 0);
                    }
                };
                channels(std::integral_constant<int, 0>{});
                channels(std::integral_constant<int, 1>{});
                if constexpr (NC == 8) {
                    channels(std::integral_constant<int, 2>{});
                    channels(std::integral_constant<int, 3>{});
                }
                load_v<D>(v, vc, vs, unit_key(u + kValuesDepth), c1);
            };
            for (int i = 0; i < n_units; i += kValuesDepth) {
#pragma unroll
                for (int u = 0; u < kValuesDepth; ++u)
                    if (i + u < n_units) unit(i + u, kt[u], vt[u]);
            }
            // lane: heads 4 q4 + i, channels NC r16 ..
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int h = 4 * q4 + i;
                const float iz = __shfl(inv_z, h, vz::kWave);  // (lane h of row 0 holds head h)
                if (h < G) {
                    float o[NC];
#pragma unroll
                    for (int t = 0; t < NC; ++t) o[t] = acc[t][i] * iz;
                    if (rows == 1) {
                        typename E::T* const dst = static_cast<typename E::T*>(a.out) +
                            (row_sl * a.Hq + g * G + h) * D + NC * r16;
#pragma unroll
                        for (int t = 0; t < NC; ++t) dst[t] = E::from_f32(o[t]);
                    } else {
                        float* const dst = part_of(a, l, it.first + c, share, g * G + h, D) + NC * r16;
#pragma unroll
                        for (int t = 0; t < NC; ++t) dst[t] = o[t];
                    }
                }
            }
        }
        __syncthreads();
        // the sums of this round's KV heads, in head order
#pragma unroll
        for (int i = 0; i < KEYS_PER_THREAD; ++i) {
            const int key = threadIdx.x + i * kThreads;
            if (c0 + key < c1)
                for (int v = 0; v < kWaves && first + v < items; ++v)
                    if (v % shares == key / kUnit % shares) total[i] += s_sum[v][key];
        }
        __syncthreads();
    }
    float* const sc = a.score + static_cast<size_t>(l) * a.plane + it.base + c0;
#pragma unroll
    for (int i = 0; i < KEYS_PER_THREAD; ++i) {
        const int key = threadIdx.x + i * kThreads;
        if (c0 + key < c1) sc[key] = fmaf(a.gamma, c0 + key < it.len ? sc[key] : 0.f, total[i]);  // (zero pad for the new slot)
    }
}

// One (layer, sequence, head)'s output row from its chunks', thread = channel;
// in a ragged call the sequence's status too.
template <int DT, int D, bool RAG>
__global__ __launch_bounds__(D) void finish_kernel(const Q4Args a) {
    const int l = blockIdx.y, h = blockIdx.x % a.Hq, s = blockIdx.x / a.Hq, t = threadIdx.x;
    int first = 0, nc = a.n_chunks;
    if constexpr (RAG) {
        const int st = vz::ragged_decode_status(a.rag, s);
        nc = seq_chunks(a.rag, s, a.log2_chunk);
        first = vz::ragged_first(s, a.nc_max, [&](int u) { return seq_chunks(a.rag, u, a.log2_chunk); });
        const bool ok = st == VZ_OK && first >= 0 && first + nc <= a.nc_max;
        if (a.rag.status && h == 0 && l == 0 && t == 0)
            a.rag.status[s] = ok ? VZ_OK : (st != VZ_OK ? st : VZ_ERR_CAPACITY);
        if (!ok) return;
    }
    const int rows = nc * a.shares;
    if (rows == 1) return;
    const size_t step = static_cast<size_t>(a.Hq) * D;
    const float* const p = part_of(a, l, first, 0, h, D) + t;
    float o = 0.f;
#pragma unroll 8
    for (int r = 0; r < rows; ++r) o += p[r * step];
    static_cast<typename vz::Elem<DT>::T*>(a.out)[((static_cast<size_t>(s) * a.L + l) * a.Hq + h) * D + t] =
        vz::Elem<DT>::from_f32(o);
}

constexpr int kMostProducts = 6;  // float32, d = 128, groups of more than 8 heads

// Keys per chunk (log2) of a call over `keys` keys per layer: the smallest
// chunks that leave at most kTargetChunks of them over all layers.
constexpr int kTargetChunks = 512, kLeastChunks = 8;
int log2_chunk_for(int32_t L, int64_t keys) {
    const int64_t most = std::max<int64_t>(kLeastChunks, kTargetChunks / L);
    int lg = kMinChunkLog2;
    while (lg < kMaxChunkLog2 && ((keys + (int64_t(1) << lg) - 1) >> lg) > most) ++lg;
    return lg;
}

// Chunk rows per layer that a workspace for planes of `plane` slots holds.
int64_t chunk_rows(int32_t L, int64_t plane, int32_t n_seqs) {
    if (n_seqs > 0) {
        const int lg = log2_chunk_for(L, plane);
        return (plane >> lg) + n_seqs;
    }
    // a single sequence of any length up to the plane's: chunks grow with it
    int64_t most = 0;
    for (int lg = kMinChunkLog2; lg <= kMaxChunkLog2; ++lg) {
        const int64_t limit = std::max<int64_t>(kLeastChunks, kTargetChunks / L) << lg;  // longest at this size
        const int64_t keys = lg == kMaxChunkLog2 ? plane : std::min(plane, limit);
        most = std::max(most, (keys + (int64_t(1) << lg) - 1) >> lg);
    }
    return most;
}

template <int DT, int D, bool RAG, bool PACK>
hipError_t launch(const VzDecodeArgs& v, const VzQ4Cache& c, hipStream_t stream) {
    Q4Args a{};
    a.q = v.q;
    a.k_new = v.k_new;
    a.v_new = v.v_new;
    a.c = c;
    a.pos = v.pos;
    a.score = v.score;
    a.out = v.out;
    a.Hq = v.Hq;
    a.Hkv = v.Hkv;
    a.L = v.L;
    a.plane = RAG ? v.rag.total : v.cap;
    a.nc_max = static_cast<int32_t>(chunk_rows(v.L, a.plane, v.rag.n));
    a.log2_chunk = log2_chunk_for(v.L, RAG ? a.plane : v.len + 1);
    a.shares = shares_of(v.Hkv);
    const size_t rows = static_cast<size_t>(v.L) * a.nc_max * a.shares * v.Hq;
    a.part = static_cast<float*>(v.ws);
    a.ml = reinterpret_cast<float2*>(a.part + rows * D);
    a.parts = reinterpret_cast<uint32_t*>(a.ml + rows);
    static_assert(Queries<DT, D, PACK>::kProducts <= kMostProducts, "room in the workspace");
    a.scale_log2 = (v.sm_scale > 0.f ? v.sm_scale : 1.0f / sqrtf(static_cast<float>(D))) * kLog2e;
    a.gamma = v.gamma;
    a.rag = v.rag;
    int chunks = a.nc_max;
    if (!RAG) {
        a.len = v.len;
        a.next_pos = v.next_pos;
        a.n_chunks = chunks = (v.len >> a.log2_chunk) + 1;
    }
    hipLaunchKernelGGL((stats_kernel<DT, D, RAG, PACK>), dim3(chunks, a.L, (a.Hkv * a.shares + kWaves - 1) / kWaves), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((values_kernel<DT, D, RAG, PACK>), dim3(chunks, a.L), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess || (!RAG && chunks * a.shares == 1)) return e;
    hipLaunchKernelGGL((finish_kernel<DT, D, RAG>), dim3(a.Hq * (RAG ? v.rag.n : 1), a.L), dim3(D), 0, stream, a);
    return hipGetLastError();
}

template <int DT, int D>
hipError_t launch_any(const VzDecodeArgs& v, const VzQ4Cache& c, hipStream_t stream) {
    const bool pack = v.Hq / v.Hkv <= 8;
    if (v.rag.n > 0) return pack ? launch<DT, D, true, true>(v, c, stream) : launch<DT, D, true, false>(v, c, stream);
    return pack ? launch<DT, D, false, true>(v, c, stream) : launch<DT, D, false, false>(v, c, stream);
}

}  // namespace

size_t vz_decode_q4_ws_bytes(int32_t L, int32_t Hq, int32_t Hkv, int32_t d, int64_t plane, int32_t n_seqs) {
    const size_t rows = static_cast<size_t>(L) * chunk_rows(L, plane, n_seqs) * shares_of(Hkv) * Hq;
    const size_t queries = static_cast<size_t>(std::max(n_seqs, 1)) * L * Hkv;
    return rows * (d * sizeof(float) + sizeof(float2)) + queries * 7 * kMostProducts * vz::kWave * sizeof(uint32_t);
}

hipError_t vz_launch_decode_q4(const VzDecodeArgs& a, const VzQ4Cache& c, hipStream_t stream) {
    if (a.dtype == VZ_BF16 && a.d == 128) return launch_any<VZ_BF16, 128>(a, c, stream);
    if (a.dtype == VZ_BF16 && a.d == 64) return launch_any<VZ_BF16, 64>(a, c, stream);
    if (a.dtype == VZ_F32 && a.d == 128) return launch_any<VZ_F32, 128>(a, c, stream);
    if (a.dtype == VZ_F32 && a.d == 64) return launch_any<VZ_F32, 64>(a, c, stream);
    return hipErrorInvalidValue;
}
