// The pieces of the decode step over a 4-bit cache (q4_decode.hip): chunks of
// keys, a wave's share of K and V, queries and new rows as operands.
//
// K Q^T: v_mfma_scale_f32_16x16x128_f8f6f4 takes K's rows as they lie in the
// cache -- a lane the 16 bytes of a block's codes, its scale byte the
// instruction's scale operand -- so K is never converted.  The queries are its
// e2m3 operand (6 bits), in six parts: q = sum over i of part_i 2^(s_i), each
// part the nearest to what the ones before leave, 4 or 5 bits further down,
// which leaves less than 2^-28 of a block's largest channel.  (Four would hold
// all bits of bfloat16 channels within 2^-10 of it; but a block with one
// large channel, where K holds little, loses what the others say: logits off by
// 2^-18 of it times K.  48 layers of 8193 slots: 71.7 us with four, 72.6 with six.)
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
// the other in registers, as bfloat16 parts: two (16 bits) in a bfloat16 call,
// whose outputs are then off by their own rounding alone (in one part by a fifth
// more, 2.0e-3 of their size for 1.6e-3; 48 layers of 8193 slots: 72.8 us with one,
// 74.2 with two), three (24 bits) in a float32 call.
#pragma once

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "q4.h"
#include "q4_calls.h"

namespace vz_q4 {

using vz::SeqItem;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x6 __attribute__((ext_vector_type(6)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / vz::kWave;
constexpr int kUnit = 32;                  // keys per wave and round
constexpr int kBufferDword3 = 0x00020000;  // raw buffer descriptor word 3 (32-bit data format)
constexpr float kLog2e = 1.4426950408889634f;

struct AttendArgs {
    const void* q;
    const void* k_new;
    const void* v_new;
    VzQ4Cache c;
    float* score;
    int32_t* pos;
    void* out;
    int32_t len, next_pos, n_chunks;  // single sequence
    int32_t nc_max;                   // chunk rows per layer
    int32_t chunk, shares;            // keys per chunk (a multiple of 32); waves that share a KV head's chunk
    int32_t Hq, Hkv, L;
    int64_t plane;
    float scale_log2, gamma;
    VzRagged rag;
};

// Waves that share the chunk of a KV head.
__host__ __device__ inline int shares_of(int Hkv) { return Hkv >= kWaves ? 1 : kWaves / Hkv; }

// ---- chunks of a ragged call (as the helpers of vz_internal.h, for any chunk size) ----
__device__ __forceinline__ int seq_chunks(const VzRagged& r, int s, int chunk) {
    const int n = r.len[s];
    return vz::decode_served(r.base[s], r.cap[s], n, r.next_pos[s], r.total) ? n / chunk + 1 : 0;
}
// Flat chunk f of a layer, by a whole wave; false when it holds no work.
template <bool RAG>
__device__ __forceinline__ bool resolve_chunk(const AttendArgs& a, int f, SeqItem& it, int& c) {
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
            const int n = ok ? ln / a.chunk + 1 : 0;
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
__device__ __forceinline__ int block_of_lane(int lane) {
    return (lane >> 4) % (D / kBlock);
}

template <int D>
__device__ __forceinline__ void load_k(KTile& k, int lane, const uint8_t* codes, const uint8_t* scales, int k0, int n) {
    using R = Rows<D>;
    const int r16 = lane & 15;
    const __amdgpu_buffer_rsrc_t rc = keys_of(codes, k0, n, kUnit, R::kCodes);
    const __amdgpu_buffer_rsrc_t rs = keys_of(scales, k0, n, kUnit, R::kScales);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int off = (16 * t + r16) * R::kCodes + 16 * block_of_lane<D>(lane);
        const auto y = __builtin_amdgcn_raw_buffer_load_b128(rc, off, 0, 0);
        __builtin_memcpy(k.w[t], &y, 16);
        if constexpr (D == 128) k.s[t] = __builtin_amdgcn_raw_buffer_load_b32(rs, (16 * t + r16) * 4, 0, 0);
        else k.s[t] = __builtin_amdgcn_raw_buffer_load_b16(rs, (16 * t + r16) * 2, 0, 0);
    }
}

template <int D>
__device__ __forceinline__ void load_v(VTile<D>& v, int lane, const uint8_t* codes, const uint8_t* scales, int k0,
                                       int n) {
    using R = Rows<D>;
    const int q4 = lane >> 4, r16 = lane & 15;
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
    static constexpr int kParts = 6;
    static constexpr int kSlots = (PACK ? 2 : 1) * (128 / D);  // parts per product
    static constexpr int kProducts = (kParts + kSlots - 1) / kSlots;
    i32x8 q[kProducts];  // 6 words of 6-bit codes
    int s[kProducts];    // scale bytes
    __device__ __forceinline__ void load(const void* q0, int lane, int G) {
        using T = typename vz::Elem<DT>::T;
        const int q4 = lane >> 4, r16 = lane & 15;
        const int h = PACK ? r16 & 7 : r16, slot = (PACK ? r16 >> 3 : 0) + (D == 64 ? q4 >> 1 : 0) * (PACK ? 2 : 1);
        const T* const row = static_cast<const T*>(q0) + static_cast<size_t>(min(h, G - 1)) * D +
                             kBlock * block_of_lane<D>(lane);
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
        e = min(max(e, -102), 126);  // (every part's scale a normal float)
#pragma unroll
        for (int j = 0; j < kProducts; ++j) {
            q[j] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
            s[j] = 0;
        }
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int ep = e - (p == 0 ? 0 : 5 * p - 1) + 127;
            const float scale = __uint_as_float(static_cast<uint32_t>(ep) << 23);
            // Both conversions write registers before they have read all of their sources, and the compiler lets the
            // two overlap (the last part came out wrong, float32 logits off by up to 2^-20 of a block's largest channel):
            // the sources stay in use past them.
            u32x6 c = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(lo, hi, scale);
            asm volatile("" : "+v"(c) : "v"(lo), "v"(hi), "v"(scale));
            if (p + 1 < kParts) {
                f32x32 v = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(c, scale);
                asm volatile("" : "+v"(v) : "v"(c), "v"(scale));
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    lo[i] -= v[2 * i];
                    hi[i] -= v[2 * i + 1];
                }
            }
            const bool mine = (kSlots == 1 || p % kSlots == slot) && h < G;
#pragma unroll
            for (int i = 0; i < 6; ++i) q[p / kSlots][i] = mine ? static_cast<int>(c[i]) : q[p / kSlots][i];
            s[p / kSlots] = mine ? (bad ? kNoScale : ep) : s[p / kSlots];
        }
    }
    // The parts are there from here on, and not formed later, between loads that hold the registers it takes.
    __device__ __forceinline__ void make() {
#pragma unroll
        for (int j = 0; j < kProducts; ++j) {
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                int v = q[j][i];
                asm volatile("" : "+v"(v));
                q[j][i] = v;
            }
            asm volatile("" : "+v"(s[j]));
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
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

// Q . K of 32 keys (not yet scaled), -inf for keys at or past n (MASK).  PACK
// (groups of at most 8 heads): set 0 holds head r16 & 7, keys 16 (r16 >> 3) +
// 4 q4 + i, so that every exp2 serves a key and a head that exist; else set t
// holds head r16, keys 16 t + 4 q4 + i.
template <int DT, int D, bool PACK>
__device__ __forceinline__ void dots_of(const KTile& k, const Queries<DT, D, PACK>& q, int lane, int k0, int n,
                                        float (&x)[PACK ? 1 : 2][4]) {
    const int q4 = lane >> 4, r16 = lane & 15;
    f32x4 acc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const i32x8 w = {static_cast<int>(k.w[t][0]), static_cast<int>(k.w[t][1]), static_cast<int>(k.w[t][2]),
                         static_cast<int>(k.w[t][3]), 0, 0, 0, 0};
        const int s = static_cast<int>(k.s[t] >> (8 * block_of_lane<D>(lane)));  // (the low byte counts)
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
// stored at their slot; K's codes and scales also to LDS (codes, then scales).
// Lane: channels 2 lane and 2 lane + 1, a block per 16 lanes.
template <int D>
constexpr int kNewWords = (Rows<D>::kCodes + 16) / 4;
template <int DT, int D>
__device__ __forceinline__ void append(const AttendArgs& a, int lane, size_t new_row, size_t slot,
                                       uint32_t* s_new) {
    using T = typename vz::Elem<DT>::T;
    using R = Rows<D>;
    const int ch = min(2 * lane, D - 2);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const T* const x = static_cast<const T*>(which ? a.v_new : a.k_new) + new_row * D + ch;
        const float x0 = vz::Elem<DT>::to_f32(x[0]), x1 = vz::Elem<DT>::to_f32(x[1]);
        const float a0 = fabsf(x0), a1 = fabsf(x1);
        float top = a0 < INFINITY && a1 < INFINITY ? fmaxf(a0, a1) : INFINITY;
        top = vz::row16_max(top);
        const Scale s = scale_for(top, 1.0);
        const uint32_t b = code_of(x0, s.unit) | (code_of(x1, s.unit) << 4);
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

// Row `key` of a wave's 32 keys replaced by the new one's in LDS.
template <int D>
__device__ __forceinline__ void put_new_k(KTile& k, int lane, int key, const uint32_t* s_new) {
    const int r16 = lane & 15;
#pragma unroll
    for (int t = 0; t < 2; ++t)
        if (16 * t + r16 == key) {
#pragma unroll
            for (int j = 0; j < 4; ++j) k.w[t][j] = s_new[4 * block_of_lane<D>(lane) + j];
            k.s[t] = s_new[Rows<D>::kCodes / 4];
        }
}

// acc[t] += P V of 32 keys: p of the lane's head (row of the result) and keys
// 16 (e / 4) + 4 (lane / 16) + e % 4, in NP bfloat16 parts; lane: channels
// D / 16 (lane % 16) + t of heads 4 (lane / 16) + i.
template <int NP, int D>
__device__ __forceinline__ void add_values(const float (&p)[8], const VTile<D>& v, int lane, f32x4 (&acc)[D / 16]) {
    const int rot = scale_rot(D / 16 * (lane & 15) / kBlock);
    bf16x8_t pp[NP];
    parts_of<NP>(p, pp);
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = scale_of(v.s[e / 4][e % 4], rot);
    // channels 2 b and 2 b + 1 of the eight keys, then the keys of a channel side by side
    auto channels = [&](auto byte) {
        constexpr int B = decltype(byte)::value;
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = pair_bf16<B>(v.w[e / 4][e % 4], s[e]);
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
    if constexpr (D == 128) {
        channels(std::integral_constant<int, 2>{});
        channels(std::integral_constant<int, 3>{});
    }
}

// The arguments of a call over chunks of `chunk` keys, nc_max rows of them per layer in the workspace.
inline AttendArgs attend_args(const VzDecodeArgs& v, const VzQ4Cache& c, int32_t nc_max, int32_t chunk) {
    AttendArgs a{};
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
    a.plane = v.rag.n > 0 ? v.rag.total : v.cap;
    a.nc_max = nc_max;
    a.chunk = chunk;
    a.shares = shares_of(v.Hkv);
    a.scale_log2 = (v.sm_scale > 0.f ? v.sm_scale : 1.0f / sqrtf(static_cast<float>(v.d))) * kLog2e;
    a.gamma = v.gamma;
    a.rag = v.rag;
    if (v.rag.n == 0) {
        a.len = v.len;
        a.next_pos = v.next_pos;
        a.n_chunks = v.len / chunk + 1;
    }
    return a;
}

}  // namespace vz_q4
