// Rows into and out of a 4-bit cache.
//
// fuse:   Stage-1 fusion (Sec. 3.2.1, Eq. 4-5) whose rows are quantised where
//         they are formed: x_j = (sum over span j of x_r + n_j a_j) / n_j, then
//         the block scales and codes of q4.h.  A span of length 1 packs its row
//         as it stands, so this is also how full-precision rows enter the cache.
// unpack: the values that codes and scales stand for.
//
// A lane group of d / (16 bytes) lanes owns one (layer, KV head, K-or-V, span),
// each lane 16 contiguous bytes of the row, as in fuse.hip; a block's 32
// channels lie in 4 (bfloat16) or 8 (float32) neighbouring lanes, whose maximum
// is two or three DPP steps.  Sums are 64-bit: sums of bfloat16 and float32
// rows are then exact but for extreme spreads, so a value's code does not turn
// on the order of the rows, and a mean on a code's border is on it here as in
// the definition.  gfx950 adds, compares and converts float64 at the float32
// rate; an element in is an unpacking, a conversion and an addition, one out
// about ten instructions, so the kernel is near both its limits.  48 layers of
// 32,768 rows (4 KV heads of 128, mean span 4): 719 us, 4.8 TB/s; with rows past
// a span added as zeros and every code from comparisons: 946.  Unpacking runs at
// 6.0 TB/s.
#include <algorithm>

#include "fuse_args.h"
#include "q4.h"
#include "q4_calls.h"

namespace {

using vz_fuse::FuseArgs;

constexpr int kSwap1 = 0xB1;        // quad_perm [1, 0, 3, 2]
constexpr int kSwap2 = 0x4E;        // quad_perm [2, 3, 0, 1]
constexpr int kHalfMirror = 0x141;  // row_half_mirror: the other quad of eight lanes

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, 0xF, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, 0xF, 0xF, false);
    return __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
}
// The largest of a block's lanes (4 or 8 neighbours).
template <int BLANES, typename F>
__device__ __forceinline__ F block_max(F v) {
    F o = dpp<kSwap1>(v);
    v = o > v ? o : v;
    o = dpp<kSwap2>(v);
    v = o > v ? o : v;
    if constexpr (BLANES == 8) {
        o = dpp<kHalfMirror>(v);
        v = o > v ? o : v;
    }
    return v;
}
// max(|a|, |b|, c), a NaN being nothing
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, |%1|, |%2|, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// 1 / n to within 2^-51: two Newton steps on the instruction's estimate.
__device__ __forceinline__ double inverse(double n) {
    double r = __builtin_amdgcn_rcp(n);
    r = __builtin_fma(__builtin_fma(-n, r, 1.0), r, r);
    return __builtin_fma(__builtin_fma(-n, r, 1.0), r, r);
}

// acc += the lane's channels of rows b .. e of a plane; O holds the plane's byte offsets.
template <int DT, int D, typename O>
__device__ __forceinline__ void add_rows(const typename vz::Elem<DT>::T* __restrict__ src, int32_t b, int32_t e,
                                         int lane, double (&acc)[vz::Elem<DT>::kPer16B]) {
    constexpr int PER = vz::Elem<DT>::kPer16B;
    constexpr uint32_t STEP = D * sizeof(typename vz::Elem<DT>::T);
    constexpr int ROWS = 8;
    if (b >= e) return;
    const char* const base = reinterpret_cast<const char*>(src);
    O at = static_cast<O>(b) * STEP + lane * 16;
    const O last = static_cast<O>(e - 1) * STEP + lane * 16;
    // eight rows' loads at a time, those past the span reading its last row again and adding nothing
    for (int32_t left = e - b; left > 0; left -= ROWS, at += ROWS * STEP) {
        uint4 x[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const O o = at + u * STEP;
            // (32 bits: the offset may wrap in the plane's last rows)
            x[u] = *reinterpret_cast<const uint4*>(base + (u < left ? o : last));
        }
        // (all loads are on their way before the first branch, behind which the compiler would move each of its own:
        // one layer of 65,536 rows takes 36 us, with four rows in flight 42, with the loads behind their branches 54)
#pragma unroll
        for (int u = 0; u < ROWS; ++u) asm volatile("" : "+v"(x[u].x), "+v"(x[u].y), "+v"(x[u].z), "+v"(x[u].w));
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (u < left) {
                float f[PER];
                vz::unpack16<DT>(x[u], f);
#pragma unroll
                for (int i = 0; i < PER; ++i) acc[i] += f[i];
            }
        }
    }
}

// Codes of sums that are float32 numbers, which those of bfloat16 rows nearly
// always are, come from the conversion instruction (nearest, ties to even, the
// scale's exponent taken off first), applied to x / n rounded to 64 bits and
// then to 32.  That is code_of's answer: x = M g and a border times n, B = m h,
// are multiples of powers of two g and h, where M < 2^24 and x <= 28 n h, so
// they are equal or differ by the smaller of g and h at least, which is more
// than (1 + 2^-24) 2^-24 x for n below 2^19; x / n then is on the border, or more
// than half a float32 step and 2^-48 of it away, and stays on its side.  (Not
// where x / n may lie below the normal floats.)
constexpr double kMostExact = 1 << 19;
constexpr int kFuseThreads = 256;
template <int DT, int D>
constexpr int kSpansPerBlock = kFuseThreads / (D / vz::Elem<DT>::kPer16B);

// The spans of one sequence, and where its rows begin in their planes.
struct Spans {
    int T_in, n_spans;
    const int32_t* off;
    int64_t in_row, out_row;
};

// One block's spans, number bx of its sequence's, in one plane.
template <int DT, int D, bool RAG>
__device__ __forceinline__ void fuse_block(const FuseArgs& a, const VzQ4Cache& out, const Spans& q, int bx, int l,
                                           int h, int which, int thread) {
    using E = vz::Elem<DT>;
    using T = typename E::T;
    using R = vz_q4::Rows<D>;
    constexpr int PER = E::kPer16B;              // elements per 16-byte vector
    constexpr int LANES = D / PER;               // lanes per span row
    constexpr int BLANES = vz_q4::kBlock / PER;  // lanes per block of channels
    const int sub = thread / LANES;
    const int lane = thread % LANES;
    const int T_in = q.T_in, n_spans = q.n_spans;
    const int64_t in_row = q.in_row, out_row = q.out_row;
    const int32_t* const off = q.off;
    const int64_t j = static_cast<int64_t>(bx) * kSpansPerBlock<DT, D> + sub;
    if (j >= n_spans) return;

    int32_t b = off[j], e = off[j + 1];
    b = b < 0 ? 0 : (b > T_in ? T_in : b);
    e = e < b ? b : (e > T_in ? T_in : e);

    const T* const src = static_cast<const T*>(which ? a.v_in : a.k_in) +
                         ((static_cast<size_t>(l) * a.H + h) * static_cast<size_t>(a.in_plane) + in_row) * D;
    double acc[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = 0.0;
    if (T_in <= (INT64_C(1) << 32) / (D * static_cast<int>(sizeof(T))))
        add_rows<DT, D, uint32_t>(src, b, e, lane, acc);
    else
        add_rows<DT, D, uint64_t>(src, b, e, lane, acc);
    const double n = max(e - b, 1);
    const T* anchor = static_cast<const T*>(which ? a.av : a.ak);
    const size_t orow = (static_cast<size_t>(l) * a.H + h) * static_cast<size_t>(a.out_plane) + out_row + j;
    if (anchor) {
        // single sequence: [L][H][n_spans][d]; ragged: laid out like the output
        const size_t arow = RAG ? orow : (static_cast<size_t>(l) * a.H + h) * static_cast<size_t>(n_spans) + j;
        const uint4 x = *reinterpret_cast<const uint4*>(anchor + arow * D + lane * PER);
        float f[PER];
        vz::unpack16<DT>(x, f);
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] = __builtin_fma(n, f[i], acc[i]);
    }
    float sum[PER];
    bool exact = true;  // every sum of this lane is a float32
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        sum[i] = static_cast<float>(acc[i]);
        exact = exact && static_cast<double>(sum[i]) == acc[i];
    }
#pragma unroll
    for (int i = 0; i < PER; i += 2) top = max_abs(sum[i], sum[i + 1], top);
    vz_q4::Scale s = vz_q4::scale_for(block_max<BLANES>(top), n);
    uint32_t w = 0;
    if (__all(exact && s.byte != vz_q4::kNoScale && (s.byte > vz_q4::kMinExp + 127 || top == 0.f) && n < kMostExact)) {
        const double inv = inverse(n);
        const float scale = __uint_as_float(static_cast<uint32_t>(s.byte) << 23);
        float y[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) y[i] = static_cast<float>(acc[i] * inv);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
        if constexpr (PER == 8) {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
        }
    } else {
        double most = 0.0;
        bool fine = true;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            most = __builtin_fmax(most, __builtin_fabs(acc[i]));
            fine = fine && __builtin_fabs(acc[i]) < INFINITY;  // (a NaN is lost in the maximum)
        }
        s = vz_q4::scale_for(block_max<BLANES>(fine ? most : INFINITY), n);
#pragma unroll
        for (int i = 0; i < PER; ++i) w |= vz_q4::code_of(acc[i], s.unit) << (4 * i);
    }
    uint8_t* const codes = (which ? out.vc : out.kc) + orow * R::kCodes;
    if constexpr (PER == 8) {
        *reinterpret_cast<uint32_t*>(codes + 4 * lane) = w;
    } else {  // four codes a lane: the even lane stores its neighbour's too
        const uint32_t other = __builtin_amdgcn_update_dpp(0, static_cast<int>(w), kSwap1, 0xF, 0xF, false);
        if ((lane & 1) == 0) *reinterpret_cast<uint32_t*>(codes + 2 * lane) = w | (other << 16);
    }
    if (lane % BLANES == 0)
        ((which ? out.vs : out.ks) + orow * R::kScales)[lane / BLANES] = static_cast<uint8_t>(s.byte);

    if (which == 0 && h == 0 && lane == 0) {
        const size_t prow = static_cast<size_t>(l) * a.out_plane + out_row + j;
        a.pos_out[prow] = static_cast<int32_t>(j);
        a.score_out[prow] = 0.f;
    }
}

// Grid: (blocks, 2 x KV heads, layers); y: KV head, K or V.
template <int DT, int D>
__global__ __launch_bounds__(kFuseThreads) void fuse_q4_kernel(const FuseArgs a, const VzQ4Cache out) {
    const Spans q{a.T_in, a.n_spans, a.off, 0, 0};
    fuse_block<DT, D, false>(a, out, q, blockIdx.x, blockIdx.z, blockIdx.y >> 1, blockIdx.y & 1, threadIdx.x);
}

// A ragged batch, a workgroup for each block of spans that a sequence may have.
template <int DT, int D>
__global__ __launch_bounds__(kFuseThreads) void fuse_q4_ragged_kernel(const FuseArgs a, const VzQ4Cache out) {
    const int l = blockIdx.z, s = blockIdx.x / a.blocks_per_seq, bx = blockIdx.x - s * a.blocks_per_seq;
    const int st = vz_fuse::ragged_fuse_status(a, s);
    if (a.status && bx == 0 && blockIdx.y == 0 && l == 0 && threadIdx.x == 0) a.status[s] = st;
    if (st != VZ_OK) return;
    const Spans q{a.T_in_s[s], a.n_spans_s[s], a.off + a.off_base[s], a.in_base[s], a.base[s]};
    fuse_block<DT, D, true>(a, out, q, bx, l, blockIdx.y >> 1, blockIdx.y & 1, threadIdx.x);
}

// The same with as many workgroups as fill the GPU: a plane's blocks of spans
// are numbered over its served sequences, and each workgroup takes every
// gridDim.x-th.
template <int DT, int D>
__global__ __launch_bounds__(kFuseThreads, 7) void fuse_q4_batch_kernel(const FuseArgs a, const VzQ4Cache out) {
    constexpr int SPB = kSpansPerBlock<DT, D>;
    const int l = blockIdx.z, lane = threadIdx.x % vz::kWave;
    if (a.status && blockIdx.x == 0 && blockIdx.y == 0 && l == 0)
        for (int s = threadIdx.x; s < a.n_seqs; s += kFuseThreads) a.status[s] = vz_fuse::ragged_fuse_status(a, s);
    // 64 sequences at a time, one per lane: their blocks, and those up to each
    int s0 = 0, before = 0, blocks = 0, upto = 0;
    auto count = [&] {
        const int s = min(s0 + lane, a.n_seqs - 1);
        const bool served = vz_fuse::ragged_fuse_status(a, s) == VZ_OK && s0 + lane < a.n_seqs;
        blocks = served ? (a.n_spans_s[s] + SPB - 1) / SPB : 0;
        upto = vz::wave_incl_scan(blocks);
    };
    count();
    for (int f = blockIdx.x;; f += gridDim.x) {
        while (f >= before + __builtin_amdgcn_readlane(upto, vz::kWave - 1)) {
            before += __builtin_amdgcn_readlane(upto, vz::kWave - 1);
            s0 += vz::kWave;
            if (s0 >= a.n_seqs) return;
            count();
        }
        const int src = __builtin_ctzll(__ballot(before + upto > f));
        const int s = s0 + src;
        const int bx = f - before - __builtin_amdgcn_readlane(upto, src) + __builtin_amdgcn_readlane(blocks, src);
        const Spans q{a.T_in_s[s], a.n_spans_s[s], a.off + a.off_base[s], a.in_base[s], a.base[s]};
        // (what a thread's number gives is formed again each time: over the loop it would take the loads' registers)
        int thread = threadIdx.x;
        asm volatile("" : "+v"(thread));
        fuse_block<DT, D, true>(a, out, q, bx, l, blockIdx.y >> 1, blockIdx.y & 1, thread);
    }
}

// A workgroup that finds no spans costs the time of its dispatch, and the host
// knows no sequence's length.  Many of them outweigh what looking the blocks up
// costs: 12 layers of 16 sequences of up to 9000 tokens (215,000 workgroups), all
// but one of 10: 175 us with a workgroup for each, 67 with 8192; four of 2k-9k
// (53,760): 128 and 129, four of 4938 114 and 129.
constexpr int64_t kFuseMany = 65536, kFuseFill = 8192;
template <int DT, int D>
hipError_t launch(FuseArgs a, const VzQ4Cache& out, int32_t L, hipStream_t stream) {
    constexpr int SPB = kSpansPerBlock<DT, D>;
    const int planes = 2 * a.H;
    if (a.n_seqs > 0) {
        a.blocks_per_seq = std::max(1, (a.max_spans + SPB - 1) / SPB);  // at least one reports the status
        const int64_t blocks = static_cast<int64_t>(a.blocks_per_seq) * a.n_seqs, all = blocks * planes * L;
        if (all <= kFuseMany) {
            const dim3 grid(static_cast<unsigned>(blocks), planes, L);
            hipLaunchKernelGGL((fuse_q4_ragged_kernel<DT, D>), grid, dim3(kFuseThreads), 0, stream, a, out);
        } else {
            const int64_t fill = std::max<int64_t>(1, kFuseFill / (static_cast<int64_t>(planes) * L));
            const dim3 grid(static_cast<unsigned>(std::min(blocks, fill)), planes, L);
            hipLaunchKernelGGL((fuse_q4_batch_kernel<DT, D>), grid, dim3(kFuseThreads), 0, stream, a, out);
        }
        return hipGetLastError();
    }
    if (a.n_spans == 0) return hipSuccess;
    const dim3 grid((a.n_spans + SPB - 1) / SPB, planes, L);
    hipLaunchKernelGGL((fuse_q4_kernel<DT, D>), grid, dim3(kFuseThreads), 0, stream, a, out);
    return hipGetLastError();
}

hipError_t dispatch(const FuseArgs& a, const VzQ4Cache& out, int32_t L, int32_t d, int32_t dtype, hipStream_t stream) {
    if (dtype == VZ_BF16 && d == 128) return launch<VZ_BF16, 128>(a, out, L, stream);
    if (dtype == VZ_BF16 && d == 64) return launch<VZ_BF16, 64>(a, out, L, stream);
    if (dtype == VZ_F32 && d == 128) return launch<VZ_F32, 128>(a, out, L, stream);
    if (dtype == VZ_F32 && d == 64) return launch<VZ_F32, 64>(a, out, L, stream);
    return hipErrorInvalidValue;
}

// One 16-byte piece of the output per thread and round: eight bfloat16 from a
// word of codes, or four float32 from half a word.
constexpr int kUnpackRounds = 4;
template <int DT>
__global__ __launch_bounds__(256) void unpack_kernel(const uint8_t* __restrict__ codes,
                                                     const uint8_t* __restrict__ scales, uint4* __restrict__ out,
                                                     int64_t n) {
    constexpr int PER = vz::Elem<DT>::kPer16B;
    const int64_t i0 = static_cast<int64_t>(blockIdx.x) * (256 * kUnpackRounds) + threadIdx.x;
#pragma unroll
    for (int r = 0; r < kUnpackRounds; ++r) {
        const int64_t i = i0 + r * 256;
        if (i >= n) return;
        const float s = __uint_as_float(static_cast<uint32_t>(scales[i / (vz_q4::kBlock / PER)]) << 23);
        if constexpr (DT == VZ_BF16) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[i];
            out[i] = make_uint4(vz_q4::pair_bf16<0>(w, s), vz_q4::pair_bf16<1>(w, s), vz_q4::pair_bf16<2>(w, s),
                                vz_q4::pair_bf16<3>(w, s));
        } else {
            const uint32_t w = reinterpret_cast<const uint16_t*>(codes)[i];
            const vz_q4::f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
            const vz_q4::f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
            out[i] = make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]),
                                __float_as_uint(b[1]));
        }
    }
}

}  // namespace

hipError_t vz_launch_fuse_q4(const void* k_in, const void* v_in, int32_t T_in, const int32_t* off, int32_t n_spans,
                             const void* ak, const void* av, const VzQ4Cache& out, float* score_out, int32_t* pos_out,
                             int32_t L, int32_t H, int32_t d, int32_t cap_out, int32_t dtype, hipStream_t stream) {
    const FuseArgs a = vz_fuse::fuse_args(k_in, v_in, T_in, off, n_spans, ak, av, score_out, pos_out, H, d, cap_out);
    return dispatch(a, out, L, d, dtype, stream);
}

hipError_t vz_launch_fuse_q4_ragged(const VzFuseRaggedArgs& g, const VzQ4Cache& out, hipStream_t stream) {
    return dispatch(vz_fuse::fuse_args(g), out, g.L, g.d, g.dtype, stream);
}

hipError_t vz_launch_unpack_q4(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t d, void* out,
                               int32_t dtype, hipStream_t stream) {
    const int64_t n = rows * (d / (dtype == VZ_BF16 ? 8 : 4));
    if (n == 0) return hipSuccess;
    const dim3 grid(static_cast<unsigned>((n + 256 * kUnpackRounds - 1) / (256 * kUnpackRounds)));
    if (dtype == VZ_BF16)
        hipLaunchKernelGGL((unpack_kernel<VZ_BF16>), grid, dim3(256), 0, stream, codes, scales,
                           static_cast<uint4*>(out), n);
    else
        hipLaunchKernelGGL((unpack_kernel<VZ_F32>), grid, dim3(256), 0, stream, codes, scales,
                           static_cast<uint4*>(out), n);
    return hipGetLastError();
}
