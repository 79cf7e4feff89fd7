// Stage-2 eviction (Sec. 3.2.2, Eq. 7-9) of a 4-bit cache: the selection of
// select.h on scores and positions, one 1024-thread block per layer (and
// sequence), as in evict.hip; the rows that fill the freed slots are codes and
// scales.  A moved row is d / 32 16-byte pieces of codes and one piece of
// scales, for K and for V of every KV head.
#include <algorithm>
#include <type_traits>

#include "evict_args.h"
#include "q4.h"
#include "q4_calls.h"

namespace {

using namespace vz_sel;
using namespace vz_evict;

// Piece i of the moves of n rows between the slots src[r] -> dst[r] of one
// layer (base: its slot 0's row in the planes; head_rows: rows per KV head).
template <int D>
__device__ __forceinline__ int64_t move_pieces(int n, int Hkv) {
    return static_cast<int64_t>(n) * Hkv * 2 * (vz_q4::Rows<D>::kCodes / 16 + 1);
}
template <int D>
__device__ __forceinline__ void move_piece(const VzQ4Cache& c, size_t base, size_t head_rows, int Hkv,
                                           const int32_t* src, const int32_t* dst, int64_t i) {
    using R = vz_q4::Rows<D>;
    constexpr int CH = R::kCodes / 16, PIECES = CH + 1;
    const int p = static_cast<int>(i % PIECES);
    int64_t t = i / PIECES;
    const int which = static_cast<int>(t & 1);
    t >>= 1;
    const int h = static_cast<int>(t % Hkv), r = static_cast<int>(t / Hkv);
    const size_t row = base + h * head_rows, from = row + src[r], to = row + dst[r];
    if (p < CH) {
        uint8_t* const codes = (which ? c.vc : c.kc) + 16 * p;
        *reinterpret_cast<uint4*>(codes + to * R::kCodes) = *reinterpret_cast<const uint4*>(codes + from * R::kCodes);
    } else {
        using S = std::conditional_t<R::kScales == 4, uint32_t, uint16_t>;
        S* const scales = reinterpret_cast<S*>(which ? c.vs : c.ks);
        scales[to] = scales[from];
    }
}

// The selection and the moves of one layer by the whole block.
template <int D, bool LK, class SH>
__device__ void evict_layer(const SelJob<uint16_t>& job, const VzQ4Cache& c, size_t base, size_t head_rows, SH& sh) {
    auto move = [&](int n_moves, const int32_t* src, const int32_t* dst) -> bool {
        for (int r = threadIdx.x; r < n_moves; r += kSel) {
            job.A[dst[r]] = job.A[src[r]];
            job.P[dst[r]] = job.P[src[r]];
        }
        if (job.inline_kv)
            for (int64_t i = threadIdx.x; i < move_pieces<D>(n_moves, job.Hkv); i += kSel)
                move_piece<D>(c, base, head_rows, job.Hkv, src, dst, i);
        return true;
    };
    // (the element type and row size count for the row moves only, which are done here)
    select_body<kSel, VZ_BF16, 128, LK, SH, false>(job, sh, move);
}

template <int D, bool LK>
__global__ __launch_bounds__(kSel) void select_q4_kernel(const VzEvictArgs a, const VzQ4Cache c,
                                                         int32_t* __restrict__ ws_n, int32_t* __restrict__ ws_src,
                                                         int32_t* __restrict__ ws_dst, int inline_kv) {
    __shared__ SelSh<LK> sh;
    const int l = blockIdx.x;
    const size_t row = static_cast<size_t>(l) * a.cap;
    SelJob<uint16_t> job{};
    job.A = a.score + row;
    job.P = a.pos + row;
    job.src_g = ws_src + row;
    job.dst_g = ws_dst + row;
    job.n_out = ws_n + l;
    job.kept = a.kept_pos_out ? a.kept_pos_out + static_cast<size_t>(l) * a.budget : nullptr;
    job.len = a.len;
    job.budget = a.budget;
    job.n_sink = a.n_sink;
    job.M = a.n_recent;
    job.next_pos = a.next_pos;
    job.Hkv = a.Hkv;
    job.inline_kv = inline_kv;
    evict_layer<D, LK>(job, c, row * a.Hkv, a.cap, sh);
}

template <int D>
__global__ __launch_bounds__(kSel) void select_q4_ragged_kernel(const VzEvictArgs a, const VzQ4Cache c,
                                                                int32_t* __restrict__ ws_n,
                                                                int32_t* __restrict__ ws_src,
                                                                int32_t* __restrict__ ws_dst) {
    __shared__ SelSh<true> sh;
    const int l = blockIdx.x, s = blockIdx.y;
    const VzRagged& r = a.rag;
    int32_t* const n_out = ws_n + static_cast<size_t>(s) * a.L + l;
    const int st = ragged_evict_status(r, s, a.n_sink, a.n_recent, a.kept_pos_out != nullptr);
    const int len = r.len[s], budget = r.budget[s];
    if (l == 0 && threadIdx.x == 0) {
        if (r.status) r.status[s] = st;
        if (a.new_len_out) a.new_len_out[s] = st == VZ_OK && len > budget ? budget : len;
    }
    const int E = len > budget ? len - budget : 0;
    if (st != VZ_OK || (E == 0 && a.kept_pos_out == nullptr)) {
        if (threadIdx.x == 0) *n_out = 0;
        return;
    }
    const size_t row = static_cast<size_t>(l) * r.total + r.base[s];
    SelJob<uint16_t> job{};
    job.A = a.score + row;
    job.P = a.pos + row;
    job.src_g = ws_src + row;
    job.dst_g = ws_dst + row;
    job.n_out = n_out;
    job.kept = a.kept_pos_out ? a.kept_pos_out + row : nullptr;
    job.len = len;
    job.budget = budget;
    job.n_sink = a.n_sink;
    job.M = a.n_recent < 0 ? budget / 5 : a.n_recent;
    job.next_pos = r.next_pos[s];
    job.Hkv = a.Hkv;
    job.inline_kv = E <= kInlineRows ? 1 : 0;
    const size_t base = static_cast<size_t>(l) * a.Hkv * r.total + r.base[s];
    if (len <= kLdsSlots) evict_layer<D, true>(job, c, base, r.total, sh);
    else evict_layer<D, false>(job, c, base, r.total, sh);
}

// Layers with many moved rows: grid (jobs, y); job x = (sequence, layer), whose
// gridDim.y blocks split its moves.
template <int D, bool RAG>
__global__ __launch_bounds__(256) void compact_q4_kernel(const VzEvictArgs a, const VzQ4Cache c,
                                                         const int32_t* __restrict__ ws_n,
                                                         const int32_t* __restrict__ ws_src,
                                                         const int32_t* __restrict__ ws_dst) {
    const int job = blockIdx.x;
    const int n = ws_n[job];
    if (n == 0) return;
    const int l = RAG ? job % a.L : job;
    const int64_t plane = RAG ? a.rag.total : a.cap;
    const int64_t first = RAG ? a.rag.base[job / a.L] : 0;
    const size_t row = static_cast<size_t>(l) * plane + first;
    const int64_t total = move_pieces<D>(n, a.Hkv);
    for (int64_t i = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x; i < total;
         i += static_cast<int64_t>(gridDim.y) * 256)
        move_piece<D>(c, static_cast<size_t>(l) * a.Hkv * plane + first, plane, a.Hkv, ws_src + row, ws_dst + row, i);
}

template <int D>
hipError_t launch(const VzEvictArgs& a, const VzQ4Cache& c, hipStream_t stream) {
    if (a.rag.n > 0) {
        const int64_t jobs = static_cast<int64_t>(a.rag.n) * a.L;
        EvictWs w(a.ws, jobs, a.L, a.rag.total);
        hipLaunchKernelGGL((select_q4_ragged_kernel<D>), dim3(a.L, a.rag.n), dim3(kSel), 0, stream, a, c, w.n, w.src,
                           w.dst);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int gy = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(64, 4096 / jobs)));
        hipLaunchKernelGGL((compact_q4_kernel<D, true>), dim3(static_cast<unsigned>(jobs), gy), dim3(256), 0, stream, a,
                           c, w.n, w.src, w.dst);
        return hipGetLastError();
    }
    const int E = a.len > a.budget ? a.len - a.budget : 0;
    if (E == 0 && a.kept_pos_out == nullptr) return hipSuccess;
    EvictWs w(a.ws, a.L, a.L, a.cap);
    const int inline_kv = E <= kInlineRows ? 1 : 0;
    if (a.len <= kLdsSlots)
        hipLaunchKernelGGL((select_q4_kernel<D, true>), dim3(a.L), dim3(kSel), 0, stream, a, c, w.n, w.src, w.dst,
                           inline_kv);
    else
        hipLaunchKernelGGL((select_q4_kernel<D, false>), dim3(a.L), dim3(kSel), 0, stream, a, c, w.n, w.src, w.dst,
                           inline_kv);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || inline_kv) return e;
    const int64_t pieces = static_cast<int64_t>(E) * a.Hkv * 2 * (vz_q4::Rows<D>::kCodes / 16 + 1);
    const int gy = static_cast<int>(std::min<int64_t>((pieces + 255) / 256, 2048));
    hipLaunchKernelGGL((compact_q4_kernel<D, false>), dim3(a.L, gy), dim3(256), 0, stream, a, c, w.n, w.src, w.dst);
    return hipGetLastError();
}

}  // namespace

hipError_t vz_launch_evict_q4(const VzEvictArgs& a, const VzQ4Cache& c, hipStream_t stream) {
    return a.d == 128 ? launch<128>(a, c, stream) : launch<64>(a, c, stream);
}
