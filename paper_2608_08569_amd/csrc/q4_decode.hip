// Decode step (Sec. 3.1 Eq. 1-2, Sec. 3.2.2 Eq. 6) over a 4-bit cache.
//
// Keys are split into chunks; a workgroup takes one chunk of one
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
//   finish   the output rows from the chunks' (not launched when there is one),
//            and in a generation step the eviction of one slot: the smallest of
//            the chunks' smallest rank keys, and the moved row.
//
// The softmax's statistics come before any weight is formed, so the score of
// a key is the sum of its final probabilities in float32, with nothing kept per
// (key, head): forming the logits a second time reads 68 bytes of K again per
// key and KV head (d = 128), mostly from the memory-side cache, where keeping
// eight heads' float32 logits would write and read 64 (counted, not measured).
//
// Bound by reading K twice and V once.  48 layers, 32 heads on 4, d = 128, 8193
// slots: statistics 25.9 us (4.1 TB/s), values 46.2 us (4.7 TB/s), finish 5 us;
// one layer of 1025 slots: 4.8, 6.9 and 2.9 us, three launches' latency, which
// makes such a step slower than over a bfloat16 cache (13.6 us from a graph for
// 10.0).
#include "q4_attend.h"

namespace {

using namespace vz_q4;

constexpr int kStatsDepth = 4, kValuesDepth = 1;  // units whose loads are in flight per wave
constexpr int kMostKeys = 1024;                   // of a chunk

struct Q4Args : AttendArgs {
    uint32_t* parts;  // the queries as operands, per (sequence, layer, KV head)
    float2* ml;       // max and sum of exp2 per (layer, head, chunk row, share) [L][Hq][nc_max][shares]
    float* part;      // the chunks' outputs [L][nc_max][shares][Hq][D], each over the sequence's sum of exp2
    // a single sequence's eviction of one slot (ev_budget > 0): the finishing launch lets the slot past the budget
    // fill the freed one
    uint64_t* least;  // per (layer, chunk): the smallest rank key of the slots that compete (~0: none), and its slot
    int32_t ev_budget, ev_sink, ev_M;
};

// Places in the workspace.
__device__ __forceinline__ float2* ml_of(const Q4Args& a, int l, int h, int chunk_row) {
    return a.ml + ((static_cast<size_t>(l) * a.Hq + h) * a.nc_max + chunk_row) * a.shares;
}
// Output row of a head of a chunk row's share (channel 0).
__device__ __forceinline__ float* part_of(const Q4Args& a, int l, int chunk_row, int share, int h, int d) {
    return a.part + (((static_cast<size_t>(l) * a.nc_max + chunk_row) * a.shares + share) * a.Hq + h) * d;
}

// The parts of a KV head's queries in the workspace (row: (sequence, layer, KV head)).
template <int DT, int D, bool PACK>
__device__ __forceinline__ uint32_t* parts_of_query(const Q4Args& a, size_t row) {
    return a.parts + row * Queries<DT, D, PACK>::kWords;
}

template <int DT, int D, bool RAG, bool PACK>
__global__ __launch_bounds__(kThreads, 4) void stats_kernel(const Q4Args a) {
    using R = Rows<D>;
    __shared__ __align__(16) uint32_t s_new[kWaves][kNewWords<D>];
    const int l = blockIdx.y;
    SeqItem it;
    int c;
    if (!resolve_chunk<RAG>(a, blockIdx.x, it, c)) return;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / vz::kWave), lane = threadIdx.x % vz::kWave;
    const int q4 = lane >> 4, r16 = lane & 15;
    const int G = a.Hq / a.Hkv, shares = a.shares;
    const int c0 = c * a.chunk, c1 = min(c0 + a.chunk, it.len + 1);  // the chunk's keys
    const size_t row_sl = static_cast<size_t>(it.s) * a.L + l;
    const bool newest = it.len < c1 && it.len >= c0;
    if (newest && threadIdx.x == 0 && blockIdx.z == 0)
        a.pos[static_cast<size_t>(l) * a.plane + it.base + it.len] = it.next_pos;
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
        const int old = min(c1, it.len);  // end of the chunk's keys that the cache holds
        KTile kt[kStatsDepth];
        Queries<DT, D, PACK> q;
        q.load(static_cast<const typename vz::Elem<DT>::T*>(a.q) + row_g * G * D, lane, G);
        if (c == 0 && share == 0) q.store(parts_of_query<DT, D, PACK>(a, row_g));
        q.make();  // (the registers of the parts' making are the loads' then)
#pragma unroll
        for (int u = 0; u < kStatsDepth; ++u) load_k<D>(kt[u], lane, kc, ks, unit_key(u), old);
        // the unit that holds the new key, when it is this wave's
        const int u_new = (it.len - c0) / kUnit;
        const bool mine = newest && u_new % shares == share;
        if (mine) append<DT, D>(a, lane, row_g, head + it.len, s_new[w]);
        // the largest logit, the same scaled, and the sum of exp2 relative to it.  While no key has a finite logit the
        // scaled one is -inf, and the first that has one takes the empty sum by a factor of 0: by exp2 from any finite
        // start it would be infinity times 0 where the logits lie far below it.
        float m = -INFINITY, top = -INFINITY, z = 0.f;
        auto unit = [&](int i, KTile& k) {
            const int k0 = unit_key(i);
            if (mine && k0 + kUnit > it.len) put_new_k<D>(k, lane, it.len - k0, s_new[w]);
            float x[PACK ? 1 : 2][4];
            dots_of<DT, D, PACK>(k, q, lane, k0, c1, x);
            load_k<D>(k, lane, kc, ks, unit_key(i + kStatsDepth), old);  // (past the chunk: nothing)
            m = fmaxf(m, fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])));
            if constexpr (!PACK) m = fmaxf(m, fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
            const float last = top;
            top = m * a.scale_log2;
            const float ref = finite_ref(top);
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
        float mw = vz::rows_max(top);
        if constexpr (PACK) mw = fmaxf(mw, vz::ror16<8>(mw));
        z *= __builtin_amdgcn_exp2f(top - finite_ref(mw));
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
        constexpr int CTRL = decltype(ctrl)::value;
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
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

// Three workgroups per CU, and two where the parts and the outputs of sixteen
// heads of 128 channels would spill (24 layers of 8192 slots, 16 heads on one KV
// head: float32 34 us with the spills, 31 without; bfloat16 29.2 and 26.9).
template <int DT, int D, bool RAG, bool PACK>
__global__ __launch_bounds__(kThreads, D == 128 && !PACK ? 2 : 3) void values_kernel(const Q4Args a) {
    using R = Rows<D>;
    using E = vz::Elem<DT>;
    constexpr int NP = DT == VZ_F32 ? 3 : 2;                     // bfloat16 parts of p
    constexpr int NC = D / 16;                                   // channels per lane of V and of an output row
    constexpr int KEYS_PER_THREAD = kMostKeys / kThreads;
    __shared__ float s_sum[kWaves][kMostKeys];  // per key: the sum of p over a wave's heads
    __shared__ uint64_t s_least[kWaves];
    // The chunks in the opposite order of the statistics': the keys read last are in the memory-side cache still
    // (eight sequences, 370 MB of keys: 260 -> 253 us).
    const int l = gridDim.y - 1 - blockIdx.y;
    SeqItem it;
    int c;
    if (!resolve_chunk<RAG>(a, gridDim.x - 1 - blockIdx.x, it, c)) return;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / vz::kWave), lane = threadIdx.x % vz::kWave;
    const int q4 = lane >> 4, r16 = lane & 15;
    const int hc = PACK ? r16 & 7 : r16, half = PACK ? r16 >> 3 : 0;  // the lane's head, and 16 keys of a unit
    const int G = a.Hq / a.Hkv, shares = a.shares, items = a.Hkv * shares;
    const int c0 = c * a.chunk, c1 = min(c0 + a.chunk, it.len + 1);
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
                load_k<D>(kt[u], lane, kc, ks, unit_key(u), c1);
                load_v<D>(vt[u], lane, vc, vs, unit_key(u), c1);
            }
            const float2 st = merge_pairs<PACK>(ml_of(a, l, g * G + min(hc, G - 1), it.first), rows);
            // (columns past the group: weights and sums of 0)
            const float ref = hc < G ? finite_ref(st.x) : INFINITY;
            const float inv_z = hc < G ? 1.0f / st.y : 0.f;
            f32x4 acc[NC];
#pragma unroll
            for (int t = 0; t < NC; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto unit = [&](int u, KTile& k, VTile<D>& v) {
                const int k0 = unit_key(u);
                float x[PACK ? 1 : 2][4];
                dots_of<DT, D, PACK>(k, q, lane, k0, c1, x);
                load_k<D>(k, lane, kc, ks, unit_key(u + kValuesDepth), c1);  // (past the chunk: nothing)
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
                add_values<NP, D>(p, v, lane, acc);
                load_v<D>(v, lane, vc, vs, unit_key(u + kValuesDepth), c1);
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
        // the sums of these KV heads, in head order
#pragma unroll
        for (int i = 0; i < KEYS_PER_THREAD; ++i) {
            const int key = threadIdx.x + i * kThreads;
            if (c0 + key < c1)
                for (int v = 0; v < kWaves && first + v < items; ++v)
                    if (v % shares == key / kUnit % shares) total[i] += s_sum[v][key];
        }
        __syncthreads();
    }
    // ---- Eq. (6), and the chunk's smallest rank key ----
    const size_t slots = static_cast<size_t>(l) * a.plane + it.base + c0;
    uint64_t best = ~0ull;
    int best_key = 0;
#pragma unroll
    for (int i = 0; i < KEYS_PER_THREAD; ++i) {
        const int key = threadIdx.x + i * kThreads;
        if (c0 + key >= c1) continue;
        // (zero pad for the new slot)
        const float now = fmaf(a.gamma, c0 + key < it.len ? a.score[slots + key] : 0.f, total[i]);
        a.score[slots + key] = now;
        if (!RAG && a.ev_budget > 0) {
            const int32_t p = a.pos[slots + key];
            const uint64_t k = vz::rank_key(now, p);
            if (p >= a.ev_sink && p < it.next_pos + 1 - a.ev_M && k < best) {
                best = k;
                best_key = key;
            }
        }
    }
    if (!RAG && a.ev_budget > 0) {
        const uint64_t wb = vz::wave_min_u64(best);
        if (lane == 0) s_least[w] = wb;
        __syncthreads();
        uint64_t b = s_least[0];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) b = s_least[v] < b ? s_least[v] : b;
        if (b == ~0ull ? threadIdx.x == 0 : best == b) {  // (keys hold the position: one thread has it)
            uint64_t* const out = a.least + 2 * (static_cast<size_t>(l) * a.n_chunks + c);
            out[0] = b;
            out[1] = c0 + best_key;
        }
    }
}

// Four-element pieces of a sequence's output rows: `groups` threads of a block
// each add up a part of a piece's chunks.  Blocks per (layer, sequence).
__host__ __device__ inline int out_blocks(int Hq, int D, int groups) {
    return (Hq * D / 4 * groups + kThreads - 1) / kThreads;
}

// Blocks [0, out_blocks x sequences) of a layer: output rows from the chunks';
// in a ragged call the sequence's status too.  A block after them, where one
// slot is evicted: the slot past the budget fills the one with the smallest key.
template <int DT, int D, bool RAG, int GROUPS>
__global__ __launch_bounds__(kThreads) void finish_kernel(const Q4Args a) {
    using R = Rows<D>;
    using T = typename vz::Elem<DT>::T;
    const int l = blockIdx.y, t = threadIdx.x, blocks = out_blocks(a.Hq, D, GROUPS);
    const int s = blockIdx.x / blocks, part = blockIdx.x - s * blocks;
    if (!RAG && s > 0) {
        __shared__ uint64_t s_least[kWaves];
        __shared__ int s_slot;
        uint64_t best = ~0ull, slot = 0;
        for (int i = t; i < a.n_chunks; i += kThreads) {
            const uint64_t* const e = a.least + 2 * (static_cast<size_t>(l) * a.n_chunks + i);
            if (e[0] < best) {
                best = e[0];
                slot = e[1];
            }
        }
        const uint64_t wb = vz::wave_min_u64(best);
        if (t % vz::kWave == 0) s_least[t / vz::kWave] = wb;
        if (t == 0) s_slot = a.ev_budget;
        __syncthreads();
        uint64_t b = s_least[0];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) b = s_least[v] < b ? s_least[v] : b;
        if (b != ~0ull && best == b) s_slot = static_cast<int>(slot);
        __syncthreads();
        const int to = s_slot, from = a.ev_budget;
        if (to >= from) return;  // the slot past the budget goes, or none competes
        const size_t slots = static_cast<size_t>(l) * a.plane;
        if (t == 0) {
            a.score[slots + to] = a.score[slots + from];
            a.pos[slots + to] = a.pos[slots + from];
        }
        constexpr int CH = R::kCodes / 16;
        using S = std::conditional_t<R::kScales == 4, uint32_t, uint16_t>;
        for (int i = t; i < a.Hkv * 2 * (CH + 1); i += kThreads) {
            const int p = i % (CH + 1), which = i / (CH + 1) & 1;
            const size_t row = (static_cast<size_t>(l) * a.Hkv + i / (2 * (CH + 1))) * a.plane;
            if (p < CH) {
                uint8_t* const codes = (which ? a.c.vc : a.c.kc) + 16 * p;
                *reinterpret_cast<uint4*>(codes + (row + to) * R::kCodes) =
                    *reinterpret_cast<const uint4*>(codes + (row + from) * R::kCodes);
            } else {
                S* const scales = reinterpret_cast<S*>(which ? a.c.vs : a.c.ks);
                scales[row + to] = scales[row + from];
            }
        }
        return;
    }
    int first = 0, nc = a.n_chunks;
    if constexpr (RAG) {
        const int st = vz::ragged_decode_status(a.rag, s);
        nc = seq_chunks(a.rag, s, a.chunk);
        first = vz::ragged_first(s, a.nc_max, [&](int u) { return seq_chunks(a.rag, u, a.chunk); });
        const bool ok = st == VZ_OK && first >= 0 && first + nc <= a.nc_max;
        if (a.rag.status && part == 0 && l == 0 && t == 0)
            a.rag.status[s] = ok ? VZ_OK : (st != VZ_OK ? st : VZ_ERR_CAPACITY);
        if (!ok) return;
    }
    const int rows = nc * a.shares, n = a.Hq * D;
    if (rows == 1) return;
    constexpr int PIECES = kThreads / GROUPS;
    const int group = t / PIECES, e = 4 * (part * PIECES + t % PIECES);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4& x) {
        o.x += x.x;
        o.y += x.y;
        o.z += x.z;
        o.w += x.w;
    };
    if (e < n) {
        const float* const p = part_of(a, l, first, 0, 0, D) + e;
#pragma unroll 8
        for (int r = group; r < rows; r += GROUPS)
            add(*reinterpret_cast<const float4*>(p + static_cast<size_t>(r) * n));
    }
    if constexpr (GROUPS > 1) {
        __shared__ float4 s_part[GROUPS][PIECES];
        s_part[group][t % PIECES] = o;
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int r = 1; r < GROUPS; ++r) add(s_part[r][t]);
    }
    if (group != 0 || e >= n) return;
    T* const dst = static_cast<T*>(a.out) + (static_cast<size_t>(s) * a.L + l) * n + e;
    dst[0] = vz::Elem<DT>::from_f32(o.x);
    dst[1] = vz::Elem<DT>::from_f32(o.y);
    dst[2] = vz::Elem<DT>::from_f32(o.z);
    dst[3] = vz::Elem<DT>::from_f32(o.w);
}

// Room for a KV head's query parts.
constexpr int query_words(int d, bool pack) {
    if (d == 64) return pack ? Queries<VZ_F32, 64, true>::kWords : Queries<VZ_F32, 64, false>::kWords;
    return pack ? Queries<VZ_F32, 128, true>::kWords : Queries<VZ_F32, 128, false>::kWords;
}
// Groups of at most 8 heads take two parts of the queries a product.
bool packs(int32_t Hq, int32_t Hkv) { return Hq / Hkv <= 8; }

// Chunks per layer:
// - two workgroups per CU over the layers where a wave then has two rounds of
//   keys or more, else one (each costs its queries, pairs and partial outputs: 24
//   layers of 4001 keys, d = 64, 19 us with two and 21 with one; 48 layers of 300
//   keys 20 and 17; 48 layers of 8193 with three 81 for 77);
// - but no more than sqrt(1.4 keys / shares): a wave's keys, keys / (chunks x
//   shares), and a sequence's pairs and rows, chunks x shares, are both gone
//   through one after the other (one layer of 8001 keys on 4 KV heads: 20.5 us
//   in 251 chunks, 15.2 in 84; on 8: 28 and 21; 16,001 keys on one: 27 and 18.5);
// - no fewer than kMostKeys asks for;
// - where that gives every CU one, as many as give each the same number (13,181
//   keys of 48 layers: 109 us in 13 chunks a layer, 103 in 16).
// The host knows of a ragged call's keys only the slots that the planes have, so
// partly filled slots get longer chunks than their keys ask for (one layer of 16
// sequences of 2000 keys, 4 KV heads: 21 us in slots of 2017, 22 of 8068, 43 of
// 32,272).
constexpr int kCus = 256;
int64_t chunks_for(int32_t L, int32_t Hkv, int64_t keys, int32_t n_seqs) {
    const int64_t rounds = keys * L / (kUnit * shares_of(Hkv));
    const int64_t target = (rounds >= 2 * 2 * kCus ? 2 * kCus : kCus) / L;
    const double few = sqrt(1.4 * static_cast<double>(keys) * std::max(n_seqs, 1) / shares_of(Hkv));
    const int64_t need = std::max<int64_t>(1, (keys + kMostKeys - 1) / kMostKeys);
    const int64_t least = std::max(std::min(target, static_cast<int64_t>(few)), need);
    return least * L < kCus ? least : (least * L + kCus - 1) / kCus * kCus / L;
}
// Keys per chunk: a multiple of what its waves take at a time, so that none of
// them leaves an empty pair and row to be read (one layer of 4401 slots, one KV
// head: 45 us in chunks of 32 keys, 20 in chunks of 128).
int chunk_for(int32_t L, int32_t Hkv, int64_t keys, int32_t n_seqs) {
    const int64_t chunks = chunks_for(L, Hkv, keys, n_seqs), even = (keys + chunks - 1) / chunks;
    const int64_t step = kUnit * shares_of(Hkv);
    return static_cast<int>((even + step - 1) / step * step);
}
// Chunk rows per layer that a workspace for planes of `plane` slots holds: a
// ragged call's; a single sequence's of any length up to the plane's.
int64_t chunk_rows(int32_t L, int32_t Hkv, int64_t plane, int32_t n_seqs) {
    if (n_seqs > 0) return plane / chunk_for(L, Hkv, plane, n_seqs) + n_seqs;
    const int step = kUnit * shares_of(Hkv);
    return std::min<int64_t>((plane + step - 1) / step, chunks_for(L, Hkv, plane, n_seqs));
}

// Threads per piece of the output rows, by the workgroups that a thread each
// makes: four where they leave CUs empty (48 layers of 8193: the step takes 72 us,
// 74 with one, 72.5 with eight), eight where they are next to none and the rows
// many (one layer of 8001 keys on 4 KV heads: 15 us, with four 16; but of 1025
// keys, 33 rows, 13.3 and 12.3), one where they fill the GPU (48 layers of a
// batch of eight: 245 us, 248 with four).
constexpr int kFewBlocks = 512, kVeryFewBlocks = 64, kManyRows = 64;
template <int DT, int D, bool RAG, int GROUPS>
hipError_t launch_finish(const Q4Args& a, hipStream_t stream) {
    const int blocks = out_blocks(a.Hq, D, GROUPS);
    const int outs = RAG ? blocks * a.rag.n : a.n_chunks * a.shares > 1 ? blocks : 0;
    // (the evicting block is found by its place behind the output blocks)
    const int grid = a.ev_budget > 0 ? blocks + 1 : outs;
    if (grid == 0) return hipSuccess;
    hipLaunchKernelGGL((finish_kernel<DT, D, RAG, GROUPS>), dim3(grid, a.L), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <int DT, int D, bool RAG, bool PACK>
hipError_t launch(const VzDecodeArgs& v, const VzQ4Cache& c, hipStream_t stream) {
    Q4Args a{};
    const int64_t plane = RAG ? v.rag.total : v.cap;
    static_cast<AttendArgs&>(a) = attend_args(v, c, static_cast<int32_t>(chunk_rows(v.L, v.Hkv, plane, v.rag.n)),
                                              chunk_for(v.L, v.Hkv, RAG ? plane : v.len + 1, v.rag.n));
    const size_t rows = static_cast<size_t>(v.L) * a.nc_max * a.shares * v.Hq;
    a.part = static_cast<float*>(v.ws);
    a.ml = reinterpret_cast<float2*>(a.part + rows * D);
    a.parts = reinterpret_cast<uint32_t*>(a.ml + rows);
    if (!RAG && v.ev) {
        a.least = reinterpret_cast<uint64_t*>(a.parts + static_cast<size_t>(v.L) * v.Hkv * query_words(D, PACK));
        a.ev_budget = v.ev_budget;
        a.ev_sink = v.ev_sink;
        a.ev_M = v.ev_M;
    }
    static_assert(Queries<DT, D, PACK>::kWords <= query_words(D, PACK), "room in the workspace");
    const int chunks = RAG ? a.nc_max : a.n_chunks, groups = (a.Hkv * a.shares + kWaves - 1) / kWaves;
    hipLaunchKernelGGL((stats_kernel<DT, D, RAG, PACK>), dim3(chunks, a.L, groups), dim3(kThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((values_kernel<DT, D, RAG, PACK>), dim3(chunks, a.L), dim3(kThreads), 0, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t blocks = static_cast<int64_t>(out_blocks(a.Hq, D, 1)) * (RAG ? v.rag.n : 1) * a.L;
    const int of_one = chunks * a.shares / (RAG ? v.rag.n : 1);  // rows of a sequence
    if (blocks < kVeryFewBlocks && of_one >= kManyRows) return launch_finish<DT, D, RAG, 8>(a, stream);
    if (blocks < kFewBlocks) return launch_finish<DT, D, RAG, 4>(a, stream);
    return launch_finish<DT, D, RAG, 1>(a, stream);
}

template <int DT, int D>
hipError_t launch_any(const VzDecodeArgs& v, const VzQ4Cache& c, hipStream_t stream) {
    const bool pack = packs(v.Hq, v.Hkv);
    if (v.rag.n > 0) return pack ? launch<DT, D, true, true>(v, c, stream) : launch<DT, D, true, false>(v, c, stream);
    return pack ? launch<DT, D, false, true>(v, c, stream) : launch<DT, D, false, false>(v, c, stream);
}

}  // namespace

size_t vz_decode_q4_ws_bytes(int32_t L, int32_t Hq, int32_t Hkv, int32_t d, int64_t plane, int32_t n_seqs) {
    const size_t rows = static_cast<size_t>(L) * chunk_rows(L, Hkv, plane, n_seqs) * shares_of(Hkv) * Hq;
    const size_t queries = static_cast<size_t>(std::max(n_seqs, 1)) * L * Hkv * query_words(d, packs(Hq, Hkv));
    const size_t least = n_seqs > 0 ? 0 : static_cast<size_t>(L) * chunk_rows(L, Hkv, plane, 0) * 2 * sizeof(uint64_t);
    return rows * (d * sizeof(float) + sizeof(float2)) + queries * sizeof(uint32_t) + least;
}

bool vz_decode_q4_evicts(const VzDecodeArgs& a, int32_t budget, bool kept) { return !kept && a.len == budget; }

hipError_t vz_launch_decode_q4(const VzDecodeArgs& a, const VzQ4Cache& c, hipStream_t stream) {
    if (a.dtype == VZ_BF16 && a.d == 128) return launch_any<VZ_BF16, 128>(a, c, stream);
    if (a.dtype == VZ_BF16 && a.d == 64) return launch_any<VZ_BF16, 64>(a, c, stream);
    if (a.dtype == VZ_F32 && a.d == 128) return launch_any<VZ_F32, 128>(a, c, stream);
    if (a.dtype == VZ_F32 && a.d == 64) return launch_any<VZ_F32, 64>(a, c, stream);
    return hipErrorInvalidValue;
}
