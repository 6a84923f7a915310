// Low-rank adapters of many requests beside the projections of a group of matrices that share their activations.
// Declarations and contract: include/w2a8.h.
//
// Mathematics.  Token m of a request with adapter a (rank r, scale s), matrix i:
//   h[j] = sum_k x[m][k] A_i[a][j][k]  (j < r),      y_i[m][n] = base_i[m][n] + sum_j B_i[a][n][j] (s h[j]).
//
// Bound: memory.  base and y are read and written once, the A and B of every adapter in the batch once; the products
// are 2 r (K + N) operations per token and matrix, far below the tensor cores' rate at the ranks of adapters.
//
// One launch, no workspace.  Every CTA sorts the tokens of the batch by adapter itself (a stable counting sort of
// 4096 tokens at a time in shared memory: all CTAs find the same order) and cuts them into tiles of up to 64 tokens
// of one adapter.  A work item is (tile, matrix, share of the channels); a cluster of C CTAs takes one at a time:
//   1. h: the K axis is split over the CTAs of the cluster and the warps of a CTA; mma.sync bf16 with the operands
//      straight from global memory (k is permuted alike on both sides so that a lane's operands of two instructions
//      are 16 consecutive bytes).  Sums of the warps are added in shared memory, of the CTAs over the cluster, both
//      in a fixed order.
//   2. y: the channels of the item are split over the CTAs and warps.  s h stays in fp32: it is cut into three bf16
//      terms by truncation, whose sum is exactly its 24 bits (two terms, 16 bits, for a bf16 result), so the product
//      with the bf16 B carries no rounding of h.  Channels are permuted so that a lane holds four consecutive ones.
#include <type_traits>

#include "w2a8_common.cuh"

namespace w2a8 {

constexpr int kLoraMaxMatrices = 4;
constexpr int kLoraMaxAdapters = 1024;
constexpr int kLoraMaxRank = 128;
constexpr int kLoraThreads = 256;
constexpr int kLoraWarps = kLoraThreads / 32;
constexpr int kLoraTile = 64;            // tokens per tile
constexpr int kLoraChunk = 4096;         // tokens that are sorted at a time
constexpr int kLoraMaxCluster = 8;

struct LoraParams {
    const uint16_t *x;
    const int32_t *adapter, *rank;       // rank: nullptr = rank_max for all
    const float *scale;                  // nullptr = 1
    const uint16_t *A[kLoraMaxMatrices], *B[kLoraMaxMatrices];
    const void *base[kLoraMaxMatrices];  // nullptr = 0
    void *y[kLoraMaxMatrices];
    int N[kLoraMaxMatrices];
    int count, adapters, rank_max, M, K, C;
};

__device__ __forceinline__ float4 lora_ld_cluster(uint32_t local, uint32_t rank) {
    uint32_t remote;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
    return v;
}

// Shared memory of an instance: RK ranks at most, RP of them in a pass of step 1.
template <int RK>
struct LoraSmem {
    static constexpr int RP = RK < 64 ? RK : 64;
    static constexpr int RSTR = RP + 4;          // floats between rows of a warp's sums: no bank conflicts
    static constexpr int HSTR = RK + 4;          // of h
    union Scratch {
        struct {
            uint16_t hist[kLoraWarps][kLoraMaxAdapters + 1];
            uint16_t within[kLoraChunk];         // place of a token among those of its warp and adapter
        } sort;
        float sums[kLoraWarps][16 * RSTR];       // per warp
        float h[kLoraTile * HSTR];               // after the cluster's sum: s h
    };
    alignas(16) Scratch u;
    alignas(16) float part[kLoraTile * HSTR];    // this CTA's share of K, read by the cluster
    uint16_t perm[kLoraChunk];                   // tokens of the chunk in order of their adapters
    uint16_t first[kLoraMaxAdapters + 2];        // first place in perm of each adapter's tokens
    uint16_t tiles[kLoraMaxAdapters + 2];        // tiles of the adapters before this one
    uint32_t scan[kLoraWarps];
};

__device__ __forceinline__ uint32_t pack_hi16(float lo, float hi) {      // the upper halves of two values
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}
__device__ __forceinline__ float trunc_bf16(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }

// Cut v into T bf16 terms by truncation: 8 significant bits each, the differences are exact.  An infinity or NaN is
// its own first term.
template <int T>
__device__ __forceinline__ void cut_pair(float a, float b, uint32_t (&term)[T]) {
#pragma unroll
    for (int i = 0; i < T; ++i) {
        term[i] = pack_hi16(a, b);
        const bool fa = (__float_as_uint(a) & 0x7F800000u) != 0x7F800000u;
        const bool fb = (__float_as_uint(b) & 0x7F800000u) != 0x7F800000u;
        a = fa ? a - trunc_bf16(a) : 0.0f;
        b = fb ? b - trunc_bf16(b) : 0.0f;
    }
}

// keep the first `n` of eight / four bf16 values (n <= 0: none)
__device__ __forceinline__ uint32_t keep2(uint32_t w, int n) { return n >= 2 ? w : n == 1 ? (w & 0xFFFFu) : 0u; }

template <int RK, bool Y16>
__global__ void __launch_bounds__(kLoraThreads)
w2a8_lora_kernel(const LoraParams p) {
    using Smem = LoraSmem<RK>;
    constexpr int RP = Smem::RP, NT = RP / 8, RSTR = Smem::RSTR, HSTR = Smem::HSTR;
    constexpr int TERMS = Y16 ? 2 : 3;
    constexpr int KS = RK / 16;                  // steps of 16 ranks in step 2
    extern __shared__ __align__(16) char smem_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;       // row and column pair of a lane in the tiles of mma.sync
    const int C = p.C, crank = C > 1 ? (int)cluster_ctarank() : 0;
    const int cluster = blockIdx.x / C, clusters = gridDim.x / C;
    const int L = p.adapters;
    pdl_launch_dependents();
    pdl_wait();

    bool reading = false;                        // an open cluster barrier phase: others may read `part`
    int turn = 0;                                // items of the chunks before, modulo the clusters
    for (int chunk = 0; chunk < p.M; chunk += kLoraChunk) {
        const int n_tok = min(kLoraChunk, p.M - chunk);
        // ---- sort: places of the tokens, adapter `L` standing for none ------------------------------------------
        __syncthreads();
        for (int i = tid; i < kLoraWarps * (kLoraMaxAdapters + 1); i += kLoraThreads) {
            const int a = i % (kLoraMaxAdapters + 1);
            if (a <= L) (&sm.u.sort.hist[0][0])[i] = 0;
        }
        __syncthreads();
        const int per_warp = (n_tok + kLoraThreads - 1) / kLoraThreads * 32;
        const int w0 = min(n_tok, warp * per_warp), w1 = min(n_tok, w0 + per_warp);
        auto adapter_of = [&](int i) {
            const int a = p.adapter[chunk + i];
            return a < 0 || a >= L ? L : a;
        };
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            const int a = i < w1 ? adapter_of(i) : -1;
            const unsigned same = __match_any_sync(0xFFFFFFFFu, a);
            const int before = __popc(same & ((1u << lane) - 1u));
            int had = 0;
            if (a >= 0) had = sm.u.sort.hist[warp][a];
            __syncwarp();
            if (a >= 0) {
                sm.u.sort.within[i] = (uint16_t)(had + before);
                if (before == 0) sm.u.sort.hist[warp][a] = (uint16_t)(had + __popc(same));
            }
            __syncwarp();
        }
        __syncthreads();
        // exclusive sums over the adapters, of tokens (low half) and of tiles (high half); thread i has `each` of them
        {
            const int each = (L + 1 + kLoraThreads - 1) / kLoraThreads;
            const int a0 = min(L + 1, tid * each), a1 = min(L + 1, a0 + each);
            uint32_t mine = 0;
            for (int a = a0; a < a1; ++a) {
                uint32_t n = 0;
                for (int w = 0; w < kLoraWarps; ++w) {
                    const uint32_t c = sm.u.sort.hist[w][a];
                    sm.u.sort.hist[w][a] = (uint16_t)n;              // tokens of this adapter in the warps before
                    n += c;
                }
                sm.first[a] = (uint16_t)n;
                mine += n + ((n + kLoraTile - 1) / kLoraTile << 16);
            }
            uint32_t incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += v;
            }
            if (lane == 31) sm.scan[warp] = incl;
            __syncthreads();
            uint32_t at = incl - mine;
            for (int w = 0; w < warp; ++w) at += sm.scan[w];
            for (int a = a0; a < a1; ++a) {
                const uint32_t n = sm.first[a];
                sm.first[a] = (uint16_t)at;
                sm.tiles[a] = (uint16_t)(at >> 16);
                at += n + ((n + kLoraTile - 1) / kLoraTile << 16);
            }
            if (a1 == L + 1 && a0 < a1) { sm.first[L + 1] = (uint16_t)at; sm.tiles[L + 1] = (uint16_t)(at >> 16); }
        }
        __syncthreads();
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            if (i < w1) {
                const int a = adapter_of(i);
                sm.perm[sm.first[a] + sm.u.sort.hist[warp][a] + sm.u.sort.within[i]] = (uint16_t)i;
            }
        }
        __syncthreads();

        // ---- the items of the chunk, dealt to the clusters in turn -------------------------------------------------
        const int n_tiles = sm.tiles[L + 1];
        const int whole = n_tiles * p.count;
        const int shares = max(1, clusters / max(whole, 1));         // few items: several clusters share the channels of one
        const int items = whole * shares;
        int item = cluster - turn;
        if (item < 0) item += clusters;
        for (; item < items; item += clusters) {
            const int share = item % shares, tile = item / shares / p.count, mat = item / shares % p.count;
            int a = 0;                                                // adapter of the tile: the last with tiles[a] <= tile
            for (int step = 1 << 10; step > 0; step >>= 1)
                if (a + step <= L && sm.tiles[a + step] <= tile) a += step;
            const int at = sm.first[a] + (tile - sm.tiles[a]) * kLoraTile;
            const int n = min(kLoraTile, sm.first[a + 1] - at);       // tokens of the tile
            int r = 0;
            float s = 1.0f;
            if (a < L) {
                r = p.rank ? min(max(p.rank[a], 0), p.rank_max) : p.rank_max;
                if (p.scale) s = p.scale[a];
            }
            const int N = p.N[mat];
            const uint16_t *base16 = static_cast<const uint16_t *>(p.base[mat]);
            const float *base32 = static_cast<const float *>(p.base[mat]);
            uint16_t *y16 = static_cast<uint16_t *>(p.y[mat]);
            float *y32 = static_cast<float *>(p.y[mat]);
            // blocks of 16 channels of this CTA
            const int blocks = N / 16, parts = shares * C, part_id = share * C + crank;
            const int cb0 = (int)((long long)blocks * part_id / parts), cb1 = (int)((long long)blocks * (part_id + 1) / parts);

            if (r == 0) {                                             // nothing to add
                if (p.base[mat] == p.y[mat]) continue;
                constexpr int VB = Y16 ? 2 : 4;                       // 16-byte vectors per block
                const int per = (cb1 - cb0) * VB;
                for (int i = tid; i < n * per; i += kLoraThreads) {
                    const size_t off = (size_t)(chunk + sm.perm[at + i / per]) * N * (Y16 ? 2 : 4) +
                                       (size_t)(cb0 * VB + i % per) * 16;
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (base32) v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(base32) + off);
                    *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(y32) + off) = v;
                }
                continue;
            }

            // warps: `mt` tiles of 16 tokens (1, 2 or 4) times shares of K (step 1) or of the channels (step 2)
            const int mt = n <= 16 ? 1 : n <= 32 ? 2 : 4;
            const int wm = warp & (mt - 1), wk = warp / mt, wn = kLoraWarps / mt;
            const int ra = wm * 16 + g, rb = ra + 8;                  // the lane's two tokens in the tile
            const bool live = wm * 16 < n, la = ra < n, lb = rb < n;
            const int ta = chunk + (la ? sm.perm[at + ra] : 0), tb = chunk + (lb ? sm.perm[at + rb] : 0);

            // ---- step 1 -------------------------------------------------------------------------------------------
            const int units = p.K / 64, slices = C * wn, slice = crank * wn + wk;
            const uint16_t *xa = p.x + (size_t)ta * p.K + 8 * t, *xb = p.x + (size_t)tb * p.K + 8 * t;
            const uint16_t *wrow = p.A[mat] + ((size_t)a * p.rank_max + g) * p.K + 8 * t;
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            for (int r0 = 0; r0 < r; r0 += RP) {
                float acc[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
                if (live) {
                    for (int u = slice; u < units; u += slices) {
                        uint4 va[2], vb[2], w[NT][2];
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            va[b] = la ? *reinterpret_cast<const uint4 *>(xa + u * 64 + b * 32) : zero;
                            vb[b] = lb ? *reinterpret_cast<const uint4 *>(xb + u * 64 + b * 32) : zero;
                        }
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int b = 0; b < 2; ++b)
                                w[j][b] = r0 + j * 8 + g < r
                                              ? *reinterpret_cast<const uint4 *>(wrow + (size_t)(r0 + j * 8) * p.K + u * 64 + b * 32)
                                              : zero;
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            if (r0 + j * 8 >= r) continue;
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                mma_bf16_16x8x16(acc[j], va[b].x, vb[b].x, va[b].y, vb[b].y, w[j][b].x, w[j][b].y, acc[j]);
                                mma_bf16_16x8x16(acc[j], va[b].z, vb[b].z, va[b].w, vb[b].w, w[j][b].z, w[j][b].w, acc[j]);
                            }
                        }
                    }
                }
                __syncthreads();                                      // `u` is free (sort, h or the sums before)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    float *d = &sm.u.sums[warp][g * RSTR + j * 8 + 2 * t];
                    *reinterpret_cast<float2 *>(d) = make_float2(acc[j][0], acc[j][1]);
                    *reinterpret_cast<float2 *>(d + 8 * RSTR) = make_float2(acc[j][2], acc[j][3]);
                }
                if (reading) { cluster_wait(); reading = false; }     // the shares of the item before have been read
                __syncthreads();
                for (int i = tid; i < mt * 16 * (RP / 4); i += kLoraThreads) {
                    const int row = i / (RP / 4), c4 = i % (RP / 4);
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int k = 0; k < wn; ++k) {
                        const float4 q = *reinterpret_cast<const float4 *>(
                            &sm.u.sums[k * mt + (row >> 4)][(row & 15) * RSTR + c4 * 4]);
                        v.x += q.x; v.y += q.y; v.z += q.z; v.w += q.w;
                    }
                    *reinterpret_cast<float4 *>(&sm.part[row * HSTR + r0 + c4 * 4]) = v;
                }
            }
            if (C > 1) cluster_sync(); else __syncthreads();
            {
                // columns up to the next multiple of 16 ranks; those from r on count as zero, whatever the row holds
                const int cols4 = (r + 15) / 16 * 4;
                const uint32_t part_u32 = (uint32_t)__cvta_generic_to_shared(sm.part);
                for (int i = tid; i < mt * 16 * cols4; i += kLoraThreads) {
                    const int off = (i / cols4) * HSTR + (i % cols4) * 4;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (C > 1) {
                        for (int c = 0; c < C; ++c) {
                            const float4 q = lora_ld_cluster(part_u32 + off * 4, c);
                            v.x += q.x; v.y += q.y; v.z += q.z; v.w += q.w;
                        }
                    } else {
                        v = *reinterpret_cast<const float4 *>(&sm.part[off]);
                    }
                    const int j = (i % cols4) * 4;
                    v.x = j < r ? v.x * s : 0.0f;
                    v.y = j + 1 < r ? v.y * s : 0.0f;
                    v.z = j + 2 < r ? v.z * s : 0.0f;
                    v.w = j + 3 < r ? v.w * s : 0.0f;
                    *reinterpret_cast<float4 *>(&sm.u.h[off]) = v;
                }
            }
            if (C > 1) { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); reading = true; }
            __syncthreads();

            // ---- step 2 -------------------------------------------------------------------------------------------
            if (!live) continue;
            // terms of s h: ranks 32 b + 8 t + (0 .. 7) of a lane feed steps 2 b and 2 b + 1 (RK = 16: 4 t + (0 .. 3))
            uint32_t ha[KS][4][TERMS];
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int col = RK == 16 ? 4 * t : 32 * (k / 2) + 8 * t + 4 * (k & 1);
                float4 va = make_float4(0.f, 0.f, 0.f, 0.f), vb = va;
                if (col < (r + 15) / 16 * 16) {
                    va = *reinterpret_cast<const float4 *>(&sm.u.h[ra * HSTR + col]);
                    vb = *reinterpret_cast<const float4 *>(&sm.u.h[rb * HSTR + col]);
                }
                cut_pair<TERMS>(va.x, va.y, ha[k][0]);
                cut_pair<TERMS>(vb.x, vb.y, ha[k][1]);
                cut_pair<TERMS>(va.z, va.w, ha[k][2]);
                cut_pair<TERMS>(vb.z, vb.w, ha[k][3]);
            }
            const uint16_t *brow = p.B[mat] + (size_t)a * N * p.rank_max;
            const int nrow = 4 * (g >> 1) + (g & 1);                  // channel of a block that the lane's row of B is, + 2 for the second tile
            for (int cb = cb0 + wk; cb < cb1; cb += wn) {
                const size_t oa = (size_t)ta * N + cb * 16 + 4 * t, ob = (size_t)tb * N + cb * 16 + 4 * t;
                float4 ya = make_float4(0.f, 0.f, 0.f, 0.f), yb = ya;
                if constexpr (Y16) {
                    if (base16) {
                        uint2 qa = make_uint2(0u, 0u), qb = qa;
                        if (la) qa = *reinterpret_cast<const uint2 *>(base16 + oa);
                        if (lb) qb = *reinterpret_cast<const uint2 *>(base16 + ob);
                        ya = make_float4(__uint_as_float(qa.x << 16), __uint_as_float(qa.x & 0xFFFF0000u),
                                         __uint_as_float(qa.y << 16), __uint_as_float(qa.y & 0xFFFF0000u));
                        yb = make_float4(__uint_as_float(qb.x << 16), __uint_as_float(qb.x & 0xFFFF0000u),
                                         __uint_as_float(qb.y << 16), __uint_as_float(qb.y & 0xFFFF0000u));
                    }
                } else {
                    if (base32) {
                        if (la) ya = *reinterpret_cast<const float4 *>(base32 + oa);
                        if (lb) yb = *reinterpret_cast<const float4 *>(base32 + ob);
                    }
                }
                float d[2][4] = {};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint16_t *b = brow + (size_t)(cb * 16 + nrow + 2 * j) * p.rank_max;
                    if constexpr (RK == 16) {
                        uint2 w = make_uint2(0u, 0u);
                        const int left = r - 4 * t;
                        if (left > 0) w = *reinterpret_cast<const uint2 *>(b + 4 * t);
                        if (left < 4) { w.x = keep2(w.x, left); w.y = keep2(w.y, left - 2); }
#pragma unroll
                        for (int i = 0; i < TERMS; ++i)
                            mma_bf16_16x8x16(d[j], ha[0][0][i], ha[0][1][i], ha[0][2][i], ha[0][3][i], w.x, w.y, d[j]);
                    } else {
                        uint4 w[RK / 32];
#pragma unroll
                        for (int k = 0; k < RK / 32; ++k) {
                            const int left = r - 32 * k - 8 * t;
                            w[k] = left > 0 ? *reinterpret_cast<const uint4 *>(b + 32 * k + 8 * t) : zero;
                            if (left < 8) {
                                w[k].x = keep2(w[k].x, left); w[k].y = keep2(w[k].y, left - 2);
                                w[k].z = keep2(w[k].z, left - 4); w[k].w = keep2(w[k].w, left - 6);
                            }
                        }
#pragma unroll
                        for (int k = 0; k < RK / 32; ++k) {
                            if (32 * k >= r) continue;
#pragma unroll
                            for (int i = 0; i < TERMS; ++i) {
                                mma_bf16_16x8x16(d[j], ha[2 * k][0][i], ha[2 * k][1][i], ha[2 * k][2][i], ha[2 * k][3][i],
                                                 w[k].x, w[k].y, d[j]);
                                mma_bf16_16x8x16(d[j], ha[2 * k + 1][0][i], ha[2 * k + 1][1][i], ha[2 * k + 1][2][i],
                                                 ha[2 * k + 1][3][i], w[k].z, w[k].w, d[j]);
                            }
                        }
                    }
                }
                ya.x += d[0][0]; ya.y += d[0][1]; ya.z += d[1][0]; ya.w += d[1][1];
                yb.x += d[0][2]; yb.y += d[0][3]; yb.z += d[1][2]; yb.w += d[1][3];
                if constexpr (Y16) {
                    auto pack = [](float4 v) {
                        uint2 q;
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q.x) : "f"(v.y), "f"(v.x));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(q.y) : "f"(v.w), "f"(v.z));
                        return q;
                    };
                    if (la) *reinterpret_cast<uint2 *>(y16 + oa) = pack(ya);
                    if (lb) *reinterpret_cast<uint2 *>(y16 + ob) = pack(yb);
                } else {
                    if (la) *reinterpret_cast<float4 *>(y32 + oa) = ya;
                    if (lb) *reinterpret_cast<float4 *>(y32 + ob) = yb;
                }
            }
        }
        turn = (int)(((long long)turn + items) % clusters);
    }
    if (reading) cluster_wait();                                      // nobody leaves while its sums may be read
}

template <int RK, bool Y16>
static cudaError_t launch_lora(LoraParams &p, int bound, cudaStream_t st) {
    auto kernel = w2a8_lora_kernel<RK, Y16>;
    constexpr size_t smem = sizeof(LoraSmem<RK>);
    static PerDeviceFlags configured;
    if (cudaError_t e = allow_dynamic_smem(kernel, configured, (int)smem)) return e;
    static PerDeviceTable<kLoraMaxCluster + 1> clusters;
    const int *resident = clusters.get(current_device(), [&](int *n) {
        for (int C = 1; C <= kLoraMaxCluster; ++C) {
            const int found = resident_clusters(kernel, C, kLoraThreads, smem);
            n[C] = found > 0 ? found : sm_count() / C;
        }
    });
    p.C = p.M <= 256 ? 8 : 4;
    const int forced = env_int("W2A8_LORA_C", 0);
    if (forced >= 1 && forced <= kLoraMaxCluster) p.C = forced;
    (void)bound;
    const int n = resident[p.C] > 0 ? resident[p.C] : 1;
    return launch_kernel_clusters(kernel, dim3((unsigned)(n * p.C)), dim3(kLoraThreads), smem, st, pdl_enabled(),
                                  make_uint2((unsigned)p.C, 1u), p);
}

}  // namespace w2a8

using namespace w2a8;

extern "C" int w2a8_lora_grouped(const void *x_bf16, const int32_t *adapter, int adapters, int rank_max,
                                 const int32_t *rank, const float *scale, int count, const void *const *A,
                                 const void *const *B, const void *const *base, void *const *y, int y_is_bf16,
                                 const int *N, int M, int K, void *stream) {
    EnvScope scope;
    if (!x_bf16 || !adapter || !A || !B || !y || !N) return W2A8_ERR_NULL;
    if (count < 1 || count > kLoraMaxMatrices || adapters < 1 || adapters > kLoraMaxAdapters || rank_max < 8 ||
        rank_max > kLoraMaxRank || rank_max % 8)
        return W2A8_ERR_SHAPE;
    LoraParams p = {};
    const size_t e = y_is_bf16 ? 2 : 4;
    auto small = [](const void *q) { return (reinterpret_cast<uintptr_t>(q) & 3u) == 0; };
    if (!aligned16(x_bf16) || !small(adapter) || !small(rank) || !small(scale)) return W2A8_ERR_ALIGN;
    for (int i = 0; i < count; ++i) {
        if (!shape_ok(M, N[i], K, 64, nullptr)) return W2A8_ERR_SHAPE;
        if (!A[i] || !B[i] || !y[i]) return W2A8_ERR_NULL;
        const void *b = base ? base[i] : nullptr;
        if (base && !b) return W2A8_ERR_NULL;
        if (!aligned16(A[i]) || !aligned16(B[i]) || !aligned16(y[i]) || !aligned16(b)) return W2A8_ERR_ALIGN;
        p.A[i] = static_cast<const uint16_t *>(A[i]);
        p.B[i] = static_cast<const uint16_t *>(B[i]);
        p.base[i] = b;
        p.y[i] = y[i];
        p.N[i] = N[i];
    }
    // a result may take the place of its own base and overlaps nothing else that the call reads or writes
    auto overlap = [](const void *q, size_t nq, const void *r, size_t nr) {
        const char *a = static_cast<const char *>(q), *b = static_cast<const char *>(r);
        return r && a < b + nr && b < a + nq;
    };
    for (int i = 0; i < count; ++i) {
        const size_t ny = (size_t)M * N[i] * e;
        if (overlap(y[i], ny, x_bf16, (size_t)M * K * 2)) return W2A8_ERR_SHAPE;
        for (int j = 0; j < count; ++j) {
            const size_t nj = (size_t)M * N[j] * e;
            if (j != i && overlap(y[i], ny, y[j], nj)) return W2A8_ERR_SHAPE;
            if (overlap(y[i], ny, p.base[j], nj) && !(i == j && p.base[j] == y[i])) return W2A8_ERR_SHAPE;
        }
    }
    if (int st = check_device()) return st;
    p.x = static_cast<const uint16_t *>(x_bf16);
    p.adapter = adapter; p.rank = rank; p.scale = scale;
    p.count = count; p.adapters = adapters; p.rank_max = rank_max; p.M = M; p.K = K;
    cudaStream_t st = (cudaStream_t)stream;
    auto go = [&](auto rk) {
        constexpr int RK = decltype(rk)::value;
        return y_is_bf16 ? launch_lora<RK, true>(p, 0, st) : launch_lora<RK, false>(p, 0, st);
    };
    const cudaError_t err = rank_max <= 16 ? go(std::integral_constant<int, 16>())
                          : rank_max <= 32 ? go(std::integral_constant<int, 32>())
                          : rank_max <= 64 ? go(std::integral_constant<int, 64>())
                                           : go(std::integral_constant<int, 128>());
    return err == cudaSuccess ? W2A8_OK : W2A8_ERR_CUDA;
}
