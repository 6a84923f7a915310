// Low-rank adapters of many requests beside the projections of a group of matrices that share their activations.
// Declarations and contract: include/w2a8.h.
//
// Mathematics.  Token m of a request with adapter a (rank r, scale s), matrix i:
//   h[j] = sum_k x[m][k] A_i[a][j][k]  (j < r),      y_i[m][n] = base_i[m][n] + sum_j B_i[a][n][j] (s h[j]).
//
// Bound: memory.  base and y are read and written once, the A and B of every adapter in the batch once; the products
// are 2 r (K + N) operations per token and matrix, far below the tensor cores' rate at the ranks of adapters.
//
// One launch, no workspace.  Every CTA sorts the tokens of the batch by adapter itself (a stable counting sort of some
// tokens at a time in shared memory: all CTAs find the same order) and cuts them into tiles of up to T tokens of one
// adapter.  A work item is (tile, matrix, share of the channels); a cluster of C CTAs takes one at a time:
//   1. h: the K axis is split over the CTAs of the cluster; tokens, ranks and what is left of K over the warps.  The sums
//      are added in a fixed order, over the cluster through distributed shared memory.
//   2. y: the channels of the item are split over the CTAs and warps.  s h stays in fp32: it is cut into three bf16
//      terms by truncation, whose sum is exactly its 24 bits (two terms, 16 bits, for a bf16 result), so the product
//      with the bf16 B carries no rounding of h.  Where B is infinite and a term is zero, the result is formed again without the
//      terms.  The look at each block's sums costs little at ranks of up to 64 (gate|up of the 8B layer, 32 tokens of rank 64, us without
//      and with it 38.2 / 38.2, 8192 tokens 402 / 399) and up to 4 % above (32 tokens of rank 128 61.9 / 64.1, 2048 with bf16
//      results 137 / 142).
// Both steps are fed by one ring of shared-memory stages that cp.async fills ahead (x and A, then B and base), so
// that the loads of step 2 are on their way while the sums of step 1 are added.  k is permuted alike on both sides so that a
// lane's operands of two instructions are 16 consecutive bytes, and the channels so that a lane holds four consecutive
// ones.
//
// The products are mma.sync (8 clk per m16n8k16 and scheduler): an item's accumulators have 16 to 128 columns in step 1
// and 16 rows per warp in step 2, and both have to leave the tensor core's sum early, for its truncation.  What bounds the
// kernel (device time, calls over inputs larger than L2): gate|up of the 8B layer for 8192 tokens of 16 adapters of rank 64,
// 398 us for three calls in a row, 5.1 TB/s of the 2.02 GB it cannot do without, and 450 us for sixty, when the power limit
// takes the clock from 1965 to 1700 MHz; about 30 us of an item's 200 are step 1, when the memory idles, and in step 2 the
// issue of two warps per scheduler (0.34 a clock, tensor pipe 37 %: counters of 1024 tokens of 2 adapters).  32 tokens with
// an adapter each 38 us, 2.4 TB/s: the same issue, with 15 of 16 rows of an instruction empty.  One token, q|k|v: 6.5 us of
// latencies: owners, sort, addresses, first bytes, two cluster barriers.
#include "w2a8_common.cuh"

namespace w2a8 {

constexpr int kLoraMaxMatrices = 4;
constexpr int kLoraMaxAdapters = 1024;
constexpr int kLoraMaxRank = 128;
constexpr int kLoraThreads = 256;
constexpr int kLoraWarps = kLoraThreads / 32;
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
    int tiles_guess, width_guess;        // the host's: width of a share (below) for that many tiles
};

__device__ __forceinline__ float4 lora_ld_cluster(uint32_t local, uint32_t rank) {
    uint32_t remote;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
    return v;
}
// The cluster's barriers are for whole warps, and the code in front of them branches by lane.
__device__ __forceinline__ void lora_cluster_sync() {
    __syncwarp();
    cluster_sync();
}
__device__ __forceinline__ void lora_cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void lora_cluster_wait() {
    __syncwarp();
    cluster_wait();
}
__device__ __forceinline__ void lora_copy16(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
// the same, or zeros
__device__ __forceinline__ void lora_copy16_or_zero(uint32_t to, const void *from, bool zero) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\tcp.async.cg.shared.global [%0], [%1], 16, p;\n\t}"
                 ::"r"(to), "l"(from), "r"((uint32_t)zero) : "memory");
}
// the first `bytes` of 16, zeros behind them
__device__ __forceinline__ void lora_copy_some(uint32_t to, const void *from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// D += A (16 x 16, bf16, row) * B (16 x 8, bf16, col), fp32; a pure function of its operands, so that the compiler may
// put loads and other products between a chain of them.
__device__ __forceinline__ void lora_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// An instance: tiles of T tokens, ranks of up to RK.  Everything that an address in the loops below depends on is a
// constant of it.  One CTA per SM with large stages: two with half of the shared memory each were slower (32 tokens of 32
// adapters of rank 64, gate|up of the 8B layer: 46 us, one 42; 16 tokens of one adapter 15 and 10), and the terms of s h
// want the registers.
template <int T_, int RK_>
struct LoraCfg {
    static constexpr int T = T_, RK = RK_;
    static constexpr int kChunk = T == 16 ? kLoraThreads : 4096;      // tokens that are sorted at a time
    static constexpr int MT = T / 16, NT = RK / 8;
    static constexpr int NR = MT == 4 ? 2 : NT < 8 ? NT : 8;          // step 1: shares of the ranks among the warps
    static constexpr int NK = kLoraWarps / MT / NR;                   // and of K
    static constexpr int WN = kLoraWarps / MT;                        // step 2: shares of the channels
    static constexpr int KC = T == 64 ? (RK <= 64 ? 128 : 64) : RK == 16 ? 512 : RK <= 64 ? 256 : 128;    // values of K per stage
    static constexpr int CH = T == 64 ? (RK <= 64 ? 128 : 64) : RK <= 64 ? 256 : 128;   // channels per stage
    static constexpr int kBytes1 = (T + RK) * KC * 2, kBytes2 = CH * (2 * RK + 4 * T);
    static constexpr int kStageBytes = kBytes1 > kBytes2 ? kBytes1 : kBytes2;
    static constexpr int kStages = T == 64 && RK <= 64 ? 3 : 4;
    static constexpr int HSTR = RK + 4;          // floats between rows of h: no bank conflicts
};
template <typename Cfg>
struct LoraSmem {
    union Ring {
        char stage[Cfg::kStages][Cfg::kStageBytes];
        uint16_t hist[kLoraWarps * (kLoraMaxAdapters + 1)];           // of the sort: tokens of each adapter by warp
    };
    alignas(128) Ring ring;
    alignas(16) float part[Cfg::T * Cfg::HSTR];  // this CTA's share of K, read by the cluster
    alignas(16) float h[Cfg::T * Cfg::HSTR];     // s h, all of K
    uint16_t perm[Cfg::kChunk];                  // tokens of the chunk in order of their adapters
    uint16_t first[kLoraMaxAdapters + 2];        // first place in perm of each adapter's tokens
    uint16_t tiles[kLoraMaxAdapters + 2];        // tiles of the adapters before this one
    uint8_t rank[kLoraMaxAdapters + 1];          // ranks, clamped; 0 for none
    uint32_t scan[kLoraWarps];
};

__device__ __forceinline__ uint32_t pack_hi16(float lo, float hi) {      // the upper halves of two values
    return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}
__device__ __forceinline__ float trunc_bf16(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }

// Cut a and b into T bf16 terms by truncation: 8 significant bits each, the differences are exact.  An infinity or NaN
// is its own first term.
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

// The tokens of a chunk in order of their adapters (perm), where each adapter's begin (first) and the tiles before it
// (tiles); adapter `L` stands for none.
template <typename Cfg>
__device__ __forceinline__ void lora_sort(LoraSmem<Cfg> &sm, const LoraParams &p, int chunk, int n_tok) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, L = p.adapters;
    uint16_t *hist = sm.ring.hist, *mine = hist + warp * (L + 1);
    for (int i = tid; i < kLoraWarps * (L + 1); i += kLoraThreads) hist[i] = 0;
    __syncthreads();
    constexpr int kSteps = Cfg::kChunk / kLoraThreads, T = Cfg::T;
    const int steps = (n_tok + kLoraThreads - 1) / kLoraThreads;
    const int w0 = warp * steps * 32 + lane;
    int own[kSteps], place[kSteps];              // adapter of the lane's tokens (-1: no token), place among those of the warp
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        own[i] = -1;
        if (i < steps && w0 + i * 32 < n_tok) {
            const int a = p.adapter[chunk + w0 + i * 32];
            own[i] = a < 0 || a >= L ? L : a;
        }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (i >= steps) continue;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, own[i]);
        const int before = __popc(same & ((1u << lane) - 1u));
        const int had = own[i] >= 0 ? mine[own[i]] : 0;
        place[i] = had + before;
        __syncwarp();
        if (own[i] >= 0 && before == 0) mine[own[i]] = (uint16_t)(had + __popc(same));
        __syncwarp();
    }
    __syncthreads();
    // exclusive sums over the adapters, of tokens (low half) and of tiles (high half); a thread has `each` of them
    const int each = (L + 1 + kLoraThreads - 1) / kLoraThreads;
    const int a0 = min(L + 1, tid * each), a1 = min(L + 1, a0 + each);
    uint32_t total = 0;
    for (int a = a0; a < a1; ++a) {
        uint32_t n = 0;
        for (int w = 0; w < kLoraWarps; ++w) {
            const uint32_t c = hist[w * (L + 1) + a];
            hist[w * (L + 1) + a] = (uint16_t)n;                     // tokens of this adapter in the warps before
            n += c;
        }
        sm.first[a] = (uint16_t)n;
        total += n + ((n + T - 1) / T << 16);
    }
    uint32_t incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) sm.scan[warp] = incl;
    __syncthreads();
    uint32_t at = incl - total;
    for (int w = 0; w < warp; ++w) at += sm.scan[w];
    for (int a = a0; a < a1; ++a) {
        const uint32_t n = sm.first[a];
        sm.first[a] = (uint16_t)at;
        sm.tiles[a] = (uint16_t)(at >> 16);
        at += n + ((n + T - 1) / T << 16);
    }
    if (a0 < a1 && a1 == L + 1) { sm.first[L + 1] = (uint16_t)at; sm.tiles[L + 1] = (uint16_t)(at >> 16); }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
        if (own[i] >= 0) sm.perm[sm.first[own[i]] + mine[own[i]] + place[i]] = (uint16_t)(w0 + i * 32);
    __syncthreads();
}

// How the channels of the matrices are dealt out: in shares of `width` blocks of 16 at most, `total` of them for a tile.
// A share does step 1 for itself, so shares cost; too few leave clusters idle in the last round.  The estimate of both, in
// microseconds, is of measured rates of a CTA: 64 values of K in step 1, a block in step 2, and what an item takes beside.
struct LoraShares { int width, total; float cost; };
__host__ __device__ inline int lora_shares_of(int N, int width) { return (N / 16 + width - 1) / width; }
constexpr int kLoraMaxShares = 16;       // of the widest matrix
template <int T, int RK>
__host__ __device__ inline LoraShares lora_shares(const LoraParams &p, int shares, int n_tiles, int clusters) {
    constexpr float kUnit = T == 64 ? (RK <= 64 ? 0.45f : 0.72f) : RK <= 32 ? 0.14f : RK <= 64 ? 0.25f : 0.40f;
    constexpr float kBlock = T == 64 ? (RK <= 64 ? 0.21f : 0.39f) : RK <= 32 ? 0.06f : RK <= 64 ? 0.10f : 0.16f;
    constexpr float kItem = T == 64 ? 6.0f : 4.0f;
    int widest = 0;
    for (int i = 0; i < p.count; ++i) widest = p.N[i] > widest ? p.N[i] : widest;
    LoraShares q;
    q.width = (widest / 16 + shares - 1) / shares;
    q.total = 0;
    for (int i = 0; i < p.count; ++i) q.total += lora_shares_of(p.N[i], q.width);
    const int rounds = (n_tiles * q.total + clusters - 1) / clusters;
    q.cost = rounds * (kItem + (kUnit * (p.K / 64) + kBlock * q.width) / p.C);
    return q;
}

template <int T, int RK, bool Y16>
__global__ void __launch_bounds__(kLoraThreads, 1)
w2a8_lora_kernel(const LoraParams p) {
    using Cfg = LoraCfg<T, RK>;
    using Smem = LoraSmem<Cfg>;
    constexpr int MT = Cfg::MT, NR = Cfg::NR, NK = Cfg::NK, NTW = Cfg::NT / NR, WN = Cfg::WN, KC = Cfg::KC, CH = Cfg::CH;
    constexpr int HSTR = Cfg::HSTR, S = Cfg::kStages, STAGE = Cfg::kStageBytes;
    constexpr int TERMS = Y16 ? 2 : 3;
    constexpr int KS = RK / 16;                  // steps of 16 ranks in step 2
    constexpr int E = Y16 ? 2 : 4;               // bytes of a value of base and y
    extern __shared__ __align__(128) char smem_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;       // row and column pair of a lane in the tiles of mma.sync
    const int C = p.C, crank = C > 1 ? (int)cluster_ctarank() : 0;
    const int cluster = blockIdx.x / C, clusters = gridDim.x / C;
    const int L = p.adapters;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(sm.ring.stage[0]);
    // reads of a stage, at byte offsets of the ring
    auto lds128 = [&](uint32_t at) { return *reinterpret_cast<const uint4 *>(sm.ring.stage[0] + at); };
    auto lds64 = [&](uint32_t at) { return *reinterpret_cast<const uint2 *>(sm.ring.stage[0] + at); };
    // Warps: MT tiles of 16 tokens, in step 1 times NR shares of the ranks and NK of K, in step 2 times WN of the channels.
    const int wm = warp % MT, wr = warp / MT, jr = wr % NR, jk = wr / NR;
    const int ra = wm * 16 + g, rb = ra + 8;                          // the lane's two tokens in the tile
    const int units = p.K / 64, u_per = units / C, u_more = units - u_per * C;
    const int u0 = crank * u_per + min(crank, u_more), n_units = u_per + (crank < u_more);
    constexpr int KU = KC / 64;
    const int n1 = (n_units + KU - 1) / KU;

    // Stages.  Step 1: T rows of x, RK of A, KC values each; step 2: CH rows of B, RK values each, and T rows of base, CH
    // values each.  16-byte pieces, with an odd row's halves of 128 bytes exchanged where rows are multiples of 128
    // bytes, so that the reads below meet no bank conflicts.  A thread copies the same column of rows that are an even
    // number apart, so that its addresses only move on from stage to stage.
    constexpr int CPX = KC / 8, DX = kLoraThreads / CPX, PX = (T + DX - 1) / DX, PA = (RK + DX - 1) / DX;
    constexpr int CPB = RK / 8, DB = kLoraThreads / CPB, PB = (CH + DB - 1) / DB;
    constexpr int CPY = CH * E / 16, DY = kLoraThreads / CPY, PY = (T + DY - 1) / DY;
    constexpr uint32_t FB = RK >= 64 ? 4u : 0u, FY = E == 4 ? 4u : 0u;
    constexpr uint32_t kA = T * KC * 2, kBase = CH * RK * 2;          // of A and base in a stage
    const int cx = tid % CPX, rx = tid / CPX, cb = tid % CPB, rbb = tid / CPB, cy = tid % CPY, ry = tid / CPY;
    const uint32_t to_x = rx * (KC * 2) + ((cx ^ ((rx & 1) << 2)) << 4);
    const uint32_t to_b = rbb * (RK * 2) + ((cb ^ ((rbb & 1) * FB)) << 4);
    const uint32_t to_y = kBase + ry * (CH * E) + ((cy ^ ((ry & 1) * FY)) << 4);
    pdl_launch_dependents();
    pdl_wait();
    for (int a = tid; a <= L; a += kLoraThreads)
        sm.rank[a] = (uint8_t)(a == L ? 0 : p.rank ? min(max(p.rank[a], 0), p.rank_max) : p.rank_max);

    bool reading = false;                        // an open cluster barrier phase: others may read `part`
    int turn = 0;                                // items of the chunks before, modulo the clusters
    for (int chunk = 0; chunk < p.M; chunk += Cfg::kChunk) {
        __syncthreads();
        lora_sort<Cfg>(sm, p, chunk, min(Cfg::kChunk, p.M - chunk));

        // ---- the items of the chunk, dealt to the clusters in turn -------------------------------------------------
        const int n_tiles = sm.tiles[L + 1];
        LoraShares parts;
        if (n_tiles == p.tiles_guess) {
            parts.width = p.width_guess;
            parts.total = 0;
            for (int i = 0; i < p.count; ++i) parts.total += lora_shares_of(p.N[i], parts.width);
        } else {
            parts = lora_shares<T, RK>(p, lane % kLoraMaxShares + 1, n_tiles, clusters);
#pragma unroll
            for (int o = kLoraMaxShares / 2; o > 0; o >>= 1) {       // the cheapest, of equal ones the widest
                const float cost = __shfl_xor_sync(0xFFFFFFFFu, parts.cost, o);
                const int width = __shfl_xor_sync(0xFFFFFFFFu, parts.width, o), total = __shfl_xor_sync(0xFFFFFFFFu, parts.total, o);
                if (cost < parts.cost || (cost == parts.cost && width > parts.width)) parts = {width, total, cost};
            }
        }
        const int items = n_tiles * parts.total;
        int item = cluster - turn;
        if (item < 0) item += clusters;
        for (; item < items; item += clusters) {
            const int tile = item / parts.total;
            int mat = 0, share = item - tile * parts.total;           // the tile's part: a share of a matrix's channels
            while (share >= lora_shares_of(p.N[mat], parts.width)) share -= lora_shares_of(p.N[mat++], parts.width);
            int a = 0;                                                // adapter of the tile: the last with tiles[a] <= tile
            for (int step = 1 << (31 - __clz(L)); step > 0; step >>= 1)
                if (a + step <= L && sm.tiles[a + step] <= tile) a += step;
            const int at = sm.first[a] + (tile - sm.tiles[a]) * T;
            const int n = min(T, sm.first[a + 1] - at);               // tokens of the tile
            const int r = sm.rank[a];
            const int N = p.N[mat];
            const char *base = static_cast<const char *>(p.base[mat]);
            char *y = static_cast<char *>(p.y[mat]);
            // blocks of 16 channels of this CTA
            const int blocks = N / 16, n_parts = lora_shares_of(N, parts.width) * C, part_id = share * C + crank;
            const int per = blocks / n_parts, more = blocks - per * n_parts;
            const int ch0 = (part_id * per + min(part_id, more)) * 16, n_ch = (per + (part_id < more)) * 16;

            if (r == 0) {                                             // nothing to add
                if (base == y) continue;
                // a warp takes a row; eight 16-byte pieces of a lane are on their way at a time
                constexpr int kAhead = 8;
                const int row_v = n_ch * E / 16;
                for (int row = warp; row < n; row += kLoraWarps) {
                    const size_t off = ((size_t)(chunk + sm.perm[at + row]) * N + ch0) * E;
                    const uint4 *from = reinterpret_cast<const uint4 *>(base + off);
                    uint4 *to = reinterpret_cast<uint4 *>(y + off);
                    for (int c = lane; c < row_v; c += 32 * kAhead) {
                        uint4 v[kAhead];
#pragma unroll
                        for (int i = 0; i < kAhead; ++i)
                            v[i] = base && c + 32 * i < row_v ? from[c + 32 * i] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                        for (int i = 0; i < kAhead; ++i)
                            if (c + 32 * i < row_v) to[c + 32 * i] = v[i];
                    }
                }
                continue;
            }
            const float s = p.scale ? p.scale[a] : 1.0f;
            const bool live = wm * 16 < n, la = ra < n, lb = rb < n;
            const int n2 = (n_ch + CH - 1) / CH;

            const char *src_x[PX], *src_y[PY];
#pragma unroll
            for (int i = 0; i < PX; ++i) {
                const int row = min(rx + i * DX, n - 1);              // rows behind the tile's tokens: no bytes of the last
                src_x[i] = reinterpret_cast<const char *>(p.x + (size_t)(chunk + sm.perm[at + row]) * p.K + u0 * 64 + cx * 8);
            }
#pragma unroll
            for (int i = 0; i < PY; ++i) {
                const int row = min(ry + i * DY, n - 1);
                src_y[i] = base + ((size_t)(chunk + sm.perm[at + row]) * N + ch0) * E + cy * 16;
            }
            const char *src_a = reinterpret_cast<const char *>(p.A[mat] + ((size_t)a * p.rank_max + rx) * p.K + u0 * 64 + cx * 8);
            // Ranks of B behind the adapter's last count as zero, whatever the row holds: of a piece, b_bytes are the adapter's
            const int b_bytes = min(max(r - cb * 8, 0), 8) * 2;
            const char *src_b = reinterpret_cast<const char *>(p.B[mat] + ((size_t)a * N + ch0 + rbb) * p.rank_max + (b_bytes ? cb * 8 : 0));
            const int b_step = DB * p.rank_max * 2;
            const size_t a_step = (size_t)DX * p.K * 2;
            int q_issue = 0, slot_issue = 0;
            auto issue2 = [&]() {                                     // a stage of step 2
                const uint32_t st = ring + slot_issue * STAGE;
                const int cw = n_ch - (q_issue - n1) * CH;            // channels that are left
                if (cw > 0) {
                    const char *src = src_b;
#pragma unroll
                    for (int i = 0; i < PB; ++i, src += b_step)
                        if (rbb + i * DB < cw && (CH % DB == 0 || rbb + i * DB < CH))
                            lora_copy_some(st + to_b + i * (kLoraThreads * 16), src, b_bytes);
                    src_b += (size_t)CH * p.rank_max * 2;
                    if (base && cy * (16 / E) < cw) {
#pragma unroll
                        for (int i = 0; i < PY; ++i)
                            if (ry + i * DY < n) lora_copy16(st + to_y + i * (kLoraThreads * 16), src_y[i]);
                    }
#pragma unroll
                    for (int i = 0; i < PY; ++i) src_y[i] += CH * E;
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                ++q_issue;
                slot_issue = slot_issue + 1 == S ? 0 : slot_issue + 1;
            };
            auto issue = [&]() {
                if (q_issue >= n1) { issue2(); return; }
                const uint32_t st = ring + slot_issue * STAGE;
                if (KU == 1 || cx < (n_units - q_issue * KU) * 8) {
#pragma unroll
                    for (int i = 0; i < PX; ++i)
                        if (T % DX == 0 || rx + i * DX < T)
                            lora_copy16_or_zero(st + to_x + i * (kLoraThreads * 16), src_x[i], rx + i * DX >= n);
                    const char *src = src_a;
#pragma unroll
                    for (int i = 0; i < PA; ++i, src += a_step)
                        if (rx + i * DX < r) lora_copy16(st + kA + to_x + i * (kLoraThreads * 16), src);
                }
#pragma unroll
                for (int i = 0; i < PX; ++i) src_x[i] += KC * 2;
                src_a += KC * 2;
                asm volatile("cp.async.commit_group;" ::: "memory");
                ++q_issue;
                slot_issue = slot_issue + 1 == S ? 0 : slot_issue + 1;
            };
            // every stage is one group, also an empty one: S - 2 groups may still be open when a stage is needed
            int slot = 0;
            auto arrive = [&](auto &&next) {
                asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
                __syncthreads();
                next();
                const uint32_t st = slot * STAGE;
                slot = slot + 1 == S ? 0 : slot + 1;
                return st;
            };
            __syncthreads();                                          // the stages and h of the item before are done with
#pragma unroll 1
            for (int q = 0; q < S - 1; ++q) issue();

            // ---- step 1 -------------------------------------------------------------------------------------------
            float acc[NTW][4];
#pragma unroll
            for (int j = 0; j < NTW; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
            const uint32_t flip = (g & 1) << 2;
#pragma unroll 1
            for (int q = 0; q < n1; ++q) {
                const uint32_t st = arrive(issue);
                if (!live) continue;
                const uint32_t xrow = st + ra * (KC * 2), arow = st + kA + (jr * NTW * 8 + g) * (KC * 2);
                const int k32 = KU == 1 ? 2 : 2 * (n_units - q * KU);
#pragma unroll
                for (int b0 = 0; b0 < 2 * KU; b0 += NK) {
                    const int b = b0 + jk;
                    if (KU > 1 && b >= k32) continue;
                    const uint32_t col = ((4 * b + t) ^ flip) << 4;
                    const uint4 va = lds128(xrow + col), vb = lds128(xrow + 8 * KC * 2 + col);
                    uint4 w[NTW];
#pragma unroll
                    for (int j = 0; j < NTW; ++j) w[j] = lds128(arow + j * (8 * KC * 2) + col);
                    // A sum of 32 products at a time joins the running one with a rounded addition: the instruction
                    // truncates where it aligns its addends, a bias that a long chain would add up.
                    float d[NTW][4] = {};
#pragma unroll
                    for (int j = 0; j < NTW; ++j) lora_mma(d[j], {va.x, vb.x, va.y, vb.y}, w[j].x, w[j].y);
#pragma unroll
                    for (int j = 0; j < NTW; ++j) lora_mma(d[j], {va.z, vb.z, va.w, vb.w}, w[j].z, w[j].w);
#pragma unroll
                    for (int j = 0; j < NTW; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[j][c] += d[j][c];
                }
            }
            if (reading) { lora_cluster_wait(); reading = false; }    // the shares of the item before have been read
#pragma unroll
            for (int k = NK - 1; k >= 0; --k) {
                if (jk == k && live) {
#pragma unroll
                    for (int j = 0; j < NTW; ++j) {
                        const int col = (jr * NTW + j) * 8 + 2 * t;
                        float2 *d0 = reinterpret_cast<float2 *>(&sm.part[ra * HSTR + col]);
                        float2 *d1 = reinterpret_cast<float2 *>(&sm.part[rb * HSTR + col]);
                        float2 v0 = make_float2(acc[j][0], acc[j][1]), v1 = make_float2(acc[j][2], acc[j][3]);
                        if (k != NK - 1) { v0.x += d0->x; v0.y += d0->y; v1.x += d1->x; v1.y += d1->y; }
                        *d0 = v0;
                        *d1 = v1;
                    }
                }
                if (k > 0) __syncthreads();
            }
            if (C > 1) lora_cluster_sync(); else __syncthreads();
            {
                // columns of ranks that the adapter has not (sums with whatever the stage held) count as zero
                constexpr int C4 = RK / 4;
                const uint32_t part_u32 = (uint32_t)__cvta_generic_to_shared(sm.part);
                for (int i = tid; i < n * C4; i += kLoraThreads) {
                    const int j = (i % C4) * 4, off = (i / C4) * HSTR + j;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (j < r) {
                        if (C > 1) {
                            float4 o[kLoraMaxCluster];
#pragma unroll
                            for (int c = 0; c < kLoraMaxCluster; ++c)
                                if (c < C) o[c] = lora_ld_cluster(part_u32 + off * 4, c);
#pragma unroll
                            for (int c = 0; c < kLoraMaxCluster; ++c)
                                if (c < C) { v.x += o[c].x; v.y += o[c].y; v.z += o[c].z; v.w += o[c].w; }
                        } else {
                            v = *reinterpret_cast<const float4 *>(&sm.part[off]);
                        }
                        v.x *= s;
                        v.y = j + 1 < r ? v.y * s : 0.0f;
                        v.z = j + 2 < r ? v.z * s : 0.0f;
                        v.w = j + 3 < r ? v.w * s : 0.0f;
                    }
                    *reinterpret_cast<float4 *>(&sm.h[off]) = v;
                }
            }
            if (C > 1) { lora_cluster_arrive(); reading = true; }
            __syncthreads();

            // ---- step 2 -------------------------------------------------------------------------------------------
            // terms of s h: ranks 32 b + 8 t + (0 .. 7) of a lane feed steps 2 b and 2 b + 1 (RK = 16: 4 t + (0 .. 3))
            uint32_t ha[TERMS][KS][4];
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int col = RK == 16 ? 4 * t : 32 * (k / 2) + 8 * t + 4 * (k & 1);
                float4 va = make_float4(0.f, 0.f, 0.f, 0.f), vb = va;
                if (la) va = *reinterpret_cast<const float4 *>(&sm.h[ra * HSTR + col]);
                if (lb) vb = *reinterpret_cast<const float4 *>(&sm.h[rb * HSTR + col]);
                uint32_t c0[TERMS], c1[TERMS], c2[TERMS], c3[TERMS];
                cut_pair<TERMS>(va.x, va.y, c0);
                cut_pair<TERMS>(vb.x, vb.y, c1);
                cut_pair<TERMS>(va.z, va.w, c2);
                cut_pair<TERMS>(vb.z, vb.w, c3);
#pragma unroll
                for (int i = 0; i < TERMS; ++i) { ha[i][k][0] = c0[i]; ha[i][k][1] = c1[i]; ha[i][k][2] = c2[i]; ha[i][k][3] = c3[i]; }
            }
            // channel of a block that the lane's row of B is, + 2 for the second tile: a lane's results are 4 t .. 4 t + 3
            const int nrow = 4 * (g >> 1) + (g & 1);
            bool spoilt = false;                                      // a result of the stage may be a NaN of the cut (below)
            char *ya_at = y + ((size_t)(chunk + (la ? sm.perm[at + ra] : 0)) * N + ch0 + 4 * t) * E;
            char *yb_at = y + ((size_t)(chunk + (lb ? sm.perm[at + rb] : 0)) * N + ch0 + 4 * t) * E;
            // 16 channels of the stage at byte `st` for the lane's 16 tokens: tokens are the rows of mma.sync, channels its columns
            auto block = [&](uint32_t st, int blk) {
                const uint32_t brow[2] = {st + (blk * 16 + nrow) * (RK * 2), st + (blk * 16 + nrow + 2) * (RK * 2)};
                // One sum per term: short chains of dependent products, and the small terms are added up among themselves,
                // so that the instruction's truncation of their sums is small too.
                float part[TERMS][2][4] = {};
                if constexpr (RK == 16) {
                    const uint2 w0 = lds64(brow[0] + 8 * t), w1 = lds64(brow[1] + 8 * t);
#pragma unroll
                    for (int i = 0; i < TERMS; ++i) {
                        lora_mma(part[i][0], ha[i][0], w0.x, w0.y);
                        lora_mma(part[i][1], ha[i][0], w1.x, w1.y);
                    }
                } else {
                    uint4 w[2][RK / 32];
#pragma unroll
                    for (int k = 0; k < RK / 32; ++k)
#pragma unroll
                        for (int j = 0; j < 2; ++j) w[j][k] = lds128(brow[j] + (((4 * k + t) ^ ((g & 1) * FB)) << 4));
#pragma unroll
                    for (int k = 0; k < RK / 32; ++k) {
#pragma unroll
                        for (int i = 0; i < TERMS; ++i)
#pragma unroll
                            for (int j = 0; j < 2; ++j) lora_mma(part[i][j], ha[i][2 * k], w[j][k].x, w[j][k].y);
#pragma unroll
                        for (int i = 0; i < TERMS; ++i)
#pragma unroll
                            for (int j = 0; j < 2; ++j) lora_mma(part[i][j], ha[i][2 * k + 1], w[j][k].z, w[j][k].w);
                    }
                }
                // An infinite value of B times a term that is zero is a NaN that its product with s h need not be.  The last
                // term is zero whenever one is, and then one of its sums is NaN.
                float z[2] = {0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) z[j] += part[TERMS - 1][j][c];
                spoilt |= isnan(z[0] + z[1]);
                float d[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        d[j][c] = part[TERMS - 1][j][c];
#pragma unroll
                        for (int i = TERMS - 2; i >= 0; --i) d[j][c] += part[i][j][c];
                    }
                float4 ya = make_float4(d[0][0], d[0][1], d[1][0], d[1][1]), yb = make_float4(d[0][2], d[0][3], d[1][2], d[1][3]);
                const uint32_t row_at = st + kBase + ra * (CH * E);
                if constexpr (Y16) {
                    const uint2 none = make_uint2(0u, 0u);
                    const uint2 qa = base ? lds64(row_at + blk * 32 + t * 8) : none, qb = base ? lds64(row_at + 8 * CH * E + blk * 32 + t * 8) : none;
                    ya.x += __uint_as_float(qa.x << 16); ya.y += __uint_as_float(qa.x & 0xFFFF0000u);
                    ya.z += __uint_as_float(qa.y << 16); ya.w += __uint_as_float(qa.y & 0xFFFF0000u);
                    yb.x += __uint_as_float(qb.x << 16); yb.y += __uint_as_float(qb.x & 0xFFFF0000u);
                    yb.z += __uint_as_float(qb.y << 16); yb.w += __uint_as_float(qb.y & 0xFFFF0000u);
                    auto pack = [](float4 v) {
                        uint2 o;
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o.x) : "f"(v.y), "f"(v.x));
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o.y) : "f"(v.w), "f"(v.z));
                        return o;
                    };
                    if (la) *reinterpret_cast<uint2 *>(ya_at + blk * 32) = pack(ya);
                    if (lb) *reinterpret_cast<uint2 *>(yb_at + blk * 32) = pack(yb);
                } else {
                    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
                    const uint32_t col = ((blk * 4 + t) ^ ((g & 1) * FY)) << 4;
                    const uint4 qa = base ? lds128(row_at + col) : none, qb = base ? lds128(row_at + 8 * CH * E + col) : none;
                    ya.x += __uint_as_float(qa.x); ya.y += __uint_as_float(qa.y);
                    ya.z += __uint_as_float(qa.z); ya.w += __uint_as_float(qa.w);
                    yb.x += __uint_as_float(qb.x); yb.y += __uint_as_float(qb.y);
                    yb.z += __uint_as_float(qb.z); yb.w += __uint_as_float(qb.w);
                    if (la) *reinterpret_cast<float4 *>(ya_at + blk * 64) = ya;
                    if (lb) *reinterpret_cast<float4 *>(yb_at + blk * 64) = yb;
                }
            };
            // The results of a block that are NaN, again: from s h in fp32 and what the stage still holds of B and base.  The
            // others keep their bits, so an infinite weight touches its channel alone.
            auto again = [&](uint32_t st, int blk) {
                asm volatile("" ::: "memory");                        // reads what `block` stored as another type
#pragma unroll 1
                for (int v = 0; v < 8; ++v) {
                    const int row = v < 4 ? ra : rb, ch = blk * 16 + 4 * t + (v & 3);
                    if (row >= n) continue;
                    char *to = (v < 4 ? ya_at : yb_at) + (blk * 16 + (v & 3)) * E;
                    const float got = Y16 ? __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(to) << 16) : *reinterpret_cast<const float *>(to);
                    if (got == got) continue;
                    const char *brow = sm.ring.stage[0] + st + ch * (RK * 2);
                    float sum = 0.0f;
#pragma unroll 1
                    for (int j = 0; j < r; ++j) {
                        const uint32_t w = *reinterpret_cast<const uint16_t *>(brow + (((j / 8) ^ ((ch & 1) * FB)) << 4) + j % 8 * 2);
                        sum = fmaf(sm.h[row * HSTR + j], __uint_as_float(w << 16), sum);
                    }
                    const char *own = sm.ring.stage[0] + st + kBase + row * (CH * E) + (((ch * E / 16) ^ ((row & 1) * FY)) << 4) + ch * E % 16;
                    if constexpr (Y16) {
                        if (base) sum += __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(own) << 16);
                        uint32_t o;
                        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(0.0f), "f"(sum));
                        *reinterpret_cast<uint16_t *>(to) = (uint16_t)o;
                    } else {
                        if (base) sum += *reinterpret_cast<const float *>(own);
                        *reinterpret_cast<float *>(to) = sum;
                    }
                }
            };
            int left = n_ch;                                          // channels from this stage on
#pragma unroll 1
            for (int q = 0; q < n2; ++q, left -= CH) {
                const uint32_t st = arrive(issue2);
                // a whole stage without a condition between its blocks: the products of one fill the waits of another
                auto all = [&](auto &&work) {
                    if (left >= CH) {
#pragma unroll
                        for (int b0 = 0; b0 < CH / 16; b0 += WN) work(st, b0 + wr);
                    } else {
#pragma unroll 1
                        for (int b0 = wr; b0 * 16 < left; b0 += WN) work(st, b0);
                    }
                };
                if (live) {
                    all(block);
                    if (spoilt) {
#pragma unroll 1
                        for (int b0 = wr; b0 < CH / 16 && b0 * 16 < left; b0 += WN) again(st, b0);
                        spoilt = false;
                    }
                }
                ya_at += CH * E; yb_at += CH * E;
            }
        }
        turn = (int)(((long long)turn + items) % clusters);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (reading) lora_cluster_wait();                                 // nobody leaves while its sums may be read
}

template <int T, int RK, bool Y16>
static cudaError_t launch_lora(LoraParams &p, cudaStream_t st) {
    auto kernel = w2a8_lora_kernel<T, RK, Y16>;
    constexpr size_t smem = sizeof(LoraSmem<LoraCfg<T, RK>>);
    static_assert(smem <= 227 * 1024, "does not fit an SM");
    static PerDeviceFlags configured;
    if (cudaError_t e = allow_dynamic_smem(kernel, configured, (int)smem)) return e;
    static PerDeviceTable<kLoraMaxCluster + 1> clusters;
    const int *resident = clusters.get(current_device(), [&](int *n) {
        for (int C = 1; C <= kLoraMaxCluster; ++C) {
            const int found = resident_clusters(kernel, C, kLoraThreads, smem);
            n[C] = found > 0 ? found : sm_count() / C;
        }
    });
    // The cluster size by the estimate above, for a guess of the tiles.  Decode batches: one per adapter that there is a token
    // for.  Many tokens: the full ones and one more per adapter, but no more of these than of the full ones and two (resident
    // adapters need not be in use: 600 tokens of 6 of 60 adapters of rank 16, 4096 x 4096, take 18.8 us with the clusters of
    // two that 60 tiles ask for, 15.8 with the four of this guess).  The number of clusters is for as many tiles as all tokens
    // may be in one sort (those without an adapter can be one more); where the chunks of 256 tokens of 16-token instances make
    // more, the clusters take them in turn.
    const int used = p.M < p.adapters ? p.M : p.adapters, full = p.M / T, bound = full + used + 1;
    const int more = used < full + 2 ? used : full + 2;
    const int tiles = T == 16 && p.M <= (long long)used * T ? used : p.M < (1 << 24) ? full + more : (1 << 24) / T;
    const int forced = env_int("W2A8_LORA_C", 0);
    const bool force = forced >= 1 && forced <= kLoraMaxCluster;
    int C = 0, n = 0;
    LoraShares cheapest = {};
    for (int c = force ? forced : 1; c <= (force ? forced : kLoraMaxCluster); c *= 2) {
        p.C = c;
        int most = 0;                                            // shares of a tile that there can be
        LoraShares best = {};
        for (int sh = 1; sh <= kLoraMaxShares; ++sh) {
            const LoraShares q = lora_shares<T, RK>(p, sh, tiles, resident[c]);
            if (sh == 1 || q.cost < best.cost) best = q;
            most = q.total > most ? q.total : most;
        }
        if (C && best.cost >= cheapest.cost) continue;
        C = c; cheapest = best;
        n = (long long)bound * most < resident[c] ? bound * most : resident[c];
    }
    p.C = C;
    p.tiles_guess = n == resident[C] ? tiles : 0;                // the estimate is for all clusters that fit
    p.width_guess = cheapest.width;
    return launch_kernel_clusters(kernel, dim3((unsigned)(n * p.C)), dim3(kLoraThreads), smem, st, pdl_enabled(),
                                  make_uint2((unsigned)p.C, 1u), p);
}

template <int RK>
static cudaError_t launch_lora_rank(LoraParams &p, bool y16, cudaStream_t st) {
    // Tiles of 16 tokens for decode batches: few tokens, or many adapters for the tokens.  Tiles of 16 / 64, us: 256 tokens of
    // 64 adapters of rank 64, gate|up of the 8B layer, 68 / 209, 300 tokens 90 / 185; 256 tokens of one adapter 27 / 29; 1024
    // tokens of 4 adapters of rank 32 73 / 62; 500 tokens, q|k|v, rank 32, 64 resident adapters: 64 in use 36 / 72, 5 in use
    // 31 / 22.  The host knows the adapters that are resident, not those in use, and pays where these are few: q|k|v, rank 16,
    // 2048 tokens of 5 of 256 adapters 79 / 40, 8192 tokens of 64 of 1024 290 / 176, of one of 1024 343 / 143.
    const int tile = env_int("W2A8_LORA_TILE", p.M <= 256 || p.M <= 8 * p.adapters ? 16 : 64);
    if (tile == 16) return y16 ? launch_lora<16, RK, true>(p, st) : launch_lora<16, RK, false>(p, st);
    return y16 ? launch_lora<64, RK, true>(p, st) : launch_lora<64, RK, false>(p, st);
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
        rank_max > kLoraMaxRank || rank_max % 8 || M > (1 << 30))      // tokens are counted in 32 bits, a chunk ahead
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
    // A result may take the place of its own base and overlaps nothing else that the call reads or writes: CTAs read all of
    // it while others write.
    auto overlap = [](const void *q, size_t nq, const void *r, size_t nr) {
        const char *a = static_cast<const char *>(q), *b = static_cast<const char *>(r);
        return r && a < b + nr && b < a + nq;
    };
    for (int i = 0; i < count; ++i) {
        const size_t ny = (size_t)M * N[i] * e;
        if (overlap(y[i], ny, x_bf16, (size_t)M * K * 2) || overlap(y[i], ny, adapter, (size_t)M * 4) ||
            overlap(y[i], ny, rank, (size_t)adapters * 4) || overlap(y[i], ny, scale, (size_t)adapters * 4))
            return W2A8_ERR_SHAPE;
        for (int j = 0; j < count; ++j) {
            const size_t nj = (size_t)M * N[j] * e, one = (size_t)adapters * rank_max * 2;
            if (overlap(y[i], ny, A[j], one * K) || overlap(y[i], ny, B[j], one * N[j])) return W2A8_ERR_SHAPE;
            if (j != i && overlap(y[i], ny, y[j], nj)) return W2A8_ERR_SHAPE;
            if (overlap(y[i], ny, p.base[j], nj) && !(i == j && p.base[j] == y[i])) return W2A8_ERR_SHAPE;
        }
    }
    if (int st = check_device()) return st;
    p.x = static_cast<const uint16_t *>(x_bf16);
    p.adapter = adapter; p.rank = rank; p.scale = scale;
    p.count = count; p.adapters = adapters; p.rank_max = rank_max; p.M = M; p.K = K;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t err = rank_max <= 16 ? launch_lora_rank<16>(p, y_is_bf16, st)
                          : rank_max <= 32 ? launch_lora_rank<32>(p, y_is_bf16, st)
                          : rank_max <= 64 ? launch_lora_rank<64>(p, y_is_bf16, st)
                                           : launch_lora_rank<128>(p, y_is_bf16, st);
    return err == cudaSuccess ? W2A8_OK : W2A8_ERR_CUDA;
}
