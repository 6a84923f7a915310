// Rotary positions and per-head norms of queries and keys, on the rows that the projections write.
// Declarations and contracts: include/w2a8.h.
//
// Mathematics.  A head row x of D values; z = x, or z = x * w / sqrt(mean(x^2) + eps) with the norm.  The first
// `rot` values form rot / 2 pairs (u, v): values p and p + rot / 2 (halves) or 2 p and 2 p + 1 (neighbours).  Pair p
// of a token at position t turns by the angle t * inv_freq[p]:
//   u' = amp * (u cos - v sin),  v' = amp * (v cos + u sin);   values from `rot` on are z.
// The angle grows to t * 1 radians (1e5 and more), of which 32 bits would leave some 1e-2 of a turn wrong; so it is
// formed in 64 bits, in turns, its whole turns are dropped there, and only the rest (at most half a turn, known to
// 2^-26 of a turn) goes to sincospif.  Everything else is fp32, rounded once to the result's type.
//
// Bound: memory -- every value is read once and written once, about 3 (7 with the norm) operations per value.
// A lane therefore owns V pairs of a row in 16-byte accesses (V = 4 of fp32, 8 of bf16), G lanes a row, so that the norm
// is a shuffle inside G lanes.  A group of lanes keeps its head and goes from token to token: addresses move on by one
// addition, the norm's weights stay in registers, and the rows of the next tokens are on their way into slots of shared
// memory of each thread (registers for them would cost the occupancy that keeps the memory busy).
// The sines and cosines of the CTA's tokens are computed once, one per thread, into shared memory, while the first rows
// are on their way.  8192 tokens of 72 heads of 128 (device time): fp32 to bf16 67 us, 6.7 TB/s, what a copy reaches;
// with norms from bf16 50 us, 6.0 TB/s, where the issue of the arithmetic takes about 30 us of its own.  One token: 1.6 us.
// Sizes or strides that are no multiple of 8 go value by value (V = 1), one row at a time: 8192 tokens of 25 heads of 80 of
// which 60 values turn, fp32 to bf16, 152 us and with norms 205, where 80 values take 20 and 28 and the floor is 15.
#include <math.h>

#include "w2a8_common.cuh"

namespace w2a8 {

constexpr int kRopeMaxTensors = 4;
constexpr int kRopeMaxDim = 512;
constexpr int kRopeMaxThreads = 320;
// Means of squares that need no care: the squares of all values that count in them are normal numbers, and their sum over
// kRopeMaxDim values is finite
constexpr float kRopeLeastMean = 1e-30f, kRopeMostMean = 6e35f;
constexpr int kRopeTurns = 1024;         // pairs of sine and cosine in shared memory: tokens of a CTA times pairs

struct RopeTensor {
    const void *x;
    void *out;
    const float *weight;             // of the norm, nullptr = 1
    long long xt, xh, ot, oh;        // elements between tokens / between heads, of x and out
};
struct RopeParams {
    RopeTensor t[kRopeMaxTensors];
    int end[kRopeMaxTensors];        // rows (heads) of a token up to and with tensor i
    int rows, tokens_per_block;      // heads of a token in all; tokens of a CTA
    int head_tiles;                  // CTAs that share a token's heads, next to each other in the grid
    int M, D, half;                  // half = rot / 2
    float inv_D;
    int group_log2;                  // lanes of a row = 1 << group_log2
    int interleaved;
    const int32_t *pos;
    const double *inv_freq;
    float amp, eps;
};

// V consecutive values, copied ahead into a slot of shared memory that only this thread reads (single values: into a
// register), and as fp32
template <int V, bool B16>
struct Piece {
    static constexpr int kBytes = V * (B16 ? 2 : 4), kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const char *from) {
        if constexpr (kBytes == 16) {
            const uint4 q = *reinterpret_cast<const uint4 *>(from);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else if constexpr (kBytes == 8) {
            const uint2 q = *reinterpret_cast<const uint2 *>(from);
            w[0] = q.x; w[1] = q.y;
        } else if constexpr (B16) {
            w[0] = *reinterpret_cast<const uint16_t *>(from);
        } else {
            w[0] = *reinterpret_cast<const uint32_t *>(from);
        }
    }
    static __device__ __forceinline__ void copy(uint32_t slot, const char *from) {
        if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(slot), "l"(from) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(slot), "l"(from) : "memory");
    }
    __device__ __forceinline__ void read(uint32_t slot) {
        if constexpr (kBytes == 16)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(slot) : "memory");
        else
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(slot) : "memory");
    }
    __device__ __forceinline__ float value(int i) const {
        if constexpr (B16) return __uint_as_float((i & 1) ? (w[i / 2] & 0xFFFF0000u) : (w[i / 2] << 16));
        else return __uint_as_float(w[i]);
    }
};

// two fp32 values to two bf16, to nearest, ties to even; `lo` goes to the low half
__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int N, bool B16>
__device__ __forceinline__ void store_values(void *base, long long at, const float *v) {
    if constexpr (B16) {
        uint16_t *p = reinterpret_cast<uint16_t *>(base) + at;
        if constexpr (N % 8 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 8)
                *reinterpret_cast<uint4 *>(p + i) = make_uint4(to_bf16x2(v[i], v[i + 1]), to_bf16x2(v[i + 2], v[i + 3]),
                                                               to_bf16x2(v[i + 4], v[i + 5]), to_bf16x2(v[i + 6], v[i + 7]));
        } else if constexpr (N == 4) {
            *reinterpret_cast<uint2 *>(p) = make_uint2(to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]));
        } else {
            *p = (uint16_t)to_bf16x2(v[0], 0.0f);
        }
    } else {
        float *p = reinterpret_cast<float *>(base) + at;
        if constexpr (N == 1) {
            *p = v[0];
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 4)
                *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        }
    }
}

// Rows of the norm whose squares pass fp32's range, or are lost below it with next to no eps (a bit of far_rows per token of the
// CTA): brought to about 1 by a power of two first.  One value at a time and behind the others, which keep their registers
// that way.  What the others pay for being looked at: 8192 tokens of 72 heads of 128, bf16, 49.6 us before and 50.1 with it; 333
// tokens of 25 heads of 80 3.1 and 3.2 (4.1 with this inside their loop, by one CTA less per SM).
template <int V, bool X16, bool O16, bool HALVES>
__device__ __noinline__ void rope_far_rows(const RopeParams &p, const float2 *turn, unsigned far_rows) {
    const int G = 1 << p.group_log2, lane = threadIdx.x & (G - 1), turned_units = p.half / V;
    const int tile = blockIdx.x / p.head_tiles, head_tile = blockIdx.x - tile * p.head_tiles;
    const int row = head_tile * (blockDim.x >> p.group_log2) + (threadIdx.x >> p.group_log2);
    int which = 0;
    while (row < p.rows && row >= p.end[which]) ++which;
    const RopeTensor &t = p.t[which];
    const int head = row - (which ? p.end[which - 1] : 0);
#pragma unroll 1
    for (int token = 0; token < p.tokens_per_block; ++token) {
        const bool far = far_rows >> token & 1;
        const long long m = (long long)(blockIdx.x / p.head_tiles) * p.tokens_per_block + token;
        const long long from = m * t.xt + (long long)head * t.xh, to = m * t.ot + (long long)head * t.oh;
        auto get = [&](int i) {
            if constexpr (X16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(t.x)[from + i] << 16);
            else return static_cast<const float *>(t.x)[from + i];
        };
        float most = 0.0f, sum = 0.0f;
#pragma unroll 1
        for (int i = lane; far && i < p.D; i += G) most = fmaxf(most, fabsf(get(i)));
        __syncwarp();
        for (int o = G >> 1; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        // 2^-k, k the exponent of the largest value; 2^86 is enough for the square of the smallest there is
        const int k = most <= 3.402823466e38f ? min(max((int)(__float_as_uint(most) >> 23) - 127, -86), 126) : 0;
        const float f = __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll 1
        for (int i = lane; far && i < p.D; i += G) {
            const float z = get(i) * f;
            sum = fmaf(z, z, sum);
        }
        __syncwarp();
        for (int o = G >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const float scale = __frsqrt_rn(fmaf(sum, p.inv_D, p.eps * f * f));
#pragma unroll 1
        for (int k = lane; far && k < p.D / 2; k += G) {             // pairs, those that are not rotated behind the others
            const bool turns = k < p.half;
            const int i = HALVES && turns ? k : 2 * k, j = HALVES && turns ? k + p.half : 2 * k + 1;
            float u = get(i) * f * (scale * (t.weight ? t.weight[i] : 1.0f));
            float v = get(j) * f * (scale * (t.weight ? t.weight[j] : 1.0f));
            if (turns) {
                const float2 q = turn[token * p.half + k % V * turned_units + k / V];
                const float x = u, y = v;
                u = fmaf(x, q.x, -(y * q.y));
                v = fmaf(y, q.x, x * q.y);
            }
            store_values<1, O16>(t.out, to + i, &u);
            store_values<1, O16>(t.out, to + j, &v);
        }
    }
}

// V pairs per lane and chunk, NC chunks per lane: V = 4 (8 where both sides allow it) where sizes, strides and pointers
// allow vectors, else V = 1.
// Four pairs with the norm are held to 48 registers: with 62 the CTAs of a small batch wait for one another (see above).
template <int V, int NC, bool NORM, bool X16, bool O16, bool HALVES, bool DIRECT>
__global__ void __launch_bounds__(kRopeMaxThreads, NORM && V * NC == 4 ? 4 : V * NC <= 8 && V > 1 ? 3 : 1)
w2a8_rope_kernel(const __grid_constant__ RopeParams p) {
    constexpr int X = X16 ? 2 : 4;
    using P = Piece<V, X16>;
    // rows that are on their way: kRing slots of each thread
    constexpr int kRing = DIRECT ? 1 : NC == 1 ? 4 : 2;
    __shared__ __align__(16) float2 turn[kRopeTurns];
    __shared__ __align__(16) char ring[DIRECT ? 16 : kRing * NC * 2 * P::kBytes * kRopeMaxThreads];
    pdl_launch_dependents();
    pdl_wait();                                      // the rows, and perhaps the positions, come from earlier kernels
    const int tile = blockIdx.x / p.head_tiles, head_tile = blockIdx.x - tile * p.head_tiles;
    const int token0 = tile * p.tokens_per_block;
    const int tokens = min(p.tokens_per_block, p.M - token0);
    const int G = 1 << p.group_log2;
    const int lane = threadIdx.x & (G - 1);
    const int units = p.D / (2 * V), turned_units = p.half / V;
    const int row = head_tile * (blockDim.x >> p.group_log2) + (threadIdx.x >> p.group_log2);
    const bool live = row < p.rows;

    int which = 0;
    while (live && row >= p.end[which]) ++which;
    const RopeTensor &t = p.t[which];
    const int head = row - (which ? p.end[which - 1] : 0);
    const char *src = static_cast<const char *>(t.x) + ((long long)token0 * t.xt + (long long)head * t.xh) * X;
    char *dst = static_cast<char *>(t.out) + ((long long)token0 * t.ot + (long long)head * t.oh) * (O16 ? 2 : 4);
    const long long src_step = t.xt * X, dst_step = t.ot * (O16 ? 2 : 4);

    // The values of this lane in a row, two pieces of V each: (u, v) of pairs that lie `half` apart with HALVES, else 2V
    // consecutive values, which are pairs of neighbours.  Those that are not rotated are any two pieces.
    int off_a[NC], off_b[NC];
    bool on[NC], turned[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int unit = c * G + lane;
        on[c] = live && unit < units;
        turned[c] = unit < turned_units;
        const bool h = HALVES && turned[c];
        off_a[c] = h ? unit * V : 2 * unit * V;
        off_b[c] = h ? unit * V + p.half : 2 * unit * V + V;
    }
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * P::kBytes;
    auto slot_of = [&](int slot, int c, int piece) { return mine + ((slot * NC + c) * 2 + piece) * (kRopeMaxThreads * P::kBytes); };
    int ahead = 0;                                   // tokens whose rows have been asked for
    auto ask = [&]() {
        if constexpr (!DIRECT) {
            if (ahead < tokens) {
                const int slot = ahead % kRing;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (!on[c]) continue;
                    P::copy(slot_of(slot, c, 0), src + off_a[c] * X);
                    P::copy(slot_of(slot, c, 1), src + off_b[c] * X);
                }
                src += src_step;
                ++ahead;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    // DIRECT: rows go straight into registers, one token at a time
    P now[NC][2];
    auto load_row = [&]() {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            now[c][0] = now[c][1] = P{};
            if (!on[c]) continue;
            now[c][0].load(src + off_a[c] * X);
            now[c][1].load(src + off_b[c] * X);
        }
        src += src_step;
    };
    if constexpr (DIRECT) {
        load_row();
    } else {
#pragma unroll
        for (int i = 0; i < kRing; ++i) ask();
    }
    if (p.half > 0) {
        // One angle per thread.  The pairs of a token are stored by their place in a unit, then by unit: the lanes of a
        // group read consecutive words.
        for (int i = threadIdx.x; i < tokens * p.half; i += blockDim.x) {
            const int tok = i / p.half, k = i - tok * p.half, pair = V == 1 ? k : k % turned_units * V + k / turned_units;
            const double turns = (double)p.pos[token0 + tok] * (p.inv_freq[pair] * 0.15915494309189533576888);   // 1 / (2 pi)
            float s, c;
            sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
            turn[i] = make_float2(p.amp * c, p.amp * s);
        }
        __syncthreads();
    }
    float weight[NC][2 * V];                         // of the lane's values, for the norm
    if constexpr (NORM) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j)
                weight[c][j] = t.weight && on[c] ? t.weight[j < V ? off_a[c] + j : off_b[c] + j - V] : 1.0f;
    }
    unsigned far_rows = 0;                           // tokens whose row is left for the end
    const float2 *cs = turn + lane;
#pragma unroll 1
    for (int token = 0; token < tokens; ++token, cs += p.half, dst += dst_step) {
        float e[NC][2 * V];                          // the lane's values: the two pieces
        if constexpr (!DIRECT) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int k = 0; k < 2; ++k) now[c][k].read(slot_of(token % kRing, c, k));
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < V; ++j) { e[c][j] = now[c][0].value(j); e[c][V + j] = now[c][1].value(j); }
        bool far = false;
        if constexpr (NORM) {
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (on[c]) {
#pragma unroll
                    for (int j = 0; j < 2 * V; ++j) sum = fmaf(e[c][j], e[c][j], sum);
                }
            for (int o = G >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            const float mean = fmaf(sum, p.inv_D, p.eps);
            far = live && !(mean >= kRopeLeastMean && mean <= kRopeMostMean);
            far_rows |= (unsigned)far << token;
            const float scale = __frsqrt_rn(mean);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 2 * V; ++j) e[c][j] *= scale * weight[c][j];
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (!on[c] || far) continue;
            if (turned[c]) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 q = cs[j * turned_units + c * G];
                    float &u = HALVES ? e[c][j] : e[c][2 * j], &v = HALVES ? e[c][V + j] : e[c][2 * j + 1];
                    const float x = u, y = v;
                    u = fmaf(x, q.x, -(y * q.y));
                    v = fmaf(y, q.x, x * q.y);
                }
            }
            store_values<V, O16>(dst, off_a[c], e[c]);
            store_values<V, O16>(dst, off_b[c], e[c] + V);
        }
        // the slot is free, or the registers are: the values have been used
        if constexpr (!DIRECT) ask();
        else if (token + 1 < tokens) load_row();
    }
    if constexpr (NORM)
        if (__any_sync(0xFFFFFFFFu, far_rows)) rope_far_rows<V, X16, O16, HALVES>(p, turn, far_rows);
}

template <int V, int NC, bool NORM, bool HALVES, bool DIRECT>
static cudaError_t launch_rope_types(const RopeParams &p, bool x16, bool o16, dim3 grid, int threads, cudaStream_t st) {
    auto go = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(threads), 0, st, pdl_enabled(), p); };
    if (x16) return o16 ? go(w2a8_rope_kernel<V, NC, NORM, true, true, HALVES, DIRECT>) : go(w2a8_rope_kernel<V, NC, NORM, true, false, HALVES, DIRECT>);
    if constexpr (V == 8) return cudaErrorNotSupported;       // 8 pairs per lane are for bf16 rows
    else return o16 ? go(w2a8_rope_kernel<V, NC, NORM, false, true, HALVES, DIRECT>) : go(w2a8_rope_kernel<V, NC, NORM, false, false, HALVES, DIRECT>);
}
// A CTA of one token takes its rows straight into registers (one latency instead of two), and so do single values.
template <int V, int NC, bool NORM>
static cudaError_t launch_rope_layout(const RopeParams &p, bool x16, bool o16, dim3 grid, int threads, cudaStream_t st) {
    if constexpr (V > 1)
        if (p.tokens_per_block > 1)
            return p.interleaved ? launch_rope_types<V, NC, NORM, false, false>(p, x16, o16, grid, threads, st)
                                 : launch_rope_types<V, NC, NORM, true, false>(p, x16, o16, grid, threads, st);
    return p.interleaved ? launch_rope_types<V, NC, NORM, false, true>(p, x16, o16, grid, threads, st)
                         : launch_rope_types<V, NC, NORM, true, true>(p, x16, o16, grid, threads, st);
}

// vec: values, in rows and of the rotated part, that all sizes, strides and pointers are multiples of: 16, 8 or 1
template <bool NORM>
static cudaError_t launch_rope(RopeParams &p, int vec, bool x16, bool o16, cudaStream_t st) {
    const int V = vec == 16 && x16 ? 8 : vec >= 8 ? 4 : 1;
    const int units = p.D / (2 * V);
    p.group_log2 = 0;
    while ((1 << p.group_log2) < units && p.group_log2 < 5) ++p.group_log2;
    const int G = 1 << p.group_log2, fit = kRopeMaxThreads / G;
    // Heads over CTAs of at most kRopeMaxThreads threads.  Several tokens per CTA, up to 8, while 1150 threads per SM remain
    // (about what is resident): 72 heads of 128, bf16, with norms take at one, four and eight tokens a CTA 89, 56 and 50 us
    // for 8192 tokens; for 777 tokens one takes 11.2 us and two 9.4; 40 heads of 64 for 2048 tokens 5.2 and 6.1.
    const int tiles = (p.rows + fit - 1) / fit, groups = (p.rows + tiles - 1) / tiles;
    const int threads = (groups * G + 31) / 32 * 32, gy = (p.rows * G + threads - 1) / threads;
    p.head_tiles = gy;
    p.tokens_per_block = 1;
    while (p.tokens_per_block < 8 && 2 * p.tokens_per_block * p.half <= kRopeTurns &&
           (long long)p.M / (2 * p.tokens_per_block) * gy * threads >= 1150ll * sm_count())
        p.tokens_per_block *= 2;
    const long long ctas = (long long)((p.M + p.tokens_per_block - 1) / p.tokens_per_block) * gy;
    if (ctas > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;        // rows that no memory holds
    const dim3 grid((unsigned)ctas);
    if (V == 1) return launch_rope_layout<1, 8, NORM>(p, x16, o16, grid, threads, st);
    if (V == 8) return launch_rope_layout<8, 1, NORM>(p, x16, o16, grid, threads, st);
    return units <= 32 ? launch_rope_layout<4, 1, NORM>(p, x16, o16, grid, threads, st)
                       : launch_rope_layout<4, 2, NORM>(p, x16, o16, grid, threads, st);
}

// Where the rows of a result lie, in bytes.
struct RowSet {
    const char *at;
    long long token, head;           // bytes between tokens / heads
    int M, H;
    long long row;                   // bytes of a row
    long long token_span() const { return (H - 1) * head + row; }       // all heads of a token
    long long head_span() const { return (M - 1) * token + row; }       // all tokens of a head
    long long span() const { return (M - 1) * token + (H - 1) * head + row; }
};

// Whether two sets may share bytes.  Sets inside one another's range are told apart where they are column ranges of
// the same wider rows (one stride between tokens, or between heads, and spans that fit it side by side).
static bool rows_meet(const RowSet &a, const RowSet &b) {
    const RowSet &lo = a.at <= b.at ? a : b, &hi = a.at <= b.at ? b : a;
    const long long d = hi.at - lo.at;
    if (d >= lo.span()) return false;
    auto apart = [&](long long stride, long long lo_span, long long hi_span) {
        return stride > 0 && d % stride >= lo_span && d % stride + hi_span <= stride;
    };
    if (lo.token == hi.token && apart(lo.token, lo.token_span(), hi.token_span())) return false;
    if (lo.head == hi.head && apart(lo.head, lo.head_span(), hi.head_span())) return false;
    return true;
}

// Whether a set may share bytes with a plain array, which stands as one row of the set's strides.
static bool rows_meet_array(const RowSet &a, const void *array, long long bytes) {
    return array && rows_meet(a, {static_cast<const char *>(array), a.token, a.head, 1, 1, bytes});
}

static int rope_common(bool norm, int count, const void *const *x, int x_is_bf16, void *const *out, int out_is_bf16,
                       const float *const *weight, float eps, const int *heads, const int64_t *x_strides,
                       const int64_t *out_strides, int M, int head_dim, int rot_dim, int interleaved,
                       const int32_t *positions, const double *inv_freq, float amplitude, void *stream) {
    if (!x || !out || !heads || !x_strides || !out_strides) return W2A8_ERR_NULL;
    // tokens are counted in 32 bits, a CTA's share ahead
    if (count < 1 || count > kRopeMaxTensors || M < 1 || M > (1 << 30) || head_dim < 2 || head_dim > kRopeMaxDim || head_dim % 2 ||
        rot_dim < (norm ? 0 : 2) || rot_dim > head_dim || rot_dim % 2)
        return W2A8_ERR_SHAPE;
    if (norm && !(eps >= 0.0f)) return W2A8_ERR_SHAPE;
    if (rot_dim > 0 && (!positions || !inv_freq)) return W2A8_ERR_NULL;
    RopeParams p = {};
    int vec = head_dim % 16 == 0 && rot_dim % 16 == 0 ? 16 : head_dim % 8 == 0 && rot_dim % 8 == 0 ? 8 : 1;
    const int xe = x_is_bf16 ? 2 : 4, oe = out_is_bf16 ? 2 : 4;
    int rows = 0;
    RowSet in[kRopeMaxTensors], to[kRopeMaxTensors];
    for (int i = 0; i < count; ++i) {
        if (!x[i] || !out[i]) return W2A8_ERR_NULL;
        const long long xt = x_strides[2 * i], xh = x_strides[2 * i + 1];
        const long long ot = out_strides[2 * i], oh = out_strides[2 * i + 1];
        const int H = heads[i];
        if (H < 1 || H > (1 << 17)) return W2A8_ERR_SHAPE;
        // from the first row to the last: more than any memory, and far from the end of 64 bits in what follows
        constexpr long long kMax = 1ll << 48;
        auto fits = [](long long stride, int n) { return stride >= 0 && stride <= kMax / (n > 1 ? n - 1 : 1); };
        if (!fits(xt, M) || !fits(xh, H) || !fits(ot, M) || !fits(oh, H)) return W2A8_ERR_SHAPE;
        // rows of the result must not share elements: heads inside tokens, or tokens inside heads
        const bool by_token = (H == 1 || oh >= head_dim) && (M == 1 || ot >= (long long)(H - 1) * oh + head_dim);
        const bool by_head = (M == 1 || ot >= head_dim) && (H == 1 || oh >= (long long)(M - 1) * ot + head_dim);
        if (!by_token && !by_head) return W2A8_ERR_SHAPE;
        if (norm && weight && weight[i] && (reinterpret_cast<uintptr_t>(weight[i]) & 3u)) return W2A8_ERR_ALIGN;
        in[i] = {static_cast<const char *>(x[i]), xt * xe, xh * xe, M, H, (long long)head_dim * xe};
        to[i] = {static_cast<const char *>(out[i]), ot * oe, oh * oe, M, H, (long long)head_dim * oe};
        if (xt % 8 || xh % 8 || ot % 8 || oh % 8) vec = 1;       // 16 bytes of bf16
        p.t[i] = {x[i], out[i], norm && weight ? weight[i] : nullptr, xt, xh, ot, oh};
        rows += H;
        p.end[i] = rows;
        if (rows > (1 << 17)) return W2A8_ERR_SHAPE;             // rows times lanes of a row stay small numbers of 32 bits
    }
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < count; ++j) {
            if (i < j && rows_meet(to[i], to[j])) return W2A8_ERR_SHAPE;
            // in place means: the same rows in the same type
            const bool same = i == j && in[i].at == to[i].at && xe == oe && (M == 1 || in[i].token == to[i].token) &&
                              (heads[i] == 1 || in[i].head == to[i].head);
            if (!same && rows_meet(to[i], in[j])) return W2A8_ERR_SHAPE;
            // CTAs read these while others write
            if (rows_meet_array(to[i], p.t[j].weight, head_dim * 4ll)) return W2A8_ERR_SHAPE;
        }
    for (int i = 0; rot_dim > 0 && i < count; ++i)
        if (rows_meet_array(to[i], positions, M * 4ll) || rows_meet_array(to[i], inv_freq, rot_dim * 4ll)) return W2A8_ERR_SHAPE;
    // pointers: to the accesses' size, 16 bytes or (single values) the type's
    for (int i = 0; i < count; ++i)
        if ((reinterpret_cast<uintptr_t>(x[i]) & (vec > 1 ? 15u : xe - 1u)) ||
            (reinterpret_cast<uintptr_t>(out[i]) & (vec > 1 ? 15u : oe - 1u)))
            return W2A8_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(inv_freq) & 7u)) return W2A8_ERR_ALIGN;
    if (int st = check_device()) return st;
    p.rows = rows;
    p.M = M; p.D = head_dim; p.inv_D = 1.0f / head_dim; p.half = rot_dim / 2;
    p.interleaved = interleaved != 0;
    p.pos = positions; p.inv_freq = inv_freq; p.amp = amplitude; p.eps = eps;
    const cudaError_t e = norm ? launch_rope<true>(p, vec, x_is_bf16, out_is_bf16, (cudaStream_t)stream)
                               : launch_rope<false>(p, vec, x_is_bf16, out_is_bf16, (cudaStream_t)stream);
    return e == cudaSuccess ? W2A8_OK : W2A8_ERR_CUDA;
}

}  // namespace w2a8

using namespace w2a8;

extern "C" {

int w2a8_rope(int count, const void *const *x, int x_is_bf16, void *const *out, int out_is_bf16, const int *heads,
              const int64_t *x_strides, const int64_t *out_strides, int M, int head_dim, int rot_dim, int interleaved,
              const int32_t *positions, const double *inv_freq, float amplitude, void *stream) {
    return rope_common(false, count, x, x_is_bf16, out, out_is_bf16, nullptr, 0.0f, heads, x_strides, out_strides, M,
                       head_dim, rot_dim, interleaved, positions, inv_freq, amplitude, stream);
}

int w2a8_qk_norm_rope(int count, const void *const *x, int x_is_bf16, void *const *out, int out_is_bf16,
                      const float *const *weight, float eps, const int *heads, const int64_t *x_strides,
                      const int64_t *out_strides, int M, int head_dim, int rot_dim, int interleaved,
                      const int32_t *positions, const double *inv_freq, float amplitude, void *stream) {
    return rope_common(true, count, x, x_is_bf16, out, out_is_bf16, weight, eps, heads, x_strides, out_strides, M,
                       head_dim, rot_dim, interleaved, positions, inv_freq, amplitude, stream);
}

int w2a8_rope_frequencies(int rot_dim, double base, int scaling, double factor, double low, double high,
                          int original_length, double *inv_freq, float *amplitude) {
    if (!inv_freq || !amplitude) return W2A8_ERR_NULL;
    if (rot_dim < 2 || rot_dim > kRopeMaxDim || rot_dim % 2 || !(base > 1.0) || !isfinite(base)) return W2A8_ERR_SHAPE;
    if (scaling < W2A8_ROPE_PLAIN || scaling > W2A8_ROPE_YARN) return W2A8_ERR_SHAPE;
    if (scaling != W2A8_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return W2A8_ERR_SHAPE;
    const bool bands = scaling == W2A8_ROPE_LLAMA3 || scaling == W2A8_ROPE_YARN;
    if (bands && (original_length < 1 || !(low > 0.0) || !(high > low) || !isfinite(high))) return W2A8_ERR_SHAPE;
    if (scaling == W2A8_ROPE_NTK && rot_dim < 4) return W2A8_ERR_SHAPE;
    constexpr double kTwoPi = 6.283185307179586476925;
    const int half = rot_dim / 2;
    if (scaling == W2A8_ROPE_NTK) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
    // YaRN: the pairs between those that make `high` and `low` full turns within the trained length
    double from = 0.0, to = 1.0;
    if (scaling == W2A8_ROPE_YARN) {
        from = floor(rot_dim * log(original_length / (high * kTwoPi)) / (2.0 * log(base)));
        to = ceil(rot_dim * log(original_length / (low * kTwoPi)) / (2.0 * log(base)));
        if (from < 0.0) from = 0.0;
        if (to > rot_dim - 1) to = rot_dim - 1;
        if (to < from + 1e-3) to = from + 1e-3;
    }
    for (int i = 0; i < half; ++i) {
        const double f = pow(base, -2.0 * i / rot_dim);
        double kept = 1.0;                            // share of the frequency that is left as it was
        if (scaling == W2A8_ROPE_LINEAR) kept = 0.0;
        if (scaling == W2A8_ROPE_LLAMA3) kept = (original_length * f / kTwoPi - low) / (high - low);
        if (scaling == W2A8_ROPE_YARN) kept = 1.0 - (i - from) / (to - from);
        kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
        inv_freq[i] = kept == 1.0 ? f : f * kept + f / factor * (1.0 - kept);
    }
    *amplitude = scaling == W2A8_ROPE_YARN && factor > 1.0 ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return W2A8_OK;
}

}  // extern "C"
