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
// A lane therefore owns V = 4 pairs of a row (two 16-byte loads of fp32), G lanes a row, so that the norm is a
// shuffle inside G lanes; a CTA takes the rows of one token, whose sines and cosines it computes once, into shared
// memory, while the loads of its first rows are on their way.
#include <math.h>

#include "w2a8_common.cuh"

namespace w2a8 {

constexpr int kRopeMaxTensors = 4;
constexpr int kRopeMaxDim = 512;
constexpr int kRopeMaxThreads = 320;

struct RopeTensor {
    const void *x;
    void *out;
    const float *weight;             // of the norm, nullptr = 1
    long long xt, xh, ot, oh;        // elements between tokens / between heads, of x and out
};
struct RopeParams {
    RopeTensor t[kRopeMaxTensors];
    int end[kRopeMaxTensors];        // rows (heads) of a token up to and with tensor i
    int rows, rows_per_block;        // heads of a token in all / of them, per CTA
    int M, D, half;                  // half = rot / 2
    int group_log2;                  // lanes of a row = 1 << group_log2
    int interleaved;
    const int32_t *pos;
    const double *inv_freq;
    float amp, eps;
};

// N consecutive values, N = 1, 4 or 8
template <int N, bool B16>
__device__ __forceinline__ void load_values(const void *base, long long at, float *v) {
    if constexpr (B16) {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(base) + at;
        uint32_t w[(N + 1) / 2];
        if constexpr (N == 8) {
            const uint4 q = *reinterpret_cast<const uint4 *>(p);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else if constexpr (N == 4) {
            const uint2 q = *reinterpret_cast<const uint2 *>(p);
            w[0] = q.x; w[1] = q.y;
        } else {
            w[0] = *p;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = __uint_as_float((i & 1) ? (w[i / 2] & 0xFFFF0000u) : (w[i / 2] << 16));
    } else {
        const float *p = reinterpret_cast<const float *>(base) + at;
        if constexpr (N == 1) {
            v[0] = *p;
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 q = *reinterpret_cast<const float4 *>(p + i);
                v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
            }
        }
    }
}

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
        if constexpr (N == 8)
            *reinterpret_cast<uint4 *>(p) = make_uint4(to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]),
                                                       to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7]));
        else if constexpr (N == 4)
            *reinterpret_cast<uint2 *>(p) = make_uint2(to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]));
        else
            *p = (uint16_t)to_bf16x2(v[0], 0.0f);
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

// V pairs per lane and chunk, NC chunks per lane: V = 4 where sizes, strides and pointers allow vectors, else V = 1.
template <int V, int NC, bool NORM, bool X16, bool O16>
__global__ void __launch_bounds__(kRopeMaxThreads)
w2a8_rope_kernel(const RopeParams p) {
    __shared__ float2 turn[kRopeMaxDim / 2];
    pdl_launch_dependents();
    pdl_wait();                                      // the rows, and perhaps the positions, come from earlier kernels
    const int token = blockIdx.x;
    const int G = 1 << p.group_log2;
    const int lane = threadIdx.x & (G - 1), group = threadIdx.x >> p.group_log2;
    const int groups = blockDim.x >> p.group_log2;
    const int units = p.D / (2 * V);
    const int row0 = blockIdx.y * p.rows_per_block;
    const int row1 = min(p.rows, row0 + p.rows_per_block);

    float u[NC][V], v[NC][V];
    const RopeTensor *t = nullptr;
    int head = 0;
    // the pairs of this lane: values (a + j, b + j) of the row, or 2V consecutive ones from 2 * pair on
    auto load_row = [&](int row) {
        int i = 0;
        while (row >= p.end[i]) ++i;
        t = &p.t[i];
        head = row - (i ? p.end[i - 1] : 0);
        const long long at = (long long)token * t->xt + (long long)head * t->xh;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int unit = c * G + lane;
#pragma unroll
            for (int j = 0; j < V; ++j) { u[c][j] = 0.0f; v[c][j] = 0.0f; }
            if (unit >= units) continue;
            const int pair = unit * V;
            if (pair < p.half && !p.interleaved) {
                load_values<V, X16>(t->x, at + pair, u[c]);
                load_values<V, X16>(t->x, at + pair + p.half, v[c]);
            } else if constexpr (V == 4) {
                float e[8];
                load_values<8, X16>(t->x, at + 2 * pair, e);
#pragma unroll
                for (int j = 0; j < V; ++j) { u[c][j] = e[2 * j]; v[c][j] = e[2 * j + 1]; }
            } else {
                load_values<1, X16>(t->x, at + 2 * pair, u[c]);
                load_values<1, X16>(t->x, at + 2 * pair + 1, v[c]);
            }
        }
    };

    int row = row0 + group;
    const bool first = row < row1;
    if (first) load_row(row);
    if (p.half > 0) {
        const double t64 = (double)p.pos[token];
        for (int i = threadIdx.x; i < p.half; i += blockDim.x) {
            const double turns = t64 * (p.inv_freq[i] * 0.15915494309189533576888);     // 1 / (2 pi)
            float s, c;
            sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
            turn[i] = make_float2(p.amp * c, p.amp * s);
        }
        __syncthreads();
    }
    // every lane of a warp goes the same number of rounds, for the shuffles of the norm
    for (int base = row0; base < row1; base += groups, row += groups) {
        const bool live = row < row1;
        if (base != row0 && live) load_row(row);
        if constexpr (NORM) {
            float sum = 0.0f;
            if (live) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < V; ++j) sum = fmaf(u[c][j], u[c][j], fmaf(v[c][j], v[c][j], sum));
            }
            for (int o = G >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            const float scale = 1.0f / sqrtf(sum / (float)p.D + p.eps);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) { u[c][j] *= scale; v[c][j] *= scale; }
        }
        if (!live) continue;
        const long long at = (long long)token * t->ot + (long long)head * t->oh;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int unit = c * G + lane;
            if (unit >= units) continue;
            const int pair = unit * V;
            const bool turned = pair < p.half, halves = turned && !p.interleaved;
            if constexpr (NORM) {
                if (t->weight) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        u[c][j] *= t->weight[halves ? pair + j : 2 * (pair + j)];
                        v[c][j] *= t->weight[halves ? pair + j + p.half : 2 * (pair + j) + 1];
                    }
                }
            }
            if (turned) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 cs = turn[pair + j];
                    const float a = u[c][j], b = v[c][j];
                    u[c][j] = fmaf(a, cs.x, -(b * cs.y));
                    v[c][j] = fmaf(b, cs.x, a * cs.y);
                }
            }
            if (halves) {
                store_values<V, O16>(t->out, at + pair, u[c]);
                store_values<V, O16>(t->out, at + pair + p.half, v[c]);
            } else if constexpr (V == 4) {
                float e[8];
#pragma unroll
                for (int j = 0; j < V; ++j) { e[2 * j] = u[c][j]; e[2 * j + 1] = v[c][j]; }
                store_values<8, O16>(t->out, at + 2 * pair, e);
            } else {
                store_values<1, O16>(t->out, at + 2 * pair, u[c]);
                store_values<1, O16>(t->out, at + 2 * pair + 1, v[c]);
            }
        }
    }
}

template <int V, int NC, bool NORM>
static cudaError_t launch_rope_types(const RopeParams &p, bool x16, bool o16, dim3 grid, int threads, cudaStream_t st) {
    auto go = [&](auto kernel) { return launch_kernel(kernel, grid, dim3(threads), 0, st, pdl_enabled(), p); };
    if (x16) return o16 ? go(w2a8_rope_kernel<V, NC, NORM, true, true>) : go(w2a8_rope_kernel<V, NC, NORM, true, false>);
    return o16 ? go(w2a8_rope_kernel<V, NC, NORM, false, true>) : go(w2a8_rope_kernel<V, NC, NORM, false, false>);
}

template <bool NORM>
static cudaError_t launch_rope(RopeParams &p, bool vec, bool x16, bool o16, cudaStream_t st) {
    const int units = p.D / (vec ? 8 : 2);
    p.group_log2 = 0;
    while ((1 << p.group_log2) < units && p.group_log2 < 5) ++p.group_log2;
    const int G = 1 << p.group_log2;
    // rows of a token over CTAs of at most kRopeMaxThreads threads: one round each while there are few tokens
    // (latency), all rows in as few CTAs as the rounds allow otherwise (sines and cosines once per token)
    const int fit = kRopeMaxThreads / G;
    p.rows_per_block = (long long)p.M * ((p.rows + fit - 1) / fit) <= 2 * sm_count() ? (p.rows < fit ? p.rows : fit) : p.rows;
    const int rounds = (p.rows_per_block + fit - 1) / fit;
    const int groups = (p.rows_per_block + rounds - 1) / rounds;
    const int threads = (groups * G + 31) / 32 * 32;
    const dim3 grid((unsigned)p.M, (unsigned)((p.rows + p.rows_per_block - 1) / p.rows_per_block));
    if (!vec) return launch_rope_types<1, 8, NORM>(p, x16, o16, grid, threads, st);
    return units <= 32 ? launch_rope_types<4, 1, NORM>(p, x16, o16, grid, threads, st)
                       : launch_rope_types<4, 2, NORM>(p, x16, o16, grid, threads, st);
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

static int rope_common(bool norm, int count, const void *const *x, int x_is_bf16, void *const *out, int out_is_bf16,
                       const float *const *weight, float eps, const int *heads, const int64_t *x_strides,
                       const int64_t *out_strides, int M, int head_dim, int rot_dim, int interleaved,
                       const int32_t *positions, const double *inv_freq, float amplitude, void *stream) {
    if (!x || !out || !heads || !x_strides || !out_strides) return W2A8_ERR_NULL;
    if (count < 1 || count > kRopeMaxTensors || M < 1 || head_dim < 2 || head_dim > kRopeMaxDim || head_dim % 2 ||
        rot_dim < (norm ? 0 : 2) || rot_dim > head_dim || rot_dim % 2)
        return W2A8_ERR_SHAPE;
    if (norm && !(eps >= 0.0f)) return W2A8_ERR_SHAPE;
    if (rot_dim > 0 && (!positions || !inv_freq)) return W2A8_ERR_NULL;
    RopeParams p = {};
    bool vec = head_dim % 8 == 0 && rot_dim % 8 == 0;
    const int xe = x_is_bf16 ? 2 : 4, oe = out_is_bf16 ? 2 : 4;
    int rows = 0;
    RowSet in[kRopeMaxTensors], to[kRopeMaxTensors];
    for (int i = 0; i < count; ++i) {
        if (!x[i] || !out[i]) return W2A8_ERR_NULL;
        const long long xt = x_strides[2 * i], xh = x_strides[2 * i + 1];
        const long long ot = out_strides[2 * i], oh = out_strides[2 * i + 1];
        const int H = heads[i];
        constexpr long long kMax = 1ll << 40;
        if (H < 1 || H > (1 << 20) || xt < 0 || xh < 0 || ot < 0 || oh < 0 || xt > kMax || xh > kMax || ot > kMax ||
            oh > kMax)
            return W2A8_ERR_SHAPE;
        // rows of the result must not share elements: heads inside tokens, or tokens inside heads
        const bool by_token = (H == 1 || oh >= head_dim) && (M == 1 || ot >= (long long)(H - 1) * oh + head_dim);
        const bool by_head = (M == 1 || ot >= head_dim) && (H == 1 || oh >= (long long)(M - 1) * ot + head_dim);
        if (!by_token && !by_head) return W2A8_ERR_SHAPE;
        if (!aligned16(x[i]) || !aligned16(out[i])) return W2A8_ERR_ALIGN;
        if (norm && weight && weight[i] && (reinterpret_cast<uintptr_t>(weight[i]) & 3u)) return W2A8_ERR_ALIGN;
        in[i] = {static_cast<const char *>(x[i]), xt * xe, xh * xe, M, H, (long long)head_dim * xe};
        to[i] = {static_cast<const char *>(out[i]), ot * oe, oh * oe, M, H, (long long)head_dim * oe};
        vec = vec && xt % 8 == 0 && xh % 8 == 0 && ot % 8 == 0 && oh % 8 == 0;
        p.t[i] = {x[i], out[i], norm && weight ? weight[i] : nullptr, xt, xh, ot, oh};
        rows += H;
        p.end[i] = rows;
        if (rows > (1 << 21)) return W2A8_ERR_SHAPE;
    }
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < count; ++j) {
            if (i < j && rows_meet(to[i], to[j])) return W2A8_ERR_SHAPE;
            // in place means: the same rows in the same type
            const bool same = i == j && in[i].at == to[i].at && xe == oe && (M == 1 || in[i].token == to[i].token) &&
                              (heads[i] == 1 || in[i].head == to[i].head);
            if (!same && rows_meet(to[i], in[j])) return W2A8_ERR_SHAPE;
        }
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(inv_freq) & 7u)) return W2A8_ERR_ALIGN;
    if (int st = check_device()) return st;
    p.rows = rows;
    p.M = M; p.D = head_dim; p.half = rot_dim / 2;
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
