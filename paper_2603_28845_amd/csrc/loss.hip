// Softmax cross entropy over a vocabulary, from the last layer's input and its weight, without keeping the logits:
//   z_tv = scale h_t . w_v,  lse_t = log sum_v exp(z_tv),  loss_t = lse_t - z_t,target
//   g_tv = (dloss_t + dlse_t) exp(z_tv - lse_t) - dloss_t [v = target],  dh_t = scale sum_v g_tv w_v,  dw_v = scale sum_t g_tv h_t
// Forward: tiles of logits stay in the accumulators, each leaves a maximum and a sum per token (8 bytes for 256 logits), which a
// second kernel joins in their order.  Gradients: logits are formed again, a piece of the vocabulary at a time; their gradients g
// go to memory once in the operands' type (one piece of them) and are multiplied with the weight and with the tokens' rows.
// Tokens that are left out (target outside the vocabulary) are dropped first: the others' rows are copied together, and what
// follows works on as many as there are.  No atomics; every sum has an order that the sizes and the number of kept tokens decide.
#include "product.hpp"
#include "token.hpp"
#include <type_traits>

namespace onecomp {
namespace token {
namespace {

using product::ACROSS;
using product::ALONG;
using product::Operand;
using product::PANELS_ACROSS;
using product::PANELS_ALONG;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float to_float(uint16_t x) { return block::bf16_value(x); }
__device__ __forceinline__ float to_float(float x) { return x; }

// ---- kept tokens --------------------------------------------------------------------------------------------------------
struct Gather {
    const int32_t* targets;
    const char* h;
    int64_t h_stride, width_bytes;           // bytes
    int tokens, vocab;
    int32_t *count, *index, *place;
    char* rows;                              // in panels
    int64_t panel;
    // forward: target per kept token; what left-out tokens get
    int32_t* target;
    float *loss, *lse_out;
    // gradients: (dloss + dlse, dloss, lse log2(e), target) per kept token
    float4* coef;
    const float *d_loss, *d_lse, *lse;
    float* unit;                             // bf16: what the logits' gradients are counted in
};

// Bound by HBM (16384 rows of 4096 bf16: 268 MB read and written in 51 us, 5.3 TB/s).
// A workgroup takes 64 tokens: it counts the kept ones in front of its own (reading all targets before them: 256 KB from the
// L2 for the last of 65536 tokens), numbers its own and copies a part of their rows.
__global__ __launch_bounds__(256) void gather_kernel(Gather g) {
    __shared__ int s_before[4], s_index[64];
    __shared__ float s_top[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * 64;
    int n = 0;
#pragma unroll 4
    for (int t = threadIdx.x; t < first; t += 256) n += uint32_t(g.targets[t]) < uint32_t(g.vocab);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    if (lane == 0) s_before[wave] = n;
    __syncthreads();
    const int before = s_before[0] + s_before[1] + s_before[2] + s_before[3];
    const int t = first + lane, target = t < g.tokens ? g.targets[t] : -1;
    const bool kept = uint32_t(target) < uint32_t(g.vocab);
    const unsigned long long mask = __ballot(kept);
    const int many = __popcll(mask), rank = __popcll(mask & ((1ull << lane) - 1));
    if (wave == 0 && kept) s_index[rank] = t;
    if (wave == 0 && blockIdx.y == 0) {
        if (kept) {
            const int at = before + rank;
            g.index[at] = t;
            if (g.coef) {
                const float dl = g.d_loss[t], dz = g.d_lse ? g.d_lse[t] : 0.f;
                g.coef[at] = make_float4(dl + dz, dl, g.lse[t] * LOG2E, __int_as_float(target));
            } else {
                g.target[at] = target;
            }
        } else if (t < g.tokens && !g.coef) {
            if (g.loss) g.loss[t] = 0.f;
            if (g.lse_out) g.lse_out[t] = 0.f;
        }
        if (g.place && t < g.tokens) g.place[t] = kept ? before + rank : -1;
        if (lane == 0 && first + 64 >= g.tokens) *g.count = before + many;
    }
    __syncthreads();
    product::rows_to_panels([&](int r) __attribute__((always_inline)) { return g.h + s_index[r] * g.h_stride; }, many, g.width_bytes,
                            g.rows + int64_t(before) * 64, g.panel, blockIdx.y * 4 + wave, gridDim.y * 4);
    if (!g.unit || blockIdx.y != 0 || first + 64 < g.tokens) return;
    // The last workgroup: the digits of the largest |d_loss| of a kept token, a number from 1 up to 2.
    float top = 0.f;
#pragma unroll 8
    for (int t = threadIdx.x; t < g.tokens; t += 256) {
        const float d = fabsf(g.d_loss[t]);
        if (uint32_t(g.targets[t]) < uint32_t(g.vocab) && d < __builtin_inff()) top = fmaxf(top, d);
    }
    top = wave_max(top);
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    if (threadIdx.x == 0) *g.unit = top < 0x1p-126f ? 1.f : __uint_as_float((__float_as_uint(top) & 0x007FFFFFu) | 0x3F800000u);
}

// ---- forward ------------------------------------------------------------------------------------------------------------
// What powers are taken relative to: the maximum; with one that is infinite nothing, so that a logit of +inf gives a sum of +inf.
__device__ __forceinline__ float base_of(float top) { return fabsf(top) < __builtin_inff() ? top : 0.f; }
__device__ __forceinline__ void join_two(float2& x, float2 y) {
    const float top = fmaxf(x.x, y.x), from = base_of(top);
    x = make_float2(top, x.y * __builtin_amdgcn_exp2f(x.x - from) + y.y * __builtin_amdgcn_exp2f(y.x - from));
}

struct Logits {
    Operand weight, rows;                    // rows.rows: all tokens' room; what counts is *count
    const int32_t* count;
    const int32_t* target;                   // of the kept tokens; few tokens: of all
    int64_t inner;
    int columns;                             // of the vocabulary
    float c;                                 // scale log2(e)
    float2* parts;                           // [token][part of the vocabulary]: maximum (in powers of two) and sum
    float* hit;
    int64_t tokens, n_parts;
};

// 16384 tokens over 128000 entries of 4096 bf16: 12.4 to 13.2 ms, 1.30 to 1.39 PFLOP/s, matrix pipes 75 % busy at 1.67 GHz: bound by power (L2 hits 87 %).
// 16 tokens: by reading the weight, 185 us.  fp32, 901 over 32003 of 500: 271 to 283 us, 102 to 107 TFLOP/s, pipes 78 % busy at 2.13 GHz.
template <class E, class S>
__global__ __launch_bounds__(S::ALL_THREADS, S::PER_SIMD) void logits_kernel(Logits P) {
    extern __shared__ __align__(1024) char lds[];
    const int count = *P.count;
    int tm, tn;
    if (!product::my_tile((count + S::TM - 1) / S::TM, (P.columns + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = int64_t(tn) * S::TN, m0 = int64_t(tm) * S::TM;
    P.rows.rows = count;
    float16v acc[S::FR][S::FC];
    if (!product::multiply<E, ALONG, PANELS_ALONG, S>(lds, P.weight, P.rows, n0, m0, P.inner, acc)) return;
    __syncthreads();
    // A lane holds 16 FR logits of a token: maximum, sum of powers, joined with the other half's and, through LDS, with the other
    // waves' of these tokens.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / S::WC, wc = wave % S::WC, half = lane >> 5;
    float2* red = reinterpret_cast<float2*>(lds);
    const int left = P.columns - int(n0) - wr * S::FR * 32;          // of this wave's part
    if (left < S::FR * 32) {
#pragma unroll
        for (int i = 0; i < S::FR; ++i)
#pragma unroll
            for (int j = 0; j < S::FC; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (i * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= left) acc[i][j][r] = -__builtin_inff();
    }
#pragma unroll
    for (int j = 0; j < S::FC; ++j) {
        const int col = (wc * S::FC + j) * 32 + (lane & 31);
        const int64_t m = m0 + col;
        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < S::FR; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
        top = fmaxf(top, __shfl_xor(top, 32, 64)) * P.c;
        const float from = base_of(top);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::FR; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], P.c, -from));
        sum += __shfl_xor(sum, 32, 64);
        if (half == 0) red[wr * S::TM + col] = make_float2(top, sum);
        const int target = m < count ? P.target[m] - int(n0) - wr * S::FR * 32 : -1;
        if (uint32_t(target) < uint32_t(S::FR * 32) && ((target >> 2) & 1) == half) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < S::FR; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((target >> 5) == i && ((target >> 3) & 3) * 4 + (target & 3) == r) x = acc[i][j][r];
            P.hit[m] = x * P.c;
        }
    }
    __syncthreads();
    for (int col = threadIdx.x; col < S::TM; col += S::THREADS) {
        if (m0 + col >= count) continue;
        float2 x = red[col];
#pragma unroll
        for (int w = 1; w < S::WR; ++w) join_two(x, red[w * S::TM + col]);
        P.parts[(m0 + col) * P.n_parts + tn] = x;
    }
}

// Which of up to 64 tokens are kept: every wave finds out by itself.  Returns their number; index, target: of the kept ones.
__device__ __forceinline__ int kept_of(const int32_t* targets, int tokens, int vocab, int* index, int* target) {
    const int lane = threadIdx.x & 63, t = lane < tokens ? targets[lane] : -1;
    const bool kept = uint32_t(t) < uint32_t(vocab);
    const unsigned long long mask = __ballot(kept);
    if (kept && threadIdx.x < 64) {
        const int rank = __popcll(mask & ((1ull << lane) - 1));
        index[rank] = lane;
        target[rank] = t;
    }
    __syncthreads();
    return __popcll(mask);
}

// Few tokens, taken where they lie: 32 entries of the vocabulary per workgroup, a half wave per token.  Bound by reading the weight
// once: 16 tokens over 64000 entries of 4096 bf16 114 us, 4.6 TB/s; over 128000 fp32 435 us, 4.8 TB/s.
template <class E, int TF>
__global__ __launch_bounds__(64 * product::FEW_WAVES) void few_logits_kernel(Logits P) {
    __shared__ __align__(16) char lds[product::few_lds<2, TF>()];
    __shared__ int s_index[64], s_target[64];
    const int count = kept_of(P.target, int(P.tokens), P.columns, s_index, s_target);
    const int64_t n0 = int64_t(blockIdx.x) * 32;
    if (count == 0) return;
    product::multiply_few<E, 2, TF>(lds, P.weight, P.rows, [&](int m) __attribute__((always_inline)) { return m < count ? s_index[m] : -1; }, n0, P.inner);
    const int n = threadIdx.x & 31;
    for (int m = threadIdx.x >> 5; m < count; m += 2 * product::FEW_WAVES) {
        const float x = n0 + n < P.columns ? reinterpret_cast<const float*>(lds)[m * 32 + n] : -__builtin_inff();
        float top = x;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
        top *= P.c;
        const float from = base_of(top);
        float sum = __builtin_amdgcn_exp2f(fmaf(x, P.c, -from));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        const int64_t t = s_index[m];
        if (n == 0) P.parts[t * P.n_parts + blockIdx.x] = make_float2(top, sum);
        if (s_target[m] == n0 + n) P.hit[t] = x * P.c;
    }
}

struct Join {
    const int32_t *count, *index;            // FEW_TOKENS: null; parts and hit go by token then
    const int32_t* targets;
    const float2* parts;
    const float* hit;
    int n_parts, vocab;
    float *loss, *lse;
};
// LANES threads per token: each takes every LANES-th part, then they join in a tree.
template <int LANES, bool FEW_TOKENS>
__global__ __launch_bounds__(256) void join_kernel(Join P) {
    __shared__ float2 red[4];
    const int m = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, l = threadIdx.x % LANES;
    float2 x = make_float2(-__builtin_inff(), 0.f);
    const bool there = FEW_TOKENS ? uint32_t(P.targets[m]) < uint32_t(P.vocab) : m < *P.count;
    if (there) {
        const float2* const from = P.parts + int64_t(m) * P.n_parts;
#pragma unroll 4
        for (int i = l; i < P.n_parts; i += LANES) join_two(x, from[i]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) join_two(x, make_float2(__shfl_xor(x.x, o, 64), __shfl_xor(x.y, o, 64)));
    if constexpr (LANES == 256) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
        __syncthreads();
        x = red[0];
        for (int w = 1; w < 4; ++w) join_two(x, red[w]);
    }
    if (l != 0 || (!there && !FEW_TOKENS)) return;
    const float lse2 = x.x + __builtin_amdgcn_logf(x.y);           // of two
    const int t = FEW_TOKENS ? m : P.index[m];
    if (P.loss) P.loss[t] = there ? (lse2 - P.hit[m]) * LN2 : 0.f;
    if (P.lse) P.lse[t] = there ? lse2 * LN2 : 0.f;
}

// ---- gradients ----------------------------------------------------------------------------------------------------------
struct LogitGrads {
    Operand weight, rows;                    // weight: from the piece's first row on
    const int32_t* count;
    const float4* coef;
    int64_t inner;
    int first, columns;                      // of the piece
    float c;
    char* piece;                             // the gradients, tokens as rows, in panels
    int64_t panel;
    const float* unit;                       // bf16
};

__device__ __forceinline__ void store_four(uint16_t* p, const float (&x)[4]) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = static_cast<__bf16>(x[e]);
    *reinterpret_cast<bf16x4*>(p) = v;
}
__device__ __forceinline__ void store_four(float* p, const float (&x)[4]) {
    float4v v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = x[e];
    *reinterpret_cast<float4v*>(p) = v;
}

// The logits again and, in place of their sums, their gradients: rounded to the operands' type, since the two products that follow take
// them so (32-bit gradients' products would cost eight times as much).  In bf16 they are counted in units of the largest weight's
// digits: where all kept tokens have one weight d, as in a mean, the targets' -d (1 - p), which are most of the gradient, are then off
// by p or a 512th at most and not all by the same up to 1/256 that d itself is rounded by.  Errors of dh and dweight against
// 64 bits, where their own rounding alone is 0.00166: one weight 0.00166 to 0.0017 (700 tokens over 4000 entries of 1024 and 8192 over 128000 of
// 4096; counted in ones 0.00167 to 0.00207, and a weight of 1.0039 made all results 0.0037 too small), weights all different 0.0022.  4915 kept
// tokens over 64000 entries of 4096: 2.2 ms, 1.16 to 1.18 PFLOP/s, pipes 63 % busy at 1.79 GHz, the stores of a tile between its products
// and the next tile's.
template <class E, class S>
__global__ __launch_bounds__(S::ALL_THREADS, S::PER_SIMD) void logit_grads_kernel(LogitGrads P) {
    extern __shared__ __align__(1024) char lds[];
    const int count = *P.count;
    int tm, tn;
    if (!product::my_tile((count + S::TM - 1) / S::TM, (P.columns + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = int64_t(tn) * S::TN, m0 = int64_t(tm) * S::TM;
    P.rows.rows = count;
    float16v acc[S::FR][S::FC];
    if (!product::multiply<E, ALONG, PANELS_ALONG, S>(lds, P.weight, P.rows, n0, m0, P.inner, acc)) return;
    const int wc = int(threadIdx.x >> 6) % S::WC, lane = threadIdx.x & 63;
    float4 coef[S::FC];
#pragma unroll
    for (int j = 0; j < S::FC; ++j) {
        const int64_t m = m0 + (wc * S::FC + j) * 32 + (lane & 31);
        coef[j] = m < count ? P.coef[m] : make_float4(0.f, 0.f, 0.f, 0.f);
        if constexpr (E::ESZ == 2) {
            coef[j].x /= *P.unit;
            coef[j].y /= *P.unit;
        }
    }
    __syncthreads();
    product::store_tile<typename E::T, S, false>(
        lds,
        [&](float (&x)[4], int i, int j, int q, int n, int) __attribute__((always_inline)) {
            const float4 k = coef[j];
            const int at = int(n0) + n, target = __float_as_int(k.w) - P.first - at;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = k.x * __builtin_amdgcn_exp2f(fmaf(acc[i][j][4 * q + e], P.c, -k.z)) - (target == e ? k.y : 0.f);
                if (at + e >= P.columns) x[e] = 0.f;               // behind the vocabulary: nothing, for the product with the weight
            }
        },
        [&](int m) __attribute__((always_inline)) {
            return m0 + m < count ? reinterpret_cast<typename E::T*>(P.piece + n0 * E::ESZ / 64 * P.panel + (m0 + m) * 64) : nullptr;
        },
        S::TN, P.panel);
}

struct GradRows {
    Operand weight, piece;                   // ACROSS, PANELS_ALONG
    const int32_t* count;
    int columns, add;                        // of this piece; whether there is something to add to
    unsigned steps, fixed, step;             // of the largest piece: what decides on the shares
    int most;                                // shares that there is room for
    float* out;                              // [share][token][width]
    int64_t tokens;
    int width;
};
// dh of the kept tokens, a piece of the vocabulary added to those before; few tiles share out the piece's columns (shares_of).  4915 x 4096
// over 64000 bf16: 2.0 to 2.1 ms, 1.22 to 1.31 PFLOP/s, pipes 67 % busy at 1.80 GHz, L2 hits 72 %; fp32 901 x 500 over 32003: 288 to 301 us.
template <class E, class S>
__global__ __launch_bounds__(S::ALL_THREADS, S::PER_SIMD) void grad_rows_kernel(GradRows P) {
    extern __shared__ __align__(1024) char lds[];
    const int count = *P.count;
    int tm, tn;
    const int m_tiles = (count + S::TM - 1) / S::TM, n_tiles = (P.width + S::TN - 1) / S::TN;
    const int shares = __builtin_amdgcn_readfirstlane(shares_of(m_tiles * n_tiles, P.steps, P.fixed, P.step, P.most)), share = blockIdx.y;
    if (share >= shares || !product::my_tile(m_tiles, n_tiles, tm, tn)) return;
    const int each = __builtin_amdgcn_readfirstlane((int(unsigned(P.columns + shares - 1) / unsigned(shares)) + 63) & ~63), begin = share * each;
    const int inner = P.columns - begin < each ? P.columns - begin : each;
    const int64_t n0 = int64_t(tn) * S::TN, m0 = int64_t(tm) * S::TM;
    P.weight.data += int64_t(begin) * P.weight.stride;
    P.piece.data += int64_t(begin) * E::ESZ / 64 * P.piece.stride;
    P.piece.rows = count;
    float16v acc[S::FR][S::FC];
    if (!product::multiply<E, ACROSS, PANELS_ALONG, S>(lds, P.weight, P.piece, n0, m0, inner < 0 ? 0 : inner, acc)) return;
    __syncthreads();
    float* const out = P.out + share * P.tokens * P.width;
    auto value = [&](float (&x)[4], int i, int j, int q, int, int) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * q + e];
    };
    auto row = [&](int m) __attribute__((always_inline)) { return m0 + m < count ? out + (m0 + m) * P.width + n0 : nullptr; };
    if (P.add) product::store_tile<float, S, true>(lds, value, row, P.width - n0);
    else product::store_tile<float, S, false>(lds, value, row, P.width - n0);
}

struct GradWeight {
    Operand rows, piece;                     // both PANELS_ACROSS
    const int32_t* count;
    int columns, width;
    float scale;
    char* out;                               // the piece's first row of the gradient
    int64_t stride;
    const float* unit;                       // bf16
};
// dweight of a piece's rows, over the kept tokens.  64000 x 4096 over 4915 bf16: 1.92 to 1.98 ms, 1.3 PFLOP/s, pipes 73 % busy at 1.70 GHz;
// fp32 32003 x 500 over 901: 257 to 265 us, 109 to 112 TFLOP/s.
template <class E, class S>
__global__ __launch_bounds__(S::ALL_THREADS, S::PER_SIMD) void grad_weight_kernel(GradWeight P) {
    extern __shared__ __align__(1024) char lds[];
    int tm, tn;
    if (!product::my_tile((P.columns + S::TM - 1) / S::TM, (P.width + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = int64_t(tn) * S::TN, m0 = int64_t(tm) * S::TM;
    float16v acc[S::FR][S::FC];
    if (!product::multiply<E, PANELS_ACROSS, PANELS_ACROSS, S>(lds, P.rows, P.piece, n0, m0, *P.count, acc)) return;
    const float scale = E::ESZ == 2 ? P.scale * *P.unit : P.scale;
    __syncthreads();
    product::store_tile<typename E::T, S, false>(
        lds,
        [&](float (&x)[4], int i, int j, int q, int, int) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * q + e] * scale;
        },
        [&](int m) __attribute__((always_inline)) {
            return m0 + m < P.columns ? reinterpret_cast<typename E::T*>(P.out + (m0 + m) * P.stride) + n0 : nullptr;
        },
        P.width - n0);
}

struct Finish {
    const float* parts;
    const int32_t *place, *count;
    int64_t tokens;
    int width, tile_m, tile_n, most;         // as grad_rows_kernel had them
    unsigned steps, fixed, step;
    float scale;
    Rows dh;
    const float* unit;                       // bf16
};
// dh of every token from the shares' sums, zeros where it was left out.  Bound by HBM (8192 x 4096, three fifths kept: 68 us).  A wave per token and `gridDim.y`-th part of its columns.
template <class T>
__global__ __launch_bounds__(256) void finish_rows_kernel(Finish P) {
    const int64_t t = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (t >= P.tokens) return;
    const int at = P.place[t];
    const int tiles = (*P.count + P.tile_m - 1) / P.tile_m * ((P.width + P.tile_n - 1) / P.tile_n);
    const int shares = shares_of(tiles, P.steps, P.fixed, P.step, P.most);
    const float scale = sizeof(T) == 2 ? P.scale * *P.unit : P.scale;
    T* to = static_cast<T*>(P.dh.p) + t * P.dh.stride;
    for (int c = (blockIdx.y * 64 + (threadIdx.x & 63)) * 4; c < P.width; c += gridDim.y * 256) {
        float4v x = {0.f, 0.f, 0.f, 0.f};
        if (at >= 0) {
            const float* const from = P.parts + int64_t(at) * P.width + c;
            for (int s0 = 0; s0 < shares; s0 += 8) {               // eight on their way, added in their order
                float4v v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (s0 + u < shares) v[u] = *reinterpret_cast<const float4v*>(from + (s0 + u) * P.tokens * P.width);
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (s0 + u < shares) x += v[u];
            }
        }
        const float y[4] = {x[0] * scale, x[1] * scale, x[2] * scale, x[3] * scale};
        store_four(to + c, y);
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
template <class K, class A>
onecomp_status launch(K kernel, int lds, int threads, int64_t blocks, int64_t shares, const A& args, std::atomic<uint64_t>& done, hipStream_t stream) {
    if (blocks == 0) return ONECOMP_OK;
    if (const onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(kernel), lds, done)) return st;
    kernel<<<dim3(unsigned(blocks), unsigned(shares)), dim3(unsigned(threads)), lds, stream>>>(args);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

// f(shape) for the tiles that a product of m x n results over `inner` values takes
template <class E, class F>
onecomp_status with_tiles(int64_t m, int64_t n, int64_t inner, F&& f) {
    return product::with_shape<64, E::ESZ == 2, true>(choose_tiles(m, n, steps_of(inner, E::ESZ), E::ESZ == 4), f);
}

template <class E, class S>
onecomp_status run_logits(const Logits& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(logits_kernel<E, S>, S::LDS, S::ALL_THREADS, product::tile_blocks(ceil_div(P.tokens, S::TM), ceil_div(P.columns, S::TN)), 1, P, done, stream);
}
template <class E, class S>
onecomp_status run_logit_grads(const LogitGrads& P, int64_t tokens, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(logit_grads_kernel<E, S>, S::LDS, S::ALL_THREADS, product::tile_blocks(ceil_div(tokens, S::TM), ceil_div(P.columns, S::TN)), 1, P, done, stream);
}
template <class E, class S>
onecomp_status run_grad_rows(const GradRows& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(grad_rows_kernel<E, S>, S::LDS, S::ALL_THREADS, product::tile_blocks(ceil_div(P.tokens, S::TM), ceil_div(P.width, S::TN)), P.most, P, done, stream);
}
template <class E, class S>
onecomp_status run_grad_weight(const GradWeight& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(grad_weight_kernel<E, S>, S::LDS, S::ALL_THREADS, product::tile_blocks(ceil_div(P.columns, S::TM), ceil_div(P.width, S::TN)), 1, P, done, stream);
}

template <class E>
onecomp_status run_few_logits(const Logits& P, hipStream_t stream) {
    const dim3 grid(unsigned(P.n_parts)), threads(64 * product::FEW_WAVES);
    if (P.tokens <= 16) few_logits_kernel<E, 1><<<grid, threads, 0, stream>>>(P);
    else if (E::ESZ == 2 || P.tokens <= 32) few_logits_kernel<E, 2><<<grid, threads, 0, stream>>>(P);
    else if constexpr (E::ESZ == 4) few_logits_kernel<E, 4><<<grid, threads, 0, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

int64_t n_parts(int64_t tokens, int64_t width, int64_t vocab, int esz) { return ceil_div(vocab, part_columns(tokens, width, vocab, esz)); }

onecomp_status gather(const Loss& P, const LossSpace& s, int esz, bool gradient, hipStream_t stream) {
    char* ws = static_cast<char*>(P.workspace);
    Gather g{};
    g.targets = P.targets;
    g.h = static_cast<const char*>(P.h.p);
    g.h_stride = P.h.stride * esz;
    g.width_bytes = P.width * esz;
    g.tokens = int(P.tokens);
    g.vocab = int(P.vocab);
    g.count = reinterpret_cast<int32_t*>(ws + s.count);
    g.index = reinterpret_cast<int32_t*>(ws + s.index);
    g.rows = ws + s.rows;
    g.panel = P.tokens * 64;
    if (gradient) {
        g.place = reinterpret_cast<int32_t*>(ws + s.place);
        g.coef = reinterpret_cast<float4*>(ws + s.coef);
        g.d_loss = P.d_loss;
        g.d_lse = P.d_lse;
        g.lse = P.lse;
        if (esz == 2) g.unit = reinterpret_cast<float*>(ws + s.unit);
    } else {
        g.target = reinterpret_cast<int32_t*>(ws + s.coef);
        g.loss = P.loss;
        g.lse_out = P.lse;
    }
    // about two workgroups per compute unit, as long as there are 8 KB of rows for each
    const int64_t groups = P.tokens ? ceil_div(P.tokens, 64) : 1, bytes = (P.tokens < 64 ? P.tokens : 64) * g.width_bytes;
    int64_t parts = ceil_div(512, groups);
    if (parts > bytes >> 13) parts = bytes >> 13;                  // (a wave's unit of work)
    gather_kernel<<<dim3(unsigned(groups), unsigned(parts < 1 ? 1 : parts)), dim3(256), 0, stream>>>(g);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

template <class E>
onecomp_status forward(const Loss& P, hipStream_t stream) {
    const LossSpace s = loss_space(P.tokens, P.width, P.vocab, E::ESZ, n_parts(P.tokens, P.width, P.vocab, E::ESZ), false);
    char* ws = static_cast<char*>(P.workspace);
    Logits L{};
    L.weight = Operand{static_cast<const char*>(P.weight.p), P.weight.stride * E::ESZ, P.vocab};
    L.inner = P.width;
    L.columns = int(P.vocab);
    L.c = P.scale * LOG2E;
    L.parts = reinterpret_cast<float2*>(ws + s.parts);
    L.hit = reinterpret_cast<float*>(ws + s.hit);
    L.tokens = P.tokens;
    L.n_parts = n_parts(P.tokens, P.width, P.vocab, E::ESZ);
    Join J{nullptr, nullptr, P.targets, L.parts, L.hit, int(L.n_parts), int(P.vocab), P.loss, P.lse};
    if (few_rows(P.tokens, P.vocab, E::ESZ)) {
        L.rows = Operand{static_cast<const char*>(P.h.p), P.h.stride * E::ESZ, P.tokens};
        L.target = P.targets;
        if (const onecomp_status st = run_few_logits<E>(L, stream)) return st;
        join_kernel<256, true><<<dim3(unsigned(P.tokens)), dim3(256), 0, stream>>>(J);
        ONECOMP_CHECK_LAUNCH();
        return ONECOMP_OK;
    }
    if (const onecomp_status st = gather(P, s, E::ESZ, false, stream)) return st;
    L.rows = Operand{ws + s.rows, P.tokens * 64, P.tokens};
    L.count = J.count = reinterpret_cast<const int32_t*>(ws + s.count);
    L.target = reinterpret_cast<const int32_t*>(ws + s.coef);
    J.index = reinterpret_cast<const int32_t*>(ws + s.index);
    if (const onecomp_status st = with_tiles<E>(P.tokens, P.vocab, P.width, [&](auto shape) { return run_logits<E, decltype(shape)>(L, stream); })) return st;
    if (P.tokens <= 1024) join_kernel<256, false><<<dim3(unsigned(P.tokens)), dim3(256), 0, stream>>>(J);
    else join_kernel<64, false><<<dim3(unsigned(ceil_div(P.tokens, 4))), dim3(256), 0, stream>>>(J);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

template <class E>
onecomp_status backward(const Loss& P, hipStream_t stream) {
    const LossSpace s = loss_space(P.tokens, P.width, P.vocab, E::ESZ, 0, true);
    char* ws = static_cast<char*>(P.workspace);
    if (const onecomp_status st = gather(P, s, E::ESZ, true, stream)) return st;
    const int32_t* count = reinterpret_cast<const int32_t*>(ws + s.count);
    const float* unit = reinterpret_cast<const float*>(ws + s.unit);
    const int64_t panel = P.tokens * 64;     // of what has tokens for rows
    const Tiles rows_tiles = choose_rows(P.tokens, P.width, s.columns, E::ESZ);
    const TileShape tile = rows_shape(rows_tiles, E::ESZ == 4);
    const unsigned rows_steps = unsigned(steps_of(s.columns, E::ESZ));
    for (int64_t first = 0; first < P.vocab; first += s.columns) {
        const int64_t columns = P.vocab - first < s.columns ? P.vocab - first : s.columns;
        const char* const w = static_cast<const char*>(P.weight.p) + first * P.weight.stride * E::ESZ;
        LogitGrads G{};
        G.weight = Operand{w, P.weight.stride * E::ESZ, columns};
        G.rows = Operand{ws + s.rows, panel, P.tokens};
        G.count = count;
        G.coef = reinterpret_cast<const float4*>(ws + s.coef);
        G.inner = P.width;
        G.first = int(first);
        G.columns = int(columns);
        G.c = P.scale * LOG2E;
        G.piece = ws + s.piece;
        G.panel = panel;
        G.unit = unit;
        if (const onecomp_status st =
                with_tiles<E>(P.tokens, columns, P.width, [&](auto shape) { return run_logit_grads<E, decltype(shape)>(G, P.tokens, stream); }))
            return st;
        if (P.dh.p) {
            GradRows R{};
            R.weight = Operand{w, P.weight.stride * E::ESZ, P.width};
            R.piece = Operand{ws + s.piece, panel, P.tokens};
            R.count = count;
            R.columns = int(columns);
            R.steps = rows_steps;
            R.fixed = unsigned(tile.fixed);
            R.step = unsigned(tile.step);
            R.most = int(s.shares);
            R.add = first > 0;
            R.out = reinterpret_cast<float*>(ws + s.dh);
            R.tokens = P.tokens;
            R.width = int(P.width);
            if (const onecomp_status st =
                    product::with_shape<64, true, false>(rows_tiles, [&](auto shape) { return run_grad_rows<E, decltype(shape)>(R, stream); }))
                return st;
        }
        if (P.dweight.p) {
            GradWeight W{};
            W.rows = Operand{ws + s.rows, panel, P.width};
            W.piece = Operand{ws + s.piece, panel, s.columns};
            W.count = count;
            W.columns = int(columns);
            W.width = int(P.width);
            W.scale = P.scale;
            W.unit = unit;
            W.out = static_cast<char*>(P.dweight.p) + first * P.dweight.stride * E::ESZ;
            W.stride = P.dweight.stride * E::ESZ;
            if (const onecomp_status st = with_tiles<E>(columns, P.width, P.tokens, [&](auto shape) { return run_grad_weight<E, decltype(shape)>(W, stream); })) return st;
        }
    }
    if (P.dh.p && P.tokens) {
        const Finish F{reinterpret_cast<const float*>(ws + s.dh), reinterpret_cast<const int32_t*>(ws + s.place), count, P.tokens, int(P.width), tile.m, tile.n,
                       int(s.shares), rows_steps, unsigned(tile.fixed), unsigned(tile.step), P.scale, P.dh, unit};
        const int64_t groups = ceil_div(P.tokens, 4), parts = ceil_div(1024, groups), most = ceil_div(P.width, 256);
        finish_rows_kernel<typename E::T><<<dim3(unsigned(groups), unsigned(parts < most ? parts : most)), dim3(256), 0, stream>>>(F);
        ONECOMP_CHECK_LAUNCH();
    }
    return ONECOMP_OK;
}

}  // namespace

size_t loss_workspace_bytes(onecomp_dtype dtype, int64_t tokens, int64_t width, int64_t vocab, bool gradient) {
    return loss_space(tokens, width, vocab, dtype == ONECOMP_BF16 ? 2 : 4, gradient ? 0 : n_parts(tokens, width, vocab, dtype == ONECOMP_BF16 ? 2 : 4), gradient).all;
}
onecomp_status loss_forward_run(onecomp_dtype dtype, const Loss& P, hipStream_t stream) {
    return dtype == ONECOMP_BF16 ? forward<product::Bf16>(P, stream) : forward<product::F32>(P, stream);
}
onecomp_status loss_backward_run(onecomp_dtype dtype, const Loss& P, hipStream_t stream) {
    return dtype == ONECOMP_BF16 ? backward<product::Bf16>(P, stream) : backward<product::F32>(P, stream);
}

}  // namespace token
}  // namespace onecomp
