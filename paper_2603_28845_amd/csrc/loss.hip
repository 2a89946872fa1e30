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
using product::Big;
using product::Mid;
using product::Operand;

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
    char* rows;
    // forward: target per kept token; what left-out tokens get
    int32_t* target;
    float *loss, *lse_out;
    // gradients: (dloss + dlse, dloss, lse log2(e), target) per kept token
    float4* coef;
    const float *d_loss, *d_lse, *lse;
};

// A workgroup takes 64 tokens: it counts the kept ones in front of its own (reading all targets before them: 256 KB from the
// L2 for the last of 65536 tokens), numbers its own and copies their rows.
__global__ __launch_bounds__(256) void gather_kernel(Gather g) {
    __shared__ int s_before[4], s_index[64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * 64;
    int n = 0;
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
    if (wave == 0) {
        if (kept) {
            const int at = before + rank;
            s_index[rank] = t;
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
    const int chunks = int(g.width_bytes >> 4);
    for (int r = wave; r < many; r += 4) {
        const uint4v* from = reinterpret_cast<const uint4v*>(g.h + int64_t(s_index[r]) * g.h_stride);
        uint4v* to = reinterpret_cast<uint4v*>(g.rows + int64_t(before + r) * g.width_bytes);
        for (int c = lane; c < chunks; c += 64) to[c] = from[c];
    }
}

// ---- forward ------------------------------------------------------------------------------------------------------------
struct Logits {
    Operand weight, rows;                    // rows.rows: all tokens' room; what counts is *count
    const int32_t* count;
    const int32_t* target;
    int64_t inner;
    int vocab;
    float c;                                 // scale log2(e)
    float2* parts;                           // [tile of the vocabulary][token]: maximum (in powers of two) and sum
    float* hit;
    int64_t tokens;                          // row length of parts
};

template <class E, class S>
__global__ __launch_bounds__(S::THREADS, S::PER_CU) void logits_kernel(Logits P) {
    extern __shared__ __align__(1024) char lds[];
    const int count = *P.count;
    int64_t tm, tn;
    const int64_t n_tiles = (P.vocab + S::TN - 1) / S::TN;
    if (!product::tile_of(blockIdx.x, (count + S::TM - 1) / S::TM, n_tiles, tm, tn)) return;
    const int64_t n0 = tn * S::TN, m0 = tm * S::TM;
    P.rows.rows = count;
    float16v acc[S::FR][S::FC];
    product::multiply<E, ALONG, ALONG, S>(lds, P.weight, P.rows, n0, m0, P.inner, acc);
    __syncthreads();
    // A lane holds 16 FR logits of a token: maximum, sum of powers, joined with the other half's and, through LDS, with the other
    // waves' of these tokens.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / S::WC, wc = wave % S::WC, half = lane >> 5;
    float2* red = reinterpret_cast<float2*>(lds);
    const int left = P.vocab - int(n0) - wr * S::FR * 32;          // of this wave's part
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
        const float from = top == -__builtin_inff() ? 0.f : top;
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
        for (int w = 1; w < S::WR; ++w) {
            const float2 y = red[w * S::TM + col];
            const float top = fmaxf(x.x, y.x), from = top == -__builtin_inff() ? 0.f : top;
            x = make_float2(top, x.y * __builtin_amdgcn_exp2f(x.x - from) + y.y * __builtin_amdgcn_exp2f(y.x - from));
        }
        P.parts[tn * P.tokens + m0 + col] = x;
    }
}

struct Join {
    const int32_t *count, *index;
    const float2* parts;
    const float* hit;
    int64_t tokens;
    int n_parts;
    float *loss, *lse;
};
__device__ __forceinline__ void join_two(float2& x, float2 y) {
    const float top = fmaxf(x.x, y.x), from = top == -__builtin_inff() ? 0.f : top;
    x = make_float2(top, x.y * __builtin_amdgcn_exp2f(x.x - from) + y.y * __builtin_amdgcn_exp2f(y.x - from));
}
// 64 tokens per workgroup, a lane each; sixteen waves take a sixteenth of the parts each, one after the other
__global__ __launch_bounds__(1024) void join_kernel(Join P) {
    __shared__ float2 red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, count = *P.count;
    const int m = blockIdx.x * 64 + lane;
    if (int(blockIdx.x) * 64 >= count) return;
    const int each = (P.n_parts + 15) / 16, begin = wave * each, end = min(P.n_parts, begin + each);
    float2 x = make_float2(-__builtin_inff(), 0.f);
    if (m < count) {
#pragma unroll 4
        for (int i = begin; i < end; ++i) join_two(x, P.parts[int64_t(i) * P.tokens + m]);
    }
    red[wave][lane] = x;
    __syncthreads();
    if (wave != 0 || m >= count) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) join_two(x, red[w][lane]);
    const float lse2 = x.x + __builtin_amdgcn_logf(x.y);           // of two
    const int t = P.index[m];
    if (P.loss) P.loss[t] = (lse2 - P.hit[m]) * LN2;
    if (P.lse) P.lse[t] = lse2 * LN2;
}

// ---- gradients ----------------------------------------------------------------------------------------------------------
struct LogitGrads {
    Operand weight, rows;                    // weight: from the piece's first row on
    const int32_t* count;
    const float4* coef;
    int64_t inner;
    int first, columns;                      // of the piece
    float c;
    char* piece;                             // [token][column]
    int64_t stride;                          // bytes
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

template <class E, class S>
__global__ __launch_bounds__(S::THREADS, S::PER_CU) void logit_grads_kernel(LogitGrads P) {
    extern __shared__ __align__(1024) char lds[];
    const int count = *P.count;
    int64_t tm, tn;
    if (!product::tile_of(blockIdx.x, (count + S::TM - 1) / S::TM, (P.columns + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = tn * S::TN, m0 = tm * S::TM;
    P.rows.rows = count;
    float16v acc[S::FR][S::FC];
    product::multiply<E, ALONG, ALONG, S>(lds, P.weight, P.rows, n0, m0, P.inner, acc);
    const int wc = int(threadIdx.x >> 6) % S::WC, lane = threadIdx.x & 63;
    float4 coef[S::FC];
#pragma unroll
    for (int j = 0; j < S::FC; ++j) {
        const int64_t m = m0 + (wc * S::FC + j) * 32 + (lane & 31);
        coef[j] = m < count ? P.coef[m] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    product::each_four<S>([&](int i, int j, int q, int n, int m) __attribute__((always_inline)) {
        const float4 k = coef[j];
        const int at = int(n0) + n, target = __float_as_int(k.w) - P.first - at;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = k.x * __builtin_amdgcn_exp2f(fmaf(acc[i][j][4 * q + e], P.c, -k.z)) - (target == e ? k.y : 0.f);
            if (at + e >= P.columns) x[e] = 0.f;                   // behind the vocabulary: nothing, for the product with the weight
        }
        if (m0 + m < count) store_four(reinterpret_cast<typename E::T*>(P.piece + (m0 + m) * P.stride) + at, x);
    });
}

struct GradRows {
    Operand weight, piece;                   // ACROSS, ALONG
    const int32_t* count;
    int64_t columns, share;                  // of the piece; of a share of them
    int shares, add;
    float* out;                              // [share][token][width]
    int64_t tokens;
    int width;
};
template <class E, class S>
__global__ __launch_bounds__(S::THREADS, S::PER_CU) void grad_rows_kernel(GradRows P) {
    extern __shared__ __align__(1024) char lds[];
    const int count = *P.count;
    int64_t tm, tn;
    const int share = blockIdx.y;
    if (!product::tile_of(blockIdx.x, (count + S::TM - 1) / S::TM, (P.width + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = tn * S::TN, m0 = tm * S::TM, begin = share * P.share;
    const int64_t inner = P.columns - begin < P.share ? P.columns - begin : P.share;
    P.weight.data += begin * P.weight.stride;
    P.piece.data += begin * E::ESZ;
    P.piece.rows = count;
    float16v acc[S::FR][S::FC];
    product::multiply<E, ACROSS, ALONG, S>(lds, P.weight, P.piece, n0, m0, inner < 0 ? 0 : inner, acc);
    float* const out = P.out + share * P.tokens * P.width;
    product::each_four<S>([&](int i, int j, int q, int n, int m) __attribute__((always_inline)) {
        if (m0 + m >= count || n0 + n >= P.width) return;
        float4v* to = reinterpret_cast<float4v*>(out + (m0 + m) * P.width + n0 + n);
        float4v x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * q + e];
        if (P.add) x += *to;
        *to = x;
    });
}

struct GradWeight {
    Operand rows, piece;                     // both ACROSS
    const int32_t* count;
    int columns, width;
    float scale;
    char* out;                               // the piece's first row of the gradient
    int64_t stride;
};
template <class E, class S>
__global__ __launch_bounds__(S::THREADS, S::PER_CU) void grad_weight_kernel(GradWeight P) {
    extern __shared__ __align__(1024) char lds[];
    int64_t tm, tn;
    if (!product::tile_of(blockIdx.x, (P.columns + S::TM - 1) / S::TM, (P.width + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = tn * S::TN, m0 = tm * S::TM;
    float16v acc[S::FR][S::FC];
    product::multiply<E, ACROSS, ACROSS, S>(lds, P.rows, P.piece, n0, m0, *P.count, acc);
    product::each_four<S>([&](int i, int j, int q, int n, int m) __attribute__((always_inline)) {
        if (m0 + m >= P.columns || n0 + n >= P.width) return;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = acc[i][j][4 * q + e] * P.scale;
        store_four(reinterpret_cast<typename E::T*>(P.out + (m0 + m) * P.stride) + n0 + n, x);
    });
}

// dh of every token from the shares' sums: a wave per token, zeros where it was left out
template <class T>
__global__ __launch_bounds__(256) void finish_rows_kernel(const float* parts, const int32_t* place, int64_t tokens, int width, int shares, float scale, Rows dh) {
    const int64_t t = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (t >= tokens) return;
    const int at = place[t];
    T* to = static_cast<T*>(dh.p) + t * dh.stride;
    for (int c = (threadIdx.x & 63) * 4; c < width; c += 256) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (at >= 0)
            for (int s = 0; s < shares; ++s) {
                const float4v v = *reinterpret_cast<const float4v*>(parts + (s * tokens + at) * width + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] += v[e];
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= scale;
        store_four(to + c, x);
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

// 256 x 256 tiles where they are many enough
bool big_tiles(int64_t m, int64_t n) { return m > 128 && ceil_div(m, 256) * ceil_div(n, 256) >= 192; }

template <class E, class S>
onecomp_status run_logits(const Logits& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(logits_kernel<E, S>, S::LDS, S::THREADS, product::tile_blocks(ceil_div(P.tokens, S::TM), ceil_div(P.vocab, S::TN)), 1, P, done, stream);
}
template <class E, class S>
onecomp_status run_logit_grads(const LogitGrads& P, int64_t tokens, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(logit_grads_kernel<E, S>, S::LDS, S::THREADS, product::tile_blocks(ceil_div(tokens, S::TM), ceil_div(P.columns, S::TN)), 1, P, done, stream);
}
template <class E, class S>
onecomp_status run_grad_rows(const GradRows& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(grad_rows_kernel<E, S>, S::LDS, S::THREADS, product::tile_blocks(ceil_div(P.tokens, S::TM), ceil_div(P.width, S::TN)), P.shares, P, done, stream);
}
template <class E, class S>
onecomp_status run_grad_weight(const GradWeight& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    return launch(grad_weight_kernel<E, S>, S::LDS, S::THREADS, product::tile_blocks(ceil_div(P.columns, S::TM), ceil_div(P.width, S::TN)), 1, P, done, stream);
}

int64_t vocabulary_tiles(int64_t tokens, int64_t vocab) { return ceil_div(vocab, big_tiles(tokens, vocab) ? Big::TN : Mid::TN); }

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
    if (gradient) {
        g.place = reinterpret_cast<int32_t*>(ws + s.place);
        g.coef = reinterpret_cast<float4*>(ws + s.coef);
        g.d_loss = P.d_loss;
        g.d_lse = P.d_lse;
        g.lse = P.lse;
    } else {
        g.target = reinterpret_cast<int32_t*>(ws + s.coef);
        g.loss = P.loss;
        g.lse_out = P.lse;
    }
    gather_kernel<<<dim3(unsigned(P.tokens ? ceil_div(P.tokens, 64) : 1)), dim3(256), 0, stream>>>(g);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

template <class E>
onecomp_status forward(const Loss& P, hipStream_t stream) {
    const LossSpace s = loss_space(P.tokens, P.width, P.vocab, E::ESZ, vocabulary_tiles(P.tokens, P.vocab), false);
    char* ws = static_cast<char*>(P.workspace);
    if (const onecomp_status st = gather(P, s, E::ESZ, false, stream)) return st;
    Logits L{};
    L.weight = Operand{static_cast<const char*>(P.weight.p), P.weight.stride * E::ESZ, P.vocab};
    L.rows = Operand{ws + s.rows, P.width * E::ESZ, P.tokens};
    L.count = reinterpret_cast<const int32_t*>(ws + s.count);
    L.target = reinterpret_cast<const int32_t*>(ws + s.coef);
    L.inner = P.width;
    L.vocab = int(P.vocab);
    L.c = P.scale * LOG2E;
    L.parts = reinterpret_cast<float2*>(ws + s.parts);
    L.hit = reinterpret_cast<float*>(ws + s.hit);
    L.tokens = P.tokens;
    const bool big = big_tiles(P.tokens, P.vocab);
    if (const onecomp_status st = big ? run_logits<E, Big>(L, stream) : run_logits<E, Mid>(L, stream)) return st;
    const Join J{L.count, reinterpret_cast<const int32_t*>(ws + s.index), L.parts, L.hit, P.tokens, int(vocabulary_tiles(P.tokens, P.vocab)), P.loss, P.lse};
    join_kernel<<<dim3(unsigned(ceil_div(P.tokens, 64))), dim3(1024), 0, stream>>>(J);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

template <class E>
onecomp_status backward(const Loss& P, hipStream_t stream) {
    const LossSpace s = loss_space(P.tokens, P.width, P.vocab, E::ESZ, 0, true);
    char* ws = static_cast<char*>(P.workspace);
    if (const onecomp_status st = gather(P, s, E::ESZ, true, stream)) return st;
    const int32_t* count = reinterpret_cast<const int32_t*>(ws + s.count);
    const Operand rows{ws + s.rows, P.width * E::ESZ, P.tokens};
    const int64_t pitch = s.columns * E::ESZ;
    for (int64_t first = 0; first < P.vocab; first += s.columns) {
        const int64_t columns = P.vocab - first < s.columns ? P.vocab - first : s.columns;
        const char* w = static_cast<const char*>(P.weight.p) + first * P.weight.stride * E::ESZ;
        LogitGrads G{};
        G.weight = Operand{w, P.weight.stride * E::ESZ, columns};
        G.rows = rows;
        G.count = count;
        G.coef = reinterpret_cast<const float4*>(ws + s.coef);
        G.inner = P.width;
        G.first = int(first);
        G.columns = int(columns);
        G.c = P.scale * LOG2E;
        G.piece = ws + s.piece;
        G.stride = pitch;
        if (const onecomp_status st = big_tiles(P.tokens, columns) ? run_logit_grads<E, Big>(G, P.tokens, stream) : run_logit_grads<E, Mid>(G, P.tokens, stream))
            return st;
        if (P.dh.p) {
            GradRows R{};
            R.weight = Operand{w, P.weight.stride * E::ESZ, P.width};
            R.piece = Operand{ws + s.piece, pitch, P.tokens};
            R.count = count;
            R.columns = columns;
            R.shares = int(s.shares);
            R.share = ceil_div(ceil_div(columns, s.shares), 64) * 64;
            R.add = first > 0;
            R.out = reinterpret_cast<float*>(ws + s.dh);
            R.tokens = P.tokens;
            R.width = int(P.width);
            if (const onecomp_status st = big_tiles(P.tokens, P.width) ? run_grad_rows<E, Big>(R, stream) : run_grad_rows<E, Mid>(R, stream)) return st;
        }
        if (P.dweight.p) {
            GradWeight W{};
            W.rows = Operand{ws + s.rows, P.width * E::ESZ, P.width};
            W.piece = Operand{ws + s.piece, pitch, s.columns};
            W.count = count;
            W.columns = int(columns);
            W.width = int(P.width);
            W.scale = P.scale;
            W.out = static_cast<char*>(P.dweight.p) + first * P.dweight.stride * E::ESZ;
            W.stride = P.dweight.stride * E::ESZ;
            if (const onecomp_status st = big_tiles(columns, P.width) ? run_grad_weight<E, Big>(W, stream) : run_grad_weight<E, Mid>(W, stream)) return st;
        }
    }
    if (P.dh.p && P.tokens) {
        finish_rows_kernel<typename E::T><<<dim3(unsigned(ceil_div(P.tokens, 4))), dim3(256), 0, stream>>>(
            reinterpret_cast<const float*>(ws + s.dh), reinterpret_cast<const int32_t*>(ws + s.place), P.tokens, int(P.width), int(s.shares), P.scale, P.dh);
        ONECOMP_CHECK_LAUNCH();
    }
    return ONECOMP_OK;
}

}  // namespace

size_t loss_workspace_bytes(onecomp_dtype dtype, int64_t tokens, int64_t width, int64_t vocab, bool gradient) {
    return loss_space(tokens, width, vocab, dtype == ONECOMP_BF16 ? 2 : 4, gradient ? 0 : vocabulary_tiles(tokens, vocab), gradient).all;
}
onecomp_status loss_forward_run(onecomp_dtype dtype, const Loss& P, hipStream_t stream) {
    return dtype == ONECOMP_BF16 ? forward<product::Bf16>(P, stream) : forward<product::F32>(P, stream);
}
onecomp_status loss_backward_run(onecomp_dtype dtype, const Loss& P, hipStream_t stream) {
    return dtype == ONECOMP_BF16 ? backward<product::Bf16>(P, stream) : backward<product::F32>(P, stream);
}

}  // namespace token
}  // namespace onecomp
