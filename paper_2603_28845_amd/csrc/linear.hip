// Linear layers in 8-bit integers: tokens' activations to codes with a scale per token, and their product with the codes, scales
// and zero-points of a quantized layer.
//   s_t = max_k |x_tk| / 127,  c_tk = round(x_tk / s_t),  n_t = sum_k c_tk
//   y_tn = s_t s_n sum_k c_tk (q_nk - z_n) + b_n,  the sum as  sum_k c_tk (q_nk - 128) + (128 - z_n) n_t
// Sums are whole numbers of 32 bits and exact: |c (q - z)| is at most 127 255, times 65535 values of k below 2^31.
#include "product.hpp"
#include "token.hpp"

namespace onecomp {
namespace token {
namespace {

using block::load_vector;
using product::ALONG;
using product::Int8;
using product::Operand;

// Bound by HBM where there are many tokens (8192 x 4096 bf16: 101 MB in 27 us, 3.7 TB/s), by latency where there are few (2.9 us).
// A workgroup per token, whose row stays in registers (HELD 16-byte vectors a thread; what is wider is read twice).  The quotient
// is the rounded one of 32 bits (IEEE division), ties to even.  A token that holds an infinity or NaN gets codes of 0 and a
// NaN for its scale, so that its results are NaN and no others.
template <class T, int HELD>
__global__ __launch_bounds__(256) void quantize_kernel(const T* x, int64_t stride, int width, int8_t* codes, float* scales, int32_t* sums) {
    constexpr int N = 16 / int(sizeof(T)), TURN = 256 * N;
    __shared__ float s_top[4];
    __shared__ int s_sum[4], s_odd[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = threadIdx.x * N;
    const T* from = x + blockIdx.x * stride;
    float top = 0.f;
    bool odd = false;
    auto look = [&](const float (&v)[N]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            top = fmaxf(top, fabsf(v[e]));
            odd = odd || !(fabsf(v[e]) < __builtin_inff());
        }
    };
    uint4v held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        if (first + h * TURN < width) held[h] = *reinterpret_cast<const block::uint4u*>(from + first + h * TURN);
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        if (first + h * TURN < width) {
            float v[N];
            load_vector(v, reinterpret_cast<const T*>(&held[h]));
            look(v);
        }
    for (int c = first + HELD * TURN; c < width; c += TURN) {
        float v[N];
        load_vector(v, from + c);
        look(v);
    }
    top = wave_max(top);
    odd = __any(odd);
    if (lane == 0) {
        s_top[wave] = top;
        s_odd[wave] = odd;
    }
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    odd = s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3];
    const float scale = top / 127.f;
    const bool none = odd || !(scale > 0.f);
    int sum = 0;
    int8_t* const to = codes + int64_t(blockIdx.x) * width;
    auto put = [&](const float (&v)[N], int c) __attribute__((always_inline)) {
        uint32_t word[N / 4];
#pragma unroll
        for (int w = 0; w < N / 4; ++w) word[w] = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float r = rintf(v[e] / scale);
            const int code = none ? 0 : int(fminf(fmaxf(r, -127.f), 127.f));
            sum += code;
            word[e / 4] |= uint32_t(code & 255) << (8 * (e % 4));
        }
#pragma unroll
        for (int w = 0; w < N / 4; ++w) reinterpret_cast<uint32_t*>(to + c)[w] = word[w];
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h)
        if (first + h * TURN < width) {
            float v[N];
            load_vector(v, reinterpret_cast<const T*>(&held[h]));
            put(v, first + h * TURN);
        }
    for (int c = first + HELD * TURN; c < width; c += TURN) {
        float v[N];
        load_vector(v, from + c);
        put(v, c);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        scales[blockIdx.x] = odd ? __builtin_nanf("") : scale;
        sums[blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    }
}
template <class T>
onecomp_status quantize(const Rows& x, int64_t tokens, int64_t width, int8_t* codes, float* scales, int32_t* sums, hipStream_t stream) {
    const T* from = static_cast<const T*>(x.p);
    const dim3 grid{unsigned(tokens)};
    const int64_t vectors = ceil_div(width, 256 * 16 / int64_t(sizeof(T)));
    if (vectors <= 2) quantize_kernel<T, 2><<<grid, dim3(256), 0, stream>>>(from, x.stride, int(width), codes, scales, sums);
    else quantize_kernel<T, 4><<<grid, dim3(256), 0, stream>>>(from, x.stride, int(width), codes, scales, sums);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

struct Args {
    Operand q, codes;
    int64_t inner;
    const float* token_scales;
    const int32_t* token_sums;
    const float *scales, *zeros;
    const void* bias;
    void* y;
    int64_t y_stride, tokens, d_out;
};

// A column's scale, 128 less its zero-point, and bias, in LDS
struct Columns {
    float scale[256];
    int zero[256];
    float bias[256];
};
template <class T>
__device__ __forceinline__ void load_columns(Columns& c, const Args& P, int64_t n0, int count, int threads) {
    for (int n = threadIdx.x; n < count; n += threads) {
        const int64_t at = n0 + n < P.d_out ? n0 + n : P.d_out - 1;
        c.scale[n] = P.scales[at];
        c.zero[n] = 128 - int(rintf(P.zeros[at]));
        c.bias[n] = P.bias ? block::load_one(static_cast<const T*>(P.bias) + at) : 0.f;
    }
}
// y from the sum of c (q - 128)
__device__ __forceinline__ float value(int sum, int token_sum, float token_scale, float scale, int zero, float bias) {
    return fmaf(float(sum + zero * token_sum) * token_scale, scale, bias);
}

// 8192 x 4096 x 14336: 490 to 533 us, 1.80 to 1.96 POP/s, against 2.06 of a large library product; matrix pipes 45 % busy at 2.05 GHz, L2 hits
// 78 %.  Its 1792 tiles of 256 x 256 are seven for every compute unit, each only 32 steps of k long, with a beginning and an end that
// nothing of the same unit covers (tiles of 128 x 128, two a unit: 588 us where these take 538, both with the tokens' quantization).
template <class T, class S>
__global__ __launch_bounds__(S::ALL_THREADS, S::PER_SIMD) void linear_kernel(Args P) {
    extern __shared__ __align__(1024) char lds[];
    int tm, tn;
    if (!product::my_tile(int((P.tokens + S::TM - 1) / S::TM), int((P.d_out + S::TN - 1) / S::TN), tm, tn)) return;
    const int64_t n0 = int64_t(tn) * S::TN, m0 = int64_t(tm) * S::TM;
    product::int16v acc[S::FR][S::FC];
    if (!product::multiply<Int8, ALONG, ALONG, S>(lds, P.q, P.codes, n0, m0, P.inner, acc)) return;
    __syncthreads();
    static_assert(product::out_lds<T, S>() + sizeof(Columns) <= S::LDS, "room for the columns' numbers");
    Columns& c = *reinterpret_cast<Columns*>(lds + product::out_lds<T, S>());
    load_columns<T>(c, P, n0, S::TN, S::THREADS);
    const int lane = threadIdx.x & 63, wc = int(threadIdx.x >> 6) % S::WC;
    float token_scale[S::FC];
    int token_sum[S::FC];
#pragma unroll
    for (int j = 0; j < S::FC; ++j) {
        const int64_t m = m0 + (wc * S::FC + j) * 32 + (lane & 31), at = m < P.tokens ? m : P.tokens - 1;
        token_scale[j] = P.token_scales[at];
        token_sum[j] = P.token_sums[at];
    }
    __syncthreads();
    product::store_tile<T, S, false>(
        lds,
        [&](float (&x)[4], int i, int j, int q, int n, int) __attribute__((always_inline)) {
            const float4v s = *reinterpret_cast<const float4v*>(c.scale + n), b = *reinterpret_cast<const float4v*>(c.bias + n);
            const product::int4v z = *reinterpret_cast<const product::int4v*>(c.zero + n);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = value(acc[i][j][4 * q + e], token_sum[j], token_scale[j], s[e], z[e], b[e]);
        },
        [&](int m) __attribute__((always_inline)) { return m0 + m < P.tokens ? static_cast<T*>(P.y) + (m0 + m) * P.y_stride + n0 : nullptr; }, P.d_out - n0);
}

// Few tokens: bound by reading the layer's codes once.  16 x 4096 x 14336 14.8 us (59 MB, 4.0 TB/s), 1 x 4096 x 4096 4.7 us (17 MB, in
// a launch that takes about three by itself).
template <class T, int RF, int TF>
__global__ __launch_bounds__(64 * product::FEW_WAVES) void few_tokens_kernel(Args P) {
    __shared__ __align__(16) char lds[product::few_lds<RF, TF>()];
    __shared__ Columns c;
    const int64_t n0 = int64_t(blockIdx.x) * 16 * RF;
    load_columns<T>(c, P, n0, 16 * RF, 64 * product::FEW_WAVES);
    product::multiply_few<Int8, RF, TF>(lds, P.q, P.codes, [&](int m) __attribute__((always_inline)) { return m < P.tokens ? m : -1; }, n0, P.inner);
    for (int e = threadIdx.x; e < 256 * RF * TF; e += 64 * product::FEW_WAVES) {
        const int n = e % (16 * RF), m = e / (16 * RF);
        if (n0 + n < P.d_out && m < P.tokens)
            block::store_one(static_cast<T*>(P.y) + m * P.y_stride + n0 + n,
                             value(reinterpret_cast<const int*>(lds)[e], P.token_sums[m], P.token_scales[m], c.scale[n], c.zero[n], c.bias[n]));
    }
}

template <class T, class S>
onecomp_status run(const Args& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    if (const onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(linear_kernel<T, S>), S::LDS, done)) return st;
    const int64_t blocks = product::tile_blocks(ceil_div(P.tokens, S::TM), ceil_div(P.d_out, S::TN));
    linear_kernel<T, S><<<dim3(unsigned(blocks)), dim3(S::ALL_THREADS), S::LDS, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}
template <class T, int RF, int TF>
onecomp_status run_few(const Args& P, hipStream_t stream) {
    few_tokens_kernel<T, RF, TF><<<dim3(unsigned(ceil_div(P.d_out, 16 * RF))), dim3(64 * product::FEW_WAVES), 0, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}
template <class T>
onecomp_status dispatch(const Args& P, hipStream_t stream) {
    if (few_rows(P.tokens, P.d_out, 1)) {
        // 32 outputs a workgroup where these still fill the chip: the tokens' codes are read half as often
        if (P.d_out > 8192) return run_few<T, 2, 1>(P, stream);
        return P.tokens <= 16 ? run_few<T, 1, 1>(P, stream) : P.tokens <= 32 ? run_few<T, 1, 2>(P, stream) : run_few<T, 1, 4>(P, stream);
    }
    return product::with_shape<128, true, true>(choose_tiles(P.tokens, P.d_out, steps_of(P.inner, 1), false), [&](auto shape) { return run<T, decltype(shape)>(P, stream); });
}

}  // namespace

onecomp_status quantize_tokens_run(onecomp_dtype dtype, const Rows& x, int64_t tokens, int64_t width, int8_t* codes, float* scales, int32_t* sums,
                                   hipStream_t stream) {
    return dtype == ONECOMP_BF16 ? quantize<uint16_t>(x, tokens, width, codes, scales, sums, stream) : quantize<float>(x, tokens, width, codes, scales, sums, stream);
}

onecomp_status linear_run(onecomp_dtype dtype, const Linear& L, hipStream_t stream) {
    Args P{};
    P.q = Operand{reinterpret_cast<const char*>(L.q), L.d_in, L.d_out};
    P.codes = Operand{reinterpret_cast<const char*>(L.codes), L.d_in, L.tokens};
    P.inner = L.d_in;
    P.token_scales = L.token_scales;
    P.token_sums = L.token_sums;
    P.scales = L.scales;
    P.zeros = L.zeros;
    P.bias = L.bias;
    P.y = L.y.p;
    P.y_stride = L.y.stride;
    P.tokens = L.tokens;
    P.d_out = L.d_out;
    return dtype == ONECOMP_BF16 ? dispatch<uint16_t>(P, stream) : dispatch<float>(P, stream);
}

}  // namespace token
}  // namespace onecomp
