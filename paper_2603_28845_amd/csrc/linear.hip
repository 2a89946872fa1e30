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
using product::Big;
using product::Int8;
using product::Mid;
using product::Operand;

// A workgroup per token.  The quotient is the rounded one of 32 bits (IEEE division), ties to even.  A token that holds an infinity
// or NaN gets codes of 0 and a NaN for its scale, so that its results are NaN and no others.
template <class T>
__global__ __launch_bounds__(256) void quantize_kernel(const T* x, int64_t stride, int width, int8_t* codes, float* scales, int32_t* sums) {
    constexpr int N = 16 / int(sizeof(T));
    __shared__ float s_top[4];
    __shared__ int s_sum[4], s_odd[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T* from = x + blockIdx.x * stride;
    float top = 0.f;
    bool odd = false;
    for (int c = threadIdx.x * N; c < width; c += 256 * N) {
        float v[N];
        load_vector(v, from + c);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            top = fmaxf(top, fabsf(v[e]));
            odd = odd || !(fabsf(v[e]) < __builtin_inff());
        }
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
    int sum = 0;
    int8_t* to = codes + int64_t(blockIdx.x) * width;
    for (int c = threadIdx.x * N; c < width; c += 256 * N) {
        float v[N];
        load_vector(v, from + c);
        uint32_t word[N / 4];
#pragma unroll
        for (int w = 0; w < N / 4; ++w) word[w] = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float r = rintf(v[e] / scale);
            const int code = odd || !(scale > 0.f) ? 0 : int(fminf(fmaxf(r, -127.f), 127.f));
            sum += code;
            word[e / 4] |= uint32_t(code & 255) << (8 * (e % 4));
        }
#pragma unroll
        for (int w = 0; w < N / 4; ++w) reinterpret_cast<uint32_t*>(to + c)[w] = word[w];
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

template <class T>
__device__ __forceinline__ float bias_of(const void* bias, int64_t n) {
    return bias ? block::load_one(static_cast<const T*>(bias) + n) : 0.f;
}
// y from the sum of c (q - 128)
__device__ __forceinline__ float value(int sum, int token_sum, float token_scale, float scale, float zero, float bias) {
    const int all = sum + (128 - int(rintf(zero))) * token_sum;
    return fmaf(float(all) * token_scale, scale, bias);
}

template <class T, class S>
__global__ __launch_bounds__(S::THREADS, S::PER_CU) void linear_kernel(Args P) {
    extern __shared__ __align__(1024) char lds[];
    int64_t tm, tn;
    if (!product::tile_of(blockIdx.x, (P.tokens + S::TM - 1) / S::TM, (P.d_out + S::TN - 1) / S::TN, tm, tn)) return;
    const int64_t n0 = tn * S::TN, m0 = tm * S::TM;
    product::int16v acc[S::FR][S::FC];
    product::multiply<Int8, ALONG, ALONG, S>(lds, P.q, P.codes, n0, m0, P.inner, acc);
    product::each_four<S>([&](int i, int j, int q, int n, int m) __attribute__((always_inline)) {
        if (m0 + m >= P.tokens) return;
        const float ts = P.token_scales[m0 + m];
        const int sum = P.token_sums[m0 + m];
        T* to = static_cast<T*>(P.y) + (m0 + m) * P.y_stride + n0 + n;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t at = n0 + n + e;
            if (at < P.d_out) block::store_one(to + e, value(acc[i][j][4 * q + e], sum, ts, P.scales[at], P.zeros[at], bias_of<T>(P.bias, at)));
        }
    });
}

template <class T, class S>
onecomp_status run(const Args& P, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    if (const onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(linear_kernel<T, S>), S::LDS, done)) return st;
    const int64_t blocks = product::tile_blocks(ceil_div(P.tokens, S::TM), ceil_div(P.d_out, S::TN));
    linear_kernel<T, S><<<dim3(unsigned(blocks)), dim3(S::THREADS), S::LDS, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}
template <class T>
onecomp_status dispatch(const Args& P, hipStream_t stream) {
    const bool big = P.tokens > 128 && ceil_div(P.tokens, 256) * ceil_div(P.d_out, 256) >= 192;
    return big ? run<T, Big>(P, stream) : run<T, Mid>(P, stream);
}

}  // namespace

onecomp_status quantize_tokens_run(onecomp_dtype dtype, const Rows& x, int64_t tokens, int64_t width, int8_t* codes, float* scales, int32_t* sums,
                                   hipStream_t stream) {
    const dim3 grid{unsigned(tokens)};
    if (dtype == ONECOMP_BF16)
        quantize_kernel<uint16_t><<<grid, dim3(256), 0, stream>>>(static_cast<const uint16_t*>(x.p), x.stride, int(width), codes, scales, sums);
    else
        quantize_kernel<float><<<grid, dim3(256), 0, stream>>>(static_cast<const float*>(x.p), x.stride, int(width), codes, scales, sums);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

size_t linear_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

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
