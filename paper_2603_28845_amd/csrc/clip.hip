// The norm of many gradients together, and the gradients scaled to at most a given norm.
#include "block.hpp"

namespace onecomp {
namespace block {
namespace {

// Gradients of one launch, passed by value: no table in memory, nothing to copy before the kernels can start.
constexpr int MOST = 96, CHUNK = 16384;                           // tensors of a launch, entries of a workgroup's piece
struct Table {
    const void* in[MOST];
    void* out[MOST];
    int64_t n[MOST];
    int32_t first[MOST + 1];                                      // pieces before this tensor's
    uint32_t bf16[MOST / 32];                                     // bit per tensor
    int32_t tensors;
};
static_assert(sizeof(Table) <= 3072, "kernel arguments");

constexpr int PARTS = 1024;                                       // workgroups of the first pass: sums that the second adds up

// The piece's tensor: the last whose first piece is not behind it.  Wave-uniform.
__device__ __forceinline__ int tensor_of(const Table& t, int piece) {
    int lo = 0, hi = t.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= piece) lo = mid; else hi = mid;
    }
    return lo;
}

// f(entries of tensor i, and from which on): 16 bytes at a time, then what is left of the piece one by one
template <class T, class F>
__device__ __forceinline__ void each(const Table& t, int i, int64_t begin, F& f) {
    constexpr int N = 16 / int(sizeof(T));
    const T* in = static_cast<const T*>(t.in[i]) + begin;
    const int64_t left = t.n[i] - begin;
    const int n = int(left < CHUNK ? left : CHUNK), whole = n / N;
    for (int v = threadIdx.x; v < whole; v += 256) {
        float x[N];
        load_vector(x, in + N * v);
        f.template some<T>(x, i, begin + N * v);
    }
    for (int v = whole * N + threadIdx.x; v < n; v += 256) {
        float x[1] = {load_one(in + v)};
        f.template some<T>(x, i, begin + v);
    }
}
template <class F>
__device__ __forceinline__ void each(const Table& t, int piece, F& f) {
    const int i = tensor_of(t, piece);
    const int64_t begin = int64_t(piece - t.first[i]) * CHUNK;
    if (t.bf16[i >> 5] >> (i & 31) & 1) each<uint16_t>(t, i, begin, f);
    else each<float>(t, i, begin, f);
}

__device__ __forceinline__ double workgroup_sum(double x, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    __syncthreads();
    return x;
}

// Squares are added in 64 bits: exact products, no overflow of large gradients, and the rate of 64-bit additions is far above
// what memory delivers.
struct Squares {
    double sum;
    template <class T, int N>
    __device__ __forceinline__ void some(const float (&x)[N], int, int64_t) {
#pragma unroll
        for (int e = 0; e < N; ++e) sum = fma(double(x[e]), double(x[e]), sum);
    }
};

// Both passes are bound by memory: 0.87 GB of fp32 gradients read in 170 us (5.1 TB/s), read and written in 315 (5.5 TB/s); 60
// small tensors 5 and 6 us.
// Workgroup b adds up the pieces b, b + grid, ... to parts[b]; launches behind the first add to what is there.
__global__ __launch_bounds__(256) void squares_kernel(const Table t, double* parts, const int add) {
    __shared__ double lds[4];
    Squares s{0.0};
    for (int piece = blockIdx.x; piece < t.first[t.tensors]; piece += gridDim.x) each(t, piece, s);
    const double sum = workgroup_sum(s.sum, lds);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum + (add ? parts[blockIdx.x] : 0.0);
}

struct Scale {
    const Table& t;
    float f;
    template <class T, int N>
    __device__ __forceinline__ void some(const float (&x)[N], int i, int64_t at) const {
        if (f == 1.f && t.in[i] == t.out[i]) return;              // in place and nothing to clip
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[e] * f;
        T* to = static_cast<T*>(t.out[i]) + at;
        if constexpr (N == 1) store_one(to, y[0]);
        else store_vector(to, y);
    }
};

// Every workgroup adds the sums up by itself (8 KB, in one order: the same bits in all of them), then scales its pieces, from
// the last on: what the first pass read last is still in the cache.
__global__ __launch_bounds__(256) void scale_kernel(const Table t, const double* parts, const int n_parts, const float max_norm, float* norm_out) {
    __shared__ double lds[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_parts; i += 256) sum += parts[i];
    const double norm = sqrt(workgroup_sum(sum, lds));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = float(norm);
    const double f = double(max_norm) / (norm + 1e-6);
    const Scale scale{t, f < 1.0 ? float(f) : f == f ? 1.f : __builtin_nanf("")};
    const int pieces = t.first[t.tensors];
    for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) each(t, pieces - 1 - piece, scale);
}

}  // namespace

size_t clip_workspace_bytes() { return PARTS * sizeof(double); }

onecomp_status clip_run(const onecomp_gradient* grads, int n, float max_norm, float* norm, void* workspace, hipStream_t stream) {
    double* parts = static_cast<double*>(workspace);
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += ceil_div(grads[i].numel, CHUNK);
    const int used = int(all < 1 ? 1 : all < PARTS ? all : PARTS);   // workgroups of the first pass, sums that it leaves
    for (int pass = 0; pass < 2; ++pass) {
        bool first = true;
        int at = 0;
        do {
            Table t{};
            int64_t pieces = 0;
            while (at < n && t.tensors < MOST) {
                const onecomp_gradient& g = grads[at];
                if (g.numel == 0) { ++at; continue; }
                const int64_t more = ceil_div(g.numel, CHUNK);
                if (pieces + more > (1 << 30)) {
                    if (t.tensors) break;
                    return ONECOMP_ERR_UNSUPPORTED;
                }
                const int i = t.tensors++;
                t.in[i] = g.grad;
                t.out[i] = g.out;
                t.n[i] = g.numel;
                t.first[i] = int32_t(pieces);
                if (g.dtype == ONECOMP_BF16) t.bf16[i >> 5] |= 1u << (i & 31);
                pieces += more;
                ++at;
            }
            t.first[t.tensors] = int32_t(pieces);
            if (pass == 0) {
                squares_kernel<<<dim3(unsigned(used)), dim3(256), 0, stream>>>(t, parts, first ? 0 : 1);
            } else {
                const int grid = int(pieces < 4096 ? (pieces < 1 ? 1 : pieces) : 4096);
                scale_kernel<<<dim3(unsigned(grid)), dim3(256), 0, stream>>>(t, parts, used, max_norm, first ? norm : nullptr);
            }
            ONECOMP_CHECK_LAUNCH();
            first = false;
        } while (at < n);
    }
    return ONECOMP_OK;
}

}  // namespace block
}  // namespace onecomp
