// Rows of an embedding table, scaled, and the table's gradient.
//   out_t = scale table[token_t],   d table_v = base_v + scale sum over t with token_t = v of d_out_t
// Tokens outside the vocabulary mark padding: zeros forward, no part in the gradient.
//
// Gradient: three kernels.  (1) Sorting: a workgroup owns a range of the vocabulary and goes through all tokens twice, counting its
// own per wave and row, then placing them; no workgroup waits for another, and equal tokens stay in their order.  (2) Sums: waves
// add up `segment` sorted tokens each in 32 bits; rows whose tokens all lie in one segment are finished there, the others leave a
// partial sum per segment.  Rows without a token are filled by further workgroups of the same launch.  (3) Rows that cross segments
// are joined in their order.  So frequent tokens are spread over the chip, and the same inputs give the same bits.
#include "token.hpp"

namespace onecomp {
namespace token {
namespace {

using block::load_one;
using block::load_vector;
using block::store_one;
using block::store_vector;

// n of a vector's entries, at the end of a row
template <class T, int N>
__device__ __forceinline__ void load_some(float (&x)[N], const T* p, int n) {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = e < n ? load_one(p + e) : 0.f;
}
template <class T, int N>
__device__ __forceinline__ void store_some(T* p, const float (&x)[N], int n) {
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < n) store_one(p + e, x[e]);
}
template <class T, int N>
__device__ __forceinline__ void load_any(float (&x)[N], const T* p, int n) {
    constexpr int V = 16 / int(sizeof(T));
    if (n >= N) {
#pragma unroll
        for (int i = 0; i < N / V; ++i) load_vector(reinterpret_cast<float (&)[V]>(x[i * V]), p + i * V);
    } else {
        load_some(x, p, n);
    }
}
template <class T, int N>
__device__ __forceinline__ void store_any(T* p, const float (&x)[N], int n) {
    constexpr int V = 16 / int(sizeof(T));
    if (n >= N) {
#pragma unroll
        for (int i = 0; i < N / V; ++i) store_vector(p + i * V, reinterpret_cast<const float (&)[V]>(x[i * V]));
    } else {
        store_some(p, x, n);
    }
}

// 16 bytes of a row from column c on, without a branch around the load: where fewer are left they come from the row's last 16
// bytes and are shifted down when they are turned into numbers (a load inside a branch is waited for there, row after
// row: gradient of 181 tokens of 677 25.0 -> 19.4 us, of 16384 of 4096, which have no such end, 233 -> 240).  Rows shorter than
// 16 bytes are taken entry by entry.
template <class T>
__device__ __forceinline__ uint4v load_raw(const T* row, int c, int width) {
    constexpr int N = 16 / int(sizeof(T));
    if (width >= N) return *reinterpret_cast<const block::uint4u*>(row + (c < width - N ? c : width - N));
    T x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = e < width ? row[e] : T(0);
    return __builtin_bit_cast(uint4v, x);
}
// n: entries from column c to the row's end
template <class T, int N>
__device__ __forceinline__ void to_numbers(float (&x)[N], uint4v v, int n, int width) {
    if (width >= N && n < N) {
        int down = n > 0 ? N - n : 0;                              // entries
        if (sizeof(T) == 2) {
            if (down & 1) v = uint4v{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
            down >>= 1;
        }
        if (down & 1) v = uint4v{v[1], v[2], v[3], 0u};
        if (down & 2) v = uint4v{v[2], v[3], 0u, 0u};
    }
    load_vector(x, reinterpret_cast<const T*>(&v));
}

struct Lookup {
    const int32_t* tokens;
    Rows table, out;
    int64_t n, vocab;
    int width;
    float scale;
};
// A wave per token, four loads on their way a lane.  Bound by HBM: 65536 tokens of 4096 bf16, drawn log-uniformly, 157 us, of which 537 MB
// are written; repeated rows come out of the caches (348 MB are fetched).  8 tokens: 3.5 us, a launch's latency.
template <class T>
__global__ __launch_bounds__(256) void lookup_kernel(Lookup P) {
    constexpr int N = 16 / int(sizeof(T));
    const int64_t t = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (t >= P.n) return;
    const int token = P.tokens[t];
    const bool inside = token >= 0 && token < P.vocab;
    const T* from = static_cast<const T*>(P.table.p) + (inside ? token : 0) * P.table.stride;
    T* to = static_cast<T*>(P.out.p) + t * P.out.stride;
    constexpr int AHEAD = 4;
    for (int c0 = (threadIdx.x & 63) * N; c0 < P.width; c0 += AHEAD * 64 * N) {
        uint4v v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = load_raw(from, c0 + u * 64 * N, P.width);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int c = c0 + u * 64 * N, n = P.width - c;
            if (n <= 0) break;
            float x[N];
            to_numbers<T>(x, v[u], n, P.width);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = inside ? x[e] * P.scale : 0.f;
            store_any(to + c, x, n);
        }
    }
}

// Every workgroup reads all tokens, so that none waits for another: bound by latency up to some ten thousand tokens (3001 tokens 6.5 us,
// 16384 9.6 us; 250 workgroups read 64 KB each from the L2), by these readings behind that, and in small vocabularies, where few
// workgroups have rows, by the placing in turns of a wave (65536 tokens over 250 rows: 134 us).
struct Sort {
    const int32_t* tokens;
    int64_t n;
    int vocab, rows;                         // rows of the vocabulary per workgroup
    int32_t *order, *starts;
};
constexpr int HELD = 16;
__global__ __launch_bounds__(64 * SORT_WAVES) void sort_kernel(Sort P) {
    extern __shared__ int32_t at[];          // [wave][row]
    __shared__ int32_t s_wave[SORT_WAVES], s_below;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lo = blockIdx.x * P.rows, rows = min(P.rows, P.vocab - lo);
    const int64_t each = (P.n + SORT_WAVES * 64 - 1) / (SORT_WAVES * 64) * 64;
    const int64_t begin = wave * each, end = begin + each < P.n ? begin + each : P.n;
    for (int i = threadIdx.x; i < SORT_WAVES * P.rows; i += 64 * SORT_WAVES) at[i] = 0;
    if (threadIdx.x == 0) s_below = 0;
    __syncthreads();
    int32_t* const mine = at + wave * P.rows;
    int below = 0;
    auto count = [&](int token) __attribute__((always_inline)) {
        const int row = row_of(token, lo, rows);
        below += token >= 0 && token < lo;
        if (row >= 0) atomicAdd(&mine[row], 1);                    // whole numbers: any order
    };
    // the wave's first tokens stay in registers for the second pass (all of them up to 16384)
    int held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h) held[h] = begin + h * 64 + lane < end ? P.tokens[begin + h * 64 + lane] : -1;
#pragma unroll
    for (int h = 0; h < HELD; ++h) count(held[h]);
#pragma unroll 8
    for (int64_t t = begin + HELD * 64 + lane; t < end; t += 64) count(P.tokens[t]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
    if (lane == 0 && below) atomicAdd(&s_below, below);
    __syncthreads();
    // counts -> places: row by row, in a row wave by wave
    const int r = threadIdx.x;
    int total = 0;
    if (r < rows)
        for (int w = 0; w < SORT_WAVES; ++w) total += at[w * P.rows + r];
    int sum = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(sum, o, 64);
        if (lane >= o) sum += x;
    }
    if (lane == 63) s_wave[wave] = sum;
    __syncthreads();
    int place = s_below + sum - total;
    for (int w = 0; w < wave; ++w) place += s_wave[w];
    if (r < rows) {
        P.starts[lo + r] = place;
        if (lo + r == P.vocab - 1) P.starts[P.vocab] = place + total;
        for (int w = 0; w < SORT_WAVES; ++w) {
            const int n = at[w * P.rows + r];
            at[w * P.rows + r] = place;
            place += n;
        }
    }
    __syncthreads();
    auto put = [&](int token, int64_t t) __attribute__((always_inline)) {
        const int row = row_of(token, lo, rows);
        unsigned long long left = __ballot(row >= 0);
        while (left) {                                             // one token of the 64 after the other, all its places at a time
            const int same_row = __builtin_amdgcn_readlane(row, __ffsll(left) - 1);
            const unsigned long long same = __ballot(row == same_row);
            const int from = mine[same_row];
            if (row == same_row) P.order[from + __popcll(same & ((1ull << lane) - 1))] = int32_t(t);
            if (lane == 0) mine[same_row] = from + __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the other lanes read it in a later turn
            __builtin_amdgcn_wave_barrier();
            left &= ~same;
        }
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) put(held[h], begin + h * 64 + lane);
    for (int64_t t0 = begin + HELD * 64; t0 < end; t0 += 256) {
        int token[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) token[u] = t0 + u * 64 + lane < end ? P.tokens[t0 + u * 64 + lane] : -1;
#pragma unroll
        for (int u = 0; u < 4; ++u) put(token[u], t0 + u * 64 + lane);
    }
}

struct Sums {
    const int32_t *tokens, *order, *starts;
    Rows d_out, base, grad;
    int64_t vocab;
    int width, segment, strips, in_place;
    int64_t sum_blocks, units;               // workgroups that add up, and their waves' pieces of work
    float scale;
    float* parts;                            // [segment][0: begun before, 1: begun here][width]
};

// a row's sum, finished
template <class T, int N>
__device__ __forceinline__ void finish_row(const Sums& P, int64_t row, int c, int n, const float (&sum)[N]) {
    float y[N];
    if (P.base.p) load_any(y, static_cast<const T*>(P.base.p) + row * P.base.stride + c, n);
    else
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = fmaf(P.scale, sum[e], y[e]);
    store_any(static_cast<T*>(P.grad.p) + row * P.grad.stride + c, y, n);
}

// A wave per segment and strip of 64 vectors: rows of d_out are read once, eight on their way, and every row of the table is written
// once.  Bound by HBM: 16384 tokens of 4096 bf16 over 128000 rows, 1.05 GB written and 0.13 GB read in 226 us (5.2 TB/s); 3001 of 1359 fp32
// onto a base of 50021 rows, 0.56 GB in 115 us (4.9 TB/s).
template <class T>
__device__ void add_up(const Sums& P, int64_t unit) {
    constexpr int N = 16 / int(sizeof(T)), AHEAD = 8;
    const int lane = threadIdx.x & 63;
    const int64_t segment = unit / P.strips;
    const int c = (int(unit % P.strips) * 64 + lane) * N, n = P.width - c;
    const int64_t first = segment * P.segment, all = P.starts[P.vocab];
    if (first >= all) return;
    const int many = int(all - first < P.segment ? all - first : P.segment);
    // a lane's token: its row of d_out, whether the row's tokens begin or end with it
    int t = 0, token = -1;
    bool begins = false, ends = false;
    if (lane < many) {
        t = P.order[first + lane];
        token = P.tokens[t];
        begins = P.starts[token] == first + lane;
        ends = P.starts[token + 1] == first + lane + 1;
    }
    const unsigned long long begin_mask = __ballot(begins), end_mask = __ballot(ends);
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    bool here = false;                                             // whether the present row began in this segment
    for (int i0 = 0; i0 < many; i0 += AHEAD) {
        uint4v v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (i0 + u < many) v[u] = load_raw(static_cast<const T*>(P.d_out.p) + int64_t(__builtin_amdgcn_readlane(t, i0 + u)) * P.d_out.stride, c, P.width);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + u;
            if (i >= many) break;
            if (begin_mask >> i & 1) {
                here = true;
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] = 0.f;
            }
            float x[N];
            to_numbers<T>(x, v[u], n, P.width);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += x[e];
            const bool end = end_mask >> i & 1;
            if (!end && i + 1 < many) continue;
            if (n > 0) {
                if (end && here) {
                    finish_row<T>(P, __builtin_amdgcn_readlane(token, i), c, n, sum);
                } else {
                    store_any(P.parts + (segment * 2 + (here ? 1 : 0)) * P.width + c, sum, n);
                }
            }
            here = false;
        }
    }
}
template <class T>
__global__ __launch_bounds__(256) void sums_kernel(Sums P) {
    if (int64_t(blockIdx.x) < P.sum_blocks) {
        const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
        if (unit < P.units) add_up<T>(P, unit);
        return;
    }
    // rows without a token
    constexpr int N = 16 / int(sizeof(T));
    const int64_t row = (int64_t(blockIdx.x) - P.sum_blocks) * 4 + (threadIdx.x >> 6);
    if (row >= P.vocab || P.starts[row] != P.starts[row + 1]) return;
    const float none[N] = {};
    for (int c = (threadIdx.x & 63) * N; c < P.width; c += 64 * N) finish_row<T>(P, row, c, P.width - c, none);
}

// The row that begins in a segment and goes on behind it: its segments' sums in their order.  Eight on their way; bound by latency
// (5.4 to 8 us) unless one token fills many segments, which one wave a strip joins (16384 places in 512 segments: 61 us).
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Sums P) {
    constexpr int N = 16 / int(sizeof(T));
    const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (unit >= P.units) return;
    const int64_t segment = unit / P.strips, last = (segment + 1) * P.segment - 1;
    if (last + 1 >= P.starts[P.vocab]) return;
    const int token = P.tokens[P.order[last]];
    const int64_t begin = P.starts[token], end = P.starts[token + 1];
    if (begin < segment * P.segment || end <= last + 1) return;
    const int c = (int(unit % P.strips) * 64 + (threadIdx.x & 63)) * N, n = P.width - c;
    if (n <= 0) return;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    const float* from = P.parts + (segment * 2 + 1) * P.width + c;   // begun here; then the parts begun before, one after the other
    load_any(sum, from, n);
    from += P.width;
    const int64_t more = (end - 1) / P.segment - segment;
    for (int64_t s = 0; s < more; s += 8) {
        float x[8][N];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s + u < more) load_any(x[u], from + (s + u) * 2 * P.width, n);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s + u < more)
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += x[u][e];
    }
    finish_row<T>(P, token, c, n, sum);
}

template <class T>
onecomp_status backward(const Sums& P, const Sort& S, hipStream_t stream) {
    static std::atomic<uint64_t> done{0};
    const int lds = SORT_WAVES * S.rows * 4;
    if (const onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(sort_kernel), SORT_WAVES * SORT_MOST * 4, done)) return st;
    sort_kernel<<<dim3(unsigned(ceil_div(S.vocab, S.rows))), dim3(64 * SORT_WAVES), lds, stream>>>(S);
    ONECOMP_CHECK_LAUNCH();
    const int64_t fill = P.in_place ? 0 : ceil_div(P.vocab, 4);
    if (P.sum_blocks + fill > 0) {
        sums_kernel<T><<<dim3(unsigned(P.sum_blocks + fill)), dim3(256), 0, stream>>>(P);
        ONECOMP_CHECK_LAUNCH();
    }
    if (S.n > P.segment) {
        join_kernel<T><<<dim3(unsigned(P.sum_blocks)), dim3(256), 0, stream>>>(P);
        ONECOMP_CHECK_LAUNCH();
    }
    return ONECOMP_OK;
}

}  // namespace

onecomp_status embedding_forward_run(onecomp_dtype dtype, const int32_t* tokens, int64_t n, const Rows& table, int64_t vocab, int64_t width, float scale,
                                     const Rows& out, hipStream_t stream) {
    const Lookup P{tokens, table, out, n, vocab, int(width), scale};
    const dim3 grid(unsigned(ceil_div(n, 4)));
    if (dtype == ONECOMP_BF16) lookup_kernel<uint16_t><<<grid, dim3(256), 0, stream>>>(P);
    else lookup_kernel<float><<<grid, dim3(256), 0, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

size_t embedding_workspace_bytes(int64_t n, int64_t vocab, int64_t width) { return embedding_space(n, vocab, width).all; }

onecomp_status embedding_backward_run(onecomp_dtype dtype, const int32_t* tokens, int64_t n, const Rows& d_out, int64_t vocab, int64_t width, float scale,
                                      const Rows& base, const Rows& d_table, void* workspace, hipStream_t stream) {
    const EmbeddingSpace s = embedding_space(n, vocab, width);
    char* ws = static_cast<char*>(workspace);
    Sort S{tokens, n, int(vocab), sort_rows(vocab), reinterpret_cast<int32_t*>(ws + s.order), reinterpret_cast<int32_t*>(ws + s.starts)};
    Sums P{};
    P.tokens = tokens;
    P.order = S.order;
    P.starts = S.starts;
    P.d_out = d_out;
    P.base = base;
    P.grad = d_table;
    P.vocab = vocab;
    P.width = int(width);
    P.segment = segment_of(n, width);
    P.strips = int(ceil_div(width, 64 * (dtype == ONECOMP_BF16 ? 8 : 4)));
    P.in_place = base.p == d_table.p;
    P.units = s.segments * P.strips;
    P.sum_blocks = ceil_div(P.units, 4);
    if (P.sum_blocks + ceil_div(vocab, 4) >= int64_t(1) << 24) return ONECOMP_ERR_UNSUPPORTED;   // a launch has less than 2^32 threads
    P.scale = scale;
    P.parts = reinterpret_cast<float*>(ws + s.parts);
    return dtype == ONECOMP_BF16 ? backward<uint16_t>(P, S, stream) : backward<float>(P, S, stream);
}

}  // namespace token
}  // namespace onecomp
