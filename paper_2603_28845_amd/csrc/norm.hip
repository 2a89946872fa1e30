// The norms around a block, fused with its gate and residual: h' = r h + g u, n = norm(h'), u = y or norm(y), and their
// gradients.  Every tensor is read once and written once; rows stay in registers between the sums that a norm needs.
#include "block.hpp"
#include "block_plan.hpp"
#include <type_traits>

namespace onecomp {
namespace block {
namespace {

// G threads have a row: thread t of them the values VEC (t + G v) .. + VEC - 1, v < NV; 16 bytes of T each.  WHOLE: addresses,
// strides and widths of whole vectors.  Those rows, and all rows of fp32, are read and written through buffer descriptors as
// long as the row, whose bounds check, dword by dword, does what comparisons and branches around every access would.  An odd
// row of bf16 can end inside a dword: its last vector is read from where a whole one ends with the row and shifted into place
// (SHIFT), unless a thread has more than one (widths over 8192), which leaves no registers for it: entry by entry then, which
// waits for these and all loads before them.  Gradients of 32 M entries, rms, entry by entry and so: bf16 1001 wide 267 and
// 193 us, 4095 wide 257 and 170; fp32 1359 wide 379 and 249.
template <class T_, int NV, int G, bool WHOLE>
struct Part {
    typedef T_ T;
    static constexpr int VEC = 16 / int(sizeof(T)), E = VEC * NV;
    static constexpr bool RANGES = WHOLE || sizeof(T) == 4, SHIFT = !RANGES && NV == 1;
    static __device__ __forceinline__ int col(int t, int v) { return VEC * (t + G * v); }
    static __device__ __forceinline__ bool inside(int t, int e, int width) { return col(t, e / VEC) + (WHOLE ? 0 : e % VEC) < width; }
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const void* p, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
    }

    // A row on its way: loads whose values nobody has asked for yet.  Zeros behind the width.
    struct Raw {
        uint4v v[NV];
    };
    static __device__ __forceinline__ void fetch(Raw& x, const Rows& r, int64_t row, int width, int t, bool there) {
        const T* p = static_cast<const T*>(r.p) + row * r.stride;
        if constexpr (RANGES) {
            const __amdgpu_buffer_rsrc_t d = descriptor(p, there ? width * int(sizeof(T)) : 0);
#pragma unroll
            for (int v = 0; v < NV; ++v) x.v[v] = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(d, col(t, v) * int(sizeof(T)), 0, 0));
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = col(t, v);
                uint4v y = {0u, 0u, 0u, 0u};
                if (SHIFT ? width >= VEC : there && c + VEC <= width) {
                    if (there && c < width) y = *reinterpret_cast<const uint4u*>(p + (SHIFT ? min(c, width - VEC) : c));
                } else if (there && c < width) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (c + i < width) y[i / 2] |= uint32_t(reinterpret_cast<const uint16_t*>(p)[c + i]) << (16 * (i & 1));
                }
                x.v[v] = y;
            }
        }
    }
    // bf16 entries `by` .. 7 to the front, zeros behind them
    static __device__ __forceinline__ void shift(uint4v& x, int by) {
        const uint64_t lo = uint64_t(x[1]) << 32 | x[0], hi = uint64_t(x[3]) << 32 | x[2];
        const int bits = 16 * by;
        const uint64_t a = bits >= 64 ? hi >> (bits - 64) : bits ? lo >> bits | hi << (64 - bits) : lo, b = bits >= 64 ? 0 : hi >> bits;
        x = uint4v{uint32_t(a), uint32_t(a >> 32), uint32_t(b), uint32_t(b >> 32)};
    }
    static __device__ __forceinline__ void values(float (&x)[E], Raw r, int width, int t) {
        if constexpr (SHIFT) {
            const int c = col(t, 0), by = c < width && width >= VEC ? max(0, c + VEC - width) : 0;
            if (__any(by)) shift(r.v[0], by);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (sizeof(T) == 2) {
                    x[v * VEC + 2 * i] = bf16_value(r.v[v][i] & 0xffffu);
                    x[v * VEC + (2 * i + 1) % VEC] = __uint_as_float(r.v[v][i] & 0xffff0000u);
                } else {
                    x[v * VEC + i] = __uint_as_float(r.v[v][i]);
                }
            }
    }
    static __device__ __forceinline__ void load(float (&x)[E], const Rows& r, int64_t row, int width, int t, bool there) {
        Raw raw;
        fetch(raw, r, row, width, t, there);
        values(x, raw, width, t);
    }
    static __device__ __forceinline__ void store(const Rows& r, int64_t row, int width, int t, bool there, const float (&x)[E]) {
        T* p = static_cast<T*>(r.p) + row * r.stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col(t, v);
            float y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) y[i] = x[v * VEC + i];
            if constexpr (RANGES) {
                __builtin_amdgcn_raw_buffer_store_b128(packed(y), descriptor(p, there ? width * int(sizeof(T)) : 0), c * int(sizeof(T)), 0, 0);
            } else if (there && c + VEC <= width) {
                store_vector(p + c, y);
            } else if (there && c < width) {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (c + i < width) store_one(p + c + i, y[i]);
            }
        }
    }
    // this thread's entries of a parameter, in either type
    static __device__ __forceinline__ void parameter(float (&x)[E], const void* p, bool bf16, int width, int t) {
        if constexpr (WHOLE) {
            const __amdgpu_buffer_rsrc_t d = descriptor(p, width * (bf16 ? 2 : 4));
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = col(t, v);
                if (bf16) {
                    uint4v y = {0u, 0u, 0u, 0u};
                    if (VEC == 8) {
                        y = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(d, c * 2, 0, 0));
                    } else {
                        const auto z = __builtin_amdgcn_raw_buffer_load_b64(d, c * 2, 0, 0);
                        y[0] = z[0];
                        y[1] = z[1];
                    }
#pragma unroll
                    for (int i = 0; i < VEC / 2; ++i) {
                        x[v * VEC + 2 * i] = bf16_value(y[i] & 0xffffu);
                        x[v * VEC + 2 * i + 1] = __uint_as_float(y[i] & 0xffff0000u);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < VEC / 4; ++j) {
                        const uint4v y = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(d, c * 4 + 16 * j, 0, 0));
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[v * VEC + 4 * j + i] = __uint_as_float(y[i]);
                    }
                }
            }
        } else if (bf16) {
            parameter(x, static_cast<const uint16_t*>(p), width, t);
        } else {
            parameter(x, static_cast<const float*>(p), width, t);
        }
    }
    template <class W>
    static __device__ __forceinline__ void parameter(float (&x)[E], const W* p, int width, int t) {
        constexpr int N = 16 / int(sizeof(W)) < VEC ? 16 / int(sizeof(W)) : VEC;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col(t, v);
#pragma unroll
            for (int j = 0; j < VEC; j += N) {
                if (N == 16 / int(sizeof(W)) && c + j + N <= width) {
                    float y[16 / sizeof(W)];
                    load_vector(y, p + c + j);
#pragma unroll
                    for (int i = 0; i < N; ++i) x[v * VEC + j + i] = y[i];
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) x[v * VEC + j + i] = c + j + i < width ? load_one(p + c + j + i) : 0.f;
                }
            }
        }
    }
    static __device__ __forceinline__ auto packed(const float (&y)[VEC]) {
        uint4v r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(T) == 2)
                r[i] = uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(y[2 * i]))) |
                       uint32_t(__builtin_bit_cast(uint16_t, static_cast<__bf16>(y[(2 * i + 1) % VEC]))) << 16;
            else
                r[i] = __float_as_uint(y[i % VEC]);
        }
        return r;
    }
};

// Sum over the lanes up to each: the last lane has the whole wave's.  In the vector pipe; shuffles would take a trip through
// LDS for each of the six steps.
__device__ __forceinline__ float lane_sum(float x) {
    auto moved = [](float v, auto ctrl, auto rows) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
    };
    using std::integral_constant;
    x += moved(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    x += moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
    x += moved(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
    return x;
}

// Sums of K numbers (up to 4) over the G threads of each group of a workgroup.  `slot` alternates between two places in LDS, so
// that one barrier a sum is enough.  Every thread of the workgroup takes part.
template <int K, int G, int THREADS>
__device__ __forceinline__ void group_sum(float (&x)[K], float4v* lds, int& slot) {
    float4v all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) all[k] = lane_sum(x[k]);
    if (G == 64) {
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(all[k]), 63));
        return;
    }
    constexpr int WAVES = THREADS / 64, EACH = G / 64;
    float4v* to = lds + slot * WAVES;
    slot ^= 1;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) to[wave] = all;
    __syncthreads();
    const float4v* from = to + wave / EACH * EACH;
    all = from[0];
#pragma unroll
    for (int w = 1; w < EACH; ++w) all += from[w];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = all[k];
}

// x to (x - mean) / size in place: size^2 = mean of squares + eps; the mean for layer norms only
template <class Pt, int G, int THREADS>
__device__ __forceinline__ float normalise(float (&x)[Pt::E], bool layer, int width, float eps, int t, float4v* lds, int& slot) {
    const float inv_width = 1.f / float(width);
    if (layer) {
        float s[1] = {0.f};
#pragma unroll
        for (int e = 0; e < Pt::E; ++e) s[0] += x[e];
        group_sum<1, G, THREADS>(s, lds, slot);
        const float mean = s[0] * inv_width;
#pragma unroll
        for (int e = 0; e < Pt::E; ++e) x[e] = Pt::inside(t, e, width) ? x[e] - mean : 0.f;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int e = 0; e < Pt::E; ++e) s[0] = fmaf(x[e], x[e], s[0]);
    group_sum<1, G, THREADS>(s, lds, slot);
    const float inv = 1.f / sqrtf(fmaf(s[0], inv_width, eps));
#pragma unroll
    for (int e = 0; e < Pt::E; ++e) x[e] *= inv;
    return inv;
}

// x = x w + b
template <class Pt>
__device__ __forceinline__ void affine(float (&x)[Pt::E], const void* w, const void* b, bool w_bf16, int width, int t) {
    float p[Pt::E];
    if (w) {
        Pt::parameter(p, w, w_bf16, width, t);
#pragma unroll
        for (int e = 0; e < Pt::E; ++e) x[e] *= p[e];
    }
    if (b) {
        Pt::parameter(p, b, w_bf16, width, t);
#pragma unroll
        for (int e = 0; e < Pt::E; ++e) x[e] += p[e];
    }
}

// One row for each group of G threads, held in registers from its loads to its stores: the bytes are the bound.  65536 x 4096
// bf16 with y: 342 to 364 us, 5.9 TB/s (a copy of 2 GiB: 4.9); 8 rows: 3.3 us.
template <class T, int NV, int G, bool WHOLE>
__global__ __launch_bounds__(G < 256 ? 256 : G) void forward_kernel(const Params P) {
    constexpr int THREADS = G < 256 ? 256 : G;
    typedef Part<T, NV, G, WHOLE> Pt;
    __shared__ float4v lds[2 * (THREADS / 64)];
    int slot = 0;
    const int t = threadIdx.x % G;
    const int64_t row = int64_t(blockIdx.x) * (THREADS / G) + __builtin_amdgcn_readfirstlane(threadIdx.x / G);   // the same in a whole wave
    const bool there = row < P.rows;
    const int width = P.width;
    float x[Pt::E];
    if (P.y.p) {
        float u[Pt::E];
        Pt::load(u, P.y, row, width, t, there);
        Pt::load(x, P.h, row, width, t, there);
        if (P.post) {
            normalise<Pt, G, THREADS>(u, P.layer, width, P.eps, t, lds, slot);
            affine<Pt>(u, P.post_weight, P.post_bias, P.w_bf16, width, t);
        }
        if (P.gate.p) {
            float g[Pt::E];
            if (P.gate_rows) Pt::load(g, P.gate, row, width, t, there);
            else Pt::parameter(g, P.gate.p, P.w_bf16, width, t);
#pragma unroll
            for (int e = 0; e < Pt::E; ++e) u[e] *= g[e];
        }
#pragma unroll
        for (int e = 0; e < Pt::E; ++e) x[e] = fmaf(P.scale, x[e], u[e]);
        if (P.h_out.p) Pt::store(P.h_out, row, width, t, there, x);
    } else {
        Pt::load(x, P.h, row, width, t, there);
    }
    if (!P.n.p) return;
    normalise<Pt, G, THREADS>(x, P.layer, width, P.eps, t, lds, slot);
    affine<Pt>(x, P.weight, P.bias, P.w_bf16, width, t);
    Pt::store(P.n, row, width, t, there, x);
}

// Subtracts the mean of x, and of y too if it goes through a norm, from their entries.
template <class Pt, int G, int THREADS>
__device__ __forceinline__ void centre(float (&x)[Pt::E], float (&y)[Pt::E], bool both, float& mx, float& my, int width, int t, float4v* lds, int& slot) {
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < Pt::E; ++e) {
        s[0] += x[e];
        s[1] += y[e];
    }
    group_sum<2, G, THREADS>(s, lds, slot);
    mx = s[0] / float(width);
    my = both ? s[1] / float(width) : 0.f;
#pragma unroll
    for (int e = 0; e < Pt::E; ++e) {
        const bool in = Pt::inside(t, e, width);
        x[e] = in ? x[e] - mx : 0.f;
        y[e] = in ? y[e] - my : 0.f;
    }
}

// A workgroup takes rows in turn (as many at a time as it has groups of G threads) and keeps the parameters' gradients, sums
// over rows, in registers until its last row; then its groups' sums meet in LDS and go to scratch, one row per workgroup.
// With x^ = x inv the normalised row, the gradient of the rows in front of a norm is inv (d - x^ mean(d x^) - mean(d)), the
// last for layer norms only.  Both norms' squares and the first norm's means are added up in one go (mean(d x^) =
// inv mean(d x)), the second norm's means in another; layer norms take one more for the means of the rows.  16384 x 4096 bf16,
// rms on both sides, gate per channel: 187 to 203 us, 3.9 to 4.2 TB/s; registers allow 16 waves on a CU, and their loads in flight and
// 55 % of the vector pipes are the bound (512 threads a workgroup, two on a CU: 183 to 200 us, but twice the sums to join).
//
// SUMS: as said.  Wider rows leave no registers for the parameters' sums (over 8192, layer norms over 4096; spilled to memory
// they cost 4 to 8 times the rest): then only what a row's entries need is left in scratch, for strips_kernel, which adds up; not
// even that where no parameter's gradient is wanted.
//
// Registers: 128 a thread at 1024 threads a workgroup.  Spilled, rms / layer norms, whole vectors: bf16 up to 4096 wide 0 / 20, 8192
// 0 / 0, 16384 0 / 14, 32768 81 / 117; fp32 up to 4096 wide 0 / 3, 8192 0 / 0, 16384 0 / 49, 32768 112 / 170; odd rows up to 34 at
// 4096 and 480 at 32768.  The kernel's share of a wide call: 5461 x 12288 fp32 layer norms 550 us of 775, 4681 x 14336 bf16 rms
// 189 of 295.
template <class T, int NV, int G, bool WHOLE, bool LAYER, bool SUMS>
__global__ __launch_bounds__(1024) void gradient_kernel(const Params P) {
    constexpr int THREADS = 1024, GROUPS = THREADS / G;
    typedef Part<T, NV, G, WHOLE> Pt;
    constexpr int E = Pt::E;
    __shared__ float4v lds[2 * (THREADS / 64)];
    __shared__ float meet[GROUPS > 1 && SUMS ? THREADS * E : 1];
    int slot = 0;
    const int t = threadIdx.x % G, group = __builtin_amdgcn_readfirstlane(threadIdx.x / G);   // the same in a whole wave
    const int width = P.width;
    const float inv_width = 1.f / float(width);
    float sums[5][E];     // weight, bias, post_weight, post_bias, gate
#pragma unroll
    for (int i = 0; i < 5; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[i][e] = 0.f;
    // the next rows are on their way while these are worked on, where registers allow
    constexpr bool AHEAD = NV == 1;
    typename Pt::Raw raw[4];
    auto fetch = [&](int64_t row) {
        Pt::fetch(raw[0], P.h, row, width, t, row < P.rows && P.dn.p);
        Pt::fetch(raw[1], P.dn, row, width, t, row < P.rows && P.dn.p);
        Pt::fetch(raw[2], P.dh_out, row, width, t, row < P.rows && P.dh_out.p);
        Pt::fetch(raw[3], P.y, row, width, t, row < P.rows && P.y.p);
    };
    if (AHEAD) fetch(int64_t(blockIdx.x) * GROUPS + group);
    for (int64_t first = int64_t(blockIdx.x) * GROUPS; first < P.rows; first += int64_t(gridDim.x) * GROUPS) {
        const int64_t row = first + group;
        const bool there = row < P.rows;
        float x[E], y[E], dn[E], d[E];                            // h', the block's output, gradients of n and of h'
        if (!AHEAD) fetch(row);
        Pt::values(x, raw[0], width, t);
        Pt::values(dn, raw[1], width, t);
        Pt::values(d, raw[2], width, t);
        Pt::values(y, raw[3], width, t);
        typename Pt::Raw raw_gate;
        if (P.gate_rows) Pt::fetch(raw_gate, P.gate, row, width, t, there);
        if (AHEAD) fetch(row + int64_t(gridDim.x) * GROUPS);
        // parameters are read where they are used: read early they would push the sums out of the registers
        __builtin_amdgcn_sched_barrier(0);
        float mean_h = 0.f, mean_y = 0.f;
        if (LAYER) {
            centre<Pt, G, THREADS>(x, y, P.post, mean_h, mean_y, width, t, lds, slot);
        }
        float s[4] = {0.f, 0.f, 0.f, 0.f}, w[E];                  // x^2, dn w x, dn w, y^2
        if (P.weight) {
            Pt::parameter(w, P.weight, P.w_bf16, width, t);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = 1.f;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s[0] = fmaf(x[e], x[e], s[0]);
            s[1] = fmaf(dn[e] * w[e], x[e], s[1]);
            if (LAYER) s[2] = fmaf(dn[e], w[e], s[2]);
            s[3] = fmaf(y[e], y[e], s[3]);
        }
        group_sum<4, G, THREADS>(s, lds, slot);
        // a group behind the last row holds zeros, whose size is 0 without an eps: 0 times infinity would reach the parameters' sums
        const float inv_y = there ? 1.f / sqrtf(fmaf(s[3], inv_width, P.eps)) : 0.f;
        const float inv = there ? 1.f / sqrtf(fmaf(s[0], inv_width, P.eps)) : 0.f, along = s[1] * inv * inv_width, mean = LAYER ? s[2] * inv_width : 0.f;
        if (!SUMS && P.row_numbers && there && t == 0) reinterpret_cast<RowNumbers*>(P.row_numbers)[row] = RowNumbers{mean_h, inv, mean, along, mean_y, inv_y, {0.f, 0.f}};
        if (P.dn.p) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float hat = x[e] * inv;
                if (SUMS) sums[0][e] = fmaf(dn[e], hat, sums[0][e]);
                if (SUMS && LAYER) sums[1][e] += dn[e];
                d[e] += inv * (dn[e] * w[e] - mean - hat * along);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (P.dh.p) {
            float dh[E];
#pragma unroll
            for (int e = 0; e < E; ++e) dh[e] = P.scale * d[e];
            Pt::store(P.dh, row, width, t, there, dh);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!P.y.p) continue;
        if (P.post) {
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] *= inv_y;
        }
        if (P.gate.p) {
            float u[E], g[E];
#pragma unroll
            for (int e = 0; e < E; ++e) u[e] = y[e];
            if (P.post) affine<Pt>(u, P.post_weight, P.post_bias, P.w_bf16, width, t);
#pragma unroll
            for (int e = 0; e < E; ++e) u[e] *= d[e];
            if (P.gate_rows) {
                Pt::values(g, raw_gate, width, t);
                if (P.dgate.p) Pt::store(P.dgate, row, width, t, there, u);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (SUMS) sums[4][e] += there ? u[e] : 0.f;
                Pt::parameter(g, P.gate.p, P.w_bf16, width, t);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] *= g[e];
        }
        __builtin_amdgcn_sched_barrier(0);
        if (P.post) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (SUMS) sums[2][e] = fmaf(d[e], y[e], sums[2][e]);
                if (SUMS && LAYER) sums[3][e] += there ? d[e] : 0.f;
            }
            if (P.post_weight) affine<Pt>(d, P.post_weight, nullptr, P.w_bf16, width, t);
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                m[0] = fmaf(d[e], y[e], m[0]);
                if (LAYER) m[1] += Pt::inside(t, e, width) ? d[e] : 0.f;
            }
            group_sum<2, G, THREADS>(m, lds, slot);
            const float along = m[0] * inv_width, mean = m[1] * inv_width;
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = inv_y * (d[e] - mean - y[e] * along);
        }
        if (P.dy.p) Pt::store(P.dy, row, width, t, there, d);
    }
    if (!SUMS) return;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        if (!(P.wanted >> i & 1)) continue;
        float* to = P.part + (int64_t(__popc(P.wanted & ((1 << i) - 1))) * gridDim.x + blockIdx.x) * width;
        if (GROUPS == 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int c = Pt::col(t, e / Pt::VEC) + e % Pt::VEC;
                if (c < width) to[c] = sums[i][e];
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) meet[(group * E + e) * G + t] = sums[i][e];
            __syncthreads();
            for (int at = threadIdx.x; at < E * G; at += THREADS) {
                float s = 0.f;
                for (int g = 0; g < GROUPS; ++g) s += meet[g * E * G + at];
                const int e = at / G, c = Pt::col(at % G, e / Pt::VEC) + e % Pt::VEC;
                if (c < width) to[c] = s;
            }
        }
    }
}

// The parameters' gradients of wide rows: a wave has a strip of 64 vectors and goes down every fourth row of its workgroup's
// run of rows; what the rows' sums were is in scratch.  Everything is read once more (10 passes over the tensors' bytes instead
// of 6), in return for sums that stay in registers at any width.
template <class T, bool WHOLE, bool LAYER>
__global__ __launch_bounds__(256) void strips_kernel(const Params P, const int runs) {
    typedef Part<T, 1, 64, WHOLE> Pt;
    constexpr int E = Pt::E, STRIP = 64 * E;
    __shared__ float meet[4][STRIP];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // this strip of every tensor and parameter, as if it were the whole
    const int first_col = blockIdx.x * STRIP, width = min(P.width - first_col, STRIP);
    auto strip = [&](const Rows& r) { return Rows{r.p ? static_cast<T*>(r.p) + first_col : nullptr, r.stride}; };
    auto strip_of = [&](const void* p) { return p ? static_cast<const char*>(p) + first_col * (P.w_bf16 ? 2 : 4) : nullptr; };
    const Rows h = strip(P.h), y = strip(P.y), dn = strip(P.dn), dh_out = strip(P.dh_out), gate = P.gate_rows ? strip(P.gate) : P.gate;
    float w[E], pw[E], pb[E], g[E];
    auto parameter = [&](float (&x)[E], const void* p, float otherwise) {
        if (p) {
            Pt::parameter(x, strip_of(p), P.w_bf16, width, lane);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = otherwise;
        }
    };
    parameter(w, P.weight, 1.f);
    parameter(pw, P.post_weight, 1.f);
    parameter(pb, P.post_bias, 0.f);
    parameter(g, P.gate_rows ? nullptr : P.gate.p, 1.f);
    float sums[5][E];
#pragma unroll
    for (int i = 0; i < 5; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) sums[i][e] = 0.f;
    const int64_t begin = P.rows * blockIdx.y / runs, end = P.rows * (blockIdx.y + 1) / runs;
    typename Pt::Raw raw[4];
    auto fetch = [&](int64_t row) {
        Pt::fetch(raw[0], h, row, width, lane, row < end && P.dn.p);
        Pt::fetch(raw[1], dn, row, width, lane, row < end && P.dn.p);
        Pt::fetch(raw[2], dh_out, row, width, lane, row < end && P.dh_out.p);
        Pt::fetch(raw[3], y, row, width, lane, row < end && P.y.p);
    };
    fetch(begin + wave);
    for (int64_t row = begin + wave; row < end; row += 4) {
        float x[E], d[E], dx[E], u[E];
        Pt::values(x, raw[0], width, lane);
        Pt::values(dx, raw[1], width, lane);
        Pt::values(d, raw[2], width, lane);
        Pt::values(u, raw[3], width, lane);
        const RowNumbers n = reinterpret_cast<const RowNumbers*>(P.row_numbers)[row];
        if (P.gate_rows) Pt::load(g, gate, row, width, lane, true);
        fetch(row + 4);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float hat = (x[e] - n.mean_h) * n.inv_h;
            sums[0][e] = fmaf(dx[e], hat, sums[0][e]);
            if (LAYER) sums[1][e] += dx[e];
            const float total = P.dn.p ? d[e] + n.inv_h * (dx[e] * w[e] - n.mean_d - hat * n.along) : d[e];
            const float yhat = P.post ? (u[e] - n.mean_y) * n.inv_y : u[e];
            if (P.wanted & 16) sums[4][e] = fmaf(total, fmaf(yhat, pw[e], pb[e]), sums[4][e]);
            const float du = total * g[e];
            sums[2][e] = fmaf(du, yhat, sums[2][e]);
            if (LAYER) sums[3][e] += du;
        }
    }
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        if (!(P.wanted >> i & 1)) continue;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) meet[wave][lane * E + e] = sums[i][e];
        __syncthreads();
        float* to = P.part + (int64_t(__popc(P.wanted & ((1 << i) - 1))) * runs + blockIdx.y) * P.width + first_col;
        for (int c = threadIdx.x; c < width; c += 256) to[c] = (meet[0][c] + meet[1][c]) + (meet[2][c] + meet[3][c]);
    }
}

// Sums over the workgroups of the kernels above: 64 columns of one parameter per workgroup, 16 waves with every sixteenth row.
__global__ __launch_bounds__(1024) void columns_kernel(const Params P, const int n_parts) {
    __shared__ float meet[16][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane;
    const float* from = P.part + int64_t(blockIdx.y) * n_parts * P.width;
    float s = 0.f;
    if (c < P.width)
        for (int r = wave; r < n_parts; r += 16) s += from[int64_t(r) * P.width + c];
    meet[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= P.width) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += meet[w][lane];
    int which = 0;
    for (int left = int(blockIdx.y); which < 5; ++which)
        if ((P.wanted >> which & 1) && left-- == 0) break;
    if (P.w_bf16) static_cast<__bf16*>(P.d_param[which])[c] = static_cast<__bf16>(s);
    else static_cast<float*>(P.d_param[which])[c] = s;
}

int gradient_workgroups(int64_t rows, int groups) {
    const int cus = device_cus();
    const int64_t all = ceil_div(rows, groups);
    const int64_t most = cus > 0 ? cus : 256;
    return int(all < 1 ? 1 : all < most ? all : most);            // one even without rows: the sums are 0
}

// runs of rows of the strips: four workgroups for each CU at 256 entries a strip
int strip_runs(int64_t rows, int width) {
    const int64_t runs = 1024 / ((width + 511) / 512), most = ceil_div(rows, 8);
    return int(most < 1 ? 1 : runs < most ? runs : most);
}

template <class T, int NV, int G, bool WHOLE>
onecomp_status launch_whole(const Params& P, bool gradient, hipStream_t stream) {
    if (!gradient) {
        constexpr int THREADS = G < 256 ? 256 : G;
        const int64_t grid = ceil_div(P.rows, THREADS / G);
        if (grid > 0x7fffffff) return ONECOMP_ERR_UNSUPPORTED;
        forward_kernel<T, NV, G, WHOLE><<<dim3(unsigned(grid)), dim3(THREADS), 0, stream>>>(P);
        ONECOMP_CHECK_LAUNCH();
        return ONECOMP_OK;
    }
    int parts = gradient_workgroups(P.rows, 1024 / G);
    constexpr int V = 16 / int(sizeof(T));
    auto go = [&](auto layer) -> onecomp_status {
        constexpr bool LAYER = decltype(layer)::value, SUMS = own_sums(V * NV * G, LAYER);
        const int grid = parts;
        // strips read the gradients anew: where the results go over them, the rows' numbers are formed in a pass of their own
        const bool over = !SUMS && P.wanted && over_inputs({P.dh.p, P.dy.p, P.dgate.p}, {P.h.p, P.y.p, P.dn.p, P.dh_out.p, P.gate_rows ? P.gate.p : nullptr});
        Params Q = P;
        if (over) Q.dh.p = Q.dy.p = Q.dgate.p = nullptr;
        gradient_kernel<T, NV, G, WHOLE, LAYER, SUMS><<<dim3(unsigned(grid)), dim3(1024), 0, stream>>>(Q);
        ONECOMP_CHECK_LAUNCH();
        if constexpr (!SUMS) {
            if (P.wanted) {
                const int strips = (P.width + 64 * V - 1) / (64 * V);
                parts = strip_runs(P.rows, P.width);
                strips_kernel<T, WHOLE, LAYER><<<dim3(unsigned(strips), unsigned(parts)), dim3(256), 0, stream>>>(P, parts);
                ONECOMP_CHECK_LAUNCH();
            }
            if (over) {
                gradient_kernel<T, NV, G, WHOLE, LAYER, SUMS><<<dim3(unsigned(grid)), dim3(1024), 0, stream>>>(P);
                ONECOMP_CHECK_LAUNCH();
            }
        }
        return ONECOMP_OK;
    };
    if (const onecomp_status st = P.layer ? go(std::true_type{}) : go(std::false_type{})) return st;
    if (const int n = __builtin_popcount(P.wanted)) {
        columns_kernel<<<dim3(unsigned((P.width + 63) / 64), unsigned(n)), dim3(1024), 0, stream>>>(P, parts);
        ONECOMP_CHECK_LAUNCH();
    }
    return ONECOMP_OK;
}

// widths, addresses and strides of whole vectors
template <class T>
bool whole_vectors(const Params& P) {
    constexpr int V = 16 / int(sizeof(T));
    uintptr_t rest = uintptr_t(P.width % V);
    for (const Rows* r : {&P.h, &P.y, &P.h_out, &P.n, &P.dn, &P.dh_out, &P.dh, &P.dy, &P.dgate})
        if (r->p) rest |= reinterpret_cast<uintptr_t>(r->p) % 16 | uintptr_t(r->stride % V);
    if (P.gate.p) rest |= reinterpret_cast<uintptr_t>(P.gate.p) % 16 | (P.gate_rows ? uintptr_t(P.gate.stride % V) : 0);
    for (const void* p : {P.weight, P.bias, P.post_weight, P.post_bias}) rest |= reinterpret_cast<uintptr_t>(p) % 16;
    return rest == 0;
}

template <class T, int NV, int G>
onecomp_status launch(const Params& P, bool gradient, hipStream_t stream) {
    return whole_vectors<T>(P) ? launch_whole<T, NV, G, true>(P, gradient, stream) : launch_whole<T, NV, G, false>(P, gradient, stream);
}

// As few threads as hold a row with 16 bytes each: sums cross the fewest waves, and registers stay free for the parameters'
// sums.  (fp32 with two vectors a thread: gradients of 3001 rows of 1359 52 us instead of 47.)  Rows over 8192 (bf16) or 4096
// (fp32) take more per thread.
template <class T>
onecomp_status run(const Params& P, bool gradient, hipStream_t s) {
    constexpr int V = 16 / int(sizeof(T));
    const int w = P.width;
    if (w <= 64 * V) return launch<T, 1, 64>(P, gradient, s);
    if (w <= 256 * V) return launch<T, 1, 256>(P, gradient, s);
    if (w <= 512 * V) return launch<T, 1, 512>(P, gradient, s);
    if (w <= 1024 * V) return launch<T, 1, 1024>(P, gradient, s);
    if (w <= 2048 * V) return launch<T, 2, 1024>(P, gradient, s);
    if constexpr (V == 4) {
        if (w > 4096 * V) return launch<T, 8, 1024>(P, gradient, s);
    }
    return launch<T, 4, 1024>(P, gradient, s);
}

}  // namespace

size_t gradient_workspace_bytes(int64_t rows, int64_t width, int wanted) {
    const int64_t most = rows < 1 ? 1 : rows < 1024 ? rows : 1024;               // no device has more workgroups of these at a time
    return numbers_bytes(rows, width) + align_up(size_t(most) * size_t(width) * size_t(__builtin_popcount(unsigned(wanted))) * 4, 256);
}

onecomp_status norm_run(onecomp_dtype dtype, const Params& in, bool gradient, hipStream_t stream) {
    Params P = in;
    const Scratch scratch = scratch_of(P.part, P.rows, P.width, P.wanted);
    P.row_numbers = reinterpret_cast<float*>(scratch.numbers);
    P.part = reinterpret_cast<float*>(scratch.sums);
    return dtype == ONECOMP_BF16 ? run<uint16_t>(P, gradient, stream) : run<float>(P, gradient, stream);
}

}  // namespace block
}  // namespace onecomp
