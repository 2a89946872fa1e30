// Tiles of matrix products for the 32 x 32 matrix instructions, from operands of 8, 16 or 32 bits in either order.
//
//   C[m][n] = sum_k A[n][k] B[m][k]
//
// n is the axis along which results are dense in memory: in the accumulators a lane holds four neighbours of n (rows of the
// instruction's result) for one m (its column), so that sums over n stay in a lane and results go out in vectors.  An operand is
// given ALONG k (k dense in memory) or ACROSS it (n, or m, dense: rows of k).
//
// Whatever the type, a step is 64 or 128 bytes of k per row and an instruction's fragment 16 bytes per lane: lanes 0 .. 31 hold
// the first, lanes 32 .. 63 the second 16 bytes of 32 (8 bf16, 16 int8, 4 fp32 values).  Tiles reach LDS by direct loads through a
// ring of four or two steps; the fragments of 32 bytes are read while those before are multiplied, reads and loads one by one
// behind the matrix instructions.
//   ALONG   a row's bytes of a step are chunks of 16, permuted per row (Side::turn) so that rows' same chunk fall into different
//           banks.
//   ACROSS  rows of k as they are; in bf16 their chunks lie permuted by fours (Side::swizzle) and fragments are transposed
//           reads; in fp32 a fragment is four plain reads.
// What lies behind the operands' ends becomes zeros by the loads' bounds check.
//
// The loss's operands come in panels where they are written here: 64 bytes of the columns of all rows, [panel][row][64 bytes].  A
// wave's load is then 1 KB of memory instead of 64 bytes in each of 16 rows (16384 x 32000 logits, k 4096, bf16: 1.22 PFLOP/s from
// rows, 1.34 from panels).  The same panels serve products along the columns (PANELS_ALONG) and along the rows (PANELS_ACROSS).
#pragma once
#include "common.hpp"
#include "token_plan.hpp"
#include <type_traits>
#include <utility>

namespace onecomp {
namespace product {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int16v __attribute__((ext_vector_type(16)));
typedef uint4v uint4u __attribute__((aligned(2)));               // at any address of 16-bit elements

struct Bf16 {
    typedef uint16_t T;
    typedef float16v Acc;
    static constexpr int ESZ = 2;
    static __device__ __forceinline__ uint4v left(uint4v a) { return a; }
    static __device__ __forceinline__ Acc mma(uint4v a, uint4v b, Acc c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct F32 {
    typedef float T;
    typedef float16v Acc;
    static constexpr int ESZ = 4;
    static __device__ __forceinline__ uint4v left(uint4v a) { return a; }
    static __device__ __forceinline__ Acc mma(uint4v a, uint4v b, Acc c) {
        const float4v x = __builtin_bit_cast(float4v, a), y = __builtin_bit_cast(float4v, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};
// left operand unsigned, less 128 (which turns its zeros behind the end into -128, times zeros of the right one); right signed
struct Int8 {
    typedef uint8_t T;
    typedef int16v Acc;
    static constexpr int ESZ = 1;
    static __device__ __forceinline__ uint4v left(uint4v a) { return a ^ 0x80808080u; }
    static __device__ __forceinline__ Acc mma(uint4v a, uint4v b, Acc c) {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(int4v, a), __builtin_bit_cast(int4v, b), c, 0, 0, 0);
    }
};

enum Layout { ALONG, ACROSS, PANELS_ALONG, PANELS_ACROSS };
constexpr bool across(Layout l) { return l == ACROSS || l == PANELS_ACROSS; }
constexpr bool panels(Layout l) { return l == PANELS_ALONG || l == PANELS_ACROSS; }

// rows: how many n (m) there are; stride: bytes between rows of n (ALONG) or of k (ACROSS), below 2^23, or between panels; like the
// address, a multiple of 16
struct Operand {
    const char* data;
    int64_t stride, rows;
};

// WR x WC waves of FR x FC fragments each: a tile of 32 WR FR (n) by 32 WC FC (m), in steps of STEP bytes of k.  SPLIT groups of such waves share the steps of k
// out, each with a ring of its own; their sums meet in LDS in the groups' order.  PER_CU workgroups are meant to share a
// compute unit.
template <int WR_, int WC_, int FR_, int FC_, int STEP_, int SPLIT_, int PER_CU_>
struct Shape {
    static constexpr int WR = WR_, WC = WC_, FR = FR_, FC = FC_, STEP = STEP_, SPLIT = SPLIT_, PER_CU = PER_CU_, SLOTS = 256 / STEP;
    static constexpr int WAVES = WR * WC, THREADS = 64 * WAVES, ALL_THREADS = THREADS * SPLIT;   // of a group, of a workgroup
    static constexpr int PER_SIMD = PER_CU * WAVES * SPLIT / 4;                                  // waves
    static constexpr int TN = 32 * WR * FR, TM = 32 * WC * FC;
    static constexpr int STAGE = (TN + TM) * STEP, RING = SLOTS * STAGE, LDS = SPLIT * RING;
    static_assert((SPLIT - 1) * THREADS * FR * FC * 64 <= LDS, "room for the groups' sums");
};
constexpr uint32_t NOWHERE = 0xFFFFFFF0u;

// One operand's tile: how a wave brings its part of a step to LDS, and how a lane reads fragments from there.
template <class E, Layout L, int T, int WAVES, int STEP>
struct Side {
    static constexpr int LOADS = T * STEP / 1024 / WAVES, ROW_CHUNKS = STEP / 16;   // loads of 1 KB, per wave and step
    static_assert(T * STEP % (1024 * WAVES) == 0, "whole loads per wave");
    static_assert(!panels(L) || STEP == 64, "a panel is a step along the columns");
    static_assert(!across(L) || E::ESZ != 1, "no transposed reads of bytes here");
    static constexpr int ROWB = T * E::ESZ, CHUNKS = ROWB / 16;   // ACROSS: a row of k
    static constexpr int PER_PANEL = E::ESZ == 2 ? 2 : 1;         // PANELS_ACROSS: loads of a step's rows of one panel
    // along k: chunk c of row r of the tile lies at c ^ turn(r).  LDS serves 16 lanes together, 16 rows of one chunk: with 64 bytes a row
    // they lie in different banks, with 128 two and two share theirs (a turn that repeats after eight rows, those of one load;
    // without these conflicts the 8-bit products take as long: 501 and 503 us for 8192 x 4096 x 14336).
    static __device__ __forceinline__ int turn(int r) { return STEP == 64 ? (r >> 2) & 3 : r & 7; }
    // ACROSS, bf16: which group of four chunks goes where in row r of k; the same for r + 4.  Four rows of a read lie 64 bytes
    // apart in the banks (rows of 128 bytes: two and two).
    static __device__ __forceinline__ int swizzle(int r) { return CHUNKS >= 16 ? r & 3 : (r >> 1) & 1; }
    static_assert(L != ACROSS || E::ESZ != 2 || CHUNKS == 8 || CHUNKS % 16 == 0, "the swizzle stays inside a row");
    uint32_t off[LOADS], lane_at;                                 // lane_at: where the lane's 16 bytes lie in a step of a row or panel
    const char* p;
    int64_t left, step, taken;                                    // bytes: what is left of the operand (of a row, of a panel); a step's in memory, of `left`
    int read0;
    // group: of `split` that take the steps in turn
    __device__ __forceinline__ void init(const Operand& o, int64_t first, int64_t inner, int wave, int lane, int group, int split) {
        const int i16 = lane & 15, kq = i16 >> 2, half = lane >> 5, r32 = lane & 31;
        if constexpr (!across(L)) {
            const int64_t row = L == ALONG ? o.stride : 64, one = L == ALONG ? STEP : o.stride;
            p = o.data + first * row + group * one;
            left = inner * E::ESZ - group * STEP;
            step = one * split;
            taken = STEP * split;
            lane_at = uint32_t((lane % ROW_CHUNKS) ^ turn(lane / ROW_CHUNKS)) * 16u;
#pragma unroll
            for (int q = 0; q < LOADS; ++q) {
                const int r = ((wave * LOADS + q) * 64 + lane) / ROW_CHUNKS;
                off[q] = first + r < o.rows ? uint32_t(r) * uint32_t(row) + lane_at : NOWHERE;
            }
            read0 = r32 * STEP + ((half ^ turn(r32)) << 4);
        } else if constexpr (L == ACROSS) {
            const int64_t one = int64_t(STEP / E::ESZ) * o.stride;
            p = o.data + first * E::ESZ + group * one;
            left = inner * o.stride - first * E::ESZ - group * one;
            step = taken = one * split;
            lane_at = 0;
#pragma unroll
            for (int q = 0; q < LOADS; ++q) {
                const int at = (wave * LOADS + q) * 64 + lane, r = at / CHUNKS;
                const int c = (at % CHUNKS) ^ (E::ESZ == 2 ? swizzle(r) << 2 : 0);
                off[q] = first + c * (16 / E::ESZ) < o.rows ? uint32_t(r) * uint32_t(o.stride) + uint32_t(c) * 16u : NOWHERE;
            }
            // bf16: inside 16 lanes, lane 4 k + c points at four columns of row k and lane i receives column i of rows 0 .. 3
            if constexpr (E::ESZ == 2) read0 = (half * 8 + kq) * ROWB + (2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
            else read0 = half * 4 * ROWB + r32 * 4;
        } else {
            constexpr int ROWS = 64 / E::ESZ;                     // of k, per step
            p = o.data + first * E::ESZ / 64 * o.stride + group * (ROWS * 64);
            left = inner * 64 - group * (ROWS * 64);
            step = taken = int64_t(ROWS * 64) * split;
            lane_at = uint32_t(lane) * 16u;
#pragma unroll
            for (int q = 0; q < LOADS; ++q) {
                const int j = wave * LOADS + q, panel = j / PER_PANEL;
                off[q] = first + panel * (64 / E::ESZ) < o.rows ? uint32_t(panel) * uint32_t(o.stride) + uint32_t(j % PER_PANEL) * 1024u + lane_at : NOWHERE;
            }
            // a fragment's 32 columns: a panel of 64 bytes a row (bf16), two panels (fp32)
            if constexpr (E::ESZ == 2) read0 = (half * 8 + kq) * 64 + (2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
            else read0 = (r32 >> 4) * 1024 + half * 4 * 64 + (r32 & 15) * 4;
        }
    }
    struct Step {
        __amdgpu_buffer_rsrc_t rsrc;
        uint32_t mask[PER_PANEL];
    };
    // the next step: an empty range, or masks, behind the last one
    __device__ __forceinline__ Step next() {
        Step s;
        const int64_t range = L != ACROSS ? 0x7FFFFFFF : left > 0x7FFFFFFF ? 0x7FFFFFFF : left > 0 ? left : 0;
        s.rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, int(range), 0x00020000);
        const int here = left > 4096 ? 4096 : left < 0 ? 0 : int(left);
#pragma unroll
        for (int i = 0; i < PER_PANEL; ++i) s.mask[i] = L == ACROSS || int(lane_at) + i * 1024 < here ? 0u : NOWHERE;
        p += step;
        left -= taken;
        return s;
    }
    __device__ __forceinline__ void load(const Step& s, uint32_t lds, int wave, int q) const {
        const uint32_t mask = PER_PANEL == 2 && L == PANELS_ACROSS && ((wave * LOADS + q) & 1) ? s.mask[PER_PANEL - 1] : s.mask[0];
        lds_load16(lds + uint32_t(wave * LOADS + q) * 1024u, L == ACROSS ? off[q] : off[q] | mask, s.rsrc);
    }
    // fragment f of the tile (32 of n or m), 32 bytes s of the step
    __device__ __forceinline__ uint4v read(const char* tile, int f, int s, int lane) const {
        if constexpr (!across(L)) {
            return *reinterpret_cast<const uint4v*>(tile + f * 32 * STEP + (read0 ^ (s << 5)));
        } else if constexpr (E::ESZ == 2) {
            constexpr int ROW = L == ACROSS ? ROWB : 64;
            const char* a = tile + s * 16 * ROW + read0 + (L == ACROSS ? (f ^ swizzle((lane & 15) >> 2)) << 6 : f * 2048);
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ONECOMP_LDS short4v*)(a));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ONECOMP_LDS short4v*)(a + 4 * ROW));
            return __builtin_bit_cast(uint4v, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            constexpr int ROW = L == ACROSS ? ROWB : 64;
            const char* a = tile + s * 8 * ROW + read0 + f * (L == ACROSS ? 128 : 2048);
            uint4v v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t*>(a + i * ROW);
            return v;
        }
    }
};

template <int... I, class F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f) {
    (f(std::integral_constant<int, I>{}), ...);
}

// acc = the products of tile (n0, m0) over `inner` values of k, in the first group of waves; the others return false and have
// nothing left to do.  lds: S::LDS bytes, free again for the caller behind a barrier.
template <class E, Layout LA, Layout LB, class S>
__device__ __forceinline__ bool multiply(char* lds, const Operand& A, const Operand& B, int64_t n0, int64_t m0, int64_t inner,
                                         typename E::Acc (&acc)[S::FR][S::FC]) {
    constexpr int FR = S::FR, FC = S::FC, SLOTS = S::SLOTS;
    const int lane = threadIdx.x & 63, all_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = S::SPLIT == 1 ? 0 : all_wave / S::WAVES, wave = S::SPLIT == 1 ? all_wave : all_wave % S::WAVES;
    const int wr = wave / S::WC, wc = wave % S::WC;
    char* const all_lds = lds;
    lds += group * S::RING;
    typedef Side<E, LA, S::TN, S::WAVES, S::STEP> SideA;
    typedef Side<E, LB, S::TM, S::WAVES, S::STEP> SideB;
    constexpr int LOADS = SideA::LOADS + SideB::LOADS, FRAGS = FR + FC, PRODUCTS = FR * FC;
    constexpr int B_AT = S::TN * S::STEP, PARTS = S::STEP / 32;   // parts of a step: a fragment each
    SideA a;
    SideB b;
    a.init(A, n0, inner, wave, lane, group, S::SPLIT);
    b.init(B, m0, inner, wave, lane, group, S::SPLIT);
    const uint32_t lds0 = uint32_t(uintptr_t((ONECOMP_LDS char*)lds));
    struct Step {
        typename SideA::Step a;
        typename SideB::Step b;
    };
    auto next = [&]() __attribute__((always_inline)) { return Step{a.next(), b.next()}; };
    auto load = [&](const Step& s, int slot, int i) __attribute__((always_inline)) {   // number i of a step's
        if (i < SideA::LOADS) a.load(s.a, lds0 + slot * S::STAGE, wave, i);
        else b.load(s.b, lds0 + slot * S::STAGE + B_AT, wave, i - SideA::LOADS);
    };
    for (int st = 0; st < SLOTS - 1; ++st) {
        const Step s = next();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(s, st, i);
    }
#pragma unroll
    for (int i = 0; i < FR; ++i)
#pragma unroll
        for (int j = 0; j < FC; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    struct Frags {
        uint4v a[FR], b[FC];
    };
    Frags F0, F1;
    // fragment r of FRAGS, those of both operands in turn
    auto read = [&](Frags& f, int r, int slot, int s) __attribute__((always_inline)) {
        constexpr int BOTH = 2 * (FR < FC ? FR : FC);
        const bool of_a = r < BOTH ? !(r & 1) : FR > FC;
        const int i = r < BOTH ? r >> 1 : r - BOTH / 2;
        if (of_a) f.a[i] = a.read(lds + slot * S::STAGE, wr * FR + i, s, lane);
        else f.b[i] = b.read(lds + slot * S::STAGE + B_AT, wc * FC + i, s, lane);
    };
    // `behind(n)` goes behind product n
    auto products = [&](Frags& f, auto&& behind) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < PRODUCTS; ++n) {
            const int i = n / FC, j = i & 1 ? FC - 1 - n % FC : n % FC;   // one operand stays from one product to the next
            if (n % FC == 0) f.a[i] = E::left(f.a[i]);
            acc[i][j] = E::mma(f.a[i], f.b[j], acc[i][j]);
            behind(n);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const int64_t bytes = inner * E::ESZ;
    const int n_st = (int((bytes + S::STEP - 1) / S::STEP) + S::SPLIT - 1) / S::SPLIT;
    __builtin_amdgcn_s_waitcnt(wait_vmcnt(LOADS * (SLOTS - 2)));
    __syncthreads();
    {
        const Step s = next();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(s, SLOTS - 1, i);
    }
#pragma unroll
    for (int r = 0; r < FRAGS; ++r) read(F0, r, 0, 0);
    // what of `all` things goes behind product n
    auto share = [](int n, int all, auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int x = n * all / PRODUCTS; x < (n + 1) * all / PRODUCTS; ++x) f(x);
    };
    auto stage = [&](auto slot_c) __attribute__((always_inline)) {
        constexpr int slot = decltype(slot_c)::value, follow = (slot + 1) % SLOTS;
        auto early = [&](Frags& now, Frags& then, int part) __attribute__((always_inline)) {
            products(now, [&](int n) __attribute__((always_inline)) {
                if constexpr (PRODUCTS > FRAGS) {
                    if (n < FRAGS) read(then, n, slot, part);
                } else {
                    share(n, FRAGS, [&](int r) __attribute__((always_inline)) { read(then, r, slot, part); });
                }
            });
        };
#pragma unroll
        for (int part = 1; part < PARTS; ++part) early(part & 1 ? F0 : F1, part & 1 ? F1 : F0, part);
        // the next step has landed; every wave has read this one
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(LOADS * (SLOTS - 2)));
        __syncthreads();
        const Step s = next();
        products(F1, [&](int n) __attribute__((always_inline)) {
            share(n, LOADS + FRAGS, [&](int x) __attribute__((always_inline)) {
                constexpr int BOTH = 2 * (LOADS < FRAGS ? LOADS : FRAGS);
                const bool is_read = x < BOTH ? !(x & 1) : FRAGS > LOADS;
                const int i = x < BOTH ? x >> 1 : x - BOTH / 2;
                if (is_read) read(F0, i, follow, 0);
                else load(s, slot, i);
            });
        });
    };
    int st = 0;
#pragma unroll 1
    for (; st + SLOTS <= n_st; st += SLOTS) each_of(std::make_integer_sequence<int, SLOTS>{}, stage);
    const int rest = n_st - st;
    each_of(std::make_integer_sequence<int, SLOTS - 1>{}, [&](auto slot_c) __attribute__((always_inline)) {
        if (decltype(slot_c)::value < rest) stage(slot_c);
    });
    __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));                    // no LDS write may be in flight when the tile ends
    if constexpr (S::SPLIT > 1) {
        typedef std::conditional_t<std::is_same<typename E::Acc, int16v>::value, int, float> X;
        X* const sums = reinterpret_cast<X*>(all_lds) + threadIdx.x % S::THREADS;
        constexpr int EACH = FR * FC * 16 * S::THREADS;
        __syncthreads();
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FC; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sums[(group - 1) * EACH + ((i * FC + j) * 16 + r) * S::THREADS] = acc[i][j][r];
        }
        __syncthreads();
        if (group > 0) return false;
#pragma unroll
        for (int g = 0; g < S::SPLIT - 1; ++g)
#pragma unroll
            for (int i = 0; i < FR; ++i)
#pragma unroll
                for (int j = 0; j < FC; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] += sums[g * EACH + ((i * FC + j) * 16 + r) * S::THREADS];
    }
    return true;
}

// f(shape) for a choice of tiles; LARGE, SPLIT: whether the choice may be of 128 x 128 and more, of waves that share k
template <int STEP, bool LARGE, bool SPLIT, class F>
auto with_shape(token::Tiles t, F&& f) {
    if constexpr (LARGE) {
        if (t == token::BIG) return f(Shape<2, 2, 4, 4, STEP, 1, 1>{});      // 256 x 256
        if (t == token::MID) return f(Shape<2, 2, 2, 2, STEP, 1, 2>{});      // 128 x 128
    }
    if constexpr (SPLIT) {
        if (t == token::SMALL_SPLIT) return f(Shape<2, 2, 1, 1, STEP, 4, 1>{});
    }
    return t == token::HALF ? f(Shape<2, 2, 2, 1, STEP, 1, 3>{})             // 128 x 64
                            : f(Shape<2, 2, 1, 1, STEP, 1, 4>{});            // 64 x 64
}

// Rows to panels: row r of the result is row(r) of the source (nullptr: nothing is there), row_bytes long (a multiple of 16); what is
// behind a row's end in its last panel becomes zeros.  A wave takes 16 rows of eight panels at a time: 512 bytes a row in, 1 KB
// out per panel.  `units` of these are shared out over the workgroups from `unit` on in steps of `stride`.
template <class R>
__device__ __forceinline__ void rows_to_panels(R&& row, int rows, int64_t row_bytes, char* to, int64_t panel, int unit, int stride) {
    const int lane = threadIdx.x & 63, c = lane & 3;
    const int n_panels = int((row_bytes + 63) >> 6), eights = (n_panels + 7) / 8, units = (rows + 15) / 16 * eights;
    for (; unit < units; unit += stride) {
        const int r = unit / eights * 16 + (lane >> 2), first = unit % eights * 8;
        const char* const from = r < rows ? row(r) : nullptr;
        uint4v v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t at = int64_t(first + u) * 64 + c * 16;
            v[u] = uint4v{0u, 0u, 0u, 0u};
            if (from && at < row_bytes) v[u] = *reinterpret_cast<const uint4v*>(from + at);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (r < rows && first + u < n_panels) *reinterpret_cast<uint4v*>(to + (first + u) * panel + r * 64 + c * 16) = v[u];
    }
}

// tile_of for a workgroup of this launch, in scalar registers
__device__ __forceinline__ bool my_tile(int m_tiles, int n_tiles, int& tm, int& tn) {
    if (!tile_of(blockIdx.x, m_tiles, n_tiles, tm, tn)) return false;
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    return true;
}

// The tile's results to memory through LDS, in whole lines: a wave's 32 FR of n for 32 of m at a time.  Straight from the
// accumulators a store would touch 32 rows with 8 or 16 bytes each.
//   value(x, i, j, q, n, m)   four neighbours of n from acc[i][j][4 q ..]; n and m inside the tile
//   row(m)                    address of n = 0 of the tile in row m of the tile, or nullptr: no such row
//   left                      how many n there are from the tile's first on
//   panel                     0: rows are dense; else rows are 64 bytes of the tile's panels, which are so many bytes apart (all of them
//                             are written)
// ADD: added to what is there (fp32).  lds: the tile's, behind a barrier; out_lds() bytes of it are used.
template <class T, class S>
constexpr int out_lds() { return S::WAVES * 32 * (32 * S::FR * int(sizeof(T)) + 16); }

template <class T, class S, bool ADD, class V, class R>
__device__ __forceinline__ void store_tile(char* lds, V&& value, R&& row, int64_t left, int64_t panel = 0) {
    constexpr int NW = 32 * S::FR, PITCH = NW * int(sizeof(T)) + 16, CHUNKS = NW * int(sizeof(T)) / 16, N = 16 / int(sizeof(T));
    static_assert(out_lds<T, S>() <= S::LDS, "room in the tile's LDS");
    static_assert(!ADD || sizeof(T) == 4, "added in 32 bits");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / S::WC, wc = wave % S::WC;
    char* const mine = lds + wave * 32 * PITCH;
#pragma unroll
    for (int j = 0; j < S::FC; ++j) {
#pragma unroll
        for (int i = 0; i < S::FR; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = i * 32 + 8 * q + 4 * (lane >> 5);
                float x[4];
                value(x, i, j, q, wr * NW + n, (wc * S::FC + j) * 32 + (lane & 31));
                T* const to = reinterpret_cast<T*>(mine + (lane & 31) * PITCH) + n;
                if constexpr (sizeof(T) == 2) {
                    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                    bf16x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = static_cast<__bf16>(x[e]);
                    *reinterpret_cast<bf16x4*>(to) = v;
                } else {
                    float4v v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = x[e];
                    *reinterpret_cast<float4v*>(to) = v;
                }
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int it = 0; it < CHUNKS / 2; ++it) {
            const int id = it * 64 + lane;
            if (panel) {
                const int r = id % 128 / 4, c = id / 128 * 4 + id % 4;
                T* const to = row((wc * S::FC + j) * 32 + r);
                if (to) *reinterpret_cast<uint4v*>(reinterpret_cast<char*>(to) + (wr * (CHUNKS / 4) + id / 128) * panel + id % 4 * 16) = *reinterpret_cast<const uint4v*>(mine + r * PITCH + c * 16);
                continue;
            }
            const int r = id / CHUNKS, c = id % CHUNKS, n = wr * NW + c * N;
            uint4v v = *reinterpret_cast<const uint4v*>(mine + r * PITCH + c * 16);
            T* const to = row((wc * S::FC + j) * 32 + r);
            if (!to || n >= left) continue;
            if (n + N <= left) {
                if constexpr (ADD) v = __builtin_bit_cast(uint4v, __builtin_bit_cast(float4v, v) + *reinterpret_cast<const float4v*>(to + n));
                *reinterpret_cast<uint4u*>(to + n) = v;
            } else {
                const T* const from = reinterpret_cast<const T*>(mine + r * PITCH + c * 16);
                for (int e = 0; n + e < left; ++e) {
                    if constexpr (ADD) to[n + e] += from[e];
                    else to[n + e] = from[e];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- few rows of m ------------------------------------------------------------------------------------------------------
// 16 RF of n by 16 TF of m per workgroup, whose eight waves share k out: every byte of A is read once, straight into the
// registers of the 16 x 16 matrix instructions (64 bytes of k per row and step), and the waves' sums meet in LDS in their order.
template <class E> struct Few;
template <> struct Few<Bf16> {
    typedef float4v Acc;
    static __device__ __forceinline__ Acc mma(uint4v a, uint4v b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Few<F32> {
    typedef float4v Acc;
    static __device__ __forceinline__ Acc mma(uint4v a, uint4v b, Acc c) {
        const float4v x = __builtin_bit_cast(float4v, a), y = __builtin_bit_cast(float4v, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};
template <> struct Few<Int8> {
    typedef int4v Acc;
    static __device__ __forceinline__ Acc mma(uint4v a, uint4v b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(int4v, a), __builtin_bit_cast(int4v, b), c, 0, 0, 0);
    }
};

constexpr int FEW_WAVES = 8;
template <int RF, int TF>
constexpr int few_lds() { return FEW_WAVES * 16 * RF * 16 * TF * 4; }

// sums[n + 16 RF m] in the first 1024 RF TF bytes of lds, behind a barrier
// row(m): the row of B that is row m of the product, or -1 (B.rows is not looked at)
template <class E, int RF, int TF, class R>
__device__ __forceinline__ void multiply_few(char* lds, const Operand& A, const Operand& B, R&& row, int64_t n0, int64_t inner) {
    typedef typename Few<E>::Acc Acc;
    constexpr int AHEAD = RF + TF >= 5 ? 2 : 4;                   // steps on their way at a time
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bytes = int(inner) * E::ESZ, steps = (bytes + 63) >> 6;
    uint32_t at[RF], bt[TF];
    const uint32_t chunk = uint32_t(lane >> 4) * 16u;
#pragma unroll
    for (int i = 0; i < RF; ++i) {
        const int r = i * 16 + (lane & 15);
        at[i] = n0 + r < A.rows ? uint32_t(r) * uint32_t(A.stride) + chunk : NOWHERE;
    }
#pragma unroll
    for (int j = 0; j < TF; ++j) {
        const int r = row(j * 16 + (lane & 15));
        bt[j] = r >= 0 ? uint32_t(r) * uint32_t(B.stride) + chunk : NOWHERE;
    }
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(A.data + n0 * A.stride), 0, 0x7FFFFFFF, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(B.data), 0, 0x7FFFFFFF, 0x00020000);
    Acc acc[RF][TF];
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < TF; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = 0;
    // Two sets of AHEAD steps: one on its way while the other is multiplied.
    struct Set {
        uint4v a[AHEAD][RF], b[AHEAD][TF];
    };
    auto load = [&](Set& x, int s0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int k = (s0 + u) * 64;
            const bool there = k + int(chunk) < bytes;
#pragma unroll
            for (int i = 0; i < RF; ++i) x.a[u][i] = __builtin_amdgcn_raw_buffer_load_b128(ra, there && at[i] != NOWHERE ? at[i] + k : NOWHERE, 0, 0);
#pragma unroll
            for (int j = 0; j < TF; ++j)
                x.b[u][j] = __builtin_amdgcn_raw_buffer_load_b128(rb, there && bt[j] != NOWHERE ? bt[j] + k : NOWHERE, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](const Set& x) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int i = 0; i < RF; ++i) {
                const uint4v left = E::left(x.a[u][i]);
#pragma unroll
                for (int j = 0; j < TF; ++j) acc[i][j] = Few<E>::mma(left, x.b[u][j], acc[i][j]);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int TURN = FEW_WAVES * AHEAD;
    Set x, y;
    if (wave * AHEAD < steps) load(x, wave * AHEAD);
    for (int s0 = wave * AHEAD; s0 < steps; s0 += 2 * TURN) {
        if (s0 + TURN < steps) load(y, s0 + TURN);
        products(x);
        if (s0 + TURN >= steps) break;
        if (s0 + 2 * TURN < steps) load(x, s0 + 2 * TURN);
        products(y);
    }
    constexpr int ALL = 16 * RF * 16 * TF;
    typedef std::conditional_t<std::is_same<Acc, int4v>::value, int, float> X;
    X* const sums = reinterpret_cast<X*>(lds);
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < TF; ++j)
            *reinterpret_cast<Acc*>(sums + wave * ALL + (j * 16 + (lane & 15)) * 16 * RF + i * 16 + 4 * (lane >> 4)) = acc[i][j];
    __syncthreads();
    for (int e = threadIdx.x; e < ALL; e += 64 * FEW_WAVES) {
        X x = sums[e];
#pragma unroll
        for (int w = 1; w < FEW_WAVES; ++w) x += sums[w * ALL + e];
        sums[e] = x;                                              // its own place: nobody else reads it before the barrier
    }
    __syncthreads();
}

}  // namespace product
}  // namespace onecomp
