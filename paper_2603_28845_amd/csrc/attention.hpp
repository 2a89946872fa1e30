// Shared device code of the attention kernels: which sequence and tile a workgroup has, tiles on their way to LDS, and the
// two products that every kernel is made of.
//
// All scores live in registers in the layout of a 32 x 32 MFMA accumulator: lane l holds column l % 32 and the rows
// 8 (r / 4) + 4 (l / 32) + r % 4, r = 0 .. 15.  The sum over the rows that follows (probabilities times values, and its
// likes in the gradients) takes these registers as its right operand as they are: a product's inner index may run in any
// order, so the left operand is read from LDS in the order 0..3, 8..11 (lanes 0..31) and 4..7, 12..15 (lanes 32..63) and no
// score ever moves between lanes.
#pragma once
#include "common.hpp"
#include "attention_plan.hpp"

namespace onecomp {
namespace attn {

// One tensor of packed rows: [token, head, dim], the last dense.
struct View {
    const void* p;
    int64_t token, head;   // strides in elements
};

struct Params {
    View q, k, v, o;       // o: output of the forward call, input of the gradients
    View d_o, dq, dk, dv;
    float* lse;            // [heads, total_q], may be null in the forward call
    float* aux;            // scratch of the gradients: [2, heads, total_q], -lse / scale and -d_out . out
    float* part;           // scratch of calls whose keys or queries are split
    int splits_q, splits_k;   // gradients: shares of the keys for dq, of the queries for dk and dv
    const int32_t *cu_q, *cu_k, *len_k;
    int64_t total_q, total_k;
    int n_seqs, heads, kv_heads, group, dim, causal;
    int splits, run;       // few rows: runs of keys and the keys of a run; splits = 0: whole prompts
    int64_t max_q, max_k;
    float scale, c;        // c = scale log2(e): probabilities are powers of two
};

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NEG_INF = -__builtin_huge_valf();

// ---- element types ------------------------------------------------------------------------------------------------------
// DT: head dimension in units of 32, rounded up (columns behind the head dimension are zeros in LDS).
struct Bf16 {
    typedef uint16_t T;
    static constexpr int PER_CHUNK = 8;          // elements of a 16-byte chunk
    typedef bf16x8 Row;                          // a chunk as an operand whose inner index is the head dimension
    typedef bf16x8 Score;                        // eight score registers as a right operand
    // Probabilities and their gradients are rounded to bf16 here, for the matrix pipes to take them beside the inputs: each term of a
    // sum moves by 2^-9 of itself at most, at random, which leaves results 1.2 to 1.4 times as far from exact ones as their own rounding
    // does (outputs 0.0019 to 0.0022 instead of 0.0015 to 0.0017, gradients 0.0024 instead of 0.0017, root mean square).  Two bf16 halves of
    // each would take that away and double the products they enter.
    static __device__ __forceinline__ Score pack(const float* s) {
        bf16x8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = static_cast<__bf16>(s[i]);
        return r;
    }
    static __device__ __forceinline__ float16v mma(Row a, Row b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float to_float(T x) { return __uint_as_float(uint32_t(x) << 16); }
};
struct F32 {
    typedef float T;
    static constexpr int PER_CHUNK = 4;
    typedef float4v Row;
    struct Score { float s[8]; };
    static __device__ __forceinline__ Score pack(const float* s) {
        Score r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.s[i] = s[i];
        return r;
    }
    static __device__ __forceinline__ float16v mma(Row a, Row b, float16v c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ float to_float(T x) { return x; }
};

// A tile of ROWS rows in LDS.  Rows are PITCH bytes, a power of two; the 16-byte chunk c of row r lies at c ^ swizzle(r).
// Sixteen rows of one chunk (row reads) lie in different banks, and so do four chunks in a row of four rows (transposed
// reads, which go by 32 lanes).
template <class E, int DT>
struct Tile {
    static constexpr int ESZ = int(sizeof(typename E::T));
    static constexpr int PITCH = (DT == 3 ? 128 : 32 * DT) * ESZ;
    static constexpr int CHUNKS = PITCH / 16;                     // of a row
    static constexpr int STEPS = 32 * DT * ESZ / 32;              // pairs of chunks that hold data: inner steps of a row product
    static __device__ __forceinline__ int swizzle(int r) {
        const int fours = (r >> 2) & 3;
        return CHUNKS >= 16 ? (r & 3) << 2 | fours : CHUNKS == 8 ? (r >> 1 & 1) << 2 | fours : fours;
    }
    static constexpr int bytes(int rows) { return rows * PITCH; }
};

// What one thread needs to bring its part of ROWS rows from memory to LDS, WAVES waves sharing the work.
template <class E, int DT, int ROWS, int WAVES>
struct Loader {
    typedef attn::Tile<E, DT> T;
    static constexpr int LOADS = T::bytes(ROWS) / 1024;           // wave-wide loads of 64 chunks
    static constexpr int MINE = (LOADS + WAVES - 1) / WAVES;
    static constexpr int STEP = WAVES * 1024 / T::PITCH;          // rows between two loads of a wave
    // whole periods of the swizzle: the same columns again, one offset is enough
    static constexpr bool SAME = STEP % 16 == 0;
    // out of every range, and stays so with what is added to it (64 rows of 2^24 bytes)
    static constexpr uint32_t NOWHERE = 0x80000000u;
    uint32_t off[SAME ? 1 : MINE];
    uint32_t row_bytes, dim_bytes;
    __device__ __forceinline__ void init(int wave, int lane, int64_t token_stride, int dim) {
        row_bytes = uint32_t(token_stride) * T::ESZ;
        dim_bytes = uint32_t(dim) * T::ESZ;
#pragma unroll
        for (int i = 0; i < (SAME ? 1 : MINE); ++i) {
            const int at = (wave + i * WAVES) * 64 + lane, r = at / T::CHUNKS;
            const uint32_t chunk = uint32_t((at % T::CHUNKS) ^ T::swizzle(r)) * 16u;
            off[i] = chunk < dim_bytes ? uint32_t(r) * row_bytes + chunk : NOWHERE;
        }
    }
    // first: address of the tile's first row (wave-uniform); rows behind `valid` and columns behind the head dimension
    // become zeros, whatever lies there
    __device__ __forceinline__ void load(uint32_t lds, const char* first, int valid, int wave) const {
        valid = valid < 0 ? 0 : valid > ROWS ? ROWS : valid;
        const uint32_t range = valid == 0 ? 0u : uint32_t(valid - 1) * row_bytes + dim_bytes;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first), 0, int(range), 0x00020000);
#pragma unroll
        for (int i = 0; i < MINE; ++i)
            if (LOADS % WAVES == 0 || wave + i * WAVES < LOADS)
                lds_load16(lds + uint32_t(wave + i * WAVES) * 1024u, SAME ? off[0] + uint32_t(i * STEP) * row_bytes : off[i], rsrc);
    }
    // Puts zeros for what is not finite in what this wave brought, and tells f of each: (row of the tile, column, whether it raises
    // a sum, whether it lowers it); what is no number does both.
    template <class F>
    static __device__ __forceinline__ void clean(char* tile, int wave, int lane, F f) {
        typedef typename E::T X;
#pragma unroll 1
        for (int i = 0; i < MINE; ++i) {
            if (LOADS % WAVES != 0 && wave + i * WAVES >= LOADS) break;
            const int at = (wave + i * WAVES) * 64 + lane, r = at / T::CHUNKS, col = ((at % T::CHUNKS) ^ T::swizzle(r)) * E::PER_CHUNK;
            uint4v* to = reinterpret_cast<uint4v*>(tile + at * 16);
            uint4v x = *to;
            bool odd = false;
#pragma unroll
            for (int w = 0; w < 4; ++w) odd = odd || (x[w] & 0x7f800000u) == 0x7f800000u || (sizeof(X) == 2 && (x[w] & 0x7f80u) == 0x7f80u);
            if (!odd) continue;
#pragma unroll
            for (int e = 0; e < E::PER_CHUNK; ++e) {
                const int w = e * int(sizeof(X)) / 4;
                const bool low = sizeof(X) == 2 && (e & 1) == 0;
                const uint32_t bits = sizeof(X) == 4 ? x[w] : low ? x[w] << 16 : x[w] & 0xffff0000u, size = bits & 0x7fffffffu;
                if (size >= 0x7f800000u) {
                    f(r, col + e, size > 0x7f800000u || bits == size, size > 0x7f800000u || bits != size);
                    x[w] = sizeof(X) == 4 ? 0u : low ? x[w] & 0xffff0000u : x[w] & 0xffffu;
                }
            }
            *to = x;
        }
    }
};

// Reads of a tile by one lane, as left operands.
template <class E, int DT>
struct Reader {
    typedef attn::Tile<E, DT> T;
    int row, tr;                                                  // byte offsets of this lane in a tile
    __device__ __forceinline__ void init(int lane) {
        const int half = lane >> 5, r = lane & 31;
        row = r * T::PITCH + ((half ^ T::swizzle(r)) << 4);
        if (sizeof(typename E::T) == 2) {
            // transposed: inside 16 lanes, lane 4 k + c points at four columns of row k and lane i receives column i of rows 0..3
            const int k = ((lane & 15) >> 2) + 4 * half;
            tr = k * T::PITCH + (((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) ^ T::swizzle(k)) << 4) + (lane & 1) * 8;
        } else {
            tr = 4 * half * T::PITCH + ((((lane & 31) >> 2) ^ T::swizzle(4 * half)) << 4) + (lane & 3) * 4;
        }
    }
    // rows 32 block .. + 31, inner step s: chunk 2 s (lanes 0..31) and 2 s + 1
    __device__ __forceinline__ typename E::Row rows(const char* tile, int block, int s) const {
        return *reinterpret_cast<const typename E::Row*>(tile + block * 32 * T::PITCH + (row ^ (s << 5)));
    }
};

// Left operand of the sum over 16 rows from 16 step on: columns 32 n .. + 31 of the tile, transposed.
template <int DT>
__device__ __forceinline__ bf16x8 columns(const Reader<Bf16, DT>& rd, const char* tile, int step, int n) {
    typedef Tile<Bf16, DT> T;
    const char* a = tile + step * 16 * T::PITCH;
    constexpr int far = 2 << 4;                                   // swizzle(r + 8) = swizzle(r) ^ 2 for r < 8
    const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ONECOMP_LDS short4v*)(a + (rd.tr ^ (n << 6))));
    const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ONECOMP_LDS short4v*)(a + 8 * T::PITCH + (rd.tr ^ (n << 6) ^ far)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// acc[col][.] += sum over the 16 rows from 16 step of tile[row][32 n + m] p[row]: m is the accumulator's row, p the
// probabilities of these rows
template <int DT>
__device__ __forceinline__ float16v mma_t(const Reader<Bf16, DT>& rd, const char* tile, int step, int n, const Bf16::Score& p, float16v acc) {
    return Bf16::mma(columns<DT>(rd, tile, step, n), p, acc);
}
template <int DT>
__device__ __forceinline__ float16v mma_t(const Reader<F32, DT>& rd, const char* tile, int step, int n, const F32::Score& p, float16v acc) {
    typedef Tile<F32, DT> T;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = step * 16 + (i >> 2) * 8 + (i & 3);          // and r + 4 in lanes 32..63
        const int sw = T::swizzle(r) << 4;                         // swizzle(r + 4) = swizzle(r) ^ swizzle(4) for r % 8 < 4
        const float a = *reinterpret_cast<const float*>(tile + r * T::PITCH + (rd.tr ^ sw ^ (n << 7)));
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p.s[i], acc, 0, 0, 0);
    }
    return acc;
}

// ---- sequences ----------------------------------------------------------------------------------------------------------
struct Seq {
    int64_t q0, k0;        // first rows
    int nq, nk;            // lengths
    int room;              // rows of k that belong to the sequence, nk of them in use
    int shift;             // query i sees keys 0 .. i + shift (causal)
};

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// Rows from `first` on that belong to sequence i.  Behind the last sequence comes one of all rows that are left: padding,
// whose queries see no keys and whose keys no query sees.
__device__ __forceinline__ int rows_of(const int32_t* cu, int64_t total, int n_seqs, int i, int& first) {
    const int64_t at = clamp64(cu[i], 0, total);
    first = int(at);
    return int((i < n_seqs ? clamp64(cu[i + 1], at, total) : total) - at);
}

// Sums over the lanes up to each, and the largest of all lanes; in the vector pipe, with the last lane's value for the whole
// wave.  (Through LDS, as shuffles go, the search below took 3 us of each workgroup's start.)
__device__ __forceinline__ int scan_add(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
__device__ __forceinline__ int wave_add(int x) { return __builtin_amdgcn_readlane(scan_add(x), 63); }
__device__ __forceinline__ int wave_max(int x) {
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}

// What is counted: tiles of `size` queries, tiles of `size` keys with the room behind them, or pieces of work of few rows
// (blocks of 32 rows, of which every query has one per head of a group, times runs of keys).
enum What { QUERIES, KEYS, PIECES };

enum Found { NOTHING, IDLE, TILE };

// The t-th of all sequences: its sequence, its number x there and how many the sequence has; IDLE if there is no such tile but may be
// some behind it, NOTHING if there are none.  What the arrays say is cut to the tensors' rows.
//
// Sequences are counted, a lane each.  Of up to 63 the tiles come by their number x, the largest first and at the
// same x by sequence: x + 1 tiles of keys lie before a causal prompt's tile x, so that long work starts early and the last
// workgroups are short (gradients of 8 x 2048 keys: 540 us instead of 680 sequence by sequence).  Tiles of queries come
// sequence by sequence, each from its largest x down, where the last sequence cannot keep the others waiting: all are equally
// long, or the longest tile is an eighth of the work of each of 512 workgroups at most.  Then the tiles at work at a time share
// keys and values in the L2 (32 x 2048 tokens: 0.9 GB over the fabric instead of 2.8, 1.32 ms instead of 1.40).  More
// sequences come one after the other in any case: counting by number would read the arrays many times.
//
// Many sequences are not counted, which would make every workgroup read all of them before its own: slots are searched, 64 places
// at a time.  16384 prompts of 1 to 16 tokens, 8 / 2 heads of 64: 16.9 ms counted, 0.72 searched, their gradients 28 and 2.6, 500
// of 20 to 200 tokens 113 and 86 us, 128 of 100 to 500 65 and 67.  A few rows' slots stand for runs of keys that are not there too, so that
// counting pays for longer: 500 tokens 154 us counted and 247 searched, 1000 308 and 311, 4000 1500 and 175.
// Every lane of a wave takes part and gets the same answer.
template <What WHAT>
__device__ __forceinline__ Found find_tile(const Params& P, int size, int t, Seq& S, int& x, int& tiles) {
    const int lane = threadIdx.x & 63;
    if (__builtin_expect(P.n_seqs >= (WHAT == PIECES ? MANY_TOKENS : MANY), 0)) {
        const int32_t* cu = WHAT == KEYS ? P.cu_k : P.cu_q;
        const int64_t total = WHAT == KEYS ? P.total_k : P.total_q, rows = WHAT == PIECES ? P.group : 1;
        const int unit = WHAT == PIECES ? 32 : size, slot = WHAT == PIECES ? t / P.splits : t;
        if (slot >= all_slots(total * rows, unit, P.n_seqs)) return NOTHING;
        int lo = 0, hi = P.n_seqs + 1;                            // the last sequence whose slots begin at `slot` or before
        do {
            const int step = (hi - lo + 63) / 64, at = lo + lane * step;
            const unsigned long long before = __ballot(at < hi && first_slot(clamp64(cu[min(at, P.n_seqs)], 0, total) * rows, unit, at) <= slot);
            if (!before) return IDLE;                             // rows in front of the first sequence
            lo += (63 - __clzll((long long)before)) * step;
            hi = min(hi, lo + step);
        } while (hi - lo > 1);
        int q0, k0;
        const int nq = rows_of(P.cu_q, P.total_q, P.n_seqs, lo, q0), room = rows_of(P.cu_k, P.total_k, P.n_seqs, lo, k0);
        S.q0 = __builtin_amdgcn_readfirstlane(q0);
        S.k0 = __builtin_amdgcn_readfirstlane(k0);
        S.nq = __builtin_amdgcn_readfirstlane(nq);
        S.room = __builtin_amdgcn_readfirstlane(room);
        S.nk = lo == P.n_seqs ? 0 : P.len_k ? __builtin_amdgcn_readfirstlane(int(clamp64(P.len_k[lo], 0, room))) : S.room;
        S.shift = S.nk - S.nq;
        const int runs = WHAT == PIECES ? runs_of(P.run, P.splits, S.nk) : 1, split = WHAT == PIECES ? t % P.splits : 0;
        const int count = int((int64_t(WHAT == KEYS ? S.room : S.nq) * rows + unit - 1) / unit);
        const int64_t nth = slot - first_slot((WHAT == KEYS ? S.k0 : S.q0) * rows, unit, lo);
        if (nth < 0 || nth >= count || split >= runs) return IDLE;
        tiles = count * runs;
        x = (count - 1 - int(nth)) * runs + split;
        return TILE;
    }
    int done = 0;
    for (int base = 0; base <= P.n_seqs; base += 64) {
        int q0 = 0, k0 = 0, nq = 0, nk = 0, room = 0, count = 0;
        const int i = base + lane;
        if (i <= P.n_seqs) {
            nq = rows_of(P.cu_q, P.total_q, P.n_seqs, i, q0);
            room = rows_of(P.cu_k, P.total_k, P.n_seqs, i, k0);
            nk = i == P.n_seqs ? 0 : P.len_k ? int(clamp64(P.len_k[i], 0, room)) : room;
            if (WHAT == PIECES) count = int((int64_t(nq) * P.group + 31) / 32) * runs_of(P.run, P.splits, nk);
            else count = int((int64_t(WHAT == KEYS ? room : nq) + size - 1) / size);
        }
        int mine = count;                                         // tiles of this lane's sequence among those looked at
        bool by_number = false;
        if (P.n_seqs < 64) {
            const int hi0 = wave_max(count);
            by_number = true;
            if (WHAT == QUERIES && hi0 < 4096) {
                const bool even = __ballot(count != 0 && count != hi0) == 0;
                // work in tiles' worth of keys, for each of 512 workgroups at a time, against that of the longest
                const float work = float(wave_add(count * (count + 1) / 2)) * float(P.heads) * (1.f / 512.f);
                by_number = !(even || work >= 8.f * float(hi0));
            }
            if (by_number) {
                int lo = 0, hi = hi0;                             // lo: the largest x of which t + 1 tiles are at least x
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (wave_add(max(0, count - mid)) > t) lo = mid; else hi = mid;
                }
                done = wave_add(max(0, count - lo - 1));          // tiles with a larger number
                mine = count > lo ? 1 : 0;
                x = lo;
            }
        }
        const int upto = scan_add(mine);
        const unsigned long long past = __ballot(done + upto > t);
        if (past) {
            const int who = __ffsll(past) - 1;
            tiles = __builtin_amdgcn_readlane(count, who);
            if (!by_number) x = tiles - 1 - (t - done - __builtin_amdgcn_readlane(upto - mine, who));
            S.q0 = __builtin_amdgcn_readlane(q0, who);
            S.k0 = __builtin_amdgcn_readlane(k0, who);
            S.nq = __builtin_amdgcn_readlane(nq, who);
            S.nk = __builtin_amdgcn_readlane(nk, who);
            S.room = __builtin_amdgcn_readlane(room, who);
            S.shift = S.nk - S.nq;
            return x >= 0 && x < tiles ? TILE : NOTHING;          // sums of starts that make no sense may have wrapped
        }
        done += __builtin_amdgcn_readlane(upto, 63);
    }
    return NOTHING;
}

// Head of the i-th of `heads` workgroups that have the same rows.  Workgroups go round the eight XCDs one by one; the heads
// of a group, which read the same keys and values, come 8 apart where there are 8 groups, and so share an L2.
__device__ __forceinline__ int head_at(const Params& P, int i) { return (i % P.kv_heads) * P.group + i / P.kv_heads; }

template <class E>
__device__ __forceinline__ const char* at(const View& v, int64_t row, int head) {
    return reinterpret_cast<const char*>(v.p) + (row * v.token + int64_t(head) * v.head) * int64_t(sizeof(typename E::T));
}

// the other half's value of the same column
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }

__device__ __forceinline__ float16v zero16() {
    float16v z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}

// rows of an accumulator that a lane holds: row(r) = 8 (r / 4) + 4 half + r % 4
__device__ __forceinline__ int acc_row(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// acc (32 columns of the head dimension from 32 n, in rows; one token per lane) times f, to row[..] of a tensor, cut at dim
template <class E>
__device__ __forceinline__ void store_column(char* row, const float16v& acc, float f, int n, int dim, int half) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int d = 32 * n + 8 * g + 4 * half;
        if (d < dim) {
            if (sizeof(typename E::T) == 2) {
                short4v x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(short, static_cast<__bf16>(acc[4 * g + i] * f));
                *reinterpret_cast<short4v*>(row + d * 2) = x;
            } else {
                float4v x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = acc[4 * g + i] * f;
                *reinterpret_cast<float4v*>(row + d * 4) = x;
            }
        }
    }
}

// A token's row as right operands (lane: token l % 32)
template <class E, int DT>
struct Operand {
    static constexpr int STEPS = Tile<E, DT>::STEPS;
    typename E::Row x[STEPS];
    // straight from memory; zeros where the token is not there
    __device__ __forceinline__ void load(const char* row, bool there, int dim, int half) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            typename E::Row z;
#pragma unroll
            for (int i = 0; i < E::PER_CHUNK; ++i) z[i] = 0;
            x[s] = z;
            if (there && (2 * s + half) * E::PER_CHUNK < dim) x[s] = *reinterpret_cast<const typename E::Row*>(row + (2 * s + half) * 16);
        }
    }
};

// ---- rows of one wave through LDS -------------------------------------------------------------------------------------------
// The operands and results of a wave are 32 rows of which every lane holds 8 or 16 bytes here and there, rows that lie a
// token's stride apart in memory.  Through LDS they are read and written 16 lanes to a row, in whole cache lines.  (Straight
// from and to memory, 128 queries without any keys took 11 us; 32768 x 32 x 128 bf16 read and written: 175 us.)
// `tile`: LDS of 32 rows that this wave alone uses.
template <class E, int DT>
struct Rows {
    typedef attn::Tile<E, DT> T;
    static constexpr int BYTES = T::bytes(32);
    // begins to bring rows first .. first + valid - 1; they are there after a wait for the wave's loads
    static __device__ __forceinline__ void bring(uint32_t tile, const char* first, int valid, int64_t token_stride, int dim, int lane) {
        Loader<E, DT, 32, 1> l;
        l.init(0, lane, token_stride, dim);
        l.load(tile, first, valid, 0);
    }
    static __device__ __forceinline__ void take(Operand<E, DT>& x, const Reader<E, DT>& rd, const char* tile) {
#pragma unroll
        for (int s = 0; s < T::STEPS; ++s) x.x[s] = rd.rows(tile, 0, s);
    }
    // acc f (the lane's token in column, its entries in rows) to the rows whose bit is set in `which`
    static __device__ __forceinline__ void store(char* tile, const float16v (&acc)[DT], float f, char* first, int64_t token_stride, unsigned which, int dim,
                                                 int lane) {
        static_assert(sizeof(typename E::T) == 2, "bf16");
        const int half = lane >> 5, col = lane & 31;
        char* row = tile + col * T::PITCH + half * 8;
#pragma unroll
        for (int n = 0; n < DT; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                short4v x;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(short, static_cast<__bf16>(acc[n][4 * g + i] * f));
                *reinterpret_cast<short4v*>(row + (((4 * n + g) ^ T::swizzle(col)) << 4)) = x;
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // other lanes' entries are read next
        constexpr int ROWS = 64 / T::CHUNKS;                      // at a time
        const int chunk = lane % T::CHUNKS;
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) {
            const int r = i * ROWS + lane / T::CHUNKS;
            const uint4v x = *reinterpret_cast<const uint4v*>(tile + r * T::PITCH + ((chunk ^ T::swizzle(r)) << 4));
            if ((which >> r & 1) && chunk * 8 < dim) *reinterpret_cast<uint4v*>(first + int64_t(r) * token_stride * 2 + chunk * 16) = x;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
};

template <class E>
__device__ __forceinline__ void put(char* row, int d, float x) {
    if (sizeof(typename E::T) == 2) reinterpret_cast<__bf16*>(row)[d] = static_cast<__bf16>(x);
    else reinterpret_cast<float*>(row)[d] = x;
}

// ---- results that are not finite ------------------------------------------------------------------------------------------
// A score that a query must not see has probability 0, but 0 times a value that is infinite or no number is no number.  Tiles
// behind a sequence's end hold zeros, so this can only come from later tokens of the query's own prompt.  The kernels look at
// their sums once, when they have been stored, and where one is not finite its wave or workgroup takes its tiles once more, with zeros for
// what is not finite in them.  A query sees a prefix of the keys (a key is seen by a suffix of the queries), so the first (last) row of each
// column that is not finite says which results it reaches: their sums get it back at the end.  Nothing in the ordinary case, and
// one more pass where numbers have broken down, in simpler loops (2 to 7 times the clean call).

// true in the lanes whose column of the accumulators holds an entry that is not finite
template <int DT>
__device__ __forceinline__ bool not_finite(const float16v (&acc)[DT]) {
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < DT; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r & 3] = fmaf(acc[n][r], 0.f, x[r & 3]);
    x[0] = (x[0] + x[1]) + (x[2] + x[3]);
    return !(x[0] + other_half(x[0]) == 0.f);
}

// The lane again: what the second pass derives from it is formed there, not kept in registers through the first (kept, it spilled
// operands of the 128 wide bf16 gradients: 8 x 2048 tokens, forward and gradients 1340 us instead of 1285).
__device__ __forceinline__ int lane_anew() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// LDS of a workgroup for this: what its waves say, and rows: of two kinds in any column, and per column, of what raises and of what
// lowers a sum.
struct Marks {
    int said[8], any[2], column[256];
    __device__ __forceinline__ int& up(int c) { return column[c]; }
    __device__ __forceinline__ int& down(int c) { return column[128 + c]; }
};

// Whether any wave of the workgroup says so.  A barrier.
template <int WAVES>
__device__ __forceinline__ bool any_wave(Marks& marks, int wave, bool x) {
    const int mine = __any(x);
    if ((threadIdx.x & 63) == 0) marks.said[wave] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all |= marks.said[w];
    return __builtin_amdgcn_readfirstlane(all) != 0;
}

// All rows to `none`, by `threads` threads; what waits for them makes it known to others.
__device__ __forceinline__ void clear(Marks& marks, int none, int thread, int threads) {
    for (int i = thread; i < 256; i += threads) marks.column[i] = none;
    if (thread < 2) marks.any[thread] = none;
}

// One more row that is not finite: the first, or the last, stays.
__device__ __forceinline__ void mark_first(int& mark, int row) {
    if (row < mark) atomicMin(&mark, row);
}
__device__ __forceinline__ void mark_last(int& mark, int row) {
    if (row > mark) atomicMax(&mark, row);
}

// Column 32 n + .. of a result gets back what is not finite: reached(row) says whether the marked row reaches this lane's.
template <class F>
__device__ __forceinline__ void give_back(float16v& acc, Marks& marks, int n, int half, F reached) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int col = 32 * n + acc_row(r, half);
        acc[r] += (reached(marks.up(col)) ? -NEG_INF : 0.f) + (reached(marks.down(col)) ? NEG_INF : 0.f);
    }
}

size_t forward_workspace_bytes(onecomp_dtype dtype, const Params& P);
size_t backward_workspace_bytes(onecomp_dtype dtype, const Params& P);
onecomp_status forward_run(onecomp_dtype dtype, const Params& P, hipStream_t stream);
onecomp_status backward_run(onecomp_dtype dtype, const Params& P, hipStream_t stream);

}  // namespace attn
}  // namespace onecomp
