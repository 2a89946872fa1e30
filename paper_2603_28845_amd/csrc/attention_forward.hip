// Attention of packed sequences, forward: o_i = sum_j exp(s_ij - lse_i) v_j, s_ij = scale q_i . k_j.
#include "attention.hpp"
#include <cmath>

namespace onecomp {
namespace attn {
namespace {

// One pass over the keys of 32 queries (one per lane pair): the running maximum and sum of the softmax, and the weighted sum
// of the values, all fp32.
template <class E, int DT>
struct Rows32 {
    float16v o[DT];        // values' columns in rows, query in the lane
    float m, l;            // maximum (powers of two) and this half's part of the sum

    __device__ __forceinline__ void init() {
#pragma unroll
        for (int n = 0; n < DT; ++n) o[n] = zero16();
        m = NEG_INF;
        l = 0.f;
    }

    // Scores of KB blocks of 32 keys in LDS.
    template <int KB>
    static __device__ __forceinline__ void scores(float16v (&s)[KB], const Reader<E, DT>& rd, const char* kt, const Operand<E, DT>& q) {
#pragma unroll
        for (int b = 0; b < KB; ++b) s[b] = zero16();
#pragma unroll
        for (int i = 0; i < Tile<E, DT>::STEPS; ++i)
#pragma unroll
            for (int b = 0; b < KB; ++b) s[b] = E::mma(rd.rows(kt, b, i), q.x[i], s[b]);
    }

    // values() of one tile and scores() of the next in one stream of instructions, each product with its share of the
    // exponentials beside it and its operand read some products ahead:
    //   half of the next scores   | exponentials of the first 32 keys
    //   the other half, in turn with the products of these 32 | exponentials of the second 32
    //   products of the second 32 | maximum of the next scores, which it returns
    // The compiler on its own reads each operand right before its product and so waits for LDS every time.
    __device__ __forceinline__ float step(float16v (&s)[2], float16v (&next)[2], const Reader<E, DT>& rd, const char* kt, const char* vt,
                                          const Operand<E, DT>& q, float c) {
        static_assert(sizeof(typename E::T) == 2, "bf16");
        constexpr int N = 4 * DT, A = N / 2;                      // products of each kind, half of them
        constexpr int AHEAD = 4, AHEAD_V = A < 3 ? A : 3;         // operands read ahead
        const float base = m == NEG_INF ? 0.f : m;
        typename E::Row a[AHEAD], v[AHEAD_V];
        typename E::Score p[4];
        float add[4] = {l, 0.f, 0.f, 0.f}, top = NEG_INF;
        auto read_q = [&](int i) { if (i < N) a[i % AHEAD] = rd.rows(kt, i & 1, i >> 1); };
        auto read_v = [&](int i) { if (i < N) v[i % AHEAD_V] = columns<DT>(rd, vt, i / DT, i % DT); };
        auto score = [&](int i) {
            next[i & 1] = E::mma(a[i % AHEAD], q.x[i >> 1], i < 2 ? zero16() : next[i & 1]);
            read_q(i + AHEAD);
        };
        auto value = [&](int i) {
            o[i % DT] = E::mma(v[i % AHEAD_V], p[i / DT], o[i % DT]);
            read_v(i + AHEAD_V);
        };
        // exponentials of block b that belong to slot i of n
        auto exponentials = [&](int b, int i, int n) {
#pragma unroll
            for (int r = 16 * i / n; r < 16 * (i + 1) / n; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -base));
                add[r & 3] += s[b][r];
                asm volatile("" : "+v"(add[r & 3]));              // here, not where the sum is used: 32 registers less
                if (r % 8 == 7) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = s[b][r - 7 + e];
                    p[2 * b + r / 8] = E::pack(x);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) read_q(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < A; ++i) {
            score(i);
            if (i >= A - AHEAD_V) read_v(i - (A - AHEAD_V));
            exponentials(0, i, A);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < A; ++i) {
            score(A + i);
            exponentials(1, 2 * i, N);
            __builtin_amdgcn_sched_barrier(0);
            value(i);
            exponentials(1, 2 * i + 1, N);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < A; ++i) {
            value(A + i);
#pragma unroll
            for (int r = 32 * i / A; r < 32 * (i + 1) / A; ++r) top = fmaxf(top, next[r >> 4][r & 15]);
            asm volatile("" : "+v"(top));
            __builtin_amdgcn_sched_barrier(0);
        }
        l = (add[0] + add[1]) + (add[2] + add[3]);
        return top;
    }

    // Takes unseen keys out and returns the largest score of this half's keys.  last: the last key, counted from the tile's first,
    // that this lane's query sees.
    template <int KB>
    static __device__ __forceinline__ float mask(float16v (&s)[KB], int last, int half) {
        float top = NEG_INF;
        asm volatile("");                                         // a branch around this stays one: 64 selections per tile otherwise
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (32 * b + acc_row(r, half) > last) s[b][r] = NEG_INF;
                top = fmaxf(top, s[b][r]);
            }
        return top;
    }

    // Moves the maximum; top: the largest score of this half's keys.
    __device__ __forceinline__ void settle(float top, float c) {
        top = fmaxf(top, other_half(top)) * c;
        // The sums keep the maximum they began with until a score passes it by 2^8: the probabilities' rounding is relative
        // and their sum has room for that, and the many products with the new scale fall away.
        if (__any(top > m + 8.f)) {
            const float to = fmaxf(m, top), base = to == NEG_INF ? 0.f : to;
            const float f = __builtin_amdgcn_exp2f(m - base);
            l *= f;
#pragma unroll
            for (int n = 0; n < DT; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[n][r] *= f;
            m = to;
        }
    }

    // Probabilities and their sums with the values.
    template <int KB>
    __device__ __forceinline__ void values(float16v (&s)[KB], const Reader<E, DT>& rd, const char* vt, float c) {
        const float base = m == NEG_INF ? 0.f : m;
#pragma unroll
        for (int b = 0; b < KB; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -base));
            float add[4] = {s[b][0], s[b][1], s[b][2], s[b][3]};
#pragma unroll
            for (int r = 4; r < 16; ++r) add[r & 3] += s[b][r];
            l += (add[0] + add[1]) + (add[2] + add[3]);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float x[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) x[r] = s[b][8 * t + r];
                const typename E::Score p = E::pack(x);
#pragma unroll
                for (int n = 0; n < DT; ++n) o[n] = mma_t<DT>(rd, vt, 2 * b + t, n, p, o[n]);
            }
        }
    }
};

// ---- whole prompts ------------------------------------------------------------------------------------------------------
// LDS of the kernel below.
template <class E, int DT, int WAVES>
struct Whole {
    static constexpr int KB = sizeof(typename E::T) == 2 ? 2 : 1, SIZE = Tile<E, DT>::bytes(32 * KB);
    // two tiles of keys, two of values; bf16: behind them what the queries need besides the last; or a wave's own tiles of a second pass
    static constexpr int OWN = (2 * Tile<E, DT>::bytes(32) + int(sizeof(Marks)) + 1023) / 1024 * 1024, TILES = 3 * SIZE + (KB == 2 ? WAVES * Rows<E, DT>::BYTES : SIZE);
    static constexpr int LDS = TILES > WAVES * OWN ? TILES : WAVES * OWN;
};

// A workgroup has WAVES x 32 queries of one head and walks through the keys in tiles that all waves share.  Four waves, so that
// two workgroups share a CU and one's beginning or end lies beside the other's work (eight waves: 8 x 2048 tokens 384 us, four
// 361 when this was decided).  A wave's 32 queries use a quarter of its registers for the queries, a quarter for the sums of
// values and half for the scores of two tiles.  16384 tokens, 32 / 8 heads of 128: 1.89 to 1.96 ms, 1.1 PFLOP/s at 1.61 to 1.66 GHz
// (power), the matrix pipes busy 63 %; 32 x 2048: 1.19 to 1.25 ms, 47 %.  18 registers are spilled at 128 wide bf16, none of them in
// the loop.
template <class E, int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, sizeof(typename E::T) == 2 ? 2 : 1) void forward_kernel(const Params P) {
    constexpr int KB = sizeof(typename E::T) == 2 ? 2 : 1, KEYS = 32 * KB;
    typedef Tile<E, DT> T;
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = head_at(P, int(blockIdx.x) % P.heads);
    int tile, tiles;
    Seq S;
    if (find_tile<QUERIES>(P, WAVES * 32, int(blockIdx.x) / P.heads, S, tile, tiles) != TILE) return;
    const int first = tile * WAVES * 32, mine = first + wave * 32, query = mine + col;
    const bool there = query < S.nq;
    const int kv = head / P.group;

    // keys that any query of the workgroup, this wave, this lane sees: 0 .. end - 1
    const int last_q = min(first + WAVES * 32, S.nq) - 1, last_mine = min(mine + 31, S.nq - 1);
    const int end = P.causal ? max(0, min(S.nk, last_q + 1 + S.shift)) : S.nk;
    const int end_mine = mine >= S.nq ? 0 : P.causal ? max(0, min(S.nk, last_mine + 1 + S.shift)) : S.nk;
    const int end_all = P.causal ? min(S.nk, mine + 1 + S.shift) : S.nk;      // keys that every query of the wave sees
    const int last = P.causal ? min(S.nk - 1, query + S.shift) : S.nk - 1;

    constexpr bool STAGED = sizeof(typename E::T) == 2;           // rows of queries and of the output through LDS
    Operand<E, DT> q;
    if constexpr (!STAGED) q.load(at<E>(P.q, S.q0 + query, head), there, P.dim, half);

    Loader<E, DT, KEYS, WAVES> lk, lv;
    lk.init(wave, lane, P.k.token, P.dim);
    lv.init(wave, lane, P.v.token, P.dim);
    Reader<E, DT> rd;
    rd.init(lane);
    Rows32<E, DT> acc;
    acc.init();

    // Tile t's scores are formed while tile t - 1 goes through exponentials and values, so that a wave has products for the
    // matrix pipe and arithmetic for the vector pipe at the same time.  LDS: two tiles of keys, two of values.
    constexpr int SIZE = T::bytes(KEYS);
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((ONECOMP_LDS char*)lds));
    const int n = (end + KEYS - 1) / KEYS, n_mine = (end_mine + KEYS - 1) / KEYS;
    auto bring_k = [&](int t) {
        if (t < n) lk.load(base + uint32_t(t & 1) * SIZE, at<E>(P.k, S.k0 + t * KEYS, kv), end - t * KEYS, wave);
    };
    auto bring_v = [&](int t) {
        if (t < n) lv.load(base + uint32_t(2 + (t & 1)) * SIZE, at<E>(P.v, S.k0 + t * KEYS, kv), end - t * KEYS, wave);
    };
    auto next = [&](int t) {                                      // keys t + 1 and values t are there, keys t and values t - 1 done with
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
        __syncthreads();
        bring_k(t + 2);
        bring_v(t + 1);
    };
    auto step = [&](float16v(&s)[KB], float16v(&s_next)[KB], int t) {
        next(t);
        const char *kt = lds + ((t + 1) & 1) * SIZE, *vt = lds + (2 + (t & 1)) * SIZE;
        float top;
        if constexpr (KB == 2) {
            top = acc.step(s, s_next, rd, kt, vt, q, P.c);
            if ((t + 2) * KEYS > end_all) top = acc.mask(s_next, last - (t + 1) * KEYS, half);
        } else {
            acc.template scores<KB>(s_next, rd, kt, q);
            acc.template values<KB>(s, rd, vt, P.c);
            top = acc.mask(s_next, last - (t + 1) * KEYS, half);
        }
        acc.settle(top, P.c);
    };
    // queries go where the second tile of values will be, and behind it
    constexpr int AT_Q = 3 * SIZE;
    if constexpr (STAGED)
        Rows<E, DT>::bring(base + AT_Q + uint32_t(wave) * Rows<E, DT>::BYTES, at<E>(P.q, S.q0 + mine, head), S.nq - mine, P.q.token, P.dim, lane);
    bring_k(0);
    bring_v(0);
    bring_k(1);
    __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
    if constexpr (STAGED) {
        asm volatile("" ::: "memory");
        Rows<E, DT>::take(q, rd, lds + AT_Q + wave * Rows<E, DT>::BYTES);
    }
    __syncthreads();
    int t = 0;
    if (n_mine > 0) {
        float16v s0[KB], s1[KB];
        acc.template scores<KB>(s0, rd, lds, q);
        acc.settle(acc.mask(s0, last, half), P.c);
        for (; t + 2 < n_mine; t += 2) {
            step(s0, s1, t);
            step(s1, s0, t + 1);
        }
        if (t + 1 < n_mine) {
            step(s0, s1, t);
            next(t + 1);
            acc.template values<KB>(s1, rd, lds + (2 + ((t + 1) & 1)) * SIZE, P.c);
            t += 2;
        } else {
            next(t);
            acc.template values<KB>(s0, rd, lds + (2 + (t & 1)) * SIZE, P.c);
            t += 1;
        }
    }
    for (; t < n; ++t) next(t);
    constexpr int OWN = Whole<E, DT, WAVES>::OWN;
    // lane, query: as the kernel's own; true where the sums are to be looked at
    auto finish = [&](int lane, int query) {
        const int half = lane >> 5;
        const bool there = query < S.nq;
        const float l = acc.l + other_half(acc.l), f = l == 0.f ? 0.f : 1.f / l;
        if constexpr (STAGED) {
            Rows<E, DT>::store(lds + wave * OWN, acc.o, f, const_cast<char*>(at<E>(P.o, S.q0 + mine, head)), P.o.token, unsigned(__ballot(there)), P.dim, lane);
        } else if (there) {
            char* row = const_cast<char*>(at<E>(P.o, S.q0 + query, head));
#pragma unroll
            for (int n = 0; n < DT; ++n) store_column<E>(row, acc.o[n], f, n, P.dim, half);
        }
        if (there && P.lse && half == 0)
            P.lse[int64_t(head) * P.total_q + S.q0 + query] = l == 0.f ? NEG_INF : (acc.m + __builtin_amdgcn_logf(l)) * LN2;
        return there && l == l;
    };
    const bool look = P.causal && not_finite(acc.o);
    __syncthreads();                                              // every wave is done with the tiles
    if (__builtin_expect(!__any(finish(lane, query) && look), 1)) return;

    // Once more, each wave by itself.
    const int lane_2 = lane_anew(), half_2 = lane_2 >> 5, query_2 = mine + (lane_2 & 31), last_2 = min(S.nk - 1, query_2 + S.shift);
    char* own = lds + wave * OWN;
    const uint32_t own_base = base + uint32_t(wave) * OWN;
    constexpr int TILE = T::bytes(32);
    Marks& marks = *reinterpret_cast<Marks*>(own + 2 * TILE);
    clear(marks, S.nk, lane_2, 64);
    Loader<E, DT, 32, 1> keys, values;
    keys.init(0, lane_2, P.k.token, P.dim);
    values.init(0, lane_2, P.v.token, P.dim);
    Reader<E, DT> rd_2;
    rd_2.init(lane_2);
    q.load(at<E>(P.q, S.q0 + query_2, head), query_2 < S.nq, P.dim, half_2);
    acc.init();
    auto bring_2 = [&](const Loader<E, DT, 32, 1>& rows, uint32_t to, const View& from, int j) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // the last tile is read
        if (j < end_mine) rows.load(to, at<E>(from, S.k0 + j, kv), end_mine - j, 0);
    };
    bring_2(keys, own_base, P.k, 0);
    bring_2(values, own_base + TILE, P.v, 0);
    for (int j = 0; j < end_mine; j += 32) {
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
        asm volatile("" ::: "memory");
        float16v s[1];
        acc.template scores<1>(s, rd_2, own, q);
        bring_2(keys, own_base, P.k, j + 32);
        acc.settle(acc.mask(s, last_2 - j, half_2), P.c);
        values.clean(own + TILE, 0, lane_2, [&](int r, int c, bool up, bool down) {
            if (up) mark_first(marks.up(c), j + r);
            if (down) mark_first(marks.down(c), j + r);
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        acc.template values<1>(s, rd_2, own + TILE, P.c);
        bring_2(values, own_base + TILE, P.v, j + 32);
    }
#pragma unroll
    for (int n = 0; n < DT; ++n) give_back(acc.o[n], marks, n, half_2, [&](int row) { return row <= last_2; });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    finish(lane_2, query_2);
}

// ---- few rows -----------------------------------------------------------------------------------------------------------
// One or a few new tokens per sequence: the rows of a group's heads lie side by side in the 32 columns (row = query x group +
// head), so that keys and values are read once for all of them, and the keys are the work that is shared out: a workgroup has
// a run of them, its waves take tiles of 32 in turn, each through LDS of its own.  The products are no bound here; bytes in
// flight are, one tile of each wave at a time, and what a workgroup takes to begin and end.
template <class E, int DT>
struct Few {
    typedef attn::Tile<E, DT> T;
    static constexpr int SIZE = T::bytes(32);
    // two tiles of keys and of values per wave; 64 KB, so that one workgroup begins or ends beside another's work
    static constexpr int WAVES = SIZE >= 16 * 1024 ? 1 : SIZE >= 8 * 1024 ? 2 : 4;
    static constexpr int TILES = 4 * SIZE * WAVES, LDS = TILES + int(sizeof(Marks));
    static constexpr int COLS = 32 * DT;                               // of a partial sum's row
    static_assert(TILES >= WAVES * DT * 4096 + WAVES * 256, "the waves' sums meet in the same memory");
};

// Scratch: runs of each row [rows], maximum and sum of each run [splits, rows, 2], its sums of values [splits, rows, COLS].
struct Parts {
    int32_t* runs;
    float *tops, *sums;
    __device__ __forceinline__ Parts(const Params& P) {
        const int64_t rows = int64_t(P.heads) * P.total_q;
        runs = reinterpret_cast<int32_t*>(P.part);
        tops = P.part + (rows + 63) / 64 * 64;
        sums = tops + 2 * P.splits * rows;
    }
};

template <class E, int DT>
__global__ __launch_bounds__((Few<E, DT>::WAVES * 64), 1) void few_rows_kernel(const Params P) {
    typedef Few<E, DT> F;
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Parts parts(P);
    Marks& marks = *reinterpret_cast<Marks*>(lds + F::TILES);
    // pieces of work in turn, whatever number of workgroups the host thought enough
    for (int piece = blockIdx.x;; piece += gridDim.x) {
    const int kv = piece % P.kv_heads;
    int x, pieces;
    Seq S;
    const Found found = find_tile<PIECES>(P, 0, piece / P.kv_heads, S, x, pieces);
    if (found == NOTHING) return;
    if (found == IDLE) continue;
    const int run = run_of(P.run, P.splits, S.nk), runs = runs_of(P.run, P.splits, S.nk), tile = x / runs, split = x % runs;
    const int row = tile * 32 + col, query = row / P.group, head = kv * P.group + row % P.group;
    const bool there = query < S.nq;
    const int last_q = min((tile * 32 + 31) / P.group, S.nq - 1), first_q = tile * 32 / P.group;
    const int seen = P.causal ? max(0, min(S.nk, last_q + 1 + S.shift)) : S.nk;
    const Range keys = run_range(run, split, seen);
    const int begin = keys.begin, end = keys.end;
    const int end_all = P.causal ? min(S.nk, first_q + 1 + S.shift) : S.nk;
    const int last = P.causal ? min(S.nk - 1, query + S.shift) : S.nk - 1;

    // again: once more, with zeros for values that are not finite
    for (bool again = false;; again = true) {
    Rows32<E, DT> acc;
    acc.init();
    if (begin < end) {
        Operand<E, DT> q;
        q.load(at<E>(P.q, S.q0 + query, head), there, P.dim, half);
        Loader<E, DT, 32, 1> lk, lv;
        lk.init(0, lane, P.k.token, P.dim);
        lv.init(0, lane, P.v.token, P.dim);
        Reader<E, DT> rd;
        rd.init(lane);
        char* own = lds + wave * 4 * F::SIZE;
        const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((ONECOMP_LDS char*)lds)) + uint32_t(wave) * 4 * F::SIZE;
        auto bring = [&](int j, int buf) {
            lk.load(base + uint32_t(buf) * 2 * F::SIZE, at<E>(P.k, S.k0 + j, kv), end - j, 0);
            lv.load(base + uint32_t(buf) * 2 * F::SIZE + F::SIZE, at<E>(P.v, S.k0 + j, kv), end - j, 0);
        };
        constexpr int STEP = 32 * F::WAVES, LOADS = 2 * Loader<E, DT, 32, 1>::LOADS;
        int j = begin + wave * 32, buf = 0;
        if (j < end) bring(j, 0);
        for (; j < end; j += STEP, buf ^= 1) {
            // the other tile is free: this wave has read it into registers, and no other reads it
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (j + STEP < end) {
                bring(j + STEP, buf ^ 1);
                __builtin_amdgcn_s_waitcnt(wait_vmcnt(LOADS));
            } else {
                __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
            }
            asm volatile("" ::: "memory");
            if (__builtin_expect(again, 0)) {
                lv.clean(own + buf * 2 * F::SIZE + F::SIZE, 0, lane, [&](int r, int c, bool up, bool down) {
                    if (up) mark_first(marks.up(c), j + r);
                    if (down) mark_first(marks.down(c), j + r);
                });
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            float16v s[1];
            acc.template scores<1>(s, rd, own + buf * 2 * F::SIZE, q);
            acc.settle(acc.mask(s, last - j, half), P.c);
            acc.template values<1>(s, rd, own + buf * 2 * F::SIZE + F::SIZE, P.c);
        }
    }

    // the waves' sums meet: their maxima and sums, then 32 columns of the values by each wave
    float l = acc.l + other_half(acc.l);
    __syncthreads();
    float* sums = reinterpret_cast<float*>(lds);
    float* tops = sums + F::WAVES * DT * 1024;
    if (half == 0) {
        tops[wave * 64 + col] = acc.m;
        tops[wave * 64 + 32 + col] = l;
    }
#pragma unroll
    for (int n = 0; n < DT; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) sums[((wave * DT + n) * 16 + r) * 64 + lane] = acc.o[n][r];
    __syncthreads();
    float top = NEG_INF, f[F::WAVES];
#pragma unroll
    for (int w = 0; w < F::WAVES; ++w) top = fmaxf(top, tops[w * 64 + col]);
    const float zero = top == NEG_INF ? 0.f : top;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < F::WAVES; ++w) {
        const float m = tops[w * 64 + col];
        f[w] = __builtin_amdgcn_exp2f(m - zero);
        l = fmaf(f[w], tops[w * 64 + 32 + col], l);
    }
    const int64_t at_row = int64_t(head) * P.total_q + S.q0 + query, rows = int64_t(P.heads) * P.total_q;
    const bool whole = P.splits == 1;
    const float out = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    bool broken = false;
    for (int n = wave; n < DT; n += F::WAVES) {
        float16v o = zero16();
#pragma unroll
        for (int w = 0; w < F::WAVES; ++w)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[r] = fmaf(f[w], sums[((w * DT + n) * 16 + r) * 64 + lane], o[r]);
        if (__builtin_expect(again, 0)) give_back(o, marks, n, half, [&](int key) { return key <= last; });
        float16v one[1] = {o};
        broken = broken || (there && l == l && not_finite(one));
        if (there) {
            if (whole) {
                store_column<E>(const_cast<char*>(at<E>(P.o, S.q0 + query, head)), o, out, n, P.dim, half);
            } else {
                char* to = reinterpret_cast<char*>(parts.sums + (split * rows + at_row) * F::COLS);
                store_column<F32>(to, o, 1.f, n, F::COLS, half);
            }
        }
    }
    if (there && wave == 0 && half == 0) {
        if (!whole) {
            if (split == 0) parts.runs[at_row] = runs;
            parts.tops[2 * (split * rows + at_row)] = top;
            parts.tops[2 * (split * rows + at_row) + 1] = l;
        } else if (P.lse) {
            P.lse[at_row] = l == 0.f ? NEG_INF : (top + __builtin_amdgcn_logf(l)) * LN2;
        }
    }
    // a barrier in either case: the next tiles go where the sums met.  Only keys that some rows do not see can do harm.
    if (again || end <= end_all) {
        __syncthreads();
        break;
    }
    if (__builtin_expect(!any_wave<F::WAVES>(marks, wave, broken), 1)) break;
    clear(marks, S.nk, threadIdx.x, F::WAVES * 64);
    __syncthreads();
    }
    }
}

// The runs' sums of one row meet, in their order: one wave per row, a lane per two columns.
template <class E, int DT>
__global__ __launch_bounds__(256) void join_kernel(const Params P) {
    constexpr int COLS = 32 * DT;
    const int lane = threadIdx.x & 63;
    const int64_t rows = int64_t(P.heads) * P.total_q, row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int head = int(row / P.total_q);
    const int64_t token = row - int64_t(head) * P.total_q;
    const Parts parts(P);
    const int runs = min(parts.runs[row], P.splits);
    float top = NEG_INF;
    for (int s = lane; s < runs; s += 64) top = fmaxf(top, parts.tops[2 * (s * rows + row)]);
    top = onecomp::wave_max(top);
    const float zero = top == NEG_INF ? 0.f : top;
    float l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 4
    for (int s = 0; s < runs; ++s) {
        const float m = parts.tops[2 * (s * rows + row)], n = parts.tops[2 * (s * rows + row) + 1];
        const float* from = parts.sums + (s * rows + row) * COLS;
        // a run behind the row's keys has no sums, only n = 0
        const float x0 = lane < COLS ? from[lane] : 0.f, x1 = DT > 2 && lane + 64 < COLS ? from[lane + 64] : 0.f;
        if (n == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(m - zero);
        l = fmaf(f, n, l);
        o0 = fmaf(f, x0, o0);
        o1 = fmaf(f, x1, o1);
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    char* to = const_cast<char*>(at<E>(P.o, token, head));
    if (lane < P.dim) put<E>(to, lane, o0 * f);
    if (lane + 64 < P.dim) put<E>(to, lane + 64, o1 * f);
    if (P.lse && lane == 0) P.lse[row] = l == 0.f ? NEG_INF : (top + __builtin_amdgcn_logf(l)) * LN2;
}

template <class E, int DT, int WAVES>
onecomp_status launch_forward(const Params& P, hipStream_t stream) {
    constexpr int LDS = Whole<E, DT, WAVES>::LDS;
    static std::atomic<uint64_t> done{0};
    const onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(forward_kernel<E, DT, WAVES>), LDS, done);
    if (st != ONECOMP_OK) return st;
    const int64_t tiles = P.total_q / (WAVES * 32) + P.n_seqs + 1;    // no less than the sequences' tiles together
    const int64_t grid = tiles * P.heads;
    if (grid > 0x7fffffff) return ONECOMP_ERR_UNSUPPORTED;
    forward_kernel<E, DT, WAVES><<<dim3(unsigned(grid)), dim3(WAVES * 64), LDS, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

// blocks of 32 rows (a group's heads of a query) for each head of keys, about
int64_t row_blocks(const Params& P) {
    const int64_t most = ceil_div(P.total_q * P.group, 32) + P.n_seqs, even = ceil_div(P.max_q * P.group, 32) * P.n_seqs;
    return most < even || even < 1 ? most : even;
}

template <class E, int DT>
onecomp_status launch_few(const Params& P, hipStream_t stream) {
    typedef Few<E, DT> F;
    static std::atomic<uint64_t> done{0};
    const onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(few_rows_kernel<E, DT>), F::LDS, done);
    if (st != ONECOMP_OK) return st;
    const int64_t rows = P.total_q * P.heads;
    int64_t grid = row_blocks(P) * (P.splits > 1 ? ceil_div(P.total_k, int64_t(P.run) * (P.n_seqs < 1 ? 1 : P.n_seqs)) + 1 : 1) * P.kv_heads;
    if (P.n_seqs >= MANY_TOKENS) grid = all_slots(P.total_q * P.group, 32, P.n_seqs) * P.splits * P.kv_heads;
    if (grid > 0x7fffffff - 16384) return ONECOMP_ERR_UNSUPPORTED;    // pieces are counted in 32 bits
    grid = grid > 16384 ? 16384 : grid;                           // workgroups go on to further pieces
    few_rows_kernel<E, DT><<<dim3(unsigned(grid)), dim3(F::WAVES * 64), F::LDS, stream>>>(P);
    ONECOMP_CHECK_LAUNCH();
    if (P.splits > 1) {
        join_kernel<E, DT><<<dim3(unsigned((rows + 3) / 4)), dim3(256), 0, stream>>>(P);
        ONECOMP_CHECK_LAUNCH();
    }
    return ONECOMP_OK;
}

// How the keys are shared out where there are few rows; splits = 0: whole prompts.  Estimates in microseconds from
// measurements at 128 wide bf16 heads: 0.8 for 64 keys of a prompt's tile of 128 rows, two of them at a time on each CU, and
// 0.8 for 32 keys of a block of 32 rows, four on each CU, with 12 to begin, end and join.  fp32, up to 64 wide and wider: 4 and 8
// for a prompt's 64 keys, 2.5 and 8 for a block's 32 (blocks wider than 64 get two waves on a CU).  With 1 to 512 new tokens behind
// 1 x 16384, 8 x 4096 and 32 x 1024 keys, both types, 64 and 128 wide, the shape chosen is the better one, by 5 to 30 % at 16 tokens
// and 1.7 to 9 times from 64 on (512 tokens behind 16384 keys, bf16, 128 wide: 251 us whole and 1510 in blocks of 32 rows), but for
// 16 tokens of bf16 behind 16384 keys, where other runs of the same kernel take 30 and 47 us instead of 36 and 51.
void plan(onecomp_dtype dtype, Params& P) {
    P.splits = P.run = 0;
    const double tiles = double(P.heads) * (double(P.total_q) / 128 + P.n_seqs), blocks = double(row_blocks(P)) * P.kv_heads;
    const bool f32 = dtype == ONECOMP_F32, wide = P.dim > 64;
    const double prompt = ceil(tiles / 512) * (double(P.max_k) / 64) * (!f32 ? 0.8 : wide ? 8 : 4) + 5;
    const double few = ceil(blocks * (double(P.max_k) / 32) / 1024) * (!f32 ? 0.8 : wide ? 8 : 2.5) + 12;
    if (P.max_q * P.group > 32 && few > prompt) return;
    // four pieces of work for each CU, none shorter than 256 keys: 32 requests of 100 to 16384 keys 100 us, with half as many again
    // 106, with 768 in all 105
    const double each = double(P.total_k) / (P.n_seqs < 1 ? 1 : P.n_seqs);
    double run = ceil(blocks * each / 1024 / 128) * 128;
    run = run < 256 ? 256 : run > (1 << 30) ? (1 << 30) : run;
    const int64_t splits = ceil_div(P.max_k, int64_t(run));
    const int most = most_splits(P.n_seqs);
    P.splits = int(splits < 1 ? 1 : splits > most ? most : splits);
    P.run = int(run);
}

template <class E, int DT>
onecomp_status forward(const Params& P, hipStream_t stream) {
    return P.splits ? launch_few<E, DT>(P, stream) : launch_forward<E, DT, 4>(P, stream);
}

}  // namespace

size_t forward_workspace_bytes(onecomp_dtype dtype, const Params& in) {
    Params P = in;
    plan(dtype, P);
    if (P.splits < 2) return 0;
    const size_t cols = size_t(P.dim + 31) / 32 * 32;
    const size_t rows = size_t(P.total_q) * P.heads;
    return align_up((align_up(rows, 64) + P.splits * rows * (2 + cols)) * 4, 256);
}

onecomp_status forward_run(onecomp_dtype dtype, const Params& in, hipStream_t stream) {
    Params P = in;
    plan(dtype, P);
    const int dt = (P.dim + 31) / 32;
    if (dtype == ONECOMP_BF16)
        return dt == 1 ? forward<Bf16, 1>(P, stream) : dt == 2 ? forward<Bf16, 2>(P, stream) : dt == 3 ? forward<Bf16, 3>(P, stream) : forward<Bf16, 4>(P, stream);
    return dt == 1 ? forward<F32, 1>(P, stream) : dt == 2 ? forward<F32, 2>(P, stream) : dt == 3 ? forward<F32, 3>(P, stream) : forward<F32, 4>(P, stream);
}

}  // namespace attn
}  // namespace onecomp
