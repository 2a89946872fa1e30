// Gradients of the attention of packed sequences, in two kernels: one with the queries in lanes (dq, and the per-query numbers
// that both need), one with the keys in lanes (dk and dv).  Each forms the scores and the probabilities' gradients anew, seven
// products where the definition has five, and in return no sum of one workgroup depends on another's and none needs atomics.  Calls
// of too few workgroups share out their inner loops (plan()): the shares' sums of dq, dk and dv, 32 bits each, go to the
// workspace and are joined there in their order.
#include "attention.hpp"

namespace onecomp {
namespace attn {
namespace {

template <class E>
constexpr int KB = sizeof(typename E::T) == 2 ? 2 : 1;            // blocks of 32 rows in a tile

// Scores of unseen keys to -inf: their probabilities are 0.
__device__ __forceinline__ void mask(float16v& s, int last, int half) {
    asm volatile("");                                             // a branch around this stays one
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (acc_row(r, half) > last) s[r] = NEG_INF;
}

// A tile of 64 keys in one stream of instructions, products with their share of the arithmetic beside them and their operands
// read from LDS some products ahead:
//   scores and the probabilities' gradients of the first 32 keys
//   the same of the second 32        | arithmetic of the first
//   the first's products with k      | arithmetic of the second
//   the second's products with k
template <int DT>
__device__ __forceinline__ void grad_q_tile(float16v (&dq)[DT], const Reader<Bf16, DT>& rd, const char* kt, const char* vt, const Operand<Bf16, DT>& q,
                                            const Operand<Bf16, DT>& d, float c, float lse, float delta, bool all_seen, int last, int half) {
    typedef Bf16 E;
    constexpr int N = 4 * DT, AHEAD = 4, AHEAD_C = 3;             // products of one block with q and with d_out
    float16v s[2], dp[2];
    E::Row a[AHEAD], k[AHEAD_C];
    E::Score ds[4];
    auto read = [&](int i) {
        if (i < 2 * N) a[i % AHEAD] = rd.rows(i & 1 ? vt : kt, i / N, (i % N) >> 1);
    };
    auto product = [&](int i) {
        const int b = i / N, x = (i % N) >> 1;
        if (i & 1) dp[b] = E::mma(a[i % AHEAD], d.x[x], x ? dp[b] : zero16());
        else s[b] = E::mma(a[i % AHEAD], q.x[x], x ? s[b] : zero16());
        read(i + AHEAD);
    };
    auto read_k = [&](int i) {
        if (i < N) k[i % AHEAD_C] = columns<DT>(rd, kt, i / DT, i % DT);
    };
    auto arithmetic = [&](int b, int i, int n) {                  // entries of block b that belong to slot i of n
#pragma unroll
        for (int r = 16 * i / n; r < 16 * (i + 1) / n; ++r) {
            s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -lse)) * (dp[b][r] - delta);
            asm volatile("" : "+v"(s[b][r]));                     // here, not where the products need it
            if (r % 8 == 7) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = s[b][r - 7 + e];
                ds[2 * b + r / 8] = E::pack(x);
            }
        }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        product(i);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (!all_seen) mask(s[0], last, half);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        product(N + i);
        if (i >= N - AHEAD_C) read_k(i - (N - AHEAD_C));
        arithmetic(0, i, N);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (!all_seen) mask(s[1], last - 32, half);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        dq[i % DT] = E::mma(k[i % AHEAD_C], ds[i / DT], dq[i % DT]);
        read_k(i + AHEAD_C);
        if (i < N / 2) arithmetic(1, i, N / 2);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The same of 32 keys, one part after the other.
template <class E, int DT>
__device__ __forceinline__ void grad_q_block(float16v (&dq)[DT], const Reader<E, DT>& rd, const char* kt, const char* vt, const Operand<E, DT>& q,
                                             const Operand<E, DT>& d, float c, float lse, float delta, bool all_seen, int last, int half) {
    typedef Tile<E, DT> T;
    float16v s = zero16(), dp = zero16();
#pragma unroll
    for (int x = 0; x < T::STEPS; ++x) s = E::mma(rd.rows(kt, 0, x), q.x[x], s);
#pragma unroll
    for (int x = 0; x < T::STEPS; ++x) dp = E::mma(rd.rows(vt, 0, x), d.x[x], dp);
    if (!all_seen) mask(s, last, half);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse)) * (dp[r] - delta);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float x[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) x[r] = s[8 * t + r];
        const typename E::Score ds = E::pack(x);
#pragma unroll
        for (int n = 0; n < DT; ++n) dq[n] = mma_t<DT>(rd, kt, t, n, ds, dq[n]);
    }
}

// dq_i = scale sum_j ds_ij k_j for WAVES x 32 queries of one head.  Also leaves in scratch what the other kernel's sums of
// products begin with: -lse / scale for the scores and -delta_i = -d_out_i . out_i for the probabilities' gradients.  Three products
// a tile: 8 x 2048 tokens, 32 / 8 heads of 128, 435 to 475 us, 0.87 to 0.95 PFLOP/s executed, matrix pipes busy 49 %; 12 registers spilled, none
// in the loop.
template <class E, int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, sizeof(typename E::T) == 2 ? 2 : 1) void grad_q_kernel(const Params P) {
    constexpr int KEYS = 32 * KB<E>;
    typedef Tile<E, DT> T;
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = head_at(P, int(blockIdx.x) % P.heads), kv = head / P.group;
    int tile, tiles;
    Seq S;
    if (find_tile<QUERIES>(P, WAVES * 32, int(blockIdx.x) / P.heads, S, tile, tiles) != TILE) return;
    const int first = tile * WAVES * 32, mine = first + wave * 32, query = mine + col;
    const bool there = query < S.nq;
    const int last_q = min(first + WAVES * 32, S.nq) - 1, last_mine = min(mine + 31, S.nq - 1);
    const int end = P.causal ? max(0, min(S.nk, last_q + 1 + S.shift)) : S.nk;
    const int end_mine = mine >= S.nq ? 0 : P.causal ? max(0, min(S.nk, last_mine + 1 + S.shift)) : S.nk;
    const int end_all = P.causal ? min(S.nk, mine + 1 + S.shift) : S.nk;
    const int last = P.causal ? min(S.nk - 1, query + S.shift) : S.nk - 1;
    // this workgroup's share of them, where the keys are split
    const Range share = share_of(end, KEYS, P.splits_q, int(blockIdx.y));
    const int from = share.begin, to = share.end;

    Loader<E, DT, KEYS, WAVES> lk, lv;
    lk.init(wave, lane, P.k.token, P.dim);
    lv.init(wave, lane, P.v.token, P.dim);
    constexpr int SIZE = T::bytes(KEYS);
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((ONECOMP_LDS char*)lds));
    auto bring = [&](int j, int buf) {
        lk.load(base + uint32_t(buf) * 2 * SIZE, at<E>(P.k, S.k0 + j, kv), end - j, wave);
        lv.load(base + uint32_t(buf) * 2 * SIZE + SIZE, at<E>(P.v, S.k0 + j, kv), end - j, wave);
    };
    constexpr bool STAGED = sizeof(typename E::T) == 2;           // rows through LDS
    const bool own_delta = STAGED && end <= 256;
    Reader<E, DT> rd;
    rd.init(lane);
    Operand<E, DT> q, d;
    typedef Rows<E, DT> R;
    static_assert(!STAGED || WAVES * R::BYTES == 2 * SIZE, "the waves' rows fill one pair of tiles");
    const int mine_at = wave * (STAGED ? R::BYTES : 0);
    if constexpr (STAGED) {
        R::bring(base + mine_at, at<E>(P.q, S.q0 + mine, head), S.nq - mine, P.q.token, P.dim, lane);
        R::bring(base + 2 * SIZE + mine_at, at<E>(P.d_o, S.q0 + mine, head), S.nq - mine, P.d_o.token, P.dim, lane);
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
        asm volatile("" ::: "memory");
        R::take(q, rd, lds + mine_at);
        R::take(d, rd, lds + 2 * SIZE + mine_at);
        __syncthreads();
        // outputs, for delta, where the second tiles of keys and values will be
        if (!own_delta) R::bring(base + 2 * SIZE + mine_at, at<E>(P.o, S.q0 + mine, head), S.nq - mine, P.o.token, P.dim, lane);
    } else {
        q.load(at<E>(P.q, S.q0 + query, head), there, P.dim, half);
        d.load(at<E>(P.d_o, S.q0 + query, head), there, P.dim, half);
    }
    if (own_delta ? end > 0 : from < to) bring(own_delta ? 0 : from, 0);
    const int64_t at_q = int64_t(head) * P.total_q + S.q0 + query;
    float delta = 0.f, lse = there ? P.lse[at_q] * LOG2E : 0.f;
    if (lse == NEG_INF) lse = -NEG_INF;                           // a query that sees nothing: all its probabilities are 0
    // delta from the output that was stored: with a few keys in a row its rounding to bf16 weighs as much as all others of the
    // gradient together (short sequences: dq and dk 2.0 times as far off as a single rounding, 1.4 times otherwise).  Where a
    // workgroup's rows see up to 256 keys, delta_i = sum_j p_ij (d_out_i . v_j) is added up in a pass of its own: one tile in
    // 36 of a causal prompt of 2048.
    if (own_delta) {
        for (int j = 0, buf = 0; j < end; j += KEYS, buf ^= 1) {
            __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
            __syncthreads();
            if (j + KEYS < end) bring(j + KEYS, buf ^ 1);
            if (j >= end_mine) continue;
#pragma unroll 1
            for (int b = 0; b < KB<E>; ++b) {
                const char *kt = lds + buf * 2 * SIZE + b * 32 * T::PITCH, *vt = kt + SIZE;
                float16v s = zero16(), dp = zero16();
#pragma unroll
                for (int x = 0; x < T::STEPS; ++x) {
                    s = E::mma(rd.rows(kt, 0, x), q.x[x], s);
                    dp = E::mma(rd.rows(vt, 0, x), d.x[x], dp);
                }
                if (j + KEYS > end_all) mask(s, last - j - 32 * b, half);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[r], P.c, -lse));
                    delta += p == 0.f ? 0.f : p * dp[r];          // values that are not seen may be no numbers
                }
            }
        }
        __syncthreads();
        if (from < to) bring(from, 0);
    } else {
        Operand<E, DT> o;
        if constexpr (STAGED) {
            __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
            asm volatile("" ::: "memory");
            R::take(o, rd, lds + 2 * SIZE + mine_at);
        } else {
            o.load(at<E>(P.o, S.q0 + query, head), there, P.dim, half);
        }
#pragma unroll
        for (int s = 0; s < T::STEPS; ++s)
#pragma unroll
            for (int e = 0; e < E::PER_CHUNK; ++e) delta = fmaf(float(o.x[s][e]), float(d.x[s][e]), delta);
    }
    delta += other_half(delta);
    if (there && half == 0 && blockIdx.y == 0) {
        P.aux[at_q] = -lse / P.c;
        P.aux[int64_t(P.heads) * P.total_q + at_q] = -delta;
    }
    float16v dq[DT];
#pragma unroll
    for (int n = 0; n < DT; ++n) dq[n] = zero16();

    for (int j = from, buf = 0; j < to; j += KEYS, buf ^= 1) {
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
        __syncthreads();
        if (j + KEYS < to) bring(j + KEYS, buf ^ 1);
        if (j >= end_mine) continue;
        const char *kt = lds + buf * 2 * SIZE, *vt = kt + SIZE;
        const bool all_seen = j + KEYS <= end_all;
        if constexpr (KB<E> == 2) {
            grad_q_tile<DT>(dq, rd, kt, vt, q, d, P.c, lse, delta, all_seen, last - j, half);
        } else {
            grad_q_block<E, DT>(dq, rd, kt, vt, q, d, P.c, lse, delta, all_seen, last - j, half);
        }
    }
    const int64_t rows_q = int64_t(P.heads) * P.total_q;
    float* part = P.part + int64_t(blockIdx.y) * rows_q * (32 * DT);
    // lane, query: as the kernel's own
    auto finish = [&](int lane, int query) {
        const int half = lane >> 5;
        const int64_t at_q = int64_t(head) * P.total_q + S.q0 + query;
        const bool there = query < S.nq;
        if (STAGED && P.splits_q == 1) {
            if constexpr (STAGED)
                R::store(lds + mine_at, dq, P.scale, const_cast<char*>(at<E>(P.dq, S.q0 + mine, head)), P.dq.token, unsigned(__ballot(there)), P.dim, lane);
        } else if (there) {
            if (P.splits_q == 1) {
                char* row = const_cast<char*>(at<E>(P.dq, S.q0 + query, head));
#pragma unroll
                for (int n = 0; n < DT; ++n) store_column<E>(row, dq[n], P.scale, n, P.dim, half);
            } else {
#pragma unroll
                for (int n = 0; n < DT; ++n) store_column<F32>(reinterpret_cast<char*>(part + at_q * (32 * DT)), dq[n], P.scale, n, 32 * DT, half);
            }
        }
    };
    __syncthreads();                                              // every wave is done with the tiles
    finish(lane, query);
    Marks& marks = *reinterpret_cast<Marks*>(lds + 4 * SIZE);
    if (__builtin_expect(any_wave<WAVES>(marks, wave, there && lse == lse && delta == delta && not_finite(dq)), 0)) {
        // Once more.  A key or value that is not finite makes no number of every entry of the dq that it reaches.
        clear(marks, S.nk, threadIdx.x, WAVES * 64);
#pragma unroll
        for (int n = 0; n < DT; ++n) dq[n] = zero16();
        const int lane = lane_anew(), half = lane >> 5, query = mine + (lane & 31), last = P.causal ? min(S.nk - 1, query + S.shift) : S.nk - 1;
        Loader<E, DT, KEYS, WAVES> lk, lv;
        lk.init(wave, lane, P.k.token, P.dim);
        lv.init(wave, lane, P.v.token, P.dim);
        Reader<E, DT> rd;
        rd.init(lane);
        Operand<E, DT> q, d;
        q.load(at<E>(P.q, S.q0 + query, head), query < S.nq, P.dim, half);
        d.load(at<E>(P.d_o, S.q0 + query, head), query < S.nq, P.dim, half);
        for (int j = from; j < to; j += KEYS) {
            lk.load(base, at<E>(P.k, S.k0 + j, kv), end - j, wave);
            lv.load(base + SIZE, at<E>(P.v, S.k0 + j, kv), end - j, wave);
            __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
            __syncthreads();
            const auto mark = [&](int r, int, bool, bool) { mark_first(marks.any[0], j + r); };
            lk.clean(lds, wave, lane, mark);
            lv.clean(lds + SIZE, wave, lane, mark);
            __syncthreads();
            if (j < end_mine) {
#pragma unroll 1
                for (int b = 0; b < KB<E>; ++b) grad_q_block<E, DT>(dq, rd, lds + b * 32 * T::PITCH, lds + SIZE + b * 32 * T::PITCH, q, d, P.c, lse, delta, false, last - j - 32 * b, half);
            }
            __syncthreads();
        }
        if (marks.any[0] <= last) {
#pragma unroll
            for (int n = 0; n < DT; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) dq[n][r] = __builtin_nanf("");
        }
        finish(lane, query);
    }
}

// A block of 32 queries: scores and the probabilities' gradients, then arithmetic of 8 rows at a time and their products with
// d_out and with q.  numbers: what the rows' scores begin with, -lse / scale, and 64 further on what their probabilities'
// gradients begin with, -delta; in an accumulator from the start they cost neither registers nor subtractions.  first: the
// first row, counted from the block's, that sees this lane's key.  The keys' operands and sums fill three quarters of the registers: what can be had again
// from a few instructions is not kept.
template <class E, int DT>
__device__ __forceinline__ void grad_kv_block(float16v (&dk)[DT], float16v (&dv)[DT], Reader<E, DT>& rd, const char* qt, const char* dt, const float* numbers,
                                              const Operand<E, DT>& k, const Operand<E, DT>& v, float c, bool all_seen, int first, int half) {
    typedef Tile<E, DT> T;
    constexpr int N = 2 * T::STEPS, AHEAD = 2;
    asm volatile("" : "+v"(rd.row), "+v"(rd.tr));                 // offsets anew, instead of 16 registers for them
    // (fp32 adds them at the end: in front, every step of a sum of a score's size would be rounded to a log-sum-exp's)
    constexpr bool FIRST = sizeof(typename E::T) == 2;
    float16v s, dp, s0, dp0;
    typename E::Row a[AHEAD];
    auto read = [&](int i) {
        if (i < N) a[i % AHEAD] = rd.rows(i & 1 ? dt : qt, 0, i >> 1);
    };
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float4v x = *reinterpret_cast<const float4v*>(numbers + 8 * g + 4 * half), y = *reinterpret_cast<const float4v*>(numbers + 64 + 8 * g + 4 * half);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s0[4 * g + e] = x[e];
            dp0[4 * g + e] = y[e];
        }
    }
    s = FIRST ? s0 : zero16();
    dp = FIRST ? dp0 : zero16();
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int x = i >> 1;
        if (i & 1) dp = E::mma(a[i % AHEAD], v.x[x], dp);
        else s = E::mma(a[i % AHEAD], k.x[x], s);
        read(i + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (!FIRST) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] += s0[r];
            dp[r] += dp0[r];
        }
    }
    if (!all_seen) {
        asm volatile("");
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (acc_row(r, half) < first) s[r] = NEG_INF;
    }
    auto arithmetic = [&](int r) {
        s[r] = __builtin_amdgcn_exp2f(s[r] * c);
        dp[r] *= s[r];
        asm volatile("" : "+v"(s[r]), "+v"(dp[r]));
    };
    auto pack = [&](const float16v& from, int t) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from[8 * t + e];
        return E::pack(x);
    };
#pragma unroll
    for (int r = 0; r < 8; ++r) arithmetic(r);
    if constexpr (sizeof(typename E::T) == 2) {
        constexpr int M = 4 * DT;
        typename E::Row u[AHEAD];
        auto read_t = [&](int i) {
            if (i < M) u[i % AHEAD] = columns<DT>(rd, (i / DT) & 1 ? qt : dt, i / (2 * DT), i % DT);
        };
        typename E::Score p = pack(s, 0), ds = pack(dp, 0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) read_t(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < M; ++i) {
            if (i == M / 2) {
                p = pack(s, 1);
                ds = pack(dp, 1);
            }
            if ((i / DT) & 1) dk[i % DT] = E::mma(u[i % AHEAD], ds, dk[i % DT]);
            else dv[i % DT] = E::mma(u[i % AHEAD], p, dv[i % DT]);
            read_t(i + AHEAD);
            if (i < M / 2) {
#pragma unroll
                for (int r = 8 + 16 * i / M; r < 8 + 16 * (i + 1) / M; ++r) arithmetic(r);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int r = 8; r < 16; ++r) arithmetic(r);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const typename E::Score p = pack(s, t), ds = pack(dp, t);
#pragma unroll
            for (int n = 0; n < DT; ++n) dv[n] = mma_t<DT>(rd, dt, t, n, p, dv[n]);
#pragma unroll
            for (int n = 0; n < DT; ++n) dk[n] = mma_t<DT>(rd, qt, t, n, ds, dk[n]);
        }
    }
}

// dv_j = sum_i p_ij d_out_i and dk_j = scale sum_i ds_ij q_i over the queries of all heads of a group, for WAVES x 32 keys.  Four
// products a tile: 8 x 2048 tokens 500 to 550 us, 1.0 to 1.1 PFLOP/s executed, matrix pipes busy 57 %.  The registers are full:
// what spilled of the keys' operands was once read back every tile behind the loads under way, and doubled the time; the 17 that
// spill now are read back behind the loop.
template <class E, int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64, sizeof(typename E::T) == 2 ? 2 : 1) void grad_kv_kernel(const Params P) {
    constexpr int ROWS = 32 * KB<E>;
    typedef Tile<E, DT> T;
    constexpr int SIZE = T::bytes(ROWS), BUF = 2 * SIZE + 512;    // queries, d_out, 64 log-sum-exps, 64 deltas
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = int(blockIdx.x) % P.kv_heads;
    int tile, tiles;
    Seq S;
    if (find_tile<attn::KEYS>(P, WAVES * 32, int(blockIdx.x) / P.kv_heads, S, tile, tiles) != TILE) return;
    tile = tiles - 1 - tile;                                      // a causal prompt's first keys are seen by all that follow
    const int first = tile * WAVES * 32, mine = first + wave * 32, key = mine + col;
    // queries that see any key of the workgroup, of this wave: from `begin` on; from `all` on they see all of the wave's
    const int begin = first >= S.nk ? S.nq : P.causal ? min(S.nq, max(0, first - S.shift)) / ROWS * ROWS : 0;
    const int begin_mine = mine >= S.nk ? S.nq : P.causal ? max(0, mine - S.shift) : 0;
    const int all = P.causal ? mine + 31 - S.shift : 0;
    // steps through the queries of one head after the other; this workgroup's share of them
    const int steps = begin < S.nq ? (S.nq - begin + ROWS - 1) / ROWS : 0, all_steps = steps * P.group;
    const int step0 = int(int64_t(all_steps) * int(blockIdx.y) / P.splits_k), total = int(int64_t(all_steps) * (int(blockIdx.y) + 1) / P.splits_k);

    Loader<E, DT, ROWS, WAVES> lq, ld;
    lq.init(wave, lane, P.q.token, P.dim);
    ld.init(wave, lane, P.d_o.token, P.dim);
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((ONECOMP_LDS char*)lds));
    auto bring_with = [&](const Loader<E, DT, ROWS, WAVES>& lq, const Loader<E, DT, ROWS, WAVES>& ld, int lane, int head, int r, int buf) {
        const uint32_t to = base + uint32_t(buf) * BUF;
        lq.load(to, at<E>(P.q, S.q0 + r, head), S.nq - r, wave);
        ld.load(to + SIZE, at<E>(P.d_o, S.q0 + r, head), S.nq - r, wave);
        if (wave < 2) {                                           // numbers of rows that are not there: zeros
            const float* from = P.aux + (int64_t(wave) * P.heads + head) * P.total_q + S.q0 + r;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, min(S.nq - r, ROWS) * 4, 0x00020000);
            lds_load4(to + 2 * SIZE + uint32_t(wave) * 256u, uint32_t(lane) * 4u, rsrc);
        }
    };
    auto bring = [&](int head, int r, int buf) { bring_with(lq, ld, lane, head, r, buf); };
    constexpr bool STAGED = sizeof(typename E::T) == 2;           // rows through LDS
    Reader<E, DT> rd;
    rd.init(lane);
    Operand<E, DT> k, v;
    typedef Rows<E, DT> R;
    static_assert(!STAGED || WAVES * R::BYTES == 2 * SIZE, "the waves' rows fill one pair of tiles");
    const int mine_at = wave * (STAGED ? R::BYTES : 0);
    if constexpr (STAGED) {
        R::bring(base + mine_at, at<E>(P.k, S.k0 + mine, kv), S.nk - mine, P.k.token, P.dim, lane);
        R::bring(base + 2 * SIZE + mine_at, at<E>(P.v, S.k0 + mine, kv), S.nk - mine, P.v.token, P.dim, lane);
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
        asm volatile("" ::: "memory");
        R::take(k, rd, lds + mine_at);
        R::take(v, rd, lds + 2 * SIZE + mine_at);
        __syncthreads();
    } else {
        k.load(at<E>(P.k, S.k0 + key, kv), key < S.nk, P.dim, half);
        v.load(at<E>(P.v, S.k0 + key, kv), key < S.nk, P.dim, half);
    }
    const int head0 = kv * P.group;
    int head = head0, r0 = begin;
    if (step0 < total) {
        head += step0 / steps;
        r0 += step0 % steps * ROWS;
        bring(head, r0, 0);
    }
    float16v dk[DT], dv[DT];
#pragma unroll
    for (int n = 0; n < DT; ++n) dk[n] = dv[n] = zero16();

    for (int step = step0, buf = 0; step < total; ++step, buf ^= 1) {
        __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
        __syncthreads();
        int next_head = head, next = r0 + ROWS;
        if (next >= S.nq) { next = begin; ++next_head; }
        if (step + 1 < total) bring(next_head, next, buf ^ 1);
        if (r0 + ROWS > begin_mine) {
            const char *qt = lds + buf * BUF, *dt = qt + SIZE;
            const bool all_seen = r0 >= all;
#pragma unroll
            for (int b = 0; b < KB<E>; ++b)
                grad_kv_block<E, DT>(dk, dv, rd, qt + b * 32 * T::PITCH, dt + b * 32 * T::PITCH, reinterpret_cast<const float*>(qt + 2 * SIZE) + 32 * b, k, v, P.c,
                                     all_seen, key - S.shift - r0 - 32 * b, half);
        }
        head = next_head;
        r0 = next;
    }
    // sums of a share: those for dk, then those for dv
    const int64_t rows_k = int64_t(P.kv_heads) * P.total_k;
    float* part = P.part + P.splits_q * (P.splits_q > 1) * int64_t(P.heads) * P.total_q * (32 * DT) + 2 * int64_t(blockIdx.y) * rows_k * (32 * DT);
    // lane, key: as the kernel's own
    auto finish = [&](int lane, int key) {
        const int half = lane >> 5;
        if (key >= S.nk) {
#pragma unroll
            for (int n = 0; n < DT; ++n) dk[n] = dv[n] = zero16();
        }
        if (STAGED && P.splits_k == 1) {
            if constexpr (STAGED) {
                const unsigned which = unsigned(__ballot(key < S.room));
                R::store(lds + mine_at, dk, P.scale, const_cast<char*>(at<E>(P.dk, S.k0 + mine, kv)), P.dk.token, which, P.dim, lane);
                R::store(lds + 2 * SIZE + mine_at, dv, 1.f, const_cast<char*>(at<E>(P.dv, S.k0 + mine, kv)), P.dv.token, which, P.dim, lane);
            }
        } else if (key < S.room) {
            if (P.splits_k == 1) {
                char* row_k = const_cast<char*>(at<E>(P.dk, S.k0 + key, kv));
                char* row_v = const_cast<char*>(at<E>(P.dv, S.k0 + key, kv));
#pragma unroll
                for (int n = 0; n < DT; ++n) {
                    store_column<E>(row_k, dk[n], P.scale, n, P.dim, half);
                    store_column<E>(row_v, dv[n], 1.f, n, P.dim, half);
                }
            } else {
                float* to = part + (int64_t(kv) * P.total_k + S.k0 + key) * (32 * DT);
#pragma unroll
                for (int n = 0; n < DT; ++n) {
                    store_column<F32>(reinterpret_cast<char*>(to), dk[n], P.scale, n, 32 * DT, half);
                    store_column<F32>(reinterpret_cast<char*>(to + rows_k * (32 * DT)), dv[n], 1.f, n, 32 * DT, half);
                }
            }
        }
    };
    __syncthreads();                                              // every wave is done with the tiles
    finish(lane, key);
    Marks& marks = *reinterpret_cast<Marks*>(lds + 2 * BUF);
    if (__builtin_expect(any_wave<WAVES>(marks, wave, not_finite(dk) || not_finite(dv)), 0)) {
        // Once more.  A query or log-sum-exp that is not finite makes no numbers of the dk and dv that it reaches (any[0]), a row of
        // d_out or a delta of those dk (any[1]).
        clear(marks, -1, threadIdx.x, WAVES * 64);
#pragma unroll
        for (int n = 0; n < DT; ++n) dk[n] = dv[n] = zero16();
        const int lane = lane_anew(), half = lane >> 5, key = mine + (lane & 31);
        Loader<E, DT, ROWS, WAVES> lq, ld;
        lq.init(wave, lane, P.q.token, P.dim);
        ld.init(wave, lane, P.d_o.token, P.dim);
        Reader<E, DT> rd;
        rd.init(lane);
        Operand<E, DT> k, v;
        k.load(at<E>(P.k, S.k0 + key, kv), key < S.nk, P.dim, half);
        v.load(at<E>(P.v, S.k0 + key, kv), key < S.nk, P.dim, half);
        for (int step = step0; step < total; ++step) {
            const int r = begin + step % steps * ROWS;
            bring_with(lq, ld, lane, head0 + step / steps, r, 0);
            __builtin_amdgcn_s_waitcnt(wait_vmcnt(0));
            __syncthreads();
            lq.clean(lds, wave, lane, [&](int row, int, bool, bool) { mark_last(marks.any[0], r + row); });
            ld.clean(lds + SIZE, wave, lane, [&](int row, int c, bool up, bool down) {
                if (up) mark_last(marks.up(c), r + row);
                if (down) mark_last(marks.down(c), r + row);
                mark_last(marks.any[1], r + row);
            });
            if (wave < 2) {
                float& x = reinterpret_cast<float*>(lds + 2 * SIZE)[64 * wave + lane];
                // -inf in front of the scores is a query that sees nothing
                if (!(wave == 0 ? x < -NEG_INF : x * 0.f == 0.f)) {
                    mark_last(marks.any[wave], r + lane);
                    x = wave == 0 ? NEG_INF : 0.f;
                }
            }
            __syncthreads();
            if (r + ROWS > begin_mine) {
#pragma unroll 1
                for (int b = 0; b < KB<E>; ++b)
                    grad_kv_block<E, DT>(dk, dv, rd, lds + b * 32 * T::PITCH, lds + SIZE + b * 32 * T::PITCH, reinterpret_cast<const float*>(lds + 2 * SIZE) + 32 * b, k, v,
                                         P.c, r >= all, key - S.shift - r - 32 * b, half);
            }
            __syncthreads();
        }
        const int seen_from = P.causal ? max(0, key - S.shift) : 0;
        const float no_k = max(marks.any[0], marks.any[1]) >= seen_from ? __builtin_nanf("") : 0.f, no_v = marks.any[0] >= seen_from ? __builtin_nanf("") : 0.f;
#pragma unroll
        for (int n = 0; n < DT; ++n) {
            give_back(dv[n], marks, n, half, [&](int row) { return row >= seen_from; });
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                dk[n][r] += no_k;
                dv[n][r] += no_v;
            }
        }
        finish(lane, key);
    }
}

// The shares' sums of one gradient meet, in their order: out[token, head] = sum over s of part[s][head, token].
template <class E, int DT>
__global__ __launch_bounds__(256) void join_kernel(const View out, const float* part, const int splits, const int64_t stride, const int64_t tokens, const int heads,
                                                   const int dim) {
    constexpr int COLS = 32 * DT, LANES = COLS / 4;               // four columns a lane
    const int64_t at_row = (int64_t(blockIdx.x) * 256 + threadIdx.x) / LANES;
    const int d = int((int64_t(blockIdx.x) * 256 + threadIdx.x) % LANES) * 4;
    if (at_row >= tokens * heads || d >= dim) return;
    float4v sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const float4v*>(part + s * stride + at_row * COLS + d);
    const int head = int(at_row / tokens);
    char* to = const_cast<char*>(at<E>(out, at_row - int64_t(head) * tokens, head));
#pragma unroll
    for (int e = 0; e < 4; ++e) put<E>(to, d + e, sum[e]);
}

template <class E, int DT>
onecomp_status join(const View& out, const float* part, int splits, int64_t stride, int64_t tokens, int heads, int dim, hipStream_t stream) {
    const int64_t grid = ceil_div(tokens * heads * (8 * DT), 256);
    if (grid > 0x7fffffff) return ONECOMP_ERR_UNSUPPORTED;
    join_kernel<E, DT><<<dim3(unsigned(grid)), dim3(256), 0, stream>>>(out, part, splits, stride, tokens, heads, dim);
    ONECOMP_CHECK_LAUNCH();
    return ONECOMP_OK;
}

template <class E, int DT, int WQ, int WK>
onecomp_status launch_backward(const Params& P, hipStream_t stream) {
    typedef Tile<E, DT> T;
    constexpr int TILES = 4 * T::bytes(32 * KB<E>), LDS_Q = TILES + int(sizeof(Marks)), LDS_K = TILES + 1024 + int(sizeof(Marks));
    static std::atomic<uint64_t> done_q{0}, done_k{0};
    onecomp_status st = allow_dynamic_lds(reinterpret_cast<const void*>(grad_q_kernel<E, DT, WQ>), LDS_Q, done_q);
    if (st != ONECOMP_OK) return st;
    st = allow_dynamic_lds(reinterpret_cast<const void*>(grad_kv_kernel<E, DT, WK>), LDS_K, done_k);
    if (st != ONECOMP_OK) return st;
    const int64_t grid_q = (P.total_q / (WQ * 32) + P.n_seqs + 1) * P.heads, grid_k = (P.total_k / (WK * 32) + P.n_seqs + 1) * P.kv_heads;
    if (grid_q > 0x7fffffff || grid_k > 0x7fffffff) return ONECOMP_ERR_UNSUPPORTED;
    if (P.total_q > 0) {
        grad_q_kernel<E, DT, WQ><<<dim3(unsigned(grid_q), unsigned(P.splits_q)), dim3(WQ * 64), LDS_Q, stream>>>(P);
        ONECOMP_CHECK_LAUNCH();
    }
    if (P.total_k > 0) {
        grad_kv_kernel<E, DT, WK><<<dim3(unsigned(grid_k), unsigned(P.splits_k)), dim3(WK * 64), LDS_K, stream>>>(P);
        ONECOMP_CHECK_LAUNCH();
    }
    const int64_t cols = 32 * DT, part_q = P.total_q * P.heads * cols, part_k = P.total_k * P.kv_heads * cols;
    const float* parts = P.part;
    if (P.splits_q > 1) {
        if (const onecomp_status e = join<E, DT>(P.dq, parts, P.splits_q, part_q, P.total_q, P.heads, P.dim, stream)) return e;
        parts += P.splits_q * part_q;
    }
    if (P.splits_k > 1) {
        if (const onecomp_status e = join<E, DT>(P.dk, parts, P.splits_k, 2 * part_k, P.total_k, P.kv_heads, P.dim, stream)) return e;
        if (const onecomp_status e = join<E, DT>(P.dv, parts + part_k, P.splits_k, 2 * part_k, P.total_k, P.kv_heads, P.dim, stream)) return e;
    }
    return ONECOMP_OK;
}

// Where whole sequences make too few workgroups to fill the chip, their inner loops are split: the keys of dq's rows, the
// queries of dk's and dv's.  512 workgroups are two on each CU; more cost more in partial sums than they bring (2048 tokens,
// 8 / 2 heads of 128: 284 us whole, 90 with 512, 120 with 1024).  A share is worth the launches that join it from 8 tiles of 64
// on (4 x 512 tokens, 8 heads: 43 us whole, 62 in shares of 4 tiles), in fp32, whose products take longer, from the first on
// (300 tokens, 4 / 1 heads of 32: 128 us whole, 31 split).
void plan(onecomp_dtype dtype, Params& P) {
    const int64_t groups_q = (P.total_q / 128 + P.n_seqs) * P.heads, groups_k = (P.total_k / 128 + P.n_seqs) * P.kv_heads;
    auto splits = [&](int64_t groups, int64_t steps) {
        const int64_t n = groups < 1 ? 1 : 512 / groups, most = dtype == ONECOMP_F32 ? steps : steps / 8;
        return int(n < 2 || most < 2 ? 1 : n < most ? n : most);
    };
    P.splits_q = P.total_q ? splits(groups_q, ceil_div(P.max_k, 64)) : 1;
    P.splits_k = P.total_k ? splits(groups_k, ceil_div(P.max_q < P.total_q ? P.max_q : P.total_q, 64) * P.group) : 1;
}

}  // namespace

size_t backward_workspace_bytes(onecomp_dtype dtype, const Params& in) {
    Params P = in;
    plan(dtype, P);
    const size_t cols = size_t(P.dim + 31) / 32 * 32, rows_q = size_t(P.total_q) * P.heads, rows_k = size_t(P.total_k) * P.kv_heads;
    size_t floats = align_up(2 * rows_q, 64);
    if (P.splits_q > 1) floats += P.splits_q * rows_q * cols;
    if (P.splits_k > 1) floats += 2 * P.splits_k * rows_k * cols;
    return align_up(floats * 4, 256);
}

onecomp_status backward_run(onecomp_dtype dtype, const Params& in, hipStream_t stream) {
    Params P = in;
    plan(dtype, P);
    P.part = P.aux + align_up(size_t(P.total_q) * P.heads * 2, 64);
    const int dt = (P.dim + 31) / 32;
    if (dtype == ONECOMP_BF16)
        return dt == 1   ? launch_backward<Bf16, 1, 4, 4>(P, stream)
               : dt == 2 ? launch_backward<Bf16, 2, 4, 4>(P, stream)
               : dt == 3 ? launch_backward<Bf16, 3, 4, 4>(P, stream)
                         : launch_backward<Bf16, 4, 4, 4>(P, stream);
    return dt == 1   ? launch_backward<F32, 1, 4, 4>(P, stream)
           : dt == 2 ? launch_backward<F32, 2, 4, 4>(P, stream)
           : dt == 3 ? launch_backward<F32, 3, 4, 4>(P, stream)
                     : launch_backward<F32, 4, 4, 4>(P, stream);
}

}  // namespace attn
}  // namespace onecomp
