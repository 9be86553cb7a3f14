// The attention weight that new tokens give to each key, added to the keys' scores (flashd_cache_score).
//
// score_j <- decay score_j + sum over the new tokens i that see key j, and the heads of the kv group, of
// w_i exp(scale q_i.k_j - lse_i), with the queries' log-sum-exps as the attention has left them: so that one pass over K is enough, no
// sum over the keys is needed, and what belongs to a key stays in one workgroup.
//
// S = Q K^T comes with keys as columns of the matrix products, so that the sum over rows (pairs of token and head of the group) is one over a lane's own
// registers.  K is the B operand and goes from the pages to registers as it lies there; a row's w exp(-lse) is one number in
// the exponent: 2^(c s - bias).
//
// Up to 16 rows to a sequence and kv head HBM bounds it (score_few_kernel); with more the products and exponentials count as well, and in the end more than the keys
// (score_many_kernel).  Both are launched where the call may have either.
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

#include <type_traits>

namespace flashd {

constexpr int kScoreWaves = 8, kScoreThreads = kScoreWaves * kWave;
constexpr int kScoreGroups = 256;       // workgroups of a launch: one per compute unit, two wavefronts per SIMD
constexpr int kFewRows = 16;            // rows of a unit that the first kernel takes
constexpr int kBiasTiles = 128;         // tiles whose rows' bias lies in LDS
constexpr int kScoreRuns = 128;         // runs of sequences

struct ScoreRun {
    Paged c;
    ScoreArgs a;
    FastDiv group;          // query heads per kv head
};

template <typename T, int D, bool FP8> struct ScoreCfg {
    static constexpr bool F = std::is_same_v<T, F32>;
    static constexpr int ROWB = D * (F ? 4 : FP8 ? 1 : 2);       // bytes of a key
    static constexpr int QSZ = F ? 4 : 2;
    static constexpr int KPITCH = ROWB + 16;                     // of a key in LDS: 16 of them fall on all banks
    // few: 16-key blocks of a turn, and loads of 16 bytes per lane and block
    static constexpr int TURN = ROWB >= 512 ? 2 : ROWB >= 256 ? 4 : 8;
    static constexpr int FEW = 16 * TURN;
    static constexpr int NF = ROWB / 64;
    // more: 32-key blocks of a turn, as many as there are registers for, beside those of the next turn where a wavefront takes it alone; 16-byte loads of
    // a lane for a block; operands of a lane
    static constexpr int LONG = F ? (D == 128 ? 1 : 2) : 4, MID = LONG > 1 ? LONG / 2 : 1;
    static constexpr int NM = ROWB / 32;
    static constexpr int STEPS = D * QSZ / 32;
    // a tile of 32 rows in LDS, and how many of them a wavefront has.  Rows lie one behind the other as copies of 1 KB leave them, the 16-byte chunk c of row r
    // at c ^ swz(r), so that 16 rows' chunks fall on all banks.
    static constexpr int QROW = D * QSZ, CH = QROW / 16;
    static constexpr int TILE = 32 * QROW;
    static constexpr int SLOTS = TILE > 8192 ? 1 : 2;
    // Up to this many tiles lie in LDS for all of a unit's turns, beside 16 keys of each wavefront on their way to the operands; in more the workgroup shares out the tiles
    static constexpr int STAGE = kScoreWaves * 16 * KPITCH, FIT = (131072 - STAGE) / TILE, OWN = FIT < 16 ? FIT : 16;
    static __device__ __forceinline__ int swz(int row) { return CH == 8 ? row >> 1 & 7 : row & 15; }
    // Tokens of a tile: with all their heads, or one where that is more than a tile's rows, or where offsets within the tile would pass 32 bits
    static __device__ __forceinline__ int tokens(const ScoreRun& r) {
        const int heads = (int)r.group.d;
        return heads > 32 || r.a.q_stride * QSZ * 32 > (1ll << 30) ? 1 : 32 / heads;
    }
    static __device__ __forceinline__ int tiles(const ScoreRun& r, int n) {
        const int heads = (int)r.group.d, of = tokens(r);
        return heads > 32 ? n * ((heads + 31) / 32) : (n + of - 1) / of;
    }
    // Byte of a row at which a lane's operand s begins, in the order in which the loads of K bring the elements: of fp8 16 at a time
    static __device__ __forceinline__ int few_at(int s, int q) { return FP8 ? 128 * (s >> 1) + 32 * q + 16 * (s & 1) : 64 * s + 16 * q; }
    static constexpr int many_at(int s) { return FP8 ? 64 * (s >> 1) + 16 * (s & 1) : 32 * s; }
    static constexpr int kHalf = FP8 ? 32 : 16;                  // and what the upper half of the lanes adds
};

template <typename T> struct Few;
template <> struct Few<BF16> {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Few<F16> {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long same(long long x) {
    return (long long)((uint64_t)(uint32_t)same((int)(x >> 32)) << 32 | (uint32_t)same((int)x));
}

// `bytes` bytes from `at` on, the same in every lane, behind which loads bring zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const char* at, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(same((long long)(uintptr_t)at)), 0, same(bytes), 0x00020000);
}

// Waits for the loads under way, as the compiler knows: what it holds for still to come before a loop it waits for in every turn of it, and so for
// all that is asked for in the meantime.
__device__ __forceinline__ void have_loads() {
    __builtin_amdgcn_s_waitcnt(0x0f70);
    asm volatile("" ::: "memory");
}
// a / b rounded up, of whole numbers 0 <= a < 2^52 and b > 0, by a division of doubles (the rounded quotient's ceiling can be one off)
__device__ __forceinline__ long long ceil_div(long long a, long long b) {
    long long q = (long long)((double)a / (double)b);
    q = q * b >= a ? q : q + 1;
    return (q - 1) * b >= a ? q - 1 : q;
}

// The workgroup's place: neighbours in the order of the turns, which read the same queries, are on one XCD.
__device__ __forceinline__ int place_of_group() { return ((int)blockIdx.x & 7) * (kScoreGroups / 8) + ((int)blockIdx.x >> 3); }

// ---- the work of a launch -----------------------------------------------------------------------
//
// Units are (sequence, kv head), cut into turns of keys.  Turns of few rows lie in a row of which each workgroup has a stretch, those of more rows in
// another.  Of a stretch the wavefronts take turn after turn as they come to it: of the two on a SIMD the older one is served first, and with stretches
// of their own the older ones ended after 66 us, the younger after 112 (a token for each of 64 sequences of 500 to 8192 keys).
// Units of many rows, whose turns take long, are the workgroups' in turn: turn i of all of them is that of workgroup i modulo their number, every other time
// backwards, in the order of falling rows (up to 128 sequences), so that none has much more than another.
enum ScoreKind { kFew, kMid, kLong };

struct ScoreScratch {
    long long first[3][kScoreRuns];      // of each thread's run of sequences: turns of all runs before
    long long sum[3][kScoreRuns / kWave];
    int rows[kScoreRuns];
    int order[kScoreRuns];               // long ones: sequences by falling rows
    int taken;                           // turns of the workgroup's stretch
};

template <typename C>
struct ScoreWalk {
    int b, h, chunk;            // the present turn
    Seq s;
    int rows, chunks, kind;
    long long at, end;          // the stretch that is left, in turns

    __device__ __forceinline__ void enter(const ScoreRun& r, int seq) {
        b = seq;
        s = seq_at(r.c, b);
        rows = s.n * (int)r.group.d;             // (T Hq is below 2^31)
        kind = rows <= kFewRows ? kFew : C::tiles(r, s.n) <= C::OWN ? kMid : kLong;
        const int keys = kind == kFew ? C::FEW : 32 * (kind == kMid ? C::MID : C::LONG);
        chunks = s.n == 0 ? 0 : (s.len + s.n + keys - 1) / keys;
    }
    __device__ __forceinline__ long long turns(const ScoreRun& r, int of) const { return of == kind ? (long long)chunks * r.c.Hkv : 0; }
    // (Every member is the same in all lanes; said once more for the compiler, which past the loops takes them for different ones.)
    __device__ __forceinline__ void settle() {
        b = same(b);
        h = same(h);
        chunk = same(chunk);
        s = Seq{same(s.row0), same(s.n), same(s.len)};
        rows = same(rows);
        chunks = same(chunks);
        kind = same(kind);
        at = same(at);
        end = same(end);
    }
    static __device__ __forceinline__ int each(const ScoreRun& r) { return (r.c.B + kScoreRuns - 1) / kScoreRuns; }

    // Every thread takes a run of sequences, whose turns are then summed over the threads.  FROM, TO: the kinds that are asked for.
    template <int FROM, int TO>
    static __device__ __forceinline__ void begin(const ScoreRun& r, ScoreScratch* sh, long long (&total)[3]) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int n = each(r), b0 = tid * n, b1 = tid < kScoreRuns ? min(b0 + n, r.c.B) : 0;
        if (tid == 0) sh->taken = 0;
        long long mine[3] = {0, 0, 0};
        ScoreWalk any;
        any.rows = -1;
        any.kind = kFew;
        any.chunks = 0;
        for (int i = b0; i < b1; ++i) {
            any.enter(r, i);
#pragma unroll
            for (int k = 0; k < 3; ++k) mine[k] += any.turns(r, k);
        }
        if (TO == kLong && n == 1 && __syncthreads_or(mine[kLong] != 0)) {
            const int rows = any.kind == kLong ? any.rows : -1;
            if (tid < kScoreRuns) {
                sh->rows[tid] = rows;
                sh->first[kLong][tid] = mine[kLong];
            }
            __syncthreads();
            if (tid < kScoreRuns) {
                int rank = 0;
                for (int i = 0; i < kScoreRuns; ++i) rank += sh->rows[i] > rows || (sh->rows[i] == rows && i < tid);
                sh->order[rank] = tid;
            }
            __syncthreads();
            if (tid < kScoreRuns) mine[kLong] = sh->first[kLong][sh->order[tid]];
            __syncthreads();
        }
        long long in[3];
#pragma unroll
        for (int k = FROM; k <= TO; ++k) {
            in[k] = mine[k];
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const long long y = __shfl_up(in[k], d);
                if (lane >= d) in[k] += y;
            }
            if (lane == 63 && wave < kScoreRuns / kWave) sh->sum[k][wave] = in[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = FROM; k <= TO; ++k) {
            long long before = in[k] - mine[k];
            total[k] = 0;
#pragma unroll
            for (int i = 0; i < kScoreRuns / kWave; ++i) {
                before += i < wave ? sh->sum[k][i] : 0;
                total[k] += sh->sum[k][i];
            }
            total[k] = same(total[k]);
            if (tid < kScoreRuns) sh->first[k][tid] = before;
        }
        __syncthreads();
    }
    // Turn x (below the total) of the list of a kind; every wavefront for itself.
    __device__ __forceinline__ void take(const ScoreRun& r, const ScoreScratch* sh, int of, long long x) {
        // the last run that does not begin behind it
        const int lane = threadIdx.x & 63;
        int run = -1;
#pragma unroll
        for (int i = 0; i < kScoreRuns; i += kWave) {
            const uint64_t before = __builtin_amdgcn_ballot_w64(sh->first[of][i + lane] <= x);
            if (before != 0) run = i + 63 - __builtin_clzll(before);
        }
        run = same(run);
        long long first = same(sh->first[of][run]);
        const int n = each(r);
        for (int i = 0;; ++i) {
            enter(r, of == kLong && n == 1 ? same(sh->order[run]) : run * n + i);
            const long long own = turns(r, of);
            if (i + 1 == n || x < first + own) break;
            first += own;
        }
        const long long k = x - first;
        h = (int)ceil_div(k + 1, max(chunks, 1)) - 1;
        chunk = (int)(k - (long long)h * chunks);
        at = x;
        settle();
    }
    // Place `w` of `n` equal stretches of the row of a kind; false: nothing in it
    __device__ __forceinline__ bool start(const ScoreRun& r, const ScoreScratch* sh, int of, long long total, int w, int n) {
        const long long per = ceil_div(total, n), from = w * per, to = min(from + per, total);
        if (from >= to) return false;
        take(r, sh, of, from);
        end = same(to);
        return true;
    }
    // On to turn x (not before the present one) of the same list; false: not in the stretch
    __device__ __forceinline__ bool advance_to(const ScoreRun& r, long long x) {
        if (x >= end) return false;
        chunk += (int)(x - at);                  // (few turns, as a rule: no division)
        at = x;
        while (chunk >= chunks) {
            chunk -= chunks;
            if (++h == r.c.Hkv) {
                const int of = kind;
                do enter(r, b + 1);              // (there is one: the stretch has turns left)
                while (turns(r, of) == 0);
                h = 0;
            }
        }
        settle();
        return true;
    }
};

// What a row with log-sum-exp l and weight w takes from the exponent; infinite where it does not count: it sees nothing (l is -infinity), l is no
// number, or w is not positive.
__device__ __forceinline__ float bias(float l, float w, bool weighed) {
    const float inf = __builtin_inff();
    return w > 0.0f && l > -inf ? l * kLog2e - (weighed ? log2_fast(w) : 0.0f) : inf;
}
// Which of N rows, 4 from `row` on and then 8 further each time, see the new key `rel` (any below 0 is an old one): bit i for the i-th.  Row 0 is the first one of
// token t0, `heads` rows to a token (row / heads.d, or 0 where a token is more rows than there can be).
template <int N, class W>
__device__ __forceinline__ uint32_t seen_by(const ScoreRun& r, const W& u, int t0, const FastDiv& heads, int row, int rel) {
    const uint32_t all = (1u << N) - 1u;
    if (r.a.tree == nullptr) {
        // of a chain those from the token's own first row on
        const int x = heads.s2 == 31 ? (rel > t0 ? 1 << 20 : 0) : min(max(rel - t0, 0), 1 << 10) * (int)heads.d - row;
        const int before = x <= 0 ? 0 : min(4 * (x >> 3) + min(x & 7, 4), N);
        return rel >= u.s.n ? 0u : all & (all << before);
    }
    if (rel < 0) return all;
    uint32_t bits = 0;
    if (rel >= u.s.n || rel >> 5 >= r.a.words) return bits;
    const uint32_t* word = r.a.tree + (size_t)u.s.row0 * r.a.words + (rel >> 5);
    // (four at a time: all at once, around the products, they take a hundred registers)
#pragma unroll 4
    for (int i = 0; i < N; ++i) {
        const int token = min(t0 + (int)fast_div((uint32_t)(row + 8 * (i >> 2) + (i & 3)), heads), u.s.n - 1);
        bits |= (word[(size_t)token * r.a.words] >> (rel & 31) & 1u) << i;
    }
    return bits;
}
// x if bit i is set, else 0
__device__ __forceinline__ float if_bit(uint32_t bits, int i, float x) {
    return __uint_as_float(__float_as_uint(x) & (uint32_t)((int)(bits << (31 - i)) >> 31));
}

// ---- few rows ------------------------------------------------------------------------------------
//
// Lane (q, c) = (lane / 16, lane % 16): of S = Q K^T it holds key c and the rows 4 q .. 4 q + 3.
// Keys go through LDS, so that a load brings 1 KB as it lies in memory: with 64 bytes of each of 16 keys, as the operand has them, HBM gave 5.0 TB/s.
// A token for each of 64 sequences of 500 to 8192 keys, 593 MB: 105 us (5.7 TB/s); trees of 4 tokens over an fp8 cache, 312 MB: 73 us.
template <typename T, int D, bool FP8, class W>
__device__ __forceinline__ void few_rows(const ScoreRun& r, W u, int* taken, char* stage, int lane) {
    using C = ScoreCfg<T, D, FP8>;
    constexpr int TURN = C::TURN, NF = C::NF, KSTEPS = C::F ? NF : D / 32;
    const Paged& c = r.c;
    const ScoreArgs& a = r.a;
    const int col = lane & 15, q = lane >> 4, G = (int)r.group.d;
    const float c_log2 = (FP8 ? a.scale * c.kscale : a.scale) * kLog2e;
    const long long begin = u.at;

    // on to the next turn that nobody has; false: none
    auto on = [&](W& v) __attribute__((always_inline)) {
        int k = 0;
        if (lane == 0) k = atomicAdd(taken, 1);
        return v.advance_to(r, begin + same(k));
    };
    // 16 keys lie in one page: a scalar look at the table, and a window that ends at the sequence's last key
    typedef const __attribute__((address_space(4))) int* table_ptr;
    auto page_of = [&](const W& v, int t) __attribute__((always_inline)) {
        const int j = v.chunk * C::FEW + 16 * t;
        const table_ptr trow = (table_ptr)(uintptr_t)(c.table + (size_t)v.b * c.max_pages);
        const int p = j < v.s.len + v.s.n ? same(trow[j >> c.page_log2]) : -1;
        return (unsigned)p < (unsigned)c.P ? p : -1;
    };
    auto fetch = [&](const W& v, int t, int page, u32x4 (&to)[NF]) __attribute__((always_inline)) {
        const int j = v.chunk * C::FEW + 16 * t;
        const char* at = c.k + v.h * c.head_bytes + max(page, 0) * c.page_bytes + (int64_t)(j & ((1 << c.page_log2) - 1)) * C::ROWB;
        const auto w = window(at, page < 0 ? 0 : min(v.s.len + v.s.n - j, 16) * C::ROWB);
#pragma unroll
        for (int i = 0; i < NF; ++i) to[i] = kv_load<2>(w, 1024 * i + 16 * lane);
    };
    u32x4 kreg[TURN][NF], qf[KSTEPS];
    int page[TURN], ahead[TURN];
    float b[4];
    uint32_t counts = 0;
    if (!on(u)) return;
#pragma unroll
    for (int t = 0; t < TURN; ++t) page[t] = page_of(u, t);
#pragma unroll
    for (int t = 0; t < TURN; ++t) fetch(u, t, page[t], kreg[t]);
    __builtin_amdgcn_sched_barrier(0);           // (the queries' way leads over the log-sum-exps: K is asked for before)
    bool fresh = true;                           // the unit's queries are to come
    for (;;) {
        W v = u;
        const bool more = on(v);
        v.settle();
        if (fresh) {
            const int row = min(col, u.rows - 1), token = (int)fast_div((uint32_t)row, r.group);
            const char* qg = static_cast<const char*>(a.q) + ((int64_t)(u.s.row0 + token) * a.q_stride + (int64_t)(u.h * G + row - token * G) * D) * C::QSZ;
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(qg + C::few_at(s, q));
            counts = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = min(4 * q + e, u.rows - 1), token = (int)fast_div((uint32_t)row, r.group);
                const float l = a.lse[(size_t)(u.s.row0 + token) * a.Hq + u.h * G + row - token * G];
                const float w = a.weight != nullptr ? a.weight[u.s.row0 + token] : 1.0f;
                b[e] = bias(l, w, a.weight != nullptr);
                counts |= (uint32_t)(4 * q + e < u.rows && b[e] < __builtin_inff()) << e;
            }
            have_loads();
        }
#pragma unroll
        for (int t = 0; t < TURN; ++t) ahead[t] = more ? page_of(v, t) : -1;
        // the lane writes the scores of the keys `mine` + 64 i
        constexpr int PUT = (TURN + 3) / 4;
        const int mine = u.chunk * C::FEW + lane, keys = u.s.len + u.s.n;
        float* const score = a.score + ((size_t)u.b * c.Hkv + u.h) * a.score_stride;
        float old[PUT], result[PUT];
#pragma unroll
        for (int i = 0; i < PUT; ++i) {
            old[i] = result[i] = 0.0f;
            if (lane < 16 * TURN && mine + 64 * i < u.s.len && a.decay != 0.0f) old[i] = score[mine + 64 * i];
        }
#pragma unroll
        for (int t = 0; t < TURN; ++t) {
            // (the wavefront's own block of LDS, which its accesses reach in their order)
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                const int at = 1024 * i + 16 * lane;
                *reinterpret_cast<u32x4*>(stage + at / C::ROWB * C::KPITCH + at % C::ROWB) = kreg[t][i];
            }
            const int j = u.chunk * C::FEW + 16 * t, there = page[t];
            fetch(v, t, ahead[t], kreg[t]);
            page[t] = ahead[t];
            u32x4 kf[NF];
#pragma unroll
            for (int i = 0; i < NF; ++i) kf[i] = *reinterpret_cast<const u32x4*>(stage + col * C::KPITCH + 64 * i + 16 * q);
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) {
                if constexpr (C::F) {
                    const f32x4 x = __builtin_bit_cast(f32x4, qf[s]), y = __builtin_bit_cast(f32x4, kf[s]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc, 0, 0, 0);
                } else if constexpr (FP8) {
                    const u32x4 y = kf[s >> 1];
                    acc = Few<T>::mfma(qf[s], widen8<T>(y[2 * (s & 1)], y[2 * (s & 1) + 1]), acc);
                } else {
                    acc = Few<T>::mfma(qf[s], kf[s], acc);
                }
            }
            uint32_t bits = counts;
            if (j + 16 > u.s.len) bits &= seen_by<4>(r, u, 0, r.group, 4 * q, j + col - u.s.len);
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = if_bit(bits, e, exp2_fast(fmaf(acc[e], c_log2, -b[e])));
            float sum = (p[0] + p[1]) + (p[2] + p[3]);
            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
            sum = pair_sum(__uint_as_float(x[0]) + __uint_as_float(x[1]));
            if (there < 0) sum = 0.0f;
            result[t / 4] = q == t % 4 ? sum : result[t / 4];
        }
#pragma unroll
        for (int i = 0; i < PUT; ++i) {
            const int key = mine + 64 * i;
            if (lane < 16 * TURN && key < keys) score[key] = key < u.s.len && a.decay != 0.0f ? fmaf(old[i], a.decay, result[i]) : result[i];
        }
        if (!more) return;
        fresh = v.b != u.b || v.h != u.h;
        u = v;
    }
}

template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kScoreThreads, 2) void score_few_kernel(ScoreRun r) {
    using C = ScoreCfg<T, D, FP8>;
    using W = ScoreWalk<C>;
    __shared__ __align__(16) char keys[kScoreWaves][16 * C::KPITCH];
    __shared__ ScoreScratch scratch;
    const int lane = threadIdx.x & 63, wave = same((int)threadIdx.x >> 6);
    long long total[3];
    W::template begin<kFew, kFew>(r, &scratch, total);
    W u;
    if (u.start(r, &scratch, kFew, total[kFew], place_of_group(), kScoreGroups)) few_rows<T, D, FP8>(r, u, &scratch.taken, keys[wave], lane);
}

// ---- many rows -----------------------------------------------------------------------------------
//
// Lane (hh, c) = (lane / 32, lane % 32): of a tile of 32 rows it holds key c of each of KB blocks of 32 keys, and the rows 8 y + 4 hh .. + 3, y = 0 .. 3.
//
// A wavefront keeps its keys' operands in registers, of 16 bits those of 64 keys, or 128 of a turn that the workgroup shares.  A unit's rows lie in LDS for all of its turns
// if they fit, and the wavefronts take turns as they come to them, reading the keys of the next one before they weigh the present: keys bound it, and are to be under way all
// the time (32 tokens after 10000 to 32000 keys, 202 MB: 65 us, and 79 where each wavefront copied the rows a tile ahead for itself and so read its next keys late).
// Of more rows each wavefront of a shared turn takes every eighth tile, copied to a place of its own one ahead, and so waits for nobody.  The exponentials of a block run between
// the products of the next one.  Chunks of 1000 tokens after 2000 to 7000 keys, 138 GFLOP: 207 to 216 us, where rows staged with a barrier for each 128 of them took 251.
// (Without the products 142, without the exponentials 183.)  At d = 128 registers are pushed out: 57 vector and 165 scalar ones of 16 bits, 55 and 89 of f32, 45 and 167 of fp8.
template <typename C> struct ScorePlaces {
    union {
        char tile[kScoreWaves][C::SLOTS][C::TILE];
        char keys[kScoreWaves][16 * C::KPITCH];          // 16 keys of a wavefront, or all of the workgroup's, on their way to the operands
        float sums[kScoreWaves][32 * C::LONG];
        struct {
            char rows[C::OWN][C::TILE];
            char stage[kScoreWaves][16 * C::KPITCH];
        } own;
    };
    float bias[kBiasTiles][32];
};

__device__ __forceinline__ uint32_t lds_at(const void* p) {
    return (uint32_t)same((int)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p);
}
// N loads of 16 bytes per lane, at off[i] of the window, to 1 KB each of LDS from `to` on.  (The compiler does not know of copies under way, and so does not wait for them wherever LDS is
// read.  M0 holds the target, with a wait state before the copy, and is left as it was.)  What was read of LDS before is there first.
template <int N> struct Copies;
template <> struct Copies<4> {
    static __device__ __forceinline__ void start(u32x4 w, uint32_t to, const int* off) {
        uint32_t m0;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %3, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %4, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %5, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %6, %1, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "s"(w), "s"(to), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]) : "memory", "scc");
    }
};
template <> struct Copies<8> {
    static __device__ __forceinline__ void start(u32x4 w, uint32_t to, const int* off) {
        uint32_t m0;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %3, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %4, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %5, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %6, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %7, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %8, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %9, %1, 0 offen lds\n\ts_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
                     "buffer_load_dwordx4 %10, %1, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0)
                     : "s"(w), "s"(to), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "v"(off[4]), "v"(off[5]), "v"(off[6]), "v"(off[7])
                     : "memory", "scc");
    }
};
template <> struct Copies<16> {
    static __device__ __forceinline__ void start(u32x4 w, uint32_t to, const int* off) {
        Copies<8>::start(w, to, off);
        Copies<8>::start(w, to + 8192, off + 8);
    }
};

// The lane's number, asked for anew: what is kept of it across a turn is pushed out of the registers, and reading it back waits for all loads under way
__device__ __forceinline__ int lane_now() {
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
}

template <typename T, int D, bool FP8, int KB, class W> struct ManyRows {
    using C = ScoreCfg<T, D, FP8>;
    static constexpr int MANY = 32 * KB, NM = C::NM, STEPS = C::STEPS, COPIES = C::TILE / 1024;
    const ScoreRun& r;
    const W& u;
    ScorePlaces<C>& lds;
    int wave, lane, keys;
    float c_log2;
    int tpt, hpt, of_token, tiles;       // tokens and heads of a tile, tiles of a token (of tpt), of the unit
    int off[COPIES];                     // of the lane's pieces of a tile from its first row
    int qat;                             // the lane's first operand in a tile; operand s lies at qat ^ many_at(s)

    __device__ __forceinline__ ManyRows(const ScoreRun& run, const W& unit, ScorePlaces<C>& places, int wv, int ln)
        : r(run), u(unit), lds(places), wave(wv), lane(ln), keys(unit.s.len + unit.s.n), c_log2((FP8 ? run.a.scale * run.c.kscale : run.a.scale) * kLog2e) {
        const int G = (int)r.group.d;
        hpt = min(G, 32);
        of_token = (G + 31) / 32;
        tpt = C::tokens(r);
        tiles = C::tiles(r, u.s.n);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) {
            const int row = i * (1024 / C::QROW) + lane / C::CH, token = row / hpt;
            // (rows behind the tile's last lie behind its window)
            off[i] = token < tpt ? (int)(token * r.a.q_stride * C::QSZ) + (row - token * hpt) * C::QROW + 16 * (lane % C::CH ^ C::swz(row)) : 0x7ffffff0;
        }
        qat = (lane & 31) * C::QROW + (16 * C::swz(lane & 31) ^ C::kHalf * (lane >> 5));
    }
    __device__ __forceinline__ int token0(int t) const { return of_token > 1 ? t / of_token : t * tpt; }
    __device__ __forceinline__ int head0(int t) const { return of_token > 1 ? t % of_token * 32 : 0; }

    // The bias of the rows of tiles t0 .. t1 - 1, by the threads `me` of `all`
    __device__ __forceinline__ void put_bias(float (*to)[32], int t0, int t1, int me, int all) const {
        const int G = (int)r.group.d;
        for (int i = me; i < 32 * (t1 - t0); i += all) {
            const int t = t0 + i / 32, row = i % 32, token = row / hpt, head = head0(t) + row - token * hpt, at = token0(t) + token;
            float bs = __builtin_inff();
            if (token < tpt && at < u.s.n && head < G)
                bs = bias(r.a.lse[(size_t)(u.s.row0 + at) * r.a.Hq + u.h * G + head], r.a.weight != nullptr ? r.a.weight[u.s.row0 + at] : 1.0f, r.a.weight != nullptr);
            to[i / 32][row] = bs;
        }
    }

    // 16 keys of the turn, as they lie in memory, 1 KB to a load; zeros behind the sequence's last key and where there is no page
    __device__ __forceinline__ int page_of(int i) const {
        typedef const __attribute__((address_space(4))) int* table_ptr;
        const table_ptr trow = (table_ptr)(uintptr_t)(r.c.table + (size_t)u.b * r.c.max_pages);
        const int j = u.chunk * MANY + 16 * i;
        const int p = j < keys ? same(trow[j >> r.c.page_log2]) : -1;
        return (unsigned)p < (unsigned)r.c.P ? p : -1;
    }
    __device__ __forceinline__ void fetch(int i, int page, int me, u32x4 (&k)[NM / 2]) const {
        const int j = u.chunk * MANY + 16 * i;
        const char* at = r.c.k + u.h * r.c.head_bytes + max(page, 0) * r.c.page_bytes + (int64_t)(j & ((1 << r.c.page_log2) - 1)) * C::ROWB;
        const auto w = window(at, page < 0 ? 0 : min(keys - j, 16) * C::ROWB);
#pragma unroll
        for (int x = 0; x < NM / 2; ++x) k[x] = kv_load<0>(w, 16 * me + 1024 * x);
    }
    __device__ __forceinline__ void stage(char* to, const u32x4 (&k)[NM / 2]) const {
#pragma unroll
        for (int i = 0; i < NM / 2; ++i) {
            const int at = 1024 * i + 16 * lane;
            *reinterpret_cast<u32x4*>(to + at / C::ROWB * C::KPITCH + at % C::ROWB) = k[i];
        }
    }
    static __device__ __forceinline__ void widen(const u32x4 (&x)[NM], u32x4 (&kf)[STEPS]) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if constexpr (FP8) kf[s] = widen8<T>(x[s >> 1][2 * (s & 1)], x[s >> 1][2 * (s & 1) + 1]);
            else kf[s] = x[s];
        }
    }
    // whether the lane's key of block b has a page
    __device__ __forceinline__ uint32_t has_page(int b, int p0, int p1) const {
        return u.chunk * MANY + 32 * b + (lane & 31) < keys && ((lane & 16) != 0 ? p1 : p0) >= 0;
    }
    // The turn's keys through LDS to the operands, by a wavefront for itself or by the workgroup.  there: whether the lane's keys have pages, a bit for each block.
    struct Own {
        u32x4 k[2 * KB][NM / 2];
        int page[2 * KB];
    };
    __device__ __forceinline__ void fetch(Own& x) const {
#pragma unroll
        for (int i = 0; i < 2 * KB; ++i) x.page[i] = page_of(i);
        const int me = lane_now();
#pragma unroll
        for (int i = 0; i < 2 * KB; ++i) fetch(i, x.page[i], me, x.k[i]);
    }
    __device__ __forceinline__ void own_keys(const Own& own, u32x4 (&kf)[KB][STEPS], uint32_t& there) const {
        char* const mine = lds.own.stage[wave];          // (its accesses reach it in their order)
        there = 0;
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            there |= has_page(b, own.page[2 * b], own.page[2 * b + 1]) << b;
            u32x4 x[NM];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                stage(mine, own.k[2 * b + half]);
                if ((lane >> 4 & 1) == half) {
#pragma unroll
                    for (int i = 0; i < NM; ++i) x[i] = *reinterpret_cast<const u32x4*>(mine + (lane & 15) * C::KPITCH + 32 * i + 16 * (lane >> 5));
                }
            }
            widen(x, kf[b]);
        }
    }
    template <class Meanwhile> __device__ __forceinline__ void shared_keys(u32x4 (&kf)[KB][STEPS], uint32_t& there, const Meanwhile& meanwhile) const {
        static_assert(2 * KB <= kScoreWaves, "16 keys to a wavefront");
        u32x4 k[NM / 2];
        if (wave < 2 * KB) fetch(wave, page_of(wave), lane, k);
        meanwhile();
        if (wave < 2 * KB) stage(lds.keys[wave], k);
        there = 0;
#pragma unroll
        for (int b = 0; b < KB; ++b) there |= has_page(b, page_of(2 * b), page_of(2 * b + 1)) << b;
        __syncthreads();
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            u32x4 x[NM];
#pragma unroll
            for (int i = 0; i < NM; ++i)
                x[i] = *reinterpret_cast<const u32x4*>(lds.keys[2 * b + (lane >> 4 & 1)] + (lane & 15) * C::KPITCH + 32 * i + 16 * (lane >> 5));
            widen(x, kf[b]);
        }
    }

    // the copies of a tile of rows
    __device__ __forceinline__ void start(int t, const char* to) const {
        const int t0 = token0(t), h0 = head0(t), G = (int)r.group.d;
        const int64_t stride = r.a.q_stride * C::QSZ;
        const uint64_t from = (uint64_t)(static_cast<const char*>(r.a.q) + (u.s.row0 + t0) * stride + (int64_t)(u.h * G + h0) * C::QROW);
        const int bytes = (int)((min(tpt, u.s.n - t0) - 1) * stride) + min(hpt, G - h0) * C::QROW;
        const u32x4 w = {(uint32_t)same((int)from), (uint32_t)same((int)(from >> 32)), (uint32_t)same(bytes), 0x00020000u};
        Copies<COPIES>::start(w, lds_at(to), off);
    }
    // waits until all but the last LOADS loads and copies have landed
    template <int LOADS> static __device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory"); }

    static __device__ __forceinline__ void multiply(u32x4 q, u32x4 k, f32x16& acc) {
        if constexpr (C::F) {
            const f32x4 y = __builtin_bit_cast(f32x4, q), z = __builtin_bit_cast(f32x4, k);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(y[e], z[e], acc, 0, 0, 0);
        } else {
            acc = Mma<T>::mfma(q, k, acc);
        }
    }
    // The weights of one tile and all blocks, added to part.  The exponentials of a block run between the products of the next: an in-order wavefront would else wait
    // for one product after the other, and for the exponentials in turn.
    template <bool MASKED>
    __device__ __forceinline__ void weigh_tile(const u32x4 (&q)[STEPS], const u32x4 (&kf)[KB][STEPS], const f32x4 (&b)[4], const uint32_t (&bits)[KB],
                                               float (&sum)[KB]) const {
        constexpr int PER = 16 / STEPS;          // weights of a block to an operand
        static_assert(STEPS == 4 || STEPS == 8 || STEPS == 16, "weights are dealt out over the operands");
        f32x16 acc[2];
#pragma unroll
        for (int k = 0; k <= KB; ++k) {
            f32x4 part = {0.0f, 0.0f, 0.0f, 0.0f};
            if (k < KB) {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[k & 1][e] = 0.0f;
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if (k < KB) multiply(q[s], kf[k < KB ? k : 0][s], acc[k & 1]);
                if (k > 0) {
#pragma unroll
                    for (int i = s * PER; i < s * PER + PER; ++i) {
                        float p = exp2_fast(fmaf(acc[(k - 1) & 1][i], c_log2, -b[i >> 2][i & 3]));
                        if (MASKED) p = b[i >> 2][i & 3] < __builtin_inff() ? if_bit(bits[k > 0 ? k - 1 : 0], i, p) : 0.0f;
                        part[i & 3] = i < 4 ? p : part[i & 3] + p;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (k > 0) sum[k > 0 ? k - 1 : 0] += (part[0] + part[1]) + (part[2] + part[3]);
        }
    }

    // Tiles, whose bias begins at `from` with that of tile `base`
    struct Tiles {
        const float (*from)[32];
        int base, clear;                 // clear: tokens from this one on see all of the keys
        uint32_t there;
    };
    __device__ __forceinline__ void tile(const Tiles& x, int t, int next, const char* at, const u32x4 (&kf)[KB][STEPS], float (&sum)[KB]) const {
        u32x4 q[STEPS];
        f32x4 b[4];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q[s] = *reinterpret_cast<const u32x4*>(at + (qat ^ C::many_at(s)));
#pragma unroll
        for (int y = 0; y < 4; ++y) b[y] = *reinterpret_cast<const f32x4*>(&x.from[t - x.base][8 * y + 4 * (lane >> 5)]);
        if (next >= 0) start(next, at);
        // (a row that does not count has an infinite bias: one of them in 8 y + 4 hh .. + 3 makes the sum of those infinite, or NaN)
        bool off_rows = false;
#pragma unroll
        for (int y = 0; y < 4; ++y) off_rows |= !((b[y][0] + b[y][1]) + (b[y][2] + b[y][3]) < __builtin_inff());
        uint32_t bits[KB];
#pragma unroll
        for (int k = 0; k < KB; ++k) bits[k] = 0;
        // A row that does not count takes nothing, e^(s - inf) = 0, but for a product that is infinite or no number; then the tile is weighed again with the masks.
        bool masks = token0(t) < x.clear;
        if (!masks) {
            float before[KB];
#pragma unroll
            for (int k = 0; k < KB; ++k) before[k] = sum[k];
            weigh_tile<false>(q, kf, b, bits, sum);
            if (__builtin_amdgcn_ballot_w64(off_rows) != 0) {
                bool odd = false;
#pragma unroll
                for (int k = 0; k < KB; ++k) odd |= !(sum[k] < __builtin_inff());
                masks = __builtin_amdgcn_ballot_w64(odd) != 0;
                if (masks) {
#pragma unroll
                    for (int k = 0; k < KB; ++k) sum[k] = before[k];
                }
            }
        }
        if (masks) {
#pragma unroll
            for (int k = 0; k < KB; ++k)
                bits[k] = (x.there >> k & 1u) != 0 ? seen_by<16>(r, u, token0(t), of_token > 1 ? FastDiv{32, 0, 0, 31} : r.group, 4 * (lane >> 5),
                                                                 u.chunk * MANY + 32 * k + (lane & 31) - u.s.len)
                                                   : 0u;
            weigh_tile<true>(q, kf, b, bits, sum);
        }
    }
    // there: of the lane's keys
    __device__ __forceinline__ Tiles tiles_of(const float (*from)[32], int base, uint32_t there) const {
        const int j0 = u.chunk * MANY;
        const bool all_there = __builtin_amdgcn_ballot_w64(there != (1u << KB) - 1u) == 0;
        // (none before the end in a tree's new keys)
        return Tiles{from, base, !all_there ? 0x7fffffff : j0 + MANY <= u.s.len ? 0 : r.a.tree == nullptr ? j0 + MANY - 1 - u.s.len : 0x7fffffff, there};
    }
    __device__ __forceinline__ void run(int t, int end, const u32x4 (&kf)[KB][STEPS], const Tiles& x, float (&sum)[KB]) const {
        constexpr int step = kScoreWaves;
        if (t >= end) return;
        const char (*const slots)[C::TILE] = lds.tile[wave];
        start(t, slots[0]);
        int slot = 0;
        if constexpr (C::SLOTS == 2) {
            if (t + step < end) start(t + step, slots[1]);
        }
#pragma unroll 1
        for (; t + step < end; t += step) {
            if constexpr (C::SLOTS == 2) {
                landed<COPIES>();
                tile(x, t, t + 2 * step < end ? t + 2 * step : -1, slots[slot], kf, sum);
                slot ^= 1;
            } else {
                landed<0>();
                tile(x, t, t + step, slots[0], kf, sum);
            }
        }
        landed<0>();
        tile(x, t, -1, slots[slot], kf, sum);
    }
    // A turn: sum is over half of the rows, the other half is in the other half of the lanes.
    __device__ __forceinline__ int first_tile() const {
        // a chain's first one with a row that sees a key of the turn
        const int rel = u.chunk * MANY - u.s.len;
        return r.a.tree == nullptr && rel > 0 ? rel / tpt * of_token : 0;
    }
    // The unit's tiles and their bias, by the workgroup
    __device__ __forceinline__ void take_rows() const {
        for (int t = wave; t < tiles; t += kScoreWaves) start(t, lds.own.rows[t]);
        put_bias(lds.bias, 0, tiles, threadIdx.x, kScoreThreads);
        landed<0>();
    }
    // `ahead` starts loads of the next turn's keys
    template <class Ahead> __device__ __forceinline__ void own_turn(const Own& own, float (&sum)[KB], const Ahead& ahead) const {
        u32x4 kf[KB][STEPS];
        uint32_t there;
#pragma unroll
        for (int k = 0; k < KB; ++k) sum[k] = 0.0f;
        own_keys(own, kf, there);
        ahead();
        const Tiles x = tiles_of(lds.bias, 0, there);
#pragma unroll 1
        for (int t = first_tile(); t < tiles; ++t) tile(x, t, -1, lds.own.rows[t], kf, sum);
    }
    __device__ __forceinline__ void shared_turn(float (&sum)[KB]) const {
        u32x4 kf[KB][STEPS];
        uint32_t there;
#pragma unroll
        for (int k = 0; k < KB; ++k) sum[k] = 0.0f;
        int base = first_tile(), end = min(base + kBiasTiles, tiles);
        // (nobody reads the turn before any more)
        shared_keys(kf, there, [&] { put_bias(lds.bias, base, end, threadIdx.x, kScoreThreads); });
        for (;;) {
            __syncthreads();             // the keys have been read, and the bias is there
            have_loads();
            run(base + wave, end, kf, tiles_of(lds.bias, base, there), sum);
            base = end;
            if (base >= tiles) return;
            end = min(base + kBiasTiles, tiles);
            __syncthreads();             // the tiles before have been read
            put_bias(lds.bias, base, end, threadIdx.x, kScoreThreads);
        }
    }
    // The sum over all rows of the turn's key `j` becomes its score.
    __device__ __forceinline__ void put(int j, float all) const {
        if (j < keys) {
            float* to = r.a.score + ((size_t)u.b * r.c.Hkv + u.h) * r.a.score_stride + j;
            *to = j < u.s.len && r.a.decay != 0.0f ? fmaf(*to, r.a.decay, all) : all;
        }
    }
};

template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kScoreThreads, 2) void score_many_kernel(ScoreRun r) {
    using C = ScoreCfg<T, D, FP8>;
    using W = ScoreWalk<C>;
    __shared__ __align__(1024) ScorePlaces<C> places;
    __shared__ ScoreScratch scratch;
    const int lane = threadIdx.x & 63, wave = same((int)threadIdx.x >> 6), w = place_of_group();
    long long total[3];
    W::template begin<kMid, kLong>(r, &scratch, total);
    W u;
    for (long long i = 0; i < total[kLong]; i += kScoreGroups) {
        const long long x = i + ((i & kScoreGroups) != 0 ? kScoreGroups - 1 - w : w);
        if (x >= total[kLong]) continue;
        u.end = 0;
        u.take(r, &scratch, kLong, x);
        const ManyRows<T, D, FP8, C::LONG, W> m(r, u, places, wave, lane);
        float sum[C::LONG];
        m.shared_turn(sum);
        __syncthreads();                 // all tiles have been read
#pragma unroll
        for (int k = 0; k < C::LONG; ++k) {
            const float all = pair_sum(sum[k]);
            if (lane < 32) places.sums[wave][32 * k + lane] = all;
        }
        // the wavefronts' sums one after the other
        __syncthreads();
        for (int j = threadIdx.x; j < 32 * C::LONG; j += kScoreThreads) {
            float all = 0.0f;
#pragma unroll
            for (int v = 0; v < kScoreWaves; ++v) all += places.sums[v][j];
            m.put(u.chunk * 32 * C::LONG + j, all);
        }
        __syncthreads();
    }
    if (!u.start(r, &scratch, kMid, total[kMid], w, kScoreGroups)) return;
    using M = ManyRows<T, D, FP8, C::MID, W>;
    for (;;) {
        // the turns of the stretch that are this unit's: the wavefronts begin with one each, and take more as they come to them
        const int from = u.chunk, n = (int)min((long long)(u.chunks - from), u.end - u.at);
        bool any = wave < n;
        u.chunk = from + wave;
        typename M::Own own;
        if (any) M(r, u, places, wave, lane).fetch(own);
        __syncthreads();                 // the unit before is done
        if (threadIdx.x == 0) scratch.taken = kScoreWaves;
        M(r, u, places, wave, lane).take_rows();
        __syncthreads();
        while (any) {
            const M m(r, u, places, wave, lane);
            W v = u;
            float sum[C::MID];
            m.own_turn(own, sum, [&] {
                int k = 0;
                if (lane == 0) k = atomicAdd(&scratch.taken, 1);
                k = same(k);
                any = k < n;
                v.chunk = from + k;
                if (any) M(r, v, places, wave, lane).fetch(own);
            });
#pragma unroll
            for (int k = 0; k < C::MID; ++k) {
                const float all = pair_sum(sum[k]);
                const int me = lane_now();
                if (me < 32) m.put(u.chunk * 32 * C::MID + 32 * k + me, all);
            }
            u.chunk = v.chunk;
        }
        u.chunk = from;
        if (!u.advance_to(r, u.at + n)) return;
    }
}

template <typename T, int D, bool FP8>
static hipError_t launch_score_d(const ScoreRun& r, hipStream_t st) {
    // (units of more than a few rows: there are none where all of the call's rows are not more)
    if ((int64_t)r.c.T * r.group.d > kFewRows) {
        hipLaunchKernelGGL((score_many_kernel<T, D, FP8>), dim3(kScoreGroups), dim3(kScoreThreads), 0, st, r);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (r.group.d > kFewRows) return hipSuccess;
    hipLaunchKernelGGL((score_few_kernel<T, D, FP8>), dim3(kScoreGroups), dim3(kScoreThreads), 0, st, r);
    return hipGetLastError();
}
template <typename T, bool FP8>
static hipError_t launch_score_t(const ScoreRun& r, hipStream_t st) {
    return r.c.d == 64 ? launch_score_d<T, 64, FP8>(r, st) : launch_score_d<T, 128, FP8>(r, st);
}

hipError_t launch_cache_score(const Paged& c, const ScoreArgs& a, hipStream_t st) {
    ScoreRun r;
    r.c = c;
    r.a = a;
    r.group = make_fast_div((uint32_t)(a.Hq / c.Hkv));
    switch (a.dtype) {
    case 0: return launch_score_t<F32, false>(r, st);
    case 1: return a.fp8 ? launch_score_t<F16, true>(r, st) : launch_score_t<F16, false>(r, st);
    default: return a.fp8 ? launch_score_t<BF16, true>(r, st) : launch_score_t<BF16, false>(r, st);
    }
}

}  // namespace flashd
