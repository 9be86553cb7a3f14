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
// By the rows of a sequence and kv head there are three ways:
//   few   (up to 16) HBM bounds it.  Products of 16 x 16 x 32; a wavefront by itself has the queries in registers and takes 64 or 128 keys at a time, the
//         next ones under way.
//   mid   (one group of rows: 128, of f32 64) HBM, and products and exponentials.  32 x 32 x 16; the rows stay in LDS, a wavefront takes 32 keys
//         at a time, the next 64 under way.
//   long  Products and exponentials.  A workgroup keeps 256 keys while the rows go by in LDS, group by group, the next one under way; a
//         wavefront has 64 of the keys and every other tile of rows.  (With 32 keys and all tiles LDS bounded it: an operand of 1 KB read for every
//         product.)
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

#include <type_traits>

namespace flashd {

constexpr int kScoreWaves = 8, kScoreThreads = kScoreWaves * kWave;
constexpr int kScoreGroups = 256;       // workgroups of a launch: one per compute unit, two wavefronts per SIMD

struct ScoreRun {
    Paged c;
    ScoreArgs a;
    FastDiv group;          // query heads per kv head
};

template <typename T, int D, bool FP8> struct ScoreCfg {
    static constexpr bool F = std::is_same_v<T, F32>;
    static constexpr int ROWB = D * (F ? 4 : FP8 ? 1 : 2);       // bytes of a key
    static constexpr int QSZ = F ? 4 : 2;
    // few: 16-key blocks of a wavefront's turn, and loads of 16 bytes per lane and block
    static constexpr int TURN = ROWB >= 512 ? 2 : ROWB >= 256 ? 4 : 8;
    static constexpr int FEW = 16 * TURN;
    static constexpr int NF = ROWB / 64;
    static constexpr int KPITCH = ROWB + 16;                     // of a key of the block in LDS
    // mid and long: keys of a workgroup's turn; loads of a lane for 32 keys, 2 lanes to 32 bytes
    static constexpr int MANY = 32 * kScoreWaves;
    static constexpr int NM = ROWB / 32;
    // long: 32-key blocks of a wavefront, and wavefronts that share out the tiles of rows (f32 has no registers for the keys of two)
    static constexpr int KB = F ? 1 : 2;
    // rows of a group in LDS, padded so that 16 of them fall on all banks
    static constexpr int ROWS = F ? 64 : 128;
    static constexpr int PITCH = D * QSZ + 16;
    static constexpr int STEPS = D * QSZ / 32;                   // operands of a lane
    static constexpr int QL = ROWS * D * QSZ / (16 * kScoreThreads);
    // Tokens of a group: with all their heads, or one where that is more than a group's rows, or where offsets within the group would pass 32 bits
    static __device__ __forceinline__ int tokens(const ScoreRun& r) {
        const int heads = (int)r.group.d;
        return heads > ROWS || r.a.q_stride * QSZ * ROWS > (1ll << 30) ? 1 : ROWS / heads;
    }
    // Byte of a row at which a lane's operand s begins, in the order in which the loads of K bring the elements: of fp8 16 at a time
    static __device__ __forceinline__ int few_at(int s, int q) { return FP8 ? 128 * (s >> 1) + 32 * q + 16 * (s & 1) : 64 * s + 16 * q; }
    static __device__ __forceinline__ int many_at(int s, int hh) { return FP8 ? 64 * (s >> 1) + 32 * hh + 16 * (s & 1) : 32 * s + 16 * hh; }
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
// The same for these registers alone
template <int N> __device__ __forceinline__ void have(u32x4 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// a / b rounded up, of whole numbers 0 <= a < 2^52 and b > 0, by a division of doubles (the rounded quotient's ceiling can be one off)
__device__ __forceinline__ long long ceil_div(long long a, long long b) {
    long long q = (long long)((double)a / (double)b);
    q = q * b >= a ? q : q + 1;
    return (q - 1) * b >= a ? q - 1 : q;
}

// ---- the work of a launch -----------------------------------------------------------------------
//
// Units are (sequence, kv head), cut into turns of keys.  Turns of few rows lie in a row of which each workgroup has a stretch, those of mid ones in
// another.  Turns of long units take many times what
// it takes to bring their keys: turn i of all of them is that of workgroup i modulo their number, every other time backwards, in the order of falling
// rows (up to 512 sequences), so that none has much more than another.
enum ScoreKind { kFew, kMid, kLong };

struct ScoreScratch {
    long long first[3][kScoreThreads];   // of each thread's run of sequences: turns of all runs before
    long long sum[3][kScoreWaves];
    int rows[kScoreThreads];
    int order[kScoreThreads];            // long ones: sequences by falling rows
    int taken;                           // turns of the workgroup's stretch of few rows
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
        kind = rows <= 16 ? kFew : rows <= C::ROWS && s.n <= C::tokens(r) ? kMid : kLong;
        const int keys = kind == kFew ? C::FEW : C::MANY;
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
    static __device__ __forceinline__ int each(const ScoreRun& r) { return (r.c.B + kScoreThreads - 1) / kScoreThreads; }

    // Every thread takes a run of sequences, whose turns are then summed over the threads.
    static __device__ __forceinline__ void begin(const ScoreRun& r, ScoreScratch* sh, long long (&total)[3]) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int n = each(r), b0 = tid * n, b1 = min(b0 + n, r.c.B);
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
        if (n == 1 && __syncthreads_or(mine[kLong] != 0)) {
            const int rows = any.kind == kLong ? any.rows : -1;
            sh->rows[tid] = rows;
            sh->first[kLong][tid] = mine[kLong];
            __syncthreads();
            int rank = 0;
            for (int i = 0; i < kScoreThreads; ++i) rank += sh->rows[i] > rows || (sh->rows[i] == rows && i < tid);
            sh->order[rank] = tid;
            __syncthreads();
            mine[kLong] = sh->first[kLong][sh->order[tid]];
            __syncthreads();
        }
        long long in[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            in[k] = mine[k];
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const long long y = __shfl_up(in[k], d);
                if (lane >= d) in[k] += y;
            }
            if (lane == 63) sh->sum[k][wave] = in[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            long long before = in[k] - mine[k];
            total[k] = 0;
#pragma unroll
            for (int i = 0; i < kScoreWaves; ++i) {
                before += i < wave ? sh->sum[k][i] : 0;
                total[k] += sh->sum[k][i];
            }
            total[k] = same(total[k]);
            sh->first[k][tid] = before;
        }
        __syncthreads();
    }
    // Turn x (below the total) of the list of a kind; every wavefront for itself.
    __device__ __forceinline__ void take(const ScoreRun& r, const ScoreScratch* sh, int of, long long x) {
        // the last run that does not begin behind it
        const int lane = threadIdx.x & 63;
        int run = -1;
#pragma unroll
        for (int i = 0; i < kScoreThreads; i += kWave) {
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
    // Turns of this unit from the present one on that are the stretch's
    __device__ __forceinline__ int here() const { return same(end - at < chunks - chunk ? (int)(end - at) : chunks - chunk); }
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
    // past n turns of this unit
    __device__ __forceinline__ bool advance(const ScoreRun& r, int n) {
        at += n;
        if (at >= end) return false;
        chunk = 0;
        if (++h == r.c.Hkv) {
            const int of = kind;
            do enter(r, b + 1);                  // (there is one: the stretch has turns left)
            while (turns(r, of) == 0);
            h = 0;
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
//
// The wavefronts of a workgroup take the turns of its stretch one by one as they come to them: of the two on a SIMD the older one is served first, and with stretches
// of their own the older ones ended after 66 us, the younger after 112 (a token for each of 64 sequences of 500 to 8192 keys).
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

// ---- mid and long --------------------------------------------------------------------------------
//
// Lane (hh, c) = (lane / 32, lane % 32): of a tile of 32 rows it holds key c (of each of KB blocks) and the rows 8 y + 4 hh .. + 3, y = 0 .. 3.
template <typename C> struct ScoreRows {
    char q[2][C::ROWS * C::PITCH];
    float bias[2][C::ROWS];
    int off[2][kScoreWaves];             // some row of the group does not count
    float sums[kScoreWaves / 2][64];     // of wavefronts that share their keys
};

template <typename T, int D, bool FP8, int KB, class W> struct ManyRows {
    using C = ScoreCfg<T, D, FP8>;
    static constexpr int NM = C::NM, STEPS = C::STEPS, ROWS = C::ROWS, PITCH = C::PITCH, QL = C::QL, CPR = D * C::QSZ / 16;
    const ScoreRun& r;
    const W& u;
    ScoreRows<C>& lds;
    int wave, lane, keys;
    int lead, odd;               // the wavefront's first key in a turn, and its first tile: it has every KB-th
    float c_log2;
    const char* pool;
    // A group: `tpg` tokens with all their heads (one token and `hpg` of them where they are more than ROWS); its row i is head i % hpg of
    // token i / hpg.  So the lane's pieces of a group lie at fixed distances from its first token.
    int tpg, hpg, of_token;      // of_token: groups of a token (of tpg tokens)
    int voff[QL], brow;

    __device__ __forceinline__ ManyRows(const ScoreRun& run, const W& unit, ScoreRows<C>& rows, int wv, int ln)
        : r(run), u(unit), lds(rows), wave(wv), lane(ln), keys(unit.s.len + unit.s.n), lead(32 * KB * (wv / KB)), odd(wv % KB),
          c_log2((FP8 ? run.a.scale * run.c.kscale : run.a.scale) * kLog2e), pool(run.c.k + unit.h * run.c.head_bytes) {
        const int G = (int)r.group.d, tid = wave * kWave + lane;
        const int64_t stride = r.a.q_stride * C::QSZ;
        hpg = min(G, ROWS);
        of_token = (G + ROWS - 1) / ROWS;
        tpg = C::tokens(r);
#pragma unroll
        for (int i = 0; i < QL; ++i) {
            const int at = i * kScoreThreads + tid, row = at / CPR, token = row / hpg;
            // (rows behind the group's last lie behind its window)
            voff[i] = token < tpg ? (int)(token * stride) + (row - token * hpg) * (D * C::QSZ) + 16 * (at % CPR) : 0x7ffffff0;
        }
        brow = tid / hpg;
    }
    __device__ __forceinline__ int count() const { return (u.s.n + tpg - 1) / tpg * of_token; }
    __device__ __forceinline__ int token0(int g) const { return of_token > 1 ? g / of_token : g * tpg; }
    __device__ __forceinline__ int head0(int g) const { return of_token > 1 ? g % of_token * ROWS : 0; }
    __device__ __forceinline__ int rows_in(int g) const { return min(tpg, u.s.n - token0(g)) * min(hpg, (int)r.group.d - head0(g)); }

    // Rows on their way to LDS, and what their bias is made of (-infinity: no row)
    __device__ __forceinline__ void load_rows(int g, u32x4 (&x)[QL], float& l, float& wt) const {
        const int tid = wave * kWave + lane, G = (int)r.group.d, t0 = token0(g), h0 = head0(g), tokens = min(tpg, u.s.n - t0);
        const int64_t stride = r.a.q_stride * C::QSZ;
        const char* from = static_cast<const char*>(r.a.q) + (u.s.row0 + t0) * stride + (int64_t)(u.h * G + h0) * (D * C::QSZ);
        const auto w = window(from, (int)((tokens - 1) * stride) + min(hpg, G - h0) * (D * C::QSZ));
#pragma unroll
        for (int i = 0; i < QL; ++i) x[i] = kv_load<0>(w, voff[i]);
        const int head = h0 + tid - brow * hpg;
        const bool row = tid < ROWS && brow < tokens && head < G;
        l = -__builtin_inff();
        wt = 1.0f;
        if (row) l = r.a.lse[(size_t)(u.s.row0 + t0 + brow) * r.a.Hq + u.h * G + head];
        if (row && r.a.weight != nullptr) wt = r.a.weight[u.s.row0 + t0 + brow];
    }
    __device__ __forceinline__ void store_rows(int slot, const u32x4 (&x)[QL], float l, float wt) const {
        const int tid = wave * kWave + lane;
#pragma unroll
        for (int i = 0; i < QL; ++i) {
            const int at = i * kScoreThreads + tid;
            *reinterpret_cast<u32x4*>(&lds.q[slot][(at / CPR) * PITCH + 16 * (at % CPR)]) = x[i];
        }
        if (tid < ROWS) {
            const float bs = bias(l, wt, r.a.weight != nullptr);
            lds.bias[slot][tid] = bs;
            const bool off = __builtin_amdgcn_ballot_w64(!(bs < __builtin_inff())) != 0;
            if (lane == 0) lds.off[slot][wave] = off;
        }
    }
    __device__ __forceinline__ bool off(int slot) const {
        int any = 0;
#pragma unroll
        for (int i = 0; i < ROWS / kWave; ++i) any |= lds.off[slot][i];
        return same(any) != 0;
    }

    __device__ __forceinline__ int key_of(int chunk, int kb) const { return chunk * C::MANY + lead + 32 * kb + (lane & 31); }
    __device__ __forceinline__ int page_of(int chunk, int kb, int last) const {
        const int j = key_of(chunk, kb);
        return chunk < last && j < keys ? page_at(r.c, u.b, j >> r.c.page_log2) : -1;
    }
    __device__ __forceinline__ void fetch(int chunk, int kb, int page, u32x4 (&to)[NM]) const {
        // (a key without a page reads the pool's first: its column of products is dropped)
        const int j = key_of(chunk, kb) & ((1 << r.c.page_log2) - 1);
        const char* from = pool + (page < 0 ? 0 : page * r.c.page_bytes + (int64_t)j * C::ROWB) + 16 * (lane >> 5);
#pragma unroll
        for (int i = 0; i < NM; ++i) to[i] = *reinterpret_cast<const u32x4*>(from + 32 * i);
    }
    static __device__ __forceinline__ void widen(const u32x4 (&k)[NM], u32x4 (&kf)[STEPS]) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if constexpr (FP8) kf[s] = widen8<T>(k[s >> 1][2 * (s & 1)], k[s >> 1][2 * (s & 1) + 1]);
            else kf[s] = k[s];
        }
    }
    // tokens before it see none of the wavefront's keys (of a chain; all tokens where there are no keys)
    __device__ __forceinline__ int first_token(int chunk) const {
        const int j0 = chunk * C::MANY + lead;
        return j0 >= keys ? u.s.n : r.a.tree == nullptr ? max(j0 - u.s.len, 0) : 0;
    }

    // Operand s of tile t of the group in `slot`, and the bias of its rows 8 y + 4 hh .. + 3
    __device__ __forceinline__ u32x4 operand(int t, int slot, int s) const {
        return *reinterpret_cast<const u32x4*>(&lds.q[slot][(32 * t + (lane & 31)) * PITCH + C::many_at(s, lane >> 5)]);
    }
    __device__ __forceinline__ f32x4 bias_at(int t, int slot, int y) const {
        return *reinterpret_cast<const f32x4*>(&lds.bias[slot][32 * t + 8 * y + 4 * (lane >> 5)]);
    }
    static __device__ __forceinline__ void multiply(u32x4 q, u32x4 k, f32x16& acc) {
        if constexpr (C::F) {
            const f32x4 y = __builtin_bit_cast(f32x4, q), z = __builtin_bit_cast(f32x4, k);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(y[e], z[e], acc, 0, 0, 0);
        } else {
            acc = Mma<T>::mfma(q, k, acc);
        }
    }
    // A tile whose products are there and whose weights are not
    struct Pending {
        f32x16 acc[KB];
        f32x4 b[4];
        bool any;
    };
    // The weights of the pending tile are added to part; in between, NEXT: the products of a tile (operands q).  An in-order wavefront would else wait for one
    // product after the other, and for the exponentials in turn.  The operands that are used up are read for tile `then`.
    template <bool NEXT>
    __device__ __forceinline__ void step(Pending& w, u32x4 (&q)[STEPS], const u32x4 (&kf)[KB][STEPS], int then, int slot, f32x4 (&part)[KB]) const {
        constexpr int PER = 16 / STEPS;          // weights of a block to an operand
        static_assert(STEPS == 4 || STEPS == 8 || STEPS == 16, "weights are dealt out over the operands");
        f32x16 next[KB];
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e) next[k][e] = 0.0f;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                if (NEXT) multiply(q[s], kf[k][s], next[k]);
                if (NEXT && k == KB - 1) q[s] = operand(then, slot, s);
#pragma unroll
                for (int i = s * PER; i < s * PER + PER; ++i) part[k][i & 3] += exp2_fast(fmaf(w.acc[k][i], c_log2, -w.b[i >> 2][i & 3]));
                if (NEXT) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (NEXT) {
#pragma unroll
            for (int k = 0; k < KB; ++k) w.acc[k] = next[k];
        }
    }
    __device__ __forceinline__ void finish(Pending& w, const u32x4 (&kf)[KB][STEPS], f32x4 (&part)[KB]) const {
        u32x4 none[STEPS];
        if (w.any) step<false>(w, none, kf, 0, 0, part);
        w.any = false;
    }
    // The wavefront's tiles of the group in `slot`, of tokens from `from` on, the last of which may stay pending.  `first`: what the tile pending so far is added to.
    __device__ __forceinline__ void tiles(int chunk, int g, int slot, const u32x4 (&kf)[KB][STEPS], int from, const bool (&there)[KB], bool all_there,
                                          Pending& w, f32x4 (&first)[KB], f32x4 (&part)[KB]) const {
        const int j0 = chunk * C::MANY + lead, rel = j0 + (lane & 31) - u.s.len;
        const int t0 = token0(g), n = (rows_in(g) + 31) / 32;
        int t = from >= u.s.n ? n : min(max(from - t0, 0), tpg) * hpg / 32;
        // tiles from `clear` on have only rows that count and see all of the wavefront's keys: of a chain those from the last key's token on
        const int clear = off(slot) || !all_there ? n
                          : j0 + 32 * KB <= u.s.len ? t
                          : r.a.tree != nullptr || of_token > 1 ? n
                                                                : (min(max(j0 + 32 * KB - 1 - u.s.len - t0, 0), tpg) * hpg + 31) / 32;
        t += (t ^ odd) & (KB - 1);
        if (t < min(clear, n) || t >= n) finish(w, kf, first);
#pragma unroll 1
        for (; t < min(clear, n); t += KB) {
            const FastDiv heads = of_token > 1 ? FastDiv{(uint32_t)ROWS, 0, 0, 31} : r.group;
#pragma unroll 1
            for (int k = 0; k < KB; ++k) {
                const uint32_t bits = (k == 0 ? there[0] : there[KB - 1]) ? seen_by<16>(r, u, t0, heads, 32 * t + 4 * (lane >> 5), rel + 32 * k) : 0u;
                f32x16 acc;
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
                if (k == 0) {
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) multiply(operand(t, slot, s), kf[0][s], acc);
                } else {
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) multiply(operand(t, slot, s), kf[KB - 1][s], acc);
                }
                f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float b = bias_at(t, slot, i >> 2)[i & 3];
                    const float p = exp2_fast(fmaf(acc[i], c_log2, -b));
                    sum[i & 3] += b < __builtin_inff() ? if_bit(bits, i, p) : 0.0f;
                }
                if (k == 0) part[0] += sum;
                else part[KB - 1] += sum;
            }
        }
        if (t >= n) return;
        u32x4 q[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q[s] = operand(t, slot, s);
        __builtin_amdgcn_sched_barrier(0);
        if (w.any) {
            step<true>(w, q, kf, min(t + KB, n - 1), slot, first);
        } else {
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) w.acc[k][e] = 0.0f;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
#pragma unroll
                for (int k = 0; k < KB; ++k) multiply(q[s], kf[k][s], w.acc[k]);
                q[s] = operand(min(t + KB, n - 1), slot, s);
            }
        }
        w.any = true;
#pragma unroll 1
        for (;;) {
#pragma unroll
            for (int y = 0; y < 4; ++y) w.b[y] = bias_at(t, slot, y);
            __builtin_amdgcn_sched_barrier(0);
            t += KB;
            if (t >= n) break;
            step<true>(w, q, kf, min(t + KB, n - 1), slot, part);
        }
    }
    static __device__ __forceinline__ float sum_of(f32x4 x) { return (x[0] + x[1]) + (x[2] + x[3]); }
    static __device__ __forceinline__ void clear_sums(f32x4 (&x)[KB]) {
#pragma unroll
        for (int k = 0; k < KB; ++k) x[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // The sum over all rows of the lane's key (half of it in either half of the wavefront is `sum`) becomes its score.
    __device__ __forceinline__ void put(int chunk, int kb, float all) const {
        const int j = key_of(chunk, kb);
        if (lane < 32 && j < keys) {
            float* to = r.a.score + ((size_t)u.b * r.c.Hkv + u.h) * r.a.score_stride + j;
            *to = j < u.s.len && r.a.decay != 0.0f ? fmaf(*to, r.a.decay, all) : all;
        }
    }

    // n turns of a mid unit (KB 1): the rows stay, and the wavefronts go their own ways, each with its next 64 keys under way.
    __device__ __forceinline__ void one_group(int n) const {
        static_assert(KB == 1, "every wavefront has all tiles");
        const int last = u.chunk + n;
        constexpr int RING = NM > 8 ? 1 : 2;     // (of f32 with d = 128 there are registers for 32 keys)
        u32x4 ring[RING][NM];
        int page[RING + 1];              // of the present turn and those behind it
#pragma unroll
        for (int i = 0; i < RING; ++i) page[i] = page_of(u.chunk + i, 0, last);
        {
            u32x4 x[QL];
            float l, wt;
            load_rows(0, x, l, wt);
#pragma unroll
            for (int i = 0; i < RING; ++i) fetch(u.chunk + i, 0, page[i], ring[i]);
            __syncthreads();             // what another unit has left in LDS has been read
            store_rows(0, x, l, wt);
            __syncthreads();
        }
        page[RING] = page_of(u.chunk + RING, 0, last);
        Pending w;
        w.any = false;
        f32x4 part[1];
        clear_sums(part);
        u32x4 kf[1][STEPS];
        auto turn = [&](int chunk, u32x4 (&kreg)[NM]) __attribute__((always_inline)) {
            have(kreg);
            widen(kreg, kf[0]);
            have(kf[0]);
            const bool there[1] = {page[0] >= 0}, all_there = __builtin_amdgcn_ballot_w64(!there[0]) == 0;
#pragma unroll
            for (int i = 0; i < RING; ++i) page[i] = page[i + 1];
            fetch(chunk + RING, 0, page[RING], kreg);
            page[RING] = page_of(chunk + RING + 1, 0, last);
            // (the last tile of the keys before is pending still)
            f32x4 before[1] = {part[0]};
            clear_sums(part);
            tiles(chunk, 0, 0, kf, first_token(chunk), there, all_there, w, before, part);
            if (chunk > u.chunk) put(chunk - 1, 0, pair_sum(sum_of(before[0])));
        };
        for (int chunk = u.chunk; chunk < last; chunk += RING) {
            turn(chunk, ring[0]);
            if (RING == 2 && chunk + 1 < last) turn(chunk + 1, ring[RING - 1]);
        }
        finish(w, kf, part);
        put(last - 1, 0, pair_sum(sum_of(part[0])));
    }
    // One turn of a long unit: the rows go by, the next ones under way.
    __device__ __forceinline__ void groups() const {
        const int chunk = u.chunk, n = count(), from = first_token(chunk);
        // a chain's first group with a token that sees a key of the turn
        const int g0 = r.a.tree == nullptr ? max(chunk * C::MANY - u.s.len, 0) / tpg * of_token : 0;
        u32x4 x[QL], kf[KB][STEPS];
        float l, wt;
        bool there[KB], all_there = true;
        load_rows(g0, x, l, wt);
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            const int page = page_of(chunk, k, chunk + 1);
            u32x4 kreg[NM];
            fetch(chunk, k, page, kreg);
            there[k] = page >= 0;
            all_there = all_there && __builtin_amdgcn_ballot_w64(!there[k]) == 0;
            widen(kreg, kf[k]);
        }
        __syncthreads();                 // what another unit has left in LDS has been read
        store_rows(0, x, l, wt);
        have_loads();
        __syncthreads();
        Pending w;
        w.any = false;
        f32x4 part[KB];
        float sum[KB];
#pragma unroll
        for (int k = 0; k < KB; ++k) sum[k] = 0.0f;
        int slot = 0;
        for (int g = g0; g < n; ++g) {
            const bool more = g + 1 < n;
            if (more) load_rows(g + 1, x, l, wt);
            clear_sums(part);
            tiles(chunk, g, slot, kf, from, there, all_there, w, part, part);
#pragma unroll
            for (int k = 0; k < KB; ++k) sum[k] += sum_of(part[k]);
            if (more) store_rows(slot ^ 1, x, l, wt);
            __syncthreads();
            slot ^= 1;
        }
        clear_sums(part);
        finish(w, kf, part);
#pragma unroll
        for (int k = 0; k < KB; ++k) {
            sum[k] = pair_sum(sum[k] + sum_of(part[k]));
            if (KB == 2 && odd == 1 && lane < 32) lds.sums[wave / 2][32 * k + lane] = sum[k];
        }
        if (KB == 2) __syncthreads();
        if (odd == 0) {
#pragma unroll
            for (int k = 0; k < KB; ++k) put(chunk, k, KB == 2 ? sum[k] + lds.sums[wave / 2][32 * k + (lane & 31)] : sum[k]);
        }
    }
};

template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kScoreThreads, 2) void score_kernel(ScoreRun r) {
    using C = ScoreCfg<T, D, FP8>;
    using W = ScoreWalk<C>;
    __shared__ __align__(16) ScoreRows<C> lds;
    __shared__ ScoreScratch scratch;
    const int lane = threadIdx.x & 63, wave = same((int)threadIdx.x >> 6);
    // neighbours in the order of the turns, which read the same queries, are on one XCD
    const int w = ((int)blockIdx.x & 7) * (kScoreGroups / 8) + ((int)blockIdx.x >> 3);
    long long total[3];
    W::begin(r, &scratch, total);
    W u;
    for (long long i = 0; i < total[kLong]; i += kScoreGroups) {
        const long long x = i + ((i & kScoreGroups) != 0 ? kScoreGroups - 1 - w : w);
        if (x >= total[kLong]) continue;
        u.end = 0;
        u.take(r, &scratch, kLong, x);
        ManyRows<T, D, FP8, C::KB, W>(r, u, lds, wave, lane).groups();
    }
    if (u.start(r, &scratch, kMid, total[kMid], w, kScoreGroups)) {
        int n;
        do {
            n = u.here();
            ManyRows<T, D, FP8, 1, W>(r, u, lds, wave, lane).one_group(n);
        } while (u.advance(r, n));
    }
    __syncthreads();                     // the rows of mid units have been read
    static_assert(sizeof(lds.q) >= kScoreWaves * 16 * C::KPITCH, "a block of keys for each wavefront");
    if (u.start(r, &scratch, kFew, total[kFew], w, kScoreGroups))
        few_rows<T, D, FP8>(r, u, &scratch.taken, &lds.q[0][0] + wave * 16 * C::KPITCH, lane);
}

template <typename T, int D, bool FP8>
static hipError_t launch_score_d(const ScoreRun& r, hipStream_t st) {
    hipLaunchKernelGGL((score_kernel<T, D, FP8>), dim3(kScoreGroups), dim3(kScoreThreads), 0, st, r);
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
