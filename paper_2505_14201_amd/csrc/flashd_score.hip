// The attention weight that new tokens give to each key, added to the keys' scores (flashd_cache_score).
//
// score_j <- decay score_j + sum over the new tokens i that see key j, and the heads of the kv group, of
// w_i exp(scale q_i.k_j - lse_i), with the queries' log-sum-exps as the attention has left them: so that one pass over K is enough, no
// sum over the keys is needed, and what belongs to a key stays in one workgroup.
//
// S = Q K^T comes with keys as columns: lane (c, hh) = (lane % 32, lane / 32) holds key c and of a tile of 32 rows (pairs of token and head
// of the group) the rows 8 (r / 4) + 4 hh + r % 4, so that the sum over rows is one over the lane's own registers.  K is the B operand
// and stays in registers, loaded from the pages as it lies there; rows go by through LDS, in groups that the wavefronts of a workgroup read together.
// A row's w exp(-lse) is one number in the exponent: 2^(c s - bias).
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

#include <type_traits>

namespace flashd {

constexpr int kScoreWaves = 4, kScoreThreads = kScoreWaves * kWave;
constexpr int kScoreGroups = 512;       // workgroups of a launch: two per compute unit
// What K's way to the registers counts, in tiles of 32 rows, where the work is shared out.
constexpr int kScoreStart = 4;

struct ScoreRun {
    Paged c;
    ScoreArgs a;
    FastDiv group;          // query heads per kv head
};

// Types and sizes: KB 32-key blocks of a wavefront, rows of a group in LDS and the bytes of one there (padded, so that 16 rows fall on all banks)
template <typename T, int D, bool FP8> struct ScoreCfg {
    static constexpr bool F = std::is_same_v<T, F32>;
    static constexpr int KB = F ? 1 : 2;
    static constexpr int KEYS = 32 * KB * kScoreWaves;   // of a workgroup's chunk
    static constexpr int QSZ = F ? 4 : 2;
    static constexpr int ROWS = F ? 64 : 128;
    static constexpr int PITCH = D * QSZ + 16;
    static constexpr int NL = D * (F ? 4 : FP8 ? 1 : 2) / 32;   // 16-byte loads of a lane and block
    static constexpr int STEPS = F ? D / 8 : D / 16;     // operands of 16 bytes
    // byte of a row at which the lane's operand s begins: the order in which K's loads bring the elements
    static __device__ __forceinline__ int at(int s, int hh) {
        return FP8 ? 2 * (32 * (s >> 1) + 16 * hh + 8 * (s & 1)) : 32 * s + 16 * hh;
    }
};

__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A workgroup's share: units are (sequence, kv head), cut into chunks of keys that each count its row tiles; a chunk is the workgroup's in whose
// stretch of that row it begins.
template <int KEYS>
struct ScoreWalk {
    long long at, end;
    int b, h, chunk;
    Seq s;
    int rows, chunks;
    long long cost;

    struct Scratch {
        long long sum[kScoreWaves];
        long long before;
        int b;
    };

    __device__ __forceinline__ void enter(const ScoreRun& r, int seq) {
        b = seq;
        s = seq_at(r.c, b);
        rows = s.n * (int)r.group.d;             // (T Hq is below 2^31)
        chunks = s.n == 0 ? 0 : (s.len + s.n + KEYS - 1) / KEYS;
        cost = (rows + 31) / 32 + kScoreStart;
    }
    __device__ __forceinline__ void enter_same(const ScoreRun& r, int seq) {
        enter(r, seq);
        s = Seq{same(s.row0), same(s.n), same(s.len)};
        rows = same(rows);
        chunks = same(chunks);
    }
    __device__ __forceinline__ bool begin(const ScoreRun& r, Scratch* sh) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int each = (r.c.B + kScoreThreads - 1) / kScoreThreads, b0 = tid * each, b1 = min(b0 + each, r.c.B);
        long long mine = 0;
        for (int i = b0; i < b1; ++i) {
            enter(r, i);
            mine += cost * chunks * r.c.Hkv;
        }
        long long in = mine;
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
            const long long y = __shfl_up(in, k);
            if (lane >= k) in += y;
        }
        if (lane == 63) sh->sum[wave] = in;
        if (tid == 0) sh->b = -1;
        __syncthreads();
        long long before = in - mine, total = 0;
#pragma unroll
        for (int k = 0; k < kScoreWaves; ++k) {
            before += k < wave ? sh->sum[k] : 0;
            total += sh->sum[k];
        }
        // neighbours along the row, which read the same queries, go to one XCD
        const int w = ((int)blockIdx.x & 7) * ((int)gridDim.x >> 3) + ((int)blockIdx.x >> 3);
        const long long per = (total + gridDim.x - 1) / gridDim.x;
        at = w * per;
        end = min(at + per, total);
        // the first chunk that begins in the share: its sequence's places end behind the share's first place
        if (at < end && at >= before && at < before + mine) {
            int i = b0;
            for (;; ++i) {
                enter(r, i);
                const long long own = cost * chunks * r.c.Hkv;
                if (at < before + own) break;
                before += own;
            }
            sh->b = i;
            sh->before = before;
        }
        __syncthreads();
        const int found = same(sh->b);
        const long long start = sh->before;
        __syncthreads();
        if (found < 0) return false;
        enter_same(r, found);
        const long long k = (at - start + cost - 1) / cost;      // chunks of the sequence that begin before
        at = start + k * cost;
        if (at >= end) return false;
        if (k >= (long long)chunks * r.c.Hkv) {
            if (!next_seq(r)) return false;
        } else {
            h = same((int)(k / chunks));
            chunk = same((int)(k - (long long)h * chunks));
        }
        return true;
    }
    __device__ __forceinline__ bool next_seq(const ScoreRun& r) {
        do {
            if (b + 1 >= r.c.B) return false;
            enter_same(r, b + 1);
        } while (chunks == 0);
        h = 0;
        chunk = 0;
        return true;
    }
    // Chunks of this unit from the present one on that are the workgroup's
    __device__ __forceinline__ int here() const {
        const long long n = (end - at + cost - 1) / cost;
        return n < chunks - chunk ? (int)n : chunks - chunk;
    }
    // past n chunks of this unit
    __device__ __forceinline__ bool advance(const ScoreRun& r, int n) {
        at += n * cost;
        if (at >= end) return false;
        chunk += n;
        if (chunk < chunks) return true;
        chunk = 0;
        if (++h < r.c.Hkv) return true;
        return next_seq(r);
    }
};

template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kScoreThreads, 2) void score_kernel(ScoreRun r) {
    using C = ScoreCfg<T, D, FP8>;
    constexpr int KB = C::KB, NL = C::NL, STEPS = C::STEPS, ROWS = C::ROWS, PITCH = C::PITCH;
    constexpr int QL = ROWS * D * C::QSZ / (16 * kScoreThreads);         // 16-byte loads of a thread for a group of rows
    constexpr int CPR = D * C::QSZ / 16;
    __shared__ __align__(16) char qlds[ROWS * PITCH];
    __shared__ __align__(16) float bias[ROWS];
    __shared__ typename ScoreWalk<C::KEYS>::Scratch scratch;
    __shared__ int any_off[kScoreWaves];
    const Paged& c = r.c;
    const ScoreArgs& a = r.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = same(tid >> 6), col = lane & 31, hh = lane >> 5;
    const float inf = __builtin_inff();
    const float c_log2 = (FP8 ? a.scale * c.kscale : a.scale) * kLog2e;
    const int G = (int)r.group.d;

    ScoreWalk<C::KEYS> u;
    if (!u.begin(r, &scratch)) return;
    int staged_b = -1, staged_h = -1;            // whose only group of rows lies in LDS
    bool off = false;                            // some row of the group in LDS does not count
    for (;;) {
        const int n = u.here();
        const int keys = u.s.len + u.s.n;
        const int groups = (u.rows + ROWS - 1) / ROWS;
        const char* pool = c.k + u.h * c.head_bytes;

        // K of the lane's keys of a chunk: their pages' places in the table go ahead of them
        auto key_of = [&](int chunk, int kb) { return chunk * C::KEYS + wave * (32 * KB) + 32 * kb + col; };
        auto page_of = [&](int chunk, int kb) {
            const int j = key_of(chunk, kb);
            return chunk < u.chunk + n && j < keys ? page_at(c, u.b, j >> c.page_log2) : -1;
        };
        auto fetch = [&](int chunk, const int (&page)[KB], u32x4 (&to)[KB][NL]) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                // (a key without a page reads the pool's first: its column of products is dropped)
                const int j = key_of(chunk, kb) & ((1 << c.page_log2) - 1);
                const char* from = pool + (page[kb] < 0 ? 0 : page[kb] * c.page_bytes + (int64_t)j * (NL * 32)) + 16 * hh;
#pragma unroll
                for (int i = 0; i < NL; ++i) to[kb][i] = *reinterpret_cast<const u32x4*>(from + 32 * i);
            }
        };
        u32x4 kreg[KB][NL];
        int page[KB], ahead[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            page[kb] = page_of(u.chunk, kb);
            ahead[kb] = page_of(u.chunk + 1, kb);
        }
        fetch(u.chunk, page, kreg);

        for (int chunk = u.chunk; chunk < u.chunk + n; ++chunk) {
            const int j0 = chunk * C::KEYS + wave * (32 * KB);           // the wavefront's first key
            u32x4 kf[KB][NL];
            bool there[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                there[kb] = page[kb] >= 0;
#pragma unroll
                for (int i = 0; i < NL; ++i) kf[kb][i] = kreg[kb][i];
            }
            if (chunk + 1 < u.chunk + n) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    page[kb] = ahead[kb];
                    ahead[kb] = page_of(chunk + 2, kb);
                }
                fetch(chunk + 1, page, kreg);
            }
            float sum[KB];
            int rel[KB], lim[KB];                // the key's place among the new ones, and the first row of a chain that sees it
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                sum[kb] = 0.0f;
                rel[kb] = j0 + 32 * kb + col - u.s.len;
                lim[kb] = rel[kb] <= 0 ? 0 : min(rel[kb], u.s.n) * G;
            }
            const bool all_there = __builtin_amdgcn_ballot_w64(!there[0] || !there[KB - 1]) == 0;
            // rows that see none of the wavefront's keys, of a chain
            const int first_row = j0 >= keys ? 0x7fffffff : a.tree == nullptr && j0 > u.s.len ? (j0 - u.s.len) * G : 0;

            const int first_key = chunk * C::KEYS - u.s.len;
            for (int g = a.tree == nullptr && first_key > 0 ? first_key * G / ROWS : 0; g < groups; ++g) {
                if (groups > 1 || staged_b != u.b || staged_h != u.h) {
                    u32x4 x[QL];
#pragma unroll
                    for (int i = 0; i < QL; ++i) {
                        const int at = i * kScoreThreads + tid, row = min(g * ROWS + at / CPR, u.rows - 1);
                        const int token = (int)fast_div((uint32_t)row, r.group);
                        const char* from = static_cast<const char*>(a.q) +
                            ((int64_t)(u.s.row0 + token) * a.q_stride + (int64_t)(u.h * G + row - token * G) * D) * C::QSZ;
                        x[i] = *reinterpret_cast<const u32x4*>(from + 16 * (at % CPR));
                    }
                    float bs = inf;
                    if (tid < ROWS && g * ROWS + tid < u.rows) {
                        const int row = g * ROWS + tid, token = (int)fast_div((uint32_t)row, r.group);
                        const float l = a.lse[(size_t)(u.s.row0 + token) * a.Hq + u.h * G + row - token * G];
                        const float w = a.weight != nullptr ? a.weight[u.s.row0 + token] : 1.0f;
                        // rows that see nothing (-infinity), or whose weight is not positive, do not count
                        if (w > 0.0f && l > -inf) bs = l * kLog2e - (a.weight != nullptr ? log2_fast(w) : 0.0f);
                    }
                    __syncthreads();             // the group before has been read
#pragma unroll
                    for (int i = 0; i < QL; ++i) {
                        const int at = i * kScoreThreads + tid;
                        *reinterpret_cast<u32x4*>(&qlds[(at / CPR) * PITCH + 16 * (at % CPR)]) = x[i];
                    }
                    if (tid < ROWS) bias[tid] = bs;
                    const bool mine_off = __builtin_amdgcn_ballot_w64(tid < ROWS && !(bs < inf)) != 0;
                    if (lane == 0) any_off[wave] = mine_off;
                    __syncthreads();
                    off = (any_off[0] | any_off[1] | any_off[2] | any_off[3]) != 0;
                    staged_b = u.b;
                    staged_h = u.h;
                }
                const int tiles = (min(u.rows - g * ROWS, ROWS) + 31) / 32;
                const bool masked = off || !all_there || j0 + 32 * KB > u.s.len;
                for (int t = max(first_row - g * ROWS, 0) / 32; t < tiles; ++t) {
                    f32x16 acc[KB];
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[kb][e] = 0.0f;
                    const char* qrow = &qlds[(32 * t + col) * PITCH];
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        const u32x4 q = *reinterpret_cast<const u32x4*>(qrow + C::at(s, hh));
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) {
                            if constexpr (C::F) {
                                const f32x4 x = __builtin_bit_cast(f32x4, q), y = __builtin_bit_cast(f32x4, kf[kb][s]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) acc[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc[kb], 0, 0, 0);
                            } else if constexpr (FP8) {
                                const u32x4 y = kf[kb][s >> 1];
                                acc[kb] = Mma<T>::mfma(q, widen8<T>(y[2 * (s & 1)], y[2 * (s & 1) + 1]), acc[kb]);
                            } else {
                                acc[kb] = Mma<T>::mfma(q, kf[kb][s], acc[kb]);
                            }
                        }
                    }
                    float part[KB];
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) part[kb] = 0.0f;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const f32x4 bs = *reinterpret_cast<const f32x4*>(&bias[32 * t + 8 * y + 4 * hh]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
#pragma unroll
                            for (int kb = 0; kb < KB; ++kb) {
                                float p = exp2_fast(fmaf(acc[kb][4 * y + e], c_log2, -bs[e]));
                                if (masked) {
                                    const int row = g * ROWS + 32 * t + 8 * y + 4 * hh + e;
                                    bool seen = there[kb] && bs[e] < inf;
                                    if (a.tree == nullptr) {
                                        seen = seen && row >= lim[kb];
                                    } else if (rel[kb] >= 0 && seen) {
                                        const int token = (int)fast_div((uint32_t)row, r.group), word = rel[kb] >> 5;
                                        seen = word < a.words && (a.tree[(size_t)(u.s.row0 + token) * a.words + word] >> (rel[kb] & 31) & 1u) != 0;
                                    }
                                    p = seen ? p : 0.0f;
                                }
                                part[kb] += p;
                            }
                        }
                    }
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) sum[kb] += part[kb];
                }
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const float all = pair_sum(sum[kb]);
                const int j = j0 + 32 * kb + col;
                if (hh == 0 && j < keys) {
                    float* to = a.score + ((size_t)u.b * c.Hkv + u.h) * a.score_stride + j;
                    *to = j < u.s.len && a.decay != 0.0f ? fmaf(*to, a.decay, all) : all;
                }
            }
        }
        if (!u.advance(r, n)) return;
    }
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
