// Which drafted tokens stay (flashd_draft_verify): rejection sampling against the target's probabilities, from given
// random numbers.
//
// Behind token i of a sequence the target says p_i = softmax(logits_i / temperature).  The walk begins at token 0 with
// r = p_0; the tokens that continue the present one are asked in their order: x stays if u q(x) < r(x), and the walk goes on from it
// with its own row; else r <- max(r - q, 0) / its sum, or without q (drafts that were not sampled) r without x.  Where the
// walk ends the next token is drawn from r: the least v up to which r sums to more than u.
//
// All of it is in 64 bits.  V tokens cut the unit interval at V places, so that sums of 32 bits would put a random number on
// the wrong side of one of them about once in a thousand draws (131072 tokens, sums off by 1e-8); with 64 it is
// once in 1e9.  An exponential is then 17 instructions of full rate, and each logit has one.
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_paged.h"

namespace flashd {

constexpr int kChunk = 4096;            // logits of a chunk
constexpr int kStatThreads = 256;
constexpr int kEach = kChunk / kStatThreads;
constexpr int kWalkThreads = 1024;
constexpr int kWalkWaves = kWalkThreads / kWave;

// A chunk of a row of logits: its largest, the first place of it, and the sum of 2^((l - top) heat).
struct ChunkStat {
    double sum;
    float top;
    int at;
};
// A row's, and of the token the target's and the draft's probability behind the token it continues.
struct RowStat {
    double sum;
    float top;
    int at;
    double p, q;
};

struct VerifyRun {
    VerifyArgs a;
    ChunkStat* chunks;      // [T][nc]
    RowStat* rows;          // [T]
    int* refused;           // [T] tokens refused behind the present one, from the sequence's first row on
    int nc;
};

// ---- numbers ------------------------------------------------------------------------------------

// A logit as it counts: NaN like -infinity, +infinity like the largest number.
__device__ __forceinline__ float clean(float x) {
    return x != x ? -__builtin_inff() : fminf(x, 3.4028234663852886e38f);
}

// 2^x for x <= 0, by the series of e^(f ln 2) on [-1/2, 1/2]; 6e-15 off.  0 for NaN (of -infinity - -infinity, or times 0).
__device__ __forceinline__ double exp2_down(double x) {
    x = fmax(x, -1100.0);
    const double n = __builtin_rint(x), f = x - n;
    double y = 4.4455382718708115e-10;
    y = fma(y, f, 7.0549116208011233e-9);
    y = fma(y, f, 1.0178086009239699e-7);
    y = fma(y, f, 1.3215486790144310e-6);
    y = fma(y, f, 1.5252733804059840e-5);
    y = fma(y, f, 1.5403530393381609e-4);
    y = fma(y, f, 1.3333558146428443e-3);
    y = fma(y, f, 9.6181291076284771e-3);
    y = fma(y, f, 5.5504108664821580e-2);
    y = fma(y, f, 2.4022650695910072e-1);
    y = fma(y, f, 6.9314718055994531e-1);
    y = fma(y, f, 1.0);
    return ldexp(y, (int)n);
}
__device__ __forceinline__ double weight_of(float l, float top, double heat) {
    return exp2_down(((double)l - (double)top) * heat);
}

template <typename T> struct Raw;
template <> struct Raw<F32> {
    typedef float type;
    static __device__ __forceinline__ float value(type x) { return x; }
};
template <> struct Raw<F16> {
    typedef _Float16 type;
    static __device__ __forceinline__ float value(type x) { return (float)x; }
};
template <> struct Raw<BF16> {
    typedef uint16_t type;
    static __device__ __forceinline__ float value(type x) { return bf16_to_f32(x); }
};
// N consecutive elements, at any alignment of an element (the hardware takes loads of 16 bytes at such)
template <typename T> struct Elements {
    typedef typename Raw<T>::type X;
    static constexpr int E = 16 / sizeof(X);
    static __device__ __forceinline__ float one(const void* p, int64_t i) { return Raw<T>::value(static_cast<const X*>(p)[i]); }
    template <int N>
    static __device__ __forceinline__ void some(const void* p, int64_t i, float* x) {
        X h[N];
        __builtin_memcpy(h, static_cast<const X*>(p) + i, sizeof(h));
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = Raw<T>::value(h[e]);
    }
};

// N elements from v on, `none` from V on
template <typename T, int N>
__device__ __forceinline__ void elements(const void* p, int64_t row, int v, int V, float none, float (&x)[N]) {
    if (v + N <= V) {
        Elements<T>::template some<N>(p, row + v, x);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = v + e < V ? Elements<T>::one(p, row + v + e) : none;
    }
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) x += __shfl_xor(x, k);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) x = fmaxf(x, __shfl_xor(x, k));
    return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) x = min(x, __shfl_xor(x, k));
    return x;
}

// log2(e) / temperature; 0 where the sequence takes the largest logit (a temperature of 0, below, or NaN)
__device__ __forceinline__ double heat_of(float t) { return t > 0.0f ? 1.4426950408889634 / (double)t : -1.0; }

// ---- sums of chunks -----------------------------------------------------------------------------
//
// A workgroup per chunk and row.
template <typename T>
__global__ __launch_bounds__(kStatThreads) void verify_stats_kernel(VerifyRun r) {
    constexpr int E = Elements<T>::E, W = kStatThreads / kWave;
    __shared__ float tops[W];
    __shared__ double sums[W];
    __shared__ int places[W];
    __shared__ int owner;
    const VerifyArgs& a = r.a;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, v0 = blockIdx.x * kChunk;
    const float ninf = -__builtin_inff();
    for (int t = blockIdx.y; t < a.T; t += gridDim.y) {
        float x[kEach];
#pragma unroll
        for (int k = 0; k < kEach / E; ++k) {
            float y[E];
            elements<T, E>(a.logits, (int64_t)t * a.logits_stride, v0 + E * (kStatThreads * k + tid), a.V, ninf, y);
#pragma unroll
            for (int e = 0; e < E; ++e) x[E * k + e] = clean(y[e]);
        }
        double heat = 1.4426950408889634;
        if (a.temperature != nullptr) {
            if (tid == 0) owner = a.B;
            __syncthreads();
            for (int b = tid; b < a.B; b += kStatThreads) {
                const int row0 = max(a.q_start[b], 0);
                if (t >= row0 && t < row0 + tokens_of(row0, a.q_start[b + 1], a.T)) atomicMin(&owner, b);
            }
            __syncthreads();
            if (owner == a.B) {                          // (the same in every thread)
                __syncthreads();
                continue;
            }
            heat = heat_of(a.temperature[owner]);
        }
        float top = x[0];
#pragma unroll
        for (int e = 1; e < kEach; ++e) top = fmaxf(top, x[e]);
        top = wave_max(top);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = tops[0];
#pragma unroll
        for (int w = 1; w < W; ++w) top = fmaxf(top, tops[w]);
        double sum = 0.0;
        int at = 0x7fffffff;
        if (heat >= 0.0) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) sum += weight_of(x[e], top, heat);
            sum = wave_sum(sum);
        } else {
#pragma unroll
            for (int k = kEach / E - 1; k >= 0; --k)
#pragma unroll
                for (int e = E - 1; e >= 0; --e)
                    if (x[E * k + e] == top) at = v0 + E * (kStatThreads * k + tid) + e;
            at = wave_min(at);
        }
        if (lane == 0) {
            sums[wave] = sum;
            places[wave] = at;
        }
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int w = 1; w < W; ++w) {
                sum += sums[w];
                at = min(at, places[w]);
            }
            r.chunks[(size_t)t * r.nc + blockIdx.x] = ChunkStat{sum, top, at};
        }
        __syncthreads();
    }
}

// ---- the walk -----------------------------------------------------------------------------------

// What is left behind the present token: max(scale w - by q, 0) for the weights w of its row; without q the weights but those of
// the tokens refused.
struct Rest {
    int row;            // row of the packed tensors
    float top;
    double heat;
    double scale, by;   // with q
    int refused;        // without q: how many
};

struct WalkShared {
    double part[kWalkWaves];
    int found[kWalkWaves];
    Rest rest;
    int ask;            // 1: the sum of the rest is wanted
    double sum;
};

__device__ __forceinline__ double block_sum(double x, double* part) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kWalkWaves; ++w) s += part[w];
    return s;
}

// The weights of 4 tokens from v on
template <typename T, typename Q>
__device__ __forceinline__ void rest_of(const VerifyRun& r, const Rest& s, const int* refused, int v, double (&w)[4]) {
    const VerifyArgs& a = r.a;
    float x[4], q[4];
    elements<T, 4>(a.logits, (int64_t)s.row * a.logits_stride, v, a.V, -__builtin_inff(), x);
    if (a.draft != nullptr) elements<Q, 4>(a.draft, (int64_t)s.row * a.draft_stride, v, a.V, 0.0f, q);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = weight_of(clean(x[e]), s.top, s.heat);
    if (a.draft != nullptr) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = fmax(s.scale * w[e] - s.by * (double)(q[e] > 0.0f ? q[e] : 0.0f), 0.0);
    } else {
        for (int k = 0; k < s.refused; ++k) {
            const int x0 = refused[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = v + e == x0 ? 0.0 : w[e];
        }
    }
}

// A workgroup per sequence.
template <typename T, typename Q>
__global__ __launch_bounds__(kWalkThreads) void verify_walk_kernel(VerifyRun r) {
    extern __shared__ double chunk_sums[];               // [nc]
    __shared__ WalkShared sh;
    const VerifyArgs& a = r.a;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = max(a.q_start[b], 0), n = tokens_of(row0, a.q_start[b + 1], a.T);
    int* const keep = a.keep + (size_t)b * a.max_keep;
    for (int i = tid; i < a.max_keep; i += kWalkThreads) keep[i] = i == 0 && n > 0 ? 0 : -1;
    if (n == 0) {
        if (tid == 0) {
            a.n_keep[b] = 0;
            a.next[b] = -1;
        }
        return;
    }
    const double heat = a.temperature != nullptr ? heat_of(a.temperature[b]) : 1.4426950408889634;
    const float ninf = -__builtin_inff();

    // rows: their chunks joined, a wavefront each
    for (int i = wave; i < n; i += kWalkWaves) {
        const ChunkStat* of = r.chunks + (size_t)(row0 + i) * r.nc;
        float top = ninf;
        for (int c = lane; c < r.nc; c += kWave) top = fmaxf(top, of[c].top);
        top = wave_max(top);
        double sum = 0.0;
        int at = 0x7fffffff;
        for (int c = lane; c < r.nc; c += kWave) {
            const ChunkStat s = of[c];
            if (heat >= 0.0) sum += s.sum * weight_of(s.top, top, heat);
            else if (s.top == top) at = min(at, s.at);
        }
        sum = wave_sum(sum);
        at = wave_min(at);
        if (lane == 0) {
            RowStat* to = &r.rows[row0 + i];
            to->sum = sum;
            to->top = top;
            to->at = top == ninf ? -1 : at;
        }
    }
    __syncthreads();
    // tokens: their probabilities behind the one they continue
    for (int i = 1 + tid; i < n; i += kWalkThreads) {
        const int before = a.parent != nullptr ? a.parent[row0 + i] : i - 1, x = a.tokens[row0 + i];
        double p = 0.0, q = 1.0;
        if (before >= 0 && before < i && x >= 0 && x < a.V) {
            const RowStat s = r.rows[row0 + before];
            const int64_t t = row0 + before;
            if (heat < 0.0) p = x == s.at ? 1.0 : 0.0;
            else if (s.top != ninf) p = weight_of(clean(Elements<T>::one(a.logits, t * a.logits_stride + x)), s.top, heat) / s.sum;
            if (a.draft != nullptr) {
                const float d = Elements<Q>::one(a.draft, t * a.draft_stride + x);
                q = d > 0.0f ? (double)d : 0.0;
            }
        }
        r.rows[row0 + i].p = p;
        r.rows[row0 + i].q = q;
    }
    __syncthreads();

    // The walk, by the first wavefront: tokens continue earlier ones, so that one way through them in their order is enough.  The
    // others wait to be asked for the sum of what is left.
    int cur = 0, kept = 1, refused = 0;
    double scale = 1.0, by = 0.0;            // r = max(scale p - by q, 0); without q p / scale but for those refused
    double want_scale = 1.0, want_by = 0.0;  // r before it is divided by its sum
    bool open = false;                       // that sum is wanted for the next question
    int* const list = r.refused + row0;
    int j0 = 0, done = 0;                    // the window of 64 tokens, and the tokens of it that are behind
    int before = -2, x = -1;
    double p = 0.0, q = 1.0;
    float u = 0.0f;
    bool load = true;
    for (;;) {
        if (wave == 0) {
            int ask = 0;
            while (j0 < n && kept < a.max_keep) {
                if (load) {
                    const int i = j0 + lane;
                    before = -2;
                    if (i > 0 && i < n) {
                        before = a.parent != nullptr ? a.parent[row0 + i] : i - 1;
                        x = a.tokens[row0 + i];
                        u = a.uniform[row0 + i];
                        p = r.rows[row0 + i].p;
                        q = r.rows[row0 + i].q;
                        if (before >= i) before = -2;
                    }
                    load = false;
                    done = 0;
                }
                const uint64_t next = done >= 64 ? 0 : __builtin_amdgcn_ballot_w64(before == cur) >> done << done;
                if (next == 0) {
                    j0 += 64;
                    load = true;
                    continue;
                }
                if (open) {
                    ask = 1;
                    break;
                }
                const int k = __builtin_ctzll(next);
                done = k + 1;
                const int token = __builtin_amdgcn_readlane(x, k);
                const double pk = __shfl(p, k), qk = __shfl(q, k);
                const float uk = __shfl(u, k);
                double rk = pk;
                bool twice = false;
                if (heat >= 0.0) {
                    if (a.draft != nullptr) {
                        rk = fmax(scale * pk - by * qk, 0.0);
                    } else {
                        for (int i = lane; i < refused; i += kWave) twice |= list[i] == token;
                        twice = __builtin_amdgcn_ballot_w64(twice) != 0;
                        rk = twice ? 0.0 : pk / scale;
                    }
                }
                if ((double)uk * qk < rk) {
                    cur = j0 + k;
                    if (lane == 0) keep[kept] = cur;
                    ++kept;
                    refused = 0;
                    scale = 1.0;
                    by = 0.0;
                } else if (heat >= 0.0) {
                    if (a.draft != nullptr) {
                        want_scale = scale;
                        want_by = by + 1.0;
                        open = true;
                    } else if (!twice && token >= 0 && token < a.V && scale - pk > 0.0) {
                        if (lane == 0) list[refused] = token;
                        __threadfence_block();
                        ++refused;
                        scale -= pk;
                    }
                }
            }
            if (lane == 0) {
                sh.ask = ask;
                const RowStat s = r.rows[row0 + cur];
                sh.rest = Rest{row0 + cur, s.top, heat, open ? want_scale / s.sum : scale / s.sum, open ? want_by : by, refused};
            }
        }
        __syncthreads();
        const bool ask = sh.ask != 0;
        const Rest rest = sh.rest;
        if (!ask) break;
        double sum = 0.0;
        for (int v = 4 * tid; v < a.V; v += 4 * kWalkThreads) {
            double w[4];
            rest_of<T, Q>(r, rest, list, v, w);
            sum += (w[0] + w[1]) + (w[2] + w[3]);
        }
        sum = block_sum(sum, sh.part);
        if (wave == 0) {
            open = false;
            if (sum > 0.0) {                 // else nothing is left, and r stays
                scale = want_scale / sum;
                by = want_by / sum;
            }
        }
    }

    // ---- the next token
    Rest rest = sh.rest;
    __syncthreads();                         // (what the first wavefront writes now has been read)
    if (wave == 0 && lane == 0) {
        a.n_keep[b] = kept;
        sh.sum = open ? scale : 0.0;
        sh.part[0] = by;
        sh.ask = open;
    }
    __syncthreads();
    const bool was_open = sh.ask != 0;
    const double old_scale = sh.sum, old_by = sh.part[0];
    const int row = rest.row;
    const RowStat s = r.rows[row];
    if (heat < 0.0 || s.top == ninf) {
        if (tid == 0) a.next[b] = s.top == ninf ? -1 : s.at;
        return;
    }
    const bool plain = a.draft == nullptr;
    double total = 0.0;
    for (int turn = 0;; ++turn) {
        // sums of the chunks
        __syncthreads();
        if (plain || rest.by == 0.0) {
            const ChunkStat* of = r.chunks + (size_t)row * r.nc;
            for (int c = tid; c < r.nc; c += kWalkThreads) chunk_sums[c] = of[c].sum * weight_of(of[c].top, s.top, heat) * (plain ? 1.0 : rest.scale);
            __syncthreads();
            for (int k = 0; k < (plain ? rest.refused : 0); ++k) {       // chunks that lack a token are summed again
                const int c = list[k] / kChunk;
                double w[4];
                rest_of<T, Q>(r, rest, list, c * kChunk + 4 * tid, w);
                const double sum = block_sum((w[0] + w[1]) + (w[2] + w[3]), sh.part);
                if (tid == 0) chunk_sums[c] = sum;
            }
        } else {
            for (int c = wave; c < r.nc; c += kWalkWaves) {
                double sum = 0.0;
#pragma unroll 4
                for (int k = 0; k < kChunk / 256; ++k) {
                    const int v = c * kChunk + 256 * k + 4 * lane;
                    if (v >= a.V) continue;
                    double w[4];
                    rest_of<T, Q>(r, rest, list, v, w);
                    sum += (w[0] + w[1]) + (w[2] + w[3]);
                }
                sum = wave_sum(sum);
                if (lane == 0) chunk_sums[c] = sum;
            }
        }
        __syncthreads();
        double mine = 0.0;
        for (int c = tid; c < r.nc; c += kWalkThreads) mine += chunk_sums[c];
        total = block_sum(mine, sh.part);
        if (total > 0.0 || turn == 1 || !was_open) break;
        rest.scale = old_scale / s.sum;      // nothing is left: r as it was before the last refusal
        rest.by = old_by;
    }
    // the chunk with the wanted place: the first up to which the sum passes it, or the last that has any
    if (wave == 0) {
        const double place = (double)a.uniform[row0] * total;
        double before_sum = 0.0, left = 0.0;
        int chunk = -1, last = -1;
        double last_before = 0.0;
        for (int c0 = 0; c0 < r.nc && chunk < 0; c0 += kWave) {
            const int c = c0 + lane;
            const double sum = c < r.nc ? chunk_sums[c] : 0.0;
            double upto = sum;
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) {
                const double y = __shfl_up(upto, k);
                if (lane >= k) upto += y;
            }
            upto += before_sum;
            const uint64_t over = __builtin_amdgcn_ballot_w64(sum > 0.0 && upto > place), any = __builtin_amdgcn_ballot_w64(sum > 0.0);
            if (any != 0) {
                const int k = 63 - __builtin_clzll(any);
                last = c0 + k;
                last_before = __shfl(upto - sum, k);
            }
            if (over != 0) {
                const int k = __builtin_ctzll(over);
                chunk = c0 + k;
                left = place - __shfl(upto - sum, k);
            }
            before_sum = __shfl(upto, 63);
        }
        if (chunk < 0) {
            chunk = last;
            left = place - last_before;
        }
        if (lane == 0) {
            sh.found[0] = chunk;
            sh.sum = left;
        }
    }
    __syncthreads();
    const int chunk = sh.found[0];
    const double left = sh.sum;
    __syncthreads();
    if (chunk < 0) {
        if (tid == 0) a.next[b] = -1;
        return;
    }
    double w[4];
    const int v = chunk * kChunk + 4 * tid;
    rest_of<T, Q>(r, rest, list, v, w);
    const double own = (w[0] + w[1]) + (w[2] + w[3]);
    double upto = own;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const double y = __shfl_up(upto, k);
        if (lane >= k) upto += y;
    }
    if (lane == 63) sh.part[wave] = upto;
    __syncthreads();
    double sum = upto - own;
#pragma unroll
    for (int k = 0; k < kWalkWaves; ++k) sum += k < wave ? sh.part[k] : 0.0;
    int first = 0x7fffffff, last = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sum += w[e];
        if (w[e] > 0.0) {
            last = v + e;
            if (sum > left) first = min(first, v + e);
        }
    }
    first = wave_min(first);
    last = -wave_min(-last);
    if (lane == 0) sh.found[wave] = first;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWalkWaves; ++k) first = min(first, sh.found[k]);
    __syncthreads();
    if (lane == 0) sh.found[wave] = last;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWalkWaves; ++k) last = max(last, sh.found[k]);
    if (tid == 0) a.next[b] = first != 0x7fffffff ? first : last;
}

// ---- host ---------------------------------------------------------------------------------------

static int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }

size_t verify_workspace(int T, int V) {
    return (size_t)T * ((size_t)chunks_of(V) * sizeof(ChunkStat) + sizeof(RowStat) + 8);
}

template <typename T>
static hipError_t launch_verify_t(const VerifyRun& r, hipStream_t st) {
    if (r.a.T > 0) {                     // (without rows no sequence has tokens)
        const dim3 grid((unsigned)r.nc, (unsigned)(r.a.T < 65535 ? r.a.T : 65535));
        hipLaunchKernelGGL(verify_stats_kernel<T>, grid, dim3(kStatThreads), 0, st, r);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 seqs((unsigned)r.a.B), block(kWalkThreads);
    const size_t lds = (size_t)r.nc * sizeof(double);
    switch (r.a.draft_dtype) {
    case 0: hipLaunchKernelGGL((verify_walk_kernel<T, F32>), seqs, block, lds, st, r); break;
    case 1: hipLaunchKernelGGL((verify_walk_kernel<T, F16>), seqs, block, lds, st, r); break;
    default: hipLaunchKernelGGL((verify_walk_kernel<T, BF16>), seqs, block, lds, st, r); break;
    }
    return hipGetLastError();
}

hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t st) {
    VerifyRun r;
    r.a = a;
    r.nc = chunks_of(a.V);
    r.chunks = static_cast<ChunkStat*>(ws);
    r.rows = reinterpret_cast<RowStat*>(r.chunks + (size_t)a.T * r.nc);
    r.refused = reinterpret_cast<int*>(r.rows + a.T);
    switch (a.dtype) {
    case 0: return launch_verify_t<F32>(r, st);
    case 1: return launch_verify_t<F16>(r, st);
    default: return launch_verify_t<BF16>(r, st);
    }
}

}  // namespace flashd
