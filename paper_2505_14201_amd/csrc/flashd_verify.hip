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
// once in 1e9.  An exponential is then 13 instructions of full rate, and each logit has one.
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

// log2(e) / temperature, and what distances to the largest logit are cut to, -1023 / scale, which is exponent 0: no weight; a scale below 0 where the sequence takes the largest logit
// (a temperature of 0, below, or NaN).  An infinite temperature leaves the least scale with which the rules for infinities hold.
struct Heat {
    double scale, least;
};
__device__ __forceinline__ Heat heat_of(float t) {
    if (!(t > 0.0f)) return Heat{-1.0, 0.0};
    const double scale = fmax(1.4426950408889634 / (double)t, 1e-290);
    return Heat{scale, -1023.0 / scale};
}

// What is left behind the present token: max(scale w - by q, 0) for the weights w of its row; without q the weights but those of
// the tokens refused.
struct Rest {
    int row;            // row of the packed tensors
    float top;
    Heat heat;
    double scale, by;   // with q
    int refused;        // without q: how many
};

// Where a sequence's walk has ended
struct WalkEnd {
    Rest rest;
    RowStat row;        // of the rest
    double old_scale, old_by;   // of what was left before the last refusal, if that has not been divided by its sum
    int open;
    int draw;           // 0: the next token is known
};

struct VerifyRun {
    VerifyArgs a;
    ChunkStat* chunks;      // [T][nc]
    RowStat* rows;          // [T]
    WalkEnd* ends;          // [T] of a sequence at its first row, as the others:
    double* left;           // [T][nc] sums of what is left over the chunks
    uint8_t* marks;         // [longest sequences][nc * kChunk] tokens refused behind the present one
    int* refused;           // [T] their list
    int nc;
};

// ---- numbers ------------------------------------------------------------------------------------

// The largest of three numbers, none of them NaN.  (The compiler, which cannot know that, has each operand of fmaxf go through an instruction of its own.)
__device__ __forceinline__ float max3(float x, float y, float z) {
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(x), "v"(y), "v"(z));
    return m;
}
__device__ __forceinline__ bool is_odd(float x) { return __builtin_amdgcn_classf(x, 0x203); }        // NaN or +infinity
// A logit as it counts: NaN like -infinity, +infinity like the largest number.
__device__ __forceinline__ float clean(float x) {
    return x != x ? -__builtin_inff() : fminf(x, 3.4028234663852886e38f);
}

// 2^(d heat.scale) for d <= 0, by a polynomial for 2^f on [-1/2, 1/2] through its values at the ten zeros of a Chebyshev polynomial; 1.9e-14 off.  0 where
// it is below 2^-1022.5, and so for d = -infinity and NaN (of -infinity - -infinity), which `least` makes 2^-1023.
__device__ __forceinline__ double weight_of(float l, float top, Heat heat) {
    const double d = fmax((double)l - (double)top, heat.least);
    const double whole = 6755399441055744.0;                     // 1.5 2^52: what is added to it is rounded to a whole number, in its low bits
    const double t = fma(d, heat.scale, whole), f = fma(d, heat.scale, whole - t);
    double y = 1.0205905413765595e-07;
    y = fma(y, f, 1.3259645244887111e-06);
    y = fma(y, f, 1.5252672924850737e-05);
    y = fma(y, f, 1.5403433751251010e-04);
    y = fma(y, f, 1.3333558200794592e-03);
    y = fma(y, f, 9.6181291939343126e-03);
    y = fma(y, f, 5.5504108664651670e-02);
    y = fma(y, f, 2.4022650695640341e-01);
    y = fma(y, f, 6.9314718055994617e-01);
    y = fma(y, f, 1.0000000000000135);
    const int n = (int)(uint32_t)__double_as_longlong(t);
    return n > -1023 ? ldexp(y, n) : 0.0;
}

// The same where there are many, with a table of 2^(j / 256): of the exponent's 256th parts the whole ones' low 8 bits are j, the others go to the number's exponent, and
// of the rest a polynomial of degree 3 is 1.8e-14 off.  13 instructions instead of 19 (and a read of LDS, which is idle: the lanes of a wavefront meet a bank about
// three at a time).
constexpr int kParts = 256;
struct Powers {
    uint64_t bits[kParts];          // of the number less j << 44: what j adds to the exponent's place is in it already
    constexpr Powers() : bits() {
        for (int j = 0; j < kParts; ++j) {
            // e^x of x = j ln 2 / 256 < 0.7
            const double x = j * (0.69314718055994530942 / kParts);
            double y = 1.0;
            for (int k = 22; k > 0; --k) y = 1.0 + x / k * y;
            bits[j] = (uint64_t)((y - 1.0) * 4503599627370496.0) + (1023ull << 52) - ((uint64_t)j << 44);
        }
    }
};
__device__ constexpr Powers kPowers;
template <int THREADS> __device__ __forceinline__ void take_powers(uint64_t (&to)[kParts]) {
    for (int j = threadIdx.x; j < kParts; j += THREADS) to[j] = kPowers.bits[j];
}
__device__ __forceinline__ void weights_of(const float* l, float top, Heat heat, const uint64_t* powers, double (&w)[4]) {
    const double scale = heat.scale * kParts, whole = 6755399441055744.0;
    double f[4];
    uint32_t lift[4];
    uint64_t power[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double d = fmax((double)l[e] - (double)top, heat.least), t = fma(d, scale, whole);
        f[e] = fma(d, scale, whole - t);
        const uint32_t n = (uint32_t)__double_as_longlong(t);
        power[e] = powers[n & (kParts - 1)];
        lift[e] = n << 12;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        double y = 3.3083029837113951e-09;
        y = fma(y, f[e], 3.6655661567589336e-06);
        y = fma(y, f[e], 0.0027076061740622767);
        y = fma(y, f[e], 0.99999999999998246);
        w[e] = __hiloint2double((int)((uint32_t)(power[e] >> 32) + lift[e]), (int)(uint32_t)power[e]) * y;
    }
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

// What 1, 2, 4 and 8 lanes before have, then lane 15 of a row for rows 1 and 3, then lane 31 for rows 2 and 3; `none` where there is no such lane.  After all six steps lane 63
// has met all of them.
template <int STEP> __device__ __forceinline__ int lane_before(int none, int x) {
    constexpr int CTRL[6] = {0x111, 0x112, 0x114, 0x118, 0x142, 0x143}, ROWS[6] = {0xf, 0xf, 0xf, 0xf, 0xa, 0xc};
    return __builtin_amdgcn_update_dpp(none, x, CTRL[STEP], ROWS[STEP], 0xf, false);
}
template <int STEP> __device__ __forceinline__ double lane_before(double x) {
    const long long y = __double_as_longlong(x);
    return __hiloint2double(lane_before<STEP>(0, (int)(y >> 32)), lane_before<STEP>(0, (int)y));
}
template <int STEP> __device__ __forceinline__ float lane_before(float x) {
    return __int_as_float(lane_before<STEP>(__float_as_int(x), __float_as_int(x)));
}
// Sum of the lanes up to this one
__device__ __forceinline__ double sum_up_to(double x) {
    x += lane_before<0>(x);
    x += lane_before<1>(x);
    x += lane_before<2>(x);
    x += lane_before<3>(x);
    x += lane_before<4>(x);
    return x + lane_before<5>(x);
}
__device__ __forceinline__ double of_lane(double x, int lane) {
    const long long y = __double_as_longlong(x);
    return __hiloint2double(__builtin_amdgcn_readlane((int)(y >> 32), lane), __builtin_amdgcn_readlane((int)y, lane));
}
__device__ __forceinline__ double wave_sum(double x) { return of_lane(sum_up_to(x), 63); }
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, lane_before<0>(x));
    x = fmaxf(x, lane_before<1>(x));
    x = fmaxf(x, lane_before<2>(x));
    x = fmaxf(x, lane_before<3>(x));
    x = fmaxf(x, lane_before<4>(x));
    x = fmaxf(x, lane_before<5>(x));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ int wave_min(int x) {
    x = min(x, lane_before<0>(x, x));
    x = min(x, lane_before<1>(x, x));
    x = min(x, lane_before<2>(x, x));
    x = min(x, lane_before<3>(x, x));
    x = min(x, lane_before<4>(x, x));
    x = min(x, lane_before<5>(x, x));
    return __builtin_amdgcn_readlane(x, 63);
}

// ---- sums of chunks -----------------------------------------------------------------------------
//
// A workgroup per chunk and row.  f32 logits come at 4.3 TB/s (202 rows of 100003: 19 us); of 16 bits the sums of 64 bits take as long again: 75.5 MB of bf16, 288 rows of 131072,
// 29 us, of which 18 without the exponentials.  (Workgroups that take several chunks, reading the next while they sum the present one: 32 us, and 23 for the f32.)
template <typename T>
__global__ __launch_bounds__(kStatThreads) void verify_stats_kernel(VerifyRun r) {
    constexpr int E = Elements<T>::E, W = kStatThreads / kWave;
    __shared__ uint64_t powers[kParts];
    __shared__ float tops[W];
    __shared__ double sums[W];
    __shared__ int places[W];
    const VerifyArgs& a = r.a;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, v0 = blockIdx.x * kChunk;
    const float ninf = -__builtin_inff();
    take_powers<kStatThreads>(powers);
    for (int t = blockIdx.y; t < a.T; t += gridDim.y) {
        // (with temperatures: whose row it is; every wavefront looks for itself)
        Heat heat = heat_of(1.0f);
        if (a.temperature != nullptr) {
            int owner = -1;
            for (int b0 = 0; b0 < a.B && owner < 0; b0 += kWave) {
                const int b = min(b0 + lane, a.B - 1), row0 = max(a.q_start[b], 0);
                const uint64_t mine = __builtin_amdgcn_ballot_w64(t >= row0 && t < row0 + tokens_of(row0, a.q_start[b + 1], a.T));
                if (mine != 0) owner = min(b0 + __builtin_ctzll(mine), a.B - 1);
            }
            if (owner < 0) continue;                     // (the same in every wavefront)
            heat = heat_of(a.temperature[owner]);
        }
        float x[kEach];
#pragma unroll
        for (int k = 0; k < kEach / E; ++k) {
            float y[E];
            elements<T, E>(a.logits, (int64_t)t * a.logits_stride, v0 + E * (kStatThreads * k + tid), a.V, ninf, y);
#pragma unroll
            for (int e = 0; e < E; ++e) x[E * k + e] = y[e];
        }
        bool odd = false;
#pragma unroll
        for (int e = 0; e < kEach; ++e) odd |= is_odd(x[e]);
        if (__builtin_amdgcn_ballot_w64(odd) != 0) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) x[e] = clean(x[e]);
        }
        float top = ninf;
#pragma unroll
        for (int e = 0; e < kEach; e += 2) top = max3(top, x[e], x[e + 1]);
        top = wave_max(top);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = tops[0];
#pragma unroll
        for (int w = 1; w < W; ++w) top = fmaxf(top, tops[w]);
        double sum = 0.0, odd_sum = 0.0;
        int at = 0x7fffffff;
        if (heat.scale >= 0.0) {
#pragma unroll
            for (int e = 0; e < kEach; e += 4) {
                double w[4];
                weights_of(x + e, top, heat, powers, w);
                sum += w[0];
                odd_sum += w[1];
                sum += w[2];
                odd_sum += w[3];
            }
            sum = wave_sum(sum + odd_sum);
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

constexpr int kNear = 256;               // rows and refused tokens of a sequence that have a place in LDS

// Sequences of more than kNear tokens, of which there are fewer than T / kNear, have a byte for each token of the vocabulary: whether it has been refused behind the
// present one.  (By the list alone each of R refused tokens would be looked for among all others, and in every sum: R^2.)
__host__ __device__ constexpr int64_t mark_maps(int T) { return T > 0 ? (T - 1) / kNear : 0; }
__device__ __forceinline__ uint8_t* marks_of(const VerifyRun& r, int row0, int n) {
    // (starts of such sequences are more than kNear apart)
    return n > kNear ? r.marks + (int64_t)(row0 / kNear) * r.nc * kChunk : nullptr;
}

struct WalkShared {
    RowStat rows[kNear];
    int list[kNear];
    double weight[kNear];   // of a refused token
    int queue[kNear];       // chunks whose sum is to be taken again, `queued` of them
    int queued;
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

// The refused tokens: the first ones in LDS, where there are more the others in `far`, and all of them marked
struct Refused {
    int* near;
    int* far;
    uint8_t* marks;
    __device__ __forceinline__ int operator[](int k) const { return k < kNear ? near[k] : far[k]; }
    __device__ __forceinline__ void put(int k, int x) const {
        if (k < kNear) near[k] = x;
        else far[k] = x;
        if (marks != nullptr) marks[x] = 1;
    }
    // the first n of them out of the weights of 4 tokens from v on (a multiple of 4)
    __device__ __forceinline__ void out(int n, int v, double (&w)[4]) const {
        if (n > kNear) {
            const uint32_t gone = *reinterpret_cast<const uint32_t*>(marks + v);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (gone >> (8 * e) & 0xffu) != 0 ? 0.0 : w[e];
        } else {
            for (int k = 0; k < n; ++k) {
                const int x = near[k];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = v + e == x ? 0.0 : w[e];
            }
        }
    }
};

// The weights of 4 tokens from v on.  `less`: the draft's row is taken off (what it holds is not read where nothing has been refused: it may be nobody's).
template <typename T, typename Q>
__device__ __forceinline__ void rest_of(const VerifyRun& r, const Rest& s, const Refused& refused, int v, bool less, double (&w)[4],
                                        const uint64_t* powers = nullptr) {
    const VerifyArgs& a = r.a;
    float x[4], q[4];
    elements<T, 4>(a.logits, (int64_t)s.row * a.logits_stride, v, a.V, -__builtin_inff(), x);
    if (less) elements<Q, 4>(a.draft, (int64_t)s.row * a.draft_stride, v, a.V, 0.0f, q);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = clean(x[e]);
    if (powers != nullptr) {
        weights_of(x, s.top, s.heat, powers, w);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = weight_of(x[e], s.top, s.heat);
    }
    if (less) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = fmax(fma(s.scale, w[e], -(s.by * (double)(q[e] > 0.0f ? q[e] : 0.0f))), 0.0);
    } else if (a.draft != nullptr) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] *= s.scale;
    } else {
        refused.out(s.refused, v, w);
    }
}

// What is left of the chunks of a row of which no draft's row has been taken off, by the whole workgroup (without a barrier at the end).
template <typename T, typename Q>
__device__ __forceinline__ void chunks_left(const VerifyRun& r, const Rest& rest, const RowStat& s, const Refused& list, double* chunk_sums, WalkShared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const ChunkStat* of = r.chunks + (size_t)rest.row * r.nc;
    // A chunk lacks its refused tokens: their weights are taken off its sum, unless they are most of it; then what is left is summed again.
    const bool plain = r.a.draft == nullptr;
    const int refused = plain ? rest.refused : 0;
    if (tid == 0) sh.queued = 0;
    __syncthreads();
    if (refused <= kNear) {
        for (int c = tid; c < r.nc; c += kWalkThreads) {
            const double sum = of[c].sum * weight_of(of[c].top, s.top, rest.heat) * (plain ? 1.0 : rest.scale);
            double off = 0.0;
            for (int k = 0; k < refused; ++k) off += list[k] / kChunk == c ? sh.weight[k] : 0.0;
            chunk_sums[c] = sum - off;
            if (off > 0.5 * sum) sh.queue[atomicAdd(&sh.queued, 1)] = c;        // (has one of the refused)
        }
        __syncthreads();
        // four chunks at a time
        constexpr int PARTS = kWalkWaves / 4, EACH = kChunk / (4 * kWave * PARTS);
        const int queued = sh.queued;
        for (int k0 = 0; k0 < queued; k0 += 4) {
            const int k = k0 + wave / PARTS;
            if (k < queued) {
                const int v = sh.queue[k] * kChunk + 4 * (kWave * (wave % PARTS) + lane);
                double sum = 0.0;
#pragma unroll
                for (int e = 0; e < EACH; ++e) {
                    double w[4];
                    rest_of<T, Q>(r, rest, list, v + e * 4 * kWave * PARTS, false, w);
                    sum += (w[0] + w[1]) + (w[2] + w[3]);
                }
                sum = wave_sum(sum);
                if (lane == 0) sh.part[wave] = sum;
            }
            __syncthreads();
            if (k < queued && wave % PARTS == 0 && lane == 0) {
                double sum = 0.0;
#pragma unroll
                for (int e = 0; e < PARTS; ++e) sum += sh.part[wave + e];
                chunk_sums[sh.queue[k]] = sum;
            }
            __syncthreads();
        }
    } else {
        // (of so many all chunks, a wavefront each)
        for (int c = wave; c < r.nc; c += kWalkWaves) {
            double sum = 0.0;
#pragma unroll 4
            for (int k = 0; k < kChunk / 256; ++k) {
                double w[4];
                rest_of<T, Q>(r, rest, list, c * kChunk + 256 * k + 4 * lane, false, w);
                sum += (w[0] + w[1]) + (w[2] + w[3]);
            }
            sum = wave_sum(sum);
            if (lane == 0) chunk_sums[c] = sum;
        }
    }
}

// The next token, drawn from what is left where the walk has ended; by the whole workgroup.  The chunks' sums and the weights within a chunk are the same numbers (with
// `powers`, as verify_left_kernel sums them), or positive together: a chunk that is chosen has a token.
template <typename T, typename Q>
__device__ __forceinline__ void draw_next(const VerifyRun& r, int b, const WalkEnd& end, const Refused& list, int row0, double* chunk_sums, WalkShared& sh,
                                          const uint64_t* powers = nullptr) {
    const VerifyArgs& a = r.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool plain = a.draft == nullptr;
    Rest rest = end.rest;
    const RowStat s = end.row;
    double total = 0.0;
    for (int turn = 0;; ++turn) {
        // sums of the chunks
        __syncthreads();
        if (plain || rest.by == 0.0) {
            chunks_left<T, Q>(r, rest, s, list, chunk_sums, sh);
        } else if (turn == 0) {
            for (int c = tid; c < r.nc; c += kWalkThreads) chunk_sums[c] = r.left[(size_t)row0 * r.nc + c];
        } else {
            for (int c = wave; c < r.nc; c += kWalkWaves) {
                double sum = 0.0;
#pragma unroll 4
                for (int k = 0; k < kChunk / 256; ++k) {
                    const int v = c * kChunk + 256 * k + 4 * lane;
                    if (v >= a.V) continue;
                    double w[4];
                    rest_of<T, Q>(r, rest, list, v, true, w, powers);
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
        if (total > 0.0 || turn == 2) break;
        // nothing is left: r as it was before the last refusal
        if (turn == 0 && plain && rest.refused > 0) {
            --rest.refused;
            if (rest.refused >= kNear && tid == 0) list.marks[list[rest.refused]] = 0;
        } else if (turn == 0 && end.open) {
            rest.scale = end.old_scale / s.sum;
            rest.by = end.old_by;
        } else {
            // that was rounding, or random numbers were none
            rest.scale = 1.0 / s.sum;
            rest.by = 0.0;
            rest.refused = 0;
        }
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
            const double upto = sum_up_to(sum) + before_sum;
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
    rest_of<T, Q>(r, rest, list, v, rest.by != 0.0, w, powers);
    const double own = (w[0] + w[1]) + (w[2] + w[3]);
    const double upto = sum_up_to(own);
    if (lane == 63) sh.part[wave] = upto;
    __syncthreads();
    double sum = upto - own;
#pragma unroll
    for (int k = 0; k < kWalkWaves; ++k) sum += k < wave ? sh.part[k] : 0.0;
    int first = 0x7fffffff, last = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        sum += w[e];
        if (w[e] > 0.0 && v + e < a.V) {
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

// A workgroup per sequence.  Latency bounds it, reads that depend on each other: 7 us for 64 chains of up to 5 tokens with draft probabilities, 11 for one of 4 without, whose
// next token it draws, 15 to 18 for 32 trees of up to 16.  Where siblings ask for the sum of what is left, that is one workgroup's over the vocabulary (8 trees of up to 31 tokens: 9 us),
// without draft probabilities over the chunks.  6000 siblings of 9001 ids, all refused: 4.1 ms, 0.7 us each.
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
    const Heat heat = heat_of(a.temperature != nullptr ? a.temperature[b] : 1.0f);
    const float ninf = -__builtin_inff();
    uint8_t* const marks = a.draft == nullptr ? marks_of(r, row0, n) : nullptr;
    if (marks != nullptr)
        for (int v = 16 * tid; v < r.nc * kChunk; v += 16 * kWalkThreads) *reinterpret_cast<uint4*>(marks + v) = uint4{0, 0, 0, 0};

    // (read now, wanted later)
    auto before_of = [&](int i) { return a.parent != nullptr ? a.parent[row0 + i] : i - 1; };
    int before0 = -1, token0 = -1;
    float u0 = 0.0f;
    if (tid < n) {
        if (tid > 0) before0 = before_of(tid);
        token0 = a.tokens[row0 + tid];
        u0 = a.uniform[row0 + tid];
    }
    auto row_of = [&](int i) { return i < kNear ? sh.rows + i : r.rows + row0 + i; };

    // rows: their chunks joined, a wavefront each
    for (int i = wave; i < n; i += kWalkWaves) {
        const ChunkStat* of = r.chunks + (size_t)(row0 + i) * r.nc;
        const ChunkStat mine = lane < r.nc ? of[lane] : ChunkStat{0.0, ninf, 0x7fffffff};
        float top = mine.top;
        for (int c = kWave + lane; c < r.nc; c += kWave) top = fmaxf(top, of[c].top);
        top = wave_max(top);
        double sum = 0.0;
        int at = 0x7fffffff;
        for (int c = lane; c < r.nc; c += kWave) {
            const ChunkStat s = c == lane ? mine : of[c];
            if (heat.scale >= 0.0) sum += s.sum * weight_of(s.top, top, heat);
            else if (s.top == top) at = min(at, s.at);
        }
        sum = wave_sum(sum);
        at = wave_min(at);
        if (lane == 0) {
            RowStat* const to = row_of(i);
            to->sum = sum;
            to->top = top;
            to->at = top == ninf ? -1 : at;
        }
    }
    __syncthreads();
    // tokens: their probabilities behind the one they continue
    for (int i = tid; i < n; i += kWalkThreads) {
        if (i == 0) continue;
        const int before = i == tid ? before0 : before_of(i), x = i == tid ? token0 : a.tokens[row0 + i];
        double p = 0.0, q = 1.0;
        if (before >= 0 && before < i && x >= 0 && x < a.V) {
            const RowStat s = *row_of(before);
            const int64_t t = row0 + before;
            if (heat.scale < 0.0) p = x == s.at ? 1.0 : 0.0;
            else if (s.top != ninf) p = weight_of(clean(Elements<T>::one(a.logits, t * a.logits_stride + x)), s.top, heat) / s.sum;
            if (a.draft != nullptr) {
                const float d = Elements<Q>::one(a.draft, t * a.draft_stride + x);
                q = d > 0.0f ? (double)d : 0.0;
            }
        }
        RowStat* const to = row_of(i);
        to->p = p;
        to->q = q;
    }
    __syncthreads();

    // The walk, by the first wavefront: tokens continue earlier ones, so that one way through them in their order is enough.  The
    // others wait to be asked for the sum of what is left.
    int cur = 0, kept = 1, refused = 0;
    double scale = 1.0, by = 0.0;            // r = max(scale p - by q, 0); without q p / scale but for those refused
    double want_scale = 1.0, want_by = 0.0;  // r before it is divided by its sum; without q want_scale is `scale` before the last refusal
    double summed = 1.0;                     // without q: `scale` when it was last summed
    bool open = false;                       // that sum is wanted for the next question
    const Refused list{sh.list, r.refused + row0, marks};
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
                        before = j0 == 0 ? before0 : before_of(i);
                        x = j0 == 0 ? token0 : a.tokens[row0 + i];
                        u = j0 == 0 ? u0 : a.uniform[row0 + i];
                        p = row_of(i)->p;
                        q = row_of(i)->q;
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
                if (heat.scale >= 0.0) {
                    if (a.draft != nullptr) {
                        rk = fmax(scale * pk - by * qk, 0.0);
                    } else {
                        if (refused <= kNear) {
                            for (int i = lane; i < refused; i += kWave) twice |= sh.list[i] == token;
                        } else if (token >= 0 && token < a.V) {
                            twice = marks[token] != 0;
                        }
                        twice = __builtin_amdgcn_ballot_w64(twice) != 0;
                        rk = twice ? 0.0 : pk / scale;
                    }
                }
                if ((double)uk * qk < rk) {
                    cur = j0 + k;
                    if (lane == 0) keep[kept] = cur;
                    ++kept;
                    if (marks != nullptr) {
                        for (int i = lane; i < refused; i += kWave) marks[list[i]] = 0;
                        __threadfence_block();
                    }
                    refused = 0;
                    scale = summed = 1.0;
                    by = 0.0;
                } else if (heat.scale >= 0.0) {
                    if (a.draft != nullptr) {
                        want_scale = scale;
                        want_by = by + 1.0;
                        open = true;
                    } else if (!twice && token >= 0 && token < a.V) {
                        if (lane == 0) {
                            list.put(refused, token);
                            if (refused < kNear) sh.weight[refused] = pk * row_of(cur)->sum;
                        }
                        __threadfence_block();
                        ++refused;
                        // The difference is off by 4e-14, which is much of it where little is left: when half of the last sum is refused it is summed anew
                        // (chunk by chunk, and of mostly refused chunks the tokens; a border is then off by 1.2e-13 of itself at most).
                        want_scale = scale;
                        scale -= pk;
                        open = scale < 0.5 * summed;
                    }
                }
            }
            if (lane == 0) {
                sh.ask = ask;
                const RowStat s = *row_of(cur);
                sh.rest = Rest{row0 + cur, s.top, heat, open ? want_scale / s.sum : scale / s.sum, open ? want_by : by, refused};     // (without q neither counts)
            }
        }
        __syncthreads();
        const bool ask = sh.ask != 0;
        const Rest rest = sh.rest;
        if (!ask) break;
        double sum = 0.0;
        if (a.draft == nullptr) {
            chunks_left<T, Q>(r, rest, *row_of(rest.row - row0), list, chunk_sums, sh);
            __syncthreads();
            for (int c = tid; c < r.nc; c += kWalkThreads) sum += chunk_sums[c];
        } else {
            for (int v = 4 * tid; v < a.V; v += 4 * kWalkThreads) {
                double w[4];
                rest_of<T, Q>(r, rest, list, v, true, w);
                sum += (w[0] + w[1]) + (w[2] + w[3]);
            }
        }
        sum = block_sum(sum, sh.part);
        if (wave == 0) {
            open = false;
            // (where nothing is left r stays)
            if (a.draft != nullptr) {
                if (sum > 0.0) {
                    scale = want_scale / sum;
                    by = want_by / sum;
                }
            } else if (sum > 0.0) {
                scale = summed = sum / row_of(cur)->sum;
            } else {
                --refused;
                if (marks != nullptr && lane == 0) marks[list[refused]] = 0;
                __threadfence_block();
                scale = want_scale;
            }
        }
    }

    // ---- the next token
    WalkEnd end;
    end.rest = sh.rest;
    __syncthreads();                         // (what the first wavefront writes now has been read)
    if (wave == 0 && lane == 0) {
        a.n_keep[b] = kept;
        sh.sum = scale;
        sh.part[0] = by;
        sh.ask = open;
    }
    __syncthreads();
    end.open = sh.ask;
    end.old_scale = sh.sum;
    end.old_by = sh.part[0];
    const RowStat s = *row_of(end.rest.row - row0);
    end.row = s;
    end.draw = heat.scale >= 0.0 && s.top != ninf;
    if (!end.draw && tid == 0) a.next[b] = s.top == ninf ? -1 : s.at;
    if (a.draft != nullptr) {
        if (tid == 0) r.ends[row0] = end;
        return;
    }
    if (end.draw) draw_next<T, Q>(r, b, end, list, row0, chunk_sums, sh);
}

// With the drafts' probabilities: sums of what is left over a chunk of a sequence's row.  64 sequences of 131072 logits, 50 MB: 11.5 us, where the walk's workgroups took 45 for it.
template <typename T, typename Q>
__global__ __launch_bounds__(kStatThreads) void verify_left_kernel(VerifyRun r) {
    __shared__ uint64_t powers[kParts];
    __shared__ double part[kStatThreads / kWave];
    const VerifyArgs& a = r.a;
    const int tid = threadIdx.x;
    take_powers<kStatThreads>(powers);
    __syncthreads();
    for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
        const int row0 = max(a.q_start[b], 0);
        if (tokens_of(row0, a.q_start[b + 1], a.T) == 0) continue;
        const WalkEnd end = r.ends[row0];
        if (!end.draw || end.rest.by == 0.0) continue;
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < kEach / 4; ++k) {
            double w[4];
            rest_of<T, Q>(r, end.rest, Refused{}, blockIdx.x * kChunk + 4 * (kStatThreads * k + tid), true, w, powers);
            sum += (w[0] + w[1]) + (w[2] + w[3]);
        }
        sum = wave_sum(sum);
        if ((tid & 63) == 0) part[tid >> 6] = sum;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int w = 1; w < kStatThreads / kWave; ++w) sum += part[w];
            r.left[(size_t)row0 * r.nc + blockIdx.x] = sum;
        }
        __syncthreads();
    }
}
// And the next token: 7 us.
template <typename T, typename Q>
__global__ __launch_bounds__(kWalkThreads) void verify_draw_kernel(VerifyRun r) {
    extern __shared__ double chunk_sums[];               // [nc]
    __shared__ WalkShared sh;
    __shared__ uint64_t powers[kParts];
    take_powers<kWalkThreads>(powers);                   // (draw_next begins with a barrier)
    const int b = blockIdx.x, row0 = max(r.a.q_start[b], 0);
    if (tokens_of(row0, r.a.q_start[b + 1], r.a.T) == 0) return;
    const WalkEnd end = r.ends[row0];
    if (end.draw) draw_next<T, Q>(r, b, end, Refused{}, row0, chunk_sums, sh, powers);
}

// ---- host ---------------------------------------------------------------------------------------

static int chunks_of(int V) { return (V + kChunk - 1) / kChunk; }

size_t verify_workspace(int T, int V) {
    return (size_t)T * ((size_t)chunks_of(V) * (sizeof(ChunkStat) + sizeof(double)) + sizeof(RowStat) + sizeof(WalkEnd) + 8) +
           (size_t)mark_maps(T) * chunks_of(V) * kChunk;
}

template <typename T, typename Q>
static hipError_t launch_walk(const VerifyRun& r, hipStream_t st) {
    const dim3 seqs((unsigned)r.a.B), block(kWalkThreads);
    const size_t lds = (size_t)r.nc * sizeof(double);
    hipLaunchKernelGGL((verify_walk_kernel<T, Q>), seqs, block, lds, st, r);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || r.a.draft == nullptr || r.a.T == 0) return e;
    hipLaunchKernelGGL((verify_left_kernel<T, Q>), dim3((unsigned)r.nc, (unsigned)(r.a.B < 65535 ? r.a.B : 65535)), dim3(kStatThreads), 0, st, r);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_draw_kernel<T, Q>), seqs, block, lds, st, r);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_verify_t(const VerifyRun& r, hipStream_t st) {
    if (r.a.T > 0) {                     // (without rows no sequence has tokens)
        const dim3 grid((unsigned)r.nc, (unsigned)(r.a.T < 65535 ? r.a.T : 65535));
        hipLaunchKernelGGL(verify_stats_kernel<T>, grid, dim3(kStatThreads), 0, st, r);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    switch (r.a.draft_dtype) {
    case 0: return launch_walk<T, F32>(r, st);
    case 1: return launch_walk<T, F16>(r, st);
    default: return launch_walk<T, BF16>(r, st);
    }
}

hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t st) {
    VerifyRun r;
    r.a = a;
    r.nc = chunks_of(a.V);
    r.chunks = static_cast<ChunkStat*>(ws);
    static_assert(sizeof(ChunkStat) % 16 == 0, "marks lie at 16 bytes");
    r.marks = reinterpret_cast<uint8_t*>(r.chunks + (size_t)a.T * r.nc);
    r.rows = reinterpret_cast<RowStat*>(r.marks + (size_t)mark_maps(a.T) * r.nc * kChunk);
    r.ends = reinterpret_cast<WalkEnd*>(r.rows + a.T);
    r.left = reinterpret_cast<double*>(r.ends + a.T);
    r.refused = reinterpret_cast<int*>(r.left + (size_t)a.T * r.nc);
    switch (a.dtype) {
    case 0: return launch_verify_t<F32>(r, st);
    case 1: return launch_verify_t<F16>(r, st);
    default: return launch_verify_t<BF16>(r, st);
    }
}

}  // namespace flashd
