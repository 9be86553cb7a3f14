// Keys that go, by their scores (flashd_cache_evict): of a sequence that has more than its budget of keys the first ones, the last ones and those with
// the largest scores stay, in every layer and kv head those of its own, and move together in their order.
//
// Three kernels.  The first chooses, a workgroup per (layer, sequence, kv head), and leaves for each place (rank) behind the first ones the key that
// goes there; scores it moves by itself.  Rows of K and V then move within the pages, to lower places.  A place below the new length m may hold a key that stays
// and must be read before it is overwritten; the keys behind m are overwritten by nobody.  So the second kernel moves, in order, the keys that come
// from below m (they are a first run of the ranks), a wavefront for 64 bytes of every row, and the third all others, which by then depend on nothing.
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

namespace flashd {

constexpr int kChooseThreads = 1024;
constexpr int kChooseWaves = kChooseThreads / kWave;
constexpr int kDigit = 2048;            // values of a digit: a score's 32 bits are three of them
constexpr int kMoveWaves = 4;
constexpr int kFarRows = 128;           // ranks of a workgroup of the third kernel

// What the first kernel leaves of a unit: its ranks from `first` to `near` come from below m, those from there to m from behind it.
struct EvictUnit {
    int first, near, m;     // all 0: nothing moves
};

struct EvictRun {
    Paged c;
    EvictArgs a;
    EvictUnit* units;       // [layers of the launch][B][Hkv]
    int* from;              // [units][budget] the key of a rank
    int layer0, layers;     // of the launch
    int budget;             // ranks of a unit in `from`
};

// Scores in their order as unsigned numbers; NaN below all, -0 like 0
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x != x ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct ChooseShared {
    int count[kDigit];
    int wave_sum[kChooseWaves];
    int total;
    int digit, above;
    int bad;
};

// Exclusive sum over the workgroup's threads
__device__ __forceinline__ int sum_before(int x, ChooseShared& sh, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int in = lanes_up_to(x);
    __syncthreads();
    if (lane == 63) sh.wave_sum[wave] = in;
    __syncthreads();
    int before = in - x;
    total = 0;
#pragma unroll
    for (int k = 0; k < kChooseWaves; ++k) {
        before += k < wave ? sh.wave_sum[k] : 0;
        total += sh.wave_sum[k];
    }
    return before;
}

// Of the keys in [lo, hi) `need` (0 < need < hi - lo) stay.  The order of the least score among them, digit by digit from the top: each
// time the keys that agree so far are counted by the next digit, and the digit is the one in which the count from above reaches what
// is still needed.  `ties`: how many of those that have exactly this order stay.
__device__ __forceinline__ uint32_t least_kept(const float* score, int lo, int hi, int need, ChooseShared& sh, int& ties) {
    constexpr int EACH = kDigit / kChooseThreads;
    uint32_t prefix = 0;
    int shift = 21;
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass == 2 ? 10 : 11;
        for (int i = threadIdx.x; i < kDigit; i += kChooseThreads) sh.count[i] = 0;
        __syncthreads();
        for (int j = lo + threadIdx.x; j < hi; j += kChooseThreads) {
            const uint32_t x = order_of(score[j]);
            if (pass == 0 || x >> (shift + bits) == prefix) atomicAdd(&sh.count[x >> shift & ((1u << bits) - 1u)], 1);
        }
        __syncthreads();
        // from the top digit down
        int mine = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) mine += sh.count[kDigit - 1 - (threadIdx.x * EACH + e)];
        int total;
        int above = sum_before(mine, sh, total);
        if (above < need && above + mine >= need) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int d = kDigit - 1 - (threadIdx.x * EACH + e), n = sh.count[d];
                if (above < need && above + n >= need) {
                    sh.digit = d;
                    sh.above = above;
                }
                above += n;
            }
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)sh.digit;
        need -= sh.above;
        shift -= pass == 1 ? 10 : 11;
        __syncthreads();
    }
    ties = need;
    return prefix;
}

__global__ __launch_bounds__(kChooseThreads) void evict_choose_kernel(EvictRun r) {
    __shared__ ChooseShared sh;
    const Paged& c = r.c;
    const int unit = blockIdx.x, tid = threadIdx.x;
    const int h = unit % c.Hkv, b = unit / c.Hkv % c.B, y = unit / (c.Hkv * c.B);
    const int raw = c.lens[b], most = c.max_pages << c.page_log2;
    const int len = min(max(raw, 0), most);
    int m = r.a.budgets != nullptr ? min(r.a.budgets[b], r.budget) : r.budget;
    const bool asked = m >= 0 && len > m;
    m = max(m, 0);
    const int first = min(r.a.first, m), recent = min(r.a.recent, m - first);
    // a sequence whose keys have no page, or whose pages that are written to are others' as well, stays as it is
    if (tid == 0) sh.bad = 0;
    __syncthreads();
    if (asked && m > first) {
        const int col0 = first >> c.page_log2, cols = (len + (1 << c.page_log2) - 1) >> c.page_log2;
        bool bad = false;
        for (int k = col0 + tid; k < cols; k += kChooseThreads) {
            const int p = page_at(c, b, k);
            bad |= p < 0 || (k << c.page_log2 < m && r.a.refs[p] > 1);
        }
        if (bad) sh.bad = 1;
    }
    __syncthreads();
    const bool go = asked && sh.bad == 0;
    if (tid == 0 && h == 0 && y == 0 && r.layer0 == 0) r.a.lens_out[b] = go ? m : raw;
    EvictUnit* const left = r.units + unit;
    if (!go || m == first) {
        if (tid == 0) *left = EvictUnit{0, 0, 0};
        return;
    }

    float* const score = r.a.score + (r.layer0 + y) * r.a.score_layer_stride + ((int64_t)b * c.Hkv + h) * r.a.score_stride;
    int* const from = r.from + (int64_t)unit * r.budget;
    const int lo = first, hi = len - recent, need = m - first - recent;
    uint32_t least = 0xffffffffu;
    int ties = 0;
    if (need > 0) least = least_kept(score, lo, hi, need, sh, ties);

    // The keys that stay, in their order: a run of keys for each thread, so that one sum over the threads gives its ranks.
    constexpr int EACH = 4;
    int rank = first, equal = 0, near = first;
    for (int j0 = lo; j0 < len; j0 += EACH * kChooseThreads) {
        float x[EACH];
        int same[EACH], stays[EACH];
        int eq = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int j = j0 + EACH * tid + e;
            x[e] = j < len ? score[j] : 0.0f;
            const uint32_t o = order_of(x[e]);
            same[e] = j < hi && need > 0 && o == least;
            stays[e] = j < len && (j >= hi || (need > 0 && o > least));
            eq += same[e];
        }
        int all_equal;
        int before = equal + sum_before(eq, sh, all_equal);
        int n = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            if (same[e]) stays[e] = before++ < ties;
            n += stays[e];
        }
        int all;
        int at = rank + sum_before(n, sh, all);          // (its barriers: the scores of the run have been read)
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int j = j0 + EACH * tid + e;
            if (!stays[e]) continue;
            from[at] = j;
            if (at != j) score[at] = x[e];
            ++at;
        }
        equal += all_equal;
        rank += all;
        if (j0 < m) {
            int inside = 0;
#pragma unroll
            for (int e = 0; e < EACH; ++e) inside += stays[e] && j0 + EACH * tid + e < m;
            int sum;
            (void)sum_before(inside, sh, sum);
            near += sum;
        }
    }
    if (tid == 0) *left = EvictUnit{first, near, m};
}

// ---- moving rows --------------------------------------------------------------------------------

// Where key j of a unit lies
struct UnitPlace {
    const Paged& c;
    char* pool;             // K or V of the layer and head
    const int* row;         // of the table
    int row_bytes;
    // (every column that is asked for has been looked at by the first kernel; a page that is none by now is page 0 here and the row is left out)
    __device__ __forceinline__ char* at(int j, bool& there) const {
        const int p = row[j >> c.page_log2];
        there = (unsigned)p < (unsigned)c.P;
        return pool + (there ? p : 0) * c.page_bytes + (int64_t)(j & ((1 << c.page_log2) - 1)) * row_bytes;
    }
};

__device__ __forceinline__ UnitPlace place_of(const EvictRun& r, int unit, bool values) {
    const Paged& c = r.c;
    const int h = unit % c.Hkv, b = unit / c.Hkv % c.B, y = unit / (c.Hkv * c.B);
    char* const pool = (values ? c.v : c.k) + (r.layer0 + y) * c.layer_bytes + h * c.head_bytes;
    return UnitPlace{c, pool, c.table + (size_t)b * c.max_pages, c.d * c.esz};
}

// Ranks `first` to `near` in order.  A wavefront takes 64 bytes of each row, 16 rows by 4 lanes at a time and NROW of those together; it reads the next
// ones before it writes these: those come from higher places than any that are written here.
template <int NROW>
__global__ __launch_bounds__(kMoveWaves * kWave) void evict_near_kernel(EvictRun r, int slices) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long id = (long long)blockIdx.x * kMoveWaves + wave;
    const int slice = (int)(id % slices);
    const long long of = id / slices;
    const int units = r.layers * r.c.B * r.c.Hkv;
    if (of >= 2ll * units) return;
    const int unit = (int)(of >> 1);
    const EvictUnit u = r.units[unit];
    if (u.near <= u.first) return;
    const UnitPlace place = place_of(r, unit, of & 1);
    const int* const from = r.from + (int64_t)unit * r.budget;
    const int off = 64 * slice + 16 * (lane & 3), sub = lane >> 2;
    auto key = [&](int rank) { return rank < u.near ? from[rank] : -1; };
    auto load = [&](int rank, int j) {
        bool there;
        const char* p = place.at(j < 0 ? rank : j, there);
        return j > rank && there ? *reinterpret_cast<const u32x4*>(p + off) : u32x4{0, 0, 0, 0};
    };
    int j0[NROW], j1[NROW];
    u32x4 x[NROW], next[NROW];
#pragma unroll
    for (int i = 0; i < NROW; ++i) j0[i] = key(u.first + 16 * i + sub);
#pragma unroll
    for (int i = 0; i < NROW; ++i) j1[i] = key(u.first + 16 * (NROW + i) + sub);
#pragma unroll
    for (int i = 0; i < NROW; ++i) x[i] = load(min(u.first + 16 * i + sub, u.near - 1), j0[i]);
    for (int at = u.first; at < u.near; at += 16 * NROW) {
        int j2[NROW];
#pragma unroll
        for (int i = 0; i < NROW; ++i) j2[i] = key(at + 16 * (2 * NROW + i) + sub);
#pragma unroll
        for (int i = 0; i < NROW; ++i) next[i] = load(min(at + 16 * (NROW + i) + sub, u.near - 1), j1[i]);
        // (the reads above are older than the writes below, and a wavefront's accesses to one address keep their order)
#pragma unroll
        for (int i = 0; i < NROW; ++i) {
            const int rank = at + 16 * i + sub;
            if (j0[i] <= rank) continue;                 // none, or in its place
            bool there, was;
            char* to = place.at(rank, there);
            (void)place.at(j0[i], was);
            if (there && was) *reinterpret_cast<u32x4*>(to + off) = x[i];
        }
#pragma unroll
        for (int i = 0; i < NROW; ++i) {
            j0[i] = j1[i];
            j1[i] = j2[i];
            x[i] = next[i];
        }
    }
}

// Ranks `near` to m, kFarRows of them to a workgroup.
__global__ __launch_bounds__(kMoveWaves * kWave) void evict_far_kernel(EvictRun r, int slices) {
    const int units = r.layers * r.c.B * r.c.Hkv;
    const int per_row = 4 * slices, rows = kMoveWaves * kWave / per_row;
    const int off = 16 * (threadIdx.x % per_row), sub = threadIdx.x / per_row;
    for (int of = blockIdx.y; of < 2 * units; of += gridDim.y) {
        const int unit = of >> 1;
        const EvictUnit u = r.units[unit];
        const int begin = max(u.near, (int)blockIdx.x * kFarRows), end = min(u.m, ((int)blockIdx.x + 1) * kFarRows);
        if (begin >= end) continue;
        const UnitPlace place = place_of(r, unit, of & 1);
        const int* const from = r.from + (int64_t)unit * r.budget;
        for (int rank = begin + sub; rank < end; rank += rows) {
            bool there, was;
            const char* src = place.at(from[rank], was);
            char* to = place.at(rank, there);
            if (was && there) *reinterpret_cast<u32x4*>(to + off) = *reinterpret_cast<const u32x4*>(src + off);
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------

// Layers of a launch: as many as have at most 64 MB of ranks and fit a launch, so that the workspace of many layers has a bound
static int evict_layers(const Paged& c, int budget) {
    const int64_t one = (int64_t)c.B * c.Hkv * ((int64_t)budget * 4 + (int64_t)sizeof(EvictUnit));
    int64_t n = (64ll << 20) / one;
    n = n < kEvictMostUnits / (c.B * c.Hkv) ? n : kEvictMostUnits / (c.B * c.Hkv);
    return (int)(n < 1 ? 1 : n < c.layers ? n : c.layers);
}
static int ranks_of(const Paged& c, int budget) {
    const int most = c.max_pages << c.page_log2;
    return budget < most ? budget : most;
}

size_t evict_workspace(const Paged& c, int budget) {
    const int ranks = ranks_of(c, budget);
    return (size_t)evict_layers(c, ranks) * c.B * c.Hkv * ((size_t)ranks * 4 + sizeof(EvictUnit)) + 16;
}

hipError_t launch_cache_evict(const Paged& c, const EvictArgs& a, void* ws, hipStream_t st) {
    EvictRun r;
    r.c = c;
    r.a = a;
    r.budget = ranks_of(c, a.budget);
    const int layers = evict_layers(c, r.budget);
    const int64_t of_layer = (int64_t)c.B * c.Hkv;
    r.units = static_cast<EvictUnit*>(ws);
    r.from = reinterpret_cast<int*>(r.units + layers * of_layer);
    const int slices = c.d * c.esz / 64;
    for (r.layer0 = 0; r.layer0 < c.layers; r.layer0 += layers) {
        r.layers = c.layers - r.layer0 < layers ? c.layers - r.layer0 : layers;
        const int64_t units = r.layers * of_layer;
        hipLaunchKernelGGL(evict_choose_kernel, dim3((unsigned)units), dim3(kChooseThreads), 0, st, r);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || r.budget == 0) {
            if (e != hipSuccess) return e;
            continue;
        }
        const int64_t waves = 2 * units * slices;
        hipLaunchKernelGGL(evict_near_kernel<8>, dim3((unsigned)((waves + kMoveWaves - 1) / kMoveWaves)), dim3(kMoveWaves * kWave), 0, st, r, slices);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        const dim3 far((unsigned)((r.budget + kFarRows - 1) / kFarRows), (unsigned)(2 * units < 65535 ? 2 * units : 65535));
        hipLaunchKernelGGL(evict_far_kernel, far, dim3(kMoveWaves * kWave), 0, st, r, slices);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace flashd
