// Keys that go, by their scores (flashd_cache_evict): of a sequence that has more than its budget of keys the first ones, the last ones and those with
// the largest scores stay, in every layer and kv head those of its own, and move together in their order.
//
// The first kernel chooses, a workgroup per (layer, sequence, kv head), and leaves for each place (rank) behind the first ones the key that
// goes there; scores it moves by itself.  Rows of K and V then move within the pages, to lower places.  A place below the new length m may hold a key that stays
// and must be read before it is overwritten; the keys behind m are overwritten by nobody.  So the second kernel moves, in order, the keys that come
// from below m (they are a first run of the ranks), and the third all others, which by then depend on nothing.  Of many units the second one moves them all.
//
// Bytes bound it: rows that stay and move are read and written once, at 4.8 TB/s where a large copy has 4.84.  Before them stands the choice: 12 us for 1040 scores,
// 47 us for 65536 of them (five passes of one CU, by the instructions).  16 sequences of 1040 keys to 1024 keys 33 us, 8 layers of 8 prompts of 1500 to 8000 keys to 1024
// 146 us (548 MB), 2 layers of 65536 keys to 16384 123 us (274 MB).
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

namespace flashd {

constexpr int kDigit = 2048;            // values of a digit: a score's 32 bits are three of them
constexpr int kNearThreads = 1024;
constexpr int kNearRows = 4;            // rows of a thread in a round
constexpr int kFarThreads = 256;
constexpr int kFarRows = 128;           // ranks of a workgroup of the third kernel

// What the first kernel leaves of a unit: its ranks from `first`, the first one that moves, to `near` come from below m, those from there to m from behind it.
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

// Scores lie over few digits (powers of two and quarters), which lanes that add to one counter would wait for one by one: so there are some of each digit.
constexpr int kCopies = 4;
constexpr int kCopyPitch = kDigit + 8;
constexpr int kAhead = 8;               // scores of a thread on their way

template <int THREADS> struct ChooseShared {
    alignas(16) int count[kCopies][kCopyPitch];
    int wave_sum[2][THREADS / kWave];
    int digit, above;
    int bad;
    int near, first;
};

// How many lanes before this one are in the mask
__device__ __forceinline__ int lanes_before(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// A wavefront's run of keys [j0, j1), the first kAhead of a lane's scores in registers
struct Run {
    const float* score;
    int j0, j1, lane;
    float x0[kAhead];
    __device__ __forceinline__ void load(int at, float (&x)[kAhead]) const {
        if (at + 64 * kAhead <= j1) {
            const float* p = score + at;
#pragma unroll
            for (int e = 0; e < kAhead; ++e) x[e] = p[64 * e + lane];
        } else {
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                x[e] = 0.0f;
                if (at + 64 * e < j1) x[e] = score[min(at + 64 * e + lane, j1 - 1)];
            }
        }
    }
    // f(j, x, whether there is one) for all of the lane's scores, 64 keys at a time
    template <class F> __device__ __forceinline__ void over(F&& f) const {
        float x[kAhead], next[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) x[e] = x0[e];
#pragma unroll 1
        for (int at = j0; at < j1; at += 64 * kAhead) {
            if (at + 64 * kAhead < j1) load(at + 64 * kAhead, next);
            if (at + 64 * kAhead <= j1) {
#pragma unroll
                for (int e = 0; e < kAhead; ++e) f(at + 64 * e + lane, x[e], true);
            } else {
#pragma unroll
                for (int e = 0; e < kAhead; ++e) {
                    if (at + 64 * e < j1) f(at + 64 * e + lane, x[e], at + 64 * e + lane < j1);
                }
            }
#pragma unroll
            for (int e = 0; e < kAhead; ++e) x[e] = next[e];
        }
    }
};

// Of the keys of all wavefronts' runs `need` (more than 0, fewer than there are) stay.  The order of the least score among them, digit by digit from the top: each
// time the keys that agree so far are counted by the next digit, and the digit is the one in which the count from above reaches what
// is still needed.  `ties`: how many of those that have exactly this order stay.
template <int THREADS> __device__ __forceinline__ uint32_t least_kept(const Run& run, int need, ChooseShared<THREADS>& sh, int& ties) {
    constexpr int EACH = kDigit / THREADS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t prefix = 0;
    int shift = 21;
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass == 2 ? 10 : 11;
        for (int i = 4 * tid; i < kCopies * kCopyPitch; i += 4 * THREADS) *reinterpret_cast<u32x4*>(&sh.count[0][i]) = u32x4{0, 0, 0, 0};
        __syncthreads();
        int* const mine_of = sh.count[lane % kCopies];
        if (pass == 0) {
            run.over([&](int, float x, bool is) {
                if (is) atomicAdd(&mine_of[order_of(x) >> 21], 1);
            });
        } else if (prefix == 0) {
            // (NaN have order 0, and nothing else has this digit)
            if (tid == 0) mine_of[0] = need;
        } else {
            // those that agree so far have the prefix's sign, and so the order's bits are the score's, or all of them the other way
            const uint32_t flip = prefix >> (31 - shift - bits) != 0 ? 0x80000000u : 0xffffffffu;
            const uint32_t top = prefix << (shift + bits);
            run.over([&](int, float x, bool is) {
                const uint32_t o = __float_as_uint(x + 0.0f) ^ flip ^ top;
                if (is && o < 1u << (shift + bits) && x == x) atomicAdd(&mine_of[o >> shift], 1);
            });
        }
        __syncthreads();
        // from the top digit down
        int n[EACH], mine = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            n[e] = 0;
#pragma unroll
            for (int k = 0; k < kCopies; ++k) n[e] += sh.count[k][kDigit - 1 - (tid * EACH + e)];
            mine += n[e];
        }
        const int in = lanes_up_to(mine);
        if (lane == 63) sh.wave_sum[0][wave] = in;
        __syncthreads();
        int above = in - mine;
#pragma unroll
        for (int k = 0; k < THREADS / kWave; ++k) above += k < wave ? sh.wave_sum[0][k] : 0;
        if (above < need && above + mine >= need) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                if (above < need && above + n[e] >= need) {
                    sh.digit = kDigit - 1 - (tid * EACH + e);
                    sh.above = above;
                }
                above += n[e];
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

template <int THREADS> __global__ __launch_bounds__(THREADS) void evict_choose_kernel(EvictRun r) {
    __shared__ ChooseShared<THREADS> sh;
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
        for (int k = col0 + tid; k < cols; k += THREADS) {
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
    // Each wavefront has a run of keys, counts those that stay, and then knows the ranks of its own.
    const int lane = tid & 63, wave = tid >> 6;
    const int each = ((hi - lo + THREADS / kWave - 1) / (THREADS / kWave) + 63) & ~63;
    Run run;
    run.score = score;
    run.lane = lane;
    run.j0 = __builtin_amdgcn_readfirstlane(min(lo + wave * each, hi));
    run.j1 = min(run.j0 + each, hi);
    if (tid == 0) {
        sh.near = first;
        sh.first = m;
    }
    if (need > 0) {
        run.load(run.j0, run.x0);
        int ties;
        const uint32_t o = least_kept(run, need, sh, ties);
        const bool odd = o == 0;                         // the least one that stays is NaN, and all others stay
        const float least = __uint_as_float((o & 0x80000000u) != 0 ? o ^ 0x80000000u : ~o);
        int n_sure = 0, n_equal = 0;
        run.over([&](int, float x, bool is) {
            n_sure += is && (odd ? x == x : x > least);
            n_equal += is && (odd ? x != x : x == least);
        });
        n_sure = lanes_up_to(n_sure);
        n_equal = lanes_up_to(n_equal);
        if (lane == 63) {
            sh.wave_sum[0][wave] = n_sure;
            sh.wave_sum[1][wave] = n_equal;
        }
        __syncthreads();
        int rank = first, seen = 0;
        for (int k = 0; k < wave; ++k) {
            rank += sh.wave_sum[0][k];
            seen += sh.wave_sum[1][k];
        }
        rank = __builtin_amdgcn_readfirstlane(rank + min(seen, ties));
        seen = __builtin_amdgcn_readfirstlane(seen);
        run.over([&](int j, float x, bool is) {
            bool stays = is && (odd ? x == x : x > least);
            const bool equals = is && (odd ? x != x : x == least);
            const uint64_t equal = __builtin_amdgcn_ballot_w64(equals);
            if (equal != 0) {
                // the first ones of those stay
                stays |= equals && seen + lanes_before(equal) < ties;
                seen += __popcll(equal);
            }
            const uint64_t stay = __builtin_amdgcn_ballot_w64(stays);
            int* const to = from + rank;                 // (the same for all lanes)
            if (stays) to[(uint32_t)lanes_before(stay)] = j;
            rank += __popcll(stay);
        });
    }
    for (int k = tid; k < recent; k += THREADS) from[m - recent + k] = hi + k;
    __syncthreads();
    // Their scores move down: all of a round have been read before any is written, and later rounds' come from behind what is written.
    constexpr int N = 8;
    int near = 0, moved = m;             // of the wavefront: ranks from below m, the first one that moves
    for (int r0 = first; r0 < m; r0 += N * THREADS) {
        int j[N];
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) j[e] = from[min(r0 + e * THREADS + tid, m - 1)];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = score[j[e]];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int at = r0 + e * THREADS + tid;
            const bool moves = at < m && j[e] != at;
            if (moves) score[at] = x[e];
            near += __popcll(__builtin_amdgcn_ballot_w64(at < m && j[e] < m));
            const uint64_t some = __builtin_amdgcn_ballot_w64(moves);
            if (some != 0) moved = min(moved, at - lane + __builtin_ctzll(some));
        }
    }
    if (lane == 0) {
        atomicAdd(&sh.near, near);
        atomicMin(&sh.first, moved);
    }
    __syncthreads();
    if (tid == 0) *left = EvictUnit{min(sh.first, sh.near), sh.near, m};
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

// Ranks `first` to `near` in order (to m with `all`), of a unit's K or V by one workgroup, or by some that take a slice of every row each.  All rows of a round have been read before any
// is written, and the next round's are on their way by then: they come from behind all that is written.
__global__ __launch_bounds__(kNearThreads) void evict_near_kernel(EvictRun r, int slices, int all) {
    constexpr int N = kNearRows;
    const int units = r.layers * r.c.B * r.c.Hkv;
    // (slices of a row share its 128-byte lines: their workgroups are 8 apart, on one XCD)
    const long long g = blockIdx.x / (8 * slices), in = blockIdx.x % (8 * slices);
    const long long of = 8 * g + (in & 7);
    if (of >= 2ll * units) return;
    const int slice = (int)(in >> 3), unit = (int)(of >> 1);
    const EvictUnit u = r.units[unit];
    const int end = all ? u.m : u.near;
    if (end <= u.first) return;
    const UnitPlace place = place_of(r, unit, of & 1);
    const int* const from = r.from + (int64_t)unit * r.budget;
    const int pieces = place.row_bytes / 16 / slices, rows = kNearThreads / pieces;
    const int sub = threadIdx.x / pieces, off = 16 * (slice * pieces + (int)threadIdx.x % pieces);
    bool there[N], there_next[N];
    u32x4 x[N], next[N];
    int j[N];
    auto key = [&](int at) {
#pragma unroll
        for (int i = 0; i < N; ++i) j[i] = from[min(at + i * rows + sub, end - 1)];
    };
    auto load = [&](u32x4 (&to)[N], bool (&is)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = *reinterpret_cast<const u32x4*>(place.at(j[i], is[i]) + off);
    };
    key(u.first);
    load(x, there);
    key(u.first + N * rows);
    for (int at = u.first; at < end; at += N * rows) {
        load(next, there_next);
        key(at + 2 * N * rows);
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));       // this round's rows have been read
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int rank = at + i * rows + sub;
            bool is;
            char* to = place.at(min(rank, end - 1), is);
            if (rank < end && is && there[i]) *reinterpret_cast<u32x4*>(to + off) = x[i];
            x[i] = next[i];
            there[i] = there_next[i];
        }
    }
}

// Ranks `near` to m, kFarRows of them to a workgroup.  Their rows are read once (past the caches: 128 -> 116 us for 2 layers of 65536 keys to 16384).
__global__ __launch_bounds__(kFarThreads) void evict_far_kernel(EvictRun r) {
    constexpr int N = 4;
    const int units = r.layers * r.c.B * r.c.Hkv;
    for (int of = blockIdx.y; of < 2 * units; of += gridDim.y) {
        const int unit = of >> 1;
        const EvictUnit u = r.units[unit];
        const int begin = max(u.near, (int)blockIdx.x * kFarRows), end = min(u.m, ((int)blockIdx.x + 1) * kFarRows);
        if (begin >= end) continue;
        const UnitPlace place = place_of(r, unit, of & 1);
        const int* const from = r.from + (int64_t)unit * r.budget;
        const int pieces = place.row_bytes / 16, rows = kFarThreads / pieces;
        const int off = 16 * (threadIdx.x % pieces), sub = threadIdx.x / pieces;
        for (int at = begin + sub; at < end; at += N * rows) {
            int j[N];
            bool was[N];
            u32x4 x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) j[i] = from[min(at + i * rows, end - 1)];
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(place.at(j[i], was[i]) + off));
#pragma unroll
            for (int i = 0; i < N; ++i) {
                bool is;
                char* to = place.at(min(at + i * rows, end - 1), is);
                if (at + i * rows < end && is && was[i]) *reinterpret_cast<u32x4*>(to + off) = x[i];
            }
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
    for (r.layer0 = 0; r.layer0 < c.layers; r.layer0 += layers) {
        r.layers = c.layers - r.layer0 < layers ? c.layers - r.layer0 : layers;
        const int64_t units = r.layers * of_layer;
        // A unit's choice is the call's time where there are few units, and two halves as large go by turns where there are more than CUs (8 layers of 8 heads of 8 sequences
        // 156 -> 148 us, 128 units of 1040 keys 38.7 -> 37.2; 16 units of 65536 keys 115 -> 126).
        if (units < 128) hipLaunchKernelGGL(evict_choose_kernel<1024>, dim3((unsigned)units), dim3(1024), 0, st, r);
        else hipLaunchKernelGGL(evict_choose_kernel<512>, dim3((unsigned)units), dim3(512), 0, st, r);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (r.budget == 0) continue;
        // As many workgroups as take the CUs twice move the rows, each of them slices of at least 64 bytes where there are few units.  Of many units each moves all ranks
        // (128 units of 1040 keys 47 -> 39 us with their slices and without the third kernel, 512 of 1500 to 8000 keys 162 -> 156).
        const bool all = 2 * units >= 256;
        int slices = 1;
        while (2 * units * slices < 512 && c.d * c.esz / slices > 64) slices *= 2;
        hipLaunchKernelGGL(evict_near_kernel, dim3((unsigned)((2 * units + 7) / 8 * 8 * slices)), dim3(kNearThreads), 0, st, r, slices, (int)all);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (all) continue;
        const dim3 far((unsigned)((r.budget + kFarRows - 1) / kFarRows), (unsigned)(2 * units < 65535 ? 2 * units : 65535));
        hipLaunchKernelGGL(evict_far_kernel, far, dim3(kFarThreads), 0, st, r);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace flashd
