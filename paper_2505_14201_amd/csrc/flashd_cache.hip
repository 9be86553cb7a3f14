// Writing the paged cache: projected keys and values with norm and rotation on the way
// (append_kernel), and the bookkeeping of sequences that branch, grow and drop what was drafted
// (fork_kernel, reserve_kernel with copy_rows_kernel, commit_kernel).
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

#include <type_traits>

namespace flashd {

// 8 elements that are read once
template <typename T>
__device__ __forceinline__ void load_once(const void* p, size_t i, float (&x)[8]) {
    constexpr int NW = sizeof(typename T::raw) / 2;
    const u32x4* at = reinterpret_cast<const u32x4*>(static_cast<const typename T::raw*>(p) + i);
    u32x4 w[NW];
#pragma unroll
    for (int k = 0; k < NW; ++k) w[k] = __builtin_nontemporal_load(at + k);
    Store<T>::load8(w, 0, x);
}
// 8 elements, rounded to nearest even two by two (one by one in integers that took a fifth of the kernel's instructions)
template <typename T>
__device__ __forceinline__ void store8(void* p, size_t i, const float (&x)[8]) {
    if constexpr (std::is_same_v<T, F32>) {
        Store<T>::store4(p, i, {x[0], x[1], x[2], x[3]});
        Store<T>::store4(p, i + 4, {x[4], x[5], x[6], x[7]});
    } else {
        *reinterpret_cast<u32x4*>(static_cast<typename T::raw*>(p) + i) =
            Mma<T>::pack8(f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]});
    }
}

// ---- norm, rotation and cache write --------------------------------------------------------
//
// Per token and head: x <- x / sqrt(mean x^2 + eps) * w, then (u, v) <- (u cos a - v sin a,
// v cos a + u sin a) for the pairs of the first `rot` elements, a_i = position * inv_freq_i.  The angle
// is formed in fp64 and reduced to a turn there: at position 10^5 an fp32 product would be off
// by 4e-3 radians.  Everything else is fp32 with one rounding at the store.
//
// A row of d elements lies in d / 8 lanes, 8 elements each (one 16-byte load), so the partner of an
// element of a half-split pair is a whole lane away and the sum of squares takes d / 8 lanes.  A
// workgroup takes one token's rows (its q, k and v heads), so that the angles are formed once for
// all of them.
//
// PASSES: how many rows a lane's place in the workgroup takes, all loaded before anything else.  Long calls want few
// workgroups per token, as the search for its sequence and its angles are done in each of them: with one for every 16 rows 12696
// tokens of 32 + 2 x 8 heads of 128 took 92 us where this took 78.  Short ones want the rows spread.  Those tokens take 62 us now, 312 MB
// at 5.0 TB/s (a plain copy moves 5.2); 64 tokens take 4.2, all of it latency.  Workgroups that walk many tokens, the next
// one's rows on their way, were not ahead (76 to 102 where this took 78).
template <typename T, int D, bool FP8, int PASSES>
__global__ __launch_bounds__(256) void append_kernel(Paged c, AppendArgs a) {
    constexpr int LPR = D / 8;                  // lanes per row
    constexpr int RPP = 256 / LPR;              // rows per pass of the workgroup
    __shared__ float cs[D / 2], sn[D / 2];
    __shared__ int part[4];
    const int tid = threadIdx.x;
    const int t = blockIdx.x;
    const int l = tid % LPR;
    const int rows = a.Hq + 2 * c.Hkv;
    const int row0 = blockIdx.y * (RPP * PASSES) + tid / LPR;

    float x[PASSES][8];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * RPP;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[p][e] = 0.0f;
        if (row < a.Hq) load_once<T>(a.q, (size_t)t * a.q_stride + (size_t)row * D + 8 * l, x[p]);
        else if (row < a.Hq + c.Hkv) load_once<T>(a.k, (size_t)t * a.k_stride + (size_t)(row - a.Hq) * D + 8 * l, x[p]);
        else if (row < rows) load_once<T>(a.v, (size_t)t * a.v_stride + (size_t)(row - a.Hq - c.Hkv) * D + 8 * l, x[p]);
    }

    // the token's sequence: the last one that begins at or before it
    int before = 0;
    for (int i = tid; i <= c.B; i += 256) before += c.q_start[i] <= t ? 1 : 0;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) before += __shfl_xor(before, s);
    if ((tid & 63) == 0) part[tid >> 6] = before;
    __syncthreads();
    const int b = __builtin_amdgcn_readfirstlane(part[0] + part[1] + part[2] + part[3] - 1);
    if (b < 0 || b >= c.B) return;              // rows that belong to no sequence stay as they are
    const Seq s = seq_at(c, b);
    const int i = t - s.row0;
    const int key = s.len + i;
    const int page = (unsigned)i < (unsigned)s.n ? page_at(c, b, key >> c.page_log2) : -1;

    const int half = a.rot / 2;
    if (tid < half) {
        const int pos = a.positions != nullptr ? a.positions[t] : key;
        const double turns = (double)pos * (double)a.inv_freq[tid] * 0.15915494309189533577;
        float sv, cv;
        sincospif((float)(2.0 * (turns - rint(turns))), &sv, &cv);
        cs[tid] = cv;
        sn[tid] = sv;
    }
    __syncthreads();

#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int row = row0 + p * RPP;
        const bool is_q = row < a.Hq;
        const bool is_k = !is_q && row < a.Hq + c.Hkv;
        const bool turns = is_q || is_k;
        const void* wp = is_q ? a.q_weight : is_k ? a.k_weight : nullptr;
        if (a.q_weight != nullptr || a.k_weight != nullptr) {
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[p][e], x[p][e], sum);
#pragma unroll
            for (int m = LPR / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
            if (wp != nullptr) {
                float w[8];
                Store<T>::load8(wp, 8 * l, w);
                const float r = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[p][e] = x[p][e] * r * w[e];
            }
        }
        if (half > 0 && a.interleaved) {
            if (turns && 8 * l < a.rot) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float cv = cs[4 * l + e / 2], sv = sn[4 * l + e / 2];
                    const float u = x[p][e], v = x[p][e + 1];
                    x[p][e] = fmaf(u, cv, -(v * sv));
                    x[p][e + 1] = fmaf(v, cv, u * sv);
                }
            }
        } else if (half > 0) {
            // rot is a multiple of 16: half a rotation is whole lanes
            const int hl = half / 8;
            const int lane = tid & 63;
            const int from = l < hl ? lane + hl : lane - hl;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __shfl(x[p][e], from & 63);
            if (turns && l < 2 * hl) {
                const int at = 8 * (l < hl ? l : l - hl);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float sv = l < hl ? -sn[at + e] : sn[at + e];
                    x[p][e] = fmaf(x[p][e], cs[at + e], y[e] * sv);
                }
            }
        }

        if (is_q) {
            const size_t at = (size_t)t * a.qo_stride + (size_t)row * D + 8 * l;
            store8<T>(a.q_out, at, x[p]);
        } else if (row < rows && page >= 0) {
            const int h = is_k ? row - a.Hq : row - a.Hq - c.Hkv;
            char* base = (is_k ? c.k : c.v) + (size_t)page * c.page_bytes + (size_t)h * c.head_bytes;
            const size_t at = (size_t)(key & ((1 << c.page_log2) - 1)) * D + 8 * l;
            if constexpr (FP8) {
                // e4m3 ends at 448: what is larger is stored as that (NaN stays NaN)
                const float scale = is_k ? c.kscale : c.vscale;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = x[p][e] / scale;
                    x[p][e] = z > 448.0f ? 448.0f : z < -448.0f ? -448.0f : z;
                }
                u32x2 w;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    int z = __builtin_amdgcn_cvt_pk_fp8_f32(x[p][4 * e], x[p][4 * e + 1], 0, false);
                    z = __builtin_amdgcn_cvt_pk_fp8_f32(x[p][4 * e + 2], x[p][4 * e + 3], z, true);
                    w[e] = (unsigned)z;
                }
                *reinterpret_cast<u32x2*>(base + at) = w;
            } else {
                store8<T>(base, at, x[p]);
            }
        }
    }
}

template <typename T, int D, bool FP8>
static hipError_t launch_append_d(const Paged& c, const AppendArgs& a, hipStream_t st) {
    const int rows = a.Hq + 2 * c.Hkv, per = 256 / (D / 8), passes = (rows + per - 1) / per;
    const dim3 block(256);
    // a workgroup per token and 16 (32 at d = 64) rows until that fills the chip with two workgroups per compute unit
    if ((long)c.T * passes <= 512) hipLaunchKernelGGL((append_kernel<T, D, FP8, 1>), dim3((unsigned)c.T, (unsigned)passes), block, 0, st, c, a);
    else if (passes <= 2) hipLaunchKernelGGL((append_kernel<T, D, FP8, 2>), dim3((unsigned)c.T, 1), block, 0, st, c, a);
    else if (passes <= 3) hipLaunchKernelGGL((append_kernel<T, D, FP8, 3>), dim3((unsigned)c.T, 1), block, 0, st, c, a);
    else hipLaunchKernelGGL((append_kernel<T, D, FP8, 4>), dim3((unsigned)c.T, (unsigned)((passes + 3) / 4)), block, 0, st, c, a);
    return hipGetLastError();
}
template <typename T, bool FP8>
static hipError_t launch_append_t(const Paged& c, const AppendArgs& a, hipStream_t st) {
    return c.d == 64 ? launch_append_d<T, 64, FP8>(c, a, st) : launch_append_d<T, 128, FP8>(c, a, st);
}

hipError_t launch_cache_append(const Paged& c, const AppendArgs& a, hipStream_t st) {
    switch (a.dtype) {
    case 0: return launch_append_t<F32, false>(c, a, st);
    case 1: return a.fp8 ? launch_append_t<F16, true>(c, a, st) : launch_append_t<F16, false>(c, a, st);
    default: return a.fp8 ? launch_append_t<BF16, true>(c, a, st) : launch_append_t<BF16, false>(c, a, st);
    }
}

// ---- forking --------------------------------------------------------------------------------
//
// table_out[i] = table[parent[i]]; refs[p] counts the table entries that name page p, so every entry
// that changes takes one off the page it named and puts one on the page it names.  Sums of whole
// numbers: the order of the atomics does not matter.  64 sequences from 32: 3 us, the launch's latency.
__global__ __launch_bounds__(256) void fork_kernel(Paged c, int* refs, const int* parent, int B_out,
                                                   int* table_out, int* lens_out) {
    const int i = blockIdx.y;
    const int col = blockIdx.x * 256 + threadIdx.x;
    int from = -1;
    if (i < B_out) {
        from = parent[i];
        if ((unsigned)from >= (unsigned)c.B) from = -1;
        if (col == 0) lens_out[i] = from < 0 ? 0 : c.lens[from];
    }
    if (col >= c.max_pages) return;
    const int now = i < c.B ? c.table[(size_t)i * c.max_pages + col] : -1;
    const int next = from < 0 ? -1 : c.table[(size_t)from * c.max_pages + col];
    if (i < B_out) table_out[(size_t)i * c.max_pages + col] = next;
    const int page = named_page(next), was = named_page(now);
    if (page != was) {
        if ((unsigned)page < (unsigned)c.P) atomicAdd(&refs[page], 1);
        if ((unsigned)was < (unsigned)c.P) atomicSub(&refs[was], 1);
    }
}

hipError_t launch_cache_fork(const Paged& c, int* refs, const int* parent, int B_out, int* table_out,
                             int* lens_out, hipStream_t st) {
    const dim3 grid((unsigned)((c.max_pages + 255) / 256), (unsigned)(B_out > c.B ? B_out : c.B)), block(256);
    hipLaunchKernelGGL(fork_kernel, grid, block, 0, st, c, refs, parent, B_out, table_out, lens_out);
    return hipGetLastError();
}

// ---- reserving ------------------------------------------------------------------------------
//
// One workgroup, so that which sequence gets which page does not depend on the order of anything:
//   1. pages behind a sequence's keys and new tokens go back (refs - 1);
//   2. so do, of a sequence with new tokens, the pages behind its keys from the first one on that another row names too (twins of
//      a sequence that had pages left over, or of one whose length was set back): what is written there is its own;
//   3. a sequence wants the pages from its first empty column to its last, and one more where its
//      last page is part filled and shared (unless it is the first of sequences that are the
//      page's only holders and all grow: that one keeps it);
//   4. free pages (refs 0) are numbered in ascending order, k-th free page -> k-th wanted page.
// Should there be too few, step 4 is left out and the number missing reported; a growing sequence's part-filled page that others name
// too is then held back (named_page()), so that a step that runs on does not write to it, until the next call.
// Latency bounds it, six reads one after the other: 3.9 us for 32 sequences (3.6 where no page lies behind a sequence's keys), 9.0 for
// 64 whose table and counts another kernel has just written (they come from beyond this die's L2).
constexpr int kReserveThreads = 1024;
constexpr int kReserveWaves = kReserveThreads / kWave;
constexpr int kReserveEach = kCacheMaxSeqs / kReserveThreads;     // sequences of a thread
constexpr int kReserveBlocks = 4096;      // the pool is counted in at most that many blocks of 256 m pages

// Exclusive prefix sum over the workgroup's threads; `total` is their sum.
__device__ __forceinline__ int block_scan(int x, int* waves, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int in = lanes_up_to(x);
    __syncthreads();                       // (the sums of an earlier scan have been read)
    if (lane == 63) waves[wave] = in;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kReserveWaves; ++w) {
        const int y = waves[w];
        before += w < wave ? y : 0;
        total += y;
    }
    return before + in - x;
}

// Of the columns lo <= col < end of a row the first whose page is named more than once or held back; `end` where there is none up to
// the first empty one.  Four columns at a time, whose reads run together.
__device__ __forceinline__ int shared_column(const int* row, const int* refs, int P, int lo, int end) {
    for (int col = lo; col < end; col += 4) {
        int page[4], held[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) page[i] = col + i < end ? row[col + i] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) held[i] = (unsigned)page[i] < (unsigned)P ? refs[page[i]] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (page[i] == -1) return end;
            if (page[i] < -1 || held[i] > 1) return col + i;
        }
    }
    return end;
}

__global__ __launch_bounds__(kReserveThreads) void reserve_kernel(Paged c, int* refs, int* report) {
    __shared__ int at[kCacheMaxSeqs + 1];        // wanted pages of the sequences before b
    __shared__ __align__(16) int last[kCacheMaxSeqs];        // part-filled last page of a sequence that grows, or -1
    __shared__ int2 cols[kCacheMaxSeqs];         // that page's column (kShared: others name the page, kCopy: a copy is wanted), and the column behind the last
    __shared__ int count[kReserveBlocks];        // free pages of the blocks before
    __shared__ int waves[kReserveWaves];
    __shared__ unsigned long long beyond;
    __shared__ int shared_behind;                // some sequence has a shared page behind its keys
    constexpr int kCopy = 1 << 30, kShared = 1 << 29;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int mask = (1 << c.page_log2) - 1;
    const int each = (c.B + kReserveThreads - 1) / kReserveThreads;
    if (tid == 0) beyond = 0, shared_behind = 0;
    if (tid < (-c.B & 3)) last[c.B + tid] = -1;          // read four at a time

    // 1. back to the pool.  (`from`: the first column that the row may want a page for; `lo_page`, `end_page`: what it has there and in the
    // last one, read here beside the others)
    int from[kReserveEach], lo_page[kReserveEach], end_page[kReserveEach];
    unsigned long long lacking = 0;
#pragma unroll
    for (int k = 0; k < kReserveEach; ++k) {
        const int b = k * kReserveThreads + tid;
        from[k] = 0;
        lo_page[k] = end_page[k] = -1;
        if (b >= c.B) continue;
        const int next = c.q_start[b + 1];
        const Seq s = seq_of(c.q_start[b], next, c.lens[b], c.T, c.max_pages << c.page_log2);
        int* row = c.table + (size_t)b * c.max_pages;
        const int end = (s.len + s.n + mask) >> c.page_log2, lo = (s.len + mask) >> c.page_log2, first = s.len >> c.page_log2;
        const int tail = lo > 0 ? row[lo - 1] : 0;
        int part = lo > first ? tail : -1, p = end < c.max_pages ? row[end] : -1;
        if (lo < end) {
            lo_page[k] = row[lo];
            end_page[k] = row[end - 1];
        }
        if (part < -1) row[first] = part = named_page(part);        // held back by an earlier call that found too few pages
        for (int col = end; p != -1;) {          // owned pages come first in a row
            row[col] = -1;
            const int page = named_page(p);
            if (page < c.P) atomicSub(&refs[page], 1);
            p = ++col < c.max_pages ? row[col] : -1;
        }
        from[k] = s.n > 0 ? lo : end;
        if (s.n > 0 && tail == -1) {             // not even its keys have pages
            int z = lo - 1;
            from[k] = 0;
            while (from[k] < z) {
                const int mid = (from[k] + z) >> 1;
                if (row[mid] == -1) z = mid;
                else from[k] = mid + 1;
            }
        }
        last[b] = s.n > 0 && part < c.P ? part : -1;
        cols[b] = int2{first, end};
        // tokens that the table has no columns for
        lacking += (unsigned long long)columns_beyond(tokens_of(s.row0, next, c.T), s.n, c.page_log2);
    }
    // (refs have not been read yet, so what follows finds them as these atomics, waited for at the barrier,
    // have left them)
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (lacking > 0) atomicAdd(&beyond, lacking);

    // The pool is counted by blocks of 256 m pages that each fall to one wavefront.  Its first block is kept, as long as it is
    // one read per lane and 64 pages; it is on its way while rows are looked at.
    const int m = (c.P + 256 * kReserveBlocks - 1) / (256 * kReserveBlocks);
    const int blocks = (c.P + 256 * m - 1) / (256 * m);
    int held[4], shares[kReserveEach];           // shares: how many rows name the part-filled page
    auto look = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = wave * 256 + 64 * i + lane;
            held[i] = m == 1 && p < c.P ? refs[p] : 1;
        }
#pragma unroll
        for (int k = 0; k < kReserveEach; ++k) {
            const int b = k * kReserveThreads + tid;
            shares[k] = k < each && b < c.B && last[b] >= 0 ? refs[last[b]] : 0;
        }
    };
    look();

    // 2. pages behind the keys.  All are looked at before any goes back, so that all see the same counts.
    int cut[kReserveEach];                       // the column from which they go
#pragma unroll
    for (int k = 0; k < kReserveEach; ++k) {
        cut[k] = 0x7fffffff;
        if (lo_page[k] == -1) continue;
        const int b = k * kReserveThreads + tid, p = lo_page[k], end = cols[b].y;
        cut[k] = p < -1 || (p < c.P && refs[p] > 1) ? from[k] : shared_column(c.table + (size_t)b * c.max_pages, refs, c.P, from[k] + 1, end);
        if (cut[k] < end) shared_behind = 1;
    }
    __syncthreads();
    if (shared_behind != 0) {
#pragma unroll
        for (int k = 0; k < kReserveEach; ++k) {
            const int b = k * kReserveThreads + tid;
            if (lo_page[k] == -1 || cut[k] >= cols[b].y) continue;
            int* row = c.table + (size_t)b * c.max_pages;
            for (int col = cut[k]; col < cols[b].y; ++col) {
                const int p = row[col];
                if (p == -1) break;
                row[col] = -1;
                const int page = named_page(p);
                if (page < c.P) atomicSub(&refs[page], 1);
            }
            end_page[k] = -1;
            if (cut[k] == from[k]) lo_page[k] = -1;
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        // counts that this compute unit has read lie in its cache as they were
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        look();
    }

    // 3. what each wants
    int run = 0;
#pragma unroll
    for (int k = 0; k < kReserveEach; ++k) {
        if (k >= each) break;
        const int b = k * kReserveThreads + tid;
        int want = 0;
        bool copy = false;
        if (b < c.B) {
            const int* row = c.table + (size_t)b * c.max_pages;
            const int end = cols[b].y, p = last[b];
            int lo = from[k], hi = end;
            if (lo < hi) {
                if (lo_page[k] == -1) hi = lo;
                else if (end_page[k] != -1) lo = hi;
            }
            while (lo < hi) {                    // the first empty column
                const int mid = (lo + hi) >> 1;
                if (row[mid] == -1) hi = mid;
                else lo = mid + 1;
            }
            want = end - lo;
            if (shares[k] > 1) {
                int holders = 0, before = 0;
#pragma unroll 4
                for (int o = 0; o < c.B; o += 4) {
                    const int4 x = *reinterpret_cast<const int4*>(&last[o]);
                    const int four[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool same = four[i] == p;
                        holders += same ? 1 : 0;
                        before += same && o + i < b ? 1 : 0;
                    }
                }
                copy = holders < shares[k] || before > 0;
                cols[b].x |= copy ? kCopy | kShared : kShared;
            }
            report[1 + b] = copy ? p : -1;
        }
        int all;
        const int ex = block_scan(want + (copy ? 1 : 0), waves, all);
        if (b < c.B) at[b] = run + ex;
        run += all;
    }
    if (tid == 0) at[c.B] = run;

    // free pages
    for (int k = wave; k < blocks; k += kReserveWaves) {
        int n = 0;
        if (k == wave && m == 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(held[i] == 0));
            if (lane == 0) count[k] = n;
            continue;
        }
        for (int j = 0; j < 4 * m; j += 4) {
            bool is[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int p = k * 256 * m + 64 * (j + i) + lane;
                is[i] = p < c.P && refs[p] == 0;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(is[i]));
        }
        if (lane == 0) count[k] = n;
    }
    __syncthreads();
    int free_pages = 0;
    for (int k0 = 0; k0 < blocks; k0 += kReserveThreads) {
        const int k = k0 + tid;
        int all;
        const int ex = block_scan(k < blocks ? count[k] : 0, waves, all);
        if (k < blocks) count[k] = free_pages + ex;
        free_pages += all;
    }
    __syncthreads();
    const int missing = (int)min((unsigned long long)max(run - free_pages, 0) + beyond, 0x7fffffffull);
    if (tid == 0) report[0] = missing;
    if (missing > 0) {
        for (int b = tid; b < c.B; b += kReserveThreads) {
            report[1 + b] = -1;
            // a shared page stays unchanged though its copy is missing: what would be written to it has no page
            const int x = cols[b].x;
            if (x & kShared) c.table[(size_t)b * c.max_pages + (x & (kShared - 1))] = -2 - last[b];
        }
        return;
    }

    // 4. the k-th free page to the k-th wanted one
    for (int k = wave; k < blocks; k += kReserveWaves) {
        int rank = count[k];
        for (int j = 0; j < 4 * m && rank < run; ++j) {
            const int p = k * 256 * m + 64 * j + lane;
            bool is = false;
            if (k != wave || m != 1) is = p < c.P && refs[p] == 0;
            else is = (j == 0 ? held[0] : j == 1 ? held[1] : j == 2 ? held[2] : held[3]) == 0;
            const uint64_t all = __ballot(is);
            const int mine = rank + __popcll(all & ((1ull << lane) - 1));
            if (is && mine < run) {
                int lo = 0, hi = c.B;            // the sequence: the last with at[b] <= mine
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (at[mid] <= mine) lo = mid;
                    else hi = mid;
                }
                const int2 to = cols[lo];
                const bool copied = mine == at[lo] && (to.x & kCopy) != 0;
                if (copied) atomicSub(&refs[last[lo]], 1);
                // (of the fresh pages the last one goes to the last column)
                c.table[(size_t)lo * c.max_pages + (copied ? to.x & (kShared - 1) : to.y - (at[lo + 1] - mine))] = p;
                refs[p] = 1;
            }
            rank += __popcll(all);
        }
    }
}

// Rows of the part-filled page that report names into the page that the sequence now has there.
// Workgroup (b, j) takes every gridDim.y-th of the 2 * layers * Hkv pieces.  67 MB, read and written, in 13 us: 5.1 TB/s.
__global__ __launch_bounds__(256) void copy_rows_kernel(Paged c, const int* report) {
    const int b = blockIdx.x;
    const int from = report[1 + b];
    if ((unsigned)from >= (unsigned)c.P) return;
    const Seq s = seq_at(c, b);
    const int to = page_at(c, b, s.len >> c.page_log2);
    if (to < 0) return;
    const int64_t bytes = (int64_t)(s.len & ((1 << c.page_log2) - 1)) * c.d * c.esz;
    for (int j = blockIdx.y; j < 2 * c.layers * c.Hkv; j += gridDim.y) {
        const int h = j % c.Hkv, layer = j / c.Hkv >> 1;
        char* base = (j / c.Hkv & 1 ? c.v : c.k) + (size_t)layer * c.layer_bytes + (size_t)h * c.head_bytes;
        const u32x4* src = reinterpret_cast<const u32x4*>(base + (size_t)from * c.page_bytes);
        u32x4* dst = reinterpret_cast<u32x4*>(base + (size_t)to * c.page_bytes);
        for (int64_t i = threadIdx.x; i < bytes / 16; i += 256) dst[i] = src[i];
    }
}

hipError_t launch_cache_reserve(const Paged& c, int* refs, int* report, hipStream_t st) {
    hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kReserveThreads), 0, st, c, refs, report);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const long pieces = 2L * c.layers * c.Hkv;
    hipLaunchKernelGGL(copy_rows_kernel, dim3((unsigned)c.B, (unsigned)(pieces < 64 ? pieces : 64)), dim3(256), 0,
                       st, c, report);
    return hipGetLastError();
}

// ---- committing -----------------------------------------------------------------------------
//
// Of a sequence's new tokens those that keep[] names (ascending) move together behind its keys: key
// len + keep[i] -> len + i.  As keep[i] >= i, rows may be moved in ascending groups, each group read whole
// before it is written: what a group writes lies before everything that later groups read.  A
// wavefront moves the rows of one (layer, K or V, head), eight such pieces under way.  Up to 6 rows for each of 32 sequences, 32
// layers of 2 x 8 heads of 128: 42 MB, read and written, in 9.5 us, 4.4 TB/s.
template <int RB>       // bytes of a row
__global__ __launch_bounds__(256) void commit_kernel(Paged c, const int* keep, int max_keep,
                                                     const int* n_keep, int* lens_out) {
    constexpr int LPR = RB / 16;                  // lanes per row
    constexpr int GROUP = kWave / LPR;            // rows per load
    constexpr int GROUPS = GROUP >= 8 ? 1 : GROUP >= 4 ? 2 : 4;     // loads of a piece under way
    constexpr int PIECES = 4 / GROUPS * 2;        // pieces under way
    const int b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Seq s = seq_at(c, b);
    int kept = n_keep != nullptr ? min(max(n_keep[b], 0), s.n) : s.n;
    const int* list = keep != nullptr ? keep + (size_t)b * max_keep : nullptr;
    if (keep != nullptr) {
        // the list ends where it stops ascending or leaves the sequence's tokens
        kept = min(kept, max_keep);
        int good = 0;
        for (int i0 = 0; i0 < kept; i0 += kWave) {
            const int i = i0 + lane;
            const int x = i < kept ? list[i] : 0;
            const int y = i > 0 && i < kept ? list[i - 1] : -1;
            const uint64_t bad = __ballot(i < kept && !(x > y && x < s.n));
            const int here = min(kept - i0, kWave);
            if (bad != 0) {
                good += min(here, (int)__builtin_ctzll(bad));
                break;
            }
            good += here;
        }
        kept = good;
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) lens_out[b] = s.len + kept;
    if (keep == nullptr) return;

    // Where the rows of a group lie is the same in every piece.
    const int mask = (1 << c.page_log2) - 1;
    const int all = 2 * c.layers * c.Hkv;
    const int first = blockIdx.y * 4 + wave, step = 4 * gridDim.y;
    for (int i0 = 0; i0 < kept; i0 += GROUP * GROUPS) {
        int64_t from[GROUPS], to[GROUPS];
        bool moves[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const int i = i0 + g * GROUP + lane / LPR;
            const int x = i < kept ? list[i] : i;
            const int sk = s.len + x, dk = s.len + i;
            const int sp = x != i ? page_at(c, b, sk >> c.page_log2) : -1, dp = x != i ? page_at(c, b, dk >> c.page_log2) : -1;
            moves[g] = sp >= 0 && dp >= 0;
            from[g] = (int64_t)sp * c.page_bytes + (sk & mask) * RB + 16 * (lane % LPR);
            to[g] = (int64_t)dp * c.page_bytes + (dk & mask) * RB + 16 * (lane % LPR);
        }
        for (int j0 = first; j0 < all; j0 += PIECES * step) {
            u32x4 x[PIECES][GROUPS];
            char* base[PIECES];
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const int j = j0 + k * step;
                const int h = j % c.Hkv, layer = j / c.Hkv >> 1;
                base[k] = (j / c.Hkv & 1 ? c.v : c.k) + (size_t)layer * c.layer_bytes + (size_t)h * c.head_bytes;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
                    if (j < all && moves[g]) x[k][g] = *reinterpret_cast<const u32x4*>(base[k] + from[g]);
            }
            // the wavefront's loads have all returned before the first of its stores is issued
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
            for (int k = 0; k < PIECES; ++k)
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
                    if (j0 + k * step < all && moves[g]) *reinterpret_cast<u32x4*>(base[k] + to[g]) = x[k][g];
        }
    }
}

hipError_t launch_cache_commit(const Paged& c, const int* keep, int max_keep, const int* n_keep,
                               int* lens_out, hipStream_t st) {
    const long pieces = 2L * c.layers * c.Hkv;
    // four wavefronts a workgroup, two rounds of their pieces each, unless that leaves compute units without work
    long y = keep == nullptr ? 1 : (pieces + 31) / 32;
    if (keep != nullptr && y * c.B < 512) y = (512 + c.B - 1) / c.B;
    if (keep != nullptr && y > (pieces + 3) / 4) y = (pieces + 3) / 4;
    const dim3 grid((unsigned)c.B, (unsigned)y), block(256);
    switch (c.d * c.esz) {
    case 64: hipLaunchKernelGGL(commit_kernel<64>, grid, block, 0, st, c, keep, max_keep, n_keep, lens_out); break;
    case 128: hipLaunchKernelGGL(commit_kernel<128>, grid, block, 0, st, c, keep, max_keep, n_keep, lens_out); break;
    case 256: hipLaunchKernelGGL(commit_kernel<256>, grid, block, 0, st, c, keep, max_keep, n_keep, lens_out); break;
    default: hipLaunchKernelGGL(commit_kernel<512>, grid, block, 0, st, c, keep, max_keep, n_keep, lens_out); break;
    }
    return hipGetLastError();
}

}  // namespace flashd
