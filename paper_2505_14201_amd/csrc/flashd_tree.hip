// Attention of each sequence's new tokens over its keys in the paged cache and, as a chain or a
// tree, over each other (flashd_attn_fwd_tree).
//
// For the new token i of sequence b and query head h, o = sum_j softmax_j(scale q.k_j) v_j over the
// keys j < len (all of them) and the new keys len + j that the token's bits name (a chain: j <= i).
// The heads of a kv group read the same keys, so the rows of a unit of work are pairs (token, head of the
// group), 16 to 128 of them to a tile (tree_rows()), and a unit is (sequence, kv head, row tile).
//
// Sequences differ in length by orders of magnitude and the host does not know by how much, so the
// launch has a fixed number of workgroups and each finds its share of the work by itself: the units'
// blocks of 32 or 64 keys form one long row, of which each workgroup takes a stretch whose length depends only on the
// row's (Walk).  A unit that ends up in several workgroups is
// left as partial states (at most two per workgroup: its first unit, begun by the one before, and its
// last) that merge_tree_kernel joins in the order of the keys: the result does not depend on timing.
//
// LSE: the rows' log-sum-exps are wanted as well.  Where rows are divided by the sum of the rounded weights (bf16) the sum of the unrounded ones is then
// carried beside it: what later weights are held against is the true one.  Instances of their own: the others are as they were.
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"
#include "flashd_rows.h"
#include "flashd_tile_parts.h"

#include <type_traits>

namespace flashd {

constexpr int kTreeBlock = 32;          // keys of a block: a wavefront's step
constexpr int kTreeWaves = 4;
constexpr int kTreeMostGroups = 768;    // workgroups of a launch at most: three per compute unit (rows_per_cu(); f32_per_cu() and two elsewhere)
// What the start of a unit counts, in blocks (of 64 keys in the tile kernel): with 0, 1, 2, 3, 4 and 6 the tile kernel took 28.8,
// 27.8, 26.8, 26.3, 25.4 and 25.8 us for 128 units of 17 to 64 tiles, and for long units it made no difference; the rows kernel
// took 103.8 us with 0 and 103.7 with 8, its own steps being shorter.
constexpr int kRowsStart = 0, kTileStart = 3;
// By how many 64ths the first workgroup of a compute unit gets more than the mean and the second less: the older wavefronts are
// served first, so that with equal shares the first ones of the tile kernel ended after 309 us and the second after 384 (chunks
// of 1000 tokens).  With 0, 4, 6, 8, 10 and 14 the kernel took 365, 355, 351, 345, 343 and 352 us, for trees of 16 tokens with 0, 2,
// 4, 6, 8 and 10 111, 109, 110, 109, 108 and 110.  The rows kernel is bound by HBM from first to last: 177 and 176 us with 0 to 20.
constexpr int kRowsLead = 0, kTileLead = 8;

// Waits until all but the last N loads have arrived.
template <int N> __device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
}

template <typename T> struct Mma16;
template <> struct Mma16<BF16> {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma16<F16> {
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// What a unit that is split leaves for the merge: its place and its number of parts (0: none).
struct TreeSplit {
    int row0;       // first row of the packed tensors
    int h;          // kv head
    int first;      // first row (token, head of the group) of the tile
    int rows;       // rows of the tile
    int parts;
    int w;          // place along the row of blocks of the workgroup with its first part
};

struct TreeRun {
    Paged c;
    TreeArgs a;
    FastDiv group;          // query heads per kv head
    float* parts;           // [2 groups][rows of a tile][d] unnormalised outputs
    float2* stats;          // [2 groups][rows of a tile] reference and sum of weights
    TreeSplit* splits;      // [groups], of the unit that a workgroup begins and does not end
    float* sums;            // [2 groups][rows of a tile] sums of unrounded weights (LSE of bf16)
    int groups;             // workgroups of the launch
};

// The kernel's arguments, read anew where they are asked for.  What only the beginning and the end of a piece need
// is taken from here: kept over the loop in scalar registers, of which there are a hundred, it would push what the loop
// needs out of them.
__device__ __forceinline__ TreeRun args_now() {
    typedef const __attribute__((address_space(4))) uint32_t* words_ptr;
    words_ptr p = (words_ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    struct Words { uint32_t w[sizeof(TreeRun) / 4]; } x;
    static_assert(sizeof(TreeRun) % 4 == 0, "read word by word");
#pragma unroll
    for (size_t i = 0; i < sizeof(TreeRun) / 4; ++i) x.w[i] = p[i];
    return __builtin_bit_cast(TreeRun, x);
}

// ---- the share of a workgroup ------------------------------------------------------------------

// A value that is the same in every lane, in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x) {
    return (long long)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// lanes_up_to() of numbers that are small as a rule
__device__ __forceinline__ long long lanes_up_to(long long x) {
    if (__builtin_amdgcn_ballot_w64((x >> 24) != 0) == 0) return lanes_up_to((int)x);      // the sum has 30 bits
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const long long y = __shfl_up(x, k);
        if (lane >= k) x += y;
    }
    return x;
}

// a / b of whole numbers, 0 <= a < 2^52 and b > 0, by a division of doubles (one of 64-bit integers takes ten times the
// instructions).  The quotient is rounded, so that its floor can be one too large.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    const long long q = (long long)((double)a / (double)b);
    return q * b > a ? q - 1 : q;
}

// sum over i < n of floor((a i + b) / m), for a, b >= 0 and m > 0.  Whole multiples of m in a and b are counted directly.
// What is left counts points under a line with slope below 1; seen from the other axis, of its k = floor((a (n - 1) + b) / m)
// rows row j = 1..k lacks the first ceil((j m - b) / a) of n points: a sum of the same form with a in m's place.
__device__ __forceinline__ long long sum_of_floors(long long n, long long a, long long b, long long m) {
    long long sum = 0, sign = 1;
    while (n > 0) {
        if (a >= m) {
            const long long q = quotient(a, m);
            sum += sign * q * ((n * (n - 1)) >> 1);
            a -= q * m;
        }
        if (b >= m) {
            const long long q = quotient(b, m);
            sum += sign * q * n;
            b -= q * m;
        }
        const long long k = quotient(a * (n - 1) + b, m);
        if (k == 0) break;
        sum += sign * n * k;
        sign = -sign;
        b = m - b + a - 1;
        const long long slope = a;
        a = m;
        m = slope;
        n = k;
    }
    return sum;
}

struct WalkScratch {
    long long wave_sum[kTreeWaves];
    long long found_before, found_head;
    Seq found_seq;
    int found_b;
};

// A workgroup's way along the row of blocks, and the piece of a unit that it is at (all the same in every
// thread, in scalar registers).  M: rows of a tile; KB: keys of a block of the row.  Of a chain's row tile only the blocks count
// that its last token sees.  A unit begins with START places without a block, for the time that its first keys and its
// queries take to arrive: a workgroup with more units gets fewer blocks.  GRID: workgroups of the launch, LEAD: by how many
// 64ths the share of a compute unit's first workgroup is above the mean, and that of its last below it.
// LATE: a share that begins inside a unit takes that piece last, so that workgroups of one head, whose other units begin at
// their first key, meet the same keys at the same time.
template <int M, int KB, int GRID, int START, int LEAD, bool LATE>
struct Walk {
    static constexpr int kSlots = GRID / 256;       // workgroups of a compute unit
    static constexpr int kOfXcd = GRID / 8;         // workgroups of an XCD, 32 of each slot
    long long at, end;      // places of the long row
    long long per, lead;    // places of a workgroup, and what first and last slots have more and less
    int w;                  // the workgroup's place along the row
    int b, h, tile;         // present unit
    Seq s;
    int tiles;              // row tiles of the sequence
    int blocks;             // blocks of the unit
    int from;               // the place in the unit at which the piece begins
    int blk0, blk1;         // the piece
    int first, nrows;       // its first row (token, head of the group), and rows
    bool later = false;     // the share's first piece is still to be done: its place
    long long later_at;
    int later_b, later_h, later_tile, later_from;

    // Places of a share where there are few in all, 0 where there are not: a share of fewer ends sooner, but leaves more parts to be
    // joined.  Tile kernel (12 rows after 1000 keys, 48 after 4000, 64 each of 4 sequences; all with the merge): 15.8, 24.7, 26.1 us with 1,
    // 18.5, 22.0, 26.2 with 2, 19.7, 21.4, 23.8 with 4.  Kernels whose wavefronts share out the blocks (one sequence of 1000
    // keys, one of 4000, 8 of 100 to 1000): 13.8, 16.7, 19.4 us with 4, 14.1, 17.6, 18.2 with 8.
    static __device__ __forceinline__ int few_places(long long total) {
        if (KB == kBC) return total <= GRID / 2 ? 1 : total <= GRID ? 2 : total <= 4 * GRID ? 4 : 0;
        return total <= 2 * GRID ? kTreeWaves : total <= 2 * kTreeWaves * GRID ? 2 * kTreeWaves : 0;
    }

    // Along the row come, XCD by XCD, the 32 workgroups of each slot.
    __device__ __forceinline__ long long size(int slot) const {
        return slot == 0 ? per + lead : slot == kSlots - 1 ? per - lead : per;
    }
    __device__ __forceinline__ long long begin_of(int slot) const { return slot == 0 ? 0 : 32 * (slot * per + lead); }
    __device__ __forceinline__ int holder(long long place) const {
        const long long x = quotient(place, kOfXcd * per), r = place - x * (kOfXcd * per);
        int slot = 0;
#pragma unroll
        for (int j = 1; j < kSlots; ++j) slot = r >= begin_of(j) ? j : slot;
        return (int)x * kOfXcd + 32 * slot + (int)quotient(r - begin_of(slot), size(slot));
    }

    __device__ __forceinline__ bool whole() const { return blk0 == 0 && blk1 == blocks; }
    __device__ __forceinline__ int keys() const { return s.len + s.n; }

    __device__ __forceinline__ int blocks_of(const TreeRun& r, int t) const {
        int keys = s.len + s.n;
        if (r.a.tree == nullptr) {
            const long long end = (long long)(t + 1) * M;       // rows up to the tile's last
            const int token = end < (long long)s.n * (int)r.group.d ? (int)fast_div((uint32_t)(end - 1), r.group) : s.n - 1;
            keys = s.len + token + 1;
        }
        return (keys + KB - 1) / KB;
    }
    // Sequence `seq`.  SAME: it is the same one in every thread.
    template <bool SAME>
    __device__ __forceinline__ void enter(const TreeRun& r, int seq) {
        b = seq;
        s = seq_at(r.c, b);
        if constexpr (SAME) s = Seq{uniform(s.row0), uniform(s.n), uniform(s.len)};
        tiles = (int)(((long long)s.n * (int)r.group.d + M - 1) / M);
    }
    __device__ __forceinline__ void set_seq(const TreeRun& r, const Seq& x) {       // one that was entered before
        s = Seq{uniform(x.row0), uniform(x.n), uniform(x.len)};
        tiles = (int)(((long long)s.n * (int)r.group.d + M - 1) / M);
    }
    // Places of one kv head's units.  (A chain's tile t < tiles - 1 has ceil((len + ceil((t + 1) M / G)) / KB) blocks,
    // which is ceil((len G + (t + 1) M) / (G KB)).)
    __device__ __forceinline__ long long places(const TreeRun& r) const {
        if (tiles == 0) return 0;
        const long long last = blocks_of(r, tiles - 1) + START;
        if (r.a.tree != nullptr) return tiles * last;
        const long long G = (int)r.group.d, m = G * KB;
        return last + (long long)(tiles - 1) * START + sum_of_floors(tiles - 1, M, s.len * G + M + m - 1, m);
    }
    __device__ __forceinline__ void set_unit(const TreeRun& r) {
        blocks = blocks_of(r, tile);
        first = tile * M;
        nrows = min(M, s.n * (int)r.group.d - first);
    }
    __device__ __forceinline__ void set_piece(int place) {
        const long long left = end - at;
        from = place;
        const int to = left < START + blocks - from ? from + (int)left : START + blocks;
        blk0 = max(from - START, 0);
        blk1 = max(to - START, 0);
    }

    // Every thread of the workgroup takes a run of sequences, whose places are then summed over the threads;
    // the one that has the share's first place in its run finds the sequence.  False: no share.
    __device__ __forceinline__ bool begin(const TreeRun& r, WalkScratch* scratch) {
        long long (&wave_sum)[kTreeWaves] = scratch->wave_sum;
        long long& found_before = scratch->found_before;
        int& found_b = scratch->found_b;
        const Paged& c = r.c;
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int each = (c.B + kTreeWaves * kWave - 1) / (kTreeWaves * kWave);
        const int b0 = tid * each, b1 = min(b0 + each, c.B);
        long long mine = 0, own = 0;             // of the run, and of one kv head of its last sequence
        Walk any;
        for (int i = b0; i < b1; ++i) {
            any.template enter<false>(r, i);
            own = any.places(r);
            mine += own * c.Hkv;
        }
        const long long in = lanes_up_to(mine);
        if (lane == 63) wave_sum[wave] = in;
        if (tid == 0) found_b = -1;
        __syncthreads();
        long long before = in - mine, total = 0;
#pragma unroll
        for (int k = 0; k < kTreeWaves; ++k) {
            before += k < wave ? wave_sum[k] : 0;
            total += wave_sum[k];
        }
        total = uniform(total);
        // all workgroups, or fewer with some places each
        const int least = few_places(total);
        const bool few = least > 0;
        per = few ? least : (GRID & (GRID - 1)) == 0 ? (total + GRID - 1) / GRID : quotient(total + GRID - 1, GRID);
        lead = few ? 0 : (per * LEAD) >> 6;
        // Workgroup ids go round-robin over the 8 XCDs; neighbours along the row, which may read the same
        // keys, go to one.  An XCD's first 32 go to a compute unit each, the next 32 beside them, and so on.
        const int of_xcd = few ? ((int)(total + least - 1) / least + 7) >> 3 : kOfXcd;
        const int k = (int)blockIdx.x >> 3;
        w = ((int)blockIdx.x & 7) * of_xcd + k;
        const int place = w % kOfXcd;
        at = w / kOfXcd * (kOfXcd * per) + begin_of(place >> 5) + (place & 31) * size(place >> 5);
        end = at + size(place >> 5);
        if (k >= of_xcd || at > total) at = total;
        if (end > total) end = total;
        if (tid == 0) r.splits[blockIdx.x].parts = 0;
        if (at < end && at >= before && at < before + mine) {
            int i = b0;
            if (each > 1) {                      // (a run of one sequence: `own` is its places)
                for (;; ++i) {
                    any.template enter<false>(r, i);
                    own = any.places(r);
                    if (at < before + own * c.Hkv) break;
                    before += own * c.Hkv;
                }
            }
            found_b = i;
            found_before = before;
            scratch->found_head = own;
            scratch->found_seq = any.s;
        }
        __syncthreads();
        const int found = uniform(found_b);
        const long long in_b = at - uniform(found_before), head = uniform(scratch->found_head);
        const Seq found_seq = scratch->found_seq;
        __syncthreads();                                 // the scratch is the kernel's again
        if (found < 0) return false;
        b = found;
        set_seq(r, found_seq);
        h = uniform((int)quotient(in_b, head));
        long long rest = in_b - h * head;
        tile = 0;
        if (tiles > 1 && r.a.tree != nullptr) {
            const int each_tile = blocks_of(r, 0) + START;
            tile = uniform((int)quotient(rest, each_tile));
            rest -= (long long)tile * each_tile;
        } else if (tiles > 1) {
            // every wavefront by itself, 64 tiles at a time
            for (int t0 = 0;; t0 += kWave) {
                const int its = t0 + lane < tiles ? blocks_of(r, t0 + lane) + START : 0;
                const long long sum = lanes_up_to((long long)its);
                const uint64_t beyond = __builtin_amdgcn_ballot_w64(sum > rest);
                const int hit = beyond != 0 ? __builtin_ctzll(beyond) : kWave - 1;
                const long long upto = uniform(__shfl(sum, hit));
                if (beyond != 0) {
                    tile = t0 + hit;
                    rest -= upto - __builtin_amdgcn_readlane(its, hit);
                    break;
                }
                rest -= upto;
            }
        }
        set_unit(r);
        set_piece(uniform((int)rest));
        if constexpr (LATE) {
            if (blk0 > 0 && end - at > START + blocks - from) {
                later_at = at;
                later_b = b;
                later_h = h;
                later_tile = tile;
                later_from = from;
                later = true;
                return next(r);
            }
        }
        return blk0 < blk1 || next(r);
    }
    // On to the next piece with keys; false at the end of the share.
    __device__ __forceinline__ bool next(const TreeRun& r) {
        if (advance(r)) return true;
        if (!LATE || !later) return false;
        later = false;
        at = later_at;
        enter<true>(r, later_b);
        h = later_h;
        tile = later_tile;
        set_unit(r);
        end = at + START + blocks - later_from;
        set_piece(later_from);
        return true;
    }
    __device__ __forceinline__ bool advance(const TreeRun& r) {
        int place = from;
        do {
            at += min((long long)START + blocks - place, end - at);
            if (at >= end) return false;
            if (++tile == tiles) {
                tile = 0;
                if (++h == r.c.Hkv) {
                    h = 0;
                    do {
                        if (b + 1 >= r.c.B) return false;
                        enter<true>(r, b + 1);
                    } while (tiles == 0);
                }
            }
            set_unit(r);
            set_piece(place = 0);
        } while (blk0 == blk1);
        return true;
    }
    __device__ __forceinline__ int slot() const { return 2 * w + (blk0 == 0 ? 1 : 0); }
    __device__ __forceinline__ void note_split(const TreeRun& r) const {
        TreeSplit sp;
        sp.row0 = s.row0;
        sp.h = h;
        sp.first = first;
        sp.rows = nrows;
        sp.parts = holder(at + START + blocks - from - 1) - w + 1;
        sp.w = w;
        r.splits[blockIdx.x] = sp;
    }
};

// Element offset of row `rw` (token, head of the group) of the piece's sequence in q or o
template <class W>
__device__ __forceinline__ size_t row_at(const TreeRun& r, const W& u, int rw, int64_t stride, int d) {
    const int token = (int)fast_div((uint32_t)rw, r.group);
    return (size_t)(u.s.row0 + token) * stride + (size_t)(u.h * (int)r.group.d + rw - token * (int)r.group.d) * d;
}

// Whether the sum of the unrounded weights is carried
template <typename T, bool LSE> constexpr bool kTrueSum = LSE && std::is_same_v<T, BF16>;

// f32's weights: see tree_rows_f32_kernel.
constexpr float kF32Move = 8.0f, kF32Unit = 0x1p-40f, kF32UnitLog2 = -40.0f;

// The log-sum-exp of a row whose weights against `top` (log2 units) sum to lt; -infinity without a key
template <typename T>
__device__ __forceinline__ float lse_of(float top, float lt) {
    if (lt == 0.0f) return -__builtin_inff();
    return (top + (log2_fast(lt) - (std::is_same_v<T, F32> ? kF32UnitLog2 : 0.0f))) * kLn2;
}

// A finished row's four columns from t on: the output, or the unit's partial state.
template <typename T, int D, int M, bool LSE, class W>
__device__ __forceinline__ void put_row(const TreeRun& r, const W& u, int fr, int t, f32x4 o, float top, float lt,
                                        float vscale, float tr) {
    if (u.whole()) {
        if (lt != 0.0f) o *= vscale / lt;
        if (LSE && t == 0) r.a.lse[row_at(r, u, u.first + fr, r.a.Hq, 1)] = lse_of<T>(top, kTrueSum<T, LSE> ? tr : lt);
        Store<T>::store4(r.a.o, row_at(r, u, u.first + fr, r.a.o_stride, D) + t, {o[0], o[1], o[2], o[3]});
    } else {
        const size_t at = (size_t)u.slot() * M + fr;
        *reinterpret_cast<f32x4*>(r.parts + at * D + t) = o;
        if (t == 0) r.stats[at] = float2{top, lt};
        if (kTrueSum<T, LSE> && t == 0) r.sums[at] = tr;
    }
}

// The bits of the 32 keys from j0 on that the token `i` (row `t` of the packed tensors) sees.
__device__ __forceinline__ uint32_t seen_bits(const TreeArgs& a, const Seq& s, int i, int t, int j0) {
    const int rel = j0 - s.len;                 // the block's first key among the new ones
    if (rel + kTreeBlock <= 0) return ~0u;
    uint32_t m;
    if (a.tree == nullptr) {
        const int n = i + 1 - rel;              // keys up to the token itself
        m = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
    } else {
        const uint32_t* w = a.tree + (size_t)t * a.words;
        if (rel < 0) {
            m = (w[0] << -rel) | ((1u << -rel) - 1u);       // 0 < -rel < 32
        } else {
            const int k = rel >> 5, sh = rel & 31;
            const uint32_t lo = k < a.words ? w[k] : 0u, hi = k + 1 < a.words ? w[k + 1] : 0u;
            m = sh == 0 ? lo : (lo >> sh) | (hi << (32 - sh));
        }
    }
    const int left = s.n - rel;                 // new keys from here on
    if (left < 32) m &= left <= 0 ? 0u : (1u << left) - 1u;
    return m;
}

// Reductions over the four lanes c, c + 16, c + 32, c + 48 of a query row
__device__ __forceinline__ float quad_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(a[0]) + __uint_as_float(a[1]));
}

// ---- what every kernel does with its states -------------------------------------------------------

// A row's state in a wavefront: o = U / l, U against the reference R (log2 units); R = -inf and l = 0
// without a key.  The lane's part of U is columns 16 i + 4 q .. + 3 of row col.
//
// A block's scores, in log2 units and -inf where the row does not see the key: moves the reference
// where the top one lies more than `limit` above it and turns the scores into weights, a power of two (`unit`) at the reference.
template <bool TR, int NDB>
__device__ __forceinline__ void weigh(float (&x)[8], f32x8& p, f32x4 (&U)[NDB], float& R, float& l, float& tr, float limit, float unit = 1.0f) {
    const float ninf = -__builtin_inff();
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
    top = quad_max(top);
    if (__builtin_amdgcn_ballot_w64(top > R + limit) != 0) {
        const bool move = top > R + limit;
        const float f = move ? exp2_fast(R - top) : 1.0f;       // 0 for a row without keys
        R = move ? top : R;
        l *= f;
        if (TR) tr *= f;
#pragma unroll
        for (int i = 0; i < NDB; ++i) U[i] *= f;
    }
    const float ref = R == ninf ? 0.0f : R;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = exp2_fast(x[e] - ref) * unit;
    if (TR) tr += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
}

// Joins the four wavefronts' states of a piece whose keys they have shared out: row tiles of 16 NR rows.
// BY16: U[i] of lane (q, col) is columns 16 i + 4 q .. + 3, else 64 (i / 4) + 16 q + 4 (i % 4) .. + 3.
template <typename T, int D, int NR, bool BY16, bool LSE, class Wk>
__device__ __forceinline__ void finish_rows(const TreeRun& r, const Wk& u, const f32x4 (&U)[NR][D / 16],
                                            const float (&R)[NR], const float (&l)[NR], const float (&tr)[NR], float* fold, float vscale) {
    constexpr int W = kTreeWaves, FROW = D + 4, NDB = D / 16;
    constexpr bool TR = kTrueSum<T, LSE>;
    __shared__ float fold_r[W][16], fold_l[W][16], fold_t[TR ? W : 1][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, q = lane >> 4;
#pragma unroll
    for (int k = 0; k < NR; ++k) {
        const float lk = quad_sum(l[k]), tk = TR ? quad_sum(tr[k]) : 0.0f;
        __syncthreads();                                 // stages are dead, `fold` is their memory
#pragma unroll
        for (int i = 0; i < NDB; ++i)
            *reinterpret_cast<f32x4*>(&fold[(wave * 16 + col) * FROW + (BY16 ? 16 * i + 4 * q : 64 * (i >> 2) + 16 * q + 4 * (i & 3))]) =
                U[k][i];
        if (q == 0) {
            fold_r[wave][col] = R[k];
            fold_l[wave][col] = lk;
            if (TR) fold_t[TR ? wave : 0][col] = tk;
        }
        __syncthreads();
        for (int idx = tid; idx < min(u.nrows - 16 * k, 16) * (D / 4); idx += W * kWave) {
            const int fr = idx / (D / 4);
            const int t = 4 * (idx % (D / 4));
            float top = fold_r[0][fr];
#pragma unroll
            for (int w = 1; w < W; ++w) top = fmaxf(top, fold_r[w][fr]);
            float lt = 0.0f, tt = 0.0f;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                // a wavefront without a key of the row is left out (its U may hold 0 * infinity)
                const bool none = fold_l[w][fr] == 0.0f;
                const float f = none ? 0.0f : exp2_fast(fold_r[w][fr] - top);
                const f32x4 x = *reinterpret_cast<const f32x4*>(&fold[(w * 16 + fr) * FROW + t]);
                lt = fmaf(f, fold_l[w][fr], lt);
                if (TR) tt = fmaf(f, fold_t[TR ? w : 0][fr], tt);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(f, none ? 0.0f : x[e], o[e]);
            }
            put_row<T, D, 16 * NR, LSE>(r, u, 16 * k + fr, t, o, top, lt, vscale, tt);
        }
    }
    if (u.blk0 == 0 && !u.whole() && tid == 0) u.note_split(r);
    __syncthreads();
}

// A run of bytes behind which reads give zeros: the words of a buffer descriptor.
struct Window {
    u32x4 words;
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc() const {
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)words[1] << 32 | words[0]), 0,
                                                 (int)words[2], (int)words[3]);
    }
};

__device__ __forceinline__ Window make_window(uint64_t at, int bytes) {
    return Window{u32x4{(uint32_t)uniform((int)at), (uint32_t)uniform((int)(at >> 32)), (uint32_t)uniform(bytes), 0x00020000u}};
}

// ---- 16 rows, keys shared out over the wavefronts (f16 / bf16) -----------------------------------
//
// Wavefront w of a workgroup takes blocks w, w + 4, ... of the piece with a state of its own.
// Lane (q, c) = (lane / 16, lane % 16): S^T = K Q^T comes as two 16-key tiles of which the lane holds, for
// query row c, the keys 4 q + r and 16 + 4 q + r.  Rounded and packed, these are the eight B
// elements of the lane for O^T = V^T P^T; V^T comes from the transposing LDS read in the same key
// order.  A 16-key half of a block never crosses a page (pages have 16 keys or more), so each half
// has a base address of its own, through a buffer descriptor that ends at the sequence's last key:
// keys behind it, and pages that are none, read zeros.
//
// HBM bounds it: a token for each of 64 sequences of 500 to 8192 keys, 32 / 8 heads of 128, takes 189 us for 1.17 GB read once, 6.2 TB/s
// (median of calls one after the other; the least of 12 took 182); from fp8, four tokens each, 110 us (104) for 586 MB, 5.3 TB/s, a
// wavefront waiting for memory or for its turn three quarters of its time.  One sequence of 1000 keys takes 6.5 us, the latency of
// finding a share, its pages and its keys.
//
// In blocks with new keys a weight of zero may meet a value that is infinite or NaN (a token that some rows see
// and others do not), and 0 * infinity must not reach the others: see codes_of().

// (All of this on pairs of halves, by carries into their top bits: comparisons hand their results to scalar registers, and the
// dozens of a block's values in flight took those that the loops around hold their addresses in.)
template <typename T> struct Half {
    static constexpr bool B = Mma<T>::kRoundedSum;                          // bf16, else f16
    static constexpr uint32_t kExp = B ? 0x7f807f80u : 0x7c007c00u, kOne = B ? 0x00800080u : 0x04000400u;
    static constexpr uint32_t kMan = B ? 0x007f007fu : 0x03ff03ffu, kTop = 0x80008000u;
    static constexpr uint32_t kPlus = B ? 0x3f803f80u : 0x3c003c00u, kMinus = B ? 0x43004300u : 0x58005800u,
                              kNan = B ? 0x46804680u : 0x74007400u;         // 1, 128 and 16384
    // top bits of the halves that are infinite or NaN
    static __device__ __forceinline__ uint32_t bad(uint32_t x) { return ((x & kExp) + kOne) & kTop; }
    // top bits -> whole halves
    static __device__ __forceinline__ uint32_t spread(uint32_t top) { return (top >> 15) * 0xffffu; }
};
// all ones if bit i of x is set
__device__ __forceinline__ uint32_t bit_mask(uint32_t x, int i) { return (uint32_t)((int)(x << (31 - i)) >> 31); }

// nonzero if any of 8 values of the storage type (16 fp8 values) is infinite or NaN
template <typename T, bool FP8>
__device__ __forceinline__ uint32_t not_finite(u32x4 x) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)          // fp8: NaN is 0x7f, the only byte that adding 1 carries from
        bad |= FP8 ? ((x[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : Half<T>::bad(x[i]);
    return bad;
}

// The products of such a block: the values that are no numbers are left out of the product with the weights
// (numbers_of) and counted by one with the bits of what is seen, +infinities as 1, -infinities as 128, NaN as
// 16384 (codes_of; of at most 64 keys, so the sum is exact and keeps them apart); what_is_seen() says what a count adds to an output.
template <typename T>
__device__ __forceinline__ u32x4 numbers_of(u32x4 x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] &= ~Half<T>::spread(Half<T>::bad(x[i]));
    return x;
}
template <typename T>
__device__ __forceinline__ u32x4 codes_of(u32x4 x) {
    using H = Half<T>;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t bad = H::bad(x[i]), nan = bad & ((x[i] & H::kMan) + 0x7fff7fffu), inf = bad & ~nan;
        x[i] = (H::spread(nan) & H::kNan) | (H::spread(inf & x[i]) & H::kMinus) | (H::spread(inf & ~x[i]) & H::kPlus);
    }
    return x;
}
__device__ __forceinline__ float what_is_seen(float count) {
    const int n = (int)count;
    const float inf = __builtin_inff();
    const bool plus = (n & 127) != 0, minus = (n >> 7 & 127) != 0;
    return n >= 16384 || (plus && minus) ? __builtin_nanf("") : plus ? inf : minus ? -inf : 0.0f;
}
// 8 bits, lowest first, as ones and zeros of the storage type
template <typename T>
__device__ __forceinline__ u32x4 ones_of(uint32_t bits) {
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] = (bit_mask(bits, 2 * i) & (Mma<T>::kOnes & 0xffffu)) | (bit_mask(bits, 2 * i + 1) & (Mma<T>::kOnes & 0xffff0000u));
    return x;
}
// x if bit i of bits is set, else -inf
__device__ __forceinline__ float if_seen(uint32_t bits, int i, float x) {
    const uint32_t m = bit_mask(bits, i);
    return __uint_as_float((m & __float_as_uint(x)) | (~m & 0xff800000u));
}

// The lane's number, formed anew: what depends on it is then formed where it is used.  Kept over the loop those addresses were
// spilled, and the wait for one to come back is one for every copy under way.
__device__ __forceinline__ int lane_now() {
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
}

// Workgroups per compute unit: what one has under way is its wavefronts' next block of K and of V.  Of fp8, or at
// d = 64, that is half as much, and three workgroups' registers fit.
constexpr int rows_per_cu(int D, bool FP8, int NR) { return (D == 64 || FP8) && NR == 1 ? 3 : 2; }

template <typename T, int D, bool FP8, int NR, bool LSE>
__global__ __launch_bounds__(kTreeWaves * kWave, rows_per_cu(D, FP8, NR)) void tree_rows_kernel(TreeRun r) {
    constexpr int W = kTreeWaves;
    constexpr int NKK = D / 32;
    constexpr int NDB = D / 16;
    constexpr int ESZ = FP8 ? 1 : 2;
    constexpr int NV = kTreeBlock * D * ESZ / 1024;      // 16-byte loads of K or V per lane and block
    constexpr int CPR = D * ESZ / 16;                    // 16-byte chunks per key row
    constexpr int KROW = D + 8;
    constexpr int VROW = D + 16;
    constexpr int STAGE = kTreeBlock * VROW;
    // fp8: a lane writes 32 bytes, in two pieces.  In the second half of a row of 256 bytes pieces 2 i and 2 i + 1 change
    // places, so that the first pieces of a row's 8 lanes fall on all banks, and the addresses are formed where they are used.
    // With 32 rows that took 147 us to 138 (24 rows, 64 sequences of 500 to 8192 keys); with 16, where 44 % of the time that LDS is busy
    // goes to such conflicts, it made 111 us 114.
    constexpr bool SWAP = FP8 && D == 128 && NR == 2;
    constexpr int FROW = D + 4;
    constexpr int kLds = 2 * W * STAGE > 4 * W * 16 * FROW ? 2 * W * STAGE : 4 * W * 16 * FROW;
    __shared__ __align__(16) char lds[kLds];

    (void)r;                                             // read through args_now()
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;
    const int q = lane >> 4;
    const float ninf = -__builtin_inff();
    uint16_t* vs = reinterpret_cast<uint16_t*>(lds) + wave * STAGE;

    Walk<16 * NR, kTreeBlock, 256 * rows_per_cu(D, FP8, NR), kRowsStart, kRowsLead, false> u;
    if (!u.begin(args_now(), reinterpret_cast<WalkScratch*>(lds))) return;
    do {
        // the query rows of this lane's column; columns past the last row stand in for it
        const TreeRun now_r = args_now();
        u32x4 qf[NR][NKK];
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            const int row = u.first + min(16 * k + col, u.nrows - 1);
            const uint16_t* qg = static_cast<const uint16_t*>(now_r.a.q) + row_at(now_r, u, row, now_r.a.q_stride, D);
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) qf[k][kk] = *reinterpret_cast<const u32x4*>(qg + 32 * kk + 8 * q);
        }
        __builtin_amdgcn_sched_barrier(0);
        const float c_log2 = (FP8 ? now_r.a.scale * now_r.c.kscale : now_r.a.scale) * kLog2e;

        // What the loop needs of the arguments, each in a register of its own (see tree_tile_kernel).
        constexpr int ROWB = D * ESZ;
        const char* kpool = now_r.c.k + u.h * now_r.c.head_bytes;
        const char* vpool = now_r.c.v + u.h * now_r.c.head_bytes;
        int64_t page_bytes = now_r.c.page_bytes;
        int page_log2 = now_r.c.page_log2, pool_pages = now_r.c.P, last_key = u.keys(), blk_end = u.blk1, len = u.s.len;
        typedef const __attribute__((address_space(4))) int* table_ptr;
        table_ptr trow = (table_ptr)(uintptr_t)(now_r.c.table + (size_t)u.b * now_r.c.max_pages);
        asm volatile("" : "+s"(kpool), "+s"(vpool), "+s"(page_bytes), "+s"(page_log2), "+s"(pool_pages), "+s"(last_key),
                          "+s"(blk_end), "+s"(len), "+s"(trow));
        // page of a half of a block, by a scalar load; -1 behind the piece and behind the last key
        auto page_of = [&](int blk, int half) __attribute__((always_inline)) {
            const int key = blk * kTreeBlock + 16 * half;
            const int p = blk < blk_end && key < last_key ? trow[key >> page_log2] : -1;
            return (unsigned)p < (unsigned)pool_pages ? p : -1;
        };
        // (Always issued, with an empty window where there is nothing to fetch: with a branch around it the compiler could
        // not count the loads under way, and waited for the next block's K before it used this one's V.)
        auto fetch = [&](const char* pool, u32x4 (&reg)[NV], int blk, int p0, int p1) __attribute__((always_inline)) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int p = half ? p1 : p0, key = blk * kTreeBlock + 16 * half;
                const uint64_t at = (uint64_t)(pool + max(p, 0) * page_bytes + (key & ((1 << page_log2) - 1)) * ROWB);
                const int left = last_key - key, keys = p < 0 || left < 0 ? 0 : left < 16 ? left : 16;
                const auto w = make_window(at, keys * ROWB).rsrc();
#pragma unroll
                for (int n = 0; n < NV / 2; ++n) reg[half * (NV / 2) + n] = kv_load<2>(w, 1024 * n + 16 * lane);
            }
        };
        auto stage = [&](const u32x4 (&reg)[NV], int ROW) __attribute__((always_inline)) {
            const int x0 = SWAP ? lane_now() : lane;
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const int ch = n * kWave + x0;
                uint16_t* dst = &vs[(ch / CPR) * ROW + (FP8 ? 16 : 8) * (ch % CPR)];
                if constexpr (FP8) {
                    const int x = SWAP ? 8 * (ch % CPR >> 2) : 0;
                    *reinterpret_cast<u32x4*>(dst + x) = widen8<T>(reg[n][0], reg[n][1]);
                    *reinterpret_cast<u32x4*>(dst + (8 ^ x)) = widen8<T>(reg[n][2], reg[n][3]);
                } else {
                    *reinterpret_cast<u32x4*>(dst) = reg[n];
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        };
        auto stage_done = [&]() __attribute__((always_inline)) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };

        f32x4 U[NR][NDB];
        float R[NR], l[NR], tr[NR];
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            R[k] = ninf;
            l[k] = 0.0f;
            tr[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < NDB; ++i) U[k][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        u32x4 kreg[NV], vreg[NV];
        int blk = u.blk0 + wave;
        int p0 = page_of(blk, 0), p1 = page_of(blk, 1), n0 = page_of(blk + W, 0), n1 = page_of(blk + W, 1);
        // K before V, as in the loop: mixed, the wait for K would be one for V
        __builtin_amdgcn_sched_barrier(0);
        fetch(kpool, kreg, blk, p0, p1);
        __builtin_amdgcn_sched_barrier(0);
        fetch(vpool, vreg, blk, p0, p1);
        __builtin_amdgcn_sched_barrier(0);
        // The queries are here before the loop, as the compiler knows: in every turn of it, it would else wait for them,
        // and so for the keys under way.
        wait_loads<2 * NV>();
        for (; blk < blk_end; blk += W) {
            const int j0 = blk * kTreeBlock;
            // a half without a page, or behind the last key, has no keys
            const uint32_t have = (p0 < 0 ? 0u : 0x0000ffffu) | (p1 < 0 ? 0u : 0xffff0000u);
            const int m0 = page_of(blk + 2 * W, 0), m1 = page_of(blk + 2 * W, 1);
            stage(kreg, KROW);
            fetch(kpool, kreg, blk + W, n0, n1);
            const int z = SWAP ? lane_now() : lane, kcol = (z & 15) * KROW;
            const uint16_t* const krow[2] = {&vs[kcol + 8 * (z >> 4)], &vs[kcol + 8 * (z >> 4 ^ (SWAP ? 1 : 0))]};
            f32x4 acc[NR][2];
#pragma unroll
            for (int k = 0; k < NR; ++k)
#pragma unroll
                for (int t = 0; t < 2; ++t) acc[k][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(&krow[kk >> 1][16 * t * KROW + 32 * kk]);
#pragma unroll
                    for (int k = 0; k < NR; ++k) acc[k][t] = Mma16<T>::mfma(x, qf[k][kk], acc[k][t]);
                }
            stage_done();
            stage(vreg, VROW);
            const bool masked = have != ~0u || j0 + kTreeBlock > len;
            bool apart = false;
            if (masked) {
                uint32_t bad = 0;
#pragma unroll
                for (int n = 0; n < NV; ++n) bad |= not_finite<T, FP8>(vreg[n]);
                apart = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
            }
            fetch(vpool, vreg, blk + W, n0, n1);

            u32x4 bfrag[NR];
            uint32_t bits[NR];
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                bits[k] = ~0u;
                if (masked) {
                    const TreeRun m = args_now();
                    const int token = (int)fast_div((uint32_t)(u.first + min(16 * k + col, u.nrows - 1)), m.group);
                    bits[k] = have & seen_bits(m.a, u.s, token, u.s.row0 + token, j0);
                }
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = acc[k][e >> 2][e & 3] * c_log2;
                    if (masked) x[e] = if_seen(bits[k] >> (4 * q), 16 * (e >> 2) + (e & 3), x[e]);
                }
                f32x8 pv;
                weigh<kTrueSum<T, LSE>>(x, pv, U[k], R[k], l[k], tr[k], LazyLimit<T>::kMoveLog2);
                bfrag[k] = Mma<T>::pack8(pv);
                f32x4 ps = {0.0f, 0.0f, 0.0f, 0.0f};
                Mma<T>::sum8(pv, bfrag[k], ps);
                l[k] += (ps[0] + ps[1]) + (ps[2] + ps[3]);
            }
            const int y = SWAP ? lane_now() : lane, vrow = (4 * (y >> 4) + (y >> 2 & 3)) * VROW;
            const uint16_t* const bases[2] = {&vs[vrow + 4 * (y & 3)], &vs[vrow + (4 * (y & 3) ^ 8)]};
            typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
            auto v_operand = [&](int i) __attribute__((always_inline)) {
                const uint16_t* base = bases[SWAP && i >= 4 ? 1 : 0];
                const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_ptr)(base + 16 * i)));
                const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_ptr)(base + 16 * VROW + 16 * i)));
                return u32x4{lo[0], lo[1], hi[0], hi[1]};
            };
            if (apart) {
#pragma unroll
                for (int i = 0; i < NDB; ++i) {
                    const u32x4 codes = codes_of<T>(v_operand(i));
#pragma unroll
                    for (int k = 0; k < NR; ++k) {
                        const uint32_t mine = (bits[k] >> (4 * q) & 15u) | (bits[k] >> (16 + 4 * q) & 15u) << 4;
                        const f32x4 n = Mma16<T>::mfma(codes, ones_of<T>(mine), f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                        for (int d = 0; d < 4; ++d) U[k][i][d] += what_is_seen(n[d]);
                    }
                    __builtin_amdgcn_sched_barrier(0);           // few registers at a time
                }
                stage_done();
#pragma unroll 1
                for (int n = 0; n < D / 16; ++n) {
                    u32x4* x = reinterpret_cast<u32x4*>(&vs[(n * kWave + lane) / (D / 8) * VROW + 8 * (lane % (D / 8))]);
                    *x = numbers_of<T>(*x);
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            }
#pragma unroll
            for (int i = 0; i < NDB; ++i) {
                const u32x4 v = v_operand(i);
#pragma unroll
                for (int k = 0; k < NR; ++k) U[k][i] = Mma16<T>::mfma(v, bfrag[k], U[k][i]);
            }
            stage_done();
            p0 = n0;
            p1 = n1;
            n0 = m0;
            n1 = m1;
        }
        const TreeRun end_r = args_now();
        finish_rows<T, D, NR, true, LSE>(end_r, u, U, R, l, tr, reinterpret_cast<float*>(lds), FP8 ? end_r.c.vscale : 1.0f);
    } while (u.next(args_now()));
}

// ---- 64 or 128 rows: the wavefronts read the keys together (f16 / bf16) -----------------------------
//
// With more rows the products outweigh the keys' way through LDS, so the four wavefronts share tiles of 64 keys, in the
// layout of flashd_tile_parts.h, and the 32 x 32 x 16 products: wavefront w has rows 32 (w % RW) .. + 31 of the tile and
// every KW-th 32-key block (RW KW = 4; two wavefronts to a row's keys for up to 64 rows, none share for 128).  Each wavefront brings the 16 keys of a tile that it would
// in that layout: they lie in one page, so its copies have one scalar base.
//
// Up to 64 rows HBM bounds it: trees of 16 tokens after 500 to 8192 keys (32 sequences, 32 / 8 heads of 128) take 113 us for
// 600 MB, 5.3 TB/s (median of calls one after the other; the least of 12 took 103), one of 12 after 131000 keys 97 us (90), 5.5 TB/s; the
// start of a piece, when nothing of it has arrived, and the unequal pace of the workgroups are the rest.  With 128 rows it is the instructions:
// chunks of 573 to 1000 tokens after 3180 to 7000 keys are 277 GFLOP in 372 us, 744 TFLOP/s, as the clock falls from call to call
// (336 us and 824 at its best); of the cycles the matrix pipe works 40 %, the vector units 48 %.  A wavefront's 32 rows use each operand read
// from LDS once, and its vector instructions do not run beside its own matrix instructions: with the weights of a tile formed between the
// output products of the tile before it took 386 us.
//
// (The copies are written as instructions: where the compiler knows of a copy into LDS under way, it waits for it before
// every read of LDS that it cannot tell apart from the copy's target, and with the slot in a register it can tell
// none: the copies of tile t + 1 then ended before the math of tile t began.)
// A barrier behind the wavefront's reads and writes of LDS (__syncthreads would wait for the copies as well)
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}
template <typename T, int D, bool FP8, bool ONCE> struct TileLoader;

// straight from global memory to LDS
template <typename T, int D, bool ONCE> struct TileLoader<T, D, false, ONCE> {
    // A wavefront's copies of a tile of K or V, 1 KB each (the immediate offset counts on both sides).  M0 holds the
    // target; one wait state has to pass between writing it and the copy.  It is left as it was.
    static constexpr int NI = DmaLane<D>::NI;
    __device__ __forceinline__ void copy(const Window& w, uint16_t* to, int wave, uint32_t o0, uint32_t o1, uint32_t o2, uint32_t o3) {
        const uint32_t at = lds_address(to) + 1024 * NI * wave;
        uint32_t m0;
        if constexpr (NI == 4 && ONCE)
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %5, 0 offen nt lds\n\t"
                         "buffer_load_dwordx4 %2, %5, 0 offen offset:1024 nt lds\n\t"
                         "buffer_load_dwordx4 %3, %5, 0 offen offset:2048 nt lds\n\t"
                         "buffer_load_dwordx4 %4, %5, 0 offen offset:3072 nt lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(w.words), "s"(at) : "memory");
        else if constexpr (NI == 2 && ONCE)
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %3, 0 offen nt lds\n\t"
                         "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 nt lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(o0), "v"(o1), "s"(w.words), "s"(at) : "memory");
        else if constexpr (NI == 4)
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                         "buffer_load_dwordx4 %2, %5, 0 offen offset:1024 lds\n\t"
                         "buffer_load_dwordx4 %3, %5, 0 offen offset:2048 lds\n\t"
                         "buffer_load_dwordx4 %4, %5, 0 offen offset:3072 lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(w.words), "s"(at) : "memory");
        else
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                         "buffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(o0), "v"(o1), "s"(w.words), "s"(at) : "memory");
    }
    // (offsets as in DmaLane of flashd_tile_parts.h: copy n of K takes those of the first ^ 64 n)
    __device__ __forceinline__ void start_k(const Window& w, uint16_t* to, int wave) {
        const int lane = lane_now(), row = lane / TileCfg<D>::CPR;
        const uint32_t k0 = 2 * (row * D + 8 * ((lane % TileCfg<D>::CPR) ^ TileCfg<D>::swz_k(row)));
        copy(w, to, wave, k0, k0 ^ 64u, k0 ^ 128u, k0 ^ 192u);
    }
    __device__ __forceinline__ void start_v(const Window& w, uint16_t* to, int wave) {
        const int lane = lane_now(), row = lane / TileCfg<D>::CPR;
        const uint32_t v0 = 2 * (row * D + 8 * ((lane % TileCfg<D>::CPR) ^ TileCfg<D>::swz_v(row)));
        copy(w, to, wave, v0, v0, v0, v0);
    }
    // Waits until all but the wavefront's N last tiles (of K or of V) have landed.
    template <int N>
    static __device__ __forceinline__ void wait_but() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N * NI) : "memory"); }
};

// fp8: the bytes go straight from global memory to LDS, three tiles ahead, where each wavefront takes up its own 16 keys
// again and writes them widened to where all read them.  (Through registers there was one tile ahead, 32 KB per compute unit: 64 trees
// of 6 tokens over 500 to 8192 keys took 175 us.)
template <typename T, int D, bool ONCE> struct TileLoader<T, D, true, ONCE> {
    static constexpr int NI = D / 64;           // copies of 1 KB: the wavefront's 16 rows of D bytes
    static constexpr int LPR = D / 16;
    static constexpr int kRaw = 2 * NI * 1024;  // bytes of the wavefront's K, then its V, of a tile
    u32x4 k[NI], v[NI];
    __device__ __forceinline__ void copy(const Window& w, uint32_t at) {
        const uint32_t from = 16 * lane_now();
        uint32_t m0;
        if constexpr (NI == 2 && ONCE)
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %2, 0 offen nt lds\n\t"
                         "buffer_load_dwordx4 %1, %2, 0 offen offset:1024 nt lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(from), "s"(w.words), "s"(at) : "memory");
        else if constexpr (NI == 2)
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
                         "buffer_load_dwordx4 %1, %2, 0 offen offset:1024 lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(from), "s"(w.words), "s"(at) : "memory");
        else if constexpr (ONCE)
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %2, 0 offen nt lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(from), "s"(w.words), "s"(at) : "memory");
        else
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\t"
                         "buffer_load_dwordx4 %1, %2, 0 offen lds\n\t"
                         "s_mov_b32 m0, %0"
                         : "=&s"(m0) : "v"(from), "s"(w.words), "s"(at) : "memory");
    }
    __device__ __forceinline__ void start(const Window& kw, const Window& vw, uint16_t* raw, int wave) {
        const uint32_t at = lds_address(raw) + kRaw * wave;
        copy(kw, at);
        copy(vw, at + 1024 * NI);
    }
    // Waits until all but the wavefront's N last tiles have landed.
    template <int N>
    static __device__ __forceinline__ void wait_but() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * N * NI) : "memory"); }
    __device__ __forceinline__ void take(const uint16_t* raw, int wave) {
        const u32x4* at = reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(raw) + kRaw * wave) + lane_now();
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            k[n] = at[64 * n];
            v[n] = at[64 * (NI + n)];
        }
    }
    __device__ __forceinline__ void put(uint16_t* ks, uint16_t* vs, int wave) {
        using C = TileCfg<D>;
        const int lane = lane_now();
#pragma unroll
        for (int n = 0; n < NI; ++n) {
            const int row = 16 * wave + (64 / LPR) * n + lane / LPR;
            const int ch = 2 * (lane % LPR);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *reinterpret_cast<u32x4*>(&ks[row * D + 8 * ((ch + i) ^ C::swz_k(row))]) = widen8<T>(k[n][2 * i], k[n][2 * i + 1]);
                *reinterpret_cast<u32x4*>(&vs[row * D + 8 * ((ch + i) ^ C::swz_v(row))]) = widen8<T>(v[n][2 * i], v[n][2 * i + 1]);
            }
        }
    }
};

// The scores (acc, overwritten) of NB 32-key blocks of a row: the reference moves to their top score where that lies more
// than kMoveLog2 above it, as in top_first_pack() of flashd_rows.h, looked at once for all of them; keys that the
// row does not see are -inf and scale is positive.
template <typename T, bool TR, int NB, int NDB>
__device__ __forceinline__ void weigh_blocks(f32x16 (&acc)[NB], u32x4 (&bfrag)[2 * NB], RowState& st, f32x16 (&U)[NDB],
                                             float scale) {
    const float ninf = -__builtin_inff();
    float top[2] = {acc[0][0], acc[0][1]};
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 2 * (n == 0); e < 16; e += 2) {
            top[0] = fmaxf(top[0], acc[n][e]);
            top[1] = fmaxf(top[1], acc[n][e + 1]);
        }
    const float t = pair_max(fmaxf(top[0], top[1])) * scale;
    if (__builtin_amdgcn_ballot_w64(t > st.R + LazyLimit<T>::kMoveLog2) != 0) {
        const bool move = t > st.R + LazyLimit<T>::kMoveLog2;
        const float f = move ? exp2_fast(st.R - t) : 1.0f;       // 0 for a row without keys
        st.R = move ? t : st.R;
        st.l *= f;
        if (TR) st.ltrue *= f;
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) U[i][e] *= f;
    }
    const float ref = st.R == ninf ? 0.0f : st.R;                // no key yet: weights of zero
    f32x4 ps = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < 2 * NB; ++g) {
        f32x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = exp2_fast(fmaf(acc[g >> 1][8 * (g & 1) + e], scale, -ref));
        bfrag[g] = Mma<T>::pack8(p);
        Mma<T>::sum8(p, bfrag[g], ps);
        if (TR) st.ltrue += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    }
    st.l += (ps[0] + ps[1]) + (ps[2] + ps[3]);
}

template <typename T, int D, bool FP8, int RW, bool LSE>
__global__ __launch_bounds__(kTreeWaves * kWave, 2) void tree_tile_kernel(TreeRun r) {
    using C = TileCfg<D>;
    constexpr int KW = kTreeWaves / RW;
    constexpr int M = 32 * RW;
    constexpr int NB = 2 / KW;                  // 32-key blocks of a tile that are a wavefront's
    constexpr int NKK = D / 16;
    constexpr int NDB = D / 32;
    static_assert(32 * NB < 128, "codes_of counts the keys of a wavefront's blocks");
    constexpr int kTile = kBC * D;
    constexpr int CH = D / 4;                   // 16-byte chunks of a folded row
    // Three tiles of K and two of V, 80 KB at D = 128: all of LDS in two workgroups per compute unit.  What else needs
    // LDS lies in the same memory at other times.
    __shared__ __align__(1024) uint16_t lds[5 * kTile];
    // (fp8: one of each, as numbers of 16 bits, and three tiles of K and V as they are stored.)
    uint16_t* const vlds = lds + (FP8 ? 1 : 3) * kTile;
    uint16_t* const raw = lds + 2 * kTile;
    static_assert(!FP8 || 4 * TileLoader<T, D, true, RW == 2>::kRaw == kTile * 2, "a tile's bytes");
    constexpr bool TR = kTrueSum<T, LSE>;
    float (*fold_r)[32] = reinterpret_cast<float (*)[32]>(lds + 4 * kTile), (*fold_l)[32] = fold_r + kTreeWaves, (*fold_t)[32] = fold_l + kTreeWaves;
    static_assert(kTreeWaves * 32 * D * 4 <= 4 * kTile * 2 && 3 * kTreeWaves * 32 * 4 <= kTile * 2, "the fold lies in the tiles' LDS");

    (void)r;                                    // read through args_now()
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rw = wave & (RW - 1), kw = wave / RW;
    const float ninf = -__builtin_inff();

    Walk<M, kBC, 512, kTileStart, kTileLead, RW == 4> u;
    if (!u.begin(args_now(), reinterpret_cast<WalkScratch*>(lds))) return;

    TileLoader<T, D, FP8, RW == 2> load;        // (up to 64 rows a sequence is one row tile: its keys are read once)

    do {
        const TreeRun now_r = args_now();
        const TreeArgs& a = now_r.a;
        // keys from `clear` on may be hidden from a row of the wavefront, those from `dark` on are from all
        int clear = u.s.len, dark = u.keys();
        if (a.tree == nullptr) {
            clear += (int)fast_div((uint32_t)(u.first + min(32 * rw, u.nrows - 1)), now_r.group) + 1;
            dark = u.s.len + (int)fast_div((uint32_t)(u.first + min(32 * rw + 31, u.nrows - 1)), now_r.group) + 1;
        }
        if (32 * rw >= u.nrows) dark = 0;

        // What the loop needs of the arguments, each in a register of its own (as loaded, in groups of four and more, they
        // are spilled and fetched back group by group).
        constexpr int ROW = D * (FP8 ? 1 : 2);
        const char* kpool = now_r.c.k + u.h * now_r.c.head_bytes;
        const char* vpool = now_r.c.v + u.h * now_r.c.head_bytes;
        int64_t page_bytes = now_r.c.page_bytes;
        int page_log2 = now_r.c.page_log2, pool_pages = now_r.c.P, last_key = u.keys(), blk0 = u.blk0, tiles = u.blk1 - u.blk0;
        // The page of the wavefront's 16 keys of tile i of the piece, by a scalar load (a vector load's wait would
        // be one for the copies under way as well); -1 behind the last key.
        typedef const __attribute__((address_space(4))) int* table_ptr;
        table_ptr trow = (table_ptr)(uintptr_t)(now_r.c.table + (size_t)u.b * now_r.c.max_pages);
        asm volatile("" : "+s"(kpool), "+s"(vpool), "+s"(page_bytes), "+s"(page_log2), "+s"(pool_pages), "+s"(last_key),
                          "+s"(blk0), "+s"(tiles), "+s"(trow));
        auto page_of = [&](int i) __attribute__((always_inline)) {
            const int key = (blk0 + i) * kBC + 16 * wave;
            return i < tiles && key < last_key ? trow[key >> page_log2] : -1;
        };
        auto window = [&](const char* pool, int i, int page) __attribute__((always_inline)) {
            const int key = (blk0 + i) * kBC + 16 * wave;
            const bool there = (unsigned)page < (unsigned)pool_pages;
            const uint64_t at = (uint64_t)(pool + (there ? page : 0) * page_bytes + (key & ((1 << page_log2) - 1)) * ROW);
            const int left = last_key - key, keys = !there || left < 0 ? 0 : left < 16 ? left : 16;
            return make_window(at, keys * ROW);
        };
        // The queries and the first look at the table go ahead of the copies, and are waited for with them.
        const int lane = lane_now(), col = lane & 31, hh = lane >> 5;
        const int row = u.first + min(32 * rw + col, u.nrows - 1);
        const uint16_t* qg = static_cast<const uint16_t*>(a.q) + row_at(now_r, u, row, a.q_stride, D);
        u32x4 qf[NKK];
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) qf[kk] = *reinterpret_cast<const u32x4*>(qg + 16 * kk + 8 * hh);
        // a table with holes: which of a tile's keys have no page is looked up tile by tile
        const int first_col = (blk0 * kBC >> page_log2) + lane, last_here = min((blk0 + tiles) * kBC, last_key);
        int first_page = 0;
        if (first_col << page_log2 < last_here) first_page = now_r.c.table[(size_t)u.b * now_r.c.max_pages + first_col];
        __builtin_amdgcn_sched_barrier(0);
        // the copies of tile 0's turn; behind the last tile windows are empty and copies bring zeros
        int page1 = page_of(1), page2 = page_of(2);      // of tiles now + 1 and now + 2
        Window vnext, knext;
        if constexpr (FP8) {
            const int page0 = page_of(0), page3 = page_of(3);
            load.start(window(kpool, 0, page0), window(vpool, 0, page0), raw, wave);
            load.start(window(kpool, 1, page1), window(vpool, 1, page1), raw + kTile, wave);
            load.start(window(kpool, 2, page2), window(vpool, 2, page2), raw + 2 * kTile, wave);
            knext = window(kpool, 3, page3);
            vnext = window(vpool, 3, page3);
        } else {
            const int page0 = page_of(0);
            load.start_k(window(kpool, 0, page0), lds, wave);
            load.start_v(window(vpool, 0, page0), vlds, wave);
            load.start_k(window(kpool, 1, page1), lds + kTile, wave);
            vnext = window(vpool, 1, page1);
            knext = window(kpool, 2, page2);
        }

        f32x16 U[NDB];
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) U[i][e] = 0.0f;
        RowState st = {ninf, 0.0f, 0.0f};

        // Tile i of the piece: K in slot i % 3, V in slot i % 2, copied in the order K0 V0 K1 | V1 K2 | V2 K3 | ..., the
        // last two of these while tile i is worked on.  So a tile of V has a period to arrive and one of K two: with one
        // tile of each ahead the copies' latency was longer than the math.  Two barriers a period: at its start every
        // wavefront's copies of K_i have landed and all have done with tile i - 1, whose slots the copies to start
        // then may fill; before the output product V_i has landed.
        // (One body for all slots and both blocks: copies of it with constant operand addresses cost the code
        // that masks need several times, and with it the registers that hold U.)
        bool gaps = (unsigned)first_page >= (unsigned)pool_pages;
        for (int k = first_col + kWave; k << page_log2 < last_here; k += kWave) gaps |= page_at(now_r.c, u.b, k) < 0;
        gaps = __builtin_amdgcn_ballot_w64(gaps) != 0;
        // The queries are here to stay before the loop, as the compiler knows: it would else wait for them, and so for all copies, in every turn.
        wait_copies();
        // a negative scale is taken into Q (exact), so that the largest dot product is the top score
        float c_log2 = (FP8 ? a.scale * now_r.c.kscale : a.scale) * kLog2e;
        if (c_log2 < 0.0f) {
            c_log2 = -c_log2;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) qf[kk] ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
        }
        int kslot = 0;
#pragma unroll 1
        for (int now = 0; now < tiles; ++now) {
            const int t = blk0 + now;
            const int k1slot = kslot == 2 ? 0 : kslot + 1;
            int page4;
            if constexpr (FP8) {
                // Its 16 keys are the wavefront's own affair up to the first barrier, behind which nobody reads the tile before
                load.template wait_but<2>();
                load.take(raw + kslot * kTile, wave);
                barrier();
                load.start(knext, vnext, raw + kslot * kTile, wave);
                page4 = page_of(now + 4);
                load.put(lds, vlds, wave);
                barrier();
            } else {
                load.template wait_but<2>();
                barrier();
                load.start_v(vnext, vlds + ((now + 1) & 1) * kTile, wave);
                load.start_k(knext, lds + (k1slot == 2 ? 0 : k1slot + 1) * kTile, wave);
            }
            page1 = page2;
            page2 = page_of(now + 3);
            const uint16_t* ks = FP8 ? lds : lds + kslot * kTile;
            const uint16_t* vs = FP8 ? vlds : vlds + (now & 1) * kTile;
            uint32_t hole = 0;                           // 16-key groups of this tile without a page
            if (gaps) {
                const int key = t * kBC + 16 * (lane_now() & 3);
                const TreeRun m = args_now();
                hole = (uint32_t)__builtin_amdgcn_ballot_w64(key >= last_key || page_at(m.c, u.b, key >> page_log2) < 0) & 15u;
            }
            const int j0 = t * kBC + 32 * kw;            // first of the wavefront's keys of this tile
            const bool work = j0 < dark;
            f32x16 acc[NB];
            if (work) {
                // operand kk's address is that of the first ^ 16 kk elements, under the swizzle's exclusive or
                const int x = lane_now();
                const int kaddr = (32 * kw + (x & 31)) * D + 8 * ((x >> 5) ^ C::swz_k(x & 31));
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[n][e] = 0.0f;
                // Reads run 8 ahead of the products (LDS returns in order); the chains of the two blocks alternate.
                constexpr int AHEAD = NKK * NB < 8 ? NKK * NB : 8;
                u32x4 ka[NKK * NB];
#pragma unroll
                for (int m = 0; m < AHEAD; ++m) ka[m] = *reinterpret_cast<const u32x4*>(&ks[(kaddr ^ 16 * (m / NB)) + 32 * D * (m % NB)]);
#pragma unroll
                for (int m = 0; m < NKK * NB; ++m) {
                    acc[m % NB] = Mma<T>::mfma(ka[m], qf[m / NB], acc[m % NB]);
                    if (m + AHEAD < NKK * NB)
                        ka[m + AHEAD] = *reinterpret_cast<const u32x4*>(&ks[(kaddr ^ 16 * ((m + AHEAD) / NB)) + 32 * D * ((m + AHEAD) % NB)]);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
                for (int m = AHEAD; m < NKK * NB; ++m) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (FP8) {
                knext = window(kpool, now + 4, page4);
                vnext = window(vpool, now + 4, page4);
            } else {
                vnext = window(vpool, now + 2, page1);
                knext = window(kpool, now + 3, page2);
                load.template wait_but<3>();
                barrier();
            }
            if (work) {
                // V operands on their way while the coefficients are formed
                const int x = lane_now(), xq = (x & 15) >> 2;
                const int vaddr = (32 * kw + 4 * (x >> 5) + xq) * D + 8 * ((2 * (x >> 4 & 1) + ((x & 3) >> 1)) ^ C::swz_v(xq)) + 4 * (x & 1);
                auto v_operand = [&](int n, int m) __attribute__((always_inline)) {
                    return tile_v_operand<D>(vs, vaddr ^ 32 * (m % NDB), 32 * n + 16 * (m / NDB));
                };
                auto read_v = [&](u32x4 (&va)[2 * NDB], int n) __attribute__((always_inline)) {
#pragma unroll
                    for (int m = 0; m < 2 * NDB; ++m) va[m] = v_operand(n, m);
                    __builtin_amdgcn_sched_barrier(0);
                };
                u32x4 va[NB][2 * NDB];
                read_v(va[0], 0);

                const uint32_t lost = hole >> (2 * kw);
                const bool masked = lost != 0 || j0 + 32 * NB > clear;
                float scale = c_log2;
                uint32_t mine[NB];
                if (masked) {
                    const TreeRun m = args_now();
                    const int token = (int)fast_div((uint32_t)(u.first + min(32 * rw + (x & 31), u.nrows - 1)), m.group);
                    // (a scale of 0 or NaN would take a hidden key away from -inf: it is applied here)
                    const float by = c_log2 > 0.0f ? 1.0f : c_log2;
                    scale = c_log2 > 0.0f ? c_log2 : 1.0f;
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        uint32_t bits = seen_bits(m.a, u.s, token, u.s.row0 + token, j0 + 32 * n);
                        if (lost >> (2 * n) & 1u) bits &= 0xffff0000u;
                        if (lost >> (2 * n) & 2u) bits &= 0x0000ffffu;
                        mine[n] = bits >> (4 * (x >> 5));
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[n][e] = if_seen(mine[n], 8 * (e >> 2) + (e & 3), acc[n][e] * by);
                    }
                }
                u32x4 bfrag[2 * NB];
                weigh_blocks<T, TR, NB, NDB>(acc, bfrag, st, U, scale);
                bool apart = false;
                if (masked) {
                    // (operands are read anew here, a few at a time: the registers are taken)
                    uint32_t bad = 0;
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int m = 0; m < 2 * NDB; ++m) {
                            bad |= not_finite<T, false>(v_operand(n, m));
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    apart = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
                    if (apart) {
#pragma unroll
                        for (int i = 0; i < NDB; ++i) {
                            f32x16 count;
#pragma unroll
                            for (int e = 0; e < 16; ++e) count[e] = 0.0f;
#pragma unroll
                            for (int g = 0; g < 2 * NB; ++g) {
                                const uint32_t of = mine[g >> 1] >> (16 * (g & 1));
                                count = Mma<T>::mfma(codes_of<T>(v_operand(g >> 1, (g & 1) * NDB + i)),
                                                     ones_of<T>((of & 15u) | (of >> 8 & 15u) << 4), count);
                                __builtin_amdgcn_sched_barrier(0);
                            }
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                U[i][e] += what_is_seen(count[e]);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                    }
                }
#pragma unroll
                for (int n = 1; n < NB; ++n) read_v(va[n], n);
                if (apart) {
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int m = 0; m < 2 * NDB; ++m) va[n][m] = numbers_of<T>(va[n][m]);
                }
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int m = 0; m < 2 * NDB; ++m) U[m % NDB] = Mma<T>::mfma(va[n][m], bfrag[2 * n + m / NDB], U[m % NDB]);
            }
            kslot = k1slot;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // the last, empty copies: LDS is used otherwise now
        __syncthreads();

        // ---- rows through LDS; with KW = 2 the two states of a row are joined.  Chunk t of row c lies at t ^ c.
        const float l = pair_sum(st.l), tr = TR ? pair_sum(st.ltrue) : 0.0f;
        float* fold = reinterpret_cast<float*>(lds);
        const int elane = lane_now(), ecol = elane & 31, tid = 64 * wave + elane;
        const TreeRun end_r = args_now();
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                *reinterpret_cast<f32x4*>(&fold[((wave * 32 + ecol) * CH + ((8 * i + 2 * y + (elane >> 5)) ^ (ecol & (CH - 1)))) * 4]) =
                    f32x4{U[i][4 * y], U[i][4 * y + 1], U[i][4 * y + 2], U[i][4 * y + 3]};
        if (elane < 32) {
            fold_r[wave][ecol] = st.R;
            fold_l[wave][ecol] = l;
            if (TR) fold_t[wave][ecol] = tr;
        }
        __syncthreads();
        for (int idx = tid; idx < u.nrows * CH; idx += kTreeWaves * kWave) {
            const int fr = idx / CH, ch = idx % CH;
            const int w0 = fr >> 5, rc = fr & 31;
            float top = fold_r[w0][rc];
#pragma unroll
            for (int k = 1; k < KW; ++k) top = fmaxf(top, fold_r[w0 + RW * k][rc]);
            float lt = 0.0f, tt = 0.0f;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const int w = w0 + RW * k;
                const bool none = fold_l[w][rc] == 0.0f;
                const float f = none ? 0.0f : exp2_fast(fold_r[w][rc] - top);
                const f32x4 x = *reinterpret_cast<const f32x4*>(&fold[((w * 32 + rc) * CH + (ch ^ (rc & (CH - 1)))) * 4]);
                lt = fmaf(f, fold_l[w][rc], lt);
                if (TR) tt = fmaf(f, fold_t[w][rc], tt);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(f, none ? 0.0f : x[e], o[e]);
            }
            put_row<T, D, M, LSE>(end_r, u, fr, 4 * ch, o, top, lt, FP8 ? end_r.c.vscale : 1.0f, tt);
        }
        if (u.blk0 == 0 && !u.whole() && tid == 0) u.note_split(end_r);
        __syncthreads();
    } while (u.next(args_now()));
}

// ---- the same in fp32 ------------------------------------------------------------------------------
//
// v_mfma_f32_16x16x4_f32: lane (q, c) gives element q of the four that are summed, row (or column) c.  K as the A
// operand: the lane's float4 at dims 16 m + 4 q serves four products, each summing dims 16 m + 4 q' + e over
// q'.  The scores it gets are keys 4 q + r of its row: as B operand of O^T = V^T P^T product r sums
// the keys 4 q' + r over q'.  The lane's float4 of V[4 q + r] at columns 64 g + 4 c serves four of them, product j for the columns
// 64 g + 4 c' + j: of those the lane's results are 64 g + 16 q + 4 d + j, d = 0 .. 3.  Nothing goes through LDS; V
// of a block is on its way while K is multiplied, K of the next one while V is.
//
// NR: 16-row column tiles, which read the keys once.  With two, and at d = 128, there is one workgroup per compute unit, whose registers
// they need.  One token for each of 64 sequences of 500 to 8192 keys, 32 / 8 heads of 128: 386 us with the merge, 2.34 GB, 6.1 TB/s
// (two workgroups, with spills: 424; without anything under way in the meantime 465); d = 64: 184 us.  8 chunks of 100 to 200 tokens after
// 500 to 4000 keys: 52 GFLOP in 705 us, 74 TFLOP/s of the 154 that a large product of the library reaches: each 32 rows read the keys anew.
// A weight is at most 2^(8 - 40): 10^9 of them add up to less than 1, so that values of any size that fp32 holds have a finite sum.  The factor is
// applied to the weights: with the reference 40 above the top score the exponential's argument would be rounded to 2^-19 instead of
// 2^-22, which made outputs 9e-7 from fp64 where they are 3.4 to 4.9e-7 now (2-norm, N(0, 1) inputs).  Weights below 2^-86 of the one at the
// reference lose bits, and below 2^-109 they are zero.
constexpr int f32_per_cu(int D, int NR) { return D == 64 && NR == 1 ? 2 : 1; }
template <int D, int NR, bool LSE>
__global__ __launch_bounds__(kTreeWaves * kWave, f32_per_cu(D, NR)) void tree_rows_f32_kernel(TreeRun r) {
    constexpr int W = kTreeWaves;
    constexpr int NDB = D / 16;
    constexpr int NG = D / 64;
    __shared__ __align__(16) float fold[W * 16 * (D + 4)];

    (void)r;                                             // read through args_now()
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;
    const int q = lane >> 4;
    const float ninf = -__builtin_inff();

    Walk<16 * NR, kTreeBlock, 256 * f32_per_cu(D, NR), kRowsStart, kRowsLead, false> u;
    if (!u.begin(args_now(), reinterpret_cast<WalkScratch*>(fold))) return;
    do {
        const TreeRun now_r = args_now();
        f32x4 qf[NR][NDB];
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            const int row = u.first + min(16 * k + col, u.nrows - 1);
            const float* qg = static_cast<const float*>(now_r.a.q) + row_at(now_r, u, row, now_r.a.q_stride, D);
#pragma unroll
            for (int m = 0; m < NDB; ++m) qf[k][m] = *reinterpret_cast<const f32x4*>(qg + 16 * m + 4 * q);
        }
        __builtin_amdgcn_sched_barrier(0);
        const float c_log2 = now_r.a.scale * kLog2e;

        // as in tree_rows_kernel
        constexpr int ROWB = 4 * D;
        const char* kpool = now_r.c.k + u.h * now_r.c.head_bytes;
        const char* vpool = now_r.c.v + u.h * now_r.c.head_bytes;
        int64_t page_bytes = now_r.c.page_bytes;
        int page_log2 = now_r.c.page_log2, pool_pages = now_r.c.P, last_key = u.keys(), blk_end = u.blk1, len = u.s.len;
        typedef const __attribute__((address_space(4))) int* table_ptr;
        table_ptr trow = (table_ptr)(uintptr_t)(now_r.c.table + (size_t)u.b * now_r.c.max_pages);
        asm volatile("" : "+s"(kpool), "+s"(vpool), "+s"(page_bytes), "+s"(page_log2), "+s"(pool_pages), "+s"(last_key),
                          "+s"(blk_end), "+s"(len), "+s"(trow));
        auto page_of = [&](int blk, int half) __attribute__((always_inline)) {
            const int key = blk * kTreeBlock + 16 * half;
            const int p = blk < blk_end && key < last_key ? trow[key >> page_log2] : -1;
            return (unsigned)p < (unsigned)pool_pages ? p : -1;
        };
        auto half_window = [&](const char* pool, int blk, int half, int p) __attribute__((always_inline)) {
            const int key = blk * kTreeBlock + 16 * half;
            const uint64_t at = (uint64_t)(pool + max(p, 0) * page_bytes + (key & ((1 << page_log2) - 1)) * ROWB);
            const int left = last_key - key, keys = p < 0 || left < 0 ? 0 : left < 16 ? left : 16;
            return make_window(at, keys * ROWB).rsrc();
        };
        f32x4 kreg[2][NDB], vreg[8][NG];
        auto fetch_k = [&](int blk, int p0, int p1) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto w = half_window(kpool, blk, t, t ? p1 : p0);
#pragma unroll
                for (int m = 0; m < NDB; ++m) kreg[t][m] = __builtin_bit_cast(f32x4, kv_load<2>(w, (col * D + 16 * m + 4 * q) * 4));
            }
        };
        auto fetch_v = [&](int blk, int p0, int p1) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto w = half_window(vpool, blk, t, t ? p1 : p0);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int g = 0; g < NG; ++g)
                        vreg[4 * t + e][g] = __builtin_bit_cast(f32x4, kv_load<2>(w, ((4 * q + e) * D + 64 * g + 4 * col) * 4));
            }
        };

        f32x4 U[NR][NDB];                                // [4 g + j][d]: column 64 g + 16 q + 4 d + j
        float R[NR], l[NR], none[NR];
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            R[k] = ninf;
            l[k] = 0.0f;
            none[k] = 0.0f;
#pragma unroll
            for (int i = 0; i < NDB; ++i) U[k][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        int blk = u.blk0 + wave;
        int p0 = page_of(blk, 0), p1 = page_of(blk, 1), n0 = page_of(blk + W, 0), n1 = page_of(blk + W, 1);
        __builtin_amdgcn_sched_barrier(0);
        fetch_k(blk, p0, p1);
        __builtin_amdgcn_sched_barrier(0);
        fetch_v(blk, p0, p1);
        __builtin_amdgcn_sched_barrier(0);
        wait_loads<2 * NDB + 8 * NG>();                  // the queries are here, as the compiler knows
        for (; blk < blk_end; blk += W) {
            const int j0 = blk * kTreeBlock;
            const uint32_t have = (p0 < 0 ? 0u : 0x0000ffffu) | (p1 < 0 ? 0u : 0xffff0000u);
            const int m0 = page_of(blk + 2 * W, 0), m1 = page_of(blk + 2 * W, 1);
            f32x4 acc[NR][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int k = 0; k < NR; ++k) acc[k][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int m = 0; m < NDB; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int k = 0; k < NR; ++k)
                            acc[k][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kreg[t][m][e], qf[k][m][e], acc[k][t], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            fetch_k(blk + W, n0, n1);
            __builtin_amdgcn_sched_barrier(0);
            const bool masked = have != ~0u || j0 + kTreeBlock > len;
            uint32_t bits[NR];
            f32x8 pv[NR];
#pragma unroll
            for (int k = 0; k < NR; ++k) {
                bits[k] = ~0u;
                if (masked) {
                    const TreeRun m = args_now();
                    const int token = (int)fast_div((uint32_t)(u.first + min(16 * k + col, u.nrows - 1)), m.group);
                    bits[k] = have & seen_bits(m.a, u.s, token, u.s.row0 + token, j0);
                }
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = acc[k][e >> 2][e & 3] * c_log2;
                    if (masked) x[e] = if_seen(bits[k] >> (4 * q), 16 * (e >> 2) + (e & 3), x[e]);
                }
                weigh<false>(x, pv[k], U[k], R[k], l[k], none[k], kF32Move, kF32Unit);
                l[k] += ((pv[k][0] + pv[k][1]) + (pv[k][2] + pv[k][3])) + ((pv[k][4] + pv[k][5]) + (pv[k][6] + pv[k][7]));
            }
            bool apart = false;
            if (masked) {
                bool bad = false;
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int j = 0; j < 4; ++j) bad |= !(fabsf(vreg[e][g][j]) <= 3.4028234e38f);
                apart = __builtin_amdgcn_ballot_w64(bad) != 0;
            }
            if (apart) {
                // an infinite or NaN value: key by key, only where the row sees it
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll 1
                    for (int z = 0; z < 4; ++z)
#pragma unroll
                        for (int g = 0; g < NG; ++g)
#pragma unroll
                            for (int j = 0; j < 4; ++j)
#pragma unroll
                                for (int d = 0; d < 4; ++d) {
                                    __builtin_amdgcn_sched_barrier(0);           // few registers at a time
                                    const float y = __shfl(vreg[e][g][j], 16 * z + 4 * q + d);
#pragma unroll
                                    for (int k = 0; k < NR; ++k) {
                                        const float wt = __shfl(pv[k][e], 16 * z + col);
                                        const bool seen = (bits[k] >> (16 * (e >> 2) + 4 * z + (e & 3)) & 1u) != 0;
                                        U[k][4 * g + j][d] = seen ? fmaf(wt, y, U[k][4 * g + j][d]) : U[k][4 * g + j][d];
                                    }
                                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int k = 0; k < NR; ++k)
                                U[k][4 * g + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vreg[e][g][j], pv[k][e], U[k][4 * g + j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            fetch_v(blk + W, n0, n1);
            __builtin_amdgcn_sched_barrier(0);
            p0 = n0;
            p1 = n1;
            n0 = m0;
            n1 = m1;
        }
        // column by column, as finish_rows takes them
#pragma unroll
        for (int k = 0; k < NR; ++k)
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                f32x4 x[4];
#pragma unroll
                for (int d = 0; d < 4; ++d) x[d] = f32x4{U[k][4 * g][d], U[k][4 * g + 1][d], U[k][4 * g + 2][d], U[k][4 * g + 3][d]};
#pragma unroll
                for (int d = 0; d < 4; ++d) U[k][4 * g + d] = x[d];
            }
        finish_rows<F32, D, NR, false, LSE>(args_now(), u, U, R, l, none, fold, 1.0f);
    } while (u.next(args_now()));
}

// ---- join the parts of split units -------------------------------------------------------------
//
// The rows of all split units, one after the other, are dealt out evenly: a fixed number of workgroups, each of which
// sums up how many there are and walks its share.  D / 4 lanes take 4 columns each of a row; the 1024 / D such
// groups of a workgroup take a row each, or share the parts of one row where a unit has many (more than
// kMergeShare: one long sequence over the whole chip).  Each thread of a workgroup keeps the splits of a few of the
// launch's workgroups, and the one that holds the next rows' hands it over through LDS: between a workgroup's start
// and its rows lies one read from memory.  M: rows of a tile.  8 units of 4 rows in 8 parts take 3.5 us, 512 of 128 rows in 2 and 3
// parts (67 MB) 18.  What bounds it is the time of its reads, so that many workgroups
// are under way at once where there are many rows.
constexpr int kMergeShare = 12;
constexpr int merge_groups(int M) { return M <= 32 ? 512 : M == 64 ? 1024 : 2048; }

// One row's parts k0, k0 + step, ...: unnormalised sum against `top`.
template <int D, int M, bool TR>
__device__ __forceinline__ f32x4 merge_parts(const TreeRun& r, int w, int parts, int fr, int t, int k0, int step,
                                             float& top, float& lt, float& tr) {
    constexpr int AHEAD = 4;             // parts read together
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = k0; k < parts; k += AHEAD * step) {
        float2 st[AHEAD];
        float ts[AHEAD];
        f32x4 u[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int part = min(k + i * step, parts - 1);
            const size_t at = (size_t)(2 * (w + part) + (part == 0 ? 1 : 0)) * M + fr;
            st[i] = r.stats[at];
            ts[i] = TR ? r.sums[at] : 0.0f;
            u[i] = *reinterpret_cast<const f32x4*>(r.parts + at * D + t);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k + i * step >= parts || st[i].y == 0.0f) continue;         // no key of this row
            const float now = fmaxf(top, st[i].x);
            const float f0 = top == -__builtin_inff() ? 0.0f : exp2_fast(top - now), f1 = exp2_fast(st[i].x - now);
            lt = fmaf(lt, f0, st[i].y * f1);
            if (TR) tr = fmaf(tr, f0, ts[i] * f1);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], f0, u[i][e] * f1);
            top = now;
        }
    }
    return o;
}

template <typename T, int D, int M, bool LSE>
__global__ __launch_bounds__(256, 4) void merge_tree_kernel(TreeRun r, float vscale) {
    constexpr bool TR = kTrueSum<T, LSE>;
    constexpr int LPR = D / 4;
    constexpr int NG = 256 / LPR;
    constexpr int EACH = kTreeMostGroups / 256;
    __shared__ __align__(16) float sum[NG][D];
    __shared__ float2 part_stat[NG];
    __shared__ float part_true[TR ? NG : 1];
    __shared__ int next[sizeof(TreeSplit) / 4];
    __shared__ int next_item;
    __shared__ int wave_sum[EACH][kTreeWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float ninf = -__builtin_inff();
    // Word by word: a struct is kept in LDS, where the compiler finds its place from the launch's size, which it
    // reads from the host's memory (12 us).
    constexpr int WORDS = sizeof(TreeSplit) / 4, ROWS = offsetof(TreeSplit, rows) / 4, PARTS = offsetof(TreeSplit, parts) / 4;
    int mine[EACH][WORDS];
    int items[EACH], before[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int* sp = reinterpret_cast<const int*>(r.splits + min(256 * k + tid, r.groups - 1));
#pragma unroll
        for (int i = 0; i < WORDS; ++i) mine[k][i] = sp[i];
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int rows = mine[k][ROWS], parts = mine[k][PARTS];
        items[k] = 256 * k + tid >= r.groups || parts == 0 ? 0 : parts > kMergeShare ? rows : (rows + NG - 1) / NG;
        const int in = lanes_up_to(items[k]);
        if (lane == 63) wave_sum[k][wave] = in;
        before[k] = in - items[k];
    }
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
#pragma unroll
        for (int i = 0; i < kTreeWaves; ++i) {
            if (i == wave) before[k] += total;
            total += wave_sum[k][i];
        }
    }
    total = uniform(total);
    const int g = tid / LPR, t = 4 * (tid % LPR);
    const int G = (int)r.group.d;
    for (int item = blockIdx.x; item < total; item += gridDim.x) {
        __syncthreads();                     // the last item's sums and split are read
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            if (item >= before[k] && item - before[k] < items[k]) {
#pragma unroll
                for (int i = 0; i < WORDS; ++i) next[i] = mine[k][i];
                next_item = item - before[k];
            }
        }
        __syncthreads();
        TreeSplit sp;
        __builtin_memcpy(&sp, next, sizeof(sp));
        const int w = uniform(sp.w), parts = uniform(sp.parts), of = uniform(next_item);
        float top = ninf, lt = 0.0f, tr = 0.0f;
        f32x4 o;
        int fr;
        if (parts > kMergeShare) {
            fr = of;
            o = merge_parts<D, M, TR>(r, w, parts, fr, t, g, NG, top, lt, tr);
            *reinterpret_cast<f32x4*>(&sum[g][t]) = o;
            if (t == 0) part_stat[g] = float2{top, lt};
            if (TR && t == 0) part_true[TR ? g : 0] = tr;
            __syncthreads();
            if (g != 0) continue;
            float all = ninf;
#pragma unroll
            for (int k = 0; k < NG; ++k) all = fmaxf(all, part_stat[k].x);
            lt = 0.0f;
            tr = 0.0f;
            top = all;
            o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const float2 st = part_stat[k];
                const float f = st.y == 0.0f ? 0.0f : exp2_fast(st.x - all);
                const f32x4 u = *reinterpret_cast<const f32x4*>(&sum[k][t]);
                lt = fmaf(f, st.y, lt);
                if (TR) tr = fmaf(f, part_true[TR ? k : 0], tr);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(f, u[e], o[e]);
            }
        } else {
            fr = of * NG + g;
            if (fr >= sp.rows) continue;
            o = merge_parts<D, M, TR>(r, w, parts, fr, t, 0, 1, top, lt, tr);
        }
        if (lt != 0.0f) o *= vscale / lt;
        const int rw = sp.first + fr;
        const int tk = (int)fast_div((uint32_t)rw, r.group);
        if (LSE && t == 0) r.a.lse[(size_t)(sp.row0 + tk) * r.a.Hq + sp.h * G + rw - tk * G] = lse_of<T>(top, TR ? tr : lt);
        Store<T>::store4(r.a.o, (size_t)(sp.row0 + tk) * r.a.o_stride + (size_t)(sp.h * G + rw - tk * G) * D + t,
                         {o[0], o[1], o[2], o[3]});
    }
}

// ---- host ------------------------------------------------------------------------------------------

// Rows of a tile, chosen by how many the longest sequence has (tokens times heads of a group): the least that hold them, so that
// its keys are read once; above 64 the tiles share a sequence's keys through L2.  32 rows only pay from an fp8 cache, where the keys'
// way through LDS counts for more than their bytes: 24 rows, 64 sequences of 500 to 8192 keys, d = 128: 138 us with 32 and
// 145 with 64, d = 64: 87 and 108; from bf16, 32 such sequences: 144 and 117, d = 64: 64 and 64.  16 rows against 64 for 4 rows of
// 64 sequences: 192 and 198 us, fp8 115 and 156, one short sequence 15 and 19.  128 against 64 for chunks of 1000
// tokens: 401 and 562.  fp32, 16 against 32: 4 rows 400 and 474 us, 20 rows 263 and 249, 32 rows 403 and 270.
static int tree_rows(int Hq, int Hkv, int max_q, int dtype, bool fp8) {
    const long rows = (long)max_q * (Hq / Hkv);
    if (dtype == 0) return rows <= 16 ? 16 : 32;
    return rows <= 16 ? 16 : rows <= 32 && fp8 ? 32 : rows <= 64 ? 64 : 128;
}

size_t attn_tree_workspace(int Hq, int Hkv, int max_q, int d, int dtype) {
    const int rows = tree_rows(Hq, Hkv, max_q, dtype, false);
    return (size_t)2 * kTreeMostGroups * rows * (d + 3) * sizeof(float) + kTreeMostGroups * sizeof(TreeSplit);
}

template <typename T, int D, int M, bool LSE>
static hipError_t launch_tree_m(TreeRun& r, hipStream_t st) {
    const dim3 block(kTreeWaves * kWave);
    r.stats = reinterpret_cast<float2*>(r.parts + (size_t)2 * kTreeMostGroups * M * D);
    r.splits = reinterpret_cast<TreeSplit*>(r.stats + (size_t)2 * kTreeMostGroups * M);
    r.sums = reinterpret_cast<float*>(r.splits + kTreeMostGroups);
    auto launch = [&](auto* kernel, int groups) {
        r.groups = groups;
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), block, 0, st, r);
    };
    if constexpr (std::is_same_v<T, F32>) launch(tree_rows_f32_kernel<D, M / 16, LSE>, 256 * f32_per_cu(D, M / 16));
    else if constexpr (M == 32) launch(tree_rows_kernel<T, D, true, 2, LSE>, 256 * rows_per_cu(D, true, 2));
    else if constexpr (M == 16) {
        if (r.a.fp8) launch(tree_rows_kernel<T, D, true, 1, LSE>, 256 * rows_per_cu(D, true, 1));
        else launch(tree_rows_kernel<T, D, false, 1, LSE>, 256 * rows_per_cu(D, false, 1));
    } else {
        if (r.a.fp8) launch(tree_tile_kernel<T, D, true, M / 32, LSE>, 512);
        else launch(tree_tile_kernel<T, D, false, M / 32, LSE>, 512);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((merge_tree_kernel<T, D, M, LSE>), dim3(merge_groups(M)), block, 0, st, r,
                       r.a.fp8 ? r.c.vscale : 1.0f);
    return hipGetLastError();
}

template <typename T, int D, bool LSE>
static hipError_t launch_tree_l(TreeRun& r, hipStream_t st) {
    const int rows = tree_rows(r.a.Hq, r.c.Hkv, r.a.max_q, r.a.dtype, r.a.fp8 != 0);
    switch (rows) {
    case 16: return launch_tree_m<T, D, 16, LSE>(r, st);
    case 32: return launch_tree_m<T, D, 32, LSE>(r, st);
    }
    if constexpr (std::is_same_v<T, F32>) return hipErrorInvalidValue;          // tree_rows() has no more for it
    else return rows == 64 ? launch_tree_m<T, D, 64, LSE>(r, st) : launch_tree_m<T, D, 128, LSE>(r, st);
}
template <typename T, int D>
static hipError_t launch_tree_t(TreeRun& r, hipStream_t st) {
    return r.a.lse != nullptr ? launch_tree_l<T, D, true>(r, st) : launch_tree_l<T, D, false>(r, st);
}

hipError_t launch_attn_tree(const Paged& c, const TreeArgs& a, hipStream_t st) {
    TreeRun r;
    r.c = c;
    r.a = a;
    r.group = make_fast_div((uint32_t)(a.Hq / c.Hkv));
    r.parts = a.ws;
    const bool small = c.d == 64;
    if (a.dtype == 0) return small ? launch_tree_t<F32, 64>(r, st) : launch_tree_t<F32, 128>(r, st);
    if (a.dtype == 1) return small ? launch_tree_t<F16, 64>(r, st) : launch_tree_t<F16, 128>(r, st);
    return small ? launch_tree_t<BF16, 64>(r, st) : launch_tree_t<BF16, 128>(r, st);
}

}  // namespace flashd
