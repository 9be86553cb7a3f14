// Attention of each sequence's new tokens over its keys in the paged cache and, as a chain or a
// tree, over each other (flashd_attn_fwd_tree).
//
// For the new token i of sequence b and query head h, o = sum_j softmax_j(scale q.k_j) v_j over the
// keys j < len (all of them) and the new keys len + j that the token's bits name (a chain: j <= i).
// The heads of a kv group read the same keys, so the rows of a unit of work are pairs (token, head of the
// group), 16 of them to a tile, and a unit is (sequence, kv head, row tile).
//
// Sequences differ in length by orders of magnitude and the host does not know by how much, so the
// launch has a fixed number of workgroups and each finds its share of the work by itself: the units'
// 32-key blocks form one long row, workgroup w takes blocks [w per, (w + 1) per).  All workgroups so stream the
// same number of keys to within one block.  A unit that ends up in several workgroups is
// left as partial states (at most two per workgroup: its first unit, begun by the one before, and its
// last) that merge_tree_kernel joins in the order of the keys: the result does not depend on timing.
#include "flashd_common.h"
#include "flashd_kernels.h"
#include "flashd_mma.h"
#include "flashd_paged.h"

#include <type_traits>

namespace flashd {

constexpr int kTreeBlock = 32;          // keys per step of a wavefront
constexpr int kTreeWaves = 4;
constexpr int kTreeMostGroups = 512;    // workgroups of a launch
constexpr int kTreeMinBlocks = 4;       // blocks a workgroup takes at least, one per wavefront

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
    int pad[3];
};

struct TreeRun {
    Paged c;
    TreeArgs a;
    FastDiv group;          // query heads per kv head
    float* parts;           // [2 groups][16][d] unnormalised outputs
    float2* stats;          // [2 groups][16] reference and sum of weights
    TreeSplit* splits;      // [groups]
};

constexpr int kTreeRows = 16;

// ---- the share of a workgroup ------------------------------------------------------------------

__device__ __forceinline__ int tree_tiles(const Seq& s, int G) {
    return (int)(((long long)s.n * G + kTreeRows - 1) / kTreeRows);
}
__device__ __forceinline__ int tree_blocks(const Seq& s) {
    return (s.len + s.n + kTreeBlock - 1) / kTreeBlock;
}

// A workgroup's way along the row of blocks, and the piece of a unit that it is at (all the same in every
// thread).
struct Walk {
    long long at, end;      // blocks of the long row
    long long per;          // blocks of every workgroup
    long long in_b, in_seq; // blocks of the present sequence before `at`, and in all
    int b;                  // present sequence
    Seq s;
    int blocks, tiles;      // of the present sequence: blocks per unit, row tiles
    // the piece
    int h, first, nrows;    // kv head; first row (token, head of the group) of the tile, rows
    int blk0, blk1;         // its blocks of the unit

    __device__ __forceinline__ bool whole() const { return blk0 == 0 && blk1 == blocks; }

    __device__ __forceinline__ void enter(const Paged& c, int G, int seq) {
        b = seq;
        s = seq_at(c, b);
        blocks = tree_blocks(s);
        tiles = tree_tiles(s, G);
        in_seq = (long long)tiles * c.Hkv * blocks;
    }

    // The next piece; false at the end of the share.
    __device__ __forceinline__ bool next(const Paged& c, int G) {
        if (at >= end) return false;
        while (in_b >= in_seq) {            // on to the next sequence with new tokens
            if (b + 1 >= c.B) return false;
            enter(c, G, b + 1);
            in_b = 0;
        }
        const int unit = (int)(in_b / blocks);
        blk0 = (int)(in_b - (long long)unit * blocks);
        const long long left = end - at;
        blk1 = (int)(left < blocks - blk0 ? blk0 + left : blocks);
        h = unit / tiles;
        first = (unit - h * tiles) * kTreeRows;
        nrows = min(kTreeRows, s.n * G - first);
        return true;
    }
    __device__ __forceinline__ void done() {
        at += blk1 - blk0;
        in_b += blk1 - blk0;
    }
};

// Every thread of the workgroup takes a run of sequences, whose blocks are then summed over the threads.
__device__ __forceinline__ Walk begin_walk(const Paged& c, int G) {
    __shared__ long long wave_sum[kTreeWaves];
    __shared__ long long found_before;
    __shared__ int found_b;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (c.B + kTreeWaves * kWave - 1) / (kTreeWaves * kWave);
    const int b0 = tid * each, b1 = min(b0 + each, c.B);
    Walk r;
    long long mine = 0;
    for (int b = b0; b < b1; ++b) {
        r.enter(c, G, b);
        mine += r.in_seq;
    }
    long long in = mine;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const long long y = __shfl_up(in, s);
        if (lane >= s) in += y;
    }
    if (lane == 63) wave_sum[wave] = in;
    if (tid == 0) found_b = -1;
    __syncthreads();
    long long before = in - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kTreeWaves; ++w) {
        before += w < wave ? wave_sum[w] : 0;
        total += wave_sum[w];
    }
    long long groups = (total + kTreeMinBlocks - 1) / kTreeMinBlocks;
    if (groups > gridDim.x) groups = gridDim.x;
    r.per = groups > 0 ? (total + groups - 1) / groups : 1;
    r.at = r.per * blockIdx.x;
    r.end = r.at + r.per < total ? r.at + r.per : total;
    if (r.at < r.end && r.at >= before && r.at < before + mine) {
        for (int b = b0; b < b1; ++b) {
            r.enter(c, G, b);
            if (r.at < before + r.in_seq) {
                found_b = b;
                found_before = before;
                break;
            }
            before += r.in_seq;
        }
    }
    __syncthreads();
    const int b = __builtin_amdgcn_readfirstlane(found_b);
    if (b < 0) {
        r.end = r.at;
        return r;
    }
    r.in_b = r.at - found_before;
    r.enter(c, G, b);
    return r;
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
// where the top one lies more than `limit` above it and turns the scores into weights.
template <int NDB>
__device__ __forceinline__ void weigh(float (&x)[8], f32x8& p, f32x4 (&U)[NDB], float& R, float& l, float limit) {
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
#pragma unroll
        for (int i = 0; i < NDB; ++i) U[i] *= f;
    }
    const float ref = R == ninf ? 0.0f : R;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = exp2_fast(x[e] - ref);
}

// Joins the wavefronts' states of a piece: the output if the piece is a whole unit, else a partial state.
template <typename T, int D>
__device__ __forceinline__ void finish_piece(const TreeRun& r, const Walk& u, const f32x4 (&U)[D / 16], float R,
                                             float l, float* fold, float vscale) {
    constexpr int W = kTreeWaves, FROW = D + 4, NDB = D / 16;
    __shared__ float fold_r[W][16], fold_l[W][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, q = lane >> 4;
    l = quad_sum(l);
    __syncthreads();                                     // stages are dead, `fold` is their memory
#pragma unroll
    for (int i = 0; i < NDB; ++i)
        *reinterpret_cast<f32x4*>(&fold[(wave * 16 + col) * FROW + 16 * i + 4 * q]) = U[i];
    if (q == 0) {
        fold_r[wave][col] = R;
        fold_l[wave][col] = l;
    }
    __syncthreads();
    const bool whole = u.whole();
    const int G = (int)r.group.d;
    const int slot = 2 * (int)blockIdx.x + (u.blk0 == 0 ? 1 : 0);
    for (int idx = tid; idx < u.nrows * (D / 4); idx += W * kWave) {
        const int fr = idx / (D / 4);
        const int t = 4 * (idx % (D / 4));
        float top = fold_r[0][fr];
#pragma unroll
        for (int w = 1; w < W; ++w) top = fmaxf(top, fold_r[w][fr]);
        float lt = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            // a wavefront without a key of the row is left out (its U may hold 0 * infinity)
            const bool none = fold_l[w][fr] == 0.0f;
            const float f = none ? 0.0f : exp2_fast(fold_r[w][fr] - top);
            const f32x4 x = *reinterpret_cast<const f32x4*>(&fold[(w * 16 + fr) * FROW + t]);
            lt = fmaf(f, fold_l[w][fr], lt);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, none ? 0.0f : x[e], o[e]);
        }
        if (whole) {
            if (lt != 0.0f) o *= vscale / lt;
            const int rw = u.first + fr;
            const int tk = (int)fast_div((uint32_t)rw, r.group);
            Store<T>::store4(r.a.o, (size_t)(u.s.row0 + tk) * r.a.o_stride + (size_t)(u.h * G + rw - tk * G) * D + t,
                             {o[0], o[1], o[2], o[3]});
        } else {
            *reinterpret_cast<f32x4*>(r.parts + ((size_t)slot * kTreeRows + fr) * D + t) = o;
            if (t == 0) r.stats[slot * kTreeRows + fr] = float2{top, lt};
        }
    }
    if (u.blk0 == 0 && !whole && tid == 0) {
        TreeSplit sp;
        sp.row0 = u.s.row0;
        sp.h = u.h;
        sp.first = u.first;
        sp.rows = u.nrows;
        sp.parts = (int)((u.at + u.blocks - 1) / u.per) - (int)blockIdx.x + 1;
        sp.pad[0] = sp.pad[1] = sp.pad[2] = 0;
        r.splits[blockIdx.x] = sp;
    }
    __syncthreads();
}

// The pages of a wavefront's blocks blk0 + wave, + W, ...: looked up 32 blocks at a time, lane l for half
// l & 1 of block l / 2.  -1 where there is no page, or no key.
struct PageWindow {
    int pages, from;
    __device__ __forceinline__ int at(const Paged& c, const Walk& u, int wave, int lane, int blk, int half) {
        const int k = (blk - u.blk0) / kTreeWaves;
        if (k / 32 != from) {
            from = k / 32;
            const int mine = u.blk0 + wave + kTreeWaves * (32 * from + (lane >> 1));
            const int key = mine * kTreeBlock + 16 * (lane & 1);
            pages = -1;
            if (mine < u.blk1 && key < u.s.len + u.s.n) pages = page_at(c, u.b, key >> c.page_log2);
        }
        return __builtin_amdgcn_readlane(pages, 2 * (k & 31) + half);
    }
};

// 16 keys of a block: their bytes up to the sequence's last key, or nothing without a page.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t half_window(const Paged& c, const Walk& u, const char* pool,
                                                              int page, int key) {
    const int row = (int)(c.head_bytes >> c.page_log2);
    const char* at = pool + (int64_t)max(page, 0) * c.page_bytes + u.h * c.head_bytes +
                     (int64_t)(key & ((1 << c.page_log2) - 1)) * row;
    return kv_window(at, page < 0 ? 0 : (int64_t)min(16, u.s.len + u.s.n - key) * row);
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
// In blocks with new keys a weight of zero may meet a value that is infinite or NaN (a token that some rows see
// and others do not): 0 * infinity must not reach the others, so such blocks leave the matrix cores and
// add their visible keys one by one.

// any of 8 values of the storage type (16 fp8 values) is infinite or NaN
template <typename T, bool FP8>
__device__ __forceinline__ bool not_finite(u32x4 x) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FP8) {
            const uint32_t y = x[i] & 0x7f7f7f7fu;       // NaN is 0x7f: the only byte that adding 1 carries from
            bad |= ((y + 0x01010101u) & 0x80808080u) != 0;
        } else {
            constexpr uint32_t e = Mma<T>::kRoundedSum ? 0x7f80u : 0x7c00u;
            bad |= (x[i] & e) == e || (x[i] >> 16 & e) == e;
        }
    }
    return bad;
}

template <typename T> __device__ __forceinline__ float one_value(uint32_t half);
template <> __device__ __forceinline__ float one_value<BF16>(uint32_t half) { return __uint_as_float(half << 16); }
template <> __device__ __forceinline__ float one_value<F16>(uint32_t half) {
    return (float)__builtin_bit_cast(_Float16, (unsigned short)half);
}

template <typename T, int D, bool FP8>
__global__ __launch_bounds__(kTreeWaves * kWave, 2) void tree_rows_kernel(TreeRun r) {
    constexpr int W = kTreeWaves;
    constexpr int NKK = D / 32;
    constexpr int NDB = D / 16;
    constexpr int ESZ = FP8 ? 1 : 2;
    constexpr int NV = kTreeBlock * D * ESZ / 1024;      // 16-byte loads of K or V per lane and block
    constexpr int CPR = D * ESZ / 16;                    // 16-byte chunks per key row
    constexpr int KROW = D + 8;
    constexpr int VROW = D + 16;
    constexpr int STAGE = kTreeBlock * VROW;
    constexpr int FROW = D + 4;
    constexpr int kLds = 2 * W * STAGE > 4 * W * 16 * FROW ? 2 * W * STAGE : 4 * W * 16 * FROW;
    __shared__ __align__(16) char lds[kLds];

    const Paged& c = r.c;
    const TreeArgs& a = r.a;
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;
    const int q = lane >> 4;
    const int G = (int)r.group.d;
    const float ninf = -__builtin_inff();
    uint16_t* vs = reinterpret_cast<uint16_t*>(lds) + wave * STAGE;

    Walk u = begin_walk(c, G);
    if (tid == 0) r.splits[blockIdx.x].parts = 0;
    for (; u.next(c, G); u.done()) {
        // the query row of this lane's column; columns past the last row stand in for it
        const int row = u.first + min(col, u.nrows - 1);
        const int token = (int)fast_div((uint32_t)row, r.group);
        const int head = u.h * G + row - token * G;
        const uint16_t* qg = static_cast<const uint16_t*>(a.q) + (size_t)(u.s.row0 + token) * a.q_stride + (size_t)head * D;
        u32x4 qf[NKK];
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) qf[kk] = *reinterpret_cast<const u32x4*>(qg + 32 * kk + 8 * q);
        const float c_log2 = (FP8 ? a.scale * c.kscale : a.scale) * kLog2e;

        auto fetch = [&](const char* pool, u32x4 (&reg)[NV], int blk, int p0, int p1) __attribute__((always_inline)) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const auto w = half_window(c, u, pool, half ? p1 : p0, blk * kTreeBlock + 16 * half);
#pragma unroll
                for (int n = 0; n < NV / 2; ++n) reg[half * (NV / 2) + n] = kv_load<2>(w, 1024 * n + 16 * lane);
            }
        };
        auto stage = [&](const u32x4 (&reg)[NV], int ROW) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const int ch = n * kWave + lane;
                uint16_t* dst = &vs[(ch / CPR) * ROW + (FP8 ? 16 : 8) * (ch % CPR)];
                if constexpr (FP8) {
                    *reinterpret_cast<u32x4*>(dst) = widen8<T>(reg[n][0], reg[n][1]);
                    *reinterpret_cast<u32x4*>(dst + 8) = widen8<T>(reg[n][2], reg[n][3]);
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

        f32x4 U[NDB];
#pragma unroll
        for (int i = 0; i < NDB; ++i) U[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float R = ninf, l = 0.0f;

        PageWindow pages{-1, -1};
        u32x4 kreg[NV], vreg[NV];
        int p0 = -1, p1 = -1;
        int blk = u.blk0 + wave;
        if (blk < u.blk1) {
            p0 = pages.at(c, u, wave, lane, blk, 0);
            p1 = pages.at(c, u, wave, lane, blk, 1);
            fetch(c.k, kreg, blk, p0, p1);
            fetch(c.v, vreg, blk, p0, p1);
        }
        for (; blk < u.blk1; blk += W) {
            const int j0 = blk * kTreeBlock;
            const bool more = blk + W < u.blk1;
            // a half without a page, or behind the last key, has no keys
            const uint32_t have = (p0 < 0 ? 0u : 0x0000ffffu) | (p1 < 0 ? 0u : 0xffff0000u);
            int n0 = -1, n1 = -1;
            if (more) {
                n0 = pages.at(c, u, wave, lane, blk + W, 0);
                n1 = pages.at(c, u, wave, lane, blk + W, 1);
            }
            stage(kreg, KROW);
            if (more) fetch(c.k, kreg, blk + W, n0, n1);
            f32x4 acc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(&vs[(16 * t + col) * KROW + 32 * kk + 8 * q]);
                    acc[t] = Mma16<T>::mfma(x, qf[kk], acc[t]);
                }
            stage_done();
            stage(vreg, VROW);
            const bool masked = have != ~0u || j0 + kTreeBlock > u.s.len;
            bool apart = false;
            if (masked) {
#pragma unroll
                for (int n = 0; n < NV; ++n) apart |= not_finite<T, FP8>(vreg[n]);
                apart = __builtin_amdgcn_ballot_w64(apart) != 0;
            }
            if (more) fetch(c.v, vreg, blk + W, n0, n1);

            uint32_t bits = ~0u;
            if (masked) bits = have & seen_bits(a, u.s, token, u.s.row0 + token, j0);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = acc[e >> 2][e & 3] * c_log2;
                if (masked && !(bits >> (16 * (e >> 2) + 4 * q + (e & 3)) & 1u)) x[e] = ninf;
            }
            f32x8 pv;
            weigh(x, pv, U, R, l, LazyLimit<T>::kMoveLog2);
            const u32x4 bfrag = Mma<T>::pack8(pv);
            f32x4 ps = {0.0f, 0.0f, 0.0f, 0.0f};
            Mma<T>::sum8(pv, bfrag, ps);
            l += (ps[0] + ps[1]) + (ps[2] + ps[3]);

            if (!apart) {
                const uint16_t* base = &vs[(4 * q + (col >> 2)) * VROW + 4 * (col & 3)];
                typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
#pragma unroll
                for (int i = 0; i < NDB; ++i) {
                    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_ptr)(base + 16 * i)));
                    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_ptr)(base + 16 * VROW + 16 * i)));
                    U[i] = Mma16<T>::mfma(u32x4{lo[0], lo[1], hi[0], hi[1]}, bfrag, U[i]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float mine = one_value<T>(e & 1 ? bfrag[e >> 1] >> 16 : bfrag[e >> 1] & 0xffffu);
                    for (int k = 0; k < 4; ++k) {
                        const int j = 16 * (e >> 2) + 4 * k + (e & 3);
                        const float w = __shfl(mine, 16 * k + col);
                        const bool seen = (bits >> j & 1u) != 0;
#pragma unroll
                        for (int i = 0; i < NDB; ++i) {
                            const u32x2 y = *reinterpret_cast<const u32x2*>(&vs[j * VROW + 16 * i + 4 * q]);
#pragma unroll
                            for (int d = 0; d < 4; ++d) {
                                const float v = one_value<T>(d & 1 ? y[d >> 1] >> 16 : y[d >> 1] & 0xffffu);
                                U[i][d] = seen ? fmaf(w, v, U[i][d]) : U[i][d];
                            }
                        }
                    }
                }
            }
            stage_done();
            p0 = n0;
            p1 = n1;
        }
        finish_piece<T, D>(r, u, U, R, l, reinterpret_cast<float*>(lds), FP8 ? c.vscale : 1.0f);
    }
}

// ---- the same in fp32 ------------------------------------------------------------------------------
//
// v_mfma_f32_16x16x4_f32: lane (q, c) gives element q of the four that are summed, row (or column) c.  K as the A
// operand: the lane's float4 at dims 16 m + 4 q serves four products, each summing dims 16 m + 4 q' + e over
// q'.  The scores it gets are keys 4 q + r of its row: as B operand of O^T = V^T P^T product r sums
// the keys 4 q' + r over q', for which the lane's A element is V[4 q + r][16 i + c].  Nothing goes
// through LDS.
template <int D>
__global__ __launch_bounds__(kTreeWaves * kWave, 2) void tree_rows_f32_kernel(TreeRun r) {
    constexpr int W = kTreeWaves;
    constexpr int NDB = D / 16;
    __shared__ __align__(16) float fold[W * 16 * (D + 4)];

    const Paged& c = r.c;
    const TreeArgs& a = r.a;
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15;
    const int q = lane >> 4;
    const int G = (int)r.group.d;
    const float ninf = -__builtin_inff();

    Walk u = begin_walk(c, G);
    if (tid == 0) r.splits[blockIdx.x].parts = 0;
    for (; u.next(c, G); u.done()) {
        const int row = u.first + min(col, u.nrows - 1);
        const int token = (int)fast_div((uint32_t)row, r.group);
        const int head = u.h * G + row - token * G;
        const float* qg = static_cast<const float*>(a.q) + (size_t)(u.s.row0 + token) * a.q_stride + (size_t)head * D;
        f32x4 qf[NDB];
#pragma unroll
        for (int m = 0; m < NDB; ++m) qf[m] = *reinterpret_cast<const f32x4*>(qg + 16 * m + 4 * q);
        const float c_log2 = a.scale * kLog2e;

        f32x4 U[NDB];
#pragma unroll
        for (int i = 0; i < NDB; ++i) U[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float R = ninf, l = 0.0f;
        PageWindow pages{-1, -1};
        for (int blk = u.blk0 + wave; blk < u.blk1; blk += W) {
            const int j0 = blk * kTreeBlock;
            const int p[2] = {pages.at(c, u, wave, lane, blk, 0), pages.at(c, u, wave, lane, blk, 1)};
            const uint32_t have = (p[0] < 0 ? 0u : 0x0000ffffu) | (p[1] < 0 ? 0u : 0xffff0000u);
            f32x4 acc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                const auto w = half_window(c, u, c.k, p[t], j0 + 16 * t);
                f32x4 k[NDB];
#pragma unroll
                for (int m = 0; m < NDB; ++m) k[m] = __builtin_bit_cast(f32x4, kv_load<2>(w, (col * D + 16 * m + 4 * q) * 4));
#pragma unroll
                for (int m = 0; m < NDB; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[m][e], qf[m][e], acc[t], 0, 0, 0);
            }
            const bool masked = have != ~0u || j0 + kTreeBlock > u.s.len;
            uint32_t bits = ~0u;
            if (masked) bits = have & seen_bits(a, u.s, token, u.s.row0 + token, j0);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = acc[e >> 2][e & 3] * c_log2;
                if (masked && !(bits >> (16 * (e >> 2) + 4 * q + (e & 3)) & 1u)) x[e] = ninf;
            }
            f32x8 pv;
            weigh(x, pv, U, R, l, LazyLimit<BF16>::kMoveLog2);
            l += ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const auto w = half_window(c, u, c.v, p[e >> 2], j0 + 16 * (e >> 2));
                float v[NDB];
                bool bad = false;
#pragma unroll
                for (int i = 0; i < NDB; ++i) {
                    v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(w, ((4 * q + (e & 3)) * D + 16 * i + col) * 4, 0, 2));
                    bad |= !(fabsf(v[i]) <= 3.4028234e38f);
                }
                if (masked && __builtin_amdgcn_ballot_w64(bad) != 0) {
                    for (int k = 0; k < 4; ++k) {
                        const float wt = __shfl(pv[e], 16 * k + col);
                        const bool seen = (bits >> (16 * (e >> 2) + 4 * k + (e & 3)) & 1u) != 0;
#pragma unroll
                        for (int i = 0; i < NDB; ++i)
#pragma unroll
                            for (int d = 0; d < 4; ++d) {
                                const float y = __shfl(v[i], 16 * k + 4 * q + d);
                                U[i][d] = seen ? fmaf(wt, y, U[i][d]) : U[i][d];
                            }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < NDB; ++i)
                        U[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i], pv[e], U[i], 0, 0, 0);
                }
            }
        }
        finish_piece<F32, D>(r, u, U, R, l, fold, 1.0f);
    }
}

// ---- join the parts of split units -------------------------------------------------------------
//
// Workgroup (w, y) joins rows y, y + gridDim.y, ... of the unit that began in workgroup w and went on
// in others: D / 4 lanes take 4 columns each, 1024 / D groups of lanes share the parts.
template <typename T, int D>
__global__ __launch_bounds__(256) void merge_tree_kernel(TreeRun r, float vscale) {
    constexpr int LPR = D / 4;
    constexpr int NG = 256 / LPR;
    __shared__ __align__(16) float sum[NG][D];
    __shared__ float2 part_stat[NG];
    const TreeSplit sp = r.splits[blockIdx.x];
    if (sp.parts == 0) return;
    const int g = threadIdx.x / LPR, t = 4 * (threadIdx.x % LPR);
    const int G = (int)r.group.d;
    const float ninf = -__builtin_inff();
    for (int fr = blockIdx.y; fr < sp.rows; fr += gridDim.y) {
        float top = ninf, lt = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = g; k < sp.parts; k += NG) {
            const size_t at = (size_t)(2 * ((int)blockIdx.x + k) + (k == 0 ? 1 : 0)) * kTreeRows + fr;
            const float2 st = r.stats[at];
            if (st.y == 0.0f) continue;                  // no key of this row
            const f32x4 u = *reinterpret_cast<const f32x4*>(r.parts + at * D + t);
            const float now = fmaxf(top, st.x);
            const float f0 = top == ninf ? 0.0f : exp2_fast(top - now), f1 = exp2_fast(st.x - now);
            lt = fmaf(lt, f0, st.y * f1);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], f0, u[e] * f1);
            top = now;
        }
        __syncthreads();
        *reinterpret_cast<f32x4*>(&sum[g][t]) = o;
        if (t == 0) part_stat[g] = float2{top, lt};
        __syncthreads();
        if (g == 0) {
            float all = ninf;
#pragma unroll
            for (int k = 0; k < NG; ++k) all = fmaxf(all, part_stat[k].x);
            lt = 0.0f;
            o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const float2 st = part_stat[k];
                const float f = st.y == 0.0f ? 0.0f : exp2_fast(st.x - all);
                const f32x4 u = *reinterpret_cast<const f32x4*>(&sum[k][t]);
                lt = fmaf(f, st.y, lt);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(f, u[e], o[e]);
            }
            if (lt != 0.0f) o *= vscale / lt;
            const int rw = sp.first + fr;
            const int tk = (int)fast_div((uint32_t)rw, r.group);
            Store<T>::store4(r.a.o, (size_t)(sp.row0 + tk) * r.a.o_stride + (size_t)(sp.h * G + rw - tk * G) * D + t,
                             {o[0], o[1], o[2], o[3]});
        }
    }
}

size_t attn_tree_workspace(int Hq, int Hkv, int max_q, int d, int dtype) {
    (void)Hq; (void)Hkv; (void)max_q; (void)dtype;
    return (size_t)2 * kTreeMostGroups * kTreeRows * (d + 2) * sizeof(float) + kTreeMostGroups * sizeof(TreeSplit);
}

template <typename T, int D>
static hipError_t launch_tree_t(TreeRun& r, hipStream_t st) {
    const dim3 grid(kTreeMostGroups), block(kTreeWaves * kWave);
    if constexpr (std::is_same_v<T, F32>) {
        hipLaunchKernelGGL((tree_rows_f32_kernel<D>), grid, block, 0, st, r);
    } else {
        if (r.a.fp8) hipLaunchKernelGGL((tree_rows_kernel<T, D, true>), grid, block, 0, st, r);
        else hipLaunchKernelGGL((tree_rows_kernel<T, D, false>), grid, block, 0, st, r);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((merge_tree_kernel<T, D>), dim3(kTreeMostGroups, 4), dim3(256), 0, st, r,
                       r.a.fp8 ? r.c.vscale : 1.0f);
    return hipGetLastError();
}

hipError_t launch_attn_tree(const Paged& c, const TreeArgs& a, hipStream_t st) {
    TreeRun r;
    r.c = c;
    r.a = a;
    r.group = make_fast_div((uint32_t)(a.Hq / c.Hkv));
    r.parts = a.ws;
    r.stats = reinterpret_cast<float2*>(a.ws + (size_t)2 * kTreeMostGroups * kTreeRows * c.d);
    r.splits = reinterpret_cast<TreeSplit*>(r.stats + (size_t)2 * kTreeMostGroups * kTreeRows);
    const bool small = c.d == 64;
    if (a.dtype == 0) return small ? launch_tree_t<F32, 64>(r, st) : launch_tree_t<F32, 128>(r, st);
    if (a.dtype == 1) return small ? launch_tree_t<F16, 64>(r, st) : launch_tree_t<F16, 128>(r, st);
    return small ? launch_tree_t<BF16, 64>(r, st) : launch_tree_t<BF16, 128>(r, st);
}

}  // namespace flashd
