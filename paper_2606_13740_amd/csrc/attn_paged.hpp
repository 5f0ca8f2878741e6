// Attention of a batch of sequences that share a prefix, over a paged cache.
//
// For a row and head, o = sum_j p_j v_j / sum_j p_j with p_j = 2^(s_j - m), s_j the score in
// log2 units and m any reference near the row's maximum: one pass over the keys keeps (m, sum,
// o) and rescales when m moves.  (m, sum, o) of disjoint key sets merge the same way, so the
// keys are cut into parts that run side by side and a second kernel merges:
//   - the shared prefix, once for the rows of ALL sequences: its K/V tiles meet as many rows as
//     there are, and it is read from HBM once (rows of one sequence alone would leave a
//     32-row window at 16 flops a byte);
//   - each sequence's own keys, for its own rows.
// Both may be split further along the keys where the tiles alone do not fill the chip.
//
// Rows of the query heads of one K/V head are packed together: "virtual row" f = row * G + g
// of a K/V head (G query heads each), so that grouped heads share K/V tiles too.
//
// Products, transposed so that no operand is shuffled (16 x 16 MFMA tiles):
//   S^T (16 keys x 16 rows) = K tile (A) * Q^T (B),   O^T (16 dims x 16 rows) += V^T tile (A) * P^T (B).
//   16-bit types, 32 keys a step: key tile t takes keys 8 (r / 4) + 4 t + r % 4, so that lane group g ends
//   up with the probabilities of keys 8g .. 8g+7, which is the B operand of a 32-key product.
//   16-bit types, 32 x 32 tiles (16 deep): key tile row m takes key 16 (m / 16) + 8 (m / 4 % 2) + 4 (m / 8 %
//   2) + m % 4; a lane's 16 scores are then keys 16 j + 8g .. + 7 for j = 0, 1, the operands of
//   two 16-key products.
//   fp32 (4 keys a product): key tile t takes keys 16 t + r; lane group g has keys 16 t + 4g + i and
//   product i takes exactly key i of every group.  Dims of a 16-dim step go 4g + i the same way.
#pragma once

#include "batch_rules.hpp"
#include "common.hpp"
#include "qk_rope.hpp"

namespace dllm {

struct PagedArgs {
    const void* q;
    long ld_q;
    const void *kp, *vp;          // [n_pages][Hk][page][Dh], [n_pages][Hk][Dh][page]
    const int* table;
    int table_ld;
    const int *row0, *len, *lim;
    void* out;
    long ld_out;
    int T, B, H, Hk, G, page_shift, n_pages, shared, max_rows, max_len;
    float sl2;                    // |scale| * log2(e)
    float qmul;                   // sign of the scale (0: all scores are 0)
    int ns_s, ns_o;               // key splits of the shared part and of a sequence's own
    int nt_s, nt_o;               // row tiles of the shared part and of a sequence
    int n_s;                      // workgroups of the shared part (the first ones)
    int direct;                   // one part in all: the output is written here, not merged
    int out_f32;                  // out holds floats whatever T is (a batch step's, for the O projection's operand)
    const uint32_t* mask;         // [T][mask_ld]: which of its sequence's rows a row sees (TREE)
    int mask_ld;
    float* opart;                 // [ns_s + ns_o][T][H][Dh] unnormalised partial outputs
    float* mlpart;                // [ns_s + ns_o][T][H][2]  (reference in log2 units, sum)
};

// Largest b with row0[b] <= r, or -1 where r is no row of a sequence.
__device__ __forceinline__ int row_seq(const int* row0, int B, int r) {
    if (r < row0[0] || r >= row0[B]) return -1;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row0[mid] <= r) lo = mid;
        else hi = mid;
    }
    return lo;
}

// First position of sequence b that one of the call's rows has; those before it are cached.
__device__ __forceinline__ int seq_base(const PagedArgs& a, int b) {
    const RowRange n = row_range(a.row0[b], a.row0[b + 1], a.T, a.T);
    return max(a.len[b], 0) - (n.end - n.begin);
}
// The 32 bits of a row's mask from bit t on, w0 and w1 what stands at the words t / 32 and behind it (as far as there are ld):
// the cached positions before the mask count as set bits, what lies past it as none.
__device__ __forceinline__ uint32_t mask_bits(uint32_t w0, uint32_t w1, int t, int ld) {
    const int i = t >> 5;
    w0 = i < 0 ? 0xFFFFFFFFu : (i < ld ? w0 : 0u);
    w1 = i < -1 ? 0xFFFFFFFFu : (i + 1 < ld ? w1 : 0u);
    return __builtin_amdgcn_alignbit(w1, w0, t & 31);
}

// Item L of the sequences' own parts in a call with masks (b = -1: none), for tiles of tm virtual rows.  Sequences
// differ in their rows, and items without any must not stand between the others: the dispatcher deals workgroups to the
// shader engines in turn and waits for one that is full, so that short-lived ones leave CUs unevenly filled, and
// workgroups that would all have fitted start when the first have ended (16 trees of up to 64 rows, 28 heads over 4,
// behind 8192 + 3000, the shared part in three: 142 us, 108 so).  Where there is more than one tile a sequence, the tiles
// that have rows are counted (a wave's scan over the sequences, for up to 256 of them) and dealt as if there were no
// others, XCD x taking the x-th share of (head, split, sequence, tile), which is the same number for each.
// Otherwise the groups (sequence, head, split) go to the XCDs in turn, first tiles first.
struct TreeItem {
    int b, tile, split, hk;
};
constexpr int TREE_SCAN = 256;
__device__ __forceinline__ TreeItem tree_item(const PagedArgs& a, int tm, int L, int n_items) {
    const int xcd = L & 7, k = L >> 3, lane = threadIdx.x & 63;
    if (a.nt_o == 1 || a.B > TREE_SCAN) {
        const int groups = (n_items >> 3) / a.nt_o, tile = k / groups, i1 = xcd + 8 * (k - tile * groups);
        if (i1 >= a.B * a.Hk * a.ns_o) return TreeItem{-1, 0, 0, 0};
        const int i2 = i1 / a.ns_o;
        return TreeItem{i2 / a.Hk, tile, i1 % a.ns_o, i2 % a.Hk};
    }
    constexpr int PER = TREE_SCAN / 64;
    int at[PER + 1], tiles[PER], sum = 0;
#pragma unroll
    for (int i = 0; i <= PER; ++i) at[i] = a.row0[min(PER * lane + i, a.B)];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const RowRange n = row_range(at[i], at[i + 1], a.max_rows, a.T);
        tiles[i] = PER * lane + i < a.B ? ((n.end - n.begin) * a.G + tm - 1) / tm : 0;
        sum += tiles[i];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(inc, o);
        inc += lane >= o ? up : 0;
    }
    const int R = __builtin_amdgcn_readlane(inc, 63), N = R * a.Hk * a.ns_o;      // (N <= n_items)
    const int i = xcd * (N >> 3) + min(xcd, N & 7) + k;
    if (k >= (N >> 3) + (xcd < (N & 7))) return TreeItem{-1, 0, 0, 0};
    const int u = i / R, r = i - u * R;
    const int ln = __builtin_ctzll(__builtin_amdgcn_ballot_w64(inc > r));
    int tile = r - (__builtin_amdgcn_readlane(inc, ln) - __builtin_amdgcn_readlane(sum, ln)), b = PER * ln;
#pragma unroll
    for (int j = 0; j < PER - 1; ++j) {
        const int n = __builtin_amdgcn_readlane(tiles[j], ln);
        if (b == PER * ln + j && tile >= n) {
            tile -= n;
            ++b;
        }
    }
    return TreeItem{b, tile, u % a.ns_o, u / a.ns_o};
}

// Element type: one product step of a 16 x 16 or 32 x 32 tile (with 16-bit types 32 or 16 deep).
typedef float f32x16_t __attribute__((ext_vector_type(16)));
template <int RT> struct PagedAcc { using type = f32x4_t; };
template <> struct PagedAcc<32> { using type = f32x16_t; };
template <typename T> struct PagedElem;
template <> struct PagedElem<_Float16> {
    template <int RT> using Acc = typename PagedAcc<RT>::type;
    using x2 = _Float16 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x4_t mfma(const u32x4_t& a, const u32x4_t& b, f32x4_t c) { return mfma_f16(a, b, c); }
    static __device__ __forceinline__ f32x16_t mfma(const u32x4_t& a, const u32x4_t& b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
};
template <> struct PagedElem<__bf16> {
    template <int RT> using Acc = typename PagedAcc<RT>::type;
    using x2 = __bf16 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x4_t mfma(const u32x4_t& a, const u32x4_t& b, f32x4_t c) { return mfma_bf16(a, b, c); }
    static __device__ __forceinline__ f32x16_t mfma(const u32x4_t& a, const u32x4_t& b, f32x16_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
};
template <> struct PagedElem<float> {
    template <int RT> using Acc = typename PagedAcc<RT>::type;
    using x2 = float __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x4_t mfma(const u32x4_t& a, const u32x4_t& b, f32x4_t c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = mfma_f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c);
        return c;
    }
};

// Swizzles of a block's LDS rows (16-byte columns): the 16 lanes of one LDS cycle of a 16-byte read, which are
// lanes 0-7 and 16-23 (and so on), read distinct banks.
__device__ __forceinline__ int swz_paged(int key) { return (key & 3) | (((key >> 3) & 3) << 2); }
template <bool F32, int RT> __device__ __forceinline__ int swz_v(int dim) {
    return F32 ? dim & 7 : (RT == 32 ? ((dim >> 1) & 3) ^ ((dim >> 4) & 1) : (dim >> 1) & 3);
}

// Classes of V's elements, in the element type: what is not finite, so that sums of up to 64 of them tell
// which there are (0, 1 a +inf, 128 a -inf, 16384 a NaN: exact in every type and in an fp32 sum).
template <typename T> struct PagedClass;
template <> struct PagedClass<_Float16> { static constexpr uint32_t exp = 0x7C00u, one = 0x3C00u, c128 = 0x5800u, c16384 = 0x7400u; };
template <> struct PagedClass<__bf16> { static constexpr uint32_t exp = 0x7F80u, one = 0x3F80u, c128 = 0x4300u, c16384 = 0x4680u; };
template <> struct PagedClass<float> { static constexpr uint32_t exp = 0x7F800000u, one = 0x3F800000u, c128 = 0x43000000u, c16384 = 0x46800000u; };
// f of every element's bits
template <typename T, typename F> __device__ __forceinline__ u32x4_t map_elems(const u32x4_t& v, F f) {
    u32x4_t out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = sizeof(T) == 4 ? f(v[i]) : f(v[i] & 0xFFFFu) | (f(v[i] >> 16) << 16);
    return out;
}
template <typename T> __device__ __forceinline__ u32x4_t finite_or_zero(const u32x4_t& v) {
    return map_elems<T>(v, [](uint32_t e) { return (e & PagedClass<T>::exp) == PagedClass<T>::exp ? 0u : e; });
}
template <typename T> __device__ __forceinline__ u32x4_t class_of(const u32x4_t& v) {
    using C = PagedClass<T>;
    constexpr uint32_t sign = sizeof(T) == 4 ? 0x80000000u : 0x8000u;
    return map_elems<T>(v, [](uint32_t e) {
        const uint32_t inf = (e & sign) != 0 ? C::c128 : C::one, nan = (e & (C::exp ^ (sign - 1))) != 0 ? C::c16384 : inf;
        return (e & C::exp) == C::exp ? nan : 0u;
    });
}
template <typename T> __device__ __forceinline__ bool any_odd(const u32x4_t& v) {
    const u32x4_t c = v ^ finite_or_zero<T>(v);
    return (c[0] | c[1] | c[2] | c[3]) != 0;
}
// o with a sum of classes added
__device__ __forceinline__ float add_classes(float o, float c) {
    const int n = (int)c, pos = n & 127, neg = (n >> 7) & 127;
    if (n >= 16384 || (pos && neg)) return __builtin_nanf("");
    return pos ? o + INFINITY : (neg ? o - INFINITY : o);
}

// An output: finite sums saturate in fp16 (rounded probabilities can carry a mean of values near the largest past
// it), infinities stay.
template <typename T> __device__ __forceinline__ T attn_out(float o) {
    return __builtin_fabsf(o) == INFINITY ? (T)o : elem_from_f32<T>(o);
}

// log2-domain slack of the lazily moved reference: probabilities <= 2^8 (fits fp16)
constexpr float PAGED_SLACK = 8.f;

// Four consecutive outputs from element `at` of a.out on.
template <typename T> __device__ __forceinline__ void store_out4(const PagedArgs& a, size_t at, const float (&o)[4]) {
    if (sizeof(T) == 4 || a.out_f32) {
        *(float4*)((float*)a.out + at) = make_float4(o[0], o[1], o[2], o[3]);
    } else {
        T e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = attn_out<T>(o[i]);
        __builtin_memcpy(__builtin_assume_aligned((T*)a.out + at, 4 * sizeof(T)), e, sizeof(e));
    }
}

// Workgroup = (part, K/V head, key split, tile of QG x RT virtual rows): QG row tiles of KG waves each.
// A step is SUB blocks of 32 keys, which direct global->LDS loads stage in one of two buffers while
// the other is read; a row tile's waves take SUB / KG of the blocks each and join at the end.
// LDS rows are swizzled in 16-byte columns so that the lanes of an LDS cycle read distinct banks (no conflicts
// counted in either tile's loop).  Lane i holds the page of block 64 n + i, so a block's page is one lane read.
//
// What bounds it: many rows, the chain of products and exponentials of the two waves that a SIMD holds
// (16 sequences of 64 rows, 28 heads over 4, behind 16384 bf16 keys: 145-153 us with the merge, 850 to 900
// TFLOP/s where a large library product reaches 1100; waiting 22% of the wave cycles); rows enough for the prefix only, LDS reads and the K/V
// themselves (8 x 32 rows of 32 fp16 heads behind 4096: 46 us with the merge, 115 MB); few rows, latency (8 x 1 rows
// behind 1564: 9.8 us and 4.8, 288 workgroups of three steps, each asked for when the one before has landed).
//
// TREE: a row sees the cached positions and, of its sequence's rows, those that its mask has.  Steps whose keys are all
// cached run as without; in the others a lane takes the 32 bits of its row for a block from two words, which come to LDS
// beside the step's K/V (a load waited for inside a step would wait for the staging behind it).  What a lane needs for
// that waits in LDS too: kept in registers, the 32 x 32 tiles spilled three, and a spill's reload waits for the staging
// in every step.  Of a SIMD's two waves the one that reads and multiplies goes before the one in its exponentials: 98 us
// for 105 below, 260 for 281 with full trees behind 16384, at worst 1% (the paged calls' long case loses 3%, so not there).
// 16 trees of up to 64 rows, 28 heads over 4, behind 8192 + 3000 bf16 keys: 98 us with the merge, 740 TFLOP/s;
// 4 x 4 candidates of 32 rows, 32 fp16 heads, behind 4000: 73 us, of which the parts take 64, 270 MB of K/V at 4.2 TB/s where a
// plain read has 6.5: the waves are ready and wait to issue for 44% of their cycles, and wait for data for 29%.
template <typename T, int DH, int QG, int RT, int KG, int SUB, bool TREE>
__global__ void __launch_bounds__(QG * KG * 64)
__attribute__((amdgpu_waves_per_eu(QG * KG * (160 * 1024 / (2 * SUB * 64 * DH * (int)sizeof(T))) >= 8 ? 2 : 1)))
attn_paged_kernel(PagedArgs a) {
    using E = PagedElem<T>;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int ES = sizeof(T);
    constexpr bool R32 = RT == 32;
    constexpr int NG = 64 / RT;               // lane groups of RT lanes
    constexpr int CD = 16 / ES * NG;          // dims of one 16-byte K fragment step
    constexpr int NC = DH / CD;
    constexpr int NU = 32 / RT;               // key tiles of a block
    constexpr int NS = RT / 2;                // scores of a block per lane
    constexpr int ND = DH / RT;               // output tiles
    constexpr int NV = F32 || R32 ? 2 : 1;    // V^T fragments of a block per output tile
    using Acc = typename E::template Acc<RT>;
    constexpr int NA = RT * RT / 64;          // accumulators of a tile per lane
    constexpr int KC = DH * ES / 16;          // 16-byte columns of a key's row
    constexpr int VC = 32 * ES / 16;          // and of a dim's row of V^T
    constexpr int KPLANE = 32 * DH * ES, SBUF = 2 * KPLANE, BUF = SUB * SBUF;
    constexpr int KI = KPLANE / 1024;         // 1 KiB wave loads per plane
    constexpr int NW = QG * KG;               // waves
    constexpr int SW = SUB / KG;              // blocks of a step per wave
    static_assert(64 % SUB == 0 && SUB % KG == 0, "a step's pages lie in one chunk, its blocks are dealt evenly");
    constexpr int TM = RT * QG;               // virtual rows of a workgroup
    static_assert(KI * 1024 == KPLANE, "planes must be whole wave loads");
    static_assert(TM <= 256, "at most four virtual rows per lane");
    __shared__ __attribute__((aligned(1024))) char lds[2 * BUF];
    __shared__ uint32_t words_s[TREE ? 2 * NW * (SW + 1) * 64 : 1];      // [step & 1][wave][word][lane]
    __shared__ int lane_s[TREE ? NW * 3 * 64 : 1];                       // [wave]: limit, first masked key, mask row

    const int lane = threadIdx.x & 63, wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qw = wave % QG, kw = wave / QG;  // row tile, and the step's blocks that are this wave's
    const int r = lane % RT, g = lane / RT;

    // Which item.  The dispatcher deals consecutive workgroups to the 8 XCDs in turn; XCD x
    // takes the x-th of 8 shares, so that tiles that read the same K/V share one L2.
    const bool own = (int)blockIdx.x >= a.n_s;
    const int n_items = own ? (int)gridDim.x - a.n_s : a.n_s;
    const int L = (int)blockIdx.x - (own ? a.n_s : 0), xcd = L & 7;
    const int item = xcd * (n_items >> 3) + min(xcd, n_items & 7) + (L >> 3);
    int tile, split, hk, b, ks, ke, first, behind, most_rows, bps, part, base_own = 0;
    if (own) {
        if (TREE) {
            const TreeItem it = tree_item(a, TM, L, n_items);
            if (it.b < 0) return;
            tile = it.tile;
            split = it.split;
            hk = it.hk;
            b = it.b;
        } else {
            tile = item % a.nt_o;
            const int i1 = item / a.nt_o, i2 = i1 / a.ns_o;
            split = i1 % a.ns_o;
            hk = i2 % a.Hk;
            b = i2 / a.Hk;
        }
        first = a.row0[b];
        behind = a.row0[b + 1];
        most_rows = a.max_rows;
        ks = a.shared;
        ke = min(max(a.len[b], 0), a.max_len);
        // steps per split from the sequence's own length: a short one is still spread
        const int nst = (max(0, ke - ks) + 32 * SUB - 1) / (32 * SUB);
        bps = (nst + a.ns_o - 1) / a.ns_o;
        part = a.ns_s + split;
        if constexpr (TREE) base_own = seq_base(a, b);
    } else {
        tile = item % a.nt_s;
        const int i1 = item / a.nt_s;
        split = i1 % a.ns_s;
        hk = i1 / a.ns_s;
        b = 0;
        first = a.row0[0];
        behind = a.row0[a.B];
        most_rows = a.T;
        ks = 0;
        ke = min(a.shared, a.max_len);
        bps = ((ke + 32 * SUB - 1) / (32 * SUB) + a.ns_s - 1) / a.ns_s;
        part = split;
    }
    const int kb0 = SUB * split * bps;        // the split's first 32-key block

    // Pages of the 64 blocks of a chunk: lane i has block 64 n + i's (-1: no page), and `have` a
    // bit a block.  The first chunk, and with it the first step's K/V, is asked for before the
    // rows and their limits are known (a table row has table_ld entries whatever the length).
    const int* trow = a.table + (size_t)b * a.table_ld;
    auto chunk_pages = [&](int n) {
        const int pg = trow[min((ks + 32 * (kb0 + 64 * n + lane)) >> a.page_shift, a.table_ld - 1)];
        return pg < a.n_pages ? pg : -1;
    };
    int pgv = chunk_pages(0);
    const long page_elems = (long)DH << a.page_shift;
    const RowRange rows = row_range(first, behind, most_rows, a.T);
    const int R0 = rows.begin, R1 = rows.end;
    const int nv = (R1 - R0) * a.G;           // virtual rows of the part (n_rows * G fits 32 bits)
    const int f0 = tile * TM;
    if (f0 >= nv) return;

    // Stage step t: wave load i of a plane is its bytes [1024 i, 1024 i + 1024), taken by wave
    // i % NW.  A block without a page is staged from page 0 (and not used).
    auto stage = [&](int t, int buf) {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            const int blk = SUB * t + u;
            const int pg = max(0, __builtin_amdgcn_readlane(pgv, blk & 63));
            const int off = (ks + 32 * (kb0 + blk)) & ((1 << a.page_shift) - 1);
            const long head = ((long)pg * a.Hk + hk) * page_elems;
            const T* Kp = (const T*)a.kp + head;
            const T* Vp = (const T*)a.vp + head;
            char* base = lds + buf * BUF + u * SBUF;
#pragma unroll
            for (int j = 0; j < (KI + NW - 1) / NW; ++j) {
                const int i = wave + j * NW;
                if (KI % NW != 0 && i >= KI) break;
                const int key = (i * 64 + lane) / KC, pc = lane % KC;
                const int sw = F32 ? key & 15 : swz_paged(key);
                buffer_to_lds16(Kp, key * (DH * ES) + ((pc ^ (sw & (KC - 1))) << 4), off * (DH * ES), base + i * 1024);
            }
#pragma unroll
            for (int j = 0; j < (KI + NW - 1) / NW; ++j) {
                const int i = wave + j * NW;
                if (KI % NW != 0 && i >= KI) break;
                const int dim = (i * 64 + lane) / VC, pc = lane % VC;
                const int sw = swz_v<F32, RT>(dim);
                buffer_to_lds16(Vp, ((dim << a.page_shift) * ES) + ((pc ^ sw) << 4), off * ES, base + KPLANE + i * 1024);
            }
        }
    };
    // In the slots of a block that this wave staged, zeroes for the V^T values of keys >= end, and for the
    // infinities and NaNs of those from kz on: a key that one row of the workgroup sees and another
    // does not, whose probability of 0 would not silence them.  Returns whether there were any.
    auto clean_tail = [&](int k0, int end, int kz, char* sub) {
        bool any = false;
        char* base = sub + KPLANE;
#pragma unroll
        for (int j = 0; j < (KI + NW - 1) / NW; ++j) {
            const int i = wave + j * NW;
            if (KI % NW != 0 && i >= KI) break;
            const int dim = (i * 64 + lane) / VC, pc = lane % VC;
            const int sw = swz_v<F32, RT>(dim);
            const int key = k0 + (16 / ES) * (pc ^ sw);             // the slot's first key
            if (key + 16 / ES <= end && key < kz) continue;
            u32x4_t* slot = (u32x4_t*)(base + i * 1024 + lane * 16);
            u32x4_t v = *slot;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (F32) v[e] = key + e >= end ? 0u : v[e];
                else v[e] &= (key + 2 * e >= end ? 0u : 0x0000FFFFu) | (key + 2 * e + 1 >= end ? 0u : 0xFFFF0000u);
            }
            if (key >= kz) {
                any |= any_odd<T>(v);
                v = finite_or_zero<T>(v);
            }
            *slot = v;
        }
        return __builtin_amdgcn_ballot_w64(any);
    };

    const int most = min(SUB * bps, ((ke - ks + 31) >> 5) - kb0);      // blocks of the split, at most
    if (most > 0) stage(0, 0);

    // Key limit of virtual row f.  The rows of the shared part need their sequence's length only if some
    // sequence ends inside it.
    int short_len = 0x7FFFFFFF;
    if (!own) {
        for (int i = lane; i < a.B; i += 64) short_len = min(short_len, TREE ? seq_base(a, i) : a.len[i]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) short_len = min(short_len, __shfl_xor(short_len, o));
    }
    auto row_limit = [&](int f) {
        const int row = R0 + f / a.G;
        const int n = own || short_len >= ke ? ke : min(ke, a.len[row_seq(a.row0, a.B, row)]);
        return a.lim != nullptr ? min(n, a.lim[row]) : n;
    };
    // (TREE: short_len is the least number of cached positions) the first key of virtual row f that its mask decides
    auto row_low = [&](int f) {
        return own ? base_own : (short_len >= ke ? ke : seq_base(a, row_seq(a.row0, a.B, R0 + f / a.G)));
    };
    u32x4_t qf[NC];
    int lim, low = 0;
    int* mine = lane_s + (TREE ? wave * 3 * 64 + lane : 0);
    {
        // rows past the last repeat it (the rescale below is decided over a tile's rows)
        const int f = min(f0 + RT * qw + r, nv - 1);
        const int row = R0 + f / a.G, h = hk * a.G + f % a.G;
        const T* src = (const T*)a.q + row * a.ld_q + h * DH + (16 / ES) * g;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            qf[c] = ldg16(src + CD * c);
            if (a.qmul != 1.f) {
                constexpr uint32_t sign = F32 ? 0x80000000u : 0x80008000u;
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[c][e] = a.qmul == 0.f ? 0u : qf[c][e] ^ sign;
            }
        }
        lim = row_limit(f);
        if constexpr (TREE) {
            low = row_low(f);
            mine[0] = lim;
            mine[64] = low;
            mine[128] = row * a.mask_ld;               // (n_rows * mask_ld < 2^29)
        }
    }
    // The largest limit of the tile's rows ends its keys: what lies behind may be anything.  Keys from the
    // smallest on (kz: its 16-byte slot of V^T) are seen by some rows only.
    int ktop = ks, lim_lo;
    if (a.lim == nullptr && (own || short_len >= ke)) {
        lim_lo = ktop = max(ks, ke);
        if constexpr (TREE) {
            if (own) lim_lo = min(ktop, max(ks, base_own));
        }
    } else {
        lim_lo = 0x7FFFFFFF;
#pragma unroll
        for (int i = 0; i < (TM + 63) / 64; ++i) {
            const int f = min(f0 + (TM < 64 ? lane % TM : lane) + 64 * i, nv - 1), n = row_limit(f);
            ktop = max(ktop, n);
            lim_lo = min(lim_lo, TREE ? min(n, row_low(f)) : n);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            ktop = max(ktop, __shfl_xor(ktop, o));
            lim_lo = min(lim_lo, __shfl_xor(lim_lo, o));
        }
        ktop = __builtin_amdgcn_readfirstlane(ktop);
        lim_lo = min(ktop, max(ks, __builtin_amdgcn_readfirstlane(lim_lo)));
    }
    const int kz = lim_lo == ktop ? 0x7FFFFFFF : lim_lo & ~(16 / ES - 1);
    const int blocks = max(0, min((ktop - ks + 31) >> 5, kb0 + SUB * bps) - kb0);
    const int rounds = (blocks + SUB - 1) / SUB;
    auto chunk_have = [&](int n) { return __builtin_amdgcn_ballot_w64(pgv >= 0 && 64 * n + lane < blocks); };
    uint64_t have = chunk_have(0);

    // smallest limit of the wave's rows (or first key that a mask decides): blocks below it need no per-key mask
    int lim_w = ktop;
    const int lim_m = TREE ? min(lim, low) : lim;
#pragma unroll
    for (int i = 0; i < RT; ++i) lim_w = min(lim_w, __builtin_amdgcn_readlane(lim_m, i));

    // the mask words of this wave's blocks of step t
    auto first_key = [&](int t) { return ks + 32 * (kb0 + SUB * t + kw * SW); };
    auto words_of = [&](int t) { return words_s + ((t & 1) * NW + wave) * (SW + 1) * 64; };
    auto load_words = [&](int t) {
        if (first_key(t) + 32 * SW <= lim_w) return;
        const int i = (first_key(t) - mine[64]) >> 5, at = mine[128];
#pragma unroll
        for (int w = 0; w <= SW; ++w)
            buffer_to_lds4(a.mask, (at + min(max(i + w, 0), a.mask_ld - 1)) * 4, 0, (char*)(words_of(t) + 64 * w));
    };
    if (TREE && rounds > 0) load_words(0);

    float mrun = -INFINITY, lrun = 0.f;
    Acc oacc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < NA; ++i) oacc[dt][i] = 0.f;
    // the key that this lane reads for key tile u, and the key of its score e (see above)
    auto krow = [&](int u) {
        if constexpr (R32) return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
        else return F32 ? r + 16 * u : 8 * (r >> 2) + (r & 3) + 4 * u;
    };
    auto key_of = [&](int e) {
        if constexpr (R32) return 16 * (e >> 3) + 8 * g + (e & 7);
        else return F32 ? 16 * (e >> 2) + 4 * g + (e & 3) : 8 * g + e;
    };

    // no load outstanding past here: the compiler does not see the waits in the loop's asm and would wait again at
    // each use: for all LDS reads where a scalar load could be left, and, for Q's loads, in every step until the step's own
    // staging has landed
    __builtin_amdgcn_s_waitcnt(0x0070);
    uint64_t odd = 0;
    // a wave without rows of its own only stages
    const bool busy = f0 + RT * qw < nv;
    for (int t = 0; t < rounds; ++t) {
        const int k0 = ks + 32 * (kb0 + SUB * t), k0w = k0 + 32 * kw * SW;
        char* cur = lds + (t & 1) * BUF;
        const uint32_t there = (uint32_t)(have >> ((SUB * t) & 63)) & ((1u << SUB) - 1);      // which blocks have a page
        const bool whole = there == (1u << SUB) - 1;
        // This wave's loads of step t have landed; the barrier makes every wave's visible and frees the buffer
        // that round t - 1 read, for step t + 1.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (!whole || k0 + 32 * SUB > lim_lo) {
#pragma unroll
            for (int u = 0; u < SUB; ++u)
                odd |= clean_tail(k0 + 32 * u, (there >> u) & 1 ? ktop : 0, kz, cur + u * SBUF);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + 1 < rounds) {
            if (((SUB * (t + 1)) & 63) == 0) {
                pgv = chunk_pages((SUB * (t + 1)) >> 6);
                have = chunk_have((SUB * (t + 1)) >> 6);
            }
            stage(t + 1, (t + 1) & 1);
            if constexpr (TREE) load_words(t + 1);
        }
        if (!busy) continue;

        // all of the step's K fragments are read before the first product, its V^T fragments between
        // the scores and the softmax, which covers their latency
        if constexpr (TREE) __builtin_amdgcn_s_setprio(2);
        const char* buf = cur + kw * SW * SBUF;
        u32x4_t kf[SW][NC][NU], vf[SW][ND][NV];
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const int key = krow(u);
                    const int sw = F32 ? key & 15 : swz_paged(key);
                    kf[w][c][u] = *(const u32x4_t*)(buf + w * SBUF + key * (DH * ES) + (((NG * c + g) ^ (sw & (KC - 1))) << 4));
                }
        __builtin_amdgcn_sched_barrier(0);
        Acc s[SW][NU];
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < NA; ++i) s[w][u][i] = 0.f;
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int u = 0; u < NU; ++u) s[w][u] = E::mfma(kf[w][c][u], qf[c], s[w][u]);
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int u = 0; u < NV; ++u) {
                    const int dim = RT * dt + r;
                    const int sw = swz_v<F32, RT>(dim);
                    vf[w][dt][u] = *(const u32x4_t*)(buf + w * SBUF + KPLANE + dim * (32 * ES) + (((NG * u + g) ^ sw) << 4));
                }
        __builtin_amdgcn_sched_barrier(0);

        if constexpr (TREE) __builtin_amdgcn_s_setprio(0);
        float sv[SW][NS];
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int e = 0; e < NS; ++e) sv[w][e] = s[w][e / NA][e % NA];
        if (k0w + 32 * SW > lim_w || !whole) {
            if constexpr (TREE) {
                const int end0 = mine[0], t0 = k0w - mine[64];
                const uint32_t* words = words_of(t) + lane;
                const bool masked = k0w + 32 * SW > lim_w;              // (else the words are not there)
#pragma unroll
                for (int w = 0; w < SW; ++w) {
                    const int n = ((there >> (kw * SW + w)) & 1 ? end0 : 0) - (k0w + 32 * w);      // keys before the limit
                    uint32_t vis = masked ? mask_bits(words[64 * w], words[64 * w + 64], t0 + 32 * w, a.mask_ld) : 0xFFFFFFFFu;
                    vis = (n >= 32 ? vis : (n > 0 ? vis & ((1u << n) - 1) : 0u)) >> key_of(0);
#pragma unroll
                    for (int e = 0; e < NS; ++e)
                        if (!(vis >> (key_of(e) - key_of(0)) & 1)) sv[w][e] = -INFINITY;
                }
            } else {
#pragma unroll
                for (int w = 0; w < SW; ++w) {
                    const int end = (there >> (kw * SW + w)) & 1 ? lim : 0;
#pragma unroll
                    for (int e = 0; e < NS; ++e)
                        if (k0w + 32 * w + key_of(e) >= end) sv[w][e] = -INFINITY;
                }
            }
        }
        // the row's maximum over the step and its lane groups (max is symmetric: a swap hands a lane its
        // partner's value)
        float bm = sv[0][0];
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int e = 0; e < NS; ++e) bm = fmaxf(bm, sv[w][e]);
        const auto w32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(bm), __float_as_uint(bm), false, false);
        bm = fmaxf(__uint_as_float(w32[0]), __uint_as_float(w32[1]));
        if constexpr (!R32) {
            const auto w16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(bm), __float_as_uint(bm), false, false);
            bm = fmaxf(__uint_as_float(w16[0]), __uint_as_float(w16[1]));
        }
        const float bms = bm * a.sl2;
        // the reference moves only when some row of the tile exceeds it by PAGED_SLACK: O, sum and merge are
        // exact for any reference, and most steps skip the rescale
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(bms > mrun + PAGED_SLACK) != 0, 0)) {
            const float mnew = fmaxf(mrun, bms);
            const float alpha = (mnew == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(mrun - mnew);
            lrun *= alpha;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int i = 0; i < NA; ++i) oacc[dt][i] *= alpha;
            mrun = mnew;
        }
        const float mref = (mrun == -INFINITY) ? 0.f : mrun;
        u32x4_t pf[SW][NV];
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < SW; ++w) {
            float p[NS];
#pragma unroll
            for (int e = 0; e < NS; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(sv[w][e], a.sl2, -mref));
#pragma unroll
            for (int e = 0; e < NS; e += 4) sum += (p[e] + p[e + 1]) + (p[e + 2] + p[e + 3]);
            if constexpr (F32) {
#pragma unroll
                for (int e = 0; e < NS; ++e) pf[w][e >> 2][e & 3] = __float_as_uint(p[e]);
            } else {
                // rounded to nearest for the product with V, which takes operands of T (half a step of T a
                // probability: as much as the output's own rounding, together 1.4 times the error of a form in fp32
                // rounded once); the sum keeps fp32
#pragma unroll
                for (int e = 0; e < NS / 2; ++e)
                    pf[w][e >> 2][e & 3] = __builtin_bit_cast(uint32_t, (typename E::x2){(T)p[2 * e], (T)p[2 * e + 1]});
            }
        }
        lrun += sum;
#pragma unroll
        for (int w = 0; w < SW; ++w)
#pragma unroll
            for (int u = 0; u < NV; ++u)
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) oacc[dt] = E::mfma(vf[w][dt][u], pf[w][u], oacc[dt]);
    }

    // What clean_tail took out, for the rows that see it: sums of classes over each block's keys, V^T
    // straight from its page (a fragment's 16 bytes are consecutive keys of a dim).
    if (lim_lo < ktop) {
        __syncthreads();                                                // (the last round's reads)
        if (lane == 0) ((int*)lds)[wave] = odd != 0;
        __syncthreads();
        int any = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) any |= ((const int*)lds)[w];
        odd = __builtin_amdgcn_readfirstlane(any);
        if (KG > 1) __syncthreads();                                    // (written again below)
    }
    if (odd != 0) {
        for (int blk = kz > ks + 32 * kb0 ? (kz - ks) / 32 - kb0 : 0; blk < blocks; ++blk) {
            const int k0 = ks + 32 * (kb0 + blk), pg = trow[k0 >> a.page_shift];
            if ((KG > 1 && blk % SUB / SW != kw) || pg < 0 || pg >= a.n_pages) continue;
            const T* Vp = (const T*)a.vp + ((long)pg * a.Hk + hk) * page_elems + (k0 & ((1 << a.page_shift) - 1));
            uint32_t vis = 0xFFFFFFFFu;
            int end = lim;
            if constexpr (TREE) {
                const int t = k0 - mine[64], i = t >> 5;
                const uint32_t* words = a.mask + mine[128];
                vis = mask_bits(words[min(max(i, 0), a.mask_ld - 1)], words[min(max(i + 1, 0), a.mask_ld - 1)], t, a.mask_ld);
                end = mine[0];
            }
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                Acc c;
#pragma unroll
                for (int i = 0; i < NA; ++i) c[i] = 0.f;
#pragma unroll
                for (int u = 0; u < NV; ++u) {
                    const u32x4_t v = ldg16(Vp + ((long)(RT * dt + r) << a.page_shift) + (16 / ES) * (NG * u + g));
                    auto sees = [&](int e) {
                        const int o = key_of(16 / ES * u + e), key = k0 + o;
                        return key >= kz && key < end && (!TREE || (vis >> o & 1)) ? PagedClass<T>::one : 0u;
                    };
                    u32x4_t seen;
#pragma unroll
                    for (int i = 0; i < 4; ++i) seen[i] = F32 ? sees(i) : sees(2 * i) | (sees(2 * i + 1) << 16);
                    c = E::mfma(class_of<T>(v), seen, c);
                }
#pragma unroll
                for (int i = 0; i < NA; ++i) oacc[dt][i] = add_classes(oacc[dt][i], c[i]);
            }
        }
    }

    // the waves' key groups merge as the parts do
    if constexpr (KG > 1) {
        constexpr int REC = ND * NA / 4 + 1;                            // 16-byte records of a lane
        static_assert((KG - 1) * QG * REC * 1024 <= 2 * BUF, "the groups' sums must fit the buffers");
        __syncthreads();
        float4* rec = (float4*)lds + qw * REC * 64 + lane;
        if (kw > 0) {
            rec += (kw - 1) * QG * REC * 64;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < NA / 4; ++j)
                    rec[(dt * NA / 4 + j) * 64] = make_float4(oacc[dt][4 * j], oacc[dt][4 * j + 1], oacc[dt][4 * j + 2],
                                                              oacc[dt][4 * j + 3]);
            rec[(REC - 1) * 64] = make_float4(mrun, lrun, 0.f, 0.f);
        }
        __syncthreads();
        if (kw > 0) return;
#pragma unroll
        for (int k = 0; k < KG - 1; ++k, rec += QG * REC * 64) {
            const float4 ml = rec[(REC - 1) * 64];
            const float M = fmaxf(mrun, ml.x);
            const float w0 = mrun == M ? 1.f : __builtin_amdgcn_exp2f(mrun - M);
            const float w1 = ml.x == M ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
            mrun = M;
            lrun = lrun * w0 + ml.y * w1;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < NA / 4; ++j) {
                    const float4 o = rec[(dt * NA / 4 + j) * 64];
                    oacc[dt][4 * j] = oacc[dt][4 * j] * w0 + o.x * w1;
                    oacc[dt][4 * j + 1] = oacc[dt][4 * j + 1] * w0 + o.y * w1;
                    oacc[dt][4 * j + 2] = oacc[dt][4 * j + 2] * w0 + o.z * w1;
                    oacc[dt][4 * j + 3] = oacc[dt][4 * j + 3] * w0 + o.w * w1;
                }
        }
    }

    float l = lrun + __shfl_xor(lrun, 32);
    if constexpr (!R32) l += __shfl_xor(l, 16);
    const int f = f0 + RT * qw + r;
    if (f >= nv) return;
    const int row = R0 + f / a.G, h = hk * a.G + f % a.G;
    // (accumulators 4j .. 4j + 3 are consecutive dims)
    auto dim_of = [&](int dt, int j) { return RT * dt + (R32 ? 8 * j + 4 * g : 4 * g); };
    if (a.direct) {
        const float inv = l != 0.f ? 1.f / l : 0.f;          // (a NaN stays one)
        const size_t at = row * a.ld_out + h * DH;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int j = 0; j < NA / 4; ++j) {
                float o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = oacc[dt][4 * j + i] * inv;
                store_out4<T>(a, at + dim_of(dt, j), o);
            }
    } else {
        const size_t rec = ((size_t)part * a.T + row) * a.H + h;
        if (rounds > 0) {
            float* op = a.opart + rec * DH;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < NA / 4; ++j)
                    *(float4*)(op + dim_of(dt, j)) = make_float4(oacc[dt][4 * j], oacc[dt][4 * j + 1], oacc[dt][4 * j + 2],
                                                                 oacc[dt][4 * j + 3]);
        }
        if (g == 0) *(float2*)(a.mlpart + rec * 2) = make_float2(mrun, l);
    }
}

// Merge of the parts: o = sum_s o_s 2^(m_s - M) / sum_s l_s 2^(m_s - M).  DH / 4 lanes per
// (row, head), four dims each.  The first eight parts' outputs are asked for beside the parts'
// (m, l), of which the lanes take one each: one round trip for up to eight parts, one more for
// each eight behind them.  A part with an empty sum wrote no output: what stands there is read
// and not used.
template <typename T, int DH>
__global__ void __launch_bounds__(256) attn_paged_merge_kernel(PagedArgs a) {
    constexpr int LPP = DH / 4, MAXW = 2 * MAX_ATTN_SPLITS / LPP;      // weights per lane
    const int pair = blockIdx.x * (256 / LPP) + threadIdx.x / LPP, li = threadIdx.x % LPP;
    const RowRange rows = row_range(a.row0[0], a.row0[a.B], a.T, a.T);
    const int R0 = rows.begin, R1 = rows.end;
    const int row = min(R0 + pair / a.H, a.T - 1), h = pair % a.H;
    const size_t rec = (size_t)row * a.H + h, step = (size_t)a.T * a.H;
    const int np = a.ns_s + a.ns_o;
    const float* src = a.opart + rec * DH + 4 * li;
    float4 v[8];
    auto load8 = [&](int s0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = *(const float4*)(src + (size_t)min(s0 + j, np - 1) * step * DH);
    };
    load8(0);
    float m[MAXW], l[MAXW], M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < MAXW; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
        if (LPP * i < np && li + LPP * i < np) {
            const float2 ml = *(const float2*)(a.mlpart + ((li + LPP * i) * step + rec) * 2);
            m[i] = ml.x;
            l[i] = ml.y;
        }
        M = fmaxf(M, m[i]);
    }
#pragma unroll
    for (int o = 1; o < LPP; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
#pragma unroll
    for (int i = 0; i < MAXW; ++i) {
        m[i] = l[i] != 0.f ? exp2f(m[i] - M) : 0.f;                    // the part's weight (a NaN sum stays one)
        L += l[i] * m[i];
    }
#pragma unroll
    for (int o = 1; o < LPP; o <<= 1) L += __shfl_xor(L, o);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < MAXW; ++i) {
        for (int s0 = LPP * i; s0 < min(np, LPP * (i + 1)); s0 += 8) {
            if (s0 > 0) load8(s0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = __shfl(m[i], (s0 + j) % LPP, LPP);
                if (s0 + j < np && w > 0.f) { o.x += v[j].x * w; o.y += v[j].y * w; o.z += v[j].z * w; o.w += v[j].w * w; }
            }
        }
    }
    if (R0 + pair / a.H >= R1) return;
    const float inv = L != 0.f ? 1.f / L : 0.f;
    const float e[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
    store_out4<T>(a, row * a.ld_out + h * DH + 4 * li, e);
}

}  // namespace dllm
