// Matrix products of ragged groups of rows (regione_grouped_matmul, regione_mxfp4_grouped_matmul):
//
//     out[r, :] = act(x[r, :] W_i^T + b_i),    r in [row_begin[g], row_end[g]),  i = g mod n_weights
//
// The paper names no such operator: it takes the model's layers as given.  What its region step asks of them is here: the
// recomputed rows of a request are few, their number is known on the device only (the partition wrote it), and text and image
// rows of a block have weights of their own (Sec. 4 "Region-Aware Generation": which rows a region step recomputes).
//
// The features of W are the M side of the tensor-core product and the rows of x its N side: D^T = W x^T.  M is fixed by the
// hardware (128 lanes of tensor memory a CTA), N is any multiple of 16 or 32 up to 256 named in the instruction, so a group
// of 5 rows costs a tile of 16 or 32 and not one of 128 or 256.
//
// Two kernels.  Pairs of CTAs (cta_group::2, 256 features, up to 256 rows, a persistent cluster per pair of SMs, two accumulators so
// that sums leave while the next tile's products run) for what fills the GPU: 8192^3 in bf16 700 us = 1.57 PFLOP/s with
// the tensor pipe 92 % busy (the clock is what the power limit leaves), in 4 bits 228 us = 4.8 PFLOP/s; a library product in bf16
// takes 670.  Lone CTAs (128 features, up to 128 rows; two to an SM with tiles of up to 64 rows, of 32 in 4 bits) for less, where
// the start of a launch is what counts: 1024^3 7.9 us, in 4 bits 6.0; two rows against 2 x 6144 x 1024 weights 7.2 us (25 MB, 3.9 us
// at the copy rate), 5.2 in 4 bits.  Both can split K over the CTAs of a cluster, which add their sums in the order of the
// slices (225 rows, K 7544, N 80: 29 us whole, 10 in eight slices).  The host chooses from the capacities, the width of a pair's tiles
// is chosen on the device from the rows.
//
// What bounds them: bf16 the tensor core; 4 bits, whose operands last a quarter as long, the way from L2 into the SMs (30 KB a
// chunk in 400 ns of which the products are 272), and with K below 4096 the sums' way out; few rows the weights' way from
// device memory (64 experts of 2048 x 1408 with 4096 rows: 70 us, 62 at the copy rate).
#include "adapters.cuh"
#include "common.cuh"
#include "f32x2.cuh"
#include "grouped_plan.cuh"
#include "sm100_ptx.cuh"

#include <algorithm>
#include <type_traits>

namespace regione {

constexpr int kFeat = 128;                            // features a CTA
constexpr int kChunkBytes = 128;                      // of K: 64 bf16 or 256 4-bit elements, one swizzle row
constexpr int kTileBytes = 128 * kChunkBytes;         // 128 rows of either operand
constexpr int kMaxStages = 12;
constexpr int kMaxGroups = 512;
constexpr int kScaleA = 1024, kScaleB = 2048;         // scales of a stage: [2 of 128 elements][1 or 2 of 128 rows][512 bytes]
// Warps of a CTA: 8 (4) that take sums out of tensor memory, one that loads, one that issues products, and with 4-bit operands 8 (4) that
// bring the scales: a pair of CTAs fills its SMs, CTAs without a pair and with narrow tiles leave room for a second one.
template <bool FP4, bool PAIR> struct Roles {
    static constexpr int kEpi = PAIR ? 8 : 4, kScale = PAIR ? 8 : 4, kThreads = (kEpi + 2 + (FP4 ? kScale : 0)) * 32;
};
constexpr int kStagingBytes = 1024;                   // per epilogue warp: 16 rows of 32 features
constexpr long long kGroupedWait = 4000000000LL;      // cycles (about 2 s): bound of every wait
constexpr int kMaps = 4;                              // boxes of 16, 32, 64 and 128 rows of x

struct GroupedArgs {
    const int32_t *row_begin, *row_end;
    int groups, n_weights, rows_cap, K, N;
    int chunks;                                       // of K
    int ring_bytes;                                   // for stages: 128 rows of W and a tile's of x each, and the scales of both
    int tmem_columns, scale_column;
    int slices;                                       // of K, each a CTA or a pair of a cluster (an even number, or 1)
    int width;                                        // rows of a tile at most (lone CTAs)
    const uint16_t* bias;                             // [n_weights, N] or NULL
    int activation;
    uint16_t* out;
    long long out_stride;
    const uint8_t *x_scale, *w_scale;                 // [rows_cap, K / 32], [n_weights, N, K / 32]
    int32_t* dev_status;
    // low-rank adapters (see Product)
    const int32_t* adapter;                           // [groups], -1: none
    int n_adapters, rank, tail;                       // tail: chunks of the rank behind those of K, as often as a sum has parts
    const float* adapter_scale;                       // [n_adapters] or NULL
    const float* addend;                              // [rows_cap, N]
};

// What a launch multiplies.  kPlain: rows with the weight set of their group.  The others are the parts of a product with low-rank
// adapters beside it:
//   kInto    u = s_a x A_a^T, the adapter of the group in place of the weight set; rows of groups without one are left out.  A sum leaves
//            as its parts (see lead_part), each kind of them rows_cap rows behind the one before
//   kTail    rows with the weight set, and behind the chunks of K those of the rank, once for each part: u with B_a, into the same
//            accumulators
//   kJoined  rows with the weight set plus an fp32 row that the adapters' sums are already in; groups of a set whose ranges touch are one
//            range, so that many groups of a row or two share the tiles, and the weights are read once
enum class Product { kPlain, kInto, kTail, kJoined };
struct GroupedMaps {
    CUtensorMap w;                                    // (K, N, n_weights), box 128 bytes x 128 rows
    CUtensorMap x[kMaps];                             // (K, rows), box 128 bytes x 16 << i rows
    CUtensorMap out;                                  // (N, rows), box 32 features x 16 rows
};
struct TailMaps : GroupedMaps {
    CUtensorMap b;                                    // (rank, N, n_adapters), box 128 bytes x 128 rows
    CUtensorMap u[kMaps];                             // (rank, rows of all parts), box 128 bytes x 16 << i rows
};
template <Product OP> using MapsOf = std::conditional_t<OP == Product::kTail, TailMaps, GroupedMaps>;

struct GroupedControl {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort_flag;
    int width, total;                                 // of the plan: rows of a tile at most, tiles
    int cost[8];
    int first[kMaxGroups + 1];                        // of a group: row tiles ahead of it,
    int begin[kMaxGroups], rows[kMaxGroups];          // its first row, how many,
    int16_t widths[kMaxGroups];                       // rows of its tiles, which are even
};

struct AdapterControl : GroupedControl {
    int adapter[kMaxGroups];                          // of a group, -1: none
};
template <Product OP> constexpr bool kAdapters = OP == Product::kInto || OP == Product::kTail;
template <Product OP> using ControlOf = std::conditional_t<kAdapters<OP>, AdapterControl, GroupedControl>;
// The second launch of a product with adapters, which starts ahead of the first one's end (see the kernel).  What it reads before it has
// waited comes from L2: lines of L1 may be older than the launch in front of the first.
template <Product OP> constexpr bool kLate = OP == Product::kTail || OP == Product::kJoined;
template <Product OP, typename T> __device__ __forceinline__ T ld_input(const T* p) {
    if constexpr (kLate<OP>) return __ldcg(p);
    else return __ldg(p);
}

// ---- instructions that the pair of CTAs and the scaled product need -------------------------------------------
namespace {

template <bool PAIR> __device__ __forceinline__ void take_tmem(uint32_t slot, uint32_t columns) {
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        ptx::tmem_alloc(slot, columns);
        ptx::tmem_relinquish();
    }
}
template <bool PAIR> __device__ __forceinline__ void free_tmem(uint32_t taddr, uint32_t columns) {
    if constexpr (PAIR)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(columns) : "memory");
    else
        ptx::tmem_dealloc(taddr, columns);
}

template <bool PAIR, bool FP4>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    if constexpr (FP4 && PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else if constexpr (FP4)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        ptx::mma_ss(d, a, b, idesc, accumulate);
}

// Scales of 128 rows and 128 elements (512 bytes: row r at (r % 32) * 16 + (r / 32) * 4) to 4 columns of tensor memory, in all four
// lane groups; in a pair each CTA from its own shared memory to its own tensor memory.  Products issued behind it by the same
// thread see them.
template <bool PAIR> __device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
    if constexpr (PAIR)
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// All tcgen05 operations issued so far by this thread arrive on `bar`, in a pair on the barrier at that place in both CTAs.
template <bool PAIR> __device__ __forceinline__ void commit(uint32_t bar, uint32_t pair_mask) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)pair_mask) : "memory");
    else
        ptx::mma_commit(bar);
}

// Tiled loads; in a pair `bar` may be the leader's.
template <bool PAIR>
__device__ __forceinline__ void load_w(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void load_x(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1) : "memory");
}

// Arrival on a barrier of this CTA or, in a pair, of its leader: at the cluster's scope where that is another CTA, since a thread of that
// CTA acts on what is announced.  It releases nothing there.  An accumulator that was read out: tcgen05 operations are ordered by the
// fences of their own on both sides.  Scales: behind release_smem, which is restricted to the warp's writes to its own CTA's shared
// memory (themselves behind their proxy fence); an ordinary release at that scope waits for all memory operations of the warp that
// are on their way (17408 x 4096 x 8192 with GELU in 4 bits 347 us, in this form 234).
template <bool PAIR> __device__ __forceinline__ void release_smem(int rank) {
    if (PAIR && (rank & 1)) asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory");
}
template <bool PAIR> __device__ __forceinline__ void arrive_at(uint32_t bar, int rank) {
    if (PAIR && (rank & 1))
        asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(ptx::map_rank(bar, rank & ~1)) : "memory");
    else
        ptx::mbar_arrive(bar);
}

// 16 rows of 32 features from shared memory (64-byte swizzle) to the output; what lies behind the last feature is not written.
__device__ __forceinline__ void store_out(const CUtensorMap* map, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(c0), "r"(c1) : "memory");
}

// 16 lanes x 16 columns: thread l gets rows l / 4 and l / 4 + 8, columns 2 (l % 4) + {0, 1} and the same 8 further on.
__device__ __forceinline__ void tmem_ld_16x256b_x2(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
}
// Four 8 x 8 matrices of 16-bit elements, transposed; lane l names the place of row l % 8 of matrix l / 8.
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

}  // namespace

// ---- waits: bounded; a wait that runs out is recorded and makes the other roles of the CTA give up -----------------
// FAR: a thread of the pair's other CTA is among those that arrive.  (Where only copies and products complete, which the hardware
// announces, the scope is the CTA whichever CTA issued them; acquiring at the cluster's everywhere takes 8192^3 in 4 bits from 238 to 252 us.)
template <bool FAR> __device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    return FAR ? ptx::mbar_try_wait_cluster(bar, parity) : ptx::mbar_try_wait(bar, parity);
}
template <bool FAR>
__device__ __forceinline__ bool grouped_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* dev_status,
                                                  long long limit) {
    const long long t0 = clock64();
    while (!try_wait<FAR>(bar, parity)) {
        if (*abort_flag) return false;
        if (clock64() - t0 > limit) {
            *abort_flag = 1;
            record_status(dev_status, REGIONE_DEV_TIMEOUT);
            return false;
        }
    }
    return true;
}
template <bool FAR = false>
__device__ __forceinline__ bool grouped_wait(uint32_t bar, uint32_t parity, GroupedControl* ctl, int32_t* dev_status,
                                             long long limit = kGroupedWait) {
    return try_wait<FAR>(bar, parity) || grouped_wait_slow<FAR>(bar, parity, &ctl->abort_flag, dev_status, limit);
}

__device__ __forceinline__ float min_or_nan(float x, float y, float z) {
    float r;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// gelu(x) = x / 2 (1 + tanh(u)) = x / (1 + exp(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3), of N pairs of values; the second form keeps its
// relative accuracy where tanh(u) is near -1.  A pair shares a reciprocal, 1 / a = b / (a b): three results of the special
// function unit, which sets the pace, in place of four.  a b is below 2^118 where both are above -7.4; where one of the lane's values is
// not, or is a NaN, each takes a reciprocal of its own.  That is 0 from -10.1 on, where gelu is below 2^-122: -0 there, and NaN for
// -infinity, as the formula gives.  Step by step for all pairs, and the compiler held to it: left to interleave it keeps few in
// flight (4 bits, 16896 x 2048 x 8192: 195 us pair by pair, 175 so).
template <int N> __device__ __forceinline__ void gelu_tanh(uint64_t (&x)[N]) {
    constexpr float c = -2.0f * 1.4426950409f * 0.7978845608f;
    auto exponent = [&](int i, float& a, float& b) {  // of exp(-2 u), to base 2
        parts_of(mul2(x[i], fma2(mul2(x[i], x[i]), pair_of(c * 0.044715f, c * 0.044715f), pair_of(c, c))), a, b);
    };
    float e[2 * N], r[N], least[2 * N];
#pragma unroll
    for (int i = 0; i < N; ++i) parts_of(x[i], least[2 * i], least[2 * i + 1]);
#pragma unroll
    for (int n = 2 * N; n > 1; n = (n + 2) / 3)
#pragma unroll
        for (int i = 0; i < (n + 2) / 3; ++i)
            if (3 * i + 1 < n) least[i] = min_or_nan(least[3 * i], least[3 * i + 1], least[min(3 * i + 2, n - 1)]);
            else least[i] = least[3 * i];
    if (!(least[0] > -7.4f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            exponent(i, e[0], e[1]);
            x[i] = mul2(x[i], pair_of(reciprocal(1.0f + fast_exp2(e[0])), reciprocal(1.0f + fast_exp2(e[1]))));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) exponent(i, e[2 * i], e[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+f"(e[i]));
#pragma unroll
    for (int i = 0; i < N; ++i) parts_of(add2(pair_of(e[2 * i], e[2 * i + 1]), pair_of(1.0f, 1.0f)), e[2 * i], e[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("rcp.approx.ftz.f32 %0, %1;" : "=f"(r[i]) : "f"(e[2 * i] * e[2 * i + 1]));
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = mul2(x[i], mul2(pair_of(e[2 * i + 1], e[2 * i]), pair_of(r[i], r[i])));   // (x b could overflow)
}

// A group's rows within the buffer; false: the range as given is not within it.
template <Product OP = Product::kPlain>
__device__ __forceinline__ bool rows_of(const GroupedArgs& p, int g, int& begin, int& rows) {
    if constexpr (kLate<OP>) return cut_range(__ldcg(p.row_begin + g), __ldcg(p.row_end + g), p.rows_cap, begin, rows);
    else return cut_range(p.row_begin[g], p.row_end[g], p.rows_cap, begin, rows);
}

// A group's adapter, -1 for none; one that does not exist is none (`in`: false).
template <Product OP> __device__ __forceinline__ int adapter_of(const GroupedArgs& p, int g, bool& in) {
    const int a = ld_input<OP>(p.adapter + g);
    in = a >= -1 && a < p.n_adapters;
    return in ? a : -1;
}

// Rows [first, first + live) of a group against a feature tile; `width` = columns of the product.
struct GroupedTile {
    int first, live, width, weights, feature;
    int adapter;                                      // kTail, and with kInto the weight set
};

// Tile t of the plan, t not smaller than at the last call; `group` is where that one was.  Tiles of a group run through eight feature
// tiles before they go on to the next rows, so that the tiles in flight at one time share both operands.  PAIR: 256 features,
// widths in steps of 32.
template <bool PAIR, Product OP = Product::kPlain>
__device__ __forceinline__ GroupedTile tile_at(const GroupedArgs& p, const GroupedControl* ctl, int t, int f_tiles, int& group) {
    while (ctl->first[group + 1] * f_tiles <= t) ++group;
    const int ahead = ctl->first[group], n = ctl->first[group + 1] - ahead, width = ctl->widths[group];
    int in = t - ahead * f_tiles, block = 0;
    if (f_tiles > 8 && in >= 8 * n) {
        block = in / (8 * n);
        in -= block * 8 * n;
    }
    const int wide = min(8, f_tiles - block * 8), at = wide == 8 ? in >> 3 : in / wide;
    GroupedTile tile;
    tile.first = ctl->begin[group] + at * width;
    tile.live = min(width, ctl->rows[group] - at * width);
    tile.width = width;
    tile.weights = group < p.n_weights ? group : group % p.n_weights;
    tile.feature = (block * 8 + in - at * wide) * (PAIR ? 2 : 1) * kFeat;
    tile.adapter = -1;
    if constexpr (kAdapters<OP>) {
        tile.adapter = static_cast<const AdapterControl*>(ctl)->adapter[group];
        if (OP == Product::kInto) tile.weights = max(tile.adapter, 0);
    }
    return tile;
}

// kJoined: groups of a weight set, in their order, whose ranges touch become one, at the place of the first; the others have no rows.  The
// last one of a range is found by following links of twice the length in every round.  (All threads; ends with a barrier.)
__device__ __forceinline__ void join_groups(const GroupedArgs& p, GroupedControl* ctl) {
    int16_t* last = ctl->widths;
    bool in = true;
    for (int g = threadIdx.x; g < p.groups; g += blockDim.x) in = rows_of<Product::kJoined>(p, g, ctl->begin[g], ctl->rows[g]) && in;
    if (!in && blockIdx.x == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
    __syncthreads();
    auto joins = [&](int g) {                         // group g to the set's next one
        return g + p.n_weights < p.groups && ctl->begin[g] + ctl->rows[g] == ctl->begin[g + p.n_weights];
    };
    for (int g = threadIdx.x; g < p.groups; g += blockDim.x) last[g] = (int16_t)(joins(g) ? g + p.n_weights : g);
    __syncthreads();
    constexpr int kEach = (kMaxGroups + 191) / 192;   // of a thread (a CTA has 192 at least)
    for (int reach = p.n_weights; reach < p.groups; reach *= 2) {
        int16_t further[kEach];
        for (int i = 0, g = threadIdx.x; i < kEach && g < p.groups; ++i, g += blockDim.x) further[i] = last[last[g]];
        __syncthreads();
        for (int i = 0, g = threadIdx.x; i < kEach && g < p.groups; ++i, g += blockDim.x) last[g] = further[i];
        __syncthreads();
    }
    int rows[kEach];
    for (int i = 0, g = threadIdx.x; i < kEach && g < p.groups; ++i, g += blockDim.x)
        rows[i] = g >= p.n_weights && joins(g - p.n_weights) ? 0 : ctl->begin[last[g]] + ctl->rows[last[g]] - ctl->begin[g];
    __syncthreads();
    for (int i = 0, g = threadIdx.x; i < kEach && g < p.groups; ++i, g += blockDim.x) ctl->rows[g] = rows[i];
    __syncthreads();
}

// Scales of the tiles [t0, t_end): 8 bytes a row and chunk, from rows that lie K / 32 bytes apart to the places in shared memory that
// the copy to tensor memory reads.  A team of four warps takes a part of two chunks, 16 bytes a row, a warp every fourth group
// of 32 rows; a pair of CTAs has two teams that take turns (8192^3: 249 us with one team, 209 with two).  Loads for the next part
// are not sent ahead: the proxy fence would wait for them.  In a pair of CTAs both chunks of a part are announced behind one pair of
// fences (8192 x 4096 x 8192: 194 000 cycles with a pair each, 186 000 so; lone CTAs have less to wait for and announce each).  The stage that a team waits for is at most four chunks behind its last
// one and the ring has at least four stages: no phase of a barrier can be mistaken for the one two further on.
// VEC, rows on 16 bytes: a lane reads its row's 16 bytes, 32 rows in one load.  Else four lanes read a word each, 8 rows in one load: as
// many lines of the L1 a row (2 x 4992 x 296 for four times 764 rows: 14.9 us, a lane with the four words of its row 20.8).
// Rows behind the tile are read as its last one, words behind a row as its last: what they scale is not stored.
struct ScaleRole {
    GroupedControl* ctl;
    uint8_t* scales;
    int stages, f_tiles, workers, rank, warp, lane, c_begin, c_end;
    long long t0, t_end;
    int s, group;                                     // the ring's next stage, the last tile's group
    uint32_t phase;
};
template <bool PAIR, bool VEC>
__device__ __forceinline__ bool bring_scales(const GroupedArgs& p, const ScaleRole r) {
    constexpr int kTeams = PAIR ? 2 : 1, kGroups = PAIR ? 3 : 2;     // groups of 32 rows a warp: 128 rows of W, up to 256 (128) of x
    int s = r.s, group = r.group;
    uint32_t phase = r.phase;
    const int k32 = p.K / 32, team = r.warp >> 2, member = r.warp & 3, lane = r.lane;
    const int in_group = VEC ? (lane >> 2) + 32 * (lane & 3) : (lane >> 4) + 32 * ((lane >> 2) & 3);
    long long t = r.t0;
    int c = r.c_begin;
    bool fresh = true;                                // the next fetch is the first of its tile
    const uint8_t* src[kGroups];
    int room[kGroups];                                // rows of the matrix behind the lane's first
    auto fetch = [&](uint4 (&v)[kGroups]) {
        if (fresh) {
            const GroupedTile tile = tile_at<PAIR>(p, r.ctl, (int)t, r.f_tiles, group);
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {       // part i: 4 groups of W, then those of x
                const int row = (i == 0 ? tile.feature + (PAIR ? r.rank & 1 : 0) * kFeat : tile.first) + member * 8 + in_group + (i == 2 ? 128 : 0);
                const int last = (i == 0 ? p.N : min(p.rows_cap, tile.first + tile.width)) - 1;
                src[i] = (i == 0 ? p.w_scale + (size_t)tile.weights * p.N * k32 : p.x_scale) + (size_t)min(row, last) * k32;
                room[i] = max(last - row, 0);
            }
            fresh = false;
        }
        const int off = (c & ~1) * 8;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            if constexpr (VEC) {
                v[i] = ldg128(src[i] + off);
            } else {
                const int word = min(off + 4 * (lane & 3), k32 - 4);
                auto at = [&](int n) { return __ldg(reinterpret_cast<const uint32_t*>(src[i] + (min(2 * n, room[i]) * k32 + word))); };
                v[i] = make_uint4(at(0), at(1), at(2), at(3));
            }
        }
    };
    auto advance = [&] {                              // to the next part, of whichever team
        const int n = min(2 - (c & 1), r.c_end - c);
        c += n;
        s += n;
        if (s >= r.stages) { s -= r.stages; phase ^= 1; }
        if (c >= r.c_end) { c = r.c_begin; t += r.workers; fresh = true; }
    };
    if (kTeams == 2 && team == 1 && t < r.t_end) advance();
    uint4 v[kGroups];
    if (t < r.t_end) fetch(v);
    while (t < r.t_end) {
        const int first = c, n = min(2 - (c & 1), r.c_end - c);
        int at = s;
        uint32_t turn = phase;
        for (int k = 0; k < n; ++k) {
            if (!__all_sync(0xffffffffu, grouped_wait(ptx::smem_addr(&r.ctl->empty[at]), turn ^ 1, r.ctl, p.dev_status))) return false;
            uint32_t* base = reinterpret_cast<uint32_t*>(r.scales + at * (kScaleA + kScaleB)) + member * 32;
            const bool odd = (first + k) & 1;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                uint32_t* dst = base + (i == 0 ? 0 : kScaleA / 4 + (i == 1 ? 0 : 128));
                constexpr int kNextW = 128, kNextX = 256;             // words to the second 128 elements
                const int next = i == 0 ? kNextW : kNextX;
                if constexpr (VEC) {
                    dst[lane] = odd ? v[i].z : v[i].x;
                    dst[next + lane] = odd ? v[i].w : v[i].y;
                } else if (((lane >> 1) & 1) == odd) {
                    dst += (lane & 1) * next + (lane >> 2);
                    dst[0] = v[i].x;
                    dst[8] = v[i].y;
                    dst[16] = v[i].z;
                    dst[24] = v[i].w;
                }
            }
            if (!PAIR || k == n - 1) {
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    release_smem<PAIR>(r.rank);
                    if (PAIR && k > 0) arrive_at<PAIR>(ptx::smem_addr(&r.ctl->full[s]), r.rank);
                    arrive_at<PAIR>(ptx::smem_addr(&r.ctl->full[at]), r.rank);
                }
            }
            if (++at == r.stages) { at = 0; turn ^= 1; }
        }
        advance();
        if (kTeams == 2 && t < r.t_end) advance();
        if (t < r.t_end) fetch(v);
    }
    return true;
}

// VEC: of 4-bit operands, K is a multiple of 512 (see bring_scales).
template <bool FP4, bool PAIR, bool VEC, Product OP = Product::kPlain>
__global__ void __launch_bounds__(Roles<FP4, PAIR>::kThreads, PAIR ? 1 : 2)
grouped_kernel(const __grid_constant__ MapsOf<OP> maps, const __grid_constant__ GroupedArgs p) {
    static_assert(!FP4 || OP == Product::kPlain, "adapters are in bf16");
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr int kElems = FP4 ? 256 : 64;            // of K in a chunk
    constexpr int kMaxWidth = PAIR ? (FP4 ? 224 : 256) : 128;
    constexpr int kAcc1 = PAIR ? kMaxWidth : 0;       // column of the second accumulator
    constexpr int kEpiWarps = Roles<FP4, PAIR>::kEpi;
    constexpr int kProducer = kEpiWarps, kIssuer = kEpiWarps + 1, kScaler = kEpiWarps + 2;
    const uint32_t smem = (ptx::smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t* base = smem_raw + (smem - ptx::smem_addr(smem_raw));
    uint8_t* staging = base + p.ring_bytes;
    ControlOf<OP>* ctl = reinterpret_cast<ControlOf<OP>*>(staging + kEpiWarps * kStagingBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // a cluster has a tile's slices of K, a slice is a CTA or a pair; `half`: which of the pair
    const int cluster = (PAIR ? 2 : 1) * p.slices;
    const int rank = cluster > 1 ? (int)(blockIdx.x % cluster) : 0;
    const int half = PAIR ? rank & 1 : 0, slice = PAIR ? rank >> 1 : rank;
    const bool leader = half == 0, split = p.slices > 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            ptx::mbar_init(ptx::smem_addr(&ctl->full[s]), 1 + (FP4 ? 4 * (PAIR ? 2 : 1) : 0));
            ptx::mbar_init(ptx::smem_addr(&ctl->empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(ptx::smem_addr(&ctl->acc_full[a]), 1);
            ptx::mbar_init(ptx::smem_addr(&ctl->acc_empty[a]), kEpiWarps * (PAIR ? 2 : 1));
        }
        ctl->abort_flag = 0;
        ptx::fence_barrier_init();
    }
    if (warp == kIssuer) take_tmem<PAIR>(ptx::smem_addr(&ctl->tmem), p.tmem_columns);
    if (warp == kProducer && lane == 0) ptx::prefetch_tensormap(&maps.w);
    // The second launch of a product with adapters takes one thing from the first, and waits for it where it is read: the thread that
    // loads, ahead of the first chunk of the rank, or the threads that add.  Everything else was there before the first launch began,
    // which waited for it before it let this one in.  (Every CTA waits somewhere: what follows this launch counts on both.)
    if (!kLate<OP>) grid_dependency_wait();

    // ---- plan: from the groups' row counts, which only the device knows --------------------------------------------
    const int f_tiles = (p.N + (PAIR ? 2 : 1) * kFeat - 1) / ((PAIR ? 2 : 1) * kFeat);
    const int workers = gridDim.x / cluster;
    if constexpr (OP == Product::kJoined) join_groups(p, ctl);
    // A group's rows as the plan takes them; false: not a range of the buffer, or not an adapter.
    auto range = [&](int g, int& begin, int& rows) {
        if constexpr (OP == Product::kJoined) {
            begin = ctl->begin[g];
            rows = ctl->rows[g];
            return true;
        } else {
            bool in = rows_of<OP>(p, g, begin, rows);
            if constexpr (OP == Product::kInto) {
                bool exists;
                if (adapter_of<OP>(p, g, exists) < 0) rows = 0;
                in = in && exists;
            }
            return in;
        }
    };
    int own_begin = 0, own_rows = 0;                  // of group `lane`: read once, 800 cycles
    bool own_in = true;
    if (warp < (PAIR ? kMaxWidth / 32 : 1) && lane < p.groups) own_in = range(lane, own_begin, own_rows);
    if constexpr (PAIR) {
        // Widths of 32 .. 256 (224) rows: one warp adds up the tiles of one width.  A chunk of a tile takes the tensor core 2 cycles a row;
        // its 128 + width / 2 rows of 128 bytes arrive at about 57 bytes a cycle.  The width with the cheapest rounds of tiles is
        // taken, the larger of equals.  (4096 rows, K 4096, N 4096: rounds counted by width alone take 192, 123 us.)
        if (warp < kMaxWidth / 32) {
            const int width = 32 * (warp + 1);
            int n = (own_rows + width - 1) / width;
            for (int g = lane + 32; g < p.groups; g += 32) {
                int begin, rows;
                range(g, begin, rows);
                n += (rows + width - 1) / width;
            }
            n = min(__reduce_add_sync(0xffffffffu, n), p.rows_cap / width + p.groups);
            const int rounds = (n * f_tiles + workers - 1) / workers;
            if (lane == 0) ctl->cost[warp] = (int)min((long long)rounds * max(16 * width, 9 * (256 + width)), 0x7fffffffLL);
        }
        __syncthreads();
    }
    if (warp == 0) {
        int width = p.width;
        if constexpr (PAIR) {
            int best = kMaxWidth / 32 - 1;
            for (int i = kMaxWidth / 32 - 2; i >= 0; --i)
                if (ctl->cost[i] < ctl->cost[best]) best = i;
            width = 32 * (best + 1);
        }
        // (no more tiles than ranges without a common row have: ranges that overlap are cut there)
        const int most = p.rows_cap / width + p.groups;
        int at = 0;
        for (int g0 = 0; g0 < p.groups; g0 += 32) {
            const int g = g0 + lane;
            int n = 0;
            if (g < p.groups) {
                int begin = own_begin, rows = own_rows;
                bool in = own_in;
                if (g0 > 0) in = range(g, begin, rows);
                if (!in && blockIdx.x == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
                n = (rows + width - 1) / width;
                ctl->begin[g] = begin;
                ctl->rows[g] = rows;
                if constexpr (kAdapters<OP>) {
                    bool exists;
                    ctl->adapter[g] = adapter_of<OP>(p, g, exists);
                }
                constexpr int kStep = PAIR ? 32 : 16;
                if (n > 0) ctl->widths[g] = (int16_t)(((rows + n - 1) / n + kStep - 1) & ~(kStep - 1));
            }
            int sum = n;
            for (int d = 1; d < 32; d <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, sum, d);
                if (lane >= d) sum += up;
            }
            if (g < p.groups) ctl->first[g] = min(at + sum - n, most);
            at += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) {
            if (at > most && blockIdx.x == 0) record_status(p.dev_status, REGIONE_DEV_BOUNDS);
            at = min(at, most);
            ctl->first[p.groups] = at;
            ctl->width = width;
            ctl->total = at * f_tiles;
        }
    }
    ptx::tc_fence_before_sync();
    if (cluster > 1) ptx::cluster_sync(); else __syncthreads();
    ptx::tc_fence_after_sync();
    // (not before this CTA has its tensor memory: a CTA of the next kernel could take it and wait for this kernel's end)
    grid_launch_dependents();
    const uint32_t tmem = ctl->tmem;
    const int worker = blockIdx.x / cluster, total = ctl->total;
    // The narrower the tiles, the more stages: what bounds the loads is how many bytes are on their way (about 2 us under load).
    const int stage_bytes = kTileBytes + ctl->width * (PAIR ? kChunkBytes / 2 : kChunkBytes);
    const int stages = min(kMaxStages, p.ring_bytes / (stage_bytes + (FP4 ? kScaleA + kScaleB : 0)));
    uint8_t* scales = base + stages * stage_bytes;
    // chunks of K that this slice takes
    const int c_begin = (int)((long long)p.chunks * slice / p.slices), c_end = (int)((long long)p.chunks * (slice + 1) / p.slices);
    auto bar_at = [&](const uint64_t* bar) {          // a barrier of the pair's leader
        const uint32_t a = ptx::smem_addr(bar);
        return PAIR ? ptx::map_rank(a, rank & ~1) : a;
    };
    // What a role keeps from tile to tile: its group, its place in the ring, its tiles so far.
    int group = 0, s = 0, it = 0, sf = 0;
    uint32_t phase = 0;
    bool ok = true;
    const bool elected = ptx::elect_one();
    const uint32_t pair_mask = 3u << (rank & ~1);     // of the cluster's CTAs
    constexpr int kAccs = PAIR ? 2 : 1;
    // The chunk behind the last one of a tile: the last slice takes those of the rank, where the tile's group has an adapter.
    auto chunks_end = [&](const GroupedTile& tile) {
        return OP == Product::kTail && tile.adapter >= 0 && c_end == p.chunks ? c_end + kSumParts * p.tail : c_end;
    };

    // A cluster goes through its tiles without a stop; where slices meet, one tile at a time.
    for (long long t0 = worker; t0 < total; t0 += split ? workers : total) {
        const long long t_end = split ? t0 + 1 : total;
        if (warp == kProducer) {
            if (elected) {
                bool waited = false;
                for (long long t = t0; t < t_end && ok; t += workers) {
                    const GroupedTile tile = tile_at<PAIR, OP>(p, ctl, (int)t, f_tiles, group);
                    const int c_last = chunks_end(tile);
                    const int rows = PAIR ? tile.width / 2 : tile.width;                     // of x, for this CTA
                    const uint32_t bytes = (kTileBytes + rows * kChunkBytes) * (PAIR ? 2 : 1);
                    const int feature = tile.feature + half * kFeat, row = tile.first + half * rows;
                    for (int c = c_begin; c < c_last; ++c) {
                        if (!grouped_wait(ptx::smem_addr(&ctl->empty[s]), phase ^ 1, ctl, p.dev_status)) { ok = false; break; }
                        if (leader) ptx::mbar_arrive_expect_tx(ptx::smem_addr(&ctl->full[s]), bytes);
                        const uint32_t bar = bar_at(&ctl->full[s]), dst = smem + s * stage_bytes;
                        int at = 0;                                                  // boxes that make up the rows, the largest first
                        if constexpr (OP == Product::kTail) {
                            if (c >= p.chunks) {
                                if (!waited) {
                                    grid_dependency_wait();
                                    asm volatile("fence.proxy.async.global;" ::: "memory");
                                    waited = true;
                                }
                                const int part = (c - p.chunks) / p.tail, j = (c - p.chunks - part * p.tail) * kElems;
                                load_w<PAIR>(dst, &maps.b, bar, j, feature, tile.adapter);
#pragma unroll
                                for (int box = kMaps - 1; box >= 0; --box)
                                    if (rows & (16 << box)) {
                                        load_x<PAIR>(dst + kTileBytes + at * kChunkBytes, &maps.u[box], bar, j, part * p.rows_cap + row + at);
                                        at += 16 << box;
                                    }
                                if (++s == stages) { s = 0; phase ^= 1; }
                                continue;
                            }
                        }
                        load_w<PAIR>(dst, &maps.w, bar, c * (FP4 ? kChunkBytes : kElems), feature, tile.weights);
#pragma unroll
                        for (int box = kMaps - 1; box >= 0; --box)
                            if (rows & (16 << box)) {
                                load_x<PAIR>(dst + kTileBytes + at * kChunkBytes, &maps.x[box], bar, c * (FP4 ? kChunkBytes : kElems), row + at);
                                at += 16 << box;
                            }
                        if (++s == stages) { s = 0; phase ^= 1; }
                    }
                }
            }
        } else if (warp == kIssuer) {
            if (leader && elected) {
                constexpr uint32_t hi = ptx::smem_desc_hi_sw128(1024);              // 8-row groups 1024 bytes apart
                constexpr uint32_t hi_plain = (128u >> 4) | (1u << 14);             // scales: no swizzle, 8 rows of 16 bytes
                for (long long t = t0; t < t_end && ok; t += workers, ++it) {
                    const GroupedTile tile = tile_at<PAIR, OP>(p, ctl, (int)t, f_tiles, group);
                    const int c_last = chunks_end(tile);
                    const int a = it % kAccs, use = it / kAccs;
                    const uint32_t d = tmem + (a ? kAcc1 : 0);
                    if (use > 0 && !grouped_wait<PAIR>(ptx::smem_addr(&ctl->acc_empty[a]), (use - 1) & 1, ctl, p.dev_status)) { ok = false; break; }
                    ptx::tc_fence_after_sync();
                    // (4 bits: E2M1 operands, N, E8M0 scales, M)
                    const uint32_t idesc = FP4 ? (1u << 7) | (1u << 10) | ((uint32_t)(tile.width >> 3) << 17) | (1u << 23) |
                                                     ((PAIR ? 2u : 1u) << 27)
                                               : ptx::idesc_bf16_f32(PAIR ? 256 : 128, tile.width, false);
                    uint32_t accumulate = 0;
                    for (int c = c_begin; c < c_last; ++c) {
                        if (!grouped_wait<PAIR && FP4>(ptx::smem_addr(&ctl->full[s]), phase, ctl, p.dev_status)) { ok = false; break; }
                        ptx::tc_fence_after_sync();
                        const uint32_t at = smem + s * stage_bytes;
                        const uint32_t a_lo = ptx::smem_desc_lo(at, 16), b_lo = ptx::smem_desc_lo(at + kTileBytes, 16);
                        uint32_t sfa = 0, sfb = 0;
                        if constexpr (FP4) {
                            sfa = tmem + p.scale_column + sf * 32;
                            sfb = sfa + 8;
                            sf ^= 1;
                            const uint32_t sa = ptx::smem_addr(scales) + s * (kScaleA + kScaleB), sb = sa + kScaleA;
                            for (int k = 0; k < 2; ++k) {
                                copy_scales<PAIR>(sfa + 4 * k, ptx::smem_desc_join(ptx::smem_desc_lo(sa + k * 512, 16), hi_plain));
                                copy_scales<PAIR>(sfb + 8 * k, ptx::smem_desc_join(ptx::smem_desc_lo(sb + k * 1024, 16), hi_plain));
                                if (tile.width > 128)
                                    copy_scales<PAIR>(sfb + 8 * k + 4, ptx::smem_desc_join(ptx::smem_desc_lo(sb + k * 1024 + 512, 16), hi_plain));
                            }
                        }
                        // 32 bytes of K to an instruction; what lies behind K is zero and left out
                        const int behind = OP == Product::kTail && c >= p.chunks ? p.rank - (c - p.chunks) % p.tail * kElems : p.K - c * kElems;
                        const int left = (behind + kElems / 4 - 1) / (kElems / 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if (k >= left) break;
                            // (bits 4 and 29: which half of a scale word the two blocks of 32 have)
                            const uint32_t id = FP4 && (k & 1) ? idesc | (2u << 4) | (2u << 29) : idesc;
                            mma<PAIR, FP4>(d, ptx::smem_desc_join(a_lo + 2 * k, hi), ptx::smem_desc_join(b_lo + 2 * k, hi), id,
                                           sfa + 4 * (k >> 1), sfb + 8 * (k >> 1), accumulate);
                            accumulate = 1;
                        }
                        commit<PAIR>(ptx::smem_addr(&ctl->empty[s]), pair_mask);
                        if (++s == stages) { s = 0; phase ^= 1; }
                    }
                    if (ok) commit<PAIR>(ptx::smem_addr(&ctl->acc_full[a]), pair_mask);
                }
            }
        } else if (FP4 && warp >= kScaler) {
            const ScaleRole role = {ctl, scales, stages, f_tiles, workers, rank, warp - kScaler, lane, c_begin, c_end, t0, t_end, s, group, phase};
            ok = bring_scales<PAIR, VEC>(p, role) && ok;
            if (split) {                                  // where the ring stands behind this slice's chunks
                s += c_end - c_begin;
                while (s >= stages) { s -= stages; phase ^= 1; }
            }
        } else if (warp < kEpiWarps) {
            constexpr int kEpiCols = 16 * (kEpiWarps / 4), kOuts = OP == Product::kInto ? kSumParts : 1;
            const int sub = warp & 3, part = warp >> 2;
            const uint32_t stage = ptx::smem_addr(staging) + warp * kStagingBytes;
            for (long long t = t0; t < t_end; t += workers, ++it) {
                const GroupedTile tile = tile_at<PAIR, OP>(p, ctl, (int)t, f_tiles, group);
                const int a = it % kAccs, use = it / kAccs;
                const int feature = tile.feature + half * kFeat + 32 * sub;
                uint64_t bias[4] = {0, 0, 0, 0};          // of features lane / 4 + {0, 8, 16, 24}, twice each
                if (p.bias != nullptr && !split)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int f = min(feature + (lane >> 2) + 8 * i, p.N - 1);
                        const float b = __uint_as_float((uint32_t)ld_input<OP>(p.bias + (size_t)tile.weights * p.N + f) << 16);
                        bias[i] = pair_of(b, b);
                    }
                const float scale = OP == Product::kInto && p.adapter_scale != nullptr ? __ldg(p.adapter_scale + tile.weights) : 1.0f;
                if (!__all_sync(0xffffffffu, grouped_wait(ptx::smem_addr(&ctl->acc_full[a]), use & 1, ctl, p.dev_status)))
                    break;
                ptx::tc_fence_after_sync();
                const uint32_t acc = tmem + (a ? kAcc1 : 0) + ((uint32_t)(32 * sub) << 16);
                if (split) {
                    // this slice's sums as [row][128 features] fp32 over the stages, which nothing reads any more
                    float* sums = reinterpret_cast<float*>(base);
                    for (int c = part * 16; c < tile.live; c += kEpiCols) {
                        uint32_t r[16];
                        ptx::tmem_ld16(acc + c, r);
                        ptx::tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) sums[(c + i) * kFeat + 32 * sub + lane] = __uint_as_float(r[i]);
                    }
                } else {
                    // 16 rows at a time, the next ones on their way out of tensor memory meanwhile
                    uint32_t ahead[16];
                    auto fetch = [&](int c) {
                        tmem_ld_16x256b_x2(acc + c, ahead);
                        tmem_ld_16x256b_x2(acc + (16u << 16) + c, ahead + 8);
                    };
                    if (part * 16 < tile.live) fetch(part * 16);
                    if (OP == Product::kJoined) grid_dependency_wait();
                    for (int c = part * 16; c < tile.live; c += kEpiCols) {
                        uint64_t y[8];                                               // two rows of one feature
                        ptx::tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            y[i] = add2(pair_of(__uint_as_float(ahead[2 * i]), __uint_as_float(ahead[2 * i + 1])), bias[(i >> 2) * 2 + (i & 1)]);
                        if (c + kEpiCols < tile.live) fetch(c + kEpiCols);
                        if constexpr (OP == Product::kInto)
#pragma unroll
                            for (int i = 0; i < 8; ++i) y[i] = mul2(y[i], pair_of(scale, scale));
                        if constexpr (OP == Product::kJoined)
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                // (as the sums lie: rows 2 (l % 4) + {0, 1} of eight, features l / 4 of eight)
                                const int q = c + 8 * ((i >> 1) & 1) + 2 * (lane & 3), f = feature + (lane >> 2) + 8 * ((i >> 2) * 2 + (i & 1));
                                const float* from = p.addend + (size_t)(tile.first + q) * p.N + f;
                                y[i] = add2(y[i], pair_of(f < p.N && q < tile.live ? from[0] : 0.f, f < p.N && q + 1 < tile.live ? from[p.N] : 0.f));
                            }
                        if (p.activation == REGIONE_ACT_GELU_TANH) gelu_tanh(y);
                        // (one pass; a sum of kInto leaves in its parts)
#pragma unroll
                        for (int o = 0; o < kOuts; ++o) {
                            const int to = tile.first + c + o * p.rows_cap;
                            uint32_t z[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                float lo, hi;
                                parts_of(y[i], lo, hi);
                                if constexpr (kOuts > 1) {
                                    const float a = lead_part(lo, o + 1 == kOuts), b = lead_part(hi, o + 1 == kOuts);
                                    y[i] = pair_of(lo, hi);
                                    z[i] = pack_bf16x2(a, b);
                                } else {
                                    z[i] = pack_bf16x2(lo, hi);
                                }
                            }
                            // row of the tile t at 64 t, its 16-byte pieces (8 features) turned by t / 2 so that eight rows meet eight banks
                            const int row = (lane & 7) + 8 * (lane >> 4), piece = (lane >> 3) & 1, turn = (row >> 1) & 3;
                            if (PAIR && lane == 0) ptx::bulk_wait_read<0>();         // (the store of the step before)
                            __syncwarp();
                            stmatrix_x4_trans(stage + row * 64 + ((piece ^ turn) << 4), z[0], z[1], z[2], z[3]);
                            stmatrix_x4_trans(stage + row * 64 + (((piece + 2) ^ turn) << 4), z[4], z[5], z[6], z[7]);
                            if (PAIR && c + 16 <= tile.live) {
                                ptx::fence_proxy_async_smem();
                                __syncwarp();
                                if (lane == 0 && feature < p.N) {
                                    store_out(&maps.out, stage, feature, to);
                                    ptx::bulk_commit();
                                }
                            } else {
                                __syncwarp();
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const int q = (lane >> 2) + 8 * i, j = lane & 3;
                                    const uint4 v = *reinterpret_cast<const uint4*>(staging + warp * kStagingBytes + q * 64 + ((j ^ ((q >> 1) & 3)) << 4));
                                    if (c + q < tile.live && feature + 8 * j < p.N)
                                        *reinterpret_cast<uint4*>(p.out + (size_t)(to + q) * p.out_stride + feature + 8 * j) = v;
                                }
                                __syncwarp();
                            }
                        }
                    }
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) arrive_at<PAIR>(ptx::smem_addr(&ctl->acc_empty[a]), rank);
            }
        }
        // ---- the slices of a tile meet --------------------------------------------------------------------------------------
        __syncwarp();
        if (split) {
            ptx::cluster_sync();
            if (warp < kEpiWarps && !ctl->abort_flag) {
                const GroupedTile tile = tile_at<PAIR, OP>(p, ctl, (int)t0, f_tiles, group);
                const float scale = OP == Product::kInto && p.adapter_scale != nullptr ? __ldg(p.adapter_scale + tile.weights) : 1.0f;
                if (OP == Product::kJoined) grid_dependency_wait();
                // pieces of 8 features of a row, dealt over the slices' threads; slices are added in their order
                for (int u = threadIdx.x * p.slices + slice; u < tile.live * (kFeat / 8); u += kEpiWarps * 32 * p.slices) {
                    const int q = u / (kFeat / 8), j = u % (kFeat / 8), f = tile.feature + half * kFeat + 8 * j;
                    if (f >= p.N) continue;
                    const uint32_t at = smem + (q * kFeat + 8 * j) * 4;
                    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    // (several at a time: a load takes 1000 cycles and more; 4 bits: as many as leave the other roles their registers)
                    constexpr int kBatch = FP4 ? 2 : PAIR ? 4 : 8;
                    for (int i0 = 0; i0 < p.slices; i0 += kBatch) {
                        float4 lo[kBatch], hi[kBatch];
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) {
                            if (kBatch > 2 && i0 + i >= p.slices) break;
                            const uint32_t from = ptx::map_rank(at, PAIR ? 2 * (i0 + i) + half : i0 + i);
                            lo[i] = ptx::ld_cluster_f4(from);
                            hi[i] = ptx::ld_cluster_f4(from + 16);
                        }
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) {
                            if (kBatch > 2 && i0 + i >= p.slices) break;
                            y[0] += lo[i].x; y[1] += lo[i].y; y[2] += lo[i].z; y[3] += lo[i].w;
                            y[4] += hi[i].x; y[5] += hi[i].y; y[6] += hi[i].z; y[7] += hi[i].w;
                        }
                    }
                    if (p.bias != nullptr) {
                        const uint4 b = ld_input<OP>(reinterpret_cast<const uint4*>(p.bias + (size_t)tile.weights * p.N + f));
                        y[0] += bf16_lo(b.x); y[1] += bf16_hi(b.x); y[2] += bf16_lo(b.y); y[3] += bf16_hi(b.y);
                        y[4] += bf16_lo(b.z); y[5] += bf16_hi(b.z); y[6] += bf16_lo(b.w); y[7] += bf16_hi(b.w);
                    }
                    if constexpr (OP == Product::kInto)
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] *= scale;
                    if constexpr (OP == Product::kJoined) {
                        const float4* from = reinterpret_cast<const float4*>(p.addend + (size_t)(tile.first + q) * p.N + f);
                        const float4 lo = from[0], hi = from[1];
                        y[0] += lo.x; y[1] += lo.y; y[2] += lo.z; y[3] += lo.w;
                        y[4] += hi.x; y[5] += hi.y; y[6] += hi.z; y[7] += hi.w;
                    }
                    if (p.activation == REGIONE_ACT_GELU_TANH) {
                        uint64_t z[4] = {pair_of(y[0], y[1]), pair_of(y[2], y[3]), pair_of(y[4], y[5]), pair_of(y[6], y[7])};
                        gelu_tanh(z);
#pragma unroll
                        for (int i = 0; i < 4; ++i) parts_of(z[i], y[2 * i], y[2 * i + 1]);
                    }
                    constexpr int kOuts = OP == Product::kInto ? kSumParts : 1;
#pragma unroll
                    for (int i = 0; i < kOuts; ++i) {
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = kOuts > 1 ? lead_part(y[e], i + 1 == kOuts) : y[e];
                        uint4 o;
                        o.x = pack_bf16x2(z[0], z[1]); o.y = pack_bf16x2(z[2], z[3]);
                        o.z = pack_bf16x2(z[4], z[5]); o.w = pack_bf16x2(z[6], z[7]);
                        *reinterpret_cast<uint4*>(p.out + (size_t)(tile.first + i * p.rows_cap + q) * p.out_stride + f) = o;
                    }
                }
            }
            ptx::fence_proxy_async_smem();                // (the ring's next copies write where the sums were)
            ptx::cluster_sync();
        }
    }

    if (kLate<OP>) grid_dependency_wait();
    if (PAIR && warp < kEpiWarps && lane == 0) ptx::bulk_wait_all();
    __syncwarp();
    if ((PAIR || split) && (threadIdx.x & 31) == 0 && *(volatile int*)&ctl->abort_flag)
        for (int r = 0; r < (PAIR ? 2 : 1) * p.slices; ++r)
            asm volatile("st.relaxed.cluster.shared::cluster.s32 [%0], %1;" ::"r"(ptx::map_rank(ptx::smem_addr(&ctl->abort_flag), r)), "r"(1) : "memory");
    ptx::tc_fence_before_sync();
    if (PAIR || split) ptx::cluster_sync(); else __syncthreads();
    ptx::tc_fence_after_sync();
    // Where any role gave up (every CTA of the cluster sees it), copies and products in flight get a quarter of a second before shared and
    // tensor memory are given up.
    if (*(volatile int*)&ctl->abort_flag) {
        for (const long long t0 = clock64(); clock64() - t0 < kGroupedWait / 8;) {}
        if (PAIR || split) ptx::cluster_sync(); else __syncthreads();
    }
    if (warp == kIssuer) free_tmem<PAIR>(tmem, p.tmem_columns);
}

// The waits of the roles, run out in the harmless form: on a barrier that nothing arrives on, with no copy and no product in flight.  One
// of a lone CTA and one of a pair's with the limit, and one with a thousand times that, which sees that another role gave up.
__global__ void grouped_wait_selftest_kernel(long long limit, int32_t* dev_status, long long* out) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    GroupedControl* ctl = reinterpret_cast<GroupedControl*>(smem_raw);
    const uint32_t bar = ptx::smem_addr(&ctl->full[0]);
    if (threadIdx.x > 0) return;
    ptx::mbar_init(bar, 1);
    ptx::fence_barrier_init();
    for (int i = 0; i < 3; ++i) {
        if (i < 2) *(volatile int*)&ctl->abort_flag = 0;
        const long long t0 = clock64();
        const bool done = i == 1 ? grouped_wait<true>(bar, 0, ctl, dev_status, limit)
                                 : grouped_wait<false>(bar, 0, ctl, dev_status, i == 0 ? limit : 1000 * limit);
        const long long spent = clock64() - t0;
        if (out != nullptr) {
            out[3 * i] = done;
            out[3 * i + 1] = spent;
            out[3 * i + 2] = *(volatile int*)&ctl->abort_flag;
        }
    }
    ptx::mbar_inval(bar);
}

// ---- host side -----------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeFn grouped_encode_fn() {
    static EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeFn>(f);
    }();
    return fn;
}

// Rows of K elements (4-bit ones as K / 2 bytes), `sets` of them, in boxes of 128 bytes by `box` rows.
static bool grouped_map(CUtensorMap* map, bool fp4, int rank, const void* at, long long K, long long rows, long long sets,
                        long long row_bytes, int box) {
    EncodeFn fn = grouped_encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)(fp4 ? K / 2 : K), (cuuint64_t)rows, (cuuint64_t)sets};
    const cuuint64_t strides[2] = {(cuuint64_t)row_bytes, (cuuint64_t)(row_bytes * rows)};
    const cuuint32_t boxes[3] = {(cuuint32_t)(fp4 ? kChunkBytes : kChunkBytes / 2), (cuuint32_t)box, 1u}, ones[3] = {1u, 1u, 1u};
    return fn(map, fp4 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(at), dims,
              strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool FP4, bool PAIR, Product OP> static size_t grouped_smem(int ring_bytes) {
    return 1024 + ring_bytes + Roles<FP4, PAIR>::kEpi * kStagingBytes + sizeof(ControlOf<OP>);
}
// One CTA on an SM of a pair, two without.
constexpr int kSmemCta = 232448, kSmemHalf = 113 * 1024;
template <bool FP4, bool PAIR, Product OP> static int grouped_ring(int smem) { return (smem - (int)grouped_smem<FP4, PAIR, OP>(0)) & ~1023; }

template <bool FP4, bool PAIR> static void grouped_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, unsigned blocks, int cluster,
                                                          size_t smem, cudaStream_t st) {
    cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(Roles<FP4, PAIR>::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
}

// Clusters of pairs that the device holds at one time, by their slices of K (1, 2, 4); 0 where the kernel cannot be set up.
template <bool FP4, bool VEC, Product OP> static const int* grouped_pairs(int dev) {
    static int held[kMaxDevices][4] = {};
    int* h = held[dev];
    if (__atomic_load_n(&h[3], __ATOMIC_ACQUIRE)) return h;
    const size_t smem = grouped_smem<FP4, true, OP>(grouped_ring<FP4, true, OP>(kSmemCta));
    if (cudaFuncSetAttribute(grouped_kernel<FP4, true, VEC, OP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemCta) != cudaSuccess ||
        cudaFuncSetAttribute(grouped_kernel<FP4, false, VEC, OP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemCta) != cudaSuccess)
        return nullptr;
    for (int i = 0; i < 3; ++i) {
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[2];
        grouped_config<FP4, true>(cfg, attr, 2u << i, 2 << i, smem, nullptr);
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, grouped_kernel<FP4, true, VEC, OP>, &cfg) != cudaSuccess) {
            cudaGetLastError();
            n = 0;
        }
        __atomic_store_n(&h[i], n, __ATOMIC_RELAXED);
    }
    __atomic_store_n(&h[3], 1, __ATOMIC_RELEASE);
    return h;
}

template <bool FP4, bool PAIR, bool VEC, Product OP>
static int grouped_launch(const MapsOf<OP>& maps, const GroupedArgs& p, int clusters, cudaStream_t st) {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    const int cluster = (PAIR ? 2 : 1) * p.slices;
    grouped_config<FP4, PAIR>(cfg, attr, (unsigned)(clusters * cluster), cluster, grouped_smem<FP4, PAIR, OP>(p.ring_bytes), st);
    return launch_status(launch_counted(&cfg, grouped_kernel<FP4, PAIR, VEC, OP>, maps, p));
}

// `b`, `u`: the adapters' second factors [n_adapters, N, rank] and the rows' products with the first [parts, rows_cap, rank] (kTail).
template <bool FP4, bool VEC, Product OP = Product::kPlain>
static int grouped_run(const void* x, long long x_row_bytes, const void* w, GroupedArgs p, cudaStream_t st, const void* b = nullptr,
                       const void* u = nullptr) {
    constexpr int kElems = FP4 ? 256 : 64;
    const int dev = current_device(), sms = sm_count();
    const int* held = dev < 0 ? nullptr : grouped_pairs<FP4, VEC, OP>(dev);
    if (!held) return REGIONE_CUDA_ERROR;
    p.chunks = (p.K + kElems - 1) / kElems;
    // (joined groups: as if all were where there is one set, and none where the sets take turns)
    const int groups = std::min(OP == Product::kJoined && p.n_weights == 1 ? 1 : p.groups, p.rows_cap), each = (p.rows_cap + groups - 1) / groups;
    const int f_pairs = (p.N + 2 * kFeat - 1) / (2 * kFeat), f_tiles = (p.N + kFeat - 1) / kFeat;
    // What the launch will take, in ns, if every row of the buffer is live and the groups are alike (1280 live rows in a buffer of 8704, K 2048,
    // N 6144: as long as in one of 1280; 205 in 2304 19.4 us, in 205 17.4): what a launch takes before and behind its tiles, and rounds of tiles, each the chunks of a slice times what a chunk takes (no less than 200 by latency; 105 bytes
    // a ns to an SM; the tensor core), and the way of the slices' sums to each other.
    long long best = 0x7fffffffffffffffLL;
    int clusters = 0;
    bool pair = true;
    p.slices = 1;
    p.width = 0;
    for (int i = 0; i < 3; ++i) {
        const int slices = 1 << i;
        if (held[i] < 1 || (i > 0 && 8 * slices > p.chunks)) break;
        const int mine = (p.chunks + slices - 1) / slices;
        for (int width = 32; width <= (FP4 ? 224 : 256); width += 32) {
            const int tiles = f_pairs * groups * ((each + width - 1) / width), rounds = (tiles + held[i] - 1) / held[i];
            const int chunk = std::max(200, std::max(width * 14 / 13, 156 + width * 8 / 13));
            const long long cost = (long long)rounds * ((long long)mine * chunk + (i > 0 ? 2500 + 18 * width : 0)) + 6300;
            if (cost >= best) continue;
            best = cost;
            p.slices = slices;
            clusters = held[i];
        }
    }
    for (int width = 16; width <= 128; width *= 2) {
        const int tiles = f_tiles * (p.rows_cap / width + groups);              // at most, however the rows are spread over the groups
        const int chunk = std::max(200, 156 + width * 16 / 13);
        for (int slices = 1; slices <= 8 && 2 * slices <= std::max(p.chunks, 2); slices *= 2) {
            if (slices > 1 && tiles > sms) break;                               // (the SMs are taken)
            const int rounds = (tiles * slices + sms - 1) / sms, mine = (p.chunks + slices - 1) / slices;
            const int meet = slices > 1 ? 1500 + (slices == 8 ? 40 : 28) * width : 15 * width;
            const long long cost = (long long)rounds * ((long long)mine * chunk + meet) +
                                   (rounds - 1) * 800LL + 4300;
            if (cost >= best) continue;
            best = cost;
            pair = false;
            p.width = width;
            p.slices = slices;
            clusters = std::min(tiles, 4 * sms);
        }
    }
    if (pair && clusters == 0) return REGIONE_CUDA_ERROR;
    if (pair) {
        p.ring_bytes = grouped_ring<FP4, true, OP>(kSmemCta);
        p.tmem_columns = 512;
        p.scale_column = 448;
    } else {
        // two CTAs an SM where four stages (see the scales) leave room for them, with a slice's chunks in the ring if they fit
        const int stage = kTileBytes + p.width * kChunkBytes + (FP4 ? kScaleA + kScaleB : 0), mine = (p.chunks + p.slices - 1) / p.slices;
        p.ring_bytes = std::max(4 * stage, std::min(grouped_ring<FP4, false, OP>(kSmemHalf), std::min(kMaxStages, mine) * stage));
        p.scale_column = p.width <= 64 ? 64 : 128;
        p.tmem_columns = FP4 ? 2 * p.scale_column : std::max(32, p.width);
    }
    MapsOf<OP> maps;
    bool ok = grouped_map(&maps.w, FP4, 3, w, p.K, p.N, OP == Product::kInto ? p.n_adapters : p.n_weights, FP4 ? p.K / 2 : 2LL * p.K, 128);
    for (int i = 0; i < kMaps && ok && (pair || (16 << i) <= p.width); ++i)
        ok = grouped_map(&maps.x[i], FP4, 2, x, p.K, p.rows_cap, 1, x_row_bytes, 16 << i);
    if constexpr (OP == Product::kTail) {
        p.tail = (p.rank + kElems - 1) / kElems;
        ok = ok && grouped_map(&maps.b, false, 3, b, p.rank, p.N, p.n_adapters, 2LL * p.rank, 128);
        for (int i = 0; i < kMaps && ok && (pair || (16 << i) <= p.width); ++i)
            ok = grouped_map(&maps.u[i], false, 2, u, p.rank, (long long)kSumParts * p.rows_cap, 1, 2LL * p.rank, 16 << i);
    }
    if (ok && pair) {
        const cuuint64_t dims[2] = {(cuuint64_t)p.N, (cuuint64_t)p.rows_cap * (OP == Product::kInto ? kSumParts : 1)};
        const cuuint64_t strides[1] = {(cuuint64_t)(2 * p.out_stride)};
        const cuuint32_t box[2] = {32u, 16u}, ones[2] = {1u, 1u};
        ok = grouped_encode_fn()(&maps.out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.out, dims, strides, box, ones,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    }
    if (!ok) return REGIONE_CUDA_ERROR;
    return pair ? grouped_launch<FP4, true, VEC, OP>(maps, p, clusters, st) : grouped_launch<FP4, false, VEC, OP>(maps, p, clusters, st);
}

static GroupedArgs adapter_args(const AdapterCall& c) {
    GroupedArgs p = {};
    p.row_begin = c.row_begin; p.row_end = c.row_end; p.groups = c.groups; p.n_weights = c.n_weights; p.rows_cap = c.rows_cap;
    p.K = c.K; p.N = c.N; p.bias = c.bias; p.activation = c.activation; p.out = c.out; p.out_stride = c.out_stride; p.dev_status = c.dev_status;
    p.adapter = c.adapter; p.n_adapters = c.n_adapters; p.rank = c.rank; p.adapter_scale = c.scale;
    return p;
}

int adapters_into(const AdapterCall& c, uint16_t* u, cudaStream_t st) {
    GroupedArgs p = adapter_args(c);
    p.N = c.rank; p.bias = nullptr; p.activation = REGIONE_ACT_NONE; p.out = u; p.out_stride = c.rank;
    return grouped_run<false, false, Product::kInto>(c.x, 2 * c.x_stride, c.a, p, st);
}

int adapters_tail(const AdapterCall& c, const uint16_t* u, cudaStream_t st) {
    return grouped_run<false, false, Product::kTail>(c.x, 2 * c.x_stride, c.w, adapter_args(c), st, c.b, u);
}

int adapters_joined(const AdapterCall& c, const float* addend, cudaStream_t st) {
    GroupedArgs p = adapter_args(c);
    p.addend = addend;
    return grouped_run<false, false, Product::kJoined>(c.x, 2 * c.x_stride, c.w, p, st);
}

}  // namespace regione

using namespace regione;

int regione::check_grouped(const void* x, const void* w, const void* bias, const void* begin, const void* end, int rows_cap, int groups,
                           int n_weights, int K, int N, int activation, const void* out, long long out_stride) {
    if (!w || (rows_cap && (!x || !out)) || (groups && (!begin || !end))) return REGIONE_INVALID_ARG;
    if (rows_cap < 0 || groups < 0 || n_weights < 1 || K < 1 || N < 1) return REGIONE_INVALID_ARG;
    if (activation != REGIONE_ACT_NONE && activation != REGIONE_ACT_GELU_TANH) return REGIONE_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w) || !aligned16(out) || (bias && !aligned16(bias))) return REGIONE_INVALID_ARG;
    if (out_stride < N) return REGIONE_INVALID_ARG;
    if (N % 8 || out_stride % 8 || out_stride > (1LL << 32) || groups > kMaxGroups || n_weights > 65536 || K > (1 << 20) || N > (1 << 20) || rows_cap > (1 << 24))
        return REGIONE_UNSUPPORTED;
    // tiles are counted in 32 bits
    if (((long long)rows_cap / 16 + groups) * ((N + kFeat - 1) / kFeat) >= 0x10000000LL) return REGIONE_UNSUPPORTED;
    // the distance of two weight sets in a tensor map
    if (2LL * K * N >= 1LL << 40) return REGIONE_UNSUPPORTED;
    return REGIONE_OK;
}

extern "C" int regione_grouped_matmul(const regione_bf16* x, int64_t x_stride, const regione_bf16* w, const regione_bf16* bias,
                                      const int32_t* row_begin, const int32_t* row_end, int rows_cap, int groups, int n_weights,
                                      int K, int N, int activation, regione_bf16* out, int64_t out_stride, int32_t* dev_status,
                                      void* stream) {
    const int rc = check_grouped(x, w, bias, row_begin, row_end, rows_cap, groups, n_weights, K, N, activation, out, out_stride);
    if (rc != REGIONE_OK) return rc;
    if (x_stride < K) return REGIONE_INVALID_ARG;
    if (K % 8 || x_stride % 8 || x_stride > (1LL << 32)) return REGIONE_UNSUPPORTED;
    if (rows_cap == 0 || groups == 0) return REGIONE_OK;
    GroupedArgs p = {};
    p.row_begin = row_begin; p.row_end = row_end; p.groups = groups; p.n_weights = n_weights; p.rows_cap = rows_cap;
    p.K = K; p.N = N; p.bias = bias; p.activation = activation; p.out = out; p.out_stride = out_stride; p.dev_status = dev_status;
    return grouped_run<false, false>(x, 2 * x_stride, w, p, (cudaStream_t)stream);
}

extern "C" int regione_mxfp4_grouped_matmul(const uint8_t* x_q, const uint8_t* x_scale, const uint8_t* w_q, const uint8_t* w_scale,
                                            const regione_bf16* bias, const int32_t* row_begin, const int32_t* row_end,
                                            int rows_cap, int groups, int n_weights, int K, int N, int activation,
                                            regione_bf16* out, int64_t out_stride, int32_t* dev_status, void* stream) {
    const int rc = check_grouped(x_q, w_q, bias, row_begin, row_end, rows_cap, groups, n_weights, K, N, activation, out, out_stride);
    if (rc != REGIONE_OK) return rc;
    if ((rows_cap && !x_scale) || !w_scale || !aligned16(x_scale) || !aligned16(w_scale)) return REGIONE_INVALID_ARG;
    if (K % 128) return REGIONE_UNSUPPORTED;
    if (rows_cap == 0 || groups == 0) return REGIONE_OK;
    GroupedArgs p = {};
    p.row_begin = row_begin; p.row_end = row_end; p.groups = groups; p.n_weights = n_weights; p.rows_cap = rows_cap;
    p.K = K; p.N = N; p.bias = bias; p.activation = activation; p.out = out; p.out_stride = out_stride; p.dev_status = dev_status;
    p.x_scale = x_scale; p.w_scale = w_scale;
    return K % 512 ? grouped_run<true, false>(x_q, K / 2, w_q, p, (cudaStream_t)stream)
                   : grouped_run<true, true>(x_q, K / 2, w_q, p, (cudaStream_t)stream);
}

extern "C" int regione_selftest_group_ranges(const int32_t* row_begin, const int32_t* row_end, int rows_cap, int groups,
                                             int32_t* begin, int32_t* rows) {
    if (!row_begin || !row_end || !begin || !rows || rows_cap < 0 || groups < 0) return -1;
    int outside = 0;
    for (int g = 0; g < groups; ++g) outside += !cut_range(row_begin[g], row_end[g], rows_cap, begin[g], rows[g]);
    return outside;
}

extern "C" int regione_selftest_grouped_wait(long long limit_cycles, int32_t* dev_status, long long* out, void* stream) {
    if (limit_cycles < 1 || limit_cycles > 1000000LL) return REGIONE_INVALID_ARG;
    grouped_wait_selftest_kernel<<<1, 32, sizeof(GroupedControl), (cudaStream_t)stream>>>(limit_cycles, dev_status, out);
    return launch_status(cudaGetLastError());
}
