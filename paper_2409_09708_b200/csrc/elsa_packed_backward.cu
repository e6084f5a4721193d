// Gradient of the attention over packed sequences.  With p_ij = exp(scale q_i . k_j - lse_i), recomputed from the forward's lse, and
// delta_i = da_i . a_i:
//     ds_ij = p_ij (da_i . v_j - delta_i)
//     dq_i = scale sum_j ds_ij k_j        dk_j = scale sum_i ds_ij q_i        dv_j = sum_i p_ij da_i
// dk and dv also sum over the query heads that share the key head.  Two kernels of one form, because the two directions of the sum
// keep different rows: the first keeps 128 query rows of a head and walks the keys (dq, and delta on the way), the second keeps
// 128 key rows of a key head and walks the queries of all its heads (dk, dv).  That is seven products where one kernel would do with
// five, but no sum leaves the SM unfinished: no atomics, no partial sums in memory, the same bits every time.
//
// Per tile of 64 walked rows (X1, X2 kept; Y1, Y2 walked):      dq kernel        dk, dv kernel
//     S  = X1 Y1^T   (128 x 64 scores)                           q k^T            k q^T
//     T  = X2 Y2^T                                               da v^T           v da^T
//     acc2 += ds Y1  (ds rounded to the 16-bit type)             ds k             ds^T q
//     acc1 += p Y2   (p rounded to the 16-bit type)              -                p^T da
// fp16 has too few exponents for them as they are: of 1000 keys and da of 1e-4 ds is 1 % off, of 16384 keys and 1e-5 it is lost, and large
// ones pass 65504.  So p carries 2^12 there (twelve binary orders more for many keys, four left above 1), and ds the power of two that
// puts the bound of |da_i . (v_j - a_i)| in the sequence, 2 kD times its largest |da| and |v|, just under 2^15; both leave the sums in fp32 at the
// end.  The largest values take a pass of their own over da and v (packed_range_kernel).  bf16 has fp32's exponents.
// All products run on tcgen05; S and T go to fp32 columns of tensor memory, p and ds come back over them as A operands.  A stage of
// S and T has four warps of its own (a row a lane): one stage's exponentials run under the others' products.
// The dq kernel has room in tensor memory for X1 and X2 too: a product of 64 columns with A there takes 32 cycles, with A in shared
// memory 48, for its 6 KB at 128 bytes a cycle (dq of 16 x 1024 rows of 12 heads of 64: 146 and 129 us).
// In the dk, dv kernel lse and delta belong to the walked rows: they come with each tile into shared memory.
// What bounds it is the chain of a tile (S and T, a stage's exponentials, the sums) with as few stages under one another as tensor
// memory holds: a tile of long sequences takes 930 (dq) and 1150 cycles (dk, dv) for heads of 64 columns, where the exponentials
// take 512 and the products 384 and 640; 1340 and 1680 for heads of 128, products 768 and 1280.  Parts of 32 walked rows with twice the stages
// are slower (148 to 165 and 183 to 237 us for 2 x 4736 rows of 8 heads of 64): as many products again to issue.
#include <atomic>
#include <type_traits>

#include "elsa_packed.cuh"

namespace elsa {
namespace {

constexpr int kWalk = 64;                // walked rows of a tile

// kGroups: stages of S and T.  Heads of 128 columns have two of them on an SM.  Narrower heads have one in each of two
// CTAs, where one's beginning and end run under the other's products, or three in one, which keep the tensor core busier once they
// run: chosen by the sequences' mean length (12 heads of 64, us with one and with three: dq of 64 images of 49 to 1024 rows 191 and 224,
// of 16 x 1024 132 and 136, of 6 x 2048 158 and 154; dk and dv of the images 230 and 240, of 32 x 512 97 and 101, of 16 x 1024 166 and 154).
// The mean length stands for what an item walks, and is not the whole of it: heads of 32 cross at about 1400 and 1000 rows (16 x 1024 dq 112 and
// 120, dk and dv 129 and 126; 12 x 1408 146 and 146, 169 and 159), under a causal mask both widths at 1400 to 2000 (heads of 64, 16 x 1024, dk and
// dv 101 and 103; 8 x 2048 161 and 150), so there the two are within a tenth of one another; the group's heads are walked one after another, and
// with 12 query heads on 3 key heads three stages are ahead from 512 rows on (89 and 73; causal 71 and 58), which the rule leaves to the other form.
constexpr int kLongForQueries = 2048, kLongForKeys = 768;

template <int kD, bool kKeys, int kGroupsOf>
struct BackwardShape {
    static constexpr int kGroups = kGroupsOf;
    static constexpr int kPerSm = kGroups == 1 ? 2 : 1;
    static constexpr int kHalf = kGroups == 1 ? 2 : kGroups, kRing = 2 * kHalf;        // tiles of walked rows on their way
    static constexpr int kThreads = kGroups * 128 + 64;
    static constexpr int kTmemCols = 512 / kPerSm;
    static constexpr int kKeptBytes = TileShape<kD>::bytes(128), kWalkBytes = TileShape<kD>::bytes(kWalk);
    static constexpr int kAcc1 = 128 * kGroups, kAcc2 = kAcc1 + kD;  // tensor-memory columns; stage g: S at 128 g, T at 128 g + 64
    enum { kX1 = kAcc1, kX2 = kAcc1 + kD / 2 };                       // X1 and X2 of the first kernel, which has no acc1
    static_assert(kAcc2 + kD <= kTmemCols, "tensor memory");
    static constexpr int kVectorBytes = 2 * kWalk * 4;               // -lse log2(e), -delta
    static constexpr int kSmemBytes = 2 * kKeptBytes + kRing * (2 * kWalkBytes + kVectorBytes) + 1024 /* alignment */ + 256 /* barriers */;
};

struct BackwardParams {
    CUtensorMap map_x1, map_x2;          // boxes of 128 rows
    CUtensorMap map_y1, map_y2;          // boxes of 64 rows
    const int* plan;
    const uint16_t* a;                   // dq kernel: for delta
    const uint16_t* da;
    const uint16_t* v;                   // for the ranges
    const float* lse;                    // [heads][rows]
    float* minus_lse;                    // [heads][rows]: -lse log2(e), made by the dq kernel for the other
    float* minus_delta;                  // [heads][rows]
    uint16_t* out1;                      // dv; in the dq kernel of fp16 dk, for the key tiles' factors
    uint16_t* out2;                      // dq or dk
    const uint16_t* range;               // dq kernel of fp16: dv, where the tiles' ranges stand
    long long range_pitch;
    long long a_pitch, da_pitch, v_pitch, out1_pitch, out2_pitch;
    int rows, sequences, heads, kv_heads, group;
    int causal;
    float scale, scale_log2;
    uint32_t idesc_s, idesc_acc;
    uint32_t* dev_status;
};

// Four bytes global -> shared, zero where `in` is false; without a register in between.
__device__ __forceinline__ void copy_word(uint32_t dst, const float* src, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
// One arrival of this thread on the barrier once its copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint32_t bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// A lane's row of a kept tile, as TMA laid it in shared memory, to tensor memory as an A operand: 16 columns of the head in 8 words.
template <int kD>
__device__ __forceinline__ void keep_rows(uint32_t tile, uint32_t t_lane, int row)
{
    using T = TileShape<kD>;
    const int sw = T::kRowBytes == 128 ? row & 7 : (row >> 1) & 3;
#pragma unroll
    for (int c = 0; c < kD / 2; c += 16) {
        uint32_t x[16];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int at = c / 4 + v, half = at / (T::kCols / 8), vec = at % (T::kCols / 8);       // 16 bytes each
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[4 * v]), "=r"(x[4 * v + 1]), "=r"(x[4 * v + 2]), "=r"(x[4 * v + 3])
                         : "r"(tile + (uint32_t)(half * T::half_bytes(128) + row * T::kRowBytes + (vec ^ sw) * 16)) : "memory");
        }
        tmem_st_32x32b_x16(t_lane + (uint32_t)c, x);
    }
}

// Lane r: sum over a head's columns of x y in row r of the first rows_left of 32 rows (0 in the others).  A row is read by kD / 8 neighbouring
// lanes: with a row a lane each load touched 32 lines, and the kernel's beginning took longer than ten of its tiles
// (8192 rows, 16 heads of 128, causal: 350 to 387 us, by what the first-level cache kept; 331 so).  begin() asks for the first rows, or for all of narrow
// heads, sums() waits for them.
template <bool kBf16, int kD>
struct RowProducts {
    static constexpr int kLanes = kD / 8, kRows = 32 / kLanes;       // lanes of a row, rows of a load
    static constexpr int kAhead = kLanes < 8 ? kLanes : 8;
    uint4 u[kAhead], w[kAhead];
    const uint16_t *x, *y;
    long long x_pitch, y_pitch;
    int rows_left, lane;

    __device__ __forceinline__ static uint4 load(const uint16_t* row, bool in, int sub)
    {
        uint4 r = make_uint4(0u, 0u, 0u, 0u);
        // in its place: the loads are to be on their way while the warp waits for something else
        if (in)
            asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(reinterpret_cast<const uint4*>(row) + sub));
        return r;
    }
    __device__ __forceinline__ void begin(int i0 = 0)
    {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int r = (i0 + i) * kRows + lane / kLanes;
            u[i] = load(x + (long long)r * x_pitch, r < rows_left, lane % kLanes);
            w[i] = load(y + (long long)r * y_pitch, r < rows_left, lane % kLanes);
        }
    }
    __device__ __forceinline__ float sums()
    {
        float mine = 0.f;
#pragma unroll
        for (int i0 = 0; i0 < kLanes; i0 += kAhead) {
            if (i0 > 0) begin(i0);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const uint32_t us[4] = {u[i].x, u[i].y, u[i].z, u[i].w}, ws[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 a = raw2_to_float2<kBf16>(us[e]), b = raw2_to_float2<kBf16>(ws[e]);
                    part = fmaf(a.x, b.x, fmaf(a.y, b.y, part));
                }
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) part += __shfl_xor_sync(0xFFFFFFFFu, part, o);
                const float got = __shfl_sync(0xFFFFFFFFu, part, lane % kRows * kLanes);
                if (lane / kRows == i0 + i) mine = got;
            }
        }
        return mine;
    }
};

constexpr int kPBits = 12;               // fp16: p carries 2^12 in the dk, dv kernel

// The ranges of fp16 stand in rows of the outputs that the dk, dv kernel has yet to write (the workspace has no room for them): of a tile of 128 rows
// and key head the largest |da| and |v|, a word of two fp16, in dv at the tile's first row; the dq kernel makes the factor of a sequence from
// them and leaves it for the dk, dv kernel in dk at the first row of each tile, which only that tile's own CTA reads, before it writes there.
__device__ __forceinline__ long long range_at(long long pitch, const PackedTile& t, int tile, int kv_head, int head_dim)
{
    return (long long)(t.begin + 128 * tile) * pitch + (long long)kv_head * head_dim;
}

// Binary orders that ds carries: 2 kD |da| |v| times 2^that is in [2^14, 2^15), none where it is zero.  The largest values are finite: no overflow.
template <int kD>
__device__ __forceinline__ int ds_orders(uint32_t da_bits, uint32_t v_bits)
{
    const float most = (float)(2 * kD) * (__half2float(__ushort_as_half((unsigned short)da_bits)) * __half2float(__ushort_as_half((unsigned short)v_bits)));
    return most > 0.f ? 15 - ((int)(__float_as_uint(most) >> 23) - 126) : 0;
}
// 2^n, n far inside fp32's exponents.
__device__ __forceinline__ float power_of_two(int n) { return __uint_as_float((uint32_t)(n + 127) << 23); }

// A CTA per tile of 128 rows and key head: the largest |v|, and the largest |da| of the query heads that share it.  Infinities and NaN do not
// count: what they reach has no finite value, the rest keeps its own.  HBM bounds it, da and v are read once: 21 us for 64 images of 49 to 1024
// rows, 12 heads of 64, whose gradient takes 442 with it and 412 in bf16; a launch of 2.3 us for 8 small ones (17.0 and 14.7).  Largest norms of rows
// instead of largest values are a bound three to four orders nearer, 25 us, and more than the orders are worth.
constexpr int kRangeThreads = 256;
struct RangeParams {
    const int* plan;
    const uint16_t *da, *v;
    uint16_t* dv;
    long long da_pitch, v_pitch, dv_pitch;
    int rows, sequences, kv_heads, group;
    uint32_t* dev_status;
};
template <int kD>
__global__ void __launch_bounds__(kRangeThreads) packed_range_kernel(const RangeParams p)
{
    constexpr int kLanes = kD / 8, kRows = kRangeThreads / kLanes, kSteps = 128 / kRows;
    __shared__ uint32_t tops[kRangeThreads / 32];
    pdl_wait_for_predecessors();
    pdl_release_successors();
    PackedTile tile;
    const int kv_head = blockIdx.x % p.kv_heads, index = blockIdx.x / p.kv_heads;
    const int4 entry = plan_entry<128>(p.plan, p.rows, p.sequences, index);
    if (index >= plan_tiles<128>(p.plan, p.rows, p.sequences, p.dev_status) || !plan_tile<128>(entry, p.rows, false, tile)) return;
    const int row0 = threadIdx.x / kLanes, sub = threadIdx.x % kLanes;
    struct Rows {
        uint4 u[kSteps];
    };
    auto load = [&](Rows& r, const uint16_t* x, long long pitch, int head) {
        x += (long long)(tile.begin + tile.first + row0) * pitch + (long long)head * kD + 8 * sub;
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
            r.u[i] = tile.first + row0 + kRows * i < tile.len ? __ldg(reinterpret_cast<const uint4*>(x + (long long)(kRows * i) * pitch)) : make_uint4(0u, 0u, 0u, 0u);
    };
    // |x| of two values as 16-bit integers in order, 0x400 higher: what is not finite is below zero
    uint32_t top_v = 0u, top_da = 0u;
    auto add = [&](const Rows& r, uint32_t& top) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            top = __vmaxs2(top, (r.u[i].x & 0x7fff7fffu) + 0x04000400u);
            top = __vmaxs2(top, (r.u[i].y & 0x7fff7fffu) + 0x04000400u);
            top = __vmaxs2(top, (r.u[i].z & 0x7fff7fffu) + 0x04000400u);
            top = __vmaxs2(top, (r.u[i].w & 0x7fff7fffu) + 0x04000400u);
        }
    };
    Rows v, da;
    load(v, p.v, p.v_pitch, kv_head);
    load(da, p.da, p.da_pitch, kv_head * p.group);
    add(v, top_v);
    for (int h = 1; h < p.group; ++h) {
        const Rows had = da;
        load(da, p.da, p.da_pitch, kv_head * p.group + h);         // on its way while the head before is looked through
        add(had, top_da);
    }
    add(da, top_da);
    auto warp_top = [](uint32_t t) { return __reduce_max_sync(0xFFFFFFFFu, max(t & 0xffffu, t >> 16)); };
    const uint32_t both = warp_top(top_da) << 16 | warp_top(top_v);
    if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = both;
    __syncthreads();
    if (threadIdx.x < 32) {
        const uint32_t t = tops[threadIdx.x % (kRangeThreads / 32)];
        const uint32_t da_bits = __reduce_max_sync(0xFFFFFFFFu, t >> 16), v_bits = __reduce_max_sync(0xFFFFFFFFu, t & 0xffffu);
        auto bits = [](uint32_t t) { return t > 0x400u ? t - 0x400u : 0u; };
        if (threadIdx.x == 0)
            *reinterpret_cast<uint32_t*>(p.dv + range_at(p.dv_pitch, tile, tile.first / 128, kv_head, kD)) = bits(da_bits) << 16 | bits(v_bits);
    }
}

template <bool kBf16, int kD, bool kKeys, int kGroupsOf>
__global__ void __launch_bounds__(BackwardShape<kD, kKeys, kGroupsOf>::kThreads, BackwardShape<kD, kKeys, kGroupsOf>::kPerSm) packed_attention_backward_kernel(const __grid_constant__ BackwardParams p)
{
    using B = BackwardShape<kD, kKeys, kGroupsOf>;
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int kept_heads = kKeys ? p.kv_heads : p.heads;
    const int head = blockIdx.x % kept_heads;
    PackedTile tile;
    // under a causal mask the last query tiles and the first key tiles have the most to do
    if ((int)(blockIdx.x / kept_heads) >= plan_tiles<128>(p.plan, p.rows, p.sequences, p.dev_status)) return;
    const int4 entry = plan_entry<128>(p.plan, p.rows, p.sequences, blockIdx.x / kept_heads);
    if (!plan_tile<128>(entry, p.rows, p.causal != 0 && !kKeys, tile)) return;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t x1_smem = smem_base, x2_smem = smem_base + B::kKeptBytes;
    auto y1_smem = [&](int s) { return smem_base + (uint32_t)(2 * B::kKeptBytes + 2 * s * B::kWalkBytes); };
    auto y2_smem = [&](int s) { return y1_smem(s) + (uint32_t)B::kWalkBytes; };
    const uint32_t vectors = smem_base + (uint32_t)(2 * B::kKeptBytes + 2 * B::kRing * B::kWalkBytes);
    const uint32_t bars = vectors + B::kRing * B::kVectorBytes;
    enum { kXFull = 0, kXMoved = 1, kYFull = 2, kYEmpty = kYFull + B::kRing, kSFull = kYEmpty + B::kRing, kPFull = kSFull + B::kGroups, kDone = kPFull + B::kGroups, kBars };
    auto bar = [&](int which, int i) { return bars + (uint32_t)(8 * (which + i)); };
    const uint32_t tmem_holder_addr = bars + 8 * kBars;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem_raw + (tmem_holder_addr - smem_u32(smem_raw)));
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_holder_addr + 8 - smem_u32(smem_raw)));
    static_assert(8 * kBars + 16 <= 256, "barriers");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kGroups = B::kGroups, kRing = B::kRing, kTmaWarp = 4 * kGroups, kMmaWarp = kTmaWarp + 1;
    // walked tiles: keys from the sequence's start (causal: up to the last kept row); queries to its end (causal: from the first kept row)
    const int walk_from = kKeys && p.causal ? tile.first / kWalk : 0;
    const int walk_end = !kKeys && p.causal && tile.first + 128 < tile.len ? tile.first + 128 : tile.len;
    const int per_head = (walk_end - 1) / kWalk + 1 - walk_from;
    const int n = kKeys ? per_head * p.group : per_head;
    if (warp == kMmaWarp) {
        if (lane == 0) {
            mbar_init(bar(kXFull, 0), 1);
            mbar_init(bar(kXMoved, 0), kGroups > 1 ? 8 : 4);
            for (int s = 0; s < kRing; ++s) {
                mbar_init(bar(kYFull, s), kKeys ? 33 : 1);
                mbar_init(bar(kYEmpty, s), 1);
            }
            for (int g = 0; g < kGroups; ++g) {
                mbar_init(bar(kSFull, g), 1);
                mbar_init(bar(kPFull, g), 4);
            }
            mbar_init(bar(kDone, 0), 1);
            *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        tmem_alloc(tmem_holder_addr, B::kTmemCols);
    }
    [[maybe_unused]] int orders = 0;                                 // that ds carries, 2^orders times its value
    [[maybe_unused]] uint32_t range = 0u;
    if constexpr (!kBf16) {
        if (warp < kTmaWarp) {
            if constexpr (kKeys) {
                // ahead of the barrier: one of the warps writes there at the end
                asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(orders) : "l"(p.out2 + range_at(p.out2_pitch, tile, tile.first / 128, head, kD)) : "memory");
            } else if (lane <= (tile.len - 1) / 128) {
                asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(range) : "l"(p.range + range_at(p.range_pitch, tile, lane, head / p.group, kD)));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;

    bool ok = true;
    auto wait = [&](uint32_t b, int count, uint32_t site) {          // for the count-th completion of a barrier, from 0
        ok = packed_wait(b, (uint32_t)(count & 1), abort_flag, p.dev_status, site);
        return ok;
    };
    if (warp == kTmaWarp) {
        // ------------------------------------------------ TMA producer
        const bool elected = elect_one();
        if (elected) {
            mbar_arrive_expect_tx(bar(kXFull, 0), 2 * B::kKeptBytes);
            load_tile<kD, 128>(x1_smem, &p.map_x1, bar(kXFull, 0), head * kD, tile.begin + tile.first);
            load_tile<kD, 128>(x2_smem, &p.map_x2, bar(kXFull, 0), head * kD, tile.begin + tile.first);
        }
        __syncwarp();
        int walk_head = kKeys ? head * p.group : head / p.group, t = 0;
        for (int it = 0; it < n; ++it, ++t) {
            const int s = it % kRing;
            if (kKeys && t == per_head) { t = 0; ++walk_head; }
            const int row = (walk_from + t) * kWalk;                 // in the sequence
            if (it >= kRing && !wait(bar(kYEmpty, s), it / kRing - 1, 80)) break;
            if (elected) {
                mbar_arrive_expect_tx(bar(kYFull, s), 2 * B::kWalkBytes);
                load_tile<kD, kWalk>(y1_smem(s), &p.map_y1, bar(kYFull, s), walk_head * kD, tile.begin + row);
                load_tile<kD, kWalk>(y2_smem(s), &p.map_y2, bar(kYFull, s), walk_head * kD, tile.begin + row);
            }
            __syncwarp();
            if constexpr (kKeys) {
                const size_t at = (size_t)walk_head * (size_t)p.rows + (size_t)(tile.begin + row);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = lane + 32 * h;
                    const bool in = row + c < tile.len;
                    const uint32_t dst = vectors + (uint32_t)(s * B::kVectorBytes + 4 * c);
                    copy_word(dst, p.minus_lse + (in ? at + c : 0), in);
                    copy_word(dst + 4 * kWalk, p.minus_delta + (in ? at + c : 0), in);
                }
                copies_arrive(bar(kYFull, s));
            }
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------ MMA issuer: S and T of tile it, then the sums of tile it - 1
        using Desc = TileDesc<kD>;
        const uint32_t elected = elect_one() ? 1u : 0u;
        const uint32_t tmem_u = uniform(tmem_base);
        const int tiles = uniform(n), tiles_a_head = uniform(per_head), first_left = uniform(tile.len - walk_from * kWalk);
        const uint32_t x1_desc = Desc::k_major(uniform(smem_base)), x2_desc = x1_desc + (uint32_t)(B::kKeptBytes >> 4);
        const uint32_t y1_rows = Desc::k_major(uniform(y1_smem(0))), y1_cols = Desc::template mn_major<kWalk>(uniform(y1_smem(0)));
        constexpr uint32_t kY2 = (uint32_t)(B::kWalkBytes >> 4);
        // The loop is unrolled over half the ring, so that addresses are constants, and does little else than wait and issue: while this warp
        // works something out, or fetches code, the tensor core idles.  S and T of a tile are issued kGroups - 1 tiles ahead of the sums.
        // y_round is the offset of the half that S and T are in, as descriptors count.
        constexpr int kHalf = B::kHalf, kBehind = kGroups - 1;
        constexpr uint32_t kRound = (uint32_t)(kHalf * 2) * kY2;
        auto scores = [&](int u, uint32_t y_round) {
            const int g = u % kGroups;
            const uint32_t t_s = tmem_u + (uint32_t)(128 * g), y_at = y1_rows + y_round + (uint32_t)(u * 2) * kY2;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int k = 0; k < kD / 16; ++k) {
                    const uint64_t y = Desc::of(y_at + (uint32_t)x * kY2 + Desc::k_step(kWalk, k));
                    if constexpr (kKeys)
                        umma_f16_if(t_s + (uint32_t)(64 * x), Desc::of((x == 0 ? x1_desc : x2_desc) + Desc::k_step(128, k)), y, p.idesc_s, (uint32_t)(k != 0), elected);
                    else
                        umma_f16_ts_if(t_s + (uint32_t)(64 * x), tmem_u + (uint32_t)((x == 0 ? B::kX1 : B::kX2) + 8 * k), y, p.idesc_s, (uint32_t)(k != 0), elected);
                }
            }
            umma_commit_if(bar(kSFull, g), elected);
        };
        auto sums = [&](int u, uint32_t y_round, bool first, int steps) {
            const uint32_t t_s = tmem_u + (uint32_t)(128 * (u % kGroups)), y_at = y1_cols + y_round + (uint32_t)(u * 2) * kY2;
            auto p_step = [&](int k) {
                umma_f16_ts_if(tmem_u + B::kAcc1, t_s + (uint32_t)(8 * k), Desc::of(y_at + kY2 + (uint32_t)k * Desc::kRowsStep), p.idesc_acc,
                               k != 0 ? 1u : first ? 0u : 1u, elected);
            };
            auto ds_step = [&](int k) {
                umma_f16_ts_if(tmem_u + B::kAcc2, t_s + (uint32_t)(64 + 8 * k), Desc::of(y_at + (uint32_t)k * Desc::kRowsStep), p.idesc_acc,
                               k != 0 ? 1u : first ? 0u : 1u, elected);
            };
            if (steps == kWalk / 16) {
                if constexpr (kKeys) {
#pragma unroll
                    for (int k = 0; k < kWalk / 16; ++k) p_step(k);
                }
#pragma unroll
                for (int k = 0; k < kWalk / 16; ++k) ds_step(k);
            } else {
#pragma unroll 1
                for (int k = 0; k < steps; ++k) {
                    if constexpr (kKeys) p_step(k);
                    ds_step(k);
                }
            }
        };
        // the last tile of a head's may be ragged: rows of it, and tiles up to it
        const int last_left = first_left - (tiles_a_head - 1) * kWalk;
        const int last_steps = last_left >= kWalk ? kWalk / 16 : (last_left + 15) / 16;
        int to_last = tiles_a_head, sums_to_last = tiles_a_head;
        if (wait(bar(kKeys ? kXFull : kXMoved, 0), 0, 81)) tc_fence_after();
        uint32_t half = 0, ring_phase = 0;                           // half of the ring, phase of its barriers
        for (int it0 = 0; ok && it0 < tiles + kBehind; it0 += kHalf) {
            const uint32_t y_round = half != 0 ? kRound : 0u, y_before = kRound - y_round;
            const uint32_t round_bars = half != 0 ? 8u * kHalf : 0u, before_bars = 8u * kHalf - round_bars;
#pragma unroll
            for (int u = 0; u < kHalf; ++u) {
                const int it = it0 + u;
                if (it < tiles) {
                    if (!wait(bar(kYFull, u) + round_bars, (int)ring_phase, 82)) break;
                    if (--to_last == 0) {
                        to_last = tiles_a_head;
                        if (last_left < kWalk && (last_left & 15) != 0) {
                            const uint32_t y1 = y1_smem(u) + (half != 0 ? (uint32_t)(kHalf * 2 * B::kWalkBytes) : 0u);
                            zero_rows<kD, kWalk>(y1, last_left, (last_left + 15) & ~15, lane);
                            zero_rows<kD, kWalk>(y1 + B::kWalkBytes, last_left, (last_left + 15) & ~15, lane);
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                    }
                    tc_fence_after();
                    scores(u, y_round);
                }
                // the tile whose sums are due: kBehind tiles back, in this half of the ring or the other
                const int m = it - kBehind, mu = (u + kHalf - kBehind) % kHalf;
                const bool same = u >= kBehind;
                if (m >= 0 && m < tiles) {
                    if (!wait(bar(kPFull, mu % kGroups), kGroups == 1 ? u & 1 : (int)(same ? half : half ^ 1u), 83)) break;
                    tc_fence_after();
                    int steps = kWalk / 16;
                    if (--sums_to_last == 0) {
                        sums_to_last = tiles_a_head;
                        steps = last_steps;
                    }
                    sums(mu, same ? y_round : y_before, m == 0, steps);
                    umma_commit_if(bar(kYEmpty, mu) + (same ? round_bars : before_bars), elected);
                    if (m == tiles - 1) umma_commit_if(bar(kDone, 0), elected);
                }
            }
            if (half != 0) ring_phase ^= 1u;
            half ^= 1u;
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ p and ds, then the sums' way out: group g takes the tiles g, g + kGroups, ...
        const int g = warp >> 2, quarter = warp & 3;
        const int row0 = tile.first + 32 * quarter, row = row0 + lane;                 // kept row, in the sequence
        const bool exists = row < tile.len;
        const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16);
        // delta as the dk, dv kernel of fp16 takes it, ds's power of two less the one that is in p there
        auto handed_delta = [&](float d) { return kBf16 ? d : d * power_of_two(orders - kPBits); };
        float minus_lse = 0.f, minus_delta = 0.f;
        // all keys of the warp's rows are in the first walked tile (under a causal mask those of the first 64 rows, however long the sequence)
        [[maybe_unused]] const bool one_tile = (p.causal && row0 + 32 < tile.len ? row0 + 32 : tile.len) <= kWalk;
        if constexpr (!kKeys) {
            // delta, by each group for itself: an exchange would be one more wait, and the rows are in the caches
            RowProducts<kBf16, kD> delta;
            delta.x = p.a + (long long)(tile.begin + row0) * p.a_pitch + head * kD;
            delta.y = p.da + (long long)(tile.begin + row0) * p.da_pitch + head * kD;
            delta.x_pitch = p.a_pitch; delta.y_pitch = p.da_pitch; delta.rows_left = tile.len - row0; delta.lane = lane;
            delta.begin();
            const float lse = exists ? __ldg(p.lse + (size_t)head * (size_t)p.rows + (size_t)(tile.begin + row)) : 0.f;
            // X1 and X2 to tensor memory, a row a lane, by the first group and the second (or one after the other)
            if (g < 2 && wait(bar(kXFull, 0), 0, 87)) {
                if (g == 0) keep_rows<kD>(x1_smem, t_lane + B::kX1, 32 * quarter + lane);
                if (g == (kGroups > 1 ? 1 : 0)) keep_rows<kD>(x2_smem, t_lane + B::kX2, 32 * quarter + lane);
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kXMoved, 0));
            }
            minus_delta = -delta.sums();
            if constexpr (!kBf16) {
                for (int t = lane + 32; t <= (tile.len - 1) / 128; t += 32) {
                    uint32_t more;
                    asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(more) : "l"(p.range + range_at(p.range_pitch, tile, t, head / p.group, kD)));
                    range = __vmaxu2(range, more);
                }
                orders = ds_orders<kD>(__reduce_max_sync(0xFFFFFFFFu, range >> 16), __reduce_max_sync(0xFFFFFFFFu, range & 0xffffu));
                if (warp == 0 && lane == 0 && head % p.group == 0)
                    *reinterpret_cast<int*>(p.out1 + range_at(p.out1_pitch, tile, tile.first / 128, head / p.group, kD)) = orders;
            }
            if (exists) {
                const size_t at = (size_t)head * (size_t)p.rows + (size_t)(tile.begin + row);
                minus_lse = -1.4426950408889634f * lse;
                if (g == 0) {
                    p.minus_lse[at] = kBf16 ? minus_lse : minus_lse + (float)kPBits;
                    if (!one_tile) p.minus_delta[at] = handed_delta(minus_delta);
                }
            }
        }
        const uint64_t scale2 = f32x2(p.scale_log2, p.scale_log2);
        // fp16: the dq kernel has the power of two for ds in the exponential, the other in T and delta, since its p goes to dv
        [[maybe_unused]] const float minus_lse_ds = kBf16 ? minus_lse : minus_lse + (float)orders;
        [[maybe_unused]] const uint64_t t_factor2 = f32x2(power_of_two(orders - kPBits), power_of_two(orders - kPBits));
        for (int it = g; it < n; it += kGroups) {
            const int s = it % kRing;
            const int walked = (walk_from + it % per_head) * kWalk;                    // first walked row, in the sequence
            if constexpr (kKeys) {
                if (!wait(bar(kYFull, s), it / kRing, 84)) break;                      // lse and delta
            }
            if (!wait(bar(kSFull, g), it / kGroups, 85)) break;
            tc_fence_after();
            if (row0 < tile.len) {
                // columns [lo, hi) take part.  Walked queries behind the sequence's end need no test: their rows of q and da are zero,
                // and so are lse and delta, so that p = 1 meets zeros and ds = 0.
                const int lo = kKeys && p.causal ? row - walked : 0;
                const int hi = kKeys ? kWalk : (p.causal && row + 1 < tile.len ? row + 1 : tile.len) - walked;
                const bool whole = __all_sync(0xFFFFFFFFu, lo <= 0 && hi >= kWalk);
                const uint32_t vec = vectors + (uint32_t)(s * B::kVectorBytes);
                // With all keys of a row in one tile delta is the sum of p T, exact: from the rounded a it is off by half a step of a, as much as
                // ds itself where there are few keys (with 64 of them an eighth of that).  The first tile is the first group's, and no later one
                // has a key for these rows.
                if (!kKeys && one_tile && it == 0) {
                    float sum = 0.f;
#pragma unroll 1
                    for (int c = 0; c < kWalk; c += 16) {
                        uint32_t rs[16], rt[16];
                        tmem_ld_32x32b_x16(t_lane + (uint32_t)(128 * g + c), rs);
                        tmem_ld_32x32b_x16(t_lane + (uint32_t)(128 * g + 64 + c), rt);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float e = exp2_approx(fmaf(__uint_as_float(rs[i]), p.scale_log2, minus_lse));
                            if (c + i < hi) sum = fmaf(e, __uint_as_float(rt[i]), sum);
                        }
                    }
                    minus_delta = -sum;
                    if (exists) p.minus_delta[(size_t)head * (size_t)p.rows + (size_t)(tile.begin + row)] = handed_delta(minus_delta);
                }
                auto unit = [&](auto masked, int u) {
                    uint32_t rs[32], rt[32];
                    tmem_ld_32x32b_x32(t_lane + (uint32_t)(128 * g + 32 * u), rs);
                    tmem_ld_32x32b_x32(t_lane + (uint32_t)(128 * g + 64 + 32 * u), rt);
                    tmem_wait_ld();
                    [[maybe_unused]] uint32_t wp[16];
                    uint32_t wd[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        uint64_t l2[2], d2[2];               // -lse log2(e) and -delta of two columns each
                        if constexpr (kKeys) {
                            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(l2[0]), "=l"(l2[1]) : "r"(vec + (uint32_t)(128 * u + 8 * i)));
                            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(d2[0]), "=l"(d2[1]) : "r"(vec + (uint32_t)(4 * kWalk + 128 * u + 8 * i)));
                        } else {
                            l2[0] = l2[1] = f32x2(minus_lse_ds, minus_lse_ds);
                            d2[0] = d2[1] = f32x2(minus_delta, minus_delta);
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int c = 2 * (i + h), col = 32 * u + c;
                            const float2 e = f32x2_split(f32x2_fma(f32x2(__uint_as_float(rs[c]), __uint_as_float(rs[c + 1])), scale2, l2[h]));
                            float2 pp = make_float2(exp2_approx(e.x), exp2_approx(e.y));
                            const uint64_t t2 = f32x2(__uint_as_float(rt[c]), __uint_as_float(rt[c + 1]));
                            float2 ds = f32x2_split(f32x2_mul(f32x2(pp.x, pp.y), kBf16 || !kKeys ? f32x2_add(t2, d2[h]) : f32x2_fma(t2, t_factor2, d2[h])));
                            if constexpr (decltype(masked)::value) {
                                if (col < lo || col >= hi) pp.x = ds.x = 0.f;
                                if (col + 1 < lo || col + 1 >= hi) pp.y = ds.y = 0.f;
                            }
                            if constexpr (kKeys) wp[i + h] = pack2<kBf16>(pp.x, pp.y);
                            wd[i + h] = pack2<kBf16>(ds.x, ds.y);
                        }
                    }
                    if constexpr (kKeys) tmem_st_32x32b_x16(t_lane + (uint32_t)(128 * g + 16 * u), wp);
                    tmem_st_32x32b_x16(t_lane + (uint32_t)(128 * g + 64 + 16 * u), wd);
                };
                // no sum reads columns behind the last 16 with a walked row, and nothing is worked out where no row of the warp takes part
                auto hide = [&](int u) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = 0u;
                    if constexpr (kKeys) tmem_st_32x32b_x16(t_lane + (uint32_t)(128 * g + 16 * u), w);
                    tmem_st_32x32b_x16(t_lane + (uint32_t)(128 * g + 64 + 16 * u), w);
                };
                if (whole) {
                    unit(std::false_type{}, 0);
                    if (tile.len - walked > 32) unit(std::false_type{}, 1);
                } else {
#pragma unroll 1
                    for (int u = 0; u < 2 && 32 * u < tile.len - walked; ++u) {
                        if (__all_sync(0xFFFFFFFFu, lo >= 32 * u + 32 || hi <= 32 * u)) hide(u);
                        else unit(std::true_type{}, u);
                    }
                }
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kPFull, g));
        }
        if (ok && row0 < tile.len && wait(bar(kDone, 0), 0, 86)) {
            tc_fence_after();
            // all copies and products have ended: the ring is staging room
            const uint32_t stage = y1_smem(0) + (uint32_t)(32 * 2 * TileShape<kD>::kCols * warp);
            const long long first = tile.begin + row0;
            const float ds_scale = kBf16 ? p.scale : p.scale * power_of_two(-orders);
            if constexpr (kKeys) {
                constexpr int kCols = TileShape<kD>::kCols;
#pragma unroll
                for (int o = 0; o < 2; ++o) {                        // dv, then dk; one by each of the first two groups where there are more than one
                    if (kGroups > 1 && o != g) continue;
                    uint16_t* dst = (o == 0 ? p.out1 + first * p.out1_pitch : p.out2 + first * p.out2_pitch) + head * kD;
#pragma unroll
                    for (int c = 0; c < kD; c += kCols)
                        store_rows<kBf16, kCols>(t_lane + (uint32_t)((o == 0 ? B::kAcc1 : B::kAcc2) + c), o == 0 ? (kBf16 ? 1.f : power_of_two(-kPBits)) : ds_scale, stage, dst + c,
                                                 o == 0 ? p.out1_pitch : p.out2_pitch, tile.len - row0, lane);
                }
            } else {
                // the columns, in halves by the first two groups where there are more than one and each half has 32
                constexpr int kCols = kGroups > 1 && kD > 32 ? kD / 2 : kD;
                if (kCols * g < kD)
                    store_rows<kBf16, kCols>(t_lane + (uint32_t)(B::kAcc2 + kCols * g), ds_scale, stage, p.out2 + first * p.out2_pitch + head * kD + kCols * g,
                                             p.out2_pitch, tile.len - row0, lane);
            }
        }
    }
    if (!ok) let_copies_land();
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem_base, B::kTmemCols);
    }
}

template <bool kBf16, int kD, bool kKeys, int kGroupsOf>
elsa_status launch(const BackwardParams& p, cudaStream_t stream, const DeviceInfo& dev)
{
    using B = BackwardShape<kD, kKeys, kGroupsOf>;
    static_assert(2 * B::kRing * B::kWalkBytes >= 4 * B::kGroups * 32 * 2 * TileShape<kD>::kCols, "staging room");
    auto kernel = packed_attention_backward_kernel<kBf16, kD, kKeys, kGroupsOf>;
    static std::atomic<bool> attr_set[64];
    const int slot = dev.device & 63;
    if (!attr_set[slot].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, B::kSmemBytes) != cudaSuccess) {
            cudaError_t e = cudaGetLastError();
            return fail(ELSA_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
        }
        attr_set[slot].store(true, std::memory_order_release);
    }
    const long long items = (long long)plan_capacity(p.rows, p.sequences, 128) * (kKeys ? p.kv_heads : p.heads);
    if (items > 0x7fffffffLL) return fail(ELSA_ERR_SHAPE, "tiles * heads does not fit an int");
    ProfileScope scope(ELSA_KERNEL_PACKED_ATTENTION_BACKWARD, stream);
    cudaError_t e = launch_pdl(kernel, dim3((unsigned)items), dim3(B::kThreads), (size_t)B::kSmemBytes, stream, 1, p);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "packed attention backward launch: %s", cudaGetErrorString(e));
    return launched("packed_attention_backward");
}

template <int kD>
elsa_status launch_range(const BackwardParams& queries, const BackwardParams& keys, cudaStream_t stream)
{
    RangeParams r;
    r.plan = queries.plan; r.da = queries.da; r.v = queries.v; r.dv = keys.out1;
    r.da_pitch = queries.da_pitch; r.v_pitch = queries.v_pitch; r.dv_pitch = keys.out1_pitch;
    r.rows = queries.rows; r.sequences = queries.sequences; r.kv_heads = queries.kv_heads; r.group = queries.group;
    r.dev_status = queries.dev_status;
    const long long items = (long long)plan_capacity(r.rows, r.sequences, 128) * r.kv_heads;
    if (items > 0x7fffffffLL) return fail(ELSA_ERR_SHAPE, "tiles * heads does not fit an int");
    ProfileScope scope(ELSA_KERNEL_PACKED_ATTENTION_BACKWARD, stream);
    cudaError_t e = launch_pdl(packed_range_kernel<kD>, dim3((unsigned)items), dim3(kRangeThreads), 0, stream, 1, r);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "packed range launch: %s", cudaGetErrorString(e));
    return launched("packed_range");
}

template <bool kBf16, int kD>
elsa_status launch_both(const BackwardParams& queries, const BackwardParams& keys, cudaStream_t stream, const DeviceInfo& dev)
{
    elsa_status st;
    if constexpr (!kBf16) {
        if ((st = launch_range<kD>(queries, keys, stream)) != ELSA_OK) return st;
    }
    if constexpr (kD > 64) {
        st = launch<kBf16, kD, false, 2>(queries, stream, dev);
        return st != ELSA_OK ? st : launch<kBf16, kD, true, 2>(keys, stream, dev);
    } else {
        const int mean = queries.rows / queries.sequences;
        st = mean >= kLongForQueries ? launch<kBf16, kD, false, 3>(queries, stream, dev) : launch<kBf16, kD, false, 1>(queries, stream, dev);
        if (st != ELSA_OK) return st;
        return mean >= kLongForKeys ? launch<kBf16, kD, true, 3>(keys, stream, dev) : launch<kBf16, kD, true, 1>(keys, stream, dev);
    }
}

}  // namespace

size_t packed_attention_workspace(int rows, int heads) { return round_up((size_t)rows * (size_t)heads * sizeof(float), 256) * 2; }

elsa_status launch_packed_attention_backward(const elsa_packed_qkv& in, elsa_dtype dtype, const int* plan, int sequences, const uint16_t* a,
                                             long long a_pitch, const float* lse, const uint16_t* da, long long da_pitch, uint16_t* dq,
                                             long long dq_pitch, uint16_t* dk, long long dk_pitch, uint16_t* dv, long long dv_pitch,
                                             void* workspace, uint32_t* dev_status, cudaStream_t stream)
{
    DeviceInfo dev;
    elsa_status st = device_info(&dev);
    if (st != ELSA_OK) return st;
    const int d = in.head_dim, rows = in.rows;
    const long long wide = (long long)in.heads * d, narrow = (long long)in.kv_heads * d;
    BackwardParams q, k;
    q.plan = plan; q.a = a; q.da = da; q.lse = lse;
    q.v = static_cast<const uint16_t*>(in.v); q.v_pitch = in.v_pitch;
    q.range = dv; q.range_pitch = dv_pitch;
    q.minus_lse = static_cast<float*>(workspace);
    q.minus_delta = reinterpret_cast<float*>(static_cast<char*>(workspace) + packed_attention_workspace(rows, in.heads) / 2);
    q.a_pitch = a_pitch; q.da_pitch = da_pitch;
    q.rows = rows; q.sequences = sequences; q.heads = in.heads; q.kv_heads = in.kv_heads; q.group = in.heads / in.kv_heads;
    q.causal = in.causal ? 1 : 0;
    q.scale = in.scale; q.scale_log2 = in.scale * 1.4426950408889634f;
    q.idesc_s = packed_idesc(dtype, kWalk, false);
    q.idesc_acc = packed_idesc(dtype, d, true);
    q.dev_status = dev_status;
    k = q;
    q.out1 = dk; q.out1_pitch = dk_pitch;
    q.out2 = dq; q.out2_pitch = dq_pitch;
    k.out1 = dv; k.out1_pitch = dv_pitch;
    k.out2 = dk; k.out2_pitch = dk_pitch;
    if ((st = make_map_heads(&q.map_x1, in.q, rows, wide, in.q_pitch, d, 128, "q")) != ELSA_OK) return st;
    if ((st = make_map_heads(&q.map_x2, da, rows, wide, da_pitch, d, 128, "da")) != ELSA_OK) return st;
    if ((st = make_map_heads(&q.map_y1, in.k, rows, narrow, in.k_pitch, d, kWalk, "k")) != ELSA_OK) return st;
    if ((st = make_map_heads(&q.map_y2, in.v, rows, narrow, in.v_pitch, d, kWalk, "v")) != ELSA_OK) return st;
    if ((st = make_map_heads(&k.map_x1, in.k, rows, narrow, in.k_pitch, d, 128, "k")) != ELSA_OK) return st;
    if ((st = make_map_heads(&k.map_x2, in.v, rows, narrow, in.v_pitch, d, 128, "v")) != ELSA_OK) return st;
    if ((st = make_map_heads(&k.map_y1, in.q, rows, wide, in.q_pitch, d, kWalk, "q")) != ELSA_OK) return st;
    if ((st = make_map_heads(&k.map_y2, da, rows, wide, da_pitch, d, kWalk, "da")) != ELSA_OK) return st;
    const bool bf = dtype == ELSA_BF16;
    if (d == 32) return bf ? launch_both<true, 32>(q, k, stream, dev) : launch_both<false, 32>(q, k, stream, dev);
    if (d == 64) return bf ? launch_both<true, 64>(q, k, stream, dev) : launch_both<false, 64>(q, k, stream, dev);
    return bf ? launch_both<true, 128>(q, k, stream, dev) : launch_both<false, 128>(q, k, stream, dev);
}

}  // namespace elsa
