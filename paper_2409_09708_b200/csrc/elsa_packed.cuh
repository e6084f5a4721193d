// Pieces shared by the attention kernels over packed sequences: the plan's layout, tiles in shared memory and their way out.
#pragma once

#include "elsa_attention_common.cuh"

namespace elsa {
namespace {

// The plan: 16 words of header, then the tiles of 128 and of 256 rows that the sequences are cut into, longest sequences first,
// as {first row of the sequence, its length, number of the tile in it, 0}.
constexpr int kPlanMagic = 0x454c5031;
constexpr int kPlanHeader = 16;          // words
enum { kPlanWordMagic = 0, kPlanWordRows, kPlanWordSequences, kPlanWord128, kPlanWord256 };

__host__ __device__ inline int plan_capacity(int rows, int sequences, int tile_rows)
{
    const long long n = (long long)rows / tile_rows + sequences;      // sum of ceil(len / tile_rows) over sequences with sum(len) <= rows
    return (int)(n < rows ? n : rows);
}

struct PackedTile {
    int begin, len, first;               // the sequence's rows [begin, begin + len); the tile starts at row `first` of the sequence
};

// How many tiles of 128 or 256 rows the plan lists; -1 where it is not one of these rows and sequences (dev_status then tells).
template <int kTileRows>
__device__ __forceinline__ int plan_tiles(const int* plan, int rows, int sequences, uint32_t* dev_status)
{
    int4 head;
    int count;
    asm volatile("ld.global.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(head.x), "=r"(head.y), "=r"(head.z), "=r"(head.w) : "l"(plan));
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(count) : "l"(plan + (kTileRows == 128 ? kPlanWord128 : kPlanWord256)));
    if (head.x != kPlanMagic || head.y != rows || head.z != sequences) {
        if (dev_status != nullptr && threadIdx.x == 0 && blockIdx.x == 0) atomicCAS(dev_status, 0u, (uint32_t)ELSA_ERR_SHAPE | (79u << 8));
        return -1;
    }
    const int most = plan_capacity(rows, sequences, kTileRows);
    return count < most ? count : most;
}

// The entry of a tile, for an index below plan_capacity(): the load alone, so that it may be made ahead.
template <int kTileRows>
__device__ __forceinline__ int4 plan_entry(const int* plan, int rows, int sequences, int index)
{
    const int4* list = reinterpret_cast<const int4*>(plan + kPlanHeader) + (kTileRows == 128 ? 0 : plan_capacity(rows, sequences, 128));
    int4 e;
    asm volatile("ld.global.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(e.x), "=r"(e.y), "=r"(e.z), "=r"(e.w) : "l"(list + index));
    return e;
}

// last_first: tiles of a sequence in reverse order (the costly ones of a causal mask first).  False for an entry that is none.
template <int kTileRows>
__device__ __forceinline__ bool plan_tile(const int4& e, int rows, bool last_first, PackedTile& t)
{
    t.begin = e.x;
    t.len = e.y;
    t.first = (last_first ? (e.y - 1) / kTileRows - e.z : e.z) * kTileRows;
    return e.x >= 0 && e.y > 0 && t.first >= 0 && t.first < e.y && e.x <= rows - e.y;
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// A tile of kD columns: kD = 128 lies as two halves of 64 columns, 128-byte rows; kD = 32 has 64-byte rows.
template <int kD>
struct TileShape {
    static constexpr int kCols = kD < 64 ? kD : 64;                  // columns of a half, and of a TMA box
    static constexpr int kHalves = kD / kCols;
    static constexpr int kRowBytes = kCols * 2;
    __host__ __device__ static constexpr int bytes(int rows) { return rows * kD * 2; }
    __host__ __device__ static constexpr int half_bytes(int rows) { return rows * kRowBytes; }
};

template <int kD, int kRows>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int col, int row)
{
    using T = TileShape<kD>;
#pragma unroll
    for (int h = 0; h < T::kHalves; ++h) tma_load_2d(dst + (uint32_t)(h * T::half_bytes(kRows)), map, bar, col + h * T::kCols, row);
}

// Matrix descriptors of a tile, as the low word (its address) and a high word that is a constant: the issuing warp adds to the low
// word alone, from values that it knows to be the same in all lanes (see uniform()), or each product waits for four register moves.
// K-major: the reduction runs along the head's columns, K step k takes 16 of them.  MN-major: it runs along the tile's rows.
template <int kD>
struct TileDesc {
    using T = TileShape<kD>;
    // stride between groups of eight rows, descriptor version, swizzle of 128 or 64 bytes
    static constexpr uint32_t kHigh = (uint32_t)((8 * T::kRowBytes) >> 4) | 1u << 14 | (kD >= 64 ? 2u : 4u) << 29;
    __host__ __device__ static constexpr uint32_t k_step(int rows, int k)
    {
        return (uint32_t)(((k / (T::kCols / 16)) * T::half_bytes(rows)) >> 4) + (uint32_t)(2 * (k % (T::kCols / 16)));
    }
    static constexpr uint32_t kRowsStep = (16 * T::kRowBytes) >> 4;
    __device__ static __forceinline__ uint32_t k_major(uint32_t tile) { return (tile >> 4) | 1u << 16; }
    template <int kRows>
    __device__ static __forceinline__ uint32_t mn_major(uint32_t tile)
    {
        return (tile >> 4) | (uint32_t)(T::half_bytes(kRows) >> 4) << 16;          // leading offset: the next 64 columns
    }
    __device__ static __forceinline__ uint64_t of(uint32_t low) { return (uint64_t)kHigh << 32 | low; }
};

// The warp's bounded wait for a barrier's phase.  The common case, one test that succeeds, is all that stands where it is called; the rest
// is a function of its own, because the issuing warp's unrolled loop is fetched anew every round and each wait of it in full length
// (with its clock and its report) made that a good part of a tile's time.
__device__ __noinline__ bool packed_wait_on(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* dev_status, uint32_t site)
{
    const bool ok = mbar_wait(bar, parity, abort_flag, dev_status, site);
    return __all_sync(0xFFFFFFFFu, ok);
}
__device__ __forceinline__ bool packed_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* dev_status, uint32_t site)
{
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity))) return true;
    return packed_wait_on(bar, parity, abort_flag, dev_status, site);
}

// A value that all lanes of the (converged) warp hold, in a form that the compiler knows to be one.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __reduce_or_sync(0xFFFFFFFFu, v); }
__device__ __forceinline__ int uniform(int v) { return (int)__reduce_or_sync(0xFFFFFFFFu, (unsigned)v); }

// Rows [from, to) of a tile set to zero by a warp: what lies behind a sequence's end may be anything, and zero times NaN is NaN.
template <int kD, int kRows>
__device__ __forceinline__ void zero_rows(uint32_t tile, int from, int to, int lane)
{
    using T = TileShape<kD>;
    constexpr int kVecs = T::kRowBytes / 16;
#pragma unroll
    for (int h = 0; h < T::kHalves; ++h)
        for (int i = lane; i < (to - from) * kVecs; i += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (uint32_t)(h * T::half_bytes(kRows) + from * T::kRowBytes + i * 16)), "r"(0)
                         : "memory");
}

__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
        "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// A warp's 32 lanes x kCols fp32 columns of tensor memory, times a factor per lane, rounded once, to the first rows_left of 32
// rows of `dst`.  The rows leave through shared memory (32 * kCols * 2 bytes of the warp's own), so that a store covers whole rows.
template <bool kBf16, int kCols>
__device__ __forceinline__ void store_rows(uint32_t t_addr, float factor, uint32_t stage, uint16_t* dst, long long pitch, int rows_left, int lane)
{
    constexpr int kVecs = kCols / 8, kRowsPerStore = 32 / kVecs;
    uint32_t o[kCols / 16][16];
#pragma unroll
    for (int q = 0; q < kCols / 16; ++q) tmem_ld_32x32b_x16(t_addr + (uint32_t)(16 * q), o[q]);
    tmem_wait_ld();
    const int sw = (kVecs == 8 ? lane : lane >> 1) & (kVecs - 1);
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = pack2<kBf16>(__uint_as_float(o[v >> 1][8 * (v & 1) + 2 * e]) * factor, __uint_as_float(o[v >> 1][8 * (v & 1) + 2 * e + 1]) * factor);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + (uint32_t)((lane * kVecs + (v ^ sw)) * 16)),
                     "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                     : "memory");
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int r = i * kRowsPerStore + lane / kVecs, v = lane & (kVecs - 1);
        const int rsw = (kVecs == 8 ? r : r >> 1) & (kVecs - 1);
        uint4 w;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                     : "r"(stage + (uint32_t)((r * kVecs + (v ^ rsw)) * 16)) : "memory");
        if (r < rows_left) *reinterpret_cast<uint4*>(dst + (long long)r * pitch + 8 * v) = w;
    }
    __syncwarp();                        // the staging rows have been read
}

// Columns [0, cols) of `rows` rows, `pitch` values apart, in boxes of box_rows rows and a head's columns (at most 64).
elsa_status make_map_heads(CUtensorMap* map, const void* base, int rows, long long cols, long long pitch, int head_dim, int box_rows, const char* what)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(ELSA_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)pitch * 2};
    cuuint32_t box[2] = {(cuuint32_t)(head_dim < 64 ? head_dim : 64), (cuuint32_t)box_rows};
    cuuint32_t elem[2] = {1, 1};
    CUresult rc = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     head_dim >= 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (rc != CUDA_SUCCESS) return fail(ELSA_ERR_CUDA, "tensor map for %s rejected (CUresult %d)", what, (int)rc);
    return ELSA_OK;
}

// Instruction descriptor: fp32 accumulator, 128 rows, `cols` columns; rows_reduce: B's reduction runs along its rows in memory.
inline uint32_t packed_idesc(elsa_dtype dtype, int cols, bool rows_reduce)
{
    const uint32_t fmt = dtype == ELSA_BF16 ? 1u : 0u;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | (rows_reduce ? 1u << 16 : 0u) | ((uint32_t)(cols >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

}  // namespace
}  // namespace elsa
