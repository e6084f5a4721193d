// Softmax attention over packed sequences: images of many sizes, or prompts of patches, one after another in the rows of qkv.
//     a[i, h] = sum over j of p_ij v[j, h / group],   p_ij = softmax over j of scale q[i, h] . k[j, h / group]
// with j over the rows of i's own sequence (causal: up to i).  Sequences have any length, heads 32, 64 or 128 columns, and a group of
// query heads may share a key head.
//
// Work item = (tile of query rows of one sequence, head); the tiles come from the caller's plan, longest sequences first, and the
// hardware hands them to the SMs as they come free.  An item walks its sequence's keys in tiles of 128 with the running-reference
// form of the softmax, so scores never leave the SM:
//   1. TMA brings the Q tile once and K and V tiles through rings of two stages.
//   2. S = Q K^T on tcgen05 into 128 fp32 columns of tensor memory.
//   3. Four warps, one query row a lane: p = 2^(s scale log2(e) - ref), summed in fp32, rounded to the 16-bit type and written to
//      tensor memory as the A operand.  ref is a whole number at or below the row's maximum so far; where the probabilities of 32 keys
//      sum to more than 2^15 it is raised, and the sum, the tile's P and O are multiplied by the power of two between the two, which
//      changes no mantissa.  So there is no pass for the maximum, and no product that only rescales O.
//   4. O += P V, A from tensor memory, V as it lies in memory.  The rows of V behind a sequence's end (another sequence's, or
//      nobody's) are zeroed in shared memory first: their probabilities are zero, but zero times NaN is not.
// What bounds it is the exponentials: 128 x 128 scores cost the special-function unit 1024 cycles, the two products 512 (64 columns)
// or 1024 (128).  Heads of up to 64 columns: 128 query rows an item and two CTAs on an SM, one's softmax under the other's
// products.  Heads of 128: K and V tiles are twice as large, so one CTA has 256 query rows, two groups of softmax warps that take
// turns with the tensor core; P lies over S there, or tensor memory would not hold both tiles' S and O.
#include <atomic>
#include <type_traits>

#include "elsa_packed.cuh"

namespace elsa {
namespace {

constexpr int kKeys = 128;               // keys of a tile
constexpr int kStages = 2;

template <int kD>
struct ForwardShape {
    static constexpr int kTiles = kD > 64 ? 2 : 1;                   // tiles of 128 query rows
    static constexpr bool kPOverS = kD > 64;
    static constexpr int kThreads = kTiles * 128 + 64;
    static constexpr int kPerSm = kD > 64 ? 1 : 2;
    static constexpr int kTmemCols = kD > 64 ? 512 : 256;
    static constexpr int kPCol = kPOverS ? 0 : 128, kOCol = kPOverS ? 128 : 192;
    static constexpr int kTileBytes = TileShape<kD>::bytes(128);
    static constexpr int kSmemBytes = (kTiles + 2 * kStages) * kTileBytes + 1024 /* alignment */ + 256 /* barriers */;
};

struct ForwardParams {
    CUtensorMap map_q, map_k, map_v;     // boxes of 128 rows
    const int* plan;
    uint16_t* a;
    float* lse;                          // [heads][rows] or NULL
    long long a_pitch;
    int rows, sequences, heads, group;
    int causal;
    float scale_log2;                    // scale * log2(e)
    uint32_t idesc_s, idesc_o;
    uint32_t* dev_status;
};

template <bool kBf16, int kD>
__global__ void __launch_bounds__(ForwardShape<kD>::kThreads, ForwardShape<kD>::kPerSm)
packed_attention_kernel(const __grid_constant__ ForwardParams p)
{
    using F = ForwardShape<kD>;
    constexpr int kTiles = F::kTiles, kTileBytes = F::kTileBytes;
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int head = blockIdx.x % p.heads;
    PackedTile tile;
    if (!plan_tile<kTiles * 128>(p.plan, p.rows, p.sequences, blockIdx.x / p.heads, p.causal != 0, p.dev_status, tile)) return;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    auto q_smem = [&](int q) { return smem_base + (uint32_t)(q * kTileBytes); };
    auto k_smem = [&](int s) { return smem_base + (uint32_t)((kTiles + s) * kTileBytes); };
    auto v_smem = [&](int s) { return smem_base + (uint32_t)((kTiles + kStages + s) * kTileBytes); };
    const uint32_t bars = smem_base + (uint32_t)((kTiles + 2 * kStages) * kTileBytes);
    enum { kQFull = 0, kKFull = 1, kKEmpty = 3, kVFull = 5, kVEmpty = 7, kSFull = 9, kSEmpty = 11, kPFull = 13, kODone = 15, kBars = 17 };
    auto bar = [&](int which, int i) { return bars + (uint32_t)(8 * (which + i)); };
    const uint32_t tmem_holder_addr = bars + 8 * kBars;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem_raw + (tmem_holder_addr - smem_u32(smem_raw)));
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_holder_addr + 8 - smem_u32(smem_raw)));
    static_assert(kStages == 2 && 8 * kBars + 16 <= 256, "barriers");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kTmaWarp = 4 * kTiles, kMmaWarp = kTmaWarp + 1;
    // key tiles of query tile q: none where it has no rows
    auto key_tiles = [&](int q) {
        const int first = tile.first + 128 * q;
        if (first >= tile.len) return 0;
        const int last = p.causal && first + 128 < tile.len ? first + 128 : tile.len;
        return (last - 1) / kKeys + 1;
    };
    const int n0 = key_tiles(0), n1 = kTiles > 1 ? key_tiles(1) : 0;
    const int n = n0 > n1 ? n0 : n1;
    if (warp == kMmaWarp) {
        if (lane == 0) {
            mbar_init(bar(kQFull, 0), 1);
            for (int s = 0; s < kStages; ++s) {
                mbar_init(bar(kKFull, s), 1);
                mbar_init(bar(kKEmpty, s), 1);
                mbar_init(bar(kVFull, s), 1);
                mbar_init(bar(kVEmpty, s), 1);
            }
            for (int q = 0; q < 2; ++q) {
                mbar_init(bar(kSFull, q), 1);
                mbar_init(bar(kSEmpty, q), 4);
                mbar_init(bar(kPFull, q), 4);
                mbar_init(bar(kODone, q), 1);
            }
            *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        tmem_alloc(tmem_holder_addr, F::kTmemCols);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;

    bool ok = true;
    auto wait = [&](uint32_t b, int count, uint32_t site) {          // for the count-th completion of a barrier, from 0
        ok = mbar_wait(b, (uint32_t)(count & 1), abort_flag, p.dev_status, site);
        ok = __all_sync(0xFFFFFFFFu, ok);
        return ok;
    };
    if (warp == kTmaWarp) {
        // ------------------------------------------------ TMA producer
        const bool elected = elect_one();
        const int kv_col = head / p.group * kD;
        if (elected) {
            mbar_arrive_expect_tx(bar(kQFull, 0), (uint32_t)((n1 > 0 ? 2 : 1) * kTileBytes));
            for (int q = 0; q < (n1 > 0 ? 2 : 1); ++q) load_tile<kD, 128>(q_smem(q), &p.map_q, bar(kQFull, 0), head * kD, tile.begin + tile.first + 128 * q);
        }
        __syncwarp();
        for (int j = 0; j < n; ++j) {
            const int s = j % kStages;
            if (j >= kStages && !wait(bar(kKEmpty, s), j / kStages - 1, 70)) break;
            if (elected) {
                mbar_arrive_expect_tx(bar(kKFull, s), (uint32_t)kTileBytes);
                load_tile<kD, 128>(k_smem(s), &p.map_k, bar(kKFull, s), kv_col, tile.begin + kKeys * j);
            }
            __syncwarp();
            if (j >= kStages && !wait(bar(kVEmpty, s), j / kStages - 1, 71)) break;
            if (elected) {
                mbar_arrive_expect_tx(bar(kVFull, s), (uint32_t)kTileBytes);
                load_tile<kD, 128>(v_smem(s), &p.map_v, bar(kVFull, s), kv_col, tile.begin + kKeys * j);
            }
            __syncwarp();
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------ MMA issuer
        const uint32_t elected = elect_one() ? 1u : 0u;
        const uint32_t tmem_u = __reduce_or_sync(0xFFFFFFFFu, tmem_base);
        const int n_of[2] = {n0, n1};
        // S of key tile j for query tile q; the stage's keys are done with after the last query tile that asks for them
        auto scores = [&](int q, int j) {
            if (!wait(bar(kKFull, j % kStages), j / kStages, 72)) return false;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kD / 16; ++k)
                umma_f16_if(tmem_u + (uint32_t)(256 * q), desc_k_major<kD, 128>(q_smem(q), k), desc_k_major<kD, 128>(k_smem(j % kStages), k), p.idesc_s,
                            (uint32_t)(k != 0), elected);
            umma_commit_if(bar(kSFull, q), elected);
            if (q == (j < n1 ? 1 : 0)) umma_commit_if(bar(kKEmpty, j % kStages), elected);
            return true;
        };
        int zeroed = -1;
        auto values = [&](int q, int j) {
            const int s = j % kStages;
            if (!wait(bar(kVFull, s), j / kStages, 73)) return false;
            const int left = tile.len - kKeys * j, steps = left >= kKeys ? kKeys / 16 : (left + 15) / 16;
            if (left < 16 * steps && zeroed != j) {
                zero_rows<kD, 128>(v_smem(s), left, 16 * steps, lane);
                fence_proxy_async_smem();
                __syncwarp();
                zeroed = j;
            }
            if (!wait(bar(kPFull, q), j, 74)) return false;
            tc_fence_after();
            for (int k = 0; k < steps; ++k)
                umma_f16_ts_if(tmem_u + (uint32_t)(256 * q + F::kOCol), tmem_u + (uint32_t)(256 * q + F::kPCol + 8 * k), desc_mn_major<kD, 128>(v_smem(s), k),
                               p.idesc_o, (uint32_t)(j != 0 || k != 0), elected);
            umma_commit_if(bar(kODone, q), elected);
            if (q == (j < n1 ? 1 : 0)) umma_commit_if(bar(kVEmpty, s), elected);
            return true;
        };
        wait(bar(kQFull, 0), 0, 75);
        if constexpr (F::kPOverS) {
            for (int q = 0; ok && q < kTiles; ++q)
                if (n_of[q] > 0 && !scores(q, 0)) break;
            for (int j = 0; ok && j < n; ++j)
#pragma unroll
                for (int q = 0; q < kTiles; ++q) {
                    if (!ok || j >= n_of[q]) continue;
                    // the next scores go over this tile's P: the tensor core takes products in the order they are issued
                    if (values(q, j) && j + 1 < n_of[q]) scores(q, j + 1);
                }
        } else {
            for (int j = 0; ok && j <= n; ++j) {
                if (j < n) {
                    if (j > 0 && !wait(bar(kSEmpty, 0), j - 1, 76)) break;
                    if (!scores(0, j)) break;
                }
                if (j > 0 && !values(0, j - 1)) break;
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ softmax and output
        const int q = warp >> 2, quarter = warp & 3;
        const int nq = q == 0 ? n0 : n1;
        const int row0 = tile.first + 128 * q + 32 * quarter, row = row0 + lane;       // in the sequence
        const uint32_t t_lane = tmem_base + (uint32_t)(256 * q) + ((uint32_t)(quarter * 32) << 16);
        const uint32_t t_p = t_lane + F::kPCol, t_o = t_lane + F::kOCol;
        const int limit = row >= tile.len ? 0 : p.causal ? row + 1 : tile.len;          // keys that take part
        constexpr float kFar = 32768.f;  // no probability above it: inside the 16-bit types and far inside fp32
        const float scale = p.scale_log2;
        float ref = 0.f;
        uint64_t sum2 = f32x2(0.f, 0.f);
        for (int j = 0; j < nq; ++j) {
            if (!wait(bar(kSFull, q), j, 77)) break;
            tc_fence_after();
            const int lim = limit - kKeys * j;                                          // of this tile's keys
            if (row0 >= tile.len) {
                // none of the warp's rows exists: it only keeps its place in the barriers, and no tile ahead of the others in any of them
                if (!F::kPOverS && lane == 0) mbar_arrive(bar(kSEmpty, q));
                if (j > 0 && !wait(bar(kODone, q), j - 1, 78)) break;
                if (lane == 0) mbar_arrive(bar(kPFull, q));
                continue;
            }
            const bool whole = __all_sync(0xFFFFFFFFu, lim >= kKeys);
            const int left = tile.len - kKeys * j;
            const int read = left >= kKeys ? kKeys : (left + 15) / 16 * 16;             // keys that the second product reads
            const int most = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)(lim < 0 ? 0 : lim > kKeys ? kKeys : lim));
            const int units = (most + 31) / 32;                                         // of 32 keys with anything to exponentiate
            auto exp16 = [&](auto masked, const uint32_t* r, int col0, uint64_t& part2, uint32_t (&w)[8]) {
                const uint64_t scale2 = f32x2(scale, scale), minus_ref = f32x2(-ref, -ref);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 a = f32x2_split(f32x2_fma(f32x2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), scale2, minus_ref));
                    float e0 = exp2_approx(a.x), e1 = exp2_approx(a.y);
                    if constexpr (decltype(masked)::value) {
                        if (col0 + 2 * i >= lim) e0 = 0.f;
                        if (col0 + 2 * i + 1 >= lim) e1 = 0.f;
                    }
                    part2 = f32x2_add(part2, f32x2(e0, e1));
                    w[i] = pack2<kBf16>(e0, e1);
                }
            };
            auto top_of = [&](auto masked, const uint32_t* r, int col0) {
                float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    if (!decltype(masked)::value || col0 + i < lim) t0 = fmaxf(t0, __uint_as_float(r[i]) * scale);
                    if (!decltype(masked)::value || col0 + i + 1 < lim) t1 = fmaxf(t1, __uint_as_float(r[i + 1]) * scale);
                }
                return fmaxf(floorf(fmaxf(t0, t1)), -3.0e38f);       // finite for scores of minus infinity
            };
            auto rise = [&](float to, int written) {
                const float up = fminf(to - ref, 127.f);
                const float factor = __uint_as_float((uint32_t)(127 - (int)up) << 23);          // 2^-up, 0 from 127 on
                ref = to;
                sum2 = f32x2_mul(sum2, f32x2(factor, factor));
                tmem_wait_st();
                for (int c = 0; c < written; c += 8) {
                    uint32_t w[8];
                    tmem_ld_32x32b_x8(t_p + (uint32_t)c, w);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 v = raw2_to_float2<kBf16>(w[i]);
                        w[i] = pack2<kBf16>(v.x * factor, v.y * factor);
                    }
                    tmem_st_32x32b_x8(t_p + (uint32_t)c, w);
                }
                if (j > 0) {
                    for (int c = 0; c < kD; c += 16) {
                        uint32_t w[16];
                        tmem_ld_32x32b_x16(t_o + (uint32_t)c, w);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * factor);
                        tmem_st_32x32b_x16(t_o + (uint32_t)c, w);
                    }
                }
            };
            auto columns = [&](auto masked, const uint32_t* r, int u) {
                uint64_t part2;
                auto once = [&]() {
                    part2 = f32x2(0.f, 0.f);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t w[8];
                        exp16(masked, r + 16 * h, 32 * u + 16 * h, part2, w);
                        tmem_st_32x32b_x8(t_p + (uint32_t)(16 * u + 8 * h), w);
                    }
                };
                once();
                const float2 part = f32x2_split(part2);
                const bool far = part.x + part.y > kFar;
                if (__any_sync(0xFFFFFFFFu, far)) {
                    const float top = top_of(masked, r, 32 * u);
                    rise(far && top > ref ? top : ref, 16 * u);
                    once();
                }
                sum2 = f32x2_add(sum2, part2);
            };
            auto unit = [&](const uint32_t* r, int u) {
                if (whole) columns(std::false_type{}, r, u);
                else columns(std::true_type{}, r, u);
            };
            uint32_t ra[32], rb[32];
            tmem_ld_32x32b_x32(t_lane, ra);
            tmem_wait_ld();
            if (j == 0) ref = whole ? top_of(std::false_type{}, ra, 0) : top_of(std::true_type{}, ra, 0);
            // O takes the last tile's product before P is written again
            if (j > 0 && !wait(bar(kODone, q), j - 1, 78)) break;
            tc_fence_after();
            auto scores_read = [&]() {                               // the next tile's scores may take their place
                if constexpr (!F::kPOverS) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(kSEmpty, q));
                }
            };
            if (units == 0) scores_read();
            for (int u = 0; u < units; u += 2) {
                tmem_wait_ld();
                if (u + 1 < units) tmem_ld_32x32b_x32(t_lane + (uint32_t)(32 * (u + 1)), rb);
                else scores_read();
                unit(ra, u);
                if (u + 1 < units) {
                    tmem_wait_ld();
                    if (u + 2 < units) tmem_ld_32x32b_x32(t_lane + (uint32_t)(32 * (u + 2)), ra);
                    else scores_read();
                    unit(rb, u + 1);
                }
            }
            for (int c = 32 * units; c < read; c += 16) {
                const uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
                tmem_st_32x32b_x8(t_p + (uint32_t)(c / 2), w);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kPFull, q));
        }
        if (ok && row0 < tile.len && wait(bar(kODone, q), nq - 1, 78)) {
            tc_fence_after();
            const float2 both = f32x2_split(sum2);
            const float sum = both.x + both.y, inv = 1.0f / sum;
            if (p.lse != nullptr && row < tile.len)
                p.lse[(size_t)head * (size_t)p.rows + (size_t)(tile.begin + row)] = (ref + log2f(sum)) * 0.6931471805599453f;
            // Q has been read for the last time: its quarter is the warp's staging room
            const uint32_t stage = q_smem(q) + (uint32_t)(quarter * (kTileBytes / 4));
            uint16_t* dst = p.a + (long long)(tile.begin + row0) * p.a_pitch + head * kD;
#pragma unroll
            for (int c = 0; c < TileShape<kD>::kHalves; ++c)
                store_rows<kBf16, TileShape<kD>::kCols>(t_o + (uint32_t)(c * TileShape<kD>::kCols), inv, stage, dst + c * TileShape<kD>::kCols, p.a_pitch,
                                                        tile.len - row0, lane);
        }
    }
    if (!ok) let_copies_land();
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem_base, F::kTmemCols);
    }
}

// One CTA makes the plan: offsets that are no offsets make an empty one, and dev_status tells.  Sequences go into buckets by their number of
// 128-row tiles, most first (from 1023 tiles on they share one); where they stand inside a bucket does not matter.
__global__ void __launch_bounds__(1024) packed_plan_kernel(const int32_t* __restrict__ offsets, int sequences, int rows, int* plan, uint32_t* dev_status)
{
    __shared__ int count[2][1024], scan[2][1024];
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int tid = threadIdx.x, lane = tid & 31;
    count[0][tid] = 0;
    count[1][tid] = 0;
    int bad = 0;
    for (int i = tid; i < sequences; i += 1024) {
        const int b = __ldg(offsets + i), e = __ldg(offsets + i + 1);
        bad |= b < 0 || e < b || e > rows;
    }
    bad = __syncthreads_or(bad);
    auto bucket_of = [](int tiles) { return tiles < 1023 ? tiles : 1023; };
    if (!bad) {
        for (int i = tid; i < sequences; i += 1024) {
            const int len = __ldg(offsets + i + 1) - __ldg(offsets + i);
            if (len == 0) continue;
            const int n = (len - 1) / 128 + 1;
            atomicAdd(&count[0][bucket_of(n)], n);
            atomicAdd(&count[1][bucket_of(n)], (n + 1) / 2);
        }
    }
    __syncthreads();
    // entries of the buckets above one's own
    const int mine = 1023 - tid;
    int v[2] = {count[0][mine], count[1][mine]};
    for (int l = 0; l < 2; ++l) scan[l][tid] = v[l];
    __syncthreads();
    for (int o = 1; o < 1024; o <<= 1) {
        int add[2];
        for (int l = 0; l < 2; ++l) add[l] = tid >= o ? scan[l][tid - o] : 0;
        __syncthreads();
        for (int l = 0; l < 2; ++l) scan[l][tid] += add[l];
        __syncthreads();
    }
    if (tid == 1023) {
        plan[kPlanWordMagic] = kPlanMagic;
        plan[kPlanWordRows] = rows;
        plan[kPlanWordSequences] = sequences;
        plan[kPlanWord128] = scan[0][tid];
        plan[kPlanWord256] = scan[1][tid];
        if (bad && dev_status != nullptr) atomicCAS(dev_status, 0u, (uint32_t)ELSA_ERR_SHAPE | (69u << 8));
    }
    for (int l = 0; l < 2; ++l) count[l][mine] = scan[l][tid] - v[l];
    __syncthreads();
    if (bad) return;
    int4* list[2] = {reinterpret_cast<int4*>(plan + kPlanHeader), reinterpret_cast<int4*>(plan + kPlanHeader) + plan_capacity(rows, sequences, 128)};
    for (int base = tid - lane; base < sequences; base += 1024) {
        const int i = base + lane;
        int begin = 0, len = 0, at[2] = {0, 0};
        if (i < sequences) {
            begin = __ldg(offsets + i);
            len = __ldg(offsets + i + 1) - begin;
        }
        const int n = len > 0 ? (len - 1) / 128 + 1 : 0;
        if (n > 0) {
            at[0] = atomicAdd(&count[0][bucket_of(n)], n);
            at[1] = atomicAdd(&count[1][bucket_of(n)], (n + 1) / 2);
        }
        if (n <= 4) {
            for (int t = 0; t < n; ++t) list[0][at[0] + t] = make_int4(begin, len, t, 0);
            for (int t = 0; t < (n + 1) / 2; ++t) list[1][at[1] + t] = make_int4(begin, len, t, 0);
        }
        // long ones by the whole warp
        for (unsigned todo = __ballot_sync(0xFFFFFFFFu, n > 4); todo != 0; todo &= todo - 1) {
            const int from = __ffs(todo) - 1;
            const int b = __shfl_sync(0xFFFFFFFFu, begin, from), l = __shfl_sync(0xFFFFFFFFu, len, from), m = __shfl_sync(0xFFFFFFFFu, n, from);
            const int a0 = __shfl_sync(0xFFFFFFFFu, at[0], from), a1 = __shfl_sync(0xFFFFFFFFu, at[1], from);
            for (int t = lane; t < m; t += 32) list[0][a0 + t] = make_int4(b, l, t, 0);
            for (int t = lane; t < (m + 1) / 2; t += 32) list[1][a1 + t] = make_int4(b, l, t, 0);
        }
    }
}

template <bool kBf16, int kD>
elsa_status launch(const ForwardParams& p, cudaStream_t stream, const DeviceInfo& dev)
{
    using F = ForwardShape<kD>;
    auto kernel = packed_attention_kernel<kBf16, kD>;
    static std::atomic<bool> attr_set[64];
    const int slot = dev.device & 63;
    if (!attr_set[slot].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmemBytes) != cudaSuccess) {
            cudaError_t e = cudaGetLastError();
            return fail(ELSA_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
        }
        attr_set[slot].store(true, std::memory_order_release);
    }
    const long long items = (long long)plan_capacity(p.rows, p.sequences, F::kTiles * 128) * p.heads;
    if (items > 0x7fffffffLL) return fail(ELSA_ERR_SHAPE, "tiles * heads does not fit an int");
    ProfileScope scope(ELSA_KERNEL_PACKED_ATTENTION, stream);
    cudaError_t e = launch_pdl(kernel, dim3((unsigned)items), dim3(F::kThreads), (size_t)F::kSmemBytes, stream, 1, p);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "packed attention launch: %s", cudaGetErrorString(e));
    return launched("packed_attention");
}

}  // namespace

size_t packed_plan_bytes(int rows, int sequences)
{
    return kPlanHeader * sizeof(int) + ((size_t)plan_capacity(rows, sequences, 128) + (size_t)plan_capacity(rows, sequences, 256)) * sizeof(int4);
}

elsa_status launch_packed_plan(const int32_t* offsets, int sequences, int rows, int* plan, uint32_t* dev_status, cudaStream_t stream)
{
    DeviceInfo dev;
    elsa_status st = device_info(&dev);
    if (st != ELSA_OK) return st;
    ProfileScope scope(ELSA_KERNEL_PACKED_ATTENTION, stream);
    cudaError_t e = launch_pdl(packed_plan_kernel, dim3(1), dim3(1024), 0, stream, 1, offsets, sequences, rows, plan, dev_status);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "packed plan launch: %s", cudaGetErrorString(e));
    return launched("packed_plan");
}

elsa_status launch_packed_attention(const elsa_packed_qkv& in, elsa_dtype dtype, const int* plan, int sequences, uint16_t* a, long long a_pitch,
                                    float* lse, uint32_t* dev_status, cudaStream_t stream)
{
    DeviceInfo dev;
    elsa_status st = device_info(&dev);
    if (st != ELSA_OK) return st;
    ForwardParams p;
    const int d = in.head_dim;
    if ((st = make_map_heads(&p.map_q, in.q, in.rows, (long long)in.heads * d, in.q_pitch, d, 128, "q")) != ELSA_OK) return st;
    if ((st = make_map_heads(&p.map_k, in.k, in.rows, (long long)in.kv_heads * d, in.k_pitch, d, 128, "k")) != ELSA_OK) return st;
    if ((st = make_map_heads(&p.map_v, in.v, in.rows, (long long)in.kv_heads * d, in.v_pitch, d, 128, "v")) != ELSA_OK) return st;
    p.plan = plan; p.a = a; p.lse = lse; p.a_pitch = a_pitch;
    p.rows = in.rows; p.sequences = sequences; p.heads = in.heads; p.group = in.heads / in.kv_heads;
    p.causal = in.causal ? 1 : 0;
    p.scale_log2 = in.scale * 1.4426950408889634f;
    p.idesc_s = packed_idesc(dtype, kKeys, false);
    p.idesc_o = packed_idesc(dtype, d, true);
    p.dev_status = dev_status;
    const bool bf = dtype == ELSA_BF16;
    if (d == 32) return bf ? launch<true, 32>(p, stream, dev) : launch<false, 32>(p, stream, dev);
    if (d == 64) return bf ? launch<true, 64>(p, stream, dev) : launch<false, 64>(p, stream, dev);
    return bf ? launch<true, 128>(p, stream, dev) : launch<false, 128>(p, stream, dev);
}

}  // namespace elsa
