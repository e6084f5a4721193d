// Softmax attention over packed sequences: images of many sizes, or prompts of patches, one after another in the rows of qkv.
//     a[i, h] = sum over j of p_ij v[j, h / group],   p_ij = softmax over j of scale q[i, h] . k[j, h / group]
// with j over the rows of i's own sequence (causal: up to i).  Sequences have any length, heads 32, 64 or 128 columns, and a group of
// query heads may share a key head.
//
// Work item = (tile of query rows of one sequence, head); the tiles come from the caller's plan, longest sequences first, and the
// hardware hands them to the SMs as they come free.  An item walks its sequence's keys in tiles with the running-reference
// form of the softmax, so scores never leave the SM:
//   1. TMA brings the Q tile and the first K tile, then one stage of two at a time: V of a tile and K of the next, for which the
//      products of one step ask together.
//   2. S = Q K^T on tcgen05 into fp32 columns of tensor memory.
//   3. Four warps, one query row a lane: p = 2^(s scale log2(e) - ref), summed in fp32, rounded to the 16-bit type and written over the
//      scores it came from as the A operand.  ref is a whole number at or below the row's maximum so far; where the probabilities of a
//      chunk sum to more than 2^15 it is raised, and the sum, the tile's P and O are multiplied by the power of two between the two, which
//      changes no mantissa.  So there is no pass for the maximum, and no product that only rescales O.  The tensor core takes P in
//      the inputs' type: an error of half a step a probability, about as much in the output as its own rounding.
//   4. O += P V, A from tensor memory, V as it lies in memory, and the next tile's S into the place of this P.  The rows of V behind a
//      sequence's end (another sequence's, or nobody's) are zeroed in shared memory first: their probabilities are zero, but zero times
//      NaN is not.
// Tensor memory sets the tiles.  Heads of up to 64 columns: S of 64 keys and O are 128 columns, so four CTAs of 128 query rows share an
// SM, each waiting in its turn (16 x 1024 rows of 12 heads: two CTAs with 128 keys 122 us, the first form of four 99, now 75).  Heads of 128: S
// of 128 keys and O are 256 columns, one CTA has two query tiles whose warps take turns with the tensor core (2 x 4096 rows of 8 heads: forms
// with 64 keys 152 to 260 us, the first of this 127, now 120).  What bounds it: the special-function unit's 16 exponentials a clock, 512
// cycles for 128 x 64 scores.  The loop of narrow heads took 622 of them when 2 x 4736 rows of 8 heads took 132 us; they take 123 to 125 now (740
// TFLOP/s).  With 128 columns products of 1024 cycles for 128 x 128 scores come on top, and the two tiles' waits for them
// (8192 causal rows of 16 heads: 1.26 PFLOP/s, less at the power limit, where the clock falls from 1.96 to 1.65 GHz).
#include <atomic>
#include <type_traits>

#include "elsa_packed.cuh"

namespace elsa {
namespace {

template <int kD>
struct ForwardShape {
    static constexpr int kTiles = kD > 64 ? 2 : 1;                   // tiles of 128 query rows
    static constexpr int kKeys = kD > 64 ? 128 : 64;                 // keys of a tile
    static constexpr int kChunk = kD > 64 ? 64 : 32;                 // scores of a row in registers at a time
    static constexpr int kStages = 2;                                // of V of a tile and K of the next
    static constexpr int kThreads = kTiles * 128 + 64;
    static constexpr int kPerSm = kD > 64 ? 1 : 4;
    static constexpr int kTmemCols = 512 / kPerSm;
    static constexpr int kTileCols = kTmemCols / kTiles;             // a query tile's share: its scores, then O
    static constexpr int kOCol = kKeys;
    static constexpr int kQBytes = TileShape<kD>::bytes(128), kKvBytes = TileShape<kD>::bytes(kKeys);
    static constexpr int kSmemBytes = kTiles * kQBytes + 2 * kStages * kKvBytes + 1024 /* alignment */ + 256 /* barriers */;
    static_assert(kOCol + kD <= kTileCols, "tensor memory");
    static_assert(kStages % 2 == 0, "a tile's parity is its stage's");
};

struct ForwardParams {
    CUtensorMap map_q;                   // boxes of 128 rows
    CUtensorMap map_k, map_v;            // boxes of a key tile's rows
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
    constexpr int kTiles = F::kTiles, kKeys = F::kKeys, kStages = F::kStages;
    constexpr int kTmaWarp = 4 * kTiles, kMmaWarp = kTmaWarp + 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == kTmaWarp && lane == 0) {
        prefetch_map(&p.map_q);
        prefetch_map(&p.map_k);
        prefetch_map(&p.map_v);
    }
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int head = blockIdx.x % p.heads;
    PackedTile tile;
    if ((int)(blockIdx.x / p.heads) >= plan_tiles<kTiles * 128>(p.plan, p.rows, p.sequences, p.dev_status)) return;
    const int4 entry = plan_entry<kTiles * 128>(p.plan, p.rows, p.sequences, blockIdx.x / p.heads);
    if (!plan_tile<kTiles * 128>(entry, p.rows, p.causal != 0, tile)) return;

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    auto q_smem = [&](int q) { return smem_base + (uint32_t)(q * F::kQBytes); };
    auto k_smem = [&](int s) { return smem_base + (uint32_t)(kTiles * F::kQBytes + s * F::kKvBytes); };
    auto v_smem = [&](int s) { return k_smem(kStages + s); };
    const uint32_t bars = k_smem(2 * kStages);
    enum { kQFull = 0, kKvFull = 1, kKvEmpty = kKvFull + kStages, kSFull = kKvEmpty + kStages, kPFull = kSFull + kTiles, kODone = kPFull + kTiles,
           kBars = kODone + kTiles };
    auto bar = [&](int which, int i) { return bars + (uint32_t)(8 * (which + i)); };
    const uint32_t tmem_holder_addr = bars + 8 * kBars;
    uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem_raw + (tmem_holder_addr - smem_u32(smem_raw)));
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_holder_addr + 8 - smem_u32(smem_raw)));
    static_assert(8 * kBars + 16 <= 256, "barriers");

    // key tiles of query tile q: none where it has no rows
    auto key_tiles = [&](int q) {
        const int first = tile.first + 128 * q;
        if (first >= tile.len) return 0;
        const int last = p.causal && first + 128 < tile.len ? first + 128 : tile.len;
        return (last - 1) / kKeys + 1;
    };
    const int n0 = key_tiles(0), n1 = kTiles > 1 ? key_tiles(1) : 0;
    const int n = n0 > n1 ? n0 : n1;
    const int kv_col = head / p.group * kD;
    bool ok = true;
    auto wait = [&](uint32_t b, int count, uint32_t site) {          // for the count-th completion of a barrier, from 0
        ok = packed_wait(b, (uint32_t)(count & 1), abort_flag, p.dev_status, site);
        return ok;
    };
    // Stage j % kStages has V of tile j and K of tile j + 1, which the products of one step ask for; K of tile 0 comes with Q, into the
    // stage before the first.
    auto load_stage = [&](int j) {
        const int s = j % kStages;
        mbar_arrive_expect_tx(bar(kKvFull, s), (uint32_t)((j + 1 < n ? 2 : 1) * F::kKvBytes));
        load_tile<kD, kKeys>(v_smem(s), &p.map_v, bar(kKvFull, s), kv_col, tile.begin + kKeys * j);
        if (j + 1 < n) load_tile<kD, kKeys>(k_smem(s), &p.map_k, bar(kKvFull, s), kv_col, tile.begin + kKeys * (j + 1));
    };
    if (warp == kTmaWarp) {
        if (lane == 0) {
            mbar_init(bar(kQFull, 0), 1);
            for (int s = 0; s < kStages; ++s) {
                mbar_init(bar(kKvFull, s), 1);
                mbar_init(bar(kKvEmpty, s), 1);
            }
            for (int q = 0; q < kTiles; ++q) {
                mbar_init(bar(kSFull, q), 1);
                mbar_init(bar(kPFull, q), 4);
                mbar_init(bar(kODone, q), 1);
            }
            *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            // the first tiles are on their way before the others of the CTA are ready
            mbar_arrive_expect_tx(bar(kQFull, 0), (uint32_t)((n1 > 0 ? 2 : 1) * F::kQBytes + F::kKvBytes));
            load_tile<kD, 128>(q_smem(0), &p.map_q, bar(kQFull, 0), head * kD, tile.begin + tile.first);
            load_tile<kD, kKeys>(k_smem(kStages - 1), &p.map_k, bar(kQFull, 0), kv_col, tile.begin);
            if (n1 > 0) load_tile<kD, 128>(q_smem(kTiles - 1), &p.map_q, bar(kQFull, 0), head * kD, tile.begin + tile.first + 128);
            for (int j = 0; j < kStages - 1 && j < n; ++j) load_stage(j);
        }
        __syncwarp();
    }
    if (warp == kMmaWarp) tmem_alloc(tmem_holder_addr, F::kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_holder;

    if (warp == kTmaWarp) {
        // ------------------------------------------------ TMA producer
        for (int j = kStages - 1; j < n; ++j) {
            if (!wait(bar(kKvEmpty, j % kStages), (j + 1) / kStages - 1, 70)) break;
            if (lane == 0) load_stage(j);
            __syncwarp();
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------ MMA issuer: the first tile's scores, then P V of a tile and the scores of the next, which take its
        // place.  The tensor core idles while this warp does anything but issue (a wait that is over already costs 60 cycles, a product of 128
        // columns takes 64), so a step has one wait for K and V, and its products are unrolled with constant addresses and predicates.
        using Desc = TileDesc<kD>;
        const uint32_t elected = elect_one() ? 1u : 0u;
        const uint32_t tmem_u = uniform(tmem_base);
        const int len = uniform(tile.len), tiles0 = uniform(n0), tiles1 = uniform(n1), tiles = tiles0 > tiles1 ? tiles0 : tiles1;
        const uint32_t q_desc = Desc::k_major(uniform(smem_base)), k_desc = q_desc + (uint32_t)((kTiles * F::kQBytes) >> 4);
        const uint32_t v_desc = Desc::template mn_major<kKeys>(uniform(v_smem(0)));
        auto scores = [&](int q, int s) {
#pragma unroll
            for (int k = 0; k < kD / 16; ++k)
                umma_f16_if(tmem_u + (uint32_t)(F::kTileCols * q), Desc::of(q_desc + (uint32_t)(q * (F::kQBytes >> 4)) + Desc::k_step(128, k)),
                            Desc::of(k_desc + (uint32_t)(s * (F::kKvBytes >> 4)) + Desc::k_step(kKeys, k)), p.idesc_s, (uint32_t)(k != 0), elected);
            umma_commit_if(bar(kSFull, q), elected);
        };
        auto values = [&](int q, int s, bool first, int steps) {
            const uint32_t t_q = tmem_u + (uint32_t)(F::kTileCols * q);
            auto step = [&](int k) {
                umma_f16_ts_if(t_q + F::kOCol, t_q + (uint32_t)(8 * k), Desc::of(v_desc + (uint32_t)(s * (F::kKvBytes >> 4)) + (uint32_t)k * Desc::kRowsStep), p.idesc_o,
                               k != 0 ? 1u : first ? 0u : 1u, elected);
            };
            if (steps >= kKeys / 16) {
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k) step(k);
            } else {
#pragma unroll 1
                for (int k = 0; k < steps; ++k) step(k);
            }
        };
        if (wait(bar(kQFull, 0), 0, 75)) {
            tc_fence_after();
            scores(0, kStages - 1);
            if (kTiles > 1 && tiles1 > 0) scores(1, kStages - 1);
            umma_commit_if(bar(kKvEmpty, kStages - 1), elected);
        }
        int left = len;                                              // keys of the sequence from this tile's first on
        for (int j0 = 0, round = 0; ok && j0 < tiles; j0 += kStages, ++round) {
#pragma unroll
            for (int s = 0; s < kStages; ++s) {
                const int j = j0 + s;
                if (!ok || j >= tiles) break;
                if (!wait(bar(kKvFull, s), round, 73)) break;
                if (left < kKeys && (left & 15) != 0) {
                    zero_rows<kD, kKeys>(v_smem(s), left, (left + 15) & ~15, lane);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
#pragma unroll
                for (int q = 0; q < kTiles; ++q) {
                    const int tiles_q = q == 0 ? tiles0 : tiles1;
                    if (j >= tiles_q) continue;
                    if (!wait(bar(kPFull, q), s, 74)) break;
                    tc_fence_after();
                    values(q, s, j == 0, (left + 15) >> 4);
                    // the next scores go over this tile's P: the tensor core takes products in the order they are issued
                    if (j + 1 < tiles_q) scores(q, s);
                    else umma_commit_if(bar(kODone, q), elected);
                }
                umma_commit_if(bar(kKvEmpty, s), elected);
                left -= kKeys;
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ softmax and output
        const int q = warp >> 2, quarter = warp & 3;
        const int nq = q == 0 ? n0 : n1;
        const int row0 = tile.first + 128 * q + 32 * quarter, row = row0 + lane;       // in the sequence
        const uint32_t t_lane = tmem_base + (uint32_t)(F::kTileCols * q) + ((uint32_t)(quarter * 32) << 16);
        const uint32_t t_o = t_lane + F::kOCol;
        const int limit = row >= tile.len ? 0 : p.causal ? row + 1 : tile.len;          // keys that take part
        constexpr float kFar = 32768.f;  // no probability above it: inside the 16-bit types and far inside fp32
        const float scale = p.scale_log2;
        const uint32_t hidden = scale < 0.f ? 0x7f800000u : 0xff800000u;                // times the scale: -inf
        float ref = 0.f;
        float sum = 0.f;
        for (int j = 0; j < nq; ++j) {
            // with a tile's scores P V of the tile before has ended too: it was issued first
            if (!wait(bar(kSFull, q), j, 77)) break;
            tc_fence_after();
            if (row0 < tile.len) {
                const int lim = limit - kKeys * j;                                      // of this tile's keys
                const bool whole = __all_sync(0xFFFFFFFFu, lim >= kKeys);
                // P lies over the S of chunks that have been read
                auto chunk = [&](auto masked, int c0) {
                    uint32_t r[F::kChunk];
#pragma unroll
                    for (int c = 0; c < F::kChunk; c += 32) tmem_ld_32x32b_x32(t_lane + (uint32_t)(c0 + c), r + c);
                    tmem_wait_ld();
                    if constexpr (decltype(masked)::value) {
#pragma unroll
                        for (int c = 0; c < F::kChunk; ++c)
                            if (c0 + c >= lim) r[c] = hidden;
                    }
                    auto top = [&]() {
                        float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int c = 0; c < F::kChunk; ++c) t[c & 3] = fmaxf(t[c & 3], __uint_as_float(r[c]) * scale);
                        return fmaxf(floorf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]))), -3.0e38f);     // finite for scores of minus infinity
                    };
                    if (j == 0 && c0 == 0) ref = top();
                    uint32_t w[F::kChunk / 2];
                    float part;
                    // one value at a time: with pairs of fp32 in a register (half as many instructions, but at a quarter of the rate) 128 images of 49
                    // to 1024 rows, 12 heads of 64, take 237 us, not 225 (100 passes at 1965 MHz; 256 at 1702 MHz, the power limit's, after a second of them)
                    auto exponentials = [&]() {
                        part = 0.f;
#pragma unroll
                        for (int i = 0; i < F::kChunk / 2; ++i) {
                            const float e0 = exp2_approx(fmaf(__uint_as_float(r[2 * i]), scale, -ref)), e1 = exp2_approx(fmaf(__uint_as_float(r[2 * i + 1]), scale, -ref));
                            part += e0;
                            part += e1;
                            w[i] = pack2<kBf16>(e0, e1);
                        }
                    };
                    exponentials();
                    const bool far = part > kFar;
                    if (__any_sync(0xFFFFFFFFu, far)) {
                        const float to = far ? fmaxf(top(), ref) : ref;
                        const float factor = __uint_as_float((uint32_t)(127 - (int)fminf(to - ref, 127.f)) << 23);   // 2^(ref - to), 0 from 2^-127 on
                        ref = to;
                        sum *= factor;
                        tmem_wait_st();
#pragma unroll 1
                        for (int c = 0; c < c0 / 2; c += 8) {                           // the tile's P so far
                            uint32_t o[8];
                            tmem_ld_32x32b_x8(t_lane + (uint32_t)c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float2 v = raw2_to_float2<kBf16>(o[i]);
                                o[i] = pack2<kBf16>(v.x * factor, v.y * factor);
                            }
                            tmem_st_32x32b_x8(t_lane + (uint32_t)c, o);
                        }
#pragma unroll 1
                        for (int c = 0; j > 0 && c < kD; c += 8) {
                            uint32_t o[8];
                            tmem_ld_32x32b_x8(t_o + (uint32_t)c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * factor);
                            tmem_st_32x32b_x8(t_o + (uint32_t)c, o);
                        }
                        exponentials();
                    }
                    sum += part;
                    if constexpr (F::kChunk == 64) {
                        tmem_st_32x32b_x32(t_lane + (uint32_t)(c0 / 2), w);
                    } else {
                        tmem_st_32x32b_x16(t_lane + (uint32_t)(c0 / 2), reinterpret_cast<const uint32_t(&)[16]>(w));
                    }
                };
                // nothing of the chunk takes part in any of the warp's rows
                auto hide = [&](int c0) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = 0u;
#pragma unroll
                    for (int c = 0; c < F::kChunk / 2; c += 16) tmem_st_32x32b_x16(t_lane + (uint32_t)(c0 / 2 + c), w);
                };
                if (whole) {
#pragma unroll
                    for (int c0 = 0; c0 < kKeys; c0 += F::kChunk) chunk(std::false_type{}, c0);
                } else {
#pragma unroll 1
                    for (int c0 = 0; c0 < kKeys; c0 += F::kChunk) {
                        if (j + c0 > 0 && __all_sync(0xFFFFFFFFu, lim <= c0)) hide(c0);
                        else chunk(std::true_type{}, c0);
                    }
                }
                tmem_wait_st();
            }
            // a warp without rows only keeps its place in the barriers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kPFull, q));
        }
        if (ok && nq > 0 && row0 < tile.len && wait(bar(kODone, q), 0, 76)) {
            tc_fence_after();
            const float inv = 1.0f / sum;
            if (p.lse != nullptr && row < tile.len)
                p.lse[(size_t)head * (size_t)p.rows + (size_t)(tile.begin + row)] = (ref + log2f(sum)) * 0.6931471805599453f;
            // Q has been read for the last time: its quarter is the warp's staging room
            const uint32_t stage = q_smem(q) + (uint32_t)(quarter * (F::kQBytes / 4));
            uint16_t* dst = p.a + (long long)(tile.begin + row0) * p.a_pitch + head * kD;
            constexpr int kCols = TileShape<kD>::kCols;
#pragma unroll
            for (int c = 0; c < kD; c += kCols)
                store_rows<kBf16, kCols>(t_o + (uint32_t)c, inv, stage, dst + c, p.a_pitch, tile.len - row0, lane);
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

// Sequence i as the offsets have it now: no rows where they are no offsets.  Read in place, so that what was checked is what is used.
struct PlanSpan {
    int begin, len, tiles;               // tiles of 128 rows
    bool bad;
};
__device__ __forceinline__ PlanSpan plan_span(const int32_t* offsets, int i, int rows)
{
    int b, e;
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(b) : "l"(offsets + i));
    asm volatile("ld.global.s32 %0, [%1];" : "=r"(e) : "l"(offsets + i + 1));
    const bool bad = b < 0 || e < b || e > rows;
    const int len = bad ? 0 : e - b;
    return {b, len, len > 0 ? (len - 1) / 128 + 1 : 0, bad};
}

// One CTA makes the plan: offsets that are no offsets make an empty one, and dev_status tells.  Sequences go into buckets by their number of
// 128-row tiles, most first (from 1023 tiles on they share one); where they stand inside a bucket does not matter.  The offsets are read
// three times.  A caller keeps them as they are meanwhile; where they change all the same, the plan is worth nothing, but every span is
// checked as it is read and no entry goes behind the lists.
__global__ void __launch_bounds__(1024) packed_plan_kernel(const int32_t* offsets, int sequences, int rows, int* plan, uint32_t* dev_status)
{
    __shared__ int count[2][1024], scan[2][1024];
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int tid = threadIdx.x, lane = tid & 31;
    count[0][tid] = 0;
    count[1][tid] = 0;
    int bad = 0;
    for (int i = tid; i < sequences; i += 1024) bad |= plan_span(offsets, i, rows).bad;
    bad = __syncthreads_or(bad);
    auto bucket_of = [](int tiles) { return tiles < 1023 ? tiles : 1023; };
    if (!bad) {
        for (int i = tid; i < sequences; i += 1024) {
            const int n = plan_span(offsets, i, rows).tiles;
            if (n == 0) continue;
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
    const int most[2] = {plan_capacity(rows, sequences, 128), plan_capacity(rows, sequences, 256)};
    int4* list[2] = {reinterpret_cast<int4*>(plan + kPlanHeader), reinterpret_cast<int4*>(plan + kPlanHeader) + most[0]};
    auto put = [&](int l, int first, int t, int begin, int len) {
        const unsigned to = (unsigned)first + (unsigned)t;
        if (to < (unsigned)most[l]) list[l][to] = make_int4(begin, len, t, 0);
    };
    for (int base = tid - lane; base < sequences; base += 1024) {
        const int i = base + lane;
        PlanSpan s = {0, 0, 0, false};
        if (i < sequences) s = plan_span(offsets, i, rows);
        const int begin = s.begin, len = s.len, n = s.tiles;
        int at[2] = {0, 0};
        if (n > 0) {
            at[0] = atomicAdd(&count[0][bucket_of(n)], n);
            at[1] = atomicAdd(&count[1][bucket_of(n)], (n + 1) / 2);
        }
        if (n <= 4) {
            for (int t = 0; t < n; ++t) put(0, at[0], t, begin, len);
            for (int t = 0; t < (n + 1) / 2; ++t) put(1, at[1], t, begin, len);
        }
        // long ones by the whole warp
        for (unsigned todo = __ballot_sync(0xFFFFFFFFu, n > 4); todo != 0; todo &= todo - 1) {
            const int from = __ffs(todo) - 1;
            const int b = __shfl_sync(0xFFFFFFFFu, begin, from), l = __shfl_sync(0xFFFFFFFFu, len, from), m = __shfl_sync(0xFFFFFFFFu, n, from);
            const int a0 = __shfl_sync(0xFFFFFFFFu, at[0], from), a1 = __shfl_sync(0xFFFFFFFFu, at[1], from);
            for (int t = lane; t < m; t += 32) put(0, a0, t, b, l);
            for (int t = lane; t < (m + 1) / 2; t += 32) put(1, a1, t, b, l);
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
    const int d = in.head_dim, keys = d > 64 ? ForwardShape<128>::kKeys : ForwardShape<64>::kKeys;
    if ((st = make_map_heads(&p.map_q, in.q, in.rows, (long long)in.heads * d, in.q_pitch, d, 128, "q")) != ELSA_OK) return st;
    if ((st = make_map_heads(&p.map_k, in.k, in.rows, (long long)in.kv_heads * d, in.k_pitch, d, keys, "k")) != ELSA_OK) return st;
    if ((st = make_map_heads(&p.map_v, in.v, in.rows, (long long)in.kv_heads * d, in.v_pitch, d, keys, "v")) != ELSA_OK) return st;
    p.plan = plan; p.a = a; p.lse = lse; p.a_pitch = a_pitch;
    p.rows = in.rows; p.sequences = sequences; p.heads = in.heads; p.group = in.heads / in.kv_heads;
    p.causal = in.causal ? 1 : 0;
    // hidden scores are infinite ones times the scale, which must not be zero; 1e-30 makes as much of the others
    p.scale_log2 = in.scale == 0.f ? 1e-30f : in.scale * 1.4426950408889634f;
    p.idesc_s = packed_idesc(dtype, keys, false);
    p.idesc_o = packed_idesc(dtype, d, true);
    p.dev_status = dev_status;
    const bool bf = dtype == ELSA_BF16;
    if (d == 32) return bf ? launch<true, 32>(p, stream, dev) : launch<false, 32>(p, stream, dev);
    if (d == 64) return bf ? launch<true, 64>(p, stream, dev) : launch<false, 64>(p, stream, dev);
    return bf ? launch<true, 128>(p, stream, dev) : launch<false, 128>(p, stream, dev);
}

}  // namespace elsa
