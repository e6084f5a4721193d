// Rotary positions with several axes on the query and key columns of qkv (the patch grids of ViTs: row and column of an image,
// frame, row and column of a video).  Pair p of a head is turned by angle = position[axis(p)] * rate(p):
//     (a, b) -> (a cos - b sin, b cos + a sin)          its gradient is the turn by -angle
// Angles are held in turns of a circle as 64-bit fractions: position * turns modulo 2^64 is exact in integers, so a position of
// 2^31 is as good as one of 10 (in fp32 a position of 10^5 would be off by 4e-3); the top 32 bits become an angle in [-pi, pi),
// 2e-7 off at most, and the special-function unit's sine and cosine of it are 5e-7 off, a thousandth of a 16-bit rounding.
// HBM bounds it: a row is read and written once, its angles are made once for all heads.  A lane has two vectors of eight values, the
// same eight pairs of a head for every head it meets, and its loads are on their way while the angles are made.  50432 rows of 24 heads
// of 64: 55 us, 5.6 TB/s (59.6 with CTAs of two or three rows a warp, 62 to 71 with fewer loads in flight and more warps).
#include <math.h>

#include "elsa_row_pack.cuh"

namespace elsa {
namespace {

constexpr int kRotaryThreads = 256;
constexpr int kHeadsAhead = 3;          // heads of a lane whose vectors are asked for together

struct RotaryParams {
    const uint16_t* x;
    const int32_t* positions;
    uint16_t* y;
    long long x_pitch, y_pitch;
    int rows, heads, units;             // units of eight pairs in a head
    int row_lanes;                      // lanes of a row, a power of two
    int inverse;
    elsa_rotary_plan plan;
};

template <bool kBf16, bool kInterleaved>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryParams p)
{
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int sub = threadIdx.x % p.row_lanes;
    const int heads_step = p.row_lanes / p.units;            // heads side by side
    const int unit = sub % p.units, first_head = sub / p.units;
    const int rows_step = gridDim.x * (kRotaryThreads / p.row_lanes);
    if (first_head >= heads_step) return;                    // lanes left over by units that are no power of two
    uint64_t turns[8];
    int axis[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        turns[e] = p.plan.turns[8 * unit + e];
        if (p.inverse) turns[e] = 0ull - turns[e];
        axis[e] = p.plan.axis[8 * unit + e];
    }
    const int head_dim = 16 * p.units;
    // the unit's two vectors: side by side, or half a head apart
    const int at0 = kInterleaved ? 16 * unit : 8 * unit, at1 = kInterleaved ? at0 + 8 : at0 + head_dim / 2;
    for (int row = blockIdx.x * (kRotaryThreads / p.row_lanes) + threadIdx.x / p.row_lanes; row < p.rows; row += rows_step) {
        const uint16_t* x = p.x + (long long)row * p.x_pitch;
        uint16_t* y = p.y + (long long)row * p.y_pitch;
        float c[8], s[8];
        bool made = false;
        for (int head = first_head; head < p.heads; head += kHeadsAhead * heads_step) {
            uint4 u[kHeadsAhead], w[kHeadsAhead];
#pragma unroll
            for (int i = 0; i < kHeadsAhead; ++i) {
                const int h = head + i * heads_step;
                if (h >= p.heads) break;
                u[i] = *reinterpret_cast<const uint4*>(x + (long long)h * head_dim + at0);
                w[i] = *reinterpret_cast<const uint4*>(x + (long long)h * head_dim + at1);
            }
            if (!made) {
                const int32_t* pos = p.positions + (long long)row * p.plan.axes;
                int32_t of[4];
#pragma unroll
                for (int a = 0; a < 4; ++a) of[a] = a < p.plan.axes ? __ldg(pos + a) : 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t at = axis[e] == 0 ? of[0] : axis[e] == 1 ? of[1] : axis[e] == 2 ? of[2] : of[3];
                    const uint64_t turned = (uint64_t)(int64_t)at * turns[e];
                    const float angle = (float)(int32_t)(uint32_t)(turned >> 32) * 1.4629180792671596e-9f;      // 2 pi / 2^32
                    c[e] = __cosf(angle);
                    s[e] = __sinf(angle);
                }
                made = true;
            }
#pragma unroll
            for (int i = 0; i < kHeadsAhead; ++i) {
                const int h = head + i * heads_step;
                if (h >= p.heads) break;
                float a[8], b[8];
                unpack8<kBf16>(u[i], a);
                unpack8<kBf16>(w[i], b);
                if constexpr (kInterleaved) {
                    // pairs (2e, 2e + 1): four in either vector
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a0 = a[2 * e], a1 = a[2 * e + 1], b0 = b[2 * e], b1 = b[2 * e + 1];
                        a[2 * e] = a0 * c[e] - a1 * s[e];
                        a[2 * e + 1] = a1 * c[e] + a0 * s[e];
                        b[2 * e] = b0 * c[4 + e] - b1 * s[4 + e];
                        b[2 * e + 1] = b1 * c[4 + e] + b0 * s[4 + e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a0 = a[e], b0 = b[e];
                        a[e] = a0 * c[e] - b0 * s[e];
                        b[e] = b0 * c[e] + a0 * s[e];
                    }
                }
                *reinterpret_cast<uint4*>(y + (long long)h * head_dim + at0) = pack8<kBf16>(a);
                *reinterpret_cast<uint4*>(y + (long long)h * head_dim + at1) = pack8<kBf16>(b);
            }
        }
    }
}

}  // namespace

elsa_status launch_rotary(const uint16_t* x, long long x_pitch, const int32_t* positions, const elsa_rotary_plan& plan, int rows, int heads,
                          bool inverse, elsa_dtype dtype, uint16_t* y, long long y_pitch, cudaStream_t stream)
{
    DeviceInfo dev;
    elsa_status st = device_info(&dev);
    if (st != ELSA_OK) return st;
    RotaryParams p;
    p.x = x; p.positions = positions; p.y = y;
    p.x_pitch = x_pitch; p.y_pitch = y_pitch;
    p.rows = rows; p.heads = heads; p.units = plan.head_dim / 16;
    p.row_lanes = 1;
    while (p.row_lanes < 32 && p.row_lanes < heads * p.units) p.row_lanes *= 2;
    p.inverse = inverse ? 1 : 0;
    p.plan = plan;
    const int rows_a_block = kRotaryThreads / p.row_lanes;
    const int blocks = (rows - 1) / rows_a_block + 1, most = dev.sm_count * 2;      // one wave: the registers allow two
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    ProfileScope scope(ELSA_KERNEL_ROTARY, stream);
    cudaError_t e;
    if (dtype == ELSA_BF16)
        e = plan.interleaved ? launch_pdl(rotary_kernel<true, true>, grid, dim3(kRotaryThreads), 0, stream, 1, p)
                             : launch_pdl(rotary_kernel<true, false>, grid, dim3(kRotaryThreads), 0, stream, 1, p);
    else
        e = plan.interleaved ? launch_pdl(rotary_kernel<false, true>, grid, dim3(kRotaryThreads), 0, stream, 1, p)
                             : launch_pdl(rotary_kernel<false, false>, grid, dim3(kRotaryThreads), 0, stream, 1, p);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "rotary launch: %s", cudaGetErrorString(e));
    return launched("rotary");
}

}  // namespace elsa

extern "C" elsa_status elsa_rotary_make_plan(int head_dim, const int* sections, int axes, double base, int shared, int interleaved,
                                             elsa_rotary_plan* plan)
{
    using namespace elsa;
    if (!sections || !plan) return fail(ELSA_ERR_NULL, "sections and plan must not be NULL");
    if (head_dim < 16 || head_dim > 2 * ELSA_ROTARY_MAX_PAIRS || head_dim % 16 != 0)
        return fail(ELSA_ERR_SHAPE, "head_dim=%d must be a multiple of 16 from 16 to %d", head_dim, 2 * ELSA_ROTARY_MAX_PAIRS);
    if (axes < 1 || axes > ELSA_ROTARY_MAX_AXES) return fail(ELSA_ERR_SHAPE, "axes=%d is outside 1..%d", axes, ELSA_ROTARY_MAX_AXES);
    if (!(base >= 1.0) || isinf(base)) return fail(ELSA_ERR_SHAPE, "base=%g must be a finite number of at least 1", base);
    const int pairs = head_dim / 2;
    long long sum = 0;
    for (int a = 0; a < axes; ++a) {
        if (sections[a] < 0) return fail(ELSA_ERR_SHAPE, "section %d has %d pairs", a, sections[a]);
        sum += sections[a];
    }
    if (sum != pairs) return fail(ELSA_ERR_SHAPE, "the sections hold %lld pairs, a head of %d values has %d", sum, head_dim, pairs);
    elsa_rotary_plan made = {};
    made.head_dim = head_dim; made.axes = axes; made.interleaved = interleaved ? 1 : 0;
    int p = 0;
    for (int a = 0; a < axes; ++a)
        for (int i = 0; i < sections[a]; ++i, ++p) {
            const long double exponent = shared ? (long double)p / pairs : (long double)i / sections[a];
            const long double rate = powl((long double)base, -exponent);                               // radians, in (0, 1]
            made.axis[p] = (unsigned char)a;
            made.turns[p] = (uint64_t)(rate / (2.0L * 3.14159265358979323846264338327950288L) * 18446744073709551616.0L + 0.5L);
        }
    *plan = made;
    return ELSA_OK;
}
