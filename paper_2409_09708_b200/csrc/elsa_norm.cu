// LayerNorm as a call of its own and its gradient (ELSA, Alg. 2 trains the supernet's blocks, whose LayerNorms stand between the
// pruned linears).  With mean and rstd of a row s, xhat = (s - mean) rstd and g = dy gain:
//     y = xhat gain + bias          dx = rstd (g - mean(g) - xhat mean(g xhat)) + ds
//     dgain = sum over rows of dy xhat          dbias = sum over rows of dy
// Both are bound by HBM: every tensor is read or written once, 16 bytes a lane, the next row's loads under this row's arithmetic.
// A row belongs to kLanes lanes of a warp or to kRowWarps whole warps, each lane with the same kVpl vectors of eight columns
// of every row it meets.  So the gradients of gain and bias add up in registers, over the rows of a group, then over the groups of a
// CTA through shared memory; every CTA leaves one row of partial sums, which a second kernel adds in a fixed order: no atomics,
// the same bits every time.
#include "elsa_row_pack.cuh"

namespace elsa {
namespace {

constexpr int kMaxNormDim = 16384;      // 16 warps of 32 lanes with four vectors of eight

// kLeast: threads of a CTA where a row needs no more (256 forward, 128 for the gradient, whose registers allow CTAs of that size only in
// halves: 1384 columns 14.5 us forward, 16.2 with 128)
template <int kLanes, int kRowWarps, int kLeast>
struct Group {
    static constexpr int kThreads = kRowWarps * 32 > kLeast ? kRowWarps * 32 : kLeast;
    static constexpr int kRowLanes = kRowWarps > 1 ? kRowWarps * 32 : kLanes;   // lanes of a row
    static constexpr int kGroups = kThreads / kRowLanes;                        // rows side by side in a CTA
};

// CTAs of the gradient kernel on an SM: what its registers allow (two sums and three tensors' vectors of a row for each vector of a
// lane).  HBM bounds it: 50432 x 768 with a residual 54 us, 5.8 TB/s, 401408 x 128 71 us, 5.7 (one CTA of
// eight warps whatever the width, one row on its way: 63 and 109).
constexpr int backward_per_sm(int row_lanes, int vpl)
{
    const int warps = vpl == 1 ? 28 : vpl == 2 ? 16 : 8, cta_warps = row_lanes > 128 ? row_lanes / 32 : 4;
    return warps / cta_warps < 1 ? 1 : warps / cta_warps;
}

// Sums of a row's lanes, the same bits in each of them.  Row groups of several warps meet at a barrier of their own; two buffers
// in turn, so that one barrier a sum is enough.
template <class G, int kLanes, int kRowWarps>
__device__ __forceinline__ float2 row_sums(float2 v, float2* buffer, int& turn)
{
#pragma unroll
    for (int o = (kRowWarps > 1 ? 32 : kLanes) / 2; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if constexpr (kRowWarps > 1) {
        const int warp = threadIdx.x >> 5, group = warp / kRowWarps;
        float2* row = buffer + (turn * G::kGroups + group) * kRowWarps;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) row[warp % kRowWarps] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(kRowWarps * 32) : "memory");
        v = row[0];
#pragma unroll
        for (int w = 1; w < kRowWarps; ++w) { v.x += row[w].x; v.y += row[w].y; }
    }
    return v;
}

// Any width up to kMaxNormDim; the model widths have layer_norm_rows_kernel.
template <bool kBf16, bool kAdd, int kLanes, int kRowWarps, int kVpl>
__global__ void __launch_bounds__(Group<kLanes, kRowWarps, 256>::kThreads)
layer_norm_columns_kernel(const uint16_t* A, const uint16_t* R, uint16_t* S, const uint16_t* __restrict__ gain,
                          const uint16_t* __restrict__ beta, uint16_t* Y, float2* stats, int rows, int dim, float eps)
{
    using G = Group<kLanes, kRowWarps, 256>;
    __shared__ float2 sums[2 * G::kGroups * kRowWarps];
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int sub = threadIdx.x % G::kRowLanes, group = threadIdx.x / G::kRowLanes;
    const int vecs = dim >> 3;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    uint4 x[kVpl], w[kAdd ? kVpl : 1];
    int turn = 0;
    auto load = [&](int row) {
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            const int v = sub + G::kRowLanes * c;
            const bool in = row < rows && v < vecs;
            x[c] = in ? reinterpret_cast<const uint4*>(A + (size_t)row * (size_t)dim)[v] : zero;
            if constexpr (kAdd) w[c] = in ? reinterpret_cast<const uint4*>(R + (size_t)row * (size_t)dim)[v] : zero;
        }
    };
    const int stride = gridDim.x * G::kGroups;
    // every group of a warp makes the same number of steps: the shuffles name all lanes
    const int steps = (rows - blockIdx.x * G::kGroups + stride - 1) / stride;
    int row = blockIdx.x * G::kGroups + group;
    load(row);
    for (int step = 0; step < steps; ++step, row += stride) {
        float f[kVpl][8];
        float2 t = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            const int v = sub + G::kRowLanes * c;
            unpack8<kBf16>(x[c], f[c]);
            if constexpr (kAdd) {
                float r[8];
                unpack8<kBf16>(w[c], r);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[c][e] += r[e];
                const uint4 u = pack8<kBf16>(f[c]);
                if (row < rows && v < vecs) reinterpret_cast<uint4*>(S + (size_t)row * (size_t)dim)[v] = u;
                unpack8<kBf16>(u, f[c]);                   // the statistics are those of the row as stored
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) t.x += f[c][e];
        }
        load(row + stride);
        // a division, so that a constant row has its value as the mean, whatever the width
        const float mean = row_sums<G, kLanes, kRowWarps>(t, sums, turn).x / (float)dim;
        t.x = 0.f;
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            const bool in = sub + G::kRowLanes * c < vecs;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f[c][e] = in ? f[c][e] - mean : 0.f;
                t.x += f[c][e] * f[c][e];
            }
        }
        const float rstd = 1.0f / sqrtf(row_sums<G, kLanes, kRowWarps>(t, sums, turn).x / (float)dim + eps);
        if (row >= rows) continue;
        if (stats != nullptr && sub == 0) stats[row] = make_float2(mean, rstd);
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            const int v = sub + G::kRowLanes * c;
            if (v >= vecs) continue;
            float g[8], b[8];
            unpack8<kBf16>(__ldg(reinterpret_cast<const uint4*>(gain) + v), g);
            unpack8<kBf16>(__ldg(reinterpret_cast<const uint4*>(beta) + v), b);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[c][e] = f[c][e] * rstd * g[e] + b[e];
            reinterpret_cast<uint4*>(Y + (size_t)row * (size_t)dim)[v] = pack8<kBf16>(f[c]);
        }
    }
}

// dX may be dY's or dS's own buffer: a lane reads its vectors of a row before it writes them, and no one else touches them.
template <bool kBf16, bool kAdd, int kLanes, int kRowWarps, int kVpl>
__global__ void __launch_bounds__(Group<kLanes, kRowWarps, 128>::kThreads, backward_per_sm(Group<kLanes, kRowWarps, 128>::kRowLanes, kVpl))
layer_norm_backward_kernel(const uint16_t* dY, const uint16_t* __restrict__ S, const float2* __restrict__ stats,
                           const uint16_t* __restrict__ gain, const uint16_t* dS, uint16_t* dX, float* partial, int rows, int dim)
{
    using G = Group<kLanes, kRowWarps, 128>;
    __shared__ float2 sums[2 * G::kGroups * kRowWarps];
    extern __shared__ float4 column_sums[];                  // [2][dim], with several row groups
    float* columns = reinterpret_cast<float*>(column_sums);
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int sub = threadIdx.x % G::kRowLanes, group = threadIdx.x / G::kRowLanes;
    const int vecs = dim >> 3;
    const float inv_dim = 1.0f / (float)dim;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    // rows on their way: two where it takes eight warps with three vectors a lane to fill the registers (768 columns 60 to 54 us; with one or
    // two vectors more warps do the same, with four the registers are full)
    constexpr int kAhead = kVpl == 3 && kRowWarps <= 8 ? 2 : 1;
    struct Row {
        uint4 x[kVpl], d[kVpl], r[kAdd ? kVpl : 1];
        float2 st;
    } ahead[kAhead];
    uint4 gn[kVpl];
    // rows of more than 8192 values: 512 threads leave no registers for the sums, and one row group has the shared memory for itself
    constexpr bool kSharedSums = kRowWarps > 8;
    float dgain[kSharedSums ? 1 : kVpl][8], dbias[kSharedSums ? 1 : kVpl][8];
    int turn = 0;
#pragma unroll
    for (int c = 0; c < kVpl; ++c) {
        const int v = sub + G::kRowLanes * c;
        gn[c] = v < vecs ? __ldg(reinterpret_cast<const uint4*>(gain) + v) : zero;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (!kSharedSums) dgain[c][e] = dbias[c][e] = 0.f;
            else if (partial != nullptr && v < vecs) columns[8 * v + e] = columns[dim + 8 * v + e] = 0.f;
        }
    }
    auto load = [&](Row& a, int row) {
        a.st = row < rows ? __ldg(stats + row) : make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            const int v = sub + G::kRowLanes * c;
            const bool in = row < rows && v < vecs;
            const size_t at = (size_t)row * (size_t)dim;
            a.x[c] = in ? __ldg(reinterpret_cast<const uint4*>(S + at) + v) : zero;
            a.d[c] = in ? reinterpret_cast<const uint4*>(dY + at)[v] : zero;
            if constexpr (kAdd) a.r[c] = in ? reinterpret_cast<const uint4*>(dS + at)[v] : zero;
        }
    };
    const int stride = gridDim.x * G::kGroups;
    const int steps = (rows - blockIdx.x * G::kGroups + stride - 1) / stride;
    int row = blockIdx.x * G::kGroups + group;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) load(ahead[a], row + a * stride);
    auto one_row = [&](Row& a) {
        float xhat[kVpl][8], g[kVpl][8];
        uint4 rr[kAdd ? kVpl : 1];
        float2 t = make_float2(0.f, 0.f);
        const float rstd = a.st.y, mean = a.st.x;
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            float gv[8];
            unpack8<kBf16>(a.x[c], xhat[c]);
            unpack8<kBf16>(a.d[c], g[c]);
            unpack8<kBf16>(gn[c], gv);
            if constexpr (kAdd) rr[c] = a.r[c];
            const int v = sub + G::kRowLanes * c;
            float4* sum4 = reinterpret_cast<float4*>(columns + 8 * v);
            float had[2][8];
            if constexpr (kSharedSums) {
                if (partial != nullptr && v < vecs) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) reinterpret_cast<float4*>(had[q >> 1])[q & 1] = sum4[(q >> 1) * (dim >> 2) + (q & 1)];
                }
            }
            // columns past the row's end and rows past the last have dy = 0 and a mean and rstd that are finite: they add nothing
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xhat[c][e] = (xhat[c][e] - mean) * rstd;
                if constexpr (kSharedSums) {
                    had[0][e] += g[c][e] * xhat[c][e];
                    had[1][e] += g[c][e];
                } else {
                    dgain[c][e] += g[c][e] * xhat[c][e];
                    dbias[c][e] += g[c][e];
                }
                g[c][e] *= gv[e];
                t.x += g[c][e];
                t.y += g[c][e] * xhat[c][e];
            }
            if constexpr (kSharedSums) {
                if (partial != nullptr && v < vecs) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) sum4[(q >> 1) * (dim >> 2) + (q & 1)] = reinterpret_cast<float4*>(had[q >> 1])[q & 1];
                }
            }
        }
        load(a, row + kAhead * stride);
        const float2 m = row_sums<G, kLanes, kRowWarps>(t, sums, turn);
        if (dX == nullptr || row >= rows) return;
        const float c1 = m.x * inv_dim, c2 = m.y * inv_dim;
#pragma unroll
        for (int c = 0; c < kVpl; ++c) {
            const int v = sub + G::kRowLanes * c;
            if (v >= vecs) continue;
            float out[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if constexpr (kAdd) unpack8<kBf16>(rr[c], out);
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] += rstd * (g[c][e] - c1 - xhat[c][e] * c2);
            reinterpret_cast<uint4*>(dX + (size_t)row * (size_t)dim)[v] = pack8<kBf16>(out);
        }
    };
    for (int step = 0; step < steps; step += kAhead) {
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (step + a < steps) one_row(ahead[a]);
            row += stride;
        }
    }
    if (partial == nullptr) return;
    if constexpr (kSharedSums) {
        float4* out = reinterpret_cast<float4*>(partial + (size_t)blockIdx.x * (size_t)(2 * dim));
        for (int c = 0; c < kVpl; ++c) {
            const int v = sub + G::kRowLanes * c;
            if (v >= vecs) continue;
            for (int q = 0; q < 4; ++q) out[(q >> 1) * (dim >> 2) + 2 * v + (q & 1)] = column_sums[(q >> 1) * (dim >> 2) + 2 * v + (q & 1)];
        }
        return;
    } else {
        // the row groups of the CTA, one after another in a fixed order: columns [2][dim]
#pragma unroll 1
        for (int k = 0; k < G::kGroups; ++k) {
            if (group == k) {
#pragma unroll
                for (int c = 0; c < kVpl; ++c) {
                    const int v = sub + G::kRowLanes * c;
                    if (v >= vecs) continue;
                    float4* a = reinterpret_cast<float4*>(columns + 8 * v);
                    float4* b = reinterpret_cast<float4*>(columns + dim + 8 * v);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float4 p = make_float4(dgain[c][4 * h], dgain[c][4 * h + 1], dgain[c][4 * h + 2], dgain[c][4 * h + 3]);
                        float4 q = make_float4(dbias[c][4 * h], dbias[c][4 * h + 1], dbias[c][4 * h + 2], dbias[c][4 * h + 3]);
                        if (k > 0) {
                            const float4 p0 = a[h], q0 = b[h];
                            p.x += p0.x; p.y += p0.y; p.z += p0.z; p.w += p0.w;
                            q.x += q0.x; q.y += q0.y; q.z += q0.z; q.w += q0.w;
                        }
                        if (k + 1 < G::kGroups) {
                            a[h] = p;
                            b[h] = q;
                        } else {
                            float4* out = reinterpret_cast<float4*>(partial + (size_t)blockIdx.x * (size_t)(2 * dim));
                            out[2 * v + h] = p;
                            out[(dim >> 2) + 2 * v + h] = q;
                        }
                    }
                }
            }
            if (G::kGroups > 1) __syncthreads();
        }
    }
}

// out[c] = round16(sum over parts of partial[part][c]): 32 columns a block, the parts over its warps.
constexpr int kSumWarps = 32;
template <bool kBf16>
__global__ void __launch_bounds__(kSumWarps * 32)
norm_sums_kernel(const float* __restrict__ partial, int parts, int dim, uint16_t* dgain, uint16_t* dbias)
{
    __shared__ float sums[kSumWarps][33];
    pdl_wait_for_predecessors();
    pdl_release_successors();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    float t[4] = {0.f, 0.f, 0.f, 0.f};
    if (col < 2 * dim) {
        int p = warp;
        for (; p + 3 * kSumWarps < parts; p += 4 * kSumWarps) {
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] += __ldg(partial + (size_t)(p + kSumWarps * i) * (size_t)(2 * dim) + col);
        }
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (p + kSumWarps * i < parts) t[i] += __ldg(partial + (size_t)(p + kSumWarps * i) * (size_t)(2 * dim) + col);
    }
    sums[warp][lane] = (t[0] + t[1]) + (t[2] + t[3]);
    __syncthreads();
    // a column to a warp, its parts to the lanes
    float v = sums[lane][warp];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int out_col = blockIdx.x * 32 + warp;
    if (lane == 0 && out_col < 2 * dim) {
        uint16_t* out = out_col < dim ? dgain : dbias;
        if (out != nullptr) out[out_col < dim ? out_col : out_col - dim] = (uint16_t)(pack2<kBf16>(v, 0.f) & 0xffffu);
    }
}

// The lanes and vectors of a row of `dim` values: the fewest of them that cover it, of those the fewest lanes.
struct RowShape {
    int lanes, vpl;
};
RowShape row_shape(int dim)
{
    const int vecs = dim / 8;
    RowShape best = {512, 4};
    for (int lanes = 512; lanes >= 8; lanes >>= 1)
        for (int vpl = 1; vpl <= 4; ++vpl)
            if (lanes * vpl >= vecs && lanes * vpl <= best.lanes * best.vpl) best = {lanes, vpl};
    return best;
}

// Rows of partial sums: one of each CTA that the 148 SMs of sm_100a hold.  A constant, so that a workspace's size is the same wherever it is
// asked for.
int max_parts(int dim)
{
    const RowShape shape = row_shape(dim);
    return 148 * backward_per_sm(shape.lanes, shape.vpl);
}

#define ELSA_NORM_VPL(MACRO, LANES, WARPS)                                     \
    do {                                                                       \
        if (shape.vpl == 1) MACRO(LANES, WARPS, 1);                            \
        else if (shape.vpl == 2) MACRO(LANES, WARPS, 2);                       \
        else if (shape.vpl == 3) MACRO(LANES, WARPS, 3);                       \
        else MACRO(LANES, WARPS, 4);                                           \
    } while (0)
#define ELSA_NORM_SHAPES(MACRO)                                                \
    do {                                                                       \
        switch (shape.lanes) {                                                 \
        case 8: ELSA_NORM_VPL(MACRO, 8, 1); break;                             \
        case 16: ELSA_NORM_VPL(MACRO, 16, 1); break;                           \
        case 32: ELSA_NORM_VPL(MACRO, 32, 1); break;                           \
        case 64: ELSA_NORM_VPL(MACRO, 32, 2); break;                           \
        case 128: ELSA_NORM_VPL(MACRO, 32, 4); break;                          \
        case 256: ELSA_NORM_VPL(MACRO, 32, 8); break;                          \
        default: ELSA_NORM_VPL(MACRO, 32, 16); break;                          \
        }                                                                      \
    } while (0)

template <bool kBf16, bool kAdd>
cudaError_t forward(const RowShape& shape, const uint16_t* A, const uint16_t* R, uint16_t* S, const uint16_t* gain, const uint16_t* beta,
                    uint16_t* Y, float2* stats, int rows, int dim, float eps, cudaStream_t stream, const DeviceInfo& dev)
{
    cudaError_t e = cudaSuccess;
#define ELSA_NORM_FORWARD(LANES, WARPS, VPL)                                                                                   \
    do {                                                                                                                       \
        using G = Group<LANES, WARPS, 256>;                                                                                    \
        const int blocks = (rows - 1) / G::kGroups + 1, most = dev.sm_count * 2048 / G::kThreads;                           \
        e = launch_pdl(layer_norm_columns_kernel<kBf16, kAdd, LANES, WARPS, VPL>, dim3((unsigned)(blocks < most ? blocks : most)), \
                       dim3(G::kThreads), 0, stream, 1, A, R, S, gain, beta, Y, stats, rows, dim, eps);                        \
    } while (0)
    ELSA_NORM_SHAPES(ELSA_NORM_FORWARD);
#undef ELSA_NORM_FORWARD
    return e;
}

template <bool kBf16, bool kAdd>
cudaError_t backward(const RowShape& shape, const uint16_t* dY, const uint16_t* S, const float2* stats, const uint16_t* gain,
                     const uint16_t* dS, uint16_t* dX, float* partial, int rows, int dim, int* parts, cudaStream_t stream)
{
    cudaError_t e = cudaSuccess;
#define ELSA_NORM_BACKWARD(LANES, WARPS, VPL)                                                                                  \
    do {                                                                                                                       \
        using G = Group<LANES, WARPS, 128>;                                                                                    \
        auto kernel = layer_norm_backward_kernel<kBf16, kAdd, LANES, WARPS, VPL>;                                              \
        constexpr bool kShared = WARPS > 8;                                                                                    \
        const size_t smem = partial != nullptr && (G::kGroups > 1 || kShared) ? (size_t)dim * 8 : 0;   /* up to 16 KB, or 128 */ \
        const int blocks = (rows - 1) / G::kGroups + 1, most = max_parts(dim);                                                 \
        *parts = blocks < most ? blocks : most;                                                                                \
        if (kShared) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kMaxNormDim * (int)sizeof(float)); \
        if (e == cudaSuccess)                                                                                                  \
        e = launch_pdl(kernel, dim3((unsigned)*parts), dim3(G::kThreads), smem, stream, 1, dY, S, stats, gain, dS, dX, partial, rows, dim); \
    } while (0)
    ELSA_NORM_SHAPES(ELSA_NORM_BACKWARD);
#undef ELSA_NORM_BACKWARD
    return e;
}

}  // namespace

bool layer_norm_columns_suits(int dim) { return dim <= kMaxNormDim; }

elsa_status launch_layer_norm_columns(const uint16_t* A, const uint16_t* R, uint16_t* S, const uint16_t* gain, const uint16_t* beta,
                                      uint16_t* Y, float* stats, int rows, int dim, float eps, elsa_dtype dtype, cudaStream_t stream)
{
    DeviceInfo dev;
    elsa_status st = device_info(&dev);
    if (st != ELSA_OK) return st;
    const RowShape shape = row_shape(dim);
    float2* stats2 = reinterpret_cast<float2*>(stats);
    ProfileScope scope(ELSA_KERNEL_BLOCK_ROWWISE, stream);
    cudaError_t e;
    if (dtype == ELSA_BF16)
        e = R ? forward<true, true>(shape, A, R, S, gain, beta, Y, stats2, rows, dim, eps, stream, dev)
              : forward<true, false>(shape, A, R, S, gain, beta, Y, stats2, rows, dim, eps, stream, dev);
    else
        e = R ? forward<false, true>(shape, A, R, S, gain, beta, Y, stats2, rows, dim, eps, stream, dev)
              : forward<false, false>(shape, A, R, S, gain, beta, Y, stats2, rows, dim, eps, stream, dev);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "layer_norm launch: %s", cudaGetErrorString(e));
    return launched("layer_norm");
}

size_t layer_norm_backward_workspace(int rows, int dim)
{
    const size_t parts = (size_t)(rows < max_parts(dim) ? rows : max_parts(dim));
    return parts * (size_t)dim * 2 * sizeof(float);
}

elsa_status launch_layer_norm_backward(const uint16_t* dY, const uint16_t* S, const float* stats, const uint16_t* gain, const uint16_t* dS,
                                       int rows, int dim, elsa_dtype dtype, uint16_t* dX, uint16_t* dgain, uint16_t* dbias, float* partial,
                                       cudaStream_t stream)
{
    DeviceInfo dev;
    elsa_status st = device_info(&dev);                // a device of another kind is refused
    if (st != ELSA_OK) return st;
    const RowShape shape = row_shape(dim);
    const float2* stats2 = reinterpret_cast<const float2*>(stats);
    if (dgain == nullptr && dbias == nullptr) partial = nullptr;
    int parts = 0;
    cudaError_t e;
    {
        ProfileScope scope(ELSA_KERNEL_NORM_BACKWARD, stream);
        if (dtype == ELSA_BF16)
            e = dS ? backward<true, true>(shape, dY, S, stats2, gain, dS, dX, partial, rows, dim, &parts, stream)
                   : backward<true, false>(shape, dY, S, stats2, gain, dS, dX, partial, rows, dim, &parts, stream);
        else
            e = dS ? backward<false, true>(shape, dY, S, stats2, gain, dS, dX, partial, rows, dim, &parts, stream)
                   : backward<false, false>(shape, dY, S, stats2, gain, dS, dX, partial, rows, dim, &parts, stream);
        if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "layer_norm_backward launch: %s", cudaGetErrorString(e));
        if ((st = launched("layer_norm_backward")) != ELSA_OK || partial == nullptr) return st;
    }
    ProfileScope scope(ELSA_KERNEL_NORM_BACKWARD, stream);
    const dim3 grid((unsigned)((2 * dim + 31) / 32));
    if (dtype == ELSA_BF16) e = launch_pdl(norm_sums_kernel<true>, grid, dim3(kSumWarps * 32), 0, stream, 1, partial, parts, dim, dgain, dbias);
    else e = launch_pdl(norm_sums_kernel<false>, grid, dim3(kSumWarps * 32), 0, stream, 1, partial, parts, dim, dgain, dbias);
    if (e != cudaSuccess) return fail(ELSA_ERR_CUDA, "norm_sums launch: %s", cudaGetErrorString(e));
    return launched("norm_sums");
}

}  // namespace elsa
