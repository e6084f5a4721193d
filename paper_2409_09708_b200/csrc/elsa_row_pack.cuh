// Sixteen-byte vectors of eight 16-bit values as fp32 and back, for the row-wise kernels.
#pragma once

#include "elsa_tc_common.cuh"

namespace elsa {
namespace {

template <bool kBf16>
__device__ __forceinline__ void unpack8(const uint4& u, float (&f)[8])
{
    const float2 a = raw2_to_float2<kBf16>(u.x), b = raw2_to_float2<kBf16>(u.y), c = raw2_to_float2<kBf16>(u.z), d = raw2_to_float2<kBf16>(u.w);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
}

template <bool kBf16>
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    return make_uint4(pack2<kBf16>(f[0], f[1]), pack2<kBf16>(f[2], f[3]), pack2<kBf16>(f[4], f[5]), pack2<kBf16>(f[6], f[7]));
}

}  // namespace
}  // namespace elsa
