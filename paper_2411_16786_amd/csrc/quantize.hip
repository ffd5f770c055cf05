// Weights to 4-bit codes with one power-of-two scale per 32 columns (see mx4.hpp), and the values that the codes stand for.
//
// Scale: the smallest power of two s >= 2^-126 with max|w| <= 7 s.  A magnitude up to 7 s rounds to the largest code, 6 s, with at
// most the error that the spacing there (4, 6) allows anyway, half of 2 s; any smaller s would clip.  No s is above 2^125, where 6 s = 1.5 2^127
// is the largest number that a code and a scale stand for: with 2^126 the code of 4 is infinite.  Code: the nearest of 0, 0.5,
// 1, 1.5, 2, 3, 4, 6 to |w| / s, ties to the even code (the conversion instruction's rounding, which ends at 6).  w / s is exact: s is a power of two.
//
// Bound by memory: 32 columns are four lanes' 16-byte loads (bf16), the maximum goes round two lane exchanges, every lane
// stores its eight codes as one dword: 42 million bf16 weights with their values 34 us, 5.6 TB/s (partly from the memory-side cache; a copy 5.1).
#include "kernels.hpp"
#include "mx4.hpp"

namespace dicemoe {

template <typename T>
__global__ __launch_bounds__(256) void quantize_mx4_kernel(const T* __restrict__ W, long long n_octets, uint8_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scales, T* __restrict__ values)
{
    constexpr int V = Store<T>::kVec, L = 8 / V;                // 16-byte loads per eight columns
    const long long o = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
    if (o >= n_octets) return;                                  // (n_octets is a multiple of 4: a group's lanes stay together)
    float w[8];
#pragma unroll
    for (int i = 0; i < L; ++i) Store<T>::unpack(reinterpret_cast<const u32x4_t*>(W)[o * L + i], w + i * V);
    uint32_t top = 0;                                           // magnitudes order like their bit patterns, NaN above infinity
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(w[i]) & 0x7FFFFFFFu;
        top = a > top ? a : top;
    }
#pragma unroll
    for (int m = 1; m <= 2; m <<= 1) {
        const uint32_t other = static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), m, kWave));
        top = other > top ? other : top;
    }
    // top = 1.f 2^(e - 127) is at most 7 s = 1.75 * 4 s for s = 2^(e - 127 - 2) where 1.f <= 1.75, for twice that otherwise
    const int e = static_cast<int>(top >> 23);
    int byte = e - ((top & 0x7FFFFFu) <= 0x600000u ? 2 : 1);
    byte = byte < 1 ? 1 : byte > 252 ? 252 : byte;
    const bool finite = e < 255;
    if (!finite) byte = 255;
    uint32_t c = 0;
    const float s = mx4_scale(static_cast<uint32_t>(byte));
    if (finite) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[0], w[1], s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[2], w[3], s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[4], w[5], s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[6], w[7], s, 3);
    }
    reinterpret_cast<uint32_t*>(codes)[o] = c;
    if ((o & 3) == 0) scales[o >> 2] = static_cast<uint8_t>(byte);
    if (values == nullptr) return;
    if constexpr (V == 8) {
        reinterpret_cast<u32x4_t*>(values)[o] = u32x4_t{mx4_bf16<0>(c, s), mx4_bf16<1>(c, s), mx4_bf16<2>(c, s), mx4_bf16<3>(c, s)};
    } else {
        const f32x2_t a = mx4_f32<0>(c, s), b = mx4_f32<1>(c, s), d = mx4_f32<2>(c, s), f = mx4_f32<3>(c, s);
        f32x4_t* to = reinterpret_cast<f32x4_t*>(values) + o * 2;
        to[0] = f32x4_t{a[0], a[1], b[0], b[1]};
        to[1] = f32x4_t{d[0], d[1], f[0], f[1]};
    }
}

namespace {

template <typename T>
hipError_t launch_quantize_mx4_t(const T* W, long long octets, uint8_t* codes, uint8_t* scales, T* values, hipStream_t stream)
{
    constexpr long long kMost = 1ll << 30;                      // octets per launch: a grid holds less than 2^32 threads
    for (long long o = 0; o < octets; o += kMost) {
        const long long n = octets - o < kMost ? octets - o : kMost;
        hipLaunchKernelGGL(quantize_mx4_kernel<T>, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, W + o * 8, n, codes + o * 4,
                           scales + o / 4, values ? values + o * 8 : nullptr);
        if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_quantize_mx4(bool bf16, const void* W, long long rows, int cols, uint8_t* codes, uint8_t* scales, void* values,
                               hipStream_t stream)
{
    const long long octets = rows * (cols / 8);
    if (bf16) return launch_quantize_mx4_t(static_cast<const bf16_t*>(W), octets, codes, scales, static_cast<bf16_t*>(values), stream);
    return launch_quantize_mx4_t(static_cast<const float*>(W), octets, codes, scales, static_cast<float*>(values), stream);
}

}  // namespace dicemoe
