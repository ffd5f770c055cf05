// Gradient of the combine y_i = sum_j s_ij h_ij over the pairs that have a packed row:
//   dh[inv[p]] = s_p dy_i  (rounded once to the storage type),   ds_p = <h[inv[p]], dy_i>  (float),
// and ds_p = 0 for a pair without a row.  One wavefront per token reads dy once and its k rows of h, and writes k rows of dh; the
// dot products are summed over the lanes in a fixed order, no atomics.  Bound by memory: 1 + 2k rows moved per token
// (8192 tokens of 2048 columns in bf16, two slots: 35 us, 4.8 TB/s).
#include "common.hpp"
#include "kernels.hpp"

namespace dicemoe {

// KK > 0: k == KK, all rows of a 16-byte column slice in flight together; KK == 0: any k, slot by slot (dy from the cache again).
template <typename T, int KK>
__global__ __launch_bounds__(256) void combine_backward_kernel(const T* __restrict__ dy, const T* __restrict__ h,
                                                               const int32_t* __restrict__ inv, const float* __restrict__ scores,
                                                               int T_tok, int d, int k, T* __restrict__ dh, float* __restrict__ dscores)
{
    constexpr int V = Store<T>::kVec, KN = KK > 0 ? KK : 1;
    const int tok = blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave;
    if (tok >= T_tok) return;
    const int lane = lane_id(), nvec = d / V, kn = KK > 0 ? KK : k;
    const size_t p0 = static_cast<size_t>(tok) * kn;
    const u32x4_t* dyv = reinterpret_cast<const u32x4_t*>(dy) + static_cast<size_t>(tok) * nvec;
    const u32x4_t* hv = reinterpret_cast<const u32x4_t*>(h);
    u32x4_t* dhv = reinterpret_cast<u32x4_t*>(dh);
    for (int j0 = 0; j0 < kn; j0 += KN) {
        int row[KN];
        float s[KN], dot[KN];
#pragma unroll
        for (int j = 0; j < KN; ++j) {
            row[j] = inv[p0 + j0 + j];
            s[j] = scores[p0 + j0 + j];
            dot[j] = 0.f;
        }
        for (int c = lane; c < nvec; c += kWave) {
            const u32x4_t gv = dyv[c];
            u32x4_t v[KN];
#pragma unroll
            for (int j = 0; j < KN; ++j)
                if (row[j] >= 0) v[j] = hv[static_cast<size_t>(row[j]) * nvec + c];
            float g[V];
            Store<T>::unpack(gv, g);
#pragma unroll
            for (int j = 0; j < KN; ++j) {
                if (row[j] < 0) continue;
                float f[V], o[V];
                Store<T>::unpack(v[j], f);
#pragma unroll
                for (int t = 0; t < V; ++t) {
                    dot[j] = fmaf(f[t], g[t], dot[j]);
                    o[t] = s[j] * g[t];
                }
                const uint4 packed = Store<T>::pack(o);
                dhv[static_cast<size_t>(row[j]) * nvec + c] = u32x4_t{packed.x, packed.y, packed.z, packed.w};
            }
        }
#pragma unroll
        for (int j = 0; j < KN; ++j) {
            const float total = wave_sum(dot[j]);
            if (lane == 0) dscores[p0 + j0 + j] = total;
        }
    }
}

template <typename T>
static void launch_combine_backward_t(const void* dy, const void* h, const int32_t* inv, const float* scores, int T_tok, int d, int k,
                                      void* dh, float* dscores, hipStream_t stream)
{
#define DICEMOE_COMBINE_BWD(KK_)                                                                                              \
    hipLaunchKernelGGL((combine_backward_kernel<T, KK_>), dim3((T_tok + 3) / 4), dim3(256), 0, stream, static_cast<const T*>(dy), \
                       static_cast<const T*>(h), inv, scores, T_tok, d, k, static_cast<T*>(dh), dscores)
    if (k == 1) DICEMOE_COMBINE_BWD(1);
    else if (k == 2) DICEMOE_COMBINE_BWD(2);
    else if (k == 3) DICEMOE_COMBINE_BWD(3);
    else if (k == 4) DICEMOE_COMBINE_BWD(4);
    else DICEMOE_COMBINE_BWD(0);
#undef DICEMOE_COMBINE_BWD
}

hipError_t launch_combine_backward(bool bf16, const void* dy, const void* h_packed, const int32_t* inv, const float* scores, int T_tok,
                                   int d, int k, void* dh_packed, float* dscores, hipStream_t stream)
{
    if (T_tok == 0) return hipSuccess;
    if (bf16) launch_combine_backward_t<bf16_t>(dy, h_packed, inv, scores, T_tok, d, k, dh_packed, dscores, stream);
    else launch_combine_backward_t<float>(dy, h_packed, inv, scores, T_tok, d, k, dh_packed, dscores, stream);
    return hipGetLastError();
}

}  // namespace dicemoe
