// Gradient of router and dispatch.  With P the softmax of the logits z = x Wg^T + bg over the experts, s_j = P[idx_j] (divided
// by their sum over j if the shape renormalises) and x_packed the token rows in expert order:
//   g_e  = dP_e + sum_j [idx_j = e] ds_j            (renormalised: ds_j -> (ds_j - sum_i ds_i s_i) / sum_i P[idx_i])
//   dz   = P (g - <P, g>) + the logits' own gradient
//   dx_i = sum_j dx_packed[inv_ij]  +  sum_e dz_ie Wg_e          (float, slots in order, rounded once)
//   dWg  = dz^T x,   dbg = sum_i dz_i                            (float)
#include "common.hpp"
#include "kernels.hpp"

namespace dicemoe {

// The dispatch alone: one wavefront per token adds its rows in slot order.  Bound by memory, k + 1 rows per token.
// KK > 0: k == KK, the loads of all rows in flight together; KK == 0: any k.
template <typename T, int KK>
__global__ __launch_bounds__(256) void dispatch_backward_kernel(const T* __restrict__ dxp, const int32_t* __restrict__ inv, int T_tok,
                                                                int d, int k, T* __restrict__ dx)
{
    constexpr int V = Store<T>::kVec, KN = KK > 0 ? KK : 1;
    const int tok = blockIdx.x * (blockDim.x / kWave) + threadIdx.x / kWave;
    if (tok >= T_tok) return;
    const int nvec = d / V, kn = KK > 0 ? KK : k;
    const size_t p0 = static_cast<size_t>(tok) * kn;
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(dxp);
    int row[KN];
    if (KK > 0) {
#pragma unroll
        for (int j = 0; j < KN; ++j) row[j] = inv[p0 + j];
    }
    for (int c = lane_id(); c < nvec; c += kWave) {
        float acc[V];
#pragma unroll
        for (int t = 0; t < V; ++t) acc[t] = 0.f;
        for (int j0 = 0; j0 < kn; j0 += KN) {
            u32x4_t v[KN];
            if (KK == 0) row[0] = inv[p0 + j0];
#pragma unroll
            for (int j = 0; j < KN; ++j) v[j] = row[j] >= 0 ? from[static_cast<size_t>(row[j]) * nvec + c] : u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < KN; ++j) {
                float f[V];
                Store<T>::unpack(v[j], f);
#pragma unroll
                for (int t = 0; t < V; ++t) acc[t] += f[t];
            }
        }
        const uint4 packed = Store<T>::pack(acc);
        reinterpret_cast<u32x4_t*>(dx)[static_cast<size_t>(tok) * nvec + c] = u32x4_t{packed.x, packed.y, packed.z, packed.w};
    }
}

// A workgroup takes `chunk` tokens (a multiple of 16) and 16 x kVec columns.  It first forms dz of its tokens in LDS (16 lanes per
// token, one expert each and 16 apart), then its four wavefronts take tiles of 16 tokens.  Both products run on float matrix
// instructions (16x16x4: exact products, float sums), chosen so that one 16-byte load per lane feeds them in place: lane (g, m) =
// (l / 16, l % 16) loads columns c0 + m V .. of token 4g + v (row g of step v for dz^T x) or of expert 4s + g (step s of dz Wg),
// and component j of the 16 bytes is the operand of instruction j.  The result of dz Wg then has V consecutive columns of
// tokens 4g .. 4g + 3 in the lane that also gathers the dispatch's rows for them and stores 16 bytes.
// dz^T x stays in registers over a wavefront's tiles; the four meet in LDS in wavefront order, and workgroups write partial sums
// [token chunk][E][d] that route_backward_sum_kernel adds in chunk order (one chunk: straight to the result).
template <typename T, int NB>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteBackward a, int chunk, int columns, int chunks)
{
    constexpr int V = Store<T>::kVec, EP = 16 * NB;
    extern __shared__ float lds[];                   // dz[chunk][EP], later the four wavefronts' sums of one block of experts
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int m = lane & 15, g = lane >> 4;
    const int part = blockIdx.x / columns, column = blockIdx.x - part * columns;
    const int tok0 = part * chunk, d = a.d, E = a.E;
    const bool first = column == 0;

    for (int i = threadIdx.x / 16; i < chunk; i += 16) {
        const int tok = tok0 + i;
        const bool on = tok < a.T;
        const size_t te = static_cast<size_t>(on ? tok : 0) * E, tk = static_cast<size_t>(on ? tok : 0) * a.slots;
        float P[NB], ge[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int e = m + 16 * b;
            P[b] = e < E ? a.probs[te + e] : 0.f;
            ge[b] = a.dprobs != nullptr && e < E ? a.dprobs[te + e] : 0.f;
        }
        float total = 1.f, mean = 0.f;
        if (a.renorm) {
            total = 0.f;
            for (int j = 0; j < a.k; ++j) {
                const float p = a.probs[te + a.idx[tk + j]];
                total += p;
                mean = fmaf(a.dscores[tk + j], p, mean);
            }
            mean /= total;
        }
        for (int j = 0; j < a.k; ++j) {
            const int e = a.idx[tk + j];
            const float ds = (a.dscores[tk + j] - mean) / total;
#pragma unroll
            for (int b = 0; b < NB; ++b)
                if (e == m + 16 * b) ge[b] += ds;
        }
        float dot = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b) dot = fmaf(P[b], ge[b], dot);
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) dot += __shfl_xor(dot, x, kWave);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int e = m + 16 * b;
            float dz = P[b] * (ge[b] - dot);
            if (a.dlogits != nullptr && e < E) dz += a.dlogits[te + e];
            if (!on || e >= E) dz = 0.f;             // tokens and experts that only fill up a tile add nothing
            lds[i * EP + e] = dz;
            if (first && a.dz != nullptr && on && e < E) a.dz[te + e] = dz;
        }
    }
    __syncthreads();
    if (first && a.dbg != nullptr && threadIdx.x < E) {
        float sum = 0.f;
        for (int i = 0; i < chunk; ++i) sum += lds[i * EP + threadIdx.x];
        (chunks == 1 ? a.dbg : a.partial_dbg + static_cast<size_t>(part) * E)[threadIdx.x] = sum;
    }

    const int c = column * 16 * V + m * V;       // the lane's first column
    const bool col_on = c < d;
    const u32x4_t none = {0u, 0u, 0u, 0u};
    f32x4_t accW[NB][V];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < V; ++j) accW[b][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const T* const Wg = static_cast<const T*>(a.Wg);
    const T* const x = static_cast<const T*>(a.x);
    const T* const dxp = static_cast<const T*>(a.dx_packed);
    T* const dx = static_cast<T*>(a.dx);
    for (int t0 = wave * 16; t0 < chunk && tok0 + t0 < a.T; t0 += 64) {
        u32x4_t xv[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int tok = tok0 + t0 + 4 * g + v;
            xv[v] = a.dWg != nullptr && col_on && tok < a.T ? *reinterpret_cast<const u32x4_t*>(x + static_cast<size_t>(tok) * d + c) : none;
        }
        f32x4_t accX[V];
#pragma unroll
        for (int j = 0; j < V; ++j) accX[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int e0 = 0; e0 < E; e0 += 4) {
            const int e = e0 + g;
            const u32x4_t wv = col_on && e < E ? *reinterpret_cast<const u32x4_t*>(Wg + static_cast<size_t>(e) * d + c) : none;
            const float dz = lds[(t0 + m) * EP + e];
            float w[V];
            Store<T>::unpack(wv, w);
#pragma unroll
            for (int j = 0; j < V; ++j) accX[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(dz, w[j], accX[j], 0, 0, 0);
        }
        if (a.dWg != nullptr) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float f[V];
                Store<T>::unpack(xv[v], f);
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const float dz = lds[(t0 + 4 * g + v) * EP + m + 16 * b];
#pragma unroll
                    for (int j = 0; j < V; ++j) accW[b][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(dz, f[j], accW[b][j], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int tok = tok0 + t0 + 4 * g + v;
            if (tok >= a.T || !col_on) continue;
            float sum[V];
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] = 0.f;
            if (dxp != nullptr)
                for (int j = 0; j < a.slots; ++j) {
                    const int row = a.inv[static_cast<size_t>(tok) * a.slots + j];
                    if (row < 0) continue;
                    float f[V];
                    Store<T>::unpack(*reinterpret_cast<const u32x4_t*>(dxp + static_cast<size_t>(row) * d + c), f);
#pragma unroll
                    for (int t = 0; t < V; ++t) sum[t] += f[t];
                }
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += accX[j][v];
            const uint4 packed = Store<T>::pack(sum);
            *reinterpret_cast<u32x4_t*>(dx + static_cast<size_t>(tok) * d + c) = u32x4_t{packed.x, packed.y, packed.z, packed.w};
        }
    }
    if (a.dWg == nullptr) return;
    float* const to = chunks == 1 ? a.dWg : a.partial + static_cast<size_t>(part) * E * d;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        __syncthreads();                             // dz, or the sums of the block before, have been read
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) lds[((wave * 4 + v) * V + j) * kWave + lane] = accW[b][j][v];
        __syncthreads();
        // thread (v = wave, lane): V columns of expert 4g + v
        const int e = 16 * b + 4 * g + wave;
        if (e < E && col_on) {
            float sum[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sum[j] = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) sum[j] += lds[((w * 4 + wave) * V + j) * kWave + lane];
            }
#pragma unroll
            for (int j = 0; j < V; j += 4)
                *reinterpret_cast<f32x4_t*>(to + static_cast<size_t>(e) * d + c + j) = f32x4_t{sum[j], sum[j + 1], sum[j + 2], sum[j + 3]};
        }
    }
}

// out[i] = sum over the token chunks of partial[chunk][i], in chunk order, for the n = E d values of dWg and then the E of dbg
__global__ __launch_bounds__(256) void route_backward_sum_kernel(const float* __restrict__ partial, const float* __restrict__ partial_dbg,
                                                                 int chunks, int n, int E, float* __restrict__ dWg, float* __restrict__ dbg)
{
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n && dWg != nullptr) {
        float sum = 0.f;
        for (int c = 0; c < chunks; ++c) sum += partial[static_cast<size_t>(c) * n + i];
        dWg[i] = sum;
    }
    if (i < E && dbg != nullptr) {
        float sum = 0.f;
        for (int c = 0; c < chunks; ++c) sum += partial_dbg[static_cast<size_t>(c) * E + i];
        dbg[i] = sum;
    }
}

namespace {

// Tokens per workgroup: 64, one tile per wavefront, while that leaves a workgroup or less per compute unit; then up to 256 (128 with more
// than 32 experts, whose dz has to fit the LDS), which keeps the partial sums a small part of what is read.
int route_chunk(int T_tok, int E, int columns)
{
    int chunk = 64;
    while (chunk < (E > 32 ? 128 : 256) && static_cast<long long>((T_tok + 2 * chunk - 1) / (2 * chunk)) * columns >= 2 * kComputeUnits) chunk *= 2;
    return chunk;
}

template <typename T, int NB>
void launch_route_backward_t(const RouteBackward& a, int columns, int chunk, int chunks, hipStream_t stream)
{
    const int dz = chunk * 16 * NB, sums = 4 * 4 * Store<T>::kVec * kWave;
    hipLaunchKernelGGL((route_backward_kernel<T, NB>), dim3(columns * chunks), dim3(256), (dz > sums ? dz : sums) * sizeof(float),
                       stream, a, chunk, columns, chunks);
}

template <typename T>
void launch_dispatch_backward_t(const RouteBackward& a, hipStream_t stream)
{
    const T* const dxp = static_cast<const T*>(a.dx_packed);
    T* const dx = static_cast<T*>(a.dx);
#define DICEMOE_DISPATCH_BWD(KK_) \
    hipLaunchKernelGGL((dispatch_backward_kernel<T, KK_>), dim3((a.T + 3) / 4), dim3(256), 0, stream, dxp, a.inv, a.T, a.d, a.slots, dx)
    if (a.slots == 1) DICEMOE_DISPATCH_BWD(1);
    else if (a.slots == 2) DICEMOE_DISPATCH_BWD(2);
    else if (a.slots == 3) DICEMOE_DISPATCH_BWD(3);
    else if (a.slots == 4) DICEMOE_DISPATCH_BWD(4);
    else DICEMOE_DISPATCH_BWD(0);
#undef DICEMOE_DISPATCH_BWD
}

}  // namespace

size_t route_backward_bytes(long long T_max, int E, int d)
{
    return static_cast<size_t>((T_max + 63) / 64) * E * (static_cast<size_t>(d) + 1) * sizeof(float);
}

hipError_t launch_route_backward(bool bf16, RouteBackward a, void* workspace, hipStream_t stream)
{
    if (a.Wg == nullptr) {
        if (a.T == 0) return hipSuccess;
        if (bf16) launch_dispatch_backward_t<bf16_t>(a, stream);
        else launch_dispatch_backward_t<float>(a, stream);
        return hipGetLastError();
    }
    const int V = bf16 ? 8 : 4, columns = (a.d + 16 * V - 1) / (16 * V);
    const int chunk = route_chunk(a.T, a.E, columns), chunks = (a.T + chunk - 1) / chunk;
    a.partial = static_cast<float*>(workspace);
    a.partial_dbg = a.partial + static_cast<size_t>(chunks) * a.E * a.d;
    if (chunks > 0) {
        const int blocks = (a.E + 15) / 16;
#define DICEMOE_ROUTE_BWD(T_)                                                             \
    do {                                                                                  \
        if (blocks == 1) launch_route_backward_t<T_, 1>(a, columns, chunk, chunks, stream);      \
        else if (blocks == 2) launch_route_backward_t<T_, 2>(a, columns, chunk, chunks, stream); \
        else if (blocks == 3) launch_route_backward_t<T_, 3>(a, columns, chunk, chunks, stream); \
        else launch_route_backward_t<T_, 4>(a, columns, chunk, chunks, stream);                  \
    } while (0)
        if (bf16) DICEMOE_ROUTE_BWD(bf16_t);
        else DICEMOE_ROUTE_BWD(float);
#undef DICEMOE_ROUTE_BWD
        if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
    }
    if (chunks == 1 || (a.dWg == nullptr && a.dbg == nullptr)) return hipSuccess;
    const int n = a.E * a.d;                         // (no token: the sums are zeros)
    hipLaunchKernelGGL(route_backward_sum_kernel, dim3((n + 255) / 256), dim3(256), 0, stream, a.partial, a.partial_dbg, chunks, n, a.E, a.dWg, a.dbg);
    return hipGetLastError();
}

}  // namespace dicemoe
