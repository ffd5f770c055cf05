// Gradient of router and dispatch.  With P the softmax of the logits z = x Wg^T + bg over the experts, s_j = P[idx_j] (divided
// by their sum over j if the shape renormalises) and x_packed the token rows in expert order:
//   g_e  = dP_e + sum_j [idx_j = e] ds_j            (renormalised: ds_j -> (ds_j - sum_i ds_i s_i) / sum_i P[idx_i])
//   dz   = P (g - <P, g>) + the logits' own gradient
//   dx_i = sum_j dx_packed[inv_ij]  +  sum_e dz_ie Wg_e          (float, slots in order, rounded once)
//   dWg  = dz^T x,   dbg = sum_i dz_i                            (float)
#include <type_traits>
#include "common.hpp"
#include "kernels.hpp"
#include "route_plan.hpp"

namespace dicemoe {

// The dispatch alone: one wavefront per token adds its rows in slot order.  Bound by memory, k + 1 rows per token
// (8192 tokens of 2048 columns in bf16, two slots: 20 us, 5.0 TB/s).
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

// dz: 16 lanes per token, lane m with the experts m, m + 16, ..
template <int NB>
__global__ __launch_bounds__(256) void route_logits_kernel(RouteBackward a)
{
    const int lane = lane_id(), m = lane & 15;
    const int at = blockIdx.x * 16 + threadIdx.x / 16, tok = at < a.T ? at : a.T - 1;
    const size_t te = static_cast<size_t>(tok) * a.E, tk = static_cast<size_t>(tok) * a.slots;
    float P[NB], ge[NB], dl[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int e = m + 16 * b;
        const bool on = e < a.E;
        P[b] = on ? a.probs[te + e] : 0.f;
        ge[b] = on && a.dprobs != nullptr ? a.dprobs[te + e] : 0.f;
        dl[b] = on && a.dlogits != nullptr ? a.dlogits[te + e] : 0.f;
    }
    float total = 1.f, mean = 0.f;
    if (a.renorm) {
        total = 0.f;
        for (int j = 0; j < a.k; ++j) {
            const int e = a.idx[tk + j];
            if (e < 0 || e >= a.E) continue;             // (no expert of this router: no part in the sum)
            const float p = a.probs[te + e];
            total += p;
            mean = fmaf(a.dscores[tk + j], p, mean);
        }
        mean /= total;
    }
    for (int j = 0; j < a.k; ++j) {
        const int e = a.idx[tk + j];
        const float add = (a.dscores[tk + j] - mean) / total;
#pragma unroll
        for (int b = 0; b < NB; ++b)
            if (e == m + 16 * b) ge[b] += add;
    }
    float dot = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) dot = fmaf(P[b], ge[b], dot);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) dot += __shfl_xor(dot, o, kWave);
    if (at >= a.T) return;
#pragma unroll
    for (int b = 0; b < NB; ++b)
        if (m + 16 * b < a.E) a.dz[te + m + 16 * b] = P[b] * (ge[b] - dot) + dl[b];
}

// A workgroup takes `chunk` tokens (a multiple of 64), whose dz it keeps in LDS, and 16 x kVec columns; its four wavefronts take tiles
// of 16 tokens.  Both products run on float matrix instructions (16x16x4: exact products, float sums), chosen so that one 16-byte load
// per lane feeds them in place: lane (g, m) = (l / 16, l % 16) loads columns c0 + m V .. of token 4g + v (row g of step v for dz^T x)
// or of expert 4s + g (step s of dz Wg), and component j of the 16 bytes is the operand of instruction j.  The result of dz Wg then has V
// consecutive columns of tokens 4g .. 4g + 3 in the lane that also gathers the dispatch's rows for them and stores 16 bytes.  dz^T x stays in registers
// over a wavefront's tiles; the four meet in LDS in wavefront order, and workgroups write partial sums [token chunk][E][d] that
// route_backward_sum_kernel adds in chunk order (one chunk: straight to the result).
// Bound by memory (k + 2 rows per token); what costs is latency, so a tile's rows are asked for ahead of the products of the tile before
// it, the first one's while dz comes (8192 tokens of 2048 columns, 16 experts, two slots: 35 us, 3.9 TB/s; asked for behind those
// products, with room for three workgroups per compute unit, 41).  Forming dz here, once per column block, took 10 us more than the launch of its own.
// KK > 0: KK slots per token, their rows of a tile in flight together; KK == 0: any number, row by row.
template <typename T, int NB, int KK>
__global__ __launch_bounds__(256, NB == 1 ? 2 : 1) void route_backward_kernel(RouteBackward a, int chunk, int columns, int chunks)
{
    constexpr int V = Store<T>::kVec, EP = 16 * NB, KN = KK > 0 ? KK : 1;
    extern __shared__ float lds[];                   // dz[chunk][EP] and 256 more, later the four wavefronts' sums of one block of experts
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int m = lane & 15, g = lane >> 4;
    const int part = blockIdx.x / columns, column = blockIdx.x - part * columns;
    const int tok0 = part * chunk, d = a.d, E = a.E;
    const bool first = column == 0;
    const int c = column * 16 * V + m * V;           // the lane's first column
    const bool col_on = c < d;
    const u32x4_t none = {0u, 0u, 0u, 0u};
    const T* const Wg = static_cast<const T*>(a.Wg);
    const T* const x = static_cast<const T*>(a.x);
    const T* const dxp = static_cast<const T*>(a.dx_packed);
    T* const dx = static_cast<T*>(a.dx);
    auto router_row = [&](int e) { return col_on && e < E ? *reinterpret_cast<const u32x4_t*>(Wg + static_cast<size_t>(e) * d + c) : none; };

    // what tile t0 reads: packed rows of its tokens first, then the rows themselves and x
    u32x4_t xv[4], rv[4][KN];
    int row[4][KN];
    auto ask_places = [&](int t0) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int tok = tok0 + t0 + 4 * g + v;
#pragma unroll
            for (int j = 0; j < KN; ++j)
                row[v][j] = KK > 0 && col_on && t0 < chunk && tok < a.T && dxp != nullptr ? a.inv[static_cast<size_t>(tok) * KN + j] : -1;
        }
    };
    auto ask_rows = [&](int t0) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int tok = tok0 + t0 + 4 * g + v;
#pragma unroll
            for (int j = 0; j < KN; ++j) rv[v][j] = row[v][j] >= 0 ? *reinterpret_cast<const u32x4_t*>(dxp + static_cast<size_t>(row[v][j]) * d + c) : none;
            xv[v] = col_on && tok < a.T && a.dWg != nullptr ? *reinterpret_cast<const u32x4_t*>(x + static_cast<size_t>(tok) * d + c) : none;
        }
    };
    ask_places(wave * 16);
    {
        float dz[4];
        int i0 = threadIdx.x;
        auto ask_dz = [&]() {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + 256 * u, tok = tok0 + i / EP, e = i % EP;
                dz[u] = tok < a.T && e < E ? a.dz[static_cast<size_t>(tok) * E + e] : 0.f;      // what only fills up a tile adds nothing
            }
        };
        auto keep_dz = [&]() {
#pragma unroll
            for (int u = 0; u < 4; ++u) lds[i0 + 256 * u] = dz[u];
        };
        ask_dz();
        ask_rows(wave * 16);                         // (loads return in order: behind the first that LDS waits for)
        keep_dz();
        for (i0 += 1024; i0 < chunk * EP; i0 += 1024) {
            ask_dz();
            keep_dz();
        }
    }
    __syncthreads();
    if (first && a.dbg != nullptr) {                 // (thread: expert t % EP, every 256 / EP-th token from t / EP on)
        float* const sums = lds + chunk * EP;
        const int e = static_cast<int>(threadIdx.x) % EP, from = static_cast<int>(threadIdx.x) / EP;
        constexpr int STEP = 256 / EP;
        if (from < STEP) {
            float sum = 0.f;
#pragma unroll 4
            for (int i = from; i < chunk; i += STEP) sum += lds[i * EP + e];
            sums[from * EP + e] = sum;
        }
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < E) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < STEP; ++i) sum += sums[i * EP + threadIdx.x];
            (chunks == 1 ? a.dbg : a.partial_dbg + static_cast<size_t>(part) * E)[threadIdx.x] = sum;
        }
    }

    f32x4_t accW[NB][V];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < V; ++j) accW[b][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    u32x4_t router[4 * NB];                          // experts past E: zeros, and dz too
    auto ask_router = [&]() {
#pragma unroll
        for (int s = 0; s < 4 * NB; ++s) router[s] = router_row(4 * s + g);
    };
    if (NB == 1) ask_router();
    ask_places(wave * 16 + 64);
    for (int t0 = wave * 16; t0 < chunk && tok0 + t0 < a.T; t0 += 64) {
        const int tok = tok0 + t0 + 4 * g;           // the lane's first token
        if (NB > 1) ask_router();
        u32x4_t xc[4], rc[4][KN];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            xc[v] = xv[v];
#pragma unroll
            for (int j = 0; j < KN; ++j) rc[v][j] = rv[v][j];
        }
        if (t0 + 64 < chunk) {
            ask_rows(t0 + 64);
            ask_places(t0 + 128);
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4_t accX[V];
#pragma unroll
        for (int j = 0; j < V; ++j) accX[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4 * NB; ++s) {
            const float dz = lds[(t0 + m) * EP + 4 * s + g];
            float w[V];
            Store<T>::unpack(router[s], w);
#pragma unroll
            for (int j = 0; j < V; ++j) accX[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(dz, w[j], accX[j], 0, 0, 0);
        }
        if (a.dWg != nullptr) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float f[V];
                Store<T>::unpack(xc[v], f);
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
            if (tok + v >= a.T || !col_on) continue;
            float sum[V];
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] = 0.f;
            auto add = [&](const u32x4_t& row) {
                float f[V];
                Store<T>::unpack(row, f);
#pragma unroll
                for (int t = 0; t < V; ++t) sum[t] += f[t];
            };
            if (KK > 0) {
#pragma unroll
                for (int j = 0; j < KN; ++j) add(rc[v][j]);
            } else if (dxp != nullptr) {
                for (int j = 0; j < a.slots; ++j) {
                    const int row = a.inv[static_cast<size_t>(tok + v) * a.slots + j];
                    if (row >= 0) add(*reinterpret_cast<const u32x4_t*>(dxp + static_cast<size_t>(row) * d + c));
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += accX[j][v];
            const uint4 packed = Store<T>::pack(sum);
            *reinterpret_cast<u32x4_t*>(dx + static_cast<size_t>(tok + v) * d + c) = u32x4_t{packed.x, packed.y, packed.z, packed.w};
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

// dWg[i] = sum over the token chunks of partial[chunk][i] for its n = E d values, four at a time, and the E values of dbg (by the last
// workgroup).  Eight threads share out the chunks of a place, so that their loads do not wait for one another, and add up in LDS; the
// order is fixed.
__global__ __launch_bounds__(256) void route_backward_sum_kernel(const float* __restrict__ partial, const float* __restrict__ partial_dbg,
                                                                 int chunks, int n, int E, float* __restrict__ dWg, float* __restrict__ dbg)
{
    __shared__ f32x4_t sums[8][32];
    const int place = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int i = (blockIdx.x * 32 + place) * 4;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    if (dWg != nullptr && i < n)
        for (int c = share; c < chunks; c += 8) sum += *reinterpret_cast<const f32x4_t*>(partial + static_cast<size_t>(c) * n + i);
    sums[share][place] = sum;
    __syncthreads();
    if (share == 0 && dWg != nullptr && i < n) {
#pragma unroll
        for (int q = 1; q < 8; ++q) sum += sums[q][place];
        *reinterpret_cast<f32x4_t*>(dWg + i) = sum;
    }
    if (dbg == nullptr || blockIdx.x != gridDim.x - 1) return;
    float total = 0.f;                               // thread (share t / 64, expert t % 64)
    __shared__ float totals[4][64];
    const int e = threadIdx.x & 63, quarter = threadIdx.x >> 6;
    if (e < E)
        for (int c = quarter; c < chunks; c += 4) total += partial_dbg[static_cast<size_t>(c) * E + e];
    totals[quarter][e] = total;
    __syncthreads();
    if (quarter == 0 && e < E) dbg[e] = (total + totals[1][e]) + (totals[2][e] + totals[3][e]);
}

namespace {

template <typename T, int NB>
void launch_route_backward_t(const RouteBackward& a, int columns, int chunk, int chunks, hipStream_t stream)
{
    const int dz = chunk * 16 * NB + 256, sums = 4 * 4 * Store<T>::kVec * kWave;
    const size_t lds = (dz > sums ? dz : sums) * sizeof(float);
#define DICEMOE_ROUTE_BWD_K(KK_) \
    hipLaunchKernelGGL((route_backward_kernel<T, NB, KK_>), dim3(columns * chunks), dim3(256), lds, stream, a, chunk, columns, chunks)
    if (a.slots == 1) DICEMOE_ROUTE_BWD_K(1);
    else if (a.slots == 2) DICEMOE_ROUTE_BWD_K(2);
    else if (a.slots == 3) DICEMOE_ROUTE_BWD_K(3);
    else if (a.slots == 4) DICEMOE_ROUTE_BWD_K(4);
    else DICEMOE_ROUTE_BWD_K(0);
#undef DICEMOE_ROUTE_BWD_K
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

static int route_columns(bool bf16, int d) { return (d + (bf16 ? 128 : 64) - 1) / (bf16 ? 128 : 64); }       // 16 x kVec columns each

// partial sums by chunks of tokens, and dz if the caller does not want it
size_t route_backward_bytes(bool bf16, long long T_max, int E, int d)
{
    const size_t chunks = static_cast<size_t>(route_chunks_most(T_max, E, route_columns(bf16, d)));
    return (chunks * E * (static_cast<size_t>(d) + 1) + static_cast<size_t>(T_max) * E) * sizeof(float);
}

hipError_t launch_route_backward(bool bf16, RouteBackward a, void* workspace, hipStream_t stream)
{
    if (a.Wg == nullptr) {
        if (a.T == 0) return hipSuccess;
        if (bf16) launch_dispatch_backward_t<bf16_t>(a, stream);
        else launch_dispatch_backward_t<float>(a, stream);
        return hipGetLastError();
    }
    const int columns = route_columns(bf16, a.d);
    const int chunk = route_chunk(a.T, a.E, columns), chunks = (a.T + chunk - 1) / chunk;
    a.partial = static_cast<float*>(workspace);
    a.partial_dbg = a.partial + static_cast<size_t>(chunks) * a.E * a.d;
    if (a.dz == nullptr) a.dz = a.partial_dbg + static_cast<size_t>(chunks) * a.E;
    if (chunks > 0) {
        const int blocks = (a.E + 15) / 16;
        auto logits = [&](auto nb) { hipLaunchKernelGGL(route_logits_kernel<decltype(nb)::value>, dim3((a.T + 15) / 16), dim3(256), 0, stream, a); };
        if (blocks == 1) logits(std::integral_constant<int, 1>{});
        else if (blocks == 2) logits(std::integral_constant<int, 2>{});
        else if (blocks == 3) logits(std::integral_constant<int, 3>{});
        else logits(std::integral_constant<int, 4>{});
        if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
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
    hipLaunchKernelGGL(route_backward_sum_kernel, dim3((n + 127) / 128), dim3(256), 0, stream, a.partial, a.partial_dbg, chunks, n, a.E, a.dWg, a.dbg);
    return hipGetLastError();
}

}  // namespace dicemoe
