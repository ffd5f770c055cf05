// Expert FFN on 4-bit weights (mx4.hpp), forward and gradient of its rows, as grouped products over segments of rows.
//   forward : u = x W1_e^T + b1_e,   h = gelu(u) W2_e^T + b2_e        (gelu(u) rounded to the storage type once)
//   gradient: du = (dh W2_e) gelu'(u),   dx = du W1_e                 (du rounded to the storage type once)
// In bf16 those two roundings are the matrix instructions' own: what the second product reads is a bf16 operand, as in the FFN on bf16
// weights; two bf16 parts for each value would double its products.  They raise the distance of h and dx from the exact result from
// 0.0017 of its size, the last rounding's, to 0.0023.  (du is rounded whether or not the caller keeps it: dx has the same bits.)
// The weights are the first operand of the matrix instructions and the rows the second, so a result register holds four
// output columns of one row.  The kernels for few rows below take the weights from memory to the instruction through registers alone, converted
// on the way; the tiles for many rows (mx4_tile.hpp, mx4_tile_t.hpp) stage codes and scales through LDS.
#include <type_traits>
#include "ffn_mfma.hpp"
#include "kernels.hpp"
#include "mx4.hpp"
#include "mx4_plan.hpp"
#include "mx4_tile.hpp"
#include "mx4_tile_t.hpp"

namespace dicemoe {

__device__ __forceinline__ void store4(bf16_t* p, const float* v) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}
__device__ __forceinline__ void store4(float* p, const float* v) {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
}

// Forward product of few rows: out[r, n] = act(sum_k x[r, k] W_e[n, k] + b[n]).  A workgroup takes 16 rows and 16 NT columns n; its KS
// wavefronts share out the reduction in steps of 128 and meet in LDS.  Lane (g, m) = (l / 16, l % 16) loads the 16 bytes of
// codes, the scale and the row's values of k = 128 s + 32 g .. + 31 for its row of weights and its row of x: a lane's 16 bytes are
// exactly one scale group.  The order of k inside a step does not matter as long as both operands have the same.
// Bound by the weights' bytes and, with few of them, by one trip to memory: a wavefront asks for everything of a step at once.
template <typename T, int NT, int KS, bool GELU>
__global__ __launch_bounds__(KS * kWave) void mx4_rows_kernel(const T* __restrict__ x, const int32_t* __restrict__ row_index, int row_div,
                                                              Segments seg, int N, int K, Mx4 W, const float* __restrict__ bias,
                                                              T* __restrict__ pre, T* __restrict__ out,
                                                              const int32_t* __restrict__ out_index, int32_t* __restrict__ status)
{
    constexpr int XV = 32 / Store<T>::kVec;                     // 16-byte loads of a row per step
    __shared__ f32x4_t red[KS][NT][kWave];
    report_row_overflow(status, seg.offsets, seg.n, seg.max_rows);
    const int n_blocks = (N + 16 * NT - 1) / (16 * NT);
    const int tile = blockIdx.x / n_blocks, nb = (blockIdx.x - tile * n_blocks) * 16 * NT;
    int expert, row0, row_end;
    if (!find_tile(seg, 16, tile, expert, row0, row_end)) return;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int m = lane & 15, g = lane >> 4;

    const int r = row0 + m < row_end ? row0 + m : row_end - 1;  // rows past the end repeat the last; never stored
    const T* const xr = x + static_cast<size_t>(row_index ? row_index[r] / row_div : r) * K;
    const uint8_t *wc[NT], *ws[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        int n = nb + (m >> 2) * 4 * NT + t * 4 + (m & 3);       // result registers of a lane: 4 NT consecutive columns
        n = n < N ? n : N - 1;
        const size_t row = static_cast<size_t>(expert) * N + n;
        wc[t] = W.codes + row * (K / 2);
        ws[t] = W.scales + row * (K / kMxGroup);
    }
    f32x4_t acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // AHEAD: what the next step needs is under way behind this one's products (one token, 4608 -> 1152 6.0 us against 6.6).  With two sets
    // of weights the registers cost more where a wavefront has one or two steps (16 rows over 8 experts, 1152 -> 4608 9.4 against 7.4; 26 over
    // 16, 2048 -> 8192 46.6 against 39.5); with eight steps, 8192 -> 2048, 16 rows take 32.1 against 31.1, 26 rows 41.6 against 45.2 and 40 rows
    // 43.6 against 47.7, which is left as it is
    constexpr bool AHEAD = NT == 1;
    u32x4_t c_next[NT], x_next[XV];
    uint32_t s_next[NT];
    auto ask = [&](int k0) {
        const int k = k0 + g * 32;
        const bool on = k < K;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            c_next[t] = on ? *reinterpret_cast<const u32x4_t*>(wc[t] + k / 2) : u32x4_t{0u, 0u, 0u, 0u};
            s_next[t] = on ? ws[t][k / kMxGroup] : 0u;
        }
#pragma unroll
        for (int i = 0; i < XV; ++i) x_next[i] = on ? *reinterpret_cast<const u32x4_t*>(xr + k + i * Store<T>::kVec) : u32x4_t{0u, 0u, 0u, 0u};
    };
    if (AHEAD && wave * 128 < K) ask(wave * 128);
    for (int k0 = wave * 128; k0 < K; k0 += KS * 128) {
        u32x4_t c[NT], xv[XV];
        float s[NT];
        if (!AHEAD) ask(k0);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            c[t] = c_next[t];
            s[t] = mx4_scale(s_next[t]);
        }
#pragma unroll
        for (int i = 0; i < XV; ++i) xv[i] = x_next[i];
        if (AHEAD) {
            if (k0 + KS * 128 < K) ask(k0 + KS * 128);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) {                       // eight codes
                if constexpr (sizeof(T) == 2) {
                    const u32x4_t a = {mx4_bf16<0>(c[t][q], s[t]), mx4_bf16<1>(c[t][q], s[t]), mx4_bf16<2>(c[t][q], s[t]), mx4_bf16<3>(c[t][q], s[t])};
                    acc[t] = RowMfma<bf16_t>::step(a, xv[q], acc[t], 0);
                } else {
                    const f32x2_t p0 = mx4_f32<0>(c[t][q], s[t]), p1 = mx4_f32<1>(c[t][q], s[t]), p2 = mx4_f32<2>(c[t][q], s[t]), p3 = mx4_f32<3>(c[t][q], s[t]);
                    const float a[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], __uint_as_float(xv[2 * q + i / 4][i % 4]), acc[t], 0, 0, 0);
                }
            }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) red[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < NT; t += KS) {
        f32x4_t sum = red[0][t][lane];
#pragma unroll
        for (int w = 1; w < KS; ++w) sum += red[w][t][lane];
        const int n = nb + g * 4 * NT + t * 4;
        if (row0 + m >= row_end || n >= N) continue;
        if (bias) sum += *reinterpret_cast<const f32x4_t*>(bias + static_cast<size_t>(expert) * N + n);
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        if (pre) store4(pre + static_cast<size_t>(r) * N + n, v);
        if (GELU) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = mx4_gelu<T>(v[i]);
        }
        store4(out + static_cast<size_t>(out_index ? out_index[r] : r) * N + n, v);
    }
}

// Transposed product of few rows, for the gradient: out[r, k] = sum_n y[r, n] W_e[n, k], times gelu'(u[r, k]) with SLOPE.  A workgroup
// takes 16 rows and 16 C columns k (C = 2 CB, CB bytes of codes a lane); its KS wavefronts share out the reduction in steps of 32 rows of weights.
// Lane (g, m) loads, for n = 32 s + 8 g + q (q = 0 .. 7), the codes of columns k = kb + C m .. and their scale; matrix instruction i
// takes column i of every lane's C, i.e. its result row 4 g + v stands for column kb + (4 g + v) C + i.  In bf16 a conversion gives two columns
// of one n, and pairs along n are put together by byte permutation: one conversion and one permutation per two weights.
template <typename T, int CB, int KS, bool SLOPE>
__global__ __launch_bounds__(KS * kWave) void mx4_rows_transposed_kernel(const T* __restrict__ y, Segments seg, int N, int K, Mx4 W,
                                                                  const T* __restrict__ u, T* __restrict__ out, int32_t* __restrict__ status)
{
    constexpr int C = 2 * CB, YV = 8 / Store<T>::kVec;
    static_assert(KS >= 4 && (CB == 4 || (CB == 1 && sizeof(T) == 4)), "a thread for every C results; a dword of codes, or a byte (float)");
    __shared__ f32x4_t red[KS][C][kWave];
    report_row_overflow(status, seg.offsets, seg.n, seg.max_rows);
    const int k_blocks = (K + 16 * C - 1) / (16 * C);
    const int tile = blockIdx.x / k_blocks, kb = (blockIdx.x - tile * k_blocks) * 16 * C;
    int expert, row0, row_end;
    if (!find_tile(seg, 16, tile, expert, row0, row_end)) return;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int m = lane & 15, g = lane >> 4;
    const int r = row0 + m < row_end ? row0 + m : row_end - 1;
    const int k = kb + m * C;
    const bool on = k < K;
    const size_t first = static_cast<size_t>(expert) * N + g * 8;
    const uint8_t* const wc = W.codes + first * (K / 2) + (on ? k / 2 : 0);
    const uint8_t* const ws = W.scales + first * (K / kMxGroup) + (on ? k / kMxGroup : 0);
    const T* const yr = y + static_cast<size_t>(r) * N + g * 8;
    f32x4_t acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // (double buffer: what the next step needs is under way behind this one's products)
    uint32_t c_next[8], s_next[8];
    u32x4_t y_next[YV];
    auto ask = [&](int n0) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {                           // (columns past the end repeat the first; never stored)
            const uint8_t* const from = wc + static_cast<size_t>(n0 + q) * (K / 2);
            c_next[q] = CB == 4 ? *reinterpret_cast<const uint32_t*>(from) : *from;
            s_next[q] = ws[static_cast<size_t>(n0 + q) * (K / kMxGroup)];
        }
#pragma unroll
        for (int i = 0; i < YV; ++i) y_next[i] = *reinterpret_cast<const u32x4_t*>(yr + n0 + i * Store<T>::kVec);
    };
    if (wave * 32 < N) ask(wave * 32);
    for (int n0 = wave * 32; n0 < N; n0 += KS * 32) {
        uint32_t c[8];
        float s[8];
        u32x4_t yv[YV];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            c[q] = c_next[q];
            s[q] = mx4_scale(s_next[q]);
        }
#pragma unroll
        for (int i = 0; i < YV; ++i) yv[i] = y_next[i];
        if (n0 + KS * 32 < N) ask(n0 + KS * 32);
        __builtin_amdgcn_sched_barrier(0);
        auto columns = [&](auto B) {                            // columns 2 B and 2 B + 1
            constexpr int b = decltype(B)::value;
            if constexpr (sizeof(T) == 2) {
                u32x4_t lo, hi;
#pragma unroll
                for (int q = 0; q < 8; q += 2) {
                    const uint32_t p0 = mx4_bf16<b>(c[q], s[q]), p1 = mx4_bf16<b>(c[q + 1], s[q + 1]);
                    lo[q / 2] = __builtin_amdgcn_perm(p1, p0, 0x05040100u);
                    hi[q / 2] = __builtin_amdgcn_perm(p1, p0, 0x07060302u);
                }
                acc[2 * b] = RowMfma<bf16_t>::step(lo, yv[0], acc[2 * b], 0);
                acc[2 * b + 1] = RowMfma<bf16_t>::step(hi, yv[0], acc[2 * b + 1], 0);
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const f32x2_t p = mx4_f32<b>(c[q], s[q]);
                    const float v = __uint_as_float(yv[q / 4][q % 4]);
                    acc[2 * b] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[0], v, acc[2 * b], 0, 0, 0);
                    acc[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[1], v, acc[2 * b + 1], 0, 0, 0);
                }
            }
        };
        columns(std::integral_constant<int, 0>{});
        if constexpr (CB == 4) {
            columns(std::integral_constant<int, 1>{});
            columns(std::integral_constant<int, 2>{});
            columns(std::integral_constant<int, 3>{});
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) red[wave][i][lane] = acc[i];
    __syncthreads();
    // thread (row, place): place 4 g + v of the row's 16 C columns
    const int row = threadIdx.x >> 4, place = threadIdx.x & 15;
    const int ko = kb + place * C;
    if (row0 + row >= row_end || ko >= K || threadIdx.x >= 256) return;
    float v[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int from = (place >> 2) * 16 + row;
        v[i] = red[0][i][from][place & 3];
#pragma unroll
        for (int w = 1; w < KS; ++w) v[i] += red[w][i][from][place & 3];
    }
    const size_t at = static_cast<size_t>(row0 + row) * K + ko;
    if (SLOPE) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if constexpr (sizeof(T) == 2) v[i] *= gelu_slope<T>(bf16_to_float(u[at + i]));
            else v[i] *= gelu_slope<T>(u[at + i]);
        }
    }
    if constexpr (C == 8) {
        store4(out + at, v);
        store4(out + at + 4, v + 4);
    } else {
        *reinterpret_cast<f32x2_t*>(out + at) = f32x2_t{v[0], v[1]};
    }
}

namespace {

// A tile of the plan as its kernel takes it: 32 RT rows, 32 WN columns (64 WN in the transposed kernel), the reduction in KS shares
template <int RT_, int WN_, int KS_> struct Tile { static constexpr int RT = RT_, WN = WN_, KS = KS_; };
template <int I> using PlanTile = Tile<kTile[I].rows / 32, kTile[I].columns / 32, kTile[I].shares>;
template <int I> using PlanTileT = Tile<kTileT[I].rows / 32, kTileT[I].columns / 64, kTileT[I].shares>;

// the LDS that the plan weighs a tile by is what its kernel takes
template <int I, int K> constexpr bool kLdsAsPlanned =
    TileShape<PlanTile<I>::RT, PlanTile<I>::WN, PlanTile<I>::KS, false>::lds_bytes(K) == tile_lds(I, K, false) &&
    TileShape<PlanTile<I>::RT, PlanTile<I>::WN, PlanTile<I>::KS, true>::lds_bytes(K) == tile_lds(I, K, true);
template <int I> constexpr bool kTileAsPlanned = kTile[I].rows % 32 == 0 && kTile[I].columns % 32 == 0 && kLdsAsPlanned<I, 64> && kLdsAsPlanned<I, 1152> && kLdsAsPlanned<I, 8192>;
static_assert(kTiles == 6 && kTileAsPlanned<0> && kTileAsPlanned<1> && kTileAsPlanned<2> && kTileAsPlanned<3> && kTileAsPlanned<4> && kTileAsPlanned<5>, "mx4_plan.hpp");
static_assert(kTilesT == 3, "with_tile_t");

// Calls f with the shape of a tile and whether its scales go by chunks
template <typename F>
void with_tile(int tile, int K, F&& f)
{
    const bool chunks = tile_chunks(tile, K);
    auto go = [&](auto shape) {
        if (chunks) f(shape, std::true_type{});
        else f(shape, std::false_type{});
    };
    if (tile == 0) go(PlanTile<0>{});
    else if (tile == 1) go(PlanTile<1>{});
    else if (tile == 2) go(PlanTile<2>{});
    else if (tile == 3) go(PlanTile<3>{});
    else if (tile == 4) go(PlanTile<4>{});
    else go(PlanTile<5>{});
}

template <typename F>
void with_tile_t(int tile, F&& f)
{
    if (tile == 0) f(PlanTileT<0>{});
    else if (tile == 1) f(PlanTileT<1>{});
    else f(PlanTileT<2>{});
}

template <typename Shape>
hipError_t configure_tile()
{
    const void* const kernels[] = {reinterpret_cast<const void*>(&mx4_tile_kernel<Shape::RT, Shape::WN, Shape::KS, false, false>),
                                   reinterpret_cast<const void*>(&mx4_tile_kernel<Shape::RT, Shape::WN, Shape::KS, false, true>),
                                   reinterpret_cast<const void*>(&mx4_tile_kernel<Shape::RT, Shape::WN, Shape::KS, true, false>),
                                   reinterpret_cast<const void*>(&mx4_tile_kernel<Shape::RT, Shape::WN, Shape::KS, true, true>)};
    for (const void* kernel : kernels)
        if (hipError_t err = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes); err != hipSuccess) return err;
    return hipSuccess;
}

template <typename T, bool GELU>
void rows_product(const void* x, const int32_t* row_index, int row_div, const Segments& seg, int N, int K, const Mx4& W, const float* bias,
                  void* pre, void* out, const int32_t* out_index, int32_t* status, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        const int tile = pick_tile(seg.max_rows, seg.n, N, K);
        if (tile >= 0) {
            with_tile(tile, K, [&](auto shape, auto chunks) {
                constexpr int RT = decltype(shape)::RT, WN = decltype(shape)::WN, KS = decltype(shape)::KS;
                constexpr bool CHUNKS = decltype(chunks)::value;
                typedef TileShape<RT, WN, KS, CHUNKS> S;
                const long long blocks = (tile_bound(seg.max_rows, seg.n, S::BR) * ((N + S::BN - 1) / S::BN) + 7) / 8 * 8;
                hipLaunchKernelGGL((mx4_tile_kernel<RT, WN, KS, CHUNKS, GELU>), dim3(static_cast<unsigned>(blocks)), dim3(KS * S::kThreads), S::lds_bytes(K),
                                   stream, static_cast<const T*>(x), row_index, row_div, seg, N, K, W, bias, static_cast<T*>(pre), static_cast<T*>(out),
                                   out_index, status);
            });
            return;
        }
    }
    auto go = [&](auto sets, auto shares) {
        constexpr int NT = decltype(sets)::value, KS = decltype(shares)::value;
        const long long blocks = tile_bound(seg.max_rows, seg.n, 16) * ((N + 16 * NT - 1) / (16 * NT));
        hipLaunchKernelGGL((mx4_rows_kernel<T, NT, KS, GELU>), dim3(static_cast<unsigned>(blocks)), dim3(KS * kWave), 0, stream, static_cast<const T*>(x),
                           row_index, row_div, seg, N, K, W, bias, static_cast<T*>(pre), static_cast<T*>(out), out_index, status);
    };
    if constexpr (sizeof(T) == 4) {
        if (rows_wide(seg.max_rows, seg.n, N)) return go(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
    }
    if (rows_narrow(seg.max_rows, seg.n, N)) go(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 2>{}, std::integral_constant<int, 8>{});
}

template <typename T, bool SLOPE>
void transposed_product(const void* y, const Segments& seg, int N, int K, const Mx4& W, const void* u, void* out, int32_t* status, hipStream_t stream)
{
    if constexpr (sizeof(T) == 2) {
        const int tile = pick_tile_t(seg.max_rows, seg.n, K);
        if (tile >= 0) {
            with_tile_t(tile, [&](auto shape) {
                constexpr int RT = decltype(shape)::RT, WN = decltype(shape)::WN, KS = decltype(shape)::KS;
                typedef TileShapeT<RT, WN, KS> S;
                static_assert(KS == PlanTileT<2>::KS || S::kLds <= 64 * 1024, "prepare_expert_ffn_mx4 raises the limit of that one");
                const long long blocks = (tile_bound(seg.max_rows, seg.n, S::BR) * ((K + S::BK - 1) / S::BK) + 7) / 8 * 8;
                hipLaunchKernelGGL((mx4_tile_transposed_kernel<RT, WN, KS, SLOPE>), dim3(static_cast<unsigned>(blocks)), dim3(KS * S::kThreads), S::kLds, stream,
                                   static_cast<const T*>(y), seg, N, K, W, static_cast<const T*>(u), static_cast<T*>(out), status);
            });
            return;
        }
    }
    // Eight shares where each has three steps of 32 at least (two rows in bf16: 4608 -> 1152 13.8 us against 20.8 with four, 1536 -> 384 7.5
    // and 8.8; float, 1000 rows, 384 -> 1536 29 against 25).  Float, whose matrix instructions take an eighth of the rate: 32 columns and
    // sixteen shares where 128 columns leave half of the compute units empty (two rows, 4608 -> 1152 20 us against 47, 1152 -> 4608 17
    // both; in bf16 12 against 7 and 12 against 13).
    auto go = [&](auto bytes, auto shares) {
        constexpr int CB = decltype(bytes)::value, KS = decltype(shares)::value;
        const long long blocks = tile_bound(seg.max_rows, seg.n, 16) * ((K + 32 * CB - 1) / (32 * CB));
        hipLaunchKernelGGL((mx4_rows_transposed_kernel<T, CB, KS, SLOPE>), dim3(static_cast<unsigned>(blocks)), dim3(KS * kWave), 0, stream,
                           static_cast<const T*>(y), seg, N, K, W, static_cast<const T*>(u), static_cast<T*>(out), status);
    };
    if constexpr (sizeof(T) == 4) {
        if (2 * tile_bound(seg.max_rows, seg.n, 16) * ((K + 127) / 128) <= kComputeUnits) return go(std::integral_constant<int, 1>{}, std::integral_constant<int, 16>{});
    }
    if (N >= 768) go(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
}

template <typename T>
hipError_t ffn_t(const void* x_rows, const int32_t* row_index, int row_div, const Segments& seg, int d, int F, const Mx4& W1, const float* b1,
                 const Mx4& W2, const float* b2, void* pre, void* h_out, const int32_t* out_index, void* hidden, int32_t* status, hipStream_t stream,
                 hipEvent_t between)
{
    rows_product<T, true>(x_rows, row_index, row_div, seg, F, d, W1, b1, pre, hidden, nullptr, status, stream);
    if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
    if (between != nullptr)
        if (hipError_t err = hipEventRecord(between, stream); err != hipSuccess) return err;
    rows_product<T, false>(hidden, nullptr, 1, seg, d, F, W2, b2, nullptr, h_out, out_index, nullptr, stream);
    return hipGetLastError();
}

template <typename T>
hipError_t ffn_backward_t(const void* dh, const void* u, const Segments& seg, int d, int F, const Mx4& W1, const Mx4& W2, void* du, void* dx,
                          int32_t* status, hipStream_t stream, hipEvent_t between)
{
    transposed_product<T, true>(dh, seg, d, F, W2, u, du, status, stream);
    if (hipError_t err = hipGetLastError(); err != hipSuccess) return err;
    if (between != nullptr)
        if (hipError_t err = hipEventRecord(between, stream); err != hipSuccess) return err;
    transposed_product<T, false>(du, seg, F, d, W1, nullptr, dx, nullptr, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t prepare_expert_ffn_mx4()
{
    hipError_t err = configure_tile<PlanTile<0>>();
    if (err == hipSuccess) err = configure_tile<PlanTile<1>>();
    if (err == hipSuccess) err = configure_tile<PlanTile<2>>();
    if (err == hipSuccess) err = configure_tile<PlanTile<3>>();
    if (err == hipSuccess) err = configure_tile<PlanTile<4>>();
    if (err == hipSuccess) err = configure_tile<PlanTile<5>>();
    typedef PlanTileT<2> Shares;
    const auto shares = reinterpret_cast<const void*>(&mx4_tile_transposed_kernel<Shares::RT, Shares::WN, Shares::KS, false>);
    const auto shares_slope = reinterpret_cast<const void*>(&mx4_tile_transposed_kernel<Shares::RT, Shares::WN, Shares::KS, true>);
    for (const void* kernel : {shares, shares_slope})            // (the other transposed tiles need less than the 64 KiB that every kernel has)
        if (err == hipSuccess) err = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes);
    return err;
}

hipError_t launch_expert_ffn_mx4(bool bf16, const void* x_rows, const int32_t* row_index, int row_div, const Segments& seg, int d, int F,
                                 const Mx4& W1, const float* b1, const Mx4& W2, const float* b2, void* pre, void* h_out,
                                 const int32_t* out_index, void* hidden, int32_t* status, hipStream_t stream, hipEvent_t between)
{
    return (bf16 ? ffn_t<bf16_t> : ffn_t<float>)(x_rows, row_index, row_div, seg, d, F, W1, b1, W2, b2, pre, h_out, out_index, hidden, status, stream, between);
}

hipError_t launch_expert_ffn_mx4_backward(bool bf16, const void* dh, const void* u, const Segments& seg, int d, int F, const Mx4& W1,
                                          const Mx4& W2, void* du, void* dx, int32_t* status, hipStream_t stream, hipEvent_t between)
{
    return (bf16 ? ffn_backward_t<bf16_t> : ffn_backward_t<float>)(dh, u, seg, d, F, W1, W2, du, dx, status, stream, between);
}

}  // namespace dicemoe
