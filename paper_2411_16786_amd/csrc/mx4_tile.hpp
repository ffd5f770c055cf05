// Grouped product of many rows on 4-bit weights (bf16 rows), out[r, n] = act(sum_k x[r, k] W_e[n, k] + b_e[n]), tiled through LDS.
//
// A workgroup of WN x WR wavefronts owns BN = 32 NT WN columns n of BR = 32 RT WR rows; a wavefront NT x RT blocks of 32 x 32
// (v_mfma_f32_32x32x16_bf16, weights first operand, rows second: a result register holds columns of one row).  The
// reduction goes in stages of 64: rows take 128 bytes each, codes 32, so the weights cost a quarter of the LDS space and reads that a bf16
// operand would, and one conversion instruction per two weights, in the shadow of the NT RT matrix instructions that it feeds.
// A lane's 16 bytes of codes are one scale group: lane (h, c) = (l / 32, l % 32) holds k = 32 h .. + 31 of a stage for one weight row, instruction q
// takes its q-th dword, and the rows' operand is read in the same order (16-byte chunk 4 h + q of the row).
// Stages are double-buffered: the next stage's bytes are asked for into registers before this one's products and written to the
// other buffer behind them, one barrier per stage; two workgroups per compute unit cover each other's barriers.
#pragma once
#include "ffn_mfma.hpp"
#include "kernels.hpp"
#include "mx4.hpp"

namespace dicemoe {

// Phi(-a) for a in 0 .. 6: the polynomial that gelu_erf_fast has in its body
__device__ __forceinline__ float normal_tail(float a) {
    float p = fmaf(0x1.159ab2p-15f, a, -0x1.934b26p-11f);
    p = fmaf(p, a, 0x1.08ca02p-7f);
    p = fmaf(p, a, -0x1.b58d52p-5f);
    p = fmaf(p, a, -0x1.d5c80ep-2f);
    p = fmaf(p, a, -0x1.26b528p+0f);
    p = fmaf(p, a, -0x1.ffff18p-1f);
    return __builtin_amdgcn_exp2f(p);
}
// gelu and its slope.  The bf16 forms use that polynomial; NaN stays NaN in all of them.
template <typename T> __device__ __forceinline__ float mx4_gelu(float u);
template <> __device__ __forceinline__ float mx4_gelu<float>(float u) { return gelu_erf(u); }
template <> __device__ __forceinline__ float mx4_gelu<bf16_t>(float u) { return u != u ? u : gelu_erf_fast(u); }
// gelu'(u) = Phi(u) + u phi(u); with a = |u| it is 1 - s for u >= 0 and s below, s = Phi(-a) - a phi(a)
template <typename T> __device__ __forceinline__ float gelu_slope(float u);
template <> __device__ __forceinline__ float gelu_slope<float>(float u) {
    return 0.5f * (1.0f + erff(u * 0.70710678118654752440f)) + u * (0.39894228040143267794f * expf(-0.5f * u * u));
}
template <> __device__ __forceinline__ float gelu_slope<bf16_t>(float u) {
    const float a = fminf(fabsf(u), 6.0f);
    const float bell = 0.39894228040143267794f * __builtin_amdgcn_exp2f(-0.72134752044448170368f * a * a);
    const float s = normal_tail(a) - a * bell;
    return u != u ? u : (u >= 0.0f ? 1.0f - s : s);
}

// The segment that row tile `tile` (BM rows, tiles of a segment contiguous) belongs to, found 64 segments at a time by lanes; all lanes
// of a wavefront get the same answer.  Rows from max_rows on and segments of no known expert have no tiles.
__device__ __forceinline__ bool find_tile(const Segments& s, int BM, int tile, int& expert, int& row0, int& row_end)
{
    const int lane = lane_id();
    for (int base = 0; base < s.n; base += kWave) {
        int begin = 0, end = 0, e = -1;
        if (base + lane < s.n) {
            begin = s.offsets[base + lane];
            end = s.offsets[base + lane + 1];
            e = s.expert[base + lane];
            end = end < s.max_rows ? end : s.max_rows;
        }
        const bool used = end > begin && begin >= 0 && e >= 0 && e < s.n_experts;
        const int upto = wave_scan(used ? (end - begin + BM - 1) / BM : 0);     // tiles of the lanes up to this one
        const uint64_t past = __ballot(upto > tile);
        if (past != 0) {
            const int src = __ffsll(static_cast<unsigned long long>(past)) - 1;
            const int before = src > 0 ? __builtin_amdgcn_readlane(upto, src - 1) : 0;
            expert = __builtin_amdgcn_readlane(e, src);
            row0 = __builtin_amdgcn_readlane(begin, src) + (tile - before) * BM;
            row_end = __builtin_amdgcn_readlane(end, src);
            return true;
        }
        tile -= __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    return false;
}

__device__ __forceinline__ void store8(bf16_t* p, const float* v) {
    *reinterpret_cast<u32x4_t*>(p) = u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// Result row 8 i + 4 h + j of a 32 x 32 block lies in register 4 i + j of the lanes of half h.  Weight row 16 h + 4 i + j is loaded there,
// so that a lane ends with 16 consecutive columns.
__device__ __forceinline__ int tile_weight_row(int rho) { return 16 * ((rho >> 2) & 1) + 4 * (rho >> 3) + (rho & 3); }

// Tiles of all segments in order (segment, row tile, column block), dealt to the eight XCDs in contiguous runs: workgroups go to XCDs round
// robin and each XCD has an L2 of its own, so neighbours in the list, which share rows or weights, meet in one L2.
struct TilePlace { int expert, row0, row_end, block; };
__device__ __forceinline__ bool find_tile_on_xcd(const Segments& s, int BM, int n_blocks, int id, TilePlace& at)
{
    const int lane = lane_id();
    int total = 0;
    for (int base = 0; base < s.n; base += kWave) {
        int tiles = 0;
        if (base + lane < s.n) {
            const int begin = s.offsets[base + lane], e = s.expert[base + lane];
            int end = s.offsets[base + lane + 1];
            end = end < s.max_rows ? end : s.max_rows;
            if (end > begin && begin >= 0 && e >= 0 && e < s.n_experts) tiles = (end - begin + BM - 1) / BM;
        }
        total += __builtin_amdgcn_readlane(wave_scan(tiles), kWave - 1);
    }
    const int all = total * n_blocks, run = (all + 7) / 8;
    const int own = id >> 3, t = (id & 7) * run + own;
    if (own >= run || t >= all) return false;
    const int tile = t / n_blocks;
    at.block = t - tile * n_blocks;
    return find_tile(s, BM, tile, at.expert, at.row0, at.row_end);
}

template <int NT, int RT, int WN, int WR, bool GELU>
__global__ __launch_bounds__(64 * WN * WR, 2) void mx4_tile_kernel(const bf16_t* __restrict__ x, const int32_t* __restrict__ row_index, int row_div,
                                                                  Segments seg, int N, int K, Mx4 W, const float* __restrict__ bias,
                                                                  bf16_t* __restrict__ pre, bf16_t* __restrict__ out,
                                                                  const int32_t* __restrict__ out_index, int32_t* __restrict__ status)
{
    constexpr int BN = 32 * NT * WN, BR = 32 * RT * WR, THREADS = 64 * WN * WR;
    constexpr int XC = BR * 8 / THREADS, CC = (BN * 2 + THREADS - 1) / THREADS;      // 16-byte chunks per thread and stage
    __shared__ u32x4_t xs[2][BR * 8];
    __shared__ u32x4_t cs[2][BN * 2];
    report_row_overflow(status, seg.offsets, seg.n, seg.max_rows);
    const int n_blocks = (N + BN - 1) / BN;
    TilePlace at;
    if (!find_tile_on_xcd(seg, BR, n_blocks, blockIdx.x, at)) return;
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const int wn = wave % WN, wr = wave / WN;
    const int half = lane >> 5, c32 = lane & 31;
    const int nb = at.block * BN;

    // what this thread stages: chunk c of rows is (row c / 8, place c % 8), the place holding source chunk place ^ (row / 2 % 8), and
    // chunk c of codes (row c / 2, place c % 2) with source chunk place ^ (row / 16 % 2): reads of 32 rows then spread over all banks
    const bf16_t* xp[XC];
    const uint8_t* cp[CC];
#pragma unroll
    for (int i = 0; i < XC; ++i) {
        const int c = threadIdx.x + i * THREADS, row = c >> 3;
        const int r = at.row0 + row < at.row_end ? at.row0 + row : at.row_end - 1;       // rows past the end repeat the last; never stored
        xp[i] = x + static_cast<size_t>(row_index ? row_index[r] / row_div : r) * K + ((c & 7) ^ ((row >> 1) & 7)) * 8;
    }
#pragma unroll
    for (int i = 0; i < CC; ++i) {
        const int c = threadIdx.x + i * THREADS, row = (c >> 1) & (BN - 1);
        const int n = nb + row < N ? nb + row : N - 1;
        cp[i] = W.codes + (static_cast<size_t>(at.expert) * N + n) * (K / 2) + ((c & 1) ^ ((row >> 4) & 1)) * 16;
    }
    const uint8_t* sp[NT];
    int c_off[NT], x_off[4];
    const int wrow = tile_weight_row(c32);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = (wn * NT + t) * 32 + wrow;
        const int n = nb + row < N ? nb + row : N - 1;
        sp[t] = W.scales + (static_cast<size_t>(at.expert) * N + n) * (K / kMxGroup) + half;
        c_off[t] = row * 2 + (half ^ ((row >> 4) & 1));
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int row = wr * RT * 32 + c32;
        x_off[q] = row * 8 + ((half * 4 + q) ^ ((row >> 1) & 7));
    }

    f32x16_v acc[NT][RT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[t][r][v] = 0.f;
    const bool live = at.row0 + wr * RT * 32 < at.row_end && nb + wn * NT * 32 < N;

    u32x4_t xv[XC], cv[CC];
    uint32_t sv[NT];
    auto ask = [&](int s) {
#pragma unroll
        for (int i = 0; i < CC; ++i) cv[i] = *reinterpret_cast<const u32x4_t*>(cp[i] + s * 32);
#pragma unroll
        for (int i = 0; i < XC; ++i) xv[i] = *reinterpret_cast<const u32x4_t*>(xp[i] + s * 64);
#pragma unroll
        for (int t = 0; t < NT; ++t) sv[t] = sp[t][s * 2];
    };
    auto keep = [&](int b) {
#pragma unroll
        for (int i = 0; i < CC; ++i)
            if (BN * 2 % THREADS == 0 || static_cast<int>(threadIdx.x) + i * THREADS < BN * 2) cs[b][threadIdx.x + i * THREADS] = cv[i];
#pragma unroll
        for (int i = 0; i < XC; ++i) xs[b][threadIdx.x + i * THREADS] = xv[i];
    };
    const int stages = K / 64;
    ask(0);
    keep(0);
    float scale[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) scale[t] = mx4_scale(sv[t]);
    __syncthreads();
    for (int s = 0; s < stages; ++s) {
        const int b = s & 1;
        if (s + 1 < stages) ask(s + 1);
        if (live) {
            u32x4_t codes[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) codes[t] = cs[b][c_off[t]];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                u32x4_t rows[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) rows[r] = xs[b][x_off[q] + r * 32 * 8];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const u32x4_t a = {mx4_bf16<0>(codes[t][q], scale[t]), mx4_bf16<1>(codes[t][q], scale[t]),
                                       mx4_bf16<2>(codes[t][q], scale[t]), mx4_bf16<3>(codes[t][q], scale[t])};
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        acc[t][r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_v*>(&a),
                                                                            *reinterpret_cast<const bf16x8_v*>(&rows[r]), acc[t][r], 0, 0, 0);
                }
            }
        }
        if (s + 1 < stages) {
            keep(b ^ 1);
#pragma unroll
            for (int t = 0; t < NT; ++t) scale[t] = mx4_scale(sv[t]);
        }
        __syncthreads();
    }
    if (!live) return;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = at.row0 + (wr * RT + r) * 32 + c32;
        if (row >= at.row_end) continue;
        bf16_t* const to = out + static_cast<size_t>(out_index ? out_index[row] : row) * N;
        bf16_t* const pre_to = pre ? pre + static_cast<size_t>(row) * N : nullptr;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int n = nb + (wn * NT + t) * 32 + half * 16;
            if (n >= N) continue;
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = acc[t][r][i];
            if (bias) {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4_t add = *reinterpret_cast<const f32x4_t*>(bias + static_cast<size_t>(at.expert) * N + n + i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[i + j] += add[j];
                }
            }
            if (pre_to) {
                store8(pre_to + n, v);
                store8(pre_to + n + 8, v + 8);
            }
            if (GELU) {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = mx4_gelu<bf16_t>(v[i]);
            }
            store8(to + n, v);
            store8(to + n + 8, v + 8);
        }
    }
}

}  // namespace dicemoe
