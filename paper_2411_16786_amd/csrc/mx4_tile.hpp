// Grouped product of many rows on 4-bit weights (bf16 rows), out[r, n] = act(sum_k x[r, k] W_e[n, k] + b_e[n]), tiled through LDS.
//
// A workgroup of WN wavefronts owns 32 WN columns n of 32 RT rows; wavefront w the 32 columns from 32 w, all rows: RT blocks of 32 x 32
// (v_mfma_f32_32x32x16_bf16, weights first operand, rows second: a result register holds columns of one row).  The reduction goes in
// stages of 64: 128 bytes of a row, 32 of codes, so the weights take a quarter of the LDS space and reads of a bf16 operand and
// are converted in one wavefront only, one instruction per two weights in the shadow of the RT matrix instructions that use them.
// A lane's 16 bytes of codes are one scale group: lane (h, c) = (l / 32, l % 32) holds k = 32 h .. + 31 of a stage for one weight row, slice
// q of the stage takes its q-th dword, and the rows' operand is read in the same order (16-byte chunk 4 h + q of the row).
//
// Direct-to-LDS loads, two stages of rows and two pairs of stages of codes in the LDS: what a stage has left is asked for again behind
// its barrier, which stands before the stage's last slice, so that barrier and first reads of the next stage lie behind matrix
// instructions.  What takes the time there, by counters over 8192 rows and 8 experts, 1152 -> 4608 and 4608 -> 1152: the matrix pipes are
// busy 47 and 42 % of the cycles, a wavefront waits 37 and 45 % of its time for a stage or at a barrier and 38 and 26 % to issue; more wavefronts
// per SIMD hide both, which is why the rings are short.  That is not the limit of the instruction stream: at 8192 -> 4096, 128 stages a tile
// instead of 18, the widest tile holds 1.24 PFLOP/s against 0.98 at 1152 -> 4608.  What differs is the start and the epilogue of a tile, paid every 18
// stages, and a last round of workgroups that is partly filled (1152 tiles and more on the 512 places of two a compute unit).
// 8192 rows over 8 experts (us, medians of 54 calls; this library's bf16 GEMMs take 105 with GELU
// and 92): 1152 -> 4608 with GELU, 256 x 128 tiles 89, 128 x 128 108, 128 x 64 101; 4608 -> 1152, 128 x 64 91, 128 x 128 92,
// 256 x 128 102.  Rings of three stages, one workgroup less per compute unit: 113, 101, 105 and 103, 123, 115.  Stages through
// registers: 110 and 122 at best.
#pragma once
#include <type_traits>
#include "ffn_mfma.hpp"
#include "kernels.hpp"
#include "mx4.hpp"

namespace dicemoe {

// gelu and its slope.  The float forms take Phi(u) from erfc, which keeps its digits where Phi is small (1 + erf, a difference there, is off
// by 4 % of itself at u = -5 and by half at -5.5); the bf16 forms use normal_tail's polynomial; NaN stays NaN in all of them.
template <typename T> __device__ __forceinline__ float mx4_gelu(float u);
template <> __device__ __forceinline__ float mx4_gelu<float>(float u) {
    const float c = u < -40.0f ? -40.0f : u;                    // (-infinity times its zero is no number; gelu is zero from -15 on)
    return 0.5f * c * erfcf(c * -0.70710678118654752440f);
}
template <> __device__ __forceinline__ float mx4_gelu<bf16_t>(float u) { return u != u ? u : gelu_erf_fast(u); }
// gelu'(u) = Phi(u) + u phi(u); with a = |u| it is 1 - s for u >= 0 and s below, s = Phi(-a) - a phi(a).  The bf16 form is within 2.5e-6 of it (near 0, where
// the polynomial's Phi(-a) is furthest off; 1e-7 from 3 on), a thousandth of the rounding that du receives next.
template <typename T> __device__ __forceinline__ float gelu_slope(float u);
template <> __device__ __forceinline__ float gelu_slope<float>(float u) {
    const float a = fminf(fabsf(u), 40.0f);                     // (infinity times the bell's zero is no number; u phi(u) is zero from 15 on)
    return 0.5f * erfcf(u * -0.70710678118654752440f) + copysignf(a, u) * (0.39894228040143267794f * expf(-0.5f * a * a));
}
template <> __device__ __forceinline__ float gelu_slope<bf16_t>(float u) {
    float a;
    const float tail = normal_tail(u, a);
    const float bell = 0.39894228040143267794f * __builtin_amdgcn_exp2f(-0.72134752044448170368f * a * a);
    const float s = a < 6.0f ? tail - a * bell : 0.0f;          // (-3.6e-8 at 6, and zero soon after)
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

__device__ __forceinline__ void wait_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4)); }
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

// BN columns, BR rows.  CHUNKS: scales in chunks of 512 reduction columns (16 bytes a row, two chunks in the LDS; K % 512 == 0) instead
// of all of them at once (rows of weights are adjacent in memory, so is what is staged).
template <int RT, int WN, int KS, bool CHUNKS> struct TileShape {
    static constexpr int BN = 32 * WN, BR = 32 * RT, kThreads = 64 * WN;            // (of one share)
    static constexpr int kRowBytes = BR * 128, kCodeBytes = BN * 64;           // of a stage, of a pair of stages
    static constexpr int kRowLoads = kRowBytes / 16 / kThreads, kCodeLoads = kCodeBytes / 16 / kThreads;       // per wavefront
    static_assert(kRowBytes % (16 * kThreads) == 0 && kCodeBytes % (16 * kThreads) == 0, "whole loads");
    static constexpr int kShareBytes = 2 * kRowBytes + 2 * kCodeBytes + (CHUNKS ? 2 * BN * 16 : 0);
    static constexpr int scale_bytes(int K) { return CHUNKS ? 0 : (BN / 32 * K + 16 * KS * kThreads - 1) / (16 * KS * kThreads) * (16 * KS * kThreads); }
    static constexpr int lds_bytes(int K) { return KS * kShareBytes + scale_bytes(K); }
    static_assert((KS - 1) * RT * 64 * kThreads <= KS * kShareBytes, "the shares' sums fit where their stages were");
};

template <int RT, int WN, int KS, bool CHUNKS, bool GELU>
__global__ __launch_bounds__(64 * WN * KS, 2) void mx4_tile_kernel(const bf16_t* __restrict__ x, const int32_t* __restrict__ row_index, int row_div,
                                                           Segments seg, int N, int K, Mx4 W, const float* __restrict__ bias,
                                                           bf16_t* __restrict__ pre, bf16_t* __restrict__ out,
                                                           const int32_t* __restrict__ out_index, int32_t* __restrict__ status)
{
    typedef TileShape<RT, WN, KS, CHUNKS> S;
    constexpr int BN = S::BN, BR = S::BR, XC = S::kRowLoads, CC = S::kCodeLoads;
    extern __shared__ __attribute__((aligned(16))) char lds_all[];
    report_row_overflow(status, seg.offsets, seg.n, seg.max_rows);
    const int n_blocks = (N + BN - 1) / BN;
    TilePlace at;
    if (!find_tile_on_xcd(seg, BR, n_blocks, blockIdx.x, at)) return;
    const int lane = lane_id(), wave_all = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int wave = wave_all % WN, share = wave_all / WN;      // of the share
    const int half = lane >> 5, c32 = lane & 31;
    const int nb = at.block * BN;
    char* const lds = lds_all + share * S::kShareBytes;
    char* const code_lds = lds + 2 * S::kRowBytes;
    char* const scale_lds = CHUNKS ? code_lds + 2 * S::kCodeBytes : lds_all + KS * S::kShareBytes;

    // Rows in the LDS: 16-byte chunk c of a row's 128 bytes lies at place c ^ (row / 2 % 8).  Codes: chunk c of a row's 64 bytes at
    // place c ^ (bits 2 and 4 of the row).  Reads of 16 rows at a time then touch every bank once.
    uint32_t x_from[XC], c_from[CC], c_second[CC];              // byte offsets from x and from the tile's first code; 32 for a chunk of an odd stage
#pragma unroll
    for (int i = 0; i < XC; ++i) {
        const int row = (wave * XC + i) * 8 + (lane >> 3);
        const int r = at.row0 + row < at.row_end ? at.row0 + row : at.row_end - 1;       // rows past the end repeat the last; never stored
        x_from[i] = static_cast<uint32_t>(row_index ? row_index[r] / row_div : r) * (2u * K) + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
    const int rows_here = N - nb < BN ? N - nb : BN;            // columns past N repeat the last; never stored
#pragma unroll
    for (int i = 0; i < CC; ++i) {
        const int row = (wave * CC + i) * 16 + (lane >> 2);
        const uint32_t chunk = (lane & 3) ^ (((row >> 2) & 1) | ((row >> 3) & 2));
        c_from[i] = static_cast<uint32_t>(row < rows_here ? row : rows_here - 1) * (K / 2) + chunk * 16;
        c_second[i] = (chunk & 2) * 16;
    }
    const size_t first = static_cast<size_t>(at.expert) * N + nb;
    const char* const x_base = reinterpret_cast<const char*>(x);
    const char* const c_base = reinterpret_cast<const char*>(W.codes) + first * (K / 2);
    const char* const s_base = reinterpret_cast<const char*>(W.scales) + first * (K / kMxGroup);
    const int wrow = wave * 32 + tile_weight_row(c32);
    const int c_off = wrow * 64 + ((half ^ (((wrow >> 2) & 1) | ((wrow >> 3) & 2))) * 16);      // of an even stage; an odd one's place has bit 1 flipped
    const int s_off = CHUNKS ? wrow * 16 + half : wrow * (K / kMxGroup) + half;
    int x_off[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) x_off[q] = (c32 * 8 + ((half * 4 + q) ^ ((c32 >> 1) & 7))) * 16;

    // Stages begin .. end - 1 are this share's: whole pairs, as even as they go.  All shares pass `turns` barriers.
    const int stages = K / 64, pairs = (stages + 1) / 2;
    const int begin = 2 * (share * pairs / KS), last_end = 2 * ((share + 1) * pairs / KS);
    const int end = last_end < stages ? last_end : stages, turns = KS == 1 ? stages : 2 * ((pairs + KS - 1) / KS);
    auto ask_rows = [&](int s, int place) {
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            const char* from = x_base + static_cast<size_t>(s) * 128;
            uint32_t off = x_from[i];
            asm volatile("" : "+s"(from), "+v"(off));           // scalar base and 32-bit offset: no address arithmetic per lane
            __builtin_amdgcn_global_load_lds(DICEMOE_GLOBAL_PTR(from + off), DICEMOE_LDS_PTR(lds + place * S::kRowBytes + (wave * XC + i) * 1024), 16, 0, 0);
        }
    };
    auto ask_codes = [&](int pair) {
#pragma unroll
        for (int i = 0; i < CC; ++i) {
            const char* from = c_base + static_cast<size_t>(pair) * 64;
            uint32_t off = c_from[i];
            if (2 * pair + 1 >= stages) off -= c_second[i];     // a last pair of one stage: the first half twice, the second is never read
            asm volatile("" : "+s"(from), "+v"(off));
            __builtin_amdgcn_global_load_lds(DICEMOE_GLOBAL_PTR(from + off), DICEMOE_LDS_PTR(code_lds + (pair & 1) * S::kCodeBytes + (wave * CC + i) * 1024), 16, 0, 0);
        }
    };
    auto ask_scales = [&](int chunk) {                          // of stages 8 chunk .. + 7, 64 rows a wavefront
        if (wave * 64 < BN) {
            const int row = wave * 64 + lane;
            const char* const from = s_base + static_cast<size_t>(row < rows_here ? row : rows_here - 1) * (K / kMxGroup) + chunk * 16;
            __builtin_amdgcn_global_load_lds(DICEMOE_GLOBAL_PTR(from), DICEMOE_LDS_PTR(scale_lds + (chunk & 1) * BN * 16 + wave * 1024), 16, 0, 0);
        }
    };
    // ahead of the first stage: scales, codes and rows of stage 0, rows of stage 1, codes of stages 2 and 3
    if constexpr (CHUNKS) {
        if (begin < end) ask_scales(begin >> 3);
        if ((begin | 7) + 1 < end) ask_scales((begin >> 3) + 1);
    } else {
        const int there = rows_here * (K / kMxGroup);
        for (int to = wave_all * 1024; to < S::scale_bytes(K); to += KS * S::kThreads * 16) {
            const int mine = to + lane * 16;
            __builtin_amdgcn_global_load_lds(DICEMOE_GLOBAL_PTR(s_base + (mine < there ? mine : 0)), DICEMOE_LDS_PTR(scale_lds + to), 16, 0, 0);
        }
    }
    if (begin < end) {
        ask_codes(begin / 2);
        ask_rows(begin, 0);
        if (begin + 1 < end) ask_rows(begin + 1, 1);
        if (begin + 2 < end) ask_codes(begin / 2 + 1);
    }
    f32x16_v acc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[r][v] = 0.f;
    const bool live = nb + wave * 32 < N;

    u32x4_t codes, rows[2][RT];
    uint32_t byte = 0;
    float scale = 0.f;
    auto read_rows = [&](int set, int place, int q) {
#pragma unroll
        for (int r = 0; r < RT; ++r) rows[set][r] = *reinterpret_cast<const u32x4_t*>(lds + place * S::kRowBytes + x_off[q] + r * 4096);
    };
    auto read_weights = [&](int s, int odd) {
        codes = *reinterpret_cast<const u32x4_t*>(code_lds + ((s >> 1) & 1) * S::kCodeBytes + (c_off ^ (odd * 32)));
        byte = *reinterpret_cast<const uint8_t*>(scale_lds + s_off + (CHUNKS ? ((s >> 3) & 1) * BN * 16 + 2 * (s & 7) : 2 * s));
    };
    if (begin + 2 < end) wait_vmcnt<XC + CC>();                 // (loads return in order: all but the last ones asked for have landed)
    else wait_vmcnt<0>();
    block_barrier();

    auto stage = [&](int s, auto odd_tag, auto live_tag) {
        constexpr int ODD = decltype(odd_tag)::value;
        constexpr bool LIVE = decltype(live_tag)::value;
        const bool more = s + 1 < end;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x4_t a;
            if (LIVE) a = u32x4_t{mx4_bf16<0>(codes[q], scale), mx4_bf16<1>(codes[q], scale), mx4_bf16<2>(codes[q], scale), mx4_bf16<3>(codes[q], scale)};
            __builtin_amdgcn_sched_barrier(0);
            if (q == 3 && s + 1 < begin + turns) {
                wait_lgkmcnt0();                                // this wavefront has read all of stage s, whose place is filled next
                // The rows of stage s + 1 and all that was asked for before them have landed once only the codes asked for behind them
                // are under way: behind odd stages codes follow the rows (there are none behind the last rows)
                if (ODD || s + 2 >= end) wait_vmcnt<0>();
                else wait_vmcnt<CC>();
                block_barrier();
            }
            __builtin_amdgcn_sched_barrier(0);
            if (LIVE) {
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    acc[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_v*>(&a), *reinterpret_cast<const bf16x8_v*>(&rows[q & 1][r]),
                                                                     acc[r], 0, 0, 0);
                    if (r == 0) {                               // what the next slice needs is read behind this one's first product
                        __builtin_amdgcn_sched_barrier(0);
                        if (q < 3) {
                            read_rows((q + 1) & 1, ODD, q + 1);
                        } else if (more) {
                            read_weights(s + 1, 1 - ODD);
                            read_rows(0, 1 - ODD, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (s + 2 < end) {
            if (CHUNKS && ODD && (s & 7) == 7 && s + 9 < end) ask_scales((s >> 3) + 2);
            ask_rows(s + 2, ODD);
            if (ODD && s + 3 < end) ask_codes((s + 3) / 2);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (LIVE) scale = mx4_scale(byte);
    };
    auto run = [&](auto live_tag) {
        if (decltype(live_tag)::value) {
            read_weights(begin, 0);
            read_rows(0, 0, 0);
            scale = mx4_scale(byte);
        }
        int s = begin;
        for (; s < end; s += 2) {
            stage(s, std::integral_constant<int, 0>{}, live_tag);
            if (s + 1 < end) stage(s + 1, std::integral_constant<int, 1>{}, live_tag);
        }
        if (KS > 1)                                             // the barriers of larger shares
            for (s = end + 1; s < begin + turns; ++s) block_barrier();
    };
    if (live && begin < end) run(std::true_type{});
    else run(std::false_type{});                                // columns past N: its loads, waits and barriers only
    if constexpr (KS > 1) {                                     // the first share adds the others' sums in order
        float* const sums = reinterpret_cast<float*>(lds_all);
        wait_lgkmcnt0();
        block_barrier();                                        // all stages have been read
        if (share > 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int v = 0; v < 16; ++v) sums[(((share - 1) * RT + r) * 16 + v) * S::kThreads + wave * 64 + lane] = acc[r][v];
        }
        wait_lgkmcnt0();
        block_barrier();
        if (share > 0) return;
#pragma unroll
        for (int o = 0; o < KS - 1; ++o)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[r][v] += sums[((o * RT + r) * 16 + v) * S::kThreads + wave * 64 + lane];
    }
    if (!live) return;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = at.row0 + r * 32 + c32;
        if (row >= at.row_end) continue;
        bf16_t* const to = out + static_cast<size_t>(out_index ? out_index[row] : row) * N;
        bf16_t* const pre_to = pre ? pre + static_cast<size_t>(row) * N : nullptr;
        {
            const int n = nb + wave * 32 + half * 16;
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = acc[r][i];
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
