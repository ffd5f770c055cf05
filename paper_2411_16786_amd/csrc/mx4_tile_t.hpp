// Transposed grouped product of many rows on 4-bit weights (bf16 rows), for the gradient: out[r, k] = sum_n y[r, n] W_e[n, k], times
// gelu'(u[r, k]) with SLOPE; tiled through LDS like mx4_tile_kernel.
//
// The reduction runs over rows of weights, so the operand that a matrix instruction wants, eight consecutive n of one column k, lies in
// eight rows of codes.  The transposing LDS read (ds_read_b64_tr_b8) hands a lane the bytes of eight rows for one byte column, i.e. two
// columns k; each byte is converted with its own row's scale (two columns of one n), and byte permutations put the pairs along n
// together: one conversion and one permutation per two weights, 16 of each for the 2 RT matrix instructions of a slice of 16 n.
// Scales lie in the LDS as floats, [32-column group][n], written there by the threads (they have to be transposed as well), so that a
// slice's come with two broadcast reads.
// A workgroup of WN wavefronts owns BK = 64 WN columns of BR = 32 RT rows, a wavefront 64 columns: of its two blocks, block i has the
// columns 2 c + i.  Stages of 64 n, two in the LDS, barrier ahead of the last slice as there.
// By counters over 8192 rows and 8 experts, 64 x 256 tiles, 4608 -> 1152 and 1152 -> 4608 with the slope: matrix pipes busy 37 and 32 % of the
// cycles, a wavefront waits 42 and 41 % of its time for a stage or at a barrier, 31 and 33 % to issue (the conversions and permutations beside
// the matrix instructions).  Medians: 104 and 119 us (0.83 and 0.73 PFLOP/s) on one set of rows and two of weights, 114 and 134 (0.76 and 0.65)
// over three sets of everything, which do not fit the memory-side cache.
#pragma once
#include "mx4_tile.hpp"

namespace dicemoe {

template <int RT, int WN, int KS> struct TileShapeT {
    static constexpr int BK = 64 * WN, BR = 32 * RT, kThreads = 64 * WN;            // (of one share)
    static constexpr int kRowBytes = BR * 128, kCodePitch = BK / 2, kCodeBytes = 64 * kCodePitch;
    static constexpr int kScalePitch = 80, kScaleBytes = 2 * WN * kScalePitch * 4;        // (64 floats and 16 more: two groups and two halves on banks of their own)
    static constexpr int kRowLoads = kRowBytes / 16 / kThreads, kCodeLoads = kCodeBytes / 16 / kThreads;
    static_assert(WN == 2 || WN == 4, "the swizzles below");
    static_assert(kRowBytes % (16 * kThreads) == 0 && kCodeBytes % (16 * kThreads) == 0, "whole loads");
    static constexpr int kShareBytes = 2 * (kRowBytes + kCodeBytes + kScaleBytes), kSumBytes = (KS - 1) * 2 * RT * 64 * kThreads;
    static constexpr int kLds = KS * kShareBytes > kSumBytes ? KS * kShareBytes : kSumBytes;
    // 16-byte chunk c of row n of the codes lies at place c ^ swizzle(n): transposing reads of 16 rows then spread over all banks
    __device__ static constexpr int swizzle(int n) { return WN == 4 ? (n >> 1) & 7 : (n >> 2) & 3; }
};

template <int RT, int WN, int KS, bool SLOPE>
__global__ __launch_bounds__(64 * WN * KS, 2) void mx4_tile_transposed_kernel(const bf16_t* __restrict__ y, Segments seg, int N, int K, Mx4 W,
                                                                      const bf16_t* __restrict__ u, bf16_t* __restrict__ out,
                                                                      int32_t* __restrict__ status)
{
    typedef TileShapeT<RT, WN, KS> S;
    typedef int i32x2_t __attribute__((ext_vector_type(2)));
    constexpr int BR = S::BR, XC = S::kRowLoads, CC = S::kCodeLoads, PLACES = S::kCodePitch / 16;
    extern __shared__ __attribute__((aligned(16))) char lds_all[];
    report_row_overflow(status, seg.offsets, seg.n, seg.max_rows);
    const int k_blocks = (K + S::BK - 1) / S::BK;
    TilePlace at;
    if (!find_tile_on_xcd(seg, BR, k_blocks, blockIdx.x, at)) return;
    const int lane = lane_id(), wave_all = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const int wave = wave_all % WN, share = wave_all / WN;      // of the share
    const int half = lane >> 5, c32 = lane & 31;
    const int kb = at.block * S::BK;
    char* const lds = lds_all + share * S::kShareBytes;
    char* const code_lds = lds + 2 * S::kRowBytes;
    char* const scale_lds = code_lds + 2 * S::kCodeBytes;

    uint32_t x_from[XC], c_from[CC];
#pragma unroll
    for (int i = 0; i < XC; ++i) {
        const int row = (wave * XC + i) * 8 + (lane >> 3);
        const int r = at.row0 + row < at.row_end ? at.row0 + row : at.row_end - 1;       // rows past the end repeat the last; never stored
        x_from[i] = static_cast<uint32_t>(r) * (2u * N) + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
#pragma unroll
    for (int i = 0; i < CC; ++i) {
        const int n = (wave * CC + i) * (64 / PLACES) + lane / PLACES;
        const int chunk = (lane % PLACES) ^ S::swizzle(n);
        c_from[i] = static_cast<uint32_t>(n) * (K / 2) + (kb + chunk * 32 < K ? chunk * 16 : 0);      // columns past K repeat the first; never stored
    }
    const size_t first = static_cast<size_t>(at.expert) * N;
    const char* const y_base = reinterpret_cast<const char*>(y);
    const char* const c_base = reinterpret_cast<const char*>(W.codes) + first * (K / 2) + kb / 2;
    // scales: thread (n, pair) stages two groups of row n
    const int sn = (wave * kWave + lane) / WN, spair = (wave * kWave + lane) % WN;
    const uint8_t* const s_base = W.scales + (first + sn) * (K / kMxGroup) + kb / kMxGroup + (kb + 64 * spair < K ? 2 * spair : 0);
    float* const s_to = reinterpret_cast<float*>(scale_lds) + 2 * spair * S::kScalePitch + sn;

    const int c_off = (half * 8 + ((lane & 15) >> 1)) * S::kCodePitch + (((wave * 2 + (c32 >> 4)) ^ S::swizzle(half * 8 + ((lane & 15) >> 1))) * 16) + (lane & 1) * 8;
    const int s_off = ((wave * 2 + (c32 >> 4)) * S::kScalePitch + half * 8) * 4;
    int x_off[4];                                               // slice q: n = 16 q + 8 half .. + 7
#pragma unroll
    for (int q = 0; q < 4; ++q) x_off[q] = (c32 * 8 + ((q * 2 + half) ^ ((c32 >> 1) & 7))) * 16;

    // Stages begin .. end - 1 are this share's: whole pairs, as even as they go.  All shares pass `turns` barriers.
    const int stages = N / 64, pairs = (stages + 1) / 2;
    const int begin = 2 * (share * pairs / KS), last_end = 2 * ((share + 1) * pairs / KS);
    const int end = last_end < stages ? last_end : stages, turns = KS == 1 ? stages : 2 * ((pairs + KS - 1) / KS);
    auto ask = [&](int s, int place) {
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            const char* from = y_base + static_cast<size_t>(s) * 128;
            uint32_t off = x_from[i];
            asm volatile("" : "+s"(from), "+v"(off));           // scalar base and 32-bit offset: no address arithmetic per lane
            __builtin_amdgcn_global_load_lds(DICEMOE_GLOBAL_PTR(from + off), DICEMOE_LDS_PTR(lds + place * S::kRowBytes + (wave * XC + i) * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < CC; ++i) {
            const char* from = c_base + static_cast<size_t>(s) * 64 * (K / 2);
            uint32_t off = c_from[i];
            asm volatile("" : "+s"(from), "+v"(off));
            __builtin_amdgcn_global_load_lds(DICEMOE_GLOBAL_PTR(from + off), DICEMOE_LDS_PTR(code_lds + place * S::kCodeBytes + (wave * CC + i) * 1024), 16, 0, 0);
        }
    };
    auto ask_scales = [&](int s) { return static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(s_base + static_cast<size_t>(s) * 64 * (K / kMxGroup))); };
    auto keep_scales = [&](uint32_t two, int place) {
        s_to[place * (S::kScaleBytes / 4)] = mx4_scale(two & 0xFFu);
        s_to[place * (S::kScaleBytes / 4) + S::kScalePitch] = mx4_scale(two >> 8);
    };
    uint32_t two[2];                                            // scales on their way, by the parity of their stage
    uint32_t two0 = 0u;
    two[0] = two[1] = 0u;
    if (begin < end) {
        two0 = ask_scales(begin);
        if (begin + 1 < end) two[1] = ask_scales(begin + 1);
        if (begin + 2 < end) two[0] = ask_scales(begin + 2);
        ask(begin, 0);
        if (begin + 1 < end) ask(begin + 1, 1);
        keep_scales(two0, 0);
    }
    f32x16_v acc[2][RT];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][r][v] = 0.f;
    const bool live = kb + wave * 64 < K;

    u32x4_t rows[2][RT];
    i32x2_t codes[4];                                           // of all slices of a stage
    f32x4_t scale[2];
    auto read_rows = [&](int set, int place, int q) {
#pragma unroll
        for (int r = 0; r < RT; ++r) rows[set][r] = *reinterpret_cast<const u32x4_t*>(lds + place * S::kRowBytes + x_off[q] + r * 4096);
    };
    // All slices at once, behind the barrier and ahead of the next loads: the compiler waits for every load to the LDS before such a read
    auto read_codes = [&](int place) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            codes[q] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (__attribute__((address_space(3))) i32x2_t*)(code_lds + place * S::kCodeBytes + c_off + q * 16 * S::kCodePitch));
    };
    auto read_scales = [&](int place, int q) {
        const f32x4_t* const from = reinterpret_cast<const f32x4_t*>(scale_lds + place * S::kScaleBytes + s_off + q * 64);
        scale[0] = from[0];
        scale[1] = from[1];
    };
    if (begin + 1 < end) wait_vmcnt<XC + CC>();                 // (loads return in order: all but stage 1's have landed)
    else wait_vmcnt<0>();
    wait_lgkmcnt0();
    block_barrier();

    auto stage = [&](int s, auto odd_tag, auto live_tag) {
        constexpr int ODD = decltype(odd_tag)::value;
        constexpr bool LIVE = decltype(live_tag)::value;
        const bool more = s + 1 < end;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x4_t a[2];
            if (LIVE) {
                const uint32_t lo = codes[q][0], hi = codes[q][1];
                const uint32_t p[8] = {mx4_bf16<0>(lo, scale[0][0]), mx4_bf16<1>(lo, scale[0][1]), mx4_bf16<2>(lo, scale[0][2]), mx4_bf16<3>(lo, scale[0][3]),
                                       mx4_bf16<0>(hi, scale[1][0]), mx4_bf16<1>(hi, scale[1][1]), mx4_bf16<2>(hi, scale[1][2]), mx4_bf16<3>(hi, scale[1][3])};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    a[0][j] = __builtin_amdgcn_perm(p[2 * j + 1], p[2 * j], 0x05040100u);
                    a[1][j] = __builtin_amdgcn_perm(p[2 * j + 1], p[2 * j], 0x07060302u);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (q == 2 && more) keep_scales(two[1 - ODD], 1 - ODD);      // of stage s + 1, asked for two stages ago
            if (q == 3 && s + 1 < begin + turns) {
                wait_lgkmcnt0();                                // this wavefront has read all of stage s, whose place is filled next
                wait_vmcnt<0>();                                // its loads of stage s + 1, asked for a stage ago, have landed
                block_barrier();
            }
            __builtin_amdgcn_sched_barrier(0);
            if (LIVE) {
#pragma unroll
                for (int i = 0; i < 2 * RT; ++i) {
                    const int b = i / RT, r = i % RT;
                    acc[b][r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_v*>(&a[b]), *reinterpret_cast<const bf16x8_v*>(&rows[q & 1][r]),
                                                                        acc[b][r], 0, 0, 0);
                    if (i == 0) {                               // what the next slice needs is read behind this one's first product
                        __builtin_amdgcn_sched_barrier(0);
                        if (q < 3) {
                            read_scales(ODD, q + 1);
                            read_rows((q + 1) & 1, ODD, q + 1);
                        } else if (more) {
                            read_codes(1 - ODD);
                            read_scales(1 - ODD, 0);
                            read_rows(0, 1 - ODD, 0);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (s + 3 < end) two[1 - ODD] = ask_scales(s + 3);
        if (s + 2 < end) ask(s + 2, ODD);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto run = [&](auto live_tag) {
        if (decltype(live_tag)::value) {
            read_codes(0);
            read_scales(0, 0);
            read_rows(0, 0, 0);
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
    else run(std::false_type{});                                // columns past K: its loads, waits and barriers only
    if constexpr (KS > 1) {                                     // the first share adds the others' sums in order
        float* const sums = reinterpret_cast<float*>(lds_all);
        wait_lgkmcnt0();
        block_barrier();                                        // all stages have been read
        if (share > 0) {
#pragma unroll
            for (int i = 0; i < 2 * RT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) sums[(((share - 1) * 2 * RT + i) * 16 + v) * S::kThreads + wave * kWave + lane] = acc[i / RT][i % RT][v];
        }
        wait_lgkmcnt0();
        block_barrier();
        if (share > 0) return;
#pragma unroll
        for (int o = 0; o < KS - 1; ++o)
#pragma unroll
            for (int i = 0; i < 2 * RT; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i / RT][i % RT][v] += sums[((o * 2 * RT + i) * 16 + v) * S::kThreads + wave * kWave + lane];
    }
    if (!live) return;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = at.row0 + r * 32 + c32;
        if (row >= at.row_end) continue;
#pragma unroll
        for (int a = 0; a < 4; ++a) {                           // registers 4 a + b: columns 16 a + 8 half + 2 b + block
            const size_t to = static_cast<size_t>(row) * K + kb + wave * 64 + 16 * a + 8 * half;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = acc[i & 1][r][4 * a + (i >> 1)];
            if (SLOPE) {
                float uf[8];
                Store<bf16_t>::unpack(*reinterpret_cast<const u32x4_t*>(u + to), uf);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= gelu_slope<bf16_t>(uf[i]);
            }
            store8(out + to, v);
        }
    }
}

}  // namespace dicemoe
