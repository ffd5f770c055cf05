// How the gradient of the router cuts its tokens (route_backward.hip), and the partial sums that can take: plain C++.
#pragma once
#include <algorithm>
#include "ffn_plan.hpp"

namespace dicemoe {

constexpr int kRouteChunk = 64;                                             // tokens per workgroup at least, one tile per wavefront
constexpr int route_chunk_most(int E) { return E > 32 ? 128 : 256; }        // (with more than 32 experts their dz has to fit the LDS)
constexpr int kRouteChunksLong = 32;                                        // more chunks than that and their sum takes long

// Tokens per workgroup: 64, and up to 256 (128) while that
// leaves two workgroups per compute unit, which keeps the partial sums a small part of what is read; with more than 32 chunks, whose
// sum takes long, also while it leaves one (8 experts, 4096 tokens of 1152 columns, 64 and 32 chunks: 16.1 + 7.5 and 16.0 + 4.2 us; 16
// experts, 8192 of 1792, 64 and 32: 34.9 + 7.8 and 32.4 + 4.8; 4096 of 2048, 32 and 16: 19.2 + 4.2 and 20.5 + 4.0).
inline int route_chunk(int T_tok, int E, int columns)
{
    int chunk = kRouteChunk;
    while (chunk < route_chunk_most(E)) {
        const int least = (T_tok + chunk - 1) / chunk > kRouteChunksLong ? kComputeUnits : 2 * kComputeUnits;
        if (static_cast<long long>((T_tok + 2 * chunk - 1) / (2 * chunk)) * columns < least) break;
        chunk *= 2;
    }
    return chunk;
}

// Most chunks of any token count up to T_max.  More than 32 chunks of less than the most tokens are there only while chunks twice as long
// would leave less than a workgroup per compute unit, i.e. number at most (kComputeUnits - 1) / columns.
inline long long route_chunks_most(long long T_max, int E, int columns)
{
    const long long most = route_chunk_most(E), finest = (T_max + kRouteChunk - 1) / kRouteChunk;
    const long long few = std::max(kRouteChunksLong, 2 * ((kComputeUnits - 1) / columns));
    return std::max(std::min(finest, few), (T_max + most - 1) / most);
}

}  // namespace dicemoe
