// Row tiles of a ragged batch: the flat list (sequence, tile) that a grid walks, found by every work-group for itself.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace respec {

// Inclusive sums over the lanes of a wave.
__device__ inline int wave_scan_add(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
    return x;
}

struct Tile {
    int32_t b, index;  // sequence, tile within it
    int32_t tiles;     // of the sequence
    int32_t R;         // rows of the sequence
    int64_t q0;        // its first row
};

// Tile `tile` of the list of all sequences' tiles of `per_tile` packed rows (G of them per row); false past its end.  Every wave
// that calls it finds the same; 64 sequences are looked at at a time.
__device__ inline bool find_tile(const int32_t *q_indptr, int B, int total_q, int max_q, int G, int per_tile, int tile, Tile &out) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < B; base += 64) {
        int q0 = 0, R = 0;
        if (base + lane < B) {
            q0 = max(0, min(q_indptr[base + lane], total_q));
            R = max(0, min(min(q_indptr[base + lane + 1], total_q) - q0, max_q));
        }
        const int n = (int)(((int64_t)R * G + per_tile - 1) / per_tile);
        const int sum = wave_scan_add(n);
        const int total = __builtin_amdgcn_readlane(sum, 63);
        if (tile < total) {
            const int at = (int)__builtin_ctzll(__ballot(sum > tile));
            out.b = base + at;
            out.tiles = __builtin_amdgcn_readlane(n, at);
            out.index = tile - (__builtin_amdgcn_readlane(sum, at) - out.tiles);
            out.R = __builtin_amdgcn_readlane(R, at);
            out.q0 = __builtin_amdgcn_readlane(q0, at);
            return true;
        }
        tile -= total;
    }
    return false;
}

// As many tiles as any batch with these sizes can have.
inline int64_t tiles_bound(int32_t B, int32_t total_q, int32_t max_q, int32_t G, int32_t per_tile) {
    const int64_t by_rows = ((int64_t)total_q * G + (int64_t)B * (per_tile - 1)) / per_tile;
    const int64_t by_seqs = (int64_t)B * (((int64_t)max_q * G + per_tile - 1) / per_tile);
    return std::max<int64_t>(1, std::min(by_rows, by_seqs));
}

// Whether a grid of `blocks` work-groups can be launched: its threads are counted in 32 bits.
inline bool grid_fits(int64_t blocks, int threads) { return blocks <= 0xffffffffLL / threads; }

}  // namespace respec
