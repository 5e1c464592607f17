// 8-bit checkpoints of activations: gaf_checkpoint_pack and gaf_checkpoint_unpack (the code is described in
// gaf_layer_device.cuh).
//
// Bound by memory: 2 or 4 bytes read and 1 + 1/128 written per element, or the reverse.  A warp takes a tile of 256 columns at
// a time (16-byte loads, 8-byte stores of codes); the block's maximum is four shuffles.
#pragma once

#include "gaf_layer_device.cuh"

namespace gaf {

constexpr int kCheckpointWarps = 4;
// Tiles in flight per warp.  (Element by element, each access has a predicate and an address: 1111 columns 71 us with 2, 103 us with 4.)
__host__ __device__ constexpr int checkpoint_tiles(bool vec) { return vec ? 4 : 2; }

struct CheckpointArgs {
    const void *x;              // pack: the matrix; unpack: written instead (as `out`)
    void *out;
    unsigned char *codes, *scales;
    int64_t x_stride, codes_stride;
    int64_t d, blocks;
    unsigned int tiles_per_row, n_tiles;
};

template <typename T, bool VEC, bool PACK>
__global__ void __launch_bounds__(kCheckpointWarps * 32) checkpoint_kernel(const CheckpointArgs a) {
    constexpr int kCheckpointTiles = checkpoint_tiles(VEC);
    const int lane = threadIdx.x & 31;
    const unsigned int first = (blockIdx.x * kCheckpointWarps + (threadIdx.x >> 5)) * kCheckpointTiles;
    grid_wait();
    if (first >= a.n_tiles) return;
    // (in 32 bits: a 64-bit division was a fifth of the kernel's instructions)
    unsigned int row = first / a.tiles_per_row, tile = first - row * a.tiles_per_row;
    int64_t rows[kCheckpointTiles], cols[kCheckpointTiles];
#pragma unroll
    for (int k = 0; k < kCheckpointTiles; ++k) {
        rows[k] = row;
        cols[k] = (int64_t)tile * kTile;
        if (++tile == a.tiles_per_row) { tile = 0; ++row; }
    }
    if constexpr (PACK) {
        Share<T> s[kCheckpointTiles];
#pragma unroll
        for (int k = 0; k < kCheckpointTiles; ++k)
            if (first + k < a.n_tiles)
                load_tile<VEC>(static_cast<const T *>(a.x) + rows[k] * a.x_stride + cols[k], lane, a.d - cols[k], s[k]);
#pragma unroll
        for (int k = 0; k < kCheckpointTiles; ++k) {
            if (first + k >= a.n_tiles) break;
            float v[8];
            unsigned int c[2];
            int e[2];
            encode_share<VEC>(s[k], v, c, e);
            store_codes<VEC>(a.codes + rows[k] * a.codes_stride + cols[k], a.scales + rows[k] * a.blocks + cols[k] / kCodeBlock, lane,
                             a.d - cols[k], c, e);
        }
    } else {
        CodeShare s[kCheckpointTiles];
#pragma unroll
        for (int k = 0; k < kCheckpointTiles; ++k)
            if (first + k < a.n_tiles)
                load_codes<VEC>(a.codes + rows[k] * a.codes_stride + cols[k], a.scales + rows[k] * a.blocks + cols[k] / kCodeBlock, lane,
                                a.d - cols[k], s[k]);
#pragma unroll
        for (int k = 0; k < kCheckpointTiles; ++k) {
            if (first + k >= a.n_tiles) break;
            float v[8];
            s[k].get(v);
            store_tile<VEC>(static_cast<T *>(a.out) + rows[k] * a.x_stride + cols[k], lane, a.d - cols[k], v);
        }
    }
}

}  // namespace gaf
