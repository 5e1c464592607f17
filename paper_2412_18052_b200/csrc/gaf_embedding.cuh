// Embedding: gaf_embedding (rows of a table, scaled) and gaf_embedding_grad (the table's gradient by sorted tokens).
//
//     out[t] = scale * table[token[t]]          grad[v] = base[v] + scale * sum over t with token[t] = v of dy[t]
//
// A token outside 0 .. V-1 is padding: its row of `out` is zero and it adds nothing to any gradient.
//
// The gradient is bound by the table: V d elements are written (and read, with a base), while a microbatch touches a few of its
// rows only.  Every row is written once, by whoever adds it up, so that nothing is cleared first and no atomic touches a sum:
//   group    positions of equal tokens next to one another: counts, places, positions (one launch of one cluster; the steps
//            are separated by cluster barriers).  Integer atomics hand out the places, so which position stands where inside a
//            token's stretch differs from run to run;
//   order    therefore each stretch is put in ascending order before it is added up: up to 32 positions by the warp that adds
//            them, longer ones (a few tokens make up much of a text) by one CTA each through a bitmap of the positions;
//   sum      a warp per row and 1024 columns adds its positions in ascending order in binary32 registers, or writes zeros (or
//            base).  Stretches of more than 32 positions are cut into pieces of about the square root of their length, which
//            keeps both the pieces and the sums of a stretch's pieces short chains;
//   join     adds the pieces of such tokens in order.
#pragma once

#include "gaf_layer_device.cuh"

namespace gaf {

constexpr int kEmbedWarps = 8;
constexpr int kEmbedTiles = 4;                  // tiles per warp: 1024 columns
constexpr int kEmbedColumns = kEmbedTiles * kTile;

template <typename I>
__device__ __forceinline__ int64_t valid_token(const I *tokens, int64_t t, int64_t V) {
    const int64_t v = (int64_t)tokens[t];
    return v >= 0 && v < V ? v : -1;
}

struct EmbedArgs {
    const void *table, *tokens;
    void *out;
    int64_t table_stride, V, T, d, parts;       // parts: 1024-column stretches of a row
    float scale;
};

template <typename T, typename I, bool VEC>
__global__ void __launch_bounds__(kEmbedWarps * 32) embedding_kernel(const EmbedArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * kEmbedWarps + (threadIdx.x >> 5);
    grid_wait();
    if (unit >= a.T * a.parts) return;
    const int64_t t = unit / a.parts, c0 = (unit - t * a.parts) * kEmbedColumns;
    const int64_t v = valid_token(static_cast<const I *>(a.tokens), t, a.V);
    Share<T> s[kEmbedTiles];
#pragma unroll
    for (int k = 0; k < kEmbedTiles; ++k)
        load_tile<VEC>(static_cast<const T *>(a.table) + (v < 0 ? 0 : v) * a.table_stride + c0 + k * kTile, lane,
                       v < 0 ? 0 : a.d - c0 - k * kTile, s[k]);
#pragma unroll
    for (int k = 0; k < kEmbedTiles; ++k) {
        float x[8];
        s[k].get(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v < 0 ? 0.f : x[i] * a.scale;
        store_tile<VEC>(static_cast<T *>(a.out) + t * a.d + c0 + k * kTile, lane, a.d - c0 - k * kTile, x);
    }
}

// ---------------------------------------------------------------- gradient --

constexpr int kGroupCtas = 8;                   // one cluster
constexpr int kGroupThreads = 1024;
constexpr int kLightMost = 32;                  // longest stretch that one warp takes
constexpr int kOrderThreads = 1024;
constexpr int kOrderWords = 8192;               // positions whose bits a CTA holds at once, / 32

struct Heavy { int v, first_piece, pieces, length; };      // length: positions per piece
struct Piece { int heavy, index; };

// Words that the grouping kernel clears.
struct GroupCursors { unsigned int positions, pieces, heavies, reserved; };

struct EmbedGradArgs {
    const void *dy, *tokens, *base;
    void *grad;
    Control *ctl;
    GroupCursors *cur;
    unsigned int *count;        // [V] positions of a token
    unsigned int *start;        // [V] first place of its stretch
    unsigned int *slot;         // [T] place of a position inside its token's stretch
    unsigned int *pos;          // [T] positions, stretch by stretch
    unsigned int *ordered;      // [T] the same in ascending order, for long stretches
    Heavy *heavy;
    Piece *piece;
    float *partials;            // [piece][d]
    int64_t dy_stride, V, T, d, parts;
    float scale;
    int piece_ctas;             // CTAs of the summing kernel that take pieces
};

// Positions per piece of a stretch of n > 32: at least 32, about sqrt(n).
__device__ __forceinline__ int piece_length(unsigned int n) { return max(kLightMost, (int)ceilf(sqrtf((float)n))); }

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename I>
__global__ void __cluster_dims__(kGroupCtas, 1, 1) __launch_bounds__(kGroupThreads) embedding_group_kernel(const EmbedGradArgs a) {
    constexpr int64_t kThreads = kGroupCtas * kGroupThreads;
    const int64_t tid = (int64_t)blockIdx.x * kGroupThreads + threadIdx.x;
    const int lane = threadIdx.x & 31;
    grid_wait();
    grid_release();
    for (int64_t v = tid; v < a.V; v += kThreads) a.count[v] = 0u;
    if (tid == 0) {
        *a.cur = GroupCursors{0u, 0u, 0u, 0u};
        a.ctl->status = 0;
    }
    cluster_barrier();
    // counts; lanes with the same token take their places together
    for (int64_t t0 = tid - lane; t0 < a.T; t0 += kThreads) {
        const int64_t t = t0 + lane;
        const int v = t < a.T ? (int)valid_token(static_cast<const I *>(a.tokens), t, a.V) : -1;
        const unsigned int same = __match_any_sync(0xFFFFFFFFu, v);
        const int leader = __ffs(same) - 1;
        unsigned int first = 0u;
        if (v >= 0 && lane == leader) first = atomicAdd(a.count + v, (unsigned int)__popc(same));
        first = __shfl_sync(0xFFFFFFFFu, first, leader);
        if (v >= 0) a.slot[t] = first + (unsigned int)__popc(same & ((1u << lane) - 1u));
    }
    cluster_barrier();
    // places
    for (int64_t v0 = tid - lane; v0 < a.V; v0 += kThreads) {
        const int64_t v = v0 + lane;
        const unsigned int n = v < a.V ? __ldcg(a.count + v) : 0u;
        if (__ballot_sync(0xFFFFFFFFu, n != 0u) == 0u) continue;
        unsigned int sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned int below = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += below;
        }
        unsigned int first = 0u;
        if (lane == 31) first = atomicAdd(&a.cur->positions, sum);
        first = __shfl_sync(0xFFFFFFFFu, first, 31);
        if (n != 0u) a.start[v] = first + sum - n;
        if (n > (unsigned int)kLightMost) {
            const int length = piece_length(n), pieces = (int)((n + length - 1) / length);
            const unsigned int h = atomicAdd(&a.cur->heavies, 1u), p = atomicAdd(&a.cur->pieces, (unsigned int)pieces);
            a.heavy[h] = Heavy{(int)v, (int)p, pieces, length};
            for (int k = 0; k < pieces; ++k) a.piece[p + k] = Piece{(int)h, k};
        }
    }
    cluster_barrier();
    for (int64_t t = tid; t < a.T; t += kThreads) {
        const int64_t v = valid_token(static_cast<const I *>(a.tokens), t, a.V);
        if (v >= 0) a.pos[__ldcg(a.start + v) + a.slot[t]] = (unsigned int)t;
    }
}

// Ascending order of the positions of tokens with more than 32: a bit per position, read back in order.
__global__ void __launch_bounds__(kOrderThreads) embedding_order_kernel(const EmbedGradArgs a) {
    __shared__ unsigned int bits[kOrderWords];
    __shared__ unsigned int warp_total[32];
    constexpr int kWords = kOrderWords / kOrderThreads;     // consecutive words of a thread
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_wait();
    grid_release();
    const unsigned int heavies = a.cur->heavies;
    for (unsigned int h = blockIdx.x; h < heavies; h += gridDim.x) {
        const int v = a.heavy[h].v;
        const unsigned int n = a.count[v], first = a.start[v];
        unsigned int done = 0u;
        for (int64_t t0 = 0; t0 < a.T; t0 += (int64_t)kOrderWords * 32) {
            for (int w = threadIdx.x; w < kOrderWords; w += kOrderThreads) bits[w] = 0u;
            __syncthreads();
            for (unsigned int k = threadIdx.x; k < n; k += kOrderThreads) {
                const int64_t p = (int64_t)a.pos[first + k] - t0;
                if (p >= 0 && p < (int64_t)kOrderWords * 32) atomicOr(bits + (p >> 5), 1u << (p & 31));
            }
            __syncthreads();
            unsigned int word[kWords], mine = 0u;
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                word[k] = bits[threadIdx.x * kWords + k];
                mine += (unsigned int)__popc(word[k]);
            }
            unsigned int sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned int below = __shfl_up_sync(0xFFFFFFFFu, sum, o);
                if (lane >= o) sum += below;
            }
            if (lane == 31) warp_total[warp] = sum;
            __syncthreads();
            unsigned int at = first + done + sum - mine, total = 0u;
            for (int w = 0; w < kOrderThreads / 32; ++w) {
                const unsigned int c = warp_total[w];
                if (w < warp) at += c;
                total += c;
            }
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                const unsigned int base = (unsigned int)(t0 + (int64_t)(threadIdx.x * kWords + k) * 32);
                for (unsigned int b = word[k]; b != 0u; b &= b - 1u) a.ordered[at++] = base + (unsigned int)(__ffs(b) - 1);
            }
            done += total;
            __syncthreads();
        }
    }
}

// Adds rows of dy to acc: those at the positions that lanes 0 .. n-1 hold, in lane order.
template <typename T, bool VEC>
__device__ __forceinline__ void add_rows(const EmbedGradArgs &a, unsigned int p, int n, int64_t c0, int lane, float (&acc)[kEmbedTiles][8]) {
    constexpr int kBatch = sizeof(T) == 4 ? 2 : 4;          // rows in flight
    for (int k0 = 0; k0 < n; k0 += kBatch) {
        Share<T> s[kBatch][kEmbedTiles];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int64_t t = __shfl_sync(0xFFFFFFFFu, p, (k0 + b) & 31);
            if (k0 + b < n) {
#pragma unroll
                for (int k = 0; k < kEmbedTiles; ++k)
                    load_tile<VEC>(static_cast<const T *>(a.dy) + t * a.dy_stride + c0 + k * kTile, lane, a.d - c0 - k * kTile, s[b][k]);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (k0 + b >= n) break;
#pragma unroll
            for (int k = 0; k < kEmbedTiles; ++k) {
                float x[8];
                s[b][k].get(x);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[k][i] += x[i];
            }
        }
    }
}

// scale * sum + base, rounded once.
template <typename G, bool VEC>
__device__ __forceinline__ void write_row_tile(const EmbedGradArgs &a, int64_t v, int64_t c, int lane, float (&x)[8]) {
    const int64_t left = a.d - c;
    if (a.base) {
        float b[8];
        load_tile<VEC>(static_cast<const G *>(a.base) + v * a.d + c, lane, left, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], a.scale, b[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= a.scale;
    }
    store_tile<VEC>(static_cast<G *>(a.grad) + v * a.d + c, lane, left, x);
}

template <typename T, typename G, bool VEC>
__global__ void __launch_bounds__(kEmbedWarps * 32) embedding_sum_kernel(const EmbedGradArgs a) {
    const int lane = threadIdx.x & 31;
    float acc[kEmbedTiles][8];
    grid_wait();
    grid_release();
    if ((int)blockIdx.x < a.piece_ctas) {
        // pieces of long stretches
        const int64_t units = (int64_t)a.cur->pieces * a.parts;
        for (int64_t u = (int64_t)blockIdx.x * kEmbedWarps + (threadIdx.x >> 5); u < units; u += (int64_t)a.piece_ctas * kEmbedWarps) {
            const int64_t p = u / a.parts, c0 = (u - p * a.parts) * kEmbedColumns;
            const Piece piece = a.piece[p];
            const Heavy hv = a.heavy[piece.heavy];
            const unsigned int n_all = a.count[hv.v], from = (unsigned int)piece.index * (unsigned int)hv.length;
            const int n = (int)min((unsigned int)hv.length, n_all - from);
            const unsigned int *const at = a.ordered + a.start[hv.v] + from;
#pragma unroll
            for (int k = 0; k < kEmbedTiles; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
            for (int k0 = 0; k0 < n; k0 += 32)
                add_rows<T, VEC>(a, k0 + lane < n ? at[k0 + lane] : 0u, min(32, n - k0), c0, lane, acc);
#pragma unroll
            for (int k = 0; k < kEmbedTiles; ++k)
                store_tile<VEC>(a.partials + p * a.d + c0 + k * kTile, lane, a.d - c0 - k * kTile, acc[k]);
        }
        return;
    }
    const int64_t unit = (int64_t)(blockIdx.x - a.piece_ctas) * kEmbedWarps + (threadIdx.x >> 5);
    if (unit >= a.V * a.parts) return;
    const int64_t v = unit / a.parts, c0 = (unit - v * a.parts) * kEmbedColumns;
    const unsigned int n = a.count[v];
    if (n > (unsigned int)kLightMost) return;               // the join writes this row
#pragma unroll
    for (int k = 0; k < kEmbedTiles; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
    if (n != 0u) {
        const unsigned int p = lane < (int)n ? a.pos[a.start[v] + lane] : 0xFFFFFFFFu;
        unsigned int sorted = p;
        if (n > 1u) {
            int rank = 0;                                    // of this lane's position
            for (int j = 0; j < (int)n; ++j) rank += __shfl_sync(0xFFFFFFFFu, p, j) < p;
            for (int j = 0; j < (int)n; ++j) {
                const int r = __shfl_sync(0xFFFFFFFFu, rank, j);
                const unsigned int q = __shfl_sync(0xFFFFFFFFu, p, j);
                if (r == lane) sorted = q;
            }
        }
        add_rows<T, VEC>(a, sorted, (int)n, c0, lane, acc);
    }
#pragma unroll
    for (int k = 0; k < kEmbedTiles; ++k) write_row_tile<G, VEC>(a, v, c0 + k * kTile, lane, acc[k]);
}

// Rows of tokens with more than 32 positions: their pieces in order.  A warp per row and 256 columns.
template <typename G, bool VEC>
__global__ void __launch_bounds__(kEmbedWarps * 32) embedding_join_kernel(const EmbedGradArgs a) {
    const int lane = threadIdx.x & 31;
    grid_wait();
    const int64_t tiles = (a.d + kTile - 1) / kTile, units = (int64_t)a.cur->heavies * tiles;
    for (int64_t u = (int64_t)blockIdx.x * kEmbedWarps + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * kEmbedWarps) {
        const int64_t h = u / tiles, c = (u - h * tiles) * kTile;
        const Heavy hv = a.heavy[h];
        float acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.f;
        const float *const p = a.partials + (int64_t)hv.first_piece * a.d + c;
        constexpr int kBatch = 4;
        for (int k0 = 0; k0 < hv.pieces; k0 += kBatch) {
            Share<float> s[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
                if (k0 + b < hv.pieces) load_tile<VEC>(p + (int64_t)(k0 + b) * a.d, lane, a.d - c, s[b]);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (k0 + b >= hv.pieces) break;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += s[b].v[i];
            }
        }
        write_row_tile<G, VEC>(a, hv.v, c, lane, acc);
    }
}

}  // namespace gaf
