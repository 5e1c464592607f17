// Embedding: gaf_embedding (rows of a table, scaled) and gaf_embedding_grad (the table's gradient by sorted tokens).
//
//     out[t] = scale * table[token[t]]          grad[v] = base[v] + scale * sum over t with token[t] = v of dy[t]
//
// The lookup is a gather: 32,768 rows of 8 KB in 60 us, 8.9 TB/s of rows read and written (frequent tokens' rows come from L2).
// A token outside 0 .. V-1 is padding: its row of `out` is zero and it adds nothing to any gradient.
//
// The gradient is bound by the table: V d elements are written (and read, with a base), while a microbatch touches a few of its
// rows only.  Every row is written once, and no atomic touches a sum.  Two launches:
//   group + fill   One cluster puts the positions of equal tokens next to one another (counts, places, positions; its steps are
//            separated by cluster barriers).  Integer atomics hand out the places, so which position stands where inside a token's
//            stretch differs from run to run; stretches of more than 32 are therefore put in ascending order here (a warp each, a
//            bit per position; in texts of more than 32,768 tokens window by window, its positions put together first: two tokens in 2 M
//            positions 8.2 ms, 73 ms where every window looked through all of them), shorter ones by the warp that adds them.  All other CTAs meanwhile write the rows of tokens that do
//            not occur, of the first half of the table, each after looking through the tokens for those of its own range.  (Grouping first, then one
//            kernel that met every row and looked up its count: 67.6 and 479 us where this takes 36 and 328, at 1000
//            tokens, 50,257 x 768 binary32, and 32,768 tokens, 100,000 x 2048 with a base.)
//   sum + fill   Beside what is left to fill (half of the rows: the sums are bound by latency, the filling by bandwidth), a warp per occurring token
//            and 256 columns adds its positions in ascending order in binary32 registers.  Stretches of
//            more than 32 are cut into pieces of about the square root of their length, which keeps both a piece and the sum of a
//            stretch's pieces a short chain; the warp that finishes a stretch's last piece adds them in order.
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

constexpr int kGroupCtas = 8;                   // of a cluster
constexpr int kGroupThreads = 1024;
constexpr int kLightMost = 32;                  // longest stretch that one warp orders and adds
constexpr int kOrderWords = 1024;               // positions whose bits a warp holds at once, / 32
constexpr int kOrderWindow = kOrderWords * 32;
constexpr int kOrderWindows = 512;              // windows whose counts a warp holds at once, where the text is longer than one
constexpr int kFillRows = 1 << 16;              // rows whose bits a filling CTA holds at once
__host__ __device__ constexpr int order_words(bool one_window) { return one_window ? kOrderWords : kOrderWords + kOrderWindows; }
// (a text within one window leaves the rest to the L1 cache)
__host__ __device__ constexpr int group_smem_bytes(bool one_window) { return kGroupThreads / 32 * order_words(one_window) * 4; }
static_assert(kFillRows / 8 <= group_smem_bytes(true), "the bits of the rows fit where the bits of the positions do");

// A token with a short stretch; a piece of a long one (everything that its sum needs, in one or two loads): its token, first place and
// positions, which long stretch it belongs to, and that one's pieces.
struct alignas(16) Light { int v; unsigned int start; int n, unused; };
struct alignas(16) Piece { int v; unsigned int start; int n, heavy, first_piece, pieces, unused[2]; };

// Words that the grouping cluster clears.
struct GroupCursors { unsigned int lights, positions, pieces, heavies; };      // (the first two as one 64-bit number, too)

struct EmbedGradArgs {
    const void *dy, *tokens, *base;
    void *grad;
    GroupCursors *cur;
    unsigned int *count;        // [V] positions of a token
    unsigned int *start;        // [V] first place of its stretch
    unsigned int *slot;         // [T] place of a position inside its token's stretch
    unsigned int *pos;          // [T] positions, stretch by stretch
    unsigned int *ordered;      // [T] the same in ascending order, for long stretches
    Light *light;
    unsigned int *heavy;        // tokens with long stretches
    Piece *piece;
    unsigned int *ticket;       // [long stretch][tile] pieces that are done
    float *partials;            // [piece][d]
    int64_t dy_stride, V, T, d, tiles;      // tiles: of a row
    float scale;
    int fillers;                // CTAs of three of the summing kernel that fill rows: 1 or 2
};

// Positions per piece of a stretch of n > 32: at least 32, about sqrt(n).
__device__ __forceinline__ int piece_length(unsigned int n) { return max(kLightMost, (int)ceilf(sqrtf((float)n))); }

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned int warp_scan(unsigned int v, int lane) {      // sum of the lanes up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned int below = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += below;
    }
    return v;
}

// f of each of n positions, and of 0xFFFFFFFF, in any order.  (Sixteen loads in flight: one after the other, a text's most frequent token took
// longer than all else here.)
template <typename F>
__device__ __forceinline__ void each_position(const unsigned int *from, unsigned int n, int lane, F &&f) {
    for (unsigned int k0 = lane; k0 < n; k0 += 32 * 16) {
        unsigned int at[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) at[j] = k0 + 32 * j < n ? __ldcg(from + k0 + 32 * j) : 0xFFFFFFFFu;
#pragma unroll
        for (int j = 0; j < 16; ++j) f(at[j]);
    }
}
// n positions, all of the window of 32 * words that starts at p0, in ascending order: a bit per position, read back in order.  `to` may be `from`.
__device__ __forceinline__ void order_window(unsigned int *bits, const unsigned int *from, unsigned int n, unsigned int p0, int words, unsigned int *to,
                                             int lane) {
    for (int w = lane; w < words; w += 32) bits[w] = 0u;
    __syncwarp();
    each_position(from, n, lane, [&](unsigned int p) {
        if (p != 0xFFFFFFFFu) atomicOr(bits + ((p - p0) >> 5), 1u << (p & 31u));
    });
    __syncwarp();
    unsigned int done = 0u;
    for (int w0 = 0; w0 < words; w0 += 32) {
        const unsigned int word = w0 + lane < words ? bits[w0 + lane] : 0u;
        const unsigned int sum = warp_scan((unsigned int)__popc(word), lane);
        unsigned int at = done + sum - (unsigned int)__popc(word);
        const unsigned int base = p0 + (unsigned int)(w0 + lane) * 32u;
        for (unsigned int b = word; b != 0u; b &= b - 1u) to[at++] = base + (unsigned int)(__ffs(b) - 1);
        done += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    __syncwarp();
}

template <typename I>
__device__ __forceinline__ void group_tokens(const EmbedGradArgs &a, unsigned int *smem) {
    constexpr int64_t kThreads = kGroupCtas * kGroupThreads;
    const int64_t tid = (int64_t)blockIdx.x * kGroupThreads + threadIdx.x;
    const int lane = threadIdx.x & 31;
    for (int64_t v = tid; v < a.V; v += kThreads) a.count[v] = 0u;
    if (tid == 0) *a.cur = GroupCursors{0u, 0u, 0u, 0u};
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
    // places; the counts of several rounds together, so that a CTA asks once for all of its tokens (an atomic for each warp and round took most
    // of this kernel's time: 3000 of them on one address)
    constexpr int kRounds = 8;
    __shared__ unsigned long long warp_sum[32];
    __shared__ unsigned long long cta_first;
    for (int64_t v00 = tid - threadIdx.x; v00 < a.V; v00 += kRounds * kThreads) {
        unsigned int counts[kRounds];
        unsigned long long mine = 0ull;                      // positions of this thread's tokens, and how many short stretches
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int64_t v = v00 + r * kThreads + threadIdx.x;
            counts[r] = v < a.V ? __ldcg(a.count + v) : 0u;
        }
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            mine += ((unsigned long long)counts[r] << 32) + (counts[r] != 0u && counts[r] <= (unsigned int)kLightMost ? 1u : 0u);
        unsigned long long sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long below = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += below;
        }
        if (lane == 31) warp_sum[threadIdx.x >> 5] = sum;
        __syncthreads();
        if (threadIdx.x < 32) {
            unsigned long long s = warp_sum[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long below = __shfl_up_sync(0xFFFFFFFFu, s, o);
                if (lane >= o) s += below;
            }
            warp_sum[lane] = s;
            if (lane == 31) cta_first = atomicAdd(reinterpret_cast<unsigned long long *>(a.cur), s);
        }
        __syncthreads();
        const unsigned long long first = cta_first + (threadIdx.x >= 32 ? warp_sum[(threadIdx.x >> 5) - 1] : 0ull) + sum - mine;
        unsigned int at = (unsigned int)(first >> 32), l = (unsigned int)first;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const unsigned int n = counts[r];
            if (n == 0u) continue;
            const int64_t v = v00 + r * kThreads + threadIdx.x;
            a.start[v] = at;
            if (n <= (unsigned int)kLightMost) {
                a.light[l++] = Light{(int)v, at, (int)n, 0};
            } else {
                const int length = piece_length(n), pieces = (int)((n + length - 1) / length);
                const unsigned int h = atomicAdd(&a.cur->heavies, 1u), p = atomicAdd(&a.cur->pieces, (unsigned int)pieces);
                a.heavy[h] = (unsigned int)v;
                for (int k = 0; k < pieces; ++k)
                    a.piece[p + k] = Piece{(int)v, at + (unsigned int)(k * length), min(length, (int)n - k * length), (int)h, (int)p, pieces, {0, 0}};
                for (int64_t k = 0; k < a.tiles; ++k) a.ticket[h * a.tiles + k] = 0u;
            }
            at += n;
        }
        __syncthreads();                                     // (the next round's sums go where these were read)
    }
    cluster_barrier();
    for (int64_t t = tid; t < a.T; t += kThreads) {
        const int64_t v = valid_token(static_cast<const I *>(a.tokens), t, a.V);
        if (v >= 0) a.pos[__ldcg(a.start + v) + a.slot[t]] = (unsigned int)t;
    }
    cluster_barrier();
    // ascending order of the long stretches
    const bool one_window = a.T <= kOrderWindow;
    unsigned int *const bits = smem + (threadIdx.x >> 5) * order_words(one_window), *const count = bits + kOrderWords;
    const unsigned int heavies = __ldcg(&a.cur->heavies);
    for (unsigned int h = (unsigned int)(tid >> 5); h < heavies; h += (unsigned int)(kThreads >> 5)) {
        const unsigned int v = __ldcg(a.heavy + h);
        const unsigned int n = __ldcg(a.count + v), first = __ldcg(a.start + v);
        const unsigned int *const from = a.pos + first;
        unsigned int *to = a.ordered + first;
        if (one_window) {
            order_window(bits, from, n, 0u, (int)((a.T + 31) / 32), to, lane);
            continue;
        }
        // 512 windows at a time: the positions of each are put together, in any order, and then set right within the window
        for (int64_t t0 = 0; t0 < a.T; t0 += (int64_t)kOrderWindow * kOrderWindows) {
            auto window = [&](unsigned int p) {              // of a position, or none of these
                const int64_t w = ((int64_t)p - t0) / kOrderWindow;
                return p != 0xFFFFFFFFu && (int64_t)p >= t0 && w < kOrderWindows ? (int)w : -1;
            };
            for (int w = lane; w < kOrderWindows; w += 32) count[w] = 0u;
            __syncwarp();
            each_position(from, n, lane, [&](unsigned int p) {
                const int w = window(p);
                if (w >= 0) atomicAdd(count + w, 1u);
            });
            __syncwarp();
            unsigned int before = 0u;                        // counts become places
            for (int w0 = 0; w0 < kOrderWindows; w0 += 32) {
                const unsigned int c = count[w0 + lane], sum = warp_scan(c, lane);
                count[w0 + lane] = before + sum - c;
                before += __shfl_sync(0xFFFFFFFFu, sum, 31);
            }
            __syncwarp();
            each_position(from, n, lane, [&](unsigned int p) {
                const int w = window(p);
                if (w >= 0) to[atomicAdd(count + w, 1u)] = p;
            });
            __syncwarp();                                    // (and every place is now the next window's first)
            for (int w0 = 0; w0 < kOrderWindows; w0 += 32) {
                const unsigned int end = count[w0 + lane], begin = w0 + lane == 0 ? 0u : count[w0 + lane - 1];
                for (unsigned int some = __ballot_sync(0xFFFFFFFFu, end != begin); some != 0u; some &= some - 1u) {
                    const int k = __ffs(some) - 1;
                    const unsigned int b = __shfl_sync(0xFFFFFFFFu, begin, k), e = __shfl_sync(0xFFFFFFFFu, end, k);
                    const unsigned int p0 = (unsigned int)(t0 + (int64_t)(w0 + k) * kOrderWindow);
                    order_window(bits, to + b, e - b, p0, (int)min((int64_t)kOrderWords, (a.T - p0 + 31) / 32), to + b, lane);
                }
            }
            to += before;
        }
    }
}

// Rows of tokens that do not occur: base, or zeros.  Neighbouring rows lie next to one another, so that a run of them is one stretch of memory: as
// 16-byte pieces from its first boundary on, whatever the width (base and gradient lie alike), and single elements before and behind.
template <typename G>
__device__ __forceinline__ void fill_run(const EmbedGradArgs &a, int64_t v, int rows, int lane) {
    constexpr int kBatch = 8, kPer = 16 / sizeof(G);
    const int64_t n = rows * a.d;
    G *const out = static_cast<G *>(a.grad) + v * a.d;
    const G *const in = static_cast<const G *>(a.base) + v * a.d;
    const int64_t head = min(n, (int64_t)(((16u - (unsigned int)(reinterpret_cast<uintptr_t>(out) & 15u)) & 15u) / sizeof(G)));
    const int64_t pieces = (n - head) / kPer, tail = head + pieces * kPer;
    if (lane < head) out[lane] = a.base ? in[lane] : from_float<G>(0.f);
    if (tail + lane < n) out[tail + lane] = a.base ? in[tail + lane] : from_float<G>(0.f);
    uint4 *const to = reinterpret_cast<uint4 *>(out + head);
    const uint4 *const from = reinterpret_cast<const uint4 *>(in + head);
    for (int64_t c0 = lane; c0 < pieces; c0 += 32 * kBatch) {
        uint4 x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) x[k] = a.base && c0 + 32 * k < pieces ? from[c0 + 32 * k] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (c0 + 32 * k < pieces) to[c0 + 32 * k] = x[k];
    }
}
// Rows that a warp looks at together: enough of them for some KB.  And the runs among those of them (bits of `absent`) that do not occur.
template <typename G>
__device__ __forceinline__ int fill_group(int64_t d) { return d * (int64_t)sizeof(G) >= 1024 ? 8 : 32; }
template <typename G>
__device__ __forceinline__ void fill_absent(const EmbedGradArgs &a, int64_t v0, unsigned int absent, int lane) {
    while (absent != 0u) {
        const int first = __ffs(absent) - 1, past = __ffs(~(absent >> first)) - 1;      // (-1: ones to the end)
        const int rows = past < 0 ? 32 - first : past;
        fill_run<G>(a, v0 + first, rows, lane);
        absent &= first + rows >= 32 ? 0u : ~0u << (first + rows);
    }
}
// The first half of the rows is filled beside the grouping, the other half beside the sums.  A quarter / half / three quarters, us, L2 cold: 50,257 rows
// of 3 KB, 1000 tokens 41 / 39 / 41, 6000 55 / 52 / 52, 16,384 76 / 72 / 68; 100,000 rows of 8 KB with a base, 4000 tokens 297 / 290 / 293, 11,000 308 / 320 / 341, 32,768
// 328 / 331 / 354.
__host__ __device__ inline int64_t fill_split(int64_t V) { return V / 2; }

// Rows 0 .. fill_split(V) - 1, while the counts are not known yet.  CTA number `cta` of `ctas`.
template <typename I, typename G>
__device__ __forceinline__ void fill_rows(const EmbedGradArgs &a, unsigned int *bits, int64_t cta, int64_t ctas) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t rows = fill_split(a.V), row0 = rows * cta / ctas, row1 = rows * (cta + 1) / ctas;
    for (int64_t from = row0; from < row1; from += kFillRows) {
        const int64_t to = min(row1, from + kFillRows);
        for (int w = threadIdx.x; w < (int)((to - from + 31) / 32); w += kGroupThreads) bits[w] = 0u;
        __syncthreads();
        for (int64_t t = threadIdx.x; t < a.T; t += kGroupThreads) {
            const int64_t v = valid_token(static_cast<const I *>(a.tokens), t, a.V) - from;
            if (v >= 0 && v < to - from) atomicOr(bits + (v >> 5), 1u << (v & 31));
        }
        __syncthreads();
        const int group = fill_group<G>(a.d);
        for (int64_t v = from + warp * group; v < to; v += kGroupThreads / 32 * group) {
            const int rows = (int)min((int64_t)group, to - v);
            fill_absent<G>(a, v, ~(bits[(v - from) >> 5] >> ((v - from) & 31)) & (0xFFFFFFFFu >> (32 - rows)), lane);
        }
        __syncthreads();
    }
}

template <typename I, typename G>
__global__ void __cluster_dims__(kGroupCtas, 1, 1) __launch_bounds__(kGroupThreads, 1) embedding_group_kernel(const EmbedGradArgs a) {
    extern __shared__ unsigned int group_smem[];
    grid_wait();
    grid_release();
    if (blockIdx.x < kGroupCtas) group_tokens<I>(a, group_smem);
    // (where base is the output itself, rows that do not occur are right already)
    else if (a.base != a.grad) fill_rows<I, G>(a, group_smem, blockIdx.x - kGroupCtas, gridDim.x - kGroupCtas);
}

// Adds a tile of rows of dy to acc: of those at the positions that lanes 0 .. n-1 hold, in lane order.
template <typename T, bool VEC>
__device__ __forceinline__ void add_rows(const EmbedGradArgs &a, unsigned int p, int n, int64_t c, int lane, float (&acc)[8]) {
    constexpr int kBatch = 8;                               // rows in flight
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += kBatch) {
        Share<T> s[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int64_t t = __shfl_sync(0xFFFFFFFFu, p, (k0 + b) & 31);
            if (k0 + b < n) load_tile<VEC>(static_cast<const T *>(a.dy) + t * a.dy_stride + c, lane, a.d - c, s[b]);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (k0 + b >= n) break;
            float x[8];
            s[b].get(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += x[i];
        }
    }
}

// scale * sum + base, rounded once.
template <typename G, bool VEC>
__device__ __forceinline__ void write_row_tile(const EmbedGradArgs &a, int64_t v, int64_t c, int lane, const Share<G> &base, float (&x)[8]) {
    if (a.base) {
        float b[8];
        base.get(b);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], a.scale, b[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= a.scale;
    }
    store_tile<VEC>(static_cast<G *>(a.grad) + v * a.d + c, lane, a.d - c, x);
}

// Units of work, a tile of columns each: the pieces of long stretches, then the tokens with short ones.  What leads to a short stretch's rows is
// fetched ahead, its entry two units and its positions one, so that a unit waits for its rows only.
template <typename T, typename G, bool VEC>
__global__ void __launch_bounds__(kEmbedWarps * 32, 2) embedding_sum_kernel(const EmbedGradArgs a) {
    const int lane = threadIdx.x & 31;
    grid_wait();
    grid_release();
    // of every three CTAs the last one or two fill rows
    const int role = blockIdx.x % 3, summing = 3 - a.fillers;
    if (role >= summing) {
        if (a.base == a.grad) return;
        const int group = fill_group<G>(a.d);
        const int64_t stride = (int64_t)(gridDim.x / 3) * a.fillers * kEmbedWarps * group;
        // (the next counts are fetched before these rows are written)
        auto counts = [&](int64_t v0) { return lane < group && v0 + lane < a.V ? a.count[v0 + lane] : 1u; };
        int64_t v0 = fill_split(a.V) + ((int64_t)((blockIdx.x / 3) * a.fillers + role - summing) * kEmbedWarps + (threadIdx.x >> 5)) * group;
        unsigned int n = counts(v0);
        for (; v0 < a.V; v0 += stride) {
            const unsigned int absent = __ballot_sync(0xFFFFFFFFu, n == 0u);
            n = counts(v0 + stride);
            fill_absent<G>(a, v0, absent, lane);
        }
        return;
    }
    const unsigned int tiles = (unsigned int)a.tiles, warps = gridDim.x / 3 * summing * kEmbedWarps,
                       me = (blockIdx.x / 3 * summing + role) * kEmbedWarps + (threadIdx.x >> 5);
    const unsigned int pieces = a.cur->pieces * tiles, lights = a.cur->lights * tiles;
#pragma unroll 1
    for (unsigned int u = me; u < pieces; u += warps) {
        const unsigned int p = u / tiles, tile = u - p * tiles;
        const int64_t c = (int64_t)tile * kTile;
        const Piece piece = a.piece[p];
        const unsigned int *const at = a.ordered + piece.start;
        float acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll 1
        for (int k0 = 0; k0 < piece.n; k0 += 32)
            add_rows<T, VEC>(a, k0 + lane < piece.n ? at[k0 + lane] : 0u, min(32, piece.n - k0), c, lane, acc);
        store_tile<VEC>(a.partials + p * a.d + c, lane, a.d - c, acc);
        // the stretch's last piece to be done: all of them, in order
        __syncwarp();
        unsigned int before = 0u;
        if (lane == 0)
            asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.ticket + (size_t)piece.heavy * tiles + tile) : "memory");
        before = __shfl_sync(0xFFFFFFFFu, before, 0);
        if (before != (unsigned int)piece.pieces - 1u) continue;
        Share<G> base;
        if (a.base) load_tile<VEC>(static_cast<const G *>(a.base) + piece.v * a.d + c, lane, a.d - c, base);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.f;
        const float *const part = a.partials + (int64_t)piece.first_piece * a.d + c;
        constexpr int kBatch = 4;
#pragma unroll 1
        for (int k0 = 0; k0 < piece.pieces; k0 += kBatch) {
            float s[kBatch][8];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                // (written by other SMs during this launch: from L2)
                const float *const q = part + (int64_t)(k0 + b) * a.d;
                if (k0 + b >= piece.pieces) break;
                if (VEC) {
                    if (lane * 8 < a.d - c) {
                        const float4 f = __ldcg(reinterpret_cast<const float4 *>(q + lane * 8)), g = __ldcg(reinterpret_cast<const float4 *>(q + lane * 8) + 1);
                        s[b][0] = f.x; s[b][1] = f.y; s[b][2] = f.z; s[b][3] = f.w;
                        s[b][4] = g.x; s[b][5] = g.y; s[b][6] = g.z; s[b][7] = g.w;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[b][i] = i * 32 + lane < a.d - c ? __ldcg(q + i * 32 + lane) : 0.f;
                }
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (k0 + b >= piece.pieces) break;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += s[b][i];
            }
        }
        write_row_tile<G, VEC>(a, piece.v, c, lane, base, acc);
    }

    // (the warps that had no piece, or one less, begin here with the first ones)
    const unsigned int first = (me + warps - pieces % warps) % warps;
    auto entry = [&](unsigned int u) { return u < lights ? a.light[u / tiles] : Light{0, 0u, 0, 0}; };
    auto positions = [&](const Light &x) { return lane < x.n ? a.pos[x.start + lane] : 0xFFFFFFFFu; };
    Light x = entry(first), next = entry(first + warps);
    unsigned int p = positions(x);
#pragma unroll 1
    for (unsigned int u = first; u < lights; u += warps) {
        const int64_t c = (int64_t)(u % tiles) * kTile;
        Share<G> base;
        if (a.base) load_tile<VEC>(static_cast<const G *>(a.base) + x.v * a.d + c, lane, a.d - c, base);
        const unsigned int p_next = positions(next);
        const Light after = entry(u + 2 * warps);
        float acc[8];
        if (x.n <= 2) {                                      // most tokens of a text
            const unsigned int p0 = __shfl_sync(0xFFFFFFFFu, p, 0), p1 = __shfl_sync(0xFFFFFFFFu, p, 1);
            Share<T> s0, s1;
            load_tile<VEC>(static_cast<const T *>(a.dy) + (int64_t)min(p0, p1) * a.dy_stride + c, lane, a.d - c, s0);
            if (x.n == 2) {
                load_tile<VEC>(static_cast<const T *>(a.dy) + (int64_t)max(p0, p1) * a.dy_stride + c, lane, a.d - c, s1);
                float y[8];
                s0.get(acc);
                s1.get(y);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] += y[i];
            } else {
                s0.get(acc);
            }
        } else {
            int rank = 0;                                    // of this lane's position
            unsigned int sorted = p;
#pragma unroll 1
            for (int j = 0; j < x.n; ++j) rank += __shfl_sync(0xFFFFFFFFu, p, j) < p;
#pragma unroll 1
            for (int j = 0; j < x.n; ++j) {
                const int r = __shfl_sync(0xFFFFFFFFu, rank, j);
                const unsigned int q = __shfl_sync(0xFFFFFFFFu, p, j);
                if (r == lane) sorted = q;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = 0.f;
            add_rows<T, VEC>(a, sorted, x.n, c, lane, acc);
        }
        write_row_tile<G, VEC>(a, x.v, c, lane, base, acc);
        x = next;
        next = after;
        p = p_next;
    }
}

}  // namespace gaf
