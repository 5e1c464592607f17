// Host side of the layers' entry points of include/gaf.h (embedding, root-mean-square norm, 8-bit checkpoints, weight gradient):
// argument checks, workspace layout and launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <type_traits>

#include "../../include/gaf.h"
#include "gaf_checkpoint.cuh"
#include "gaf_embedding.cuh"
#include "gaf_host.h"
#include "gaf_launch.h"
#include "gaf_rmsnorm.cuh"
#include "gaf_weight_grad.cuh"

namespace {

using namespace gaf;

constexpr int64_t kMaxRows = INT32_MAX - 64;            // tokens, rows of a table, columns (positions and tensor-copy coordinates are 32 bits)

bool is_dtype(int t) { return t == GAF_F32 || t == GAF_BF16; }
bool in_range(int64_t n) { return n >= 0 && n <= kMaxRows; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t blocks_of(int64_t d) { return ceil_div(d, kCodeBlock); }

// Bytes from p on that a matrix of `rows` rows takes, and whether two such stretches overlap.
struct Span {
    uintptr_t from, to;
    Span(const void *p, int64_t rows, int64_t cols, int64_t stride, size_t elem)
        : from(reinterpret_cast<uintptr_t>(p)),
          to(!p || rows <= 0 || cols <= 0 ? from : from + (size_t(rows - 1) * size_t(stride) + size_t(cols)) * elem) {}
    bool meets(const Span &o) const { return from < o.to && o.from < to; }
    bool same(const Span &o) const { return from == o.from && to == o.to; }
};

// A matrix argument: present (where there are elements) and with rows that do not run into one another.
int check_matrix(const void *p, int64_t rows, int64_t cols, int64_t stride) {
    if (rows == 0 || cols == 0) return GAF_OK;
    if (!p || stride < cols || stride > (int64_t(1) << 40)) return GAF_ERR_ARG;
    return aligned16(p) ? GAF_OK : GAF_ERR_ALIGN;
}
// Codes and scales of a matrix: both or neither; rows of codes start on 16-byte boundaries.
int check_codes(const void *codes, const void *scales, int64_t rows, int64_t cols, int64_t stride) {
    if (int rc = check_matrix(codes, rows, cols, stride)) return rc;
    if (rows == 0 || cols == 0) return GAF_OK;
    if (!scales) return GAF_ERR_ARG;
    return aligned16(scales) && (rows == 1 || stride % 16 == 0) ? GAF_OK : GAF_ERR_ALIGN;
}
// Token numbers: aligned to their own size.
int check_tokens(const void *tokens, int token_type, int64_t T) {
    if (T == 0) return GAF_OK;
    if (!tokens) return GAF_ERR_ARG;
    return reinterpret_cast<uintptr_t>(tokens) % (token_type == GAF_I64 ? 8 : 4) == 0 ? GAF_OK : GAF_ERR_ALIGN;
}
#define GAF_TRY(expr) do { if (int rc_ = (expr)) return rc_; } while (0)

// The layers' kernels move 16 bytes at a time where every row of every matrix starts on a 16-byte boundary and is a multiple of 8
// elements long, and single elements otherwise.
bool wide_rows(int64_t d, int64_t rows, std::initializer_list<int64_t> strides) {
    if (d % 8 != 0) return false;
    if (rows > 1)
        for (int64_t s : strides)
            if (s % 8 != 0) return false;
    return true;
}

int launched(cudaError_t err, int launches) {
    set_last_launch_count(launches);
    if (err != cudaSuccess) { cudaGetLastError(); return GAF_ERR_CUDA; }
    return GAF_OK;
}

template <typename T> struct Tag { typedef T type; };
template <typename F> int by_type(int dtype, F &&f) { return dtype == GAF_F32 ? f(Tag<float>()) : f(Tag<__nv_bfloat16>()); }
template <bool B> struct Flag { static constexpr bool value = B; };
template <typename F> int by_flag(bool b, F &&f) { return b ? f(Flag<true>()) : f(Flag<false>()); }
template <int N> struct Count { static constexpr int value = N; };

// Threads per row and tiles per warp of the norm's kernels, by the width: as few threads as hold the row in registers.  The backward pass has
// three times as much to hold and takes twice the threads.  As many threads / twice as many, us, L2 cold: forward, coded, bfloat16 16384 x 4096 96 / 98,
// 8192 x 8192 98 / 115; backward from a matrix, bfloat16 106 / 100 and 106 / 98, binary32 8192 x 4096 100 / 102 and 4096 x 8192
// 98 / 111; from codes, bfloat16 119 / 96 and 108 / 104, binary32 102 / 88 and 102 / 88.  (Beyond 8192 columns 512 threads with four tiles each
// spill 320 to 512 bytes a thread.)
template <bool BACKWARD, typename F>
int by_width(int64_t d, F &&f) {
    if (d <= 256) return f(Count<32>(), Count<1>());
    if (d <= 512) return f(Count<32>(), Count<2>());
    if (d <= 768) return f(Count<32>(), Count<3>());
    if (d <= 1024) return f(Count<32>(), Count<4>());
    if (d <= 2048) return f(Count<128>(), Count<2>());
    if constexpr (BACKWARD) {
        if (d <= 4096) return f(Count<256>(), Count<2>());
        if (d <= 8192) return f(Count<512>(), Count<2>());
    } else {
        if (d <= 4096) return f(Count<128>(), Count<4>());
        if (d <= 8192) return f(Count<256>(), Count<4>());
    }
    return f(Count<512>(), Count<4>());
}

// ---------------------------------------------------------------- workspace --

constexpr int kNormMaxCtas = 592;                       // rows of partial sums for the norm weight's gradient
constexpr int64_t kWgMaxSplitItems = 148;               // most work items (pairs of CTAs) of a weight gradient whose tokens are split

struct EmbedLayout { size_t cursors, count, start, slot, pos, ordered, light, heavy, piece, ticket, partials, end; };
EmbedLayout embed_layout(int64_t T, int64_t d, int64_t V) {
    EmbedLayout l{};
    size_t at = kLayerScratchOffset;
    auto take = [&](size_t &field, size_t bytes) { field = at; at = round_up(at + bytes, 256); };
    // a long stretch has at least 33 positions; its pieces are 32 long or more, and a last one
    const size_t heavies = size_t(T) / (kLightMost + 1), pieces = size_t(T) / kLightMost + heavies;
    take(l.cursors, sizeof(GroupCursors));
    take(l.count, size_t(V) * 4);
    take(l.start, size_t(V) * 4);
    take(l.slot, size_t(T) * 4);
    take(l.pos, size_t(T) * 4);
    take(l.ordered, size_t(T) * 4);
    take(l.light, size_t(std::min(T, V)) * sizeof(Light));
    take(l.heavy, heavies * 4);
    take(l.piece, pieces * sizeof(Piece));
    take(l.ticket, heavies * size_t(ceil_div(d, kTile)) * 4);
    take(l.partials, pieces * size_t(d) * 4);
    l.end = at;
    return l;
}
size_t norm_grad_bytes(int64_t d) { return kLayerScratchOffset + round_up(size_t(kNormMaxCtas) * size_t(d) * 4, 256); }

// How a weight gradient is dealt to `pairs` of CTAs.  Whole tiles as long as they make full rounds; the tiles of a last round that would leave
// half of the pairs or more without work have their tokens split into as many parts as there are pairs for
// (16384 x 4096 x 4096 is 256 tiles on 74 pairs: 3 rounds of whole tiles and 34 tiles in halves).
struct WgPlan { int64_t steps_per_term, steps, tiles_m, tiles_n, whole, rest, splits, steps_per_split; };
WgPlan weight_grad_plan(int64_t T, int64_t N, int64_t M, int dtype, int64_t pairs) {
    WgPlan p{};
    p.steps_per_term = ceil_div(T, kWgK);
    p.steps = p.steps_per_term * (dtype == GAF_F32 ? 3 : 1);
    p.tiles_m = ceil_div(M, kWgPairM);
    p.tiles_n = ceil_div(N, kWgN);
    const int64_t tiles = p.tiles_m * p.tiles_n;
    p.rest = tiles % pairs;
    p.splits = p.rest > 0 ? std::min(pairs / p.rest, p.steps) : 1;
    if (p.splits > 1) {
        p.steps_per_split = ceil_div(p.steps, p.splits);
        p.splits = ceil_div(p.steps, p.steps_per_split);
    }
    if (p.splits <= 1) {
        p.splits = 1;
        p.rest = 0;
    }
    p.whole = tiles - p.rest;
    return p;
}
struct WgLayout { size_t partials, terms, end; };
// `relaid`: matrices that dy is laid out anew as.
WgLayout weight_grad_layout(const WgPlan &p, int64_t N, int relaid) {
    WgLayout l{};
    l.partials = kLayerScratchOffset;
    l.terms = l.partials + size_t(p.rest * p.splits) * kWgPairM * kWgN * 4;
    l.end = l.terms + round_up(size_t(relaid) * size_t(p.steps_per_term) * kWgK * round_up(size_t(N), 8) * 2, 256);
    return l;
}

template <typename T> T *in_workspace(void *ws, size_t offset) { return reinterpret_cast<T *>(static_cast<unsigned char *>(ws) + offset); }

// ----------------------------------------------------------------- launches --

int launch_embedding(const EmbedArgs &a, int dtype, int token_type, bool vec, cudaStream_t st) {
    const int64_t ctas = ceil_div(a.T * a.parts, kEmbedWarps);
    if (ctas > INT32_MAX) return GAF_ERR_TOO_LARGE;
    return by_type(dtype, [&](auto t) { return by_flag(token_type == GAF_I64, [&](auto i64) { return by_flag(vec, [&](auto v) {
        typedef typename decltype(t)::type T;
        typedef typename std::conditional<decltype(i64)::value, int64_t, int32_t>::type I;
        return launched(launch_dependent(embedding_kernel<T, I, decltype(v)::value>, int(ctas), kEmbedWarps * 32, st, a), 1);
    }); }); });
}

int launch_embedding_grad(const EmbedGradArgs &a, int dtype, int grad_dtype, int token_type, bool vec, const DeviceInfo &di, cudaStream_t st) {
    return by_flag(token_type == GAF_I64, [&](auto i64) { return by_type(grad_dtype, [&](auto g) { return by_flag(vec, [&](auto v) {
        typedef typename std::conditional<decltype(i64)::value, int64_t, int32_t>::type I;
        typedef typename decltype(g)::type G;
        constexpr bool kVec = decltype(v)::value;
        auto group = embedding_group_kernel<I, typename decltype(g)::type>;
        auto sum_f32 = embedding_sum_kernel<float, G, kVec>;
        auto sum_bf16 = embedding_sum_kernel<__nv_bfloat16, G, kVec>;
        // as many clusters, and as many CTAs that sum, as the device holds at once
        struct Plan { int group = 0, f32 = 0, bf16 = 0; };
        static PerDevice<Plan> table;
        GAF_TRY(plan_once(table.plan[di.dev], table.ready[di.dev], [&](Plan &pl) {
            if (cudaFuncSetAttribute(group, cudaFuncAttributeMaxDynamicSharedMemorySize, group_smem_bytes(false)) != cudaSuccess) return int(GAF_ERR_CUDA);
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(kGroupCtas); cfg.blockDim = dim3(kGroupThreads); cfg.dynamicSmemBytes = group_smem_bytes(false);
            int clusters = 0, f32 = 0, bf16 = 0;
            if (cudaOccupancyMaxActiveClusters(&clusters, group, &cfg) != cudaSuccess || clusters < 1 ||
                cudaOccupancyMaxActiveBlocksPerMultiprocessor(&f32, sum_f32, kEmbedWarps * 32, 0) != cudaSuccess || f32 < 1 ||
                cudaOccupancyMaxActiveBlocksPerMultiprocessor(&bf16, sum_bf16, kEmbedWarps * 32, 0) != cudaSuccess || bf16 < 1)
                return int(GAF_ERR_CUDA);
            pl.group = std::max(2, clusters) * kGroupCtas; pl.f32 = f32 * di.sms; pl.bf16 = bf16 * di.sms;
            return int(GAF_OK);
        }));
        const Plan &pl = table.plan[di.dev];
        cudaError_t err = launch_dependent_smem(group, a.base == a.grad ? kGroupCtas : pl.group, kGroupThreads,
                                                size_t(group_smem_bytes(a.T <= kOrderWindow)), st, a);
        if (err != cudaSuccess) return launched(err, 1);
        const int64_t need = ceil_div(3 * std::max(a.T * a.tiles, a.V / 8), kEmbedWarps);
        auto grid = [&](int resident) { return int(std::min<int64_t>(resident, need) / 3 * 3 + 3); };
        err = dtype == GAF_F32 ? launch_dependent(sum_f32, grid(pl.f32 - 3), kEmbedWarps * 32, st, a)
                               : launch_dependent(sum_bf16, grid(pl.bf16 - 3), kEmbedWarps * 32, st, a);
        return launched(err, 2);
    }); }); });
}

int launch_rms_norm(const NormArgs &a, int dtype, bool vec, cudaStream_t st) {
    return by_type(dtype, [&](auto t) { return by_flag(vec, [&](auto v) { return by_width<false>(a.d, [&](auto r, auto s) {
        constexpr int R = decltype(r)::value;
        const int64_t ctas = ceil_div(a.T, norm_threads(R) / R);
        return launched(launch_dependent(rms_norm_kernel<typename decltype(t)::type, decltype(v)::value, R, decltype(s)::value>, int(ctas),
                                         norm_threads(R), st, a), 1);
    }); }); });
}

int launch_rms_norm_grad(const NormGradArgs &a, NormFinishArgs f, int dtype, int grad_dtype, bool vec, const DeviceInfo &di, cudaStream_t st) {
    return by_type(dtype, [&](auto t) { return by_flag(vec, [&](auto v) { return by_flag(a.h_codes != nullptr, [&](auto coded) {
        return by_width<true>(a.d, [&](auto r, auto s) {
            constexpr int R = decltype(r)::value;
            auto kernel = rms_norm_grad_kernel<typename decltype(t)::type, decltype(v)::value, decltype(coded)::value, R, decltype(s)::value>;
            // as many CTAs as the device holds at once, so that each sums as many rows as possible
            struct Plan { int ctas = 0; };
            static PerDevice<Plan> table;
            GAF_TRY(plan_once(table.plan[di.dev], table.ready[di.dev], [&](Plan &pl) {
                int per_sm = 0;
                if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, norm_threads(R), 0) != cudaSuccess || per_sm < 1)
                    return int(GAF_ERR_CUDA);
                pl.ctas = std::min(per_sm * di.sms, kNormMaxCtas);
                return int(GAF_OK);
            }));
            int64_t ctas = std::min<int64_t>(table.plan[di.dev].ctas, ceil_div(a.T, norm_threads(R) / R));
            if (ctas < 1) ctas = 1;
            f.n = int(ctas);
            cudaError_t err = launch_dependent(kernel, int(ctas), norm_threads(R), st, a);
            int launches = 1;
            if (err == cudaSuccess) {
                const int grid = int(ceil_div(a.d, 32));
                err = grad_dtype == GAF_F32 ? launch_dependent(norm_grad_finish_kernel<float>, grid, 32 * kNormFinishGroups, st, f)
                                            : launch_dependent(norm_grad_finish_kernel<__nv_bfloat16>, grid, 32 * kNormFinishGroups, st, f);
                ++launches;
            }
            return launched(err, launches);
        });
    }); }); });
}

template <bool PACK>
int launch_checkpoint(const CheckpointArgs &a, int dtype, bool vec, cudaStream_t st) {
    const int64_t ctas = ceil_div(a.n_tiles, int64_t(kCheckpointWarps) * checkpoint_tiles(vec));
    return by_type(dtype, [&](auto t) { return by_flag(vec, [&](auto v) {
        return launched(launch_dependent(checkpoint_kernel<typename decltype(t)::type, decltype(v)::value, PACK>, int(ctas), kCheckpointWarps * 32,
                                         st, a), 1);
    }); });
}

// A matrix of rows for tensor copies of boxes of `box_rows` rows; false if the driver refuses it.
bool matrix_map(CUtensorMap *map, const void *p, CUtensorMapDataType type, int64_t cols, int64_t rows, int64_t pitch_bytes, int box_cols,
                int box_rows, CUtensorMapSwizzle swizzle) {
    const TensorMapEncodeFn encode = tensor_map_encoder();
    if (!encode) return false;
    const cuuint64_t dims[2] = {cuuint64_t(cols), cuuint64_t(rows)}, strides[1] = {cuuint64_t(pitch_bytes)};
    const cuuint32_t box[2] = {cuuint32_t(box_cols), cuuint32_t(box_rows)}, one[2] = {1u, 1u};
    return encode(map, type, 2, const_cast<void *>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename G>
int launch_weight_grad_tiles(const WeightGradArgs &w, const CUtensorMap &dy_map, const CUtensorMap &code_map, const DeviceInfo &di, cudaStream_t st,
                             int *launches) {
    static PerDevice<DynSmemPlan> table;
    GAF_TRY(plan_once(table.plan[di.dev], table.ready[di.dev], [&](DynSmemPlan &pl) {
        pl.dyn = kWgSmem;
        return cudaFuncSetAttribute(weight_grad_kernel<G>, cudaFuncAttributeMaxDynamicSharedMemorySize, pl.dyn) == cudaSuccess ? int(GAF_OK)
                                                                                                                          : int(GAF_ERR_CUDA);
    }));
    const int grid = 2 * std::min(w.items, int(std::min<int64_t>(di.sms / 2, kWgMaxSplitItems)));
    const cudaError_t err = launch_dependent_smem(weight_grad_kernel<G>, grid, kWgThreads, size_t(kWgSmem), st, w, dy_map, code_map);
    ++*launches;
    return launched(err, *launches);
}

}  // namespace

extern "C" {

int gaf_layer_workspace_bytes(int64_t T, int64_t width, int64_t V, int dtype, size_t *bytes_out) {
    if (!bytes_out || !in_range(T) || !in_range(width) || !in_range(V) || !is_dtype(dtype)) return GAF_ERR_ARG;
    // a weight gradient of at most width x width: the partial sums of split tokens are never more than this many tiles
    const int64_t terms = dtype == GAF_F32 ? 3 : 1, side = std::min(kWgMaxSplitItems, ceil_div(width, kWgN)),
                  tiles = std::min(kWgMaxSplitItems, side * side * std::min(kWgMaxSplitItems, ceil_div(T, kWgK) * terms));
    size_t wg = kLayerScratchOffset + size_t(tiles) * kWgPairM * kWgN * 4 + 256;
    const size_t rows = size_t(terms) * round_up(size_t(T), kWgK), pitch = round_up(size_t(width), 8) * 2;
    if (pitch > 0 && rows > (SIZE_MAX / 2) / pitch) return GAF_ERR_TOO_LARGE;
    wg += rows * pitch;
    const size_t a = embed_layout(T, width, V).end, b = norm_grad_bytes(width);
    *bytes_out = round_up(std::max(wg, std::max(a, b)), 256);
    return GAF_OK;
}

int gaf_embedding(const void *table, int64_t table_stride, int64_t V, int64_t d, int dtype, const void *tokens, int token_type, int64_t T,
                  double scale, void *out, void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(V) || !in_range(d) || !in_range(T) || !is_dtype(dtype) || (token_type != GAF_I32 && token_type != GAF_I64)) return GAF_ERR_ARG;
    GAF_TRY(check_matrix(table, V, d, table_stride));
    GAF_TRY(check_tokens(tokens, token_type, T));
    GAF_TRY(check_matrix(out, T, d, d));
    if (T == 0 || d == 0) return GAF_OK;
    const size_t e = elem_bytes(dtype);
    const Span o(out, T, d, d, e);
    if (o.meets(Span(table, V, d, table_stride, e)) || o.meets(Span(tokens, T, 1, 1, token_type == GAF_I64 ? 8 : 4))) return GAF_ERR_ALIAS;
    EmbedArgs a{};
    a.table = table; a.tokens = tokens; a.out = out; a.table_stride = table_stride; a.V = V; a.T = T; a.d = d;
    a.parts = ceil_div(d, kEmbedColumns);
    a.scale = float(scale);
    return launch_embedding(a, dtype, token_type, wide_rows(d, V, {table_stride}), static_cast<cudaStream_t>(cuda_stream));
}

int gaf_embedding_grad(const void *dy, int64_t dy_stride, int64_t T, int64_t d, int dtype, const void *tokens, int token_type, double scale,
                       const void *base, void *grad, int grad_dtype, int64_t V, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(V) || !in_range(d) || !in_range(T) || !is_dtype(dtype) || !is_dtype(grad_dtype) ||
        (token_type != GAF_I32 && token_type != GAF_I64)) return GAF_ERR_ARG;
    GAF_TRY(check_matrix(dy, T, d, dy_stride));
    GAF_TRY(check_tokens(tokens, token_type, T));
    GAF_TRY(check_matrix(grad, V, d, d));
    if (!aligned16(base)) return GAF_ERR_ALIGN;
    if (V == 0 || d == 0) return GAF_OK;
    const Span g(grad, V, d, d, elem_bytes(grad_dtype)), b(base, V, d, d, elem_bytes(grad_dtype));
    if (g.meets(Span(dy, T, d, dy_stride, elem_bytes(dtype))) || g.meets(Span(tokens, T, 1, 1, token_type == GAF_I64 ? 8 : 4)) ||
        (base && !g.same(b) && g.meets(b))) return GAF_ERR_ALIAS;
    // (units of work are counted in 32 bits)
    if (T > INT32_MAX / 4 / ceil_div(d, kTile)) return GAF_ERR_TOO_LARGE;
    const EmbedLayout l = embed_layout(T, d, V);
    GAF_TRY(check_workspace(workspace, workspace_bytes, l.end));
    DeviceInfo di;
    if (!device_info(&di)) return GAF_ERR_CUDA;
    EmbedGradArgs a{};
    a.dy = dy; a.tokens = tokens; a.base = base; a.grad = grad;
    a.cur = in_workspace<GroupCursors>(workspace, l.cursors);
    a.count = in_workspace<unsigned int>(workspace, l.count);
    a.start = in_workspace<unsigned int>(workspace, l.start);
    a.slot = in_workspace<unsigned int>(workspace, l.slot);
    a.pos = in_workspace<unsigned int>(workspace, l.pos);
    a.ordered = in_workspace<unsigned int>(workspace, l.ordered);
    a.light = in_workspace<Light>(workspace, l.light);
    a.heavy = in_workspace<unsigned int>(workspace, l.heavy);
    a.piece = in_workspace<Piece>(workspace, l.piece);
    a.ticket = in_workspace<unsigned int>(workspace, l.ticket);
    a.partials = in_workspace<float>(workspace, l.partials);
    a.dy_stride = dy_stride; a.V = V; a.T = T; a.d = d;
    a.tiles = ceil_div(d, kTile);
    a.scale = float(scale);
    // few tokens for the table: filling is most of the work, and two CTAs of three do it.  One / two, us, L2 cold: 50,257 rows of 3 KB, 1000 tokens
    // 47 / 39, 3000 48 / 44, 6000 50 / 53, 9000 57 / 65, 16,384 72 / 82; 100,000 rows of 8 KB with a base, 4000 tokens 324 / 291, 11,000 322 / 318,
    // 14,000 312 / 337, 32,768 331 / 452
    a.fillers = T < V / 8 ? 2 : 1;
    return launch_embedding_grad(a, dtype, grad_dtype, token_type, wide_rows(d, T, {dy_stride}), di, static_cast<cudaStream_t>(cuda_stream));
}

int gaf_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight, int64_t T, int64_t d, int dtype,
                 double eps, void *h, void *y, uint8_t *y_codes, int64_t y_codes_stride, uint8_t *y_scales, int coded_y, uint8_t *h_codes,
                 int64_t h_codes_stride, uint8_t *h_scales, float *rstd, void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(T) || d < 1 || !is_dtype(dtype) || !(eps >= 0.0) || std::isinf(eps)) return GAF_ERR_ARG;
    if (d > kNormMaxWidth) return GAF_ERR_TOO_LARGE;
    if (T > 0 && ((h && !residual) || (!y_codes != !y_scales) || (!h_codes != !h_scales) || (coded_y && (!y_codes || !y)) ||
                  (!h && !y && !y_codes && !h_codes && !rstd) || ((y || y_codes) && !weight))) return GAF_ERR_ARG;
    GAF_TRY(check_matrix(x, T, d, x_stride));
    if (residual) GAF_TRY(check_matrix(residual, T, d, residual_stride));
    if (y_codes) GAF_TRY(check_codes(y_codes, y_scales, T, d, y_codes_stride));
    if (h_codes) GAF_TRY(check_codes(h_codes, h_scales, T, d, h_codes_stride));
    if (!aligned16(weight) || !aligned16(h) || !aligned16(y) || !aligned16(rstd)) return GAF_ERR_ALIGN;
    if (T == 0) return GAF_OK;
    const size_t e = elem_bytes(dtype);
    const Span in[3] = {Span(x, T, d, x_stride, e), Span(residual, T, d, residual_stride, e), Span(weight, 1, d, d, e)};
    const Span out[7] = {Span(h, T, d, d, e), Span(y, T, d, d, e), Span(y_codes, T, d, y_codes_stride, 1), Span(y_scales, T, blocks_of(d), blocks_of(d), 1),
                         Span(h_codes, T, d, h_codes_stride, 1), Span(h_scales, T, blocks_of(d), blocks_of(d), 1), Span(rstd, T, 1, 1, 4)};
    for (int i = 0; i < 7; ++i) {
        for (int k = 0; k < 3; ++k)      // (h in the place of x or of the residual: every element is read by the thread that writes it)
            if (out[i].meets(in[k]) && !(i == 0 && k < 2 && out[0].same(in[k]))) return GAF_ERR_ALIAS;
        for (int k = 0; k < i; ++k)
            if (out[i].meets(out[k])) return GAF_ERR_ALIAS;
    }
    NormArgs a{};
    a.x = x; a.residual = residual; a.weight = weight; a.h = h; a.y = y;
    a.y_codes = y_codes; a.y_scales = y_scales; a.h_codes = h_codes; a.h_scales = h_scales; a.rstd = rstd;
    a.x_stride = x_stride; a.residual_stride = residual_stride; a.y_codes_stride = y_codes_stride; a.h_codes_stride = h_codes_stride;
    a.T = T; a.d = d; a.blocks = blocks_of(d); a.eps = float(eps); a.coded_y = coded_y != 0;
    return launch_rms_norm(a, dtype, wide_rows(d, T, {x_stride, residual ? residual_stride : 0}), static_cast<cudaStream_t>(cuda_stream));
}

int gaf_rms_norm_grad(const void *dy, int64_t dy_stride, const void *h, int64_t h_stride, const uint8_t *h_codes, int64_t h_codes_stride,
                      const uint8_t *h_scales, const void *weight, const float *rstd, const void *residual_grad, int64_t residual_grad_stride,
                      int64_t T, int64_t d, int dtype, void *dx, const void *base, void *dweight, int grad_dtype, void *workspace,
                      size_t workspace_bytes, void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(T) || d < 1 || !is_dtype(dtype) || !is_dtype(grad_dtype) || !weight || !dweight) return GAF_ERR_ARG;
    if (d > kNormMaxWidth) return GAF_ERR_TOO_LARGE;
    if (T > 0 && ((h != nullptr) == (h_codes != nullptr) || !rstd)) return GAF_ERR_ARG;
    GAF_TRY(check_matrix(dy, T, d, dy_stride));
    if (h) GAF_TRY(check_matrix(h, T, d, h_stride));
    if (h_codes) GAF_TRY(check_codes(h_codes, h_scales, T, d, h_codes_stride));
    if (residual_grad) GAF_TRY(check_matrix(residual_grad, T, d, residual_grad_stride));
    GAF_TRY(check_matrix(dx, T, d, d));
    if (!aligned16(weight) || !aligned16(rstd) || !aligned16(base) || !aligned16(dweight)) return GAF_ERR_ALIGN;
    const size_t e = elem_bytes(dtype), ge = elem_bytes(grad_dtype);
    const Span o_dx(dx, T, d, d, e), o_dw(dweight, 1, d, d, ge), i_dy(dy, T, d, dy_stride, e), i_res(residual_grad, T, d, residual_grad_stride, e),
        i_base(base, 1, d, d, ge);
    const Span others[5] = {Span(h, T, d, h_stride, e), Span(h_codes, T, d, h_codes_stride, 1), Span(h_scales, T, blocks_of(d), blocks_of(d), 1),
                            Span(weight, 1, d, d, e), Span(rstd, T, 1, 1, 4)};
    for (const Span &i : others)
        if (o_dx.meets(i) || o_dw.meets(i)) return GAF_ERR_ALIAS;
    // (dx in the place of dy or of the residual's gradient, dweight in that of base: every element is read by the thread that writes it)
    if (o_dx.meets(o_dw) || o_dx.meets(i_base) || o_dw.meets(i_dy) || o_dw.meets(i_res) || (o_dx.meets(i_dy) && !o_dx.same(i_dy)) ||
        (o_dx.meets(i_res) && !o_dx.same(i_res)) || (o_dw.meets(i_base) && !o_dw.same(i_base))) return GAF_ERR_ALIAS;
    GAF_TRY(check_workspace(workspace, workspace_bytes, norm_grad_bytes(d)));
    DeviceInfo di;
    if (!device_info(&di)) return GAF_ERR_CUDA;
    NormGradArgs a{};
    a.dy = dy; a.h = h; a.weight = weight; a.residual_grad = residual_grad; a.h_codes = h_codes; a.h_scales = h_scales; a.rstd = rstd; a.dx = dx;
    a.partials = in_workspace<float>(workspace, kLayerScratchOffset);
    a.dy_stride = dy_stride; a.h_stride = h_stride; a.codes_stride = h_codes_stride; a.residual_grad_stride = residual_grad_stride;
    a.T = T; a.d = d; a.blocks = blocks_of(d);
    NormFinishArgs f{};
    f.partials = a.partials; f.base = base; f.dweight = dweight; f.d = d;
    return launch_rms_norm_grad(a, f, dtype, grad_dtype, wide_rows(d, T, {dy_stride, h ? h_stride : 0, residual_grad ? residual_grad_stride : 0}), di,
                                static_cast<cudaStream_t>(cuda_stream));
}

int gaf_checkpoint_pack(const void *x, int64_t x_stride, int64_t T, int64_t d, int dtype, uint8_t *codes, int64_t codes_stride, uint8_t *scales,
                        void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(T) || !in_range(d) || !is_dtype(dtype)) return GAF_ERR_ARG;
    GAF_TRY(check_matrix(x, T, d, x_stride));
    GAF_TRY(check_codes(codes, scales, T, d, codes_stride));
    if (T == 0 || d == 0) return GAF_OK;
    const Span i(x, T, d, x_stride, elem_bytes(dtype)), c(codes, T, d, codes_stride, 1), s(scales, T, blocks_of(d), blocks_of(d), 1);
    if (i.meets(c) || i.meets(s) || c.meets(s)) return GAF_ERR_ALIAS;
    CheckpointArgs a{};
    a.x = x; a.codes = codes; a.scales = scales; a.x_stride = x_stride; a.codes_stride = codes_stride; a.d = d;
    if (T > INT32_MAX / ceil_div(d, kTile)) return GAF_ERR_TOO_LARGE;      // (tiles are counted in 32 bits)
    a.tiles_per_row = unsigned(ceil_div(d, kTile)); a.n_tiles = unsigned(T) * a.tiles_per_row; a.blocks = blocks_of(d);
    return launch_checkpoint<true>(a, dtype, wide_rows(d, T, {x_stride}), static_cast<cudaStream_t>(cuda_stream));
}

int gaf_checkpoint_unpack(const uint8_t *codes, int64_t codes_stride, const uint8_t *scales, int64_t T, int64_t d, int dtype, void *out,
                          int64_t out_stride, void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(T) || !in_range(d) || !is_dtype(dtype)) return GAF_ERR_ARG;
    GAF_TRY(check_codes(codes, scales, T, d, codes_stride));
    GAF_TRY(check_matrix(out, T, d, out_stride));
    if (T == 0 || d == 0) return GAF_OK;
    const Span o(out, T, d, out_stride, elem_bytes(dtype)), c(codes, T, d, codes_stride, 1), s(scales, T, blocks_of(d), blocks_of(d), 1);
    if (o.meets(c) || o.meets(s)) return GAF_ERR_ALIAS;
    CheckpointArgs a{};
    a.out = out; a.codes = const_cast<uint8_t *>(codes); a.scales = const_cast<uint8_t *>(scales);
    a.x_stride = out_stride; a.codes_stride = codes_stride; a.d = d;
    if (T > INT32_MAX / ceil_div(d, kTile)) return GAF_ERR_TOO_LARGE;      // (tiles are counted in 32 bits)
    a.tiles_per_row = unsigned(ceil_div(d, kTile)); a.n_tiles = unsigned(T) * a.tiles_per_row; a.blocks = blocks_of(d);
    return launch_checkpoint<false>(a, dtype, wide_rows(d, T, {out_stride}), static_cast<cudaStream_t>(cuda_stream));
}

int gaf_linear_weight_grad(const void *dy, int64_t dy_stride, int dtype, const uint8_t *codes, int64_t codes_stride, const uint8_t *scales, int64_t T,
                           int64_t N, int64_t M, const void *base, void *dweight, int grad_dtype, void *workspace, size_t workspace_bytes,
                           void *cuda_stream) {
    set_last_launch_count(0);
    if (!in_range(T) || !in_range(N) || !in_range(M) || !is_dtype(dtype) || !is_dtype(grad_dtype)) return GAF_ERR_ARG;
    GAF_TRY(check_matrix(dy, T, N, dy_stride));
    GAF_TRY(check_codes(codes, scales, T, M, codes_stride));
    GAF_TRY(check_matrix(dweight, N, M, M));
    if (!aligned16(base)) return GAF_ERR_ALIGN;
    if (N == 0 || M == 0) return GAF_OK;
    // tensor copies read bfloat16 rows that start on 16-byte boundaries; everything else is laid out anew
    const int relaid = dtype == GAF_F32 ? 3 : (T > 1 && dy_stride % 8 != 0 ? 1 : 0);
    const size_t ge = elem_bytes(grad_dtype);
    const Span o(dweight, N, M, M, ge), b(base, N, M, M, ge);
    if (o.meets(Span(dy, T, N, dy_stride, elem_bytes(dtype))) || o.meets(Span(codes, T, M, codes_stride, 1)) ||
        o.meets(Span(scales, T, blocks_of(M), blocks_of(M), 1)) || (base && !o.same(b) && o.meets(b))) return GAF_ERR_ALIAS;
    DeviceInfo di;
    if (!device_info(&di)) return GAF_ERR_CUDA;
    // (a device with more SMs than the workspace was laid out for would split no further)
    const WgPlan p = weight_grad_plan(T, N, M, dtype, std::min<int64_t>(di.sms / 2, kWgMaxSplitItems));
    // (tile coordinates are 32 bits)
    if (N > kMaxRows - kWgPairM || M > kMaxRows - kWgPairM || p.steps * kWgK > kMaxRows || p.tiles_m * p.tiles_n > INT32_MAX / kWgMaxSplitItems) return GAF_ERR_TOO_LARGE;
    const WgLayout l = weight_grad_layout(p, N, relaid);
    GAF_TRY(check_workspace(workspace, workspace_bytes, l.end));
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int launches = 0;

    WeightGradArgs w{};
    w.scales = scales; w.base = base; w.dweight = dweight;
    w.partials = in_workspace<float>(workspace, l.partials);
    w.ctl = static_cast<Control *>(workspace);
    w.T = int(T); w.N = N; w.M = M; w.blocks = int(blocks_of(M)); w.scale_bytes = T * blocks_of(M);
    w.steps = int(p.steps); w.steps_per_term = int(std::max<int64_t>(1, p.steps_per_term)); w.steps_per_split = int(p.steps_per_split);
    w.tiles_m = int(p.tiles_m); w.whole = int(p.whole); w.rest = int(p.rest); w.items = int(p.whole + p.rest * p.splits);
    w.spin_limit = test_wait_limit() ? test_wait_limit() : kWgSpinLimit;
    w.test_extra_arrival = test_withhold() & 1;

    CUtensorMap dy_map{}, code_map{};
    if (T > 0) {
        const void *y = dy;
        int64_t y_rows = T, y_pitch = (T > 1 ? dy_stride : int64_t(round_up(size_t(N), 8))) * 2;
        if (relaid) {
            WgTermsArgs t{};
            t.dy = dy; t.out = in_workspace<__nv_bfloat16>(workspace, l.terms);
            t.stride = dy_stride; t.T = T; t.N = N; t.rows = p.steps_per_term * kWgK; t.pitch = int64_t(round_up(size_t(N), 8));
            cudaLaunchConfig_t cfg{};
            cfg.gridDim = dim3(unsigned(ceil_div(t.pitch, 256)), unsigned(std::min<int64_t>(t.rows, 65535)));
            cfg.blockDim = dim3(256);
            cfg.stream = st;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            cfg.attrs = attr; cfg.numAttrs = 1;
            const cudaError_t err = dtype == GAF_F32 ? cudaLaunchKernelEx(&cfg, weight_grad_terms_kernel<float>, t)
                                                     : cudaLaunchKernelEx(&cfg, weight_grad_terms_kernel<__nv_bfloat16>, t);
            ++launches;
            if (err != cudaSuccess) return launched(err, launches);
            y = t.out; y_rows = relaid * t.rows; y_pitch = t.pitch * 2;
        }
        if (!matrix_map(&dy_map, y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, N, y_rows, y_pitch, 64, kWgK, CU_TENSOR_MAP_SWIZZLE_128B) ||
            !matrix_map(&code_map, codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, M, T, T > 1 ? codes_stride : int64_t(round_up(size_t(M), 16)),
                        kWgM, kWgK, CU_TENSOR_MAP_SWIZZLE_128B))
            return GAF_ERR_CUDA;
    }
    GAF_TRY(grad_dtype == GAF_F32 ? launch_weight_grad_tiles<float>(w, dy_map, code_map, di, st, &launches)
                                  : launch_weight_grad_tiles<__nv_bfloat16>(w, dy_map, code_map, di, st, &launches));
    if (p.rest == 0) return GAF_OK;
    WgJoinArgs j{};
    j.partials = w.partials; j.base = base; j.dweight = dweight; j.N = N; j.M = M;
    j.splits = int(p.splits); j.tiles_m = int(p.tiles_m); j.whole = int(p.whole); j.rest = int(p.rest);
    const int grid = int(p.rest) * (kWgPairM * kWgN / kWgJoinElements);
    const cudaError_t err = grad_dtype == GAF_F32 ? launch_dependent(weight_grad_join_kernel<float>, grid, kWgJoinElements / 4, st, j)
                                                  : launch_dependent(weight_grad_join_kernel<__nv_bfloat16>, grid, kWgJoinElements / 4, st, j);
    return launched(err, launches + 1);
}

}  // extern "C"
