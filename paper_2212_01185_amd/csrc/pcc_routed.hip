// Host side of the operators of include/pcc.h that stand round the grouped products: layer norm, routing, rows by expert, dropout.
#include "pcc.h"
#include "train_dropout.h"
#include "train_experts.h"
#include "train_host.h"
#include "train_norm.h"
#include "train_route.h"

using namespace pcc_train;

namespace {

bool type_ok(int type) { return type >= PCC_BF16 && type <= PCC_FP32; }
Span matrix(const void* p, size_t rows, size_t ld, size_t features, int type) { return {p, rows, ld * size_of(type), features * size_of(type)}; }

// f(type of the rows) and f(type, other type), as tags.
template <class F>
int with_type(int type, F&& f) { return type == PCC_BF16 ? f(Bf16{}) : type == PCC_FP16 ? f(Fp16{}) : f(Fp32{}); }

// ---------------------------------------------------------------------------
// Layer norm.
// ---------------------------------------------------------------------------
template <int LANES, int N>
struct RowShape {
    static constexpr int kLanes = LANES, kChunks = N;
};
// How many lanes have a row, and how many eights of it each.  us, four and two eights a lane: rows of several waves, 16,384 of 4,096 forward 58.6 and 58.4
// (8,192 in fp32 57.9 and 57.2), 8,192 of 4,096 backward 83 and 80, 8,192 of 8,192 forward 60 and 57; of one wave 65,536 of 1,024 forward 59 and 64.
template <bool FORWARD, class F>
int with_row_shape(int features, F&& f) {
    const int eights = features / 8;
    if (eights <= 8) return f(RowShape<8, 1>{});
    if (eights <= 24) return f(RowShape<8, 3>{});
    if (eights <= 32) return f(RowShape<8, 4>{});
    if (eights <= 64) return f(RowShape<16, 4>{});
    if (eights <= 128) return f(RowShape<32, 4>{});
    if (eights <= 256) return f(RowShape<64, 4>{});
    if (eights <= 512) return f(RowShape<256, 2>{});
    if (eights <= 1024) return f(RowShape<512, 2>{});
    if (eights <= 2048) {       // (without sums to keep, a thread needs few enough registers for 1024 of them: 4,096 rows of 16,384 62 us, else 67)
        if constexpr (FORWARD) return f(RowShape<1024, 2>{});
        else return f(RowShape<512, 4>{});
    }
    return f(RowShape<kLongThreads, 0>{});      // read again for each sum
}
// x and y have one type, or x is fp32 and y a 16-bit one.
template <class F>
int with_norm_types(int type, int y_type, F&& f) {
    if (type == PCC_BF16) return f(Bf16{}, Bf16{});
    if (type == PCC_FP16) return f(Fp16{}, Fp16{});
    return y_type == PCC_BF16 ? f(Fp32{}, Bf16{}) : y_type == PCC_FP16 ? f(Fp32{}, Fp16{}) : f(Fp32{}, Fp32{});
}
bool norm_ok(const int64_t* d_offsets, int groups, size_t rows, int features, int type, int y_type) {
    return type_ok(type) && type_ok(y_type) && (type == y_type || type == PCC_FP32) && features >= 1 && features <= PCC_MAX_FEATURES && groups >= 1 &&
           groups <= PCC_MAX_GROUPS && rows <= kMaxRows && (d_offsets || groups == 1) && aligned(d_offsets, 8);
}
int log2_of(int v) { return v <= 1 ? 0 : 1 + log2_of(v / 2); }

// Chunks of whole turns of a workgroup's teams, `want` of them at most if there are not too many groups for that: as many as run at once, for a
// workgroup's start (weights) and end (sums) are worth some rows.
void norm_chunks(size_t rows, int groups, int want, int teams, int& log2, uint32_t& mult) {
    const size_t whole = groups == 1 ? want : want > 2 * groups ? want - groups : want / 2 + 1, least = (rows + whole - 1) / whole;
    log2 = log2_of(teams);
    while (log2 < 24 && ((size_t)64 << log2) < least) ++log2;
    mult = (uint32_t)std::min<size_t>(std::max<size_t>((least + ((size_t)1 << log2) - 1) >> log2, 1), 64);
}
// Chunks whose sums are joined: a workgroup of 512 threads for each compute unit, five of 256 threads, whose rows are short and sums few.  us with 128, 256, 512,
// 1,024 and 1,280 chunks: 786,432 rows of 36 171, 94, 59, 49, 51, of 64 168, 95, 71, 72, 74 (256 threads); 393,216 of 160 107, 86, 90, 97, 98, 32,768 of 1,024 57, 50, 57,
// 69, 69, 8,192 of 4,096 67, 51, 57, 61, 61, 2,048 of 16,384 71, 63, 75, 102, 102 (512 threads; where registers and LDS would let two workgroups run at once, too:
// 16,384 of 2,560 103, 63, 61, 64, 67).
void sums_chunks(size_t rows, int groups, int features, int& log2, uint32_t& mult) {
    const int threads = with_row_shape<false>(features, [](auto shape) { return norm_grad_threads(decltype(shape)::kLanes, decltype(shape)::kChunks); });
    const int teams = with_row_shape<false>(features, [](auto shape) { return std::max(1, norm_grad_teams(decltype(shape)::kLanes, decltype(shape)::kChunks)); });
    norm_chunks(rows, groups, threads == 256 ? 1280 : 256, teams, log2, mult);
}

}  // namespace

extern "C" {

int pcc_layer_norm(const void* d_x, size_t ldx, const float* d_gamma, const float* d_beta, const int64_t* d_offsets, int groups, size_t rows,
                   int features, float eps, int type, void* d_y, int y_type, size_t ldy, float* d_stats, void* hip_stream) {
    if ((rows && (!d_x || !d_y)) || !norm_ok(d_offsets, groups, rows, features, type, y_type) || !ld_ok(ldx, features) || !ld_ok(ldy, features)) return PCC_E_ARG;
    if (!(eps >= 0x1p-126f && eps < __builtin_inff())) return PCC_E_ARG;
    if (!aligned(d_x, size_of(type)) || !aligned(d_y, size_of(y_type)) || !aligned(d_gamma, 4) || !aligned(d_beta, 4) || !aligned(d_stats, 4)) return PCC_E_ARG;
    if (rows == 0) return PCC_OK;
    const size_t weights = (size_t)groups * features * 4;
    const Span x = matrix(d_x, rows, ldx, features, type), gamma = piece(d_gamma, weights), beta = piece(d_beta, weights),
               offsets = piece(d_offsets, (size_t)(groups + 1) * 8), y = matrix(d_y, rows, ldy, features, y_type), stats = piece(d_stats, rows * 8);
    if (overlap(y, {x, gamma, beta, offsets, stats}) || overlap(stats, {x, gamma, beta, offsets})) return PCC_E_ARG;
    Norm a = {};
    a.x = d_x; a.gamma = d_gamma; a.beta = d_beta; a.off = d_offsets; a.y = d_y; a.stats = d_stats;
    a.ldx = ldx; a.ldy = ldy; a.rows = (int64_t)rows; a.groups = groups; a.features = features; a.eps = eps; a.inverse = 1.0f / (float)features;
    return with_row_shape<true>(features, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        norm_chunks(rows, groups, L <= 64 ? 2048 : L <= 512 ? 512 : 256, norm_teams(L), a.log2, a.mult);
        const uint64_t blocks = chunk_count(a.rows, groups, a.log2, a.mult);
        if (!launchable(blocks, norm_threads(L))) return PCC_E_ARG;
        return with_norm_types(type, y_type, [&](auto tx, auto ty) {
            if constexpr (N > 0)
                if (!allow_lds(layer_norm_kernel<decltype(tx), decltype(ty), L, N>, 2 * Weights::values(features) * sizeof(float))) { (void)hipGetLastError(); return PCC_E_HIP; }
            return launch([&] {
                const dim3 grid((uint32_t)((blocks + 7) / 8 * 8)), threads(norm_threads(L));
                if constexpr (N == 0) hipLaunchKernelGGL((layer_norm_long_kernel<decltype(tx), decltype(ty)>), grid, threads, 0, (hipStream_t)hip_stream, a);
                else hipLaunchKernelGGL((layer_norm_kernel<decltype(tx), decltype(ty), L, N>), grid, threads, 2 * Weights::values(features) * sizeof(float), (hipStream_t)hip_stream, a);
            });
        });
    });
}

size_t pcc_layer_norm_grad_workspace_bytes(size_t rows, int groups, int features) {
    if (features < 1 || features > PCC_MAX_FEATURES || groups < 1 || groups > PCC_MAX_GROUPS || rows > kMaxRows) return 0;
    int log2;
    uint32_t mult;
    sums_chunks(rows, groups, features, log2, mult);
    return shared_chunks(rows, groups, (size_t)mult << log2) * 2 * features * sizeof(float);
}

int pcc_layer_norm_grad(const void* d_dy, int y_type, size_t lddy, const void* d_x, size_t ldx, const float* d_stats, const float* d_gamma,
                        const int64_t* d_offsets, int groups, size_t rows, int features, int type, void* d_dx, size_t lddx, float* d_dgamma,
                        float* d_dbeta, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if ((rows && (!d_dy || !d_x || !d_stats)) || (!d_dx && !d_dgamma) || !d_dgamma != !d_dbeta) return PCC_E_ARG;
    if (!norm_ok(d_offsets, groups, rows, features, type, y_type) || !ld_ok(lddy, features) || !ld_ok(ldx, features) || (d_dx && !ld_ok(lddx, features))) return PCC_E_ARG;
    if (!aligned(d_dy, size_of(y_type)) || !aligned(d_x, size_of(type)) || !aligned(d_dx, size_of(type)) || !aligned(d_stats, 4) || !aligned(d_gamma, 4) ||
        !aligned(d_dgamma, 4) || !aligned(d_dbeta, 4)) return PCC_E_ARG;
    const size_t need = d_dgamma ? pcc_layer_norm_grad_workspace_bytes(rows, groups, features) : 0;
    if (need && (!d_workspace || workspace_bytes < need)) return PCC_E_SCRATCH;
    if (need && !aligned(d_workspace, 16)) return PCC_E_ARG;
    const size_t weights = (size_t)groups * features * 4;
    const Span dy = matrix(d_dy, rows, lddy, features, y_type), x = matrix(d_x, rows, ldx, features, type), stats = piece(d_stats, rows * 8),
               gamma = piece(d_gamma, weights), offsets = piece(d_offsets, (size_t)(groups + 1) * 8), dx = matrix(d_dx, rows, lddx, features, type),
               dgamma = piece(d_dgamma, weights), dbeta = piece(d_dbeta, weights), space = piece(d_workspace, need);
    if (overlap(dx, {dy, x, stats, gamma, offsets, dgamma, dbeta, space}) || overlap(dgamma, {dy, x, stats, gamma, offsets, dbeta, space}) ||
        overlap(dbeta, {dy, x, stats, gamma, offsets, space}) || overlap(space, {dy, x, stats, gamma, offsets})) return PCC_E_ARG;
    Norm a = {};
    a.x = d_x; a.dy = d_dy; a.gamma = d_gamma; a.off = d_offsets; a.y = d_dx; a.stats = const_cast<float*>(d_stats); a.dgamma = d_dgamma; a.dbeta = d_dbeta;
    a.partial = (float*)d_workspace;
    a.ldx = ldx; a.lddy = lddy; a.ldy = lddx; a.rows = (int64_t)rows; a.groups = groups; a.features = features; a.inverse = 1.0f / (float)features;
    a.shared_max = (uint32_t)std::min<size_t>(need / (2 * features * sizeof(float)), 0xFFFFFFFFu);
    hipStream_t st = (hipStream_t)hip_stream;
    const int rc = with_row_shape<false>(features, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        return with_norm_types(type, y_type, [&](auto tx, auto ty) {
            using X = decltype(tx);
            using Y = decltype(ty);
            if constexpr (N == 0) {
                if (d_dx && rows) {
                    norm_chunks(rows, groups, 2048, 1, a.log2, a.mult);
                    const uint64_t blocks = chunk_count(a.rows, groups, a.log2, a.mult);
                    if (!launchable(blocks, kLongThreads)) return PCC_E_ARG;
                    const int rc = launch([&] {
                        hipLaunchKernelGGL((layer_norm_long_dx_kernel<X, Y>), dim3((uint32_t)((blocks + 7) / 8 * 8)), dim3(kLongThreads), 0, st, a);
                    });
                    if (rc != PCC_OK) return rc;
                }
                sums_chunks(rows, groups, features, a.log2, a.mult);
                const uint64_t blocks = chunk_count(a.rows, groups, a.log2, a.mult);
                if (!d_dgamma) return PCC_OK;
                if (!launchable(blocks * 8, 256)) return PCC_E_ARG;
                return launch([&] {
                    hipLaunchKernelGGL((layer_norm_sums_kernel<X, Y>), dim3((uint32_t)((blocks + 7) / 8 * 8), std::min((features + 255) / 256, 8)), dim3(256), 0, st, a);
                });
            } else {
                sums_chunks(rows, groups, features, a.log2, a.mult);
                const uint64_t blocks = chunk_count(a.rows, groups, a.log2, a.mult);
                if (!launchable(blocks, norm_grad_threads(L, N))) return PCC_E_ARG;
                const size_t lds = Weights::values(features) * sizeof(float) * 2 * norm_grad_shares(L, N);     // sums take the weights' place
                if (!allow_lds(layer_norm_grad_kernel<X, Y, L, N>, lds)) { (void)hipGetLastError(); return PCC_E_HIP; }
                return launch([&] {
                    hipLaunchKernelGGL((layer_norm_grad_kernel<X, Y, L, N>), dim3((uint32_t)((blocks + 7) / 8 * 8)), dim3(norm_grad_threads(L, N)), lds, st, a);
                });
            }
        });
    });
    if (rc != PCC_OK || !d_dgamma || rows <= (size_t)a.mult << a.log2) return rc;        // no group can have two chunks
    return launch([&] {
        hipLaunchKernelGGL(layer_norm_join_kernel, dim3(std::min((2 * features + 63) / 64, std::max(4, 4096 / groups)), groups), dim3(kJoinThreads), 0, st, a);
    });
}

// ---------------------------------------------------------------------------
// Routing.
// ---------------------------------------------------------------------------
}  // extern "C"

namespace {

bool choices_ok(size_t tokens, int k, int experts) {
    return k >= 1 && k <= PCC_MAX_CHOICES && experts >= 1 && experts <= PCC_MAX_EXPERTS && tokens < ((size_t)1 << 31) / k;
}
template <class F>
int with_lanes(int experts, F&& f) {
    const int chunks = (experts + 7) / 8;
    if (chunks <= 1) return f(RowShape<1, 1>{});
    if (chunks <= 2) return f(RowShape<2, 1>{});
    if (chunks <= 4) return f(RowShape<4, 1>{});
    if (chunks <= 8) return f(RowShape<8, 1>{});
    if (chunks <= 16) return f(RowShape<16, 1>{});
    if (chunks <= 32) return f(RowShape<32, 1>{});
    if (chunks <= 64) return f(RowShape<64, 1>{});
    return f(RowShape<64, 2>{});
}

}  // namespace

extern "C" {

int pcc_route(const void* d_logits, size_t ldl, size_t tokens, int experts, int k, int type, int over_all, int32_t* d_expert, float* d_weight,
              void* hip_stream) {
    if ((tokens && (!d_logits || !d_expert || !d_weight)) || !choices_ok(tokens, k, experts) || k > experts || !type_ok(type) || !ld_ok(ldl, experts)) return PCC_E_ARG;
    if ((over_all != 0 && over_all != 1) || !aligned(d_logits, size_of(type)) || !aligned(d_expert, 4) || !aligned(d_weight, 4)) return PCC_E_ARG;
    if (tokens == 0) return PCC_OK;
    const Span logits = matrix(d_logits, tokens, ldl, experts, type), expert = piece(d_expert, tokens * k * 4), weight = piece(d_weight, tokens * k * 4);
    if (overlap(expert, {logits, weight}) || overlap(weight, logits)) return PCC_E_ARG;
    Route a = {};
    a.logits = d_logits; a.expert = d_expert; a.weight = d_weight; a.ldl = ldl; a.tokens = tokens; a.experts = experts; a.k = k; a.over_all = over_all;
    return with_lanes(experts, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        const uint64_t blocks = (tokens + kRouteThreads / L - 1) / (kRouteThreads / L);
        if (!launchable(blocks, kRouteThreads)) return PCC_E_ARG;
        return with_type(type, [&](auto t) {
            return launch([&] { hipLaunchKernelGGL((route_kernel<decltype(t), L, N>), dim3((uint32_t)blocks), dim3(kRouteThreads), 0, (hipStream_t)hip_stream, a); });
        });
    });
}

int pcc_route_grad(const float* d_dweight, const void* d_logits, size_t ldl, const int32_t* d_expert, const float* d_weight, size_t tokens, int experts,
                   int k, int type, int over_all, void* d_dlogits, size_t lddl, void* hip_stream) {
    if ((tokens && (!d_dweight || (over_all && !d_logits) || !d_expert || !d_weight || !d_dlogits)) || !choices_ok(tokens, k, experts) || k > experts) return PCC_E_ARG;
    if (!type_ok(type) || !ld_ok(ldl, experts) || !ld_ok(lddl, experts) || (over_all != 0 && over_all != 1)) return PCC_E_ARG;
    if (!aligned(d_dweight, 4) || !aligned(d_logits, size_of(type)) || !aligned(d_expert, 4) || !aligned(d_weight, 4) || !aligned(d_dlogits, size_of(type))) return PCC_E_ARG;
    if (tokens == 0) return PCC_OK;
    const size_t chosen = tokens * k * 4;
    if (overlap(matrix(d_dlogits, tokens, lddl, experts, type),
                {matrix(d_logits, tokens, ldl, experts, type), piece(d_dweight, chosen), piece(d_expert, chosen), piece(d_weight, chosen)})) return PCC_E_ARG;
    Route a = {};
    a.logits = d_logits; a.dweight = d_dweight; a.expert = const_cast<int32_t*>(d_expert); a.weight = const_cast<float*>(d_weight); a.dlogits = d_dlogits;
    a.ldl = ldl; a.lddl = lddl; a.tokens = tokens; a.experts = experts; a.k = k; a.over_all = over_all;
    return with_lanes(experts, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        const uint64_t blocks = (tokens + kRouteThreads / L - 1) / (kRouteThreads / L);
        if (!launchable(blocks, kRouteThreads)) return PCC_E_ARG;
        return with_type(type, [&](auto t) {
            return launch([&] { hipLaunchKernelGGL((route_grad_kernel<decltype(t), L, N>), dim3((uint32_t)blocks), dim3(kRouteThreads), 0, (hipStream_t)hip_stream, a); });
        });
    });
}

// ---------------------------------------------------------------------------
// Rows by expert.
// ---------------------------------------------------------------------------
}  // extern "C"

namespace {

// Segments of the sort: whole rounds of its waves, 256 of them at most, and with many experts fewer, since every workgroup sums all segments' counts.
uint32_t sort_segment(size_t entries, int experts) {
    const size_t most = std::min(256, std::max(64, 32768 / experts)), least = (entries + most - 1) / most;
    return (uint32_t)std::max<size_t>(4096, (least + 1023) / 1024 * 1024);
}
uint32_t sort_segments(size_t entries, int experts) {
    const uint32_t segment = sort_segment(entries, experts);
    return (uint32_t)std::max<size_t>(1, (entries + segment - 1) / segment);
}

// Rows of `features` values, their places and weights.
bool rows_ok(size_t tokens, int k, size_t rows, int features, int type) {
    return k >= 1 && k <= PCC_MAX_CHOICES && tokens < ((size_t)1 << 31) / k && rows < (size_t)1 << 31 && features >= 1 && features <= PCC_MAX_FEATURES && type_ok(type);
}
// The tokens' side has the rows' type or fp32.
template <class F>
int with_row_types(int type, int y_type, F&& f) {
    if (type == PCC_BF16) return y_type == PCC_BF16 ? f(Bf16{}, Bf16{}) : f(Bf16{}, Fp32{});
    if (type == PCC_FP16) return y_type == PCC_FP16 ? f(Fp16{}, Fp16{}) : f(Fp16{}, Fp32{});
    return f(Fp32{}, Fp32{});
}
// How many lanes have a token's row, and how many eights of it at a time each: where it is copied, as many as it has eights, so that it
// leaves in one piece.  us, 63 million values of bf16 in rows of so many features, two rows a token, by the shape before, the rule's and the one behind it: 64 features
// -, 29, 29; 136 44, 40, 64; 256 29, 28, 28; 264 41, 40, 40; 520 40, 39, 63; 1,024 28, 29, 28; 1,032 42, 41, -; 2,056 45, 39, -; 8,192 30, 29, -.
template <class F>
int with_copy_shape(int features, F&& f) {
    const int eights = features / 8;
    if (eights <= 8) return f(RowShape<8, 1>{});
    if (eights <= 16) return f(RowShape<16, 1>{});
    if (eights <= 32) return f(RowShape<32, 1>{});
    if (eights <= 64) return f(RowShape<64, 1>{});
    if (eights <= 128) return f(RowShape<64, 2>{});
    return f(RowShape<256, 1>{});
}
// Where rows are read and joined.  us as above, join / its gradient: 64 features -, 39 / 72, 52 / 96; 136 69 / 106, 41 / 68, 55 / 86; 256 39 / 68, 37 / 63, 39 / 64; 264 48 / 70,
// 42 / 68, 55 / 87; 512 38 / 65, 37 / 65, 38 / 64; 520 47 / 70, 40 / 66, 54 / 86; 1,024 37 / 66, 37 / 65, 38 / 63; 1,032 44 / 68, 39 / 65, 83 / 137; 2,048 45 / 68, 37 / 65, 50 / 81;
// 4,096 38 / 66, 37 / 63, -; 8,192 38 / 68, 37 / 65, -.  From 2,056 to about 3,000 features the shape before would be the better one: 2,056 40 / 67, 53 / 83, -; 2,500
// 44 / 73, 51 / 90, -; 3,000 40 / 69, 42 / 67, -.
template <class F>
int with_token_shape(int features, F&& f) {
    const int eights = features / 8;
    if (eights <= 8) return f(RowShape<8, 1>{});
    if (eights <= 32) return f(RowShape<16, 2>{});
    if (eights <= 64) return f(RowShape<16, 4>{});
    if (eights <= 128) return f(RowShape<32, 4>{});
    if (eights <= 256) return f(RowShape<64, 4>{});
    return f(RowShape<256, 4>{});
}
// f(workgroups) for a token's row in LANES lanes, with the workgroups of each die in `a`.
template <class F>
int with_tokens(Experts& a, int lanes, F&& f) {
    const uint64_t teams = kExpertThreads / lanes, each = ((a.tokens + teams - 1) / teams + 7) / 8;
    if (!launchable(8 * each, kExpertThreads)) return PCC_E_ARG;
    a.each = (uint32_t)each;
    return f(dim3((uint32_t)(8 * each)));
}
uint64_t chunk_blocks(uint64_t rows, uint32_t chunks, int threads) { return (rows * chunks + threads - 1) / threads; }

}  // namespace

extern "C" {

size_t pcc_expert_sort_workspace_bytes(size_t tokens, int k, int experts) {
    if (!choices_ok(tokens, k, experts)) return 0;
    const uint32_t segments = sort_segments(tokens * k, experts);
    return segments > 1 ? (size_t)segments * experts * sizeof(uint32_t) : 0;
}

int pcc_expert_sort(const int32_t* d_expert, size_t tokens, int k, int experts, int64_t* d_offsets, int32_t* d_place, void* d_workspace,
                    size_t workspace_bytes, void* hip_stream) {
    if ((tokens && (!d_expert || !d_place)) || !d_offsets || !choices_ok(tokens, k, experts)) return PCC_E_ARG;
    if (!aligned(d_expert, 4) || !aligned(d_place, 4) || !aligned(d_offsets, 8)) return PCC_E_ARG;
    const size_t need = pcc_expert_sort_workspace_bytes(tokens, k, experts);
    if (need && (!d_workspace || workspace_bytes < need)) return PCC_E_SCRATCH;
    if (need && !aligned(d_workspace, 16)) return PCC_E_ARG;
    const size_t entries = tokens * k;
    const Span expert = piece(d_expert, entries * 4), place = piece(d_place, entries * 4), offsets = piece(d_offsets, (size_t)(experts + 1) * 8),
               space = piece(d_workspace, need);
    if (overlap(place, {expert, offsets, space}) || overlap(offsets, {expert, space}) || overlap(space, expert)) return PCC_E_ARG;
    Sort a = {};
    a.expert = d_expert; a.offsets = d_offsets; a.place = d_place; a.counts = (uint32_t*)d_workspace;
    a.entries = (uint32_t)entries; a.segment = sort_segment(entries, experts); a.segments = sort_segments(entries, experts); a.experts = experts; a.bits = log2_of(experts) + 1;
    hipStream_t st = (hipStream_t)hip_stream;
    if (a.segments > 1) {
        const int rc = launch([&] { hipLaunchKernelGGL(expert_count_kernel, dim3(a.segments), dim3(kSortThreads), (size_t)experts * sizeof(uint32_t), st, a); });
        if (rc != PCC_OK) return rc;
    }
    const size_t lds = sort_lds(experts);
    if (!allow_lds(expert_place_kernel, lds)) { (void)hipGetLastError(); return PCC_E_HIP; }
    return launch([&] { hipLaunchKernelGGL(expert_place_kernel, dim3(a.segments), dim3(kSortThreads), lds, st, a); });
}

int pcc_expert_rows(const void* d_x, size_t ldx, const int32_t* d_place, size_t tokens, int k, size_t rows, int features, int type, void* d_rows,
                    size_t ldr, void* hip_stream) {
    if ((tokens && (!d_x || !d_place)) || (tokens && rows && !d_rows) || !rows_ok(tokens, k, rows, features, type) || !ld_ok(ldx, features) || !ld_ok(ldr, features)) return PCC_E_ARG;
    if (!aligned(d_x, size_of(type)) || !aligned(d_rows, size_of(type)) || !aligned(d_place, 4)) return PCC_E_ARG;
    if (tokens == 0 || rows == 0) return PCC_OK;
    if (overlap(matrix(d_rows, rows, ldr, features, type), {matrix(d_x, tokens, ldx, features, type), piece(d_place, tokens * k * 4)})) return PCC_E_ARG;
    Experts a = {};
    a.x = d_x; a.place = d_place; a.y = d_rows; a.ldx = ldx; a.ldy = ldr; a.tokens = tokens; a.rows = rows; a.k = k; a.features = features;
    // Rows of whole lines go past the caches.  us, so and not: 500,000 tokens to 2 rows of 128 bytes 41 and 52, 65,536 to 2 of 1,024 40 and 53, but
    // 393,216 to 2 of 320 (half of a line is another row's) 84 and 82.
    const bool past = features * size_of(type) % 128 == 0 && ldr * size_of(type) % 128 == 0 && aligned(d_rows, 128);
    return with_copy_shape(features, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        return with_tokens(a, L, [&](dim3 grid) {
            auto go = [&](auto kernel) { return launch([&] { hipLaunchKernelGGL(kernel, grid, dim3(kExpertThreads), 0, (hipStream_t)hip_stream, a); }); };
            if (type == PCC_FP32) return past ? go(expert_rows_kernel<Fp32, L, N, true>) : go(expert_rows_kernel<Fp32, L, N, false>);
            return past ? go(expert_rows_kernel<Bf16, L, N, true>) : go(expert_rows_kernel<Bf16, L, N, false>);     // bits are copied
        });
    });
}

int pcc_expert_join(const void* d_z, size_t ldz, const int32_t* d_place, const float* d_weight, size_t tokens, int k, size_t rows, int features, int type,
                    void* d_y, int y_type, size_t ldy, void* hip_stream) {
    if ((tokens && (!d_place || !d_y)) || (tokens && rows && !d_z) || !rows_ok(tokens, k, rows, features, type) || (y_type != type && y_type != PCC_FP32)) return PCC_E_ARG;
    if (!ld_ok(ldz, features) || !ld_ok(ldy, features) || !aligned(d_z, size_of(type)) || !aligned(d_y, size_of(y_type)) || !aligned(d_place, 4) || !aligned(d_weight, 4)) return PCC_E_ARG;
    if (tokens == 0) return PCC_OK;
    if (overlap(matrix(d_y, tokens, ldy, features, y_type), {matrix(d_z, rows, ldz, features, type), piece(d_place, tokens * k * 4), piece(d_weight, tokens * k * 4)})) return PCC_E_ARG;
    Experts a = {};
    a.z = d_z; a.place = d_place; a.weight = d_weight; a.y = d_y; a.ldz = ldz; a.ldy = ldy; a.tokens = tokens; a.rows = rows; a.k = k; a.features = features;
    return with_token_shape(features, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        return with_tokens(a, L, [&](dim3 grid) {
            return with_row_types(type, y_type, [&](auto t, auto ty) {
                return launch([&] { hipLaunchKernelGGL((expert_join_kernel<decltype(t), decltype(ty), L, N>), grid, dim3(kExpertThreads), 0, (hipStream_t)hip_stream, a); });
            });
        });
    });
}

int pcc_expert_join_grad(const void* d_dy, int y_type, size_t lddy, const void* d_z, size_t ldz, const int32_t* d_place, const float* d_weight,
                         size_t tokens, int k, size_t rows, int features, int type, void* d_dz, size_t lddz, float* d_dweight, void* hip_stream) {
    if ((tokens && (!d_dy || !d_place || (!d_dz && !d_dweight))) || (tokens && rows && d_dweight && !d_z) || !rows_ok(tokens, k, rows, features, type)) return PCC_E_ARG;
    if ((y_type != type && y_type != PCC_FP32) || !ld_ok(lddy, features) || (d_dweight && !ld_ok(ldz, features)) || (d_dz && !ld_ok(lddz, features))) return PCC_E_ARG;
    if (!aligned(d_dy, size_of(y_type)) || !aligned(d_z, size_of(type)) || !aligned(d_dz, size_of(type)) || !aligned(d_place, 4) || !aligned(d_weight, 4) ||
        !aligned(d_dweight, 4)) return PCC_E_ARG;
    if (tokens == 0) return PCC_OK;
    const Span dy = matrix(d_dy, tokens, lddy, features, y_type), z = matrix(d_dweight ? d_z : nullptr, rows, ldz, features, type), place = piece(d_place, tokens * k * 4),
               weight = piece(d_weight, tokens * k * 4), dz = matrix(d_dz, rows, lddz, features, type), dweight = piece(d_dweight, tokens * k * 4);
    if (overlap(dz, {dy, z, place, weight, dweight}) || overlap(dweight, {dy, z, place, weight})) return PCC_E_ARG;
    Experts a = {};
    a.x = d_dy; a.z = d_z; a.place = d_place; a.weight = d_weight; a.y = d_dz; a.dweight = d_dweight;
    a.ldx = lddy; a.ldz = ldz; a.ldy = lddz; a.tokens = tokens; a.rows = rows; a.k = k; a.features = features;
    return with_token_shape(features, [&](auto shape) {
        constexpr int L = decltype(shape)::kLanes, N = decltype(shape)::kChunks;
        return with_tokens(a, L, [&](dim3 grid) {
            return with_row_types(type, y_type, [&](auto t, auto ty) {
                return launch([&] { hipLaunchKernelGGL((expert_join_grad_kernel<decltype(t), decltype(ty), L, N>), grid, dim3(kExpertThreads), 0, (hipStream_t)hip_stream, a); });
            });
        });
    });
}

// ---------------------------------------------------------------------------
// Dropout.
// ---------------------------------------------------------------------------
int pcc_dropout(const void* d_x, size_t ldx, const void* d_residual, size_t ldr, size_t rows, int features, int type, double p, uint64_t seed,
                const int64_t* d_step, void* d_y, int y_type, size_t ldy, void* hip_stream) {
    if ((rows && (!d_x || !d_y)) || rows > kMaxRows || features < 1 || features > PCC_MAX_FEATURES || !(p >= 0.0 && p <= 1.0)) return PCC_E_ARG;
    if (!type_ok(type) || !type_ok(y_type) || (type != y_type && type != PCC_FP32 && y_type != PCC_FP32)) return PCC_E_ARG;
    if (!ld_ok(ldx, features) || !ld_ok(ldy, features) || (d_residual && !ld_ok(ldr, features))) return PCC_E_ARG;
    if (!aligned(d_x, size_of(type)) || !aligned(d_residual, size_of(y_type)) || !aligned(d_y, size_of(y_type)) || !aligned(d_step, 8)) return PCC_E_ARG;
    if (rows == 0) return PCC_OK;
    const Span x = matrix(d_x, rows, ldx, features, type), residual = matrix(d_residual, rows, ldr, features, y_type), y = matrix(d_y, rows, ldy, features, y_type);
    // an element is read before it is written, by the same thread
    const bool over_x = d_y == d_x && type == y_type && ldx == ldy, over_residual = d_y == d_residual && ldr == ldy;
    if ((!over_x && overlap(y, x)) || (!over_residual && overlap(y, residual)) || overlap(y, piece(d_step, 8))) return PCC_E_ARG;
    Dropout a = {};
    a.x = d_x; a.residual = d_residual; a.y = d_y; a.ldx = ldx; a.ldr = ldr; a.ldy = ldy; a.rows = rows; a.seed = seed; a.step = d_step;
    a.border = (uint32_t)(p * 65536.0 + 0.5);
    a.scale = a.border < 65536 ? (float)(65536.0 / (65536 - a.border)) : 0.0f;
    a.features = features;
    a.chunks = (uint32_t)(features + 7) / 8;
    const uint64_t blocks = chunk_blocks(rows, a.chunks, kDropoutThreads);
    if (!launchable(blocks, kDropoutThreads)) return PCC_E_ARG;
    auto go = [&](auto kernel) { return launch([&] { hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(kDropoutThreads), 0, (hipStream_t)hip_stream, a); }); };
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        if constexpr (kIs32<T>) return y_type == PCC_BF16 ? go(dropout_kernel<Fp32, Bf16>) : y_type == PCC_FP16 ? go(dropout_kernel<Fp32, Fp16>) : go(dropout_kernel<Fp32, Fp32>);
        else return y_type == PCC_FP32 ? go(dropout_kernel<T, Fp32>) : go(dropout_kernel<T, T>);
    });
}

}  // extern "C"
