// Host side of the training operators of include/pcc.h.
#include <algorithm>
#include <iterator>
#include <new>
#include <utility>
#include <vector>

#include "pcc.h"
#include "train_adamw.h"
#include "train_contexts.h"
#include "train_grouped.h"
#include "train_host.h"
#include "train_loss.h"
#include "train_narrow.h"

using namespace pcc_train;

namespace {

// ---------------------------------------------------------------------------
// Grouped products.
// ---------------------------------------------------------------------------
bool features_ok(int in, int out, int groups, size_t rows) {
    return in >= 1 && out >= 1 && in <= PCC_MAX_FEATURES && out <= PCC_MAX_FEATURES && groups >= 1 && groups <= PCC_MAX_GROUPS && rows <= kMaxRows;
}

// Rows of a chunk of the weights' gradient.  A chunk's sums go to the workspace and are added up by another kernel, so
// there are no more chunks than fill the chip (512 workgroups at a time), none of less than 256 rows, and where the groups fill it by themselves
// only a group of twice the mean or more is cut.
int weights_log2(size_t rows, int groups, int in, int out) {
    const size_t tiles = ((size_t)in + 127) / 128 * (((size_t)out + 127) / 128), want = std::max<size_t>(1, 512 / tiles);
    const size_t least = want > (size_t)groups ? (rows + want - 1) / want : 2 * (rows / groups);
    int log2 = 8;
    while (((size_t)1 << log2) < least) ++log2;
    return log2;
}
// Rows of an operand can be read in pieces of 16 bytes, which have to begin at a multiple of four.
bool even_rows(const void* p, size_t ld) { return aligned(p, 4) && ld % 2 == 0; }

template <class T, int MODE, int TILE>
int launch_tiles_of(Grouped& a, hipStream_t st) {
    a.tiles_m = (uint32_t)(((MODE == kForward ? a.out : a.in) + TILE - 1) / TILE);
    a.tiles_n = (uint32_t)((a.out + TILE - 1) / TILE);
    a.mult = 1;
    const uint64_t chunks = ((uint64_t)a.rows >> a.log2) + a.groups, blocks = chunks * a.tiles_m * (MODE == kWeights ? a.tiles_n : 1);
    if (!launchable(blocks, tile_threads(TILE))) return PCC_E_ARG;
    const bool wide = (MODE == kBackward || even_rows(a.x, a.ldx)) && (MODE == kForward || even_rows(a.dz, a.lddz)) &&
                      (MODE == kWeights || even_rows(a.w, (size_t)a.in));
    a.wide_x = aligned(a.x, 8) && a.ldx % 4 == 0;
    a.wide_dw = aligned(a.dw, 16) && (size_t)a.in * a.out % 4 == 0;
    a.wide_out = aligned(a.y, a.y32 ? 16 : 8) && a.ldy % 4 == 0;
    const uint32_t grid = (uint32_t)((blocks + 7) / 8 * 8);     // a multiple of the dies: see find_chunk
    const size_t lds = 4 * (size_t)TILE * kTileK * sizeof(u16);
    auto go = [&](auto kernel) {
        if (!allow_lds(kernel, lds)) { (void)hipGetLastError(); return PCC_E_HIP; }
        return launch([&] { hipLaunchKernelGGL(kernel, dim3(grid), dim3(tile_threads(TILE)), lds, st, a); });
    };
    return wide ? go(grouped_tile_kernel<T, MODE, true, TILE>) : go(grouped_tile_kernel<T, MODE, false, TILE>);
}

template <class T, int MODE>
int launch_tiles(Grouped& a, hipStream_t st) {
    if (MODE != kWeights) a.log2 = 7;
    return launch_tiles_of<T, MODE, 128>(a, st);
}
// Forward: tiles of 256 where the groups have the rows for them and there are as many as compute units, else of 128.  us with 128 and
// 256: four groups of 2,048 rows, 2048 to 2048, 88 and 71; sixteen of 512, 1024 to 4096, 131 and 131; 64 of five, 1024 to 1024, 28 and 34.
template <class T>
int launch_forward_tiles(Grouped& a, hipStream_t st) {
    const uint64_t of_256 = ((uint64_t)a.rows / 256 + a.groups) * ((a.out + 255) / 256);
    if (a.rows / a.groups < 512 || of_256 < 256) return launch_tiles<T, kForward>(a, st);
    a.log2 = 8;
    return launch_tiles_of<T, kForward, 256>(a, st);
}

void chunk_rows(Grouped& a, uint64_t want, int unit_log2) { pcc_train::chunk_rows(a.rows, a.groups, want, unit_log2, a.log2, a.mult); }
uint64_t chunk_count(const Grouped& a) { return pcc_train::chunk_count(a.rows, a.groups, a.log2, a.mult); }

// The forward pass with the weights in LDS: for inputs of up to 192 features, a multiple of eight, in rows that begin at even
// elements, and weights of up to 80 KB.  us for 393,216 rows with tiles and so: 32 to 160 132 and 39, 128 to 60 68 and 41, 64 to 64
// 62 and 24, 192 to 192 164 and 79, 64 to 512 275 and 130.
bool narrow_forward_fits(const Grouped& a) {
    return a.in <= 192 && a.in % 8 == 0 && even_rows(a.x, a.ldx) && aligned(a.w, 4) && narrow_forward_lds(a.in, a.out) <= kMaxLds / 2;
}

template <class T>
int launch_narrow_forward(Grouped& a, hipStream_t st) {
    chunk_rows(a, 256, 5);
    a.wide_out = aligned(a.y, 16) && a.ldy % (a.y32 ? 4 : 8) == 0;
    const uint64_t blocks = chunk_count(a);
    if (!launchable(blocks, kNarrowThreads)) return PCC_E_ARG;
    const uint32_t grid = (uint32_t)((blocks + 7) / 8 * 8);
    const size_t weights = narrow_forward_lds(a.in, a.out), rows = narrow_rows_lds(a.out, a.y32);
    const int threads = kNarrowThreads;
    a.staged = even_rows(a.y, a.ldy * (a.y32 ? 2 : 1)) && weights + threads / 64 * rows <= kMaxLds && narrow_row_pieces(a.out, a.y32) <= kMaxRowPieces;
    const size_t lds = weights + (a.staged ? threads / 64 * rows : 0);
    auto go = [&](auto kernel) {
        if (!allow_lds(kernel, lds)) { (void)hipGetLastError(); return PCC_E_HIP; }
        return launch([&] { hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), lds, st, a); });
    };
    switch ((a.in + 31) / 32) {
        case 1: return go(grouped_narrow_forward_kernel<T, 1>);
        case 2: return go(grouped_narrow_forward_kernel<T, 2>);
        case 3: return go(grouped_narrow_forward_kernel<T, 3>);
        case 4: return go(grouped_narrow_forward_kernel<T, 4>);
        case 5: return go(grouped_narrow_forward_kernel<T, 5>);
        default: return go(grouped_narrow_forward_kernel<T, 6>);
    }
}

// The backward pass in one kernel: for up to 192 features to each side, the inputs a multiple of eight and the outputs of
// two, in rows that begin at even elements.  us for 393,216 rows with tiles and so: 32 to 160 184 and 49, 160 to 128 305 and 89, 128 to 36
// 299 and 58, 192 to 192 325 and 118.
bool narrow_backward_fits(const Grouped& a) {
    return a.in <= 192 && a.out <= 192 && a.in % 8 == 0 && a.out % 2 == 0 && a.dw && even_rows(a.x, a.ldx) && even_rows(a.dz, a.lddz) &&
           (!a.y || (aligned(a.w, 4) && aligned(a.y, 4) && a.ldy % 2 == 0));
}
uint64_t backward_chunks(Grouped& a) {
    chunk_rows(a, 256, 6);
    return chunk_count(a);
}

template <class T>
int launch_narrow_backward(Grouped& a, hipStream_t st) {
    const uint64_t blocks = backward_chunks(a);
    a.wide_dw = aligned(a.dw, 16) && (size_t)a.in * a.out % 4 == 0;
    if (!launchable(blocks, kNarrowThreads)) return PCC_E_ARG;
    const uint32_t grid = (uint32_t)((blocks + 7) / 8 * 8);
    auto go = [&](auto kernel, size_t lds) {
        if (!allow_lds(kernel, lds)) { (void)hipGetLastError(); return PCC_E_HIP; }
        return launch([&] { hipLaunchKernelGGL(kernel, dim3(grid), dim3(kNarrowThreads), lds, st, a); });
    };
    auto with_out = [&](auto pairs) {
        constexpr int P = decltype(pairs)::value;
        switch ((a.out + 31) / 32) {
            case 1: case 2: return go(grouped_narrow_backward_kernel<T, P, 2>, NarrowBackward<P, 2>::kLds);
            case 3: return go(grouped_narrow_backward_kernel<T, P, 3>, NarrowBackward<P, 3>::kLds);
            case 4: return go(grouped_narrow_backward_kernel<T, P, 4>, NarrowBackward<P, 4>::kLds);
            case 5: return go(grouped_narrow_backward_kernel<T, P, 5>, NarrowBackward<P, 5>::kLds);
            default: return go(grouped_narrow_backward_kernel<T, P, 6>, NarrowBackward<P, 6>::kLds);
        }
    };
    switch ((a.in + 31) / 32) {
        case 1: return with_out(std::integral_constant<int, 1>{});
        case 2: return with_out(std::integral_constant<int, 2>{});
        case 3: case 4: return with_out(std::integral_constant<int, 4>{});
        case 5: return with_out(std::integral_constant<int, 5>{});
        default: return with_out(std::integral_constant<int, 6>{});
    }
}

}  // namespace

struct pcc_adamw {
    int device = 0;
    int grad_type = 0, copy_type = 0, state_bits = 32;
    uint32_t n_pieces = 0;
    int piece_blocks = 1;
    uint8_t* d_table = nullptr;     // rates of the step, tensors, pieces
    AdamwTensor* d_tensors = nullptr;
    AdamwPiece* d_pieces = nullptr;
};

extern "C" {

int pcc_contexts(const uint8_t* d_img, int n, int H, int W, int nbhd, int delay, void* d_x, int width, size_t ldx, void* hip_stream) {
    if (!d_img || !d_x || n < 1 || H < 1 || W < 1 || (size_t)H * W > (size_t)1 << 31) return PCC_E_ARG;
    const uint64_t pixels = (uint64_t)n * H * W;
    if (!((nbhd == 10 && delay == 2) || (nbhd == 12 && (delay == 3 || delay == 1)))) return PCC_E_ARG;
    if (width < 3 * nbhd || width > PCC_MAX_FEATURES || !ld_ok(ldx, width) || !aligned(d_x, 2)) return PCC_E_ARG;
    const uint64_t blocks = (pixels + kContextThreads - 1) / kContextThreads;
    if (pixels > kMaxRows || !launchable(blocks, kContextThreads)) return PCC_E_ARG;
    if (overlap({d_x, pixels, ldx * 2, (size_t)width * 2}, piece(d_img, pixels * 3))) return PCC_E_ARG;
    const int wide = aligned(d_x, 4) && ldx % 2 == 0 && width % 8 == 0 && width <= kContextWidth;
    auto go = [&](auto kernel) {
        return launch([&] { hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(kContextThreads), 0, (hipStream_t)hip_stream, d_img, pixels, H, W, (u16*)d_x, width, ldx, wide); });
    };
    return nbhd == 10 ? go(contexts_kernel<10, 2>) : delay == 3 ? go(contexts_kernel<12, 3>) : go(contexts_kernel<12, 1>);
}

int pcc_grouped_linear(const void* d_x, size_t ldx, const void* d_w, const float* d_bias, const int64_t* d_offsets, int groups,
                       size_t rows, int in, int out, int type, int act, void* d_y, int y_type, size_t ldy, void* hip_stream) {
    if ((rows && (!d_x || !d_y)) || !d_w || !d_offsets || !features_ok(in, out, groups, rows) || !ld_ok(ldx, in) || !ld_ok(ldy, out)) return PCC_E_ARG;
    if ((type != PCC_BF16 && type != PCC_FP16) || (y_type != type && y_type != PCC_FP32) || act < PCC_ACT_RELU || act > PCC_ACT_NONE) return PCC_E_ARG;
    if (!aligned(d_x, 2) || !aligned(d_w, 2) || !aligned(d_bias, 4) || !aligned(d_offsets, 8) || !aligned(d_y, size_of(y_type))) return PCC_E_ARG;
    if (rows == 0) return PCC_OK;
    const size_t weights = (size_t)groups * in * out, outputs = (size_t)groups * out;
    if (overlap({d_y, rows, ldy * size_of(y_type), out * size_of(y_type)},
                {{d_x, rows, ldx * 2, (size_t)in * 2}, piece(d_w, weights * 2), piece(d_bias, outputs * 4), piece(d_offsets, (size_t)(groups + 1) * 8)})) return PCC_E_ARG;
    Grouped a = {};
    a.x = (const u16*)d_x; a.w = (const u16*)d_w; a.bias = d_bias; a.off = d_offsets; a.y = d_y;
    a.ldx = ldx; a.ldy = ldy; a.rows = (int64_t)rows; a.groups = groups; a.in = in; a.out = out; a.act = act;
    a.y32 = y_type == PCC_FP32;
    hipStream_t st = (hipStream_t)hip_stream;
    if (narrow_forward_fits(a)) return type == PCC_BF16 ? launch_narrow_forward<Bf16>(a, st) : launch_narrow_forward<Fp16>(a, st);
    return type == PCC_BF16 ? launch_forward_tiles<Bf16>(a, st) : launch_forward_tiles<Fp16>(a, st);
}

size_t pcc_grouped_linear_grad_workspace_bytes(size_t rows, int groups, int in, int out) {
    if (!features_ok(in, out, groups, rows)) return 0;
    // enough for either kernel: which one runs depends on the tensors' places too
    size_t chunks = shared_chunks(rows, groups, (size_t)1 << weights_log2(rows, groups, in, out));
    if (in <= 192 && out <= 192) {
        Grouped a = {};
        a.rows = (int64_t)rows;
        a.groups = groups;
        backward_chunks(a);
        chunks = std::max(chunks, shared_chunks(rows, groups, (size_t)a.mult << a.log2));
    }
    return chunks * partial_values(in, out) * sizeof(float);
}

int pcc_grouped_linear_grad(const void* d_dz, size_t lddz, const void* d_x, size_t ldx, const void* d_w, const int64_t* d_offsets,
                            int groups, size_t rows, int in, int out, int type, int x_act, void* d_dx, size_t lddx, float* d_dw,
                            float* d_db, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if ((rows && (!d_dz || !d_x)) || !d_offsets || (rows && !d_dx && !d_dw) || (d_dx && !d_w) || (d_db && !d_dw)) return PCC_E_ARG;
    if (!features_ok(in, out, groups, rows) || !ld_ok(lddz, out) || !ld_ok(ldx, in) || (d_dx && !ld_ok(lddx, in))) return PCC_E_ARG;
    if ((type != PCC_BF16 && type != PCC_FP16) || x_act < PCC_ACT_RELU || x_act > PCC_ACT_NONE) return PCC_E_ARG;
    if (!aligned(d_dz, 2) || !aligned(d_x, 2) || !aligned(d_w, 2) || !aligned(d_offsets, 8) || !aligned(d_dx, 2) || !aligned(d_dw, 4) ||
        !aligned(d_db, 4)) return PCC_E_ARG;
    const size_t need = d_dw ? pcc_grouped_linear_grad_workspace_bytes(rows, groups, in, out) : 0;
    if (need && (!d_workspace || workspace_bytes < need)) return PCC_E_SCRATCH;
    if (need && !aligned(d_workspace, 16)) return PCC_E_ARG;
    const size_t weights = (size_t)groups * in * out, outputs = (size_t)groups * out;
    const Span dz = {d_dz, rows, lddz * 2, (size_t)out * 2}, x = {d_x, rows, ldx * 2, (size_t)in * 2}, w = piece(d_w, weights * 2),
               offsets = piece(d_offsets, (size_t)(groups + 1) * 8), dx = {d_dx, rows, lddx * 2, (size_t)in * 2}, dw = piece(d_dw, weights * 4),
               db = piece(d_db, outputs * 4), space = piece(d_workspace, need);
    if (overlap(dx, {dz, x, w, offsets, dw, db, space}) || overlap(dw, {dz, x, w, offsets, db, space}) || overlap(db, {dz, x, w, offsets, space}) ||
        overlap(space, {dz, x, w, offsets})) return PCC_E_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    Grouped a = {};
    a.x = (const u16*)d_x; a.w = (const u16*)d_w; a.dz = (const u16*)d_dz; a.off = d_offsets; a.y = d_dx; a.dw = d_dw; a.db = d_db;
    a.ldx = ldx; a.lddz = lddz; a.ldy = lddx; a.rows = (int64_t)rows; a.groups = groups; a.in = in; a.out = out; a.act = x_act;
    a.partial = (float*)d_workspace;
    a.shared_max = (uint32_t)std::min<size_t>(need / (partial_values(in, out) * sizeof(float)), 0xFFFFFFFFu);
    if (narrow_backward_fits(a)) {
        const int rc = type == PCC_BF16 ? launch_narrow_backward<Bf16>(a, st) : launch_narrow_backward<Fp16>(a, st);
        if (rc != PCC_OK) return rc;
    } else {
        if (d_dx && rows) {
            const int rc = type == PCC_BF16 ? launch_tiles<Bf16, kBackward>(a, st) : launch_tiles<Fp16, kBackward>(a, st);
            if (rc != PCC_OK) return rc;
        }
        if (!d_dw) return PCC_OK;
        a.log2 = weights_log2(rows, groups, in, out);
        const int rc = type == PCC_BF16 ? launch_tiles<Bf16, kWeights>(a, st) : launch_tiles<Fp16, kWeights>(a, st);
        if (rc != PCC_OK) return rc;
    }
    if (rows <= (size_t)a.mult << a.log2) return PCC_OK;        // no group can have two chunks
    const size_t parts = (partial_values(in, out) + 63) / 64;
    return launch([&] {
        hipLaunchKernelGGL(grouped_reduce_kernel, dim3((uint32_t)std::min<size_t>(parts, std::max(4, 4096 / groups)), groups), dim3(256), 0, st, a);
    });
}

int pcc_mixture_loss(const float* d_params, size_t ldp, const uint8_t* d_rgb, const float* d_weight, size_t count, int K, int dist,
                     float scale, float* d_bits, void* d_grad, int grad_type, size_t ldg, void* hip_stream) {
    if ((count && (!d_params || !d_rgb || (!d_bits && !d_grad))) || (K != 3 && K != 5 && K != 7) || (dist != 0 && dist != 1)) return PCC_E_ARG;
    if (!ld_ok(ldp, 12 * K) || (d_grad && (!ld_ok(ldg, 12 * K) || grad_type < PCC_BF16 || grad_type > PCC_FP32))) return PCC_E_ARG;
    if (!aligned(d_params, 4) || !aligned(d_weight, 4) || !aligned(d_bits, 4) || (d_grad && !aligned(d_grad, size_of(grad_type)))) return PCC_E_ARG;
    if (count == 0) return PCC_OK;
    const size_t length = (size_t)12 * K;
    const Span params = {d_params, count, ldp * 4, length * 4}, rgb = piece(d_rgb, count * 3), weight = piece(d_weight, count * 4), bits = piece(d_bits, count * 4),
               grad = {d_grad, count, ldg * size_of(grad_type), length * size_of(grad_type)};
    const bool in_place = d_grad == d_params && grad_type == PCC_FP32 && ldg == ldp;
    if (overlap(bits, {params, rgb, weight, grad}) || overlap(grad, {rgb, weight}) || (!in_place && overlap(grad, params))) return PCC_E_ARG;
    const size_t blocks = (count + 64 * kLossWaves - 1) / (64 * kLossWaves), lds = (size_t)kLossWaves * 64 * 12 * K * sizeof(float);
    if (!launchable(blocks, 64 * kLossWaves)) return PCC_E_ARG;
    auto go = [&](auto kernel) {
        if (!allow_lds(kernel, lds)) { (void)hipGetLastError(); return PCC_E_HIP; }
        return launch([&] {
            hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(64 * kLossWaves), lds, (hipStream_t)hip_stream, d_params, ldp, d_rgb, d_weight, count, scale,
                               d_bits, d_grad, ldg);
        });
    };
    auto with_type = [&](auto k, auto f) {
        constexpr int N = decltype(k)::value, F = decltype(f)::value;
        const int type = d_grad ? grad_type : PCC_FP32;
        return type == PCC_BF16 ? go(mixture_loss_kernel<N, F, PCC_BF16>) : type == PCC_FP16 ? go(mixture_loss_kernel<N, F, PCC_FP16>) : go(mixture_loss_kernel<N, F, PCC_FP32>);
    };
    auto with_dist = [&](auto k) { return dist == 0 ? with_type(k, std::integral_constant<int, 0>{}) : with_type(k, std::integral_constant<int, 1>{}); };
    return K == 3 ? with_dist(std::integral_constant<int, 3>{}) : K == 5 ? with_dist(std::integral_constant<int, 5>{}) : with_dist(std::integral_constant<int, 7>{});
}

int pcc_adamw_create(pcc_adamw** out, const pcc_adamw_tensor* h_tensors, int count, int grad_type, int copy_type, int state_bits,
                     int hip_device) {
    if (!out) return PCC_E_ARG;
    *out = nullptr;
    if (!h_tensors || count < 1 || grad_type < PCC_BF16 || grad_type > PCC_FP32 || (copy_type != PCC_BF16 && copy_type != PCC_FP16) ||
        (state_bits != 8 && state_bits != 32)) return PCC_E_ARG;
    const size_t state = (size_t)state_bits / 8;
    uint64_t elements = 0, pieces = 0;
    for (int i = 0; i < count; ++i) {
        const pcc_adamw_tensor& s = h_tensors[i];
        if (s.n == 0) continue;
        if (!s.d_param || !s.d_grad || !s.d_m || !s.d_v || (state_bits == 8 && (!s.d_m_scale || !s.d_v_scale))) return PCC_E_ARG;
        if (!aligned(s.d_param, 4) || !aligned(s.d_grad, size_of(grad_type)) || !aligned(s.d_copy, 2) || !aligned(s.d_m, state) || !aligned(s.d_v, state) ||
            (state_bits == 8 && (!aligned(s.d_m_scale, 4) || !aligned(s.d_v_scale, 4)))) return PCC_E_ARG;
        if (s.n > (size_t)1 << 40) return PCC_E_ARG;
        elements += s.n;
    }
    const int per_wave = piece_blocks(elements);
    const uint64_t piece = piece_elements(per_wave);
    for (int i = 0; i < count; ++i) pieces += (h_tensors[i].n + piece - 1) / piece;
    if (pieces > 0x7FFFFFFFull) return PCC_E_ARG;
    std::vector<uint8_t> table;
    const size_t at_pieces = 64 + (size_t)count * sizeof(AdamwTensor);
    try {
        table.assign(at_pieces + (size_t)pieces * sizeof(AdamwPiece), 0);
        // what a step writes is written once: a tensor that is listed twice, or shares bytes with another, has no result
        std::vector<std::pair<uintptr_t, uintptr_t>> written;
        auto add = [&](const void* p, size_t bytes) { if (p && bytes) written.emplace_back((uintptr_t)p, (uintptr_t)p + bytes); };
        for (int i = 0; i < count; ++i) {
            const pcc_adamw_tensor& s = h_tensors[i];
            const size_t scales = state_bits == 8 ? (s.n + kStateBlock - 1) / kStateBlock * sizeof(float) : 0;
            add(s.d_param, s.n * 4);
            add(s.d_copy, s.n * 2);
            add(s.d_m, s.n * state);
            add(s.d_v, s.n * state);
            add(s.d_m_scale, scales);
            add(s.d_v_scale, scales);
        }
        std::sort(written.begin(), written.end());
        for (size_t i = 1; i < written.size(); ++i)
            if (written[i].first < written[i - 1].second) return PCC_E_ARG;
        // nor may a gradient lie where a step writes, but for its own parameter's place, element by element
        for (int i = 0; i < count; ++i) {
            const pcc_adamw_tensor& s = h_tensors[i];
            if (s.n == 0 || (grad_type == PCC_FP32 && s.d_grad == s.d_param)) continue;
            const uintptr_t lo = (uintptr_t)s.d_grad, hi = lo + s.n * size_of(grad_type);
            const auto next = std::lower_bound(written.begin(), written.end(), std::make_pair(hi, (uintptr_t)0));  // the first that begins behind it
            if (next != written.begin() && std::prev(next)->second > lo) return PCC_E_ARG;
        }
    } catch (const std::bad_alloc&) {
        return PCC_E_INTERNAL;
    }
    AdamwTensor* tensors = reinterpret_cast<AdamwTensor*>(table.data() + 64);
    AdamwPiece* list = reinterpret_cast<AdamwPiece*>(table.data() + at_pieces);
    for (int i = 0; i < count; ++i) {
        const pcc_adamw_tensor& s = h_tensors[i];
        tensors[i] = {s.d_param, s.d_grad, (u16*)s.d_copy, s.d_m, s.d_v, s.d_m_scale, s.d_v_scale, s.n,
                      aligned(s.d_param, 16) && aligned(s.d_grad, 4 * size_of(grad_type)) && aligned(s.d_copy, 8) && aligned(s.d_m, 4 * state) && aligned(s.d_v, 4 * state), 0};
        for (size_t k = 0; k * piece < s.n; ++k) *list++ = {(uint32_t)i, (uint32_t)k};
    }
    DeviceGuard guard(hip_device);
    if (!guard.ok) { (void)hipGetLastError(); return PCC_E_HIP; }
    pcc_adamw* plan = new (std::nothrow) pcc_adamw();
    if (!plan) return PCC_E_INTERNAL;
    plan->device = hip_device;
    plan->grad_type = grad_type;
    plan->copy_type = copy_type;
    plan->state_bits = state_bits;
    plan->n_pieces = (uint32_t)pieces;
    plan->piece_blocks = per_wave;
    if (hipMalloc((void**)&plan->d_table, table.size()) != hipSuccess ||
        hipMemcpy(plan->d_table, table.data(), table.size(), hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        pcc_adamw_destroy(plan);
        return PCC_E_HIP;
    }
    plan->d_tensors = reinterpret_cast<AdamwTensor*>(plan->d_table + 64);
    plan->d_pieces = reinterpret_cast<AdamwPiece*>(plan->d_table + at_pieces);
    *out = plan;
    return PCC_OK;
}

void pcc_adamw_destroy(pcc_adamw* plan) {
    if (!plan) return;
    DeviceGuard guard(plan->device);
    if (plan->d_table) (void)hipFree(plan->d_table);
    delete plan;
}

int pcc_adamw_step(pcc_adamw* plan, const pcc_adamw_hyper* h, int64_t* d_step, void* hip_stream) {
    if (!plan || !h || !d_step || !aligned(d_step, 8) || !aligned(h->d_lr, 4)) return PCC_E_ARG;
    // (an eps below fp32's normal numbers has an infinite reciprocal, and a moment of 0 would make it NaN)
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0 && (h->eps == 0.0 || h->eps >= 0x1p-126))) return PCC_E_ARG;
    DeviceGuard guard(plan->device);
    if (!guard.ok) return PCC_E_HIP;
    AdamwArgs a = {};
    a.tensors = plan->d_tensors;
    a.pieces = plan->d_pieces;
    a.n_pieces = plan->n_pieces;
    a.piece_blocks = plan->piece_blocks;
    AdamwRates* rates = reinterpret_cast<AdamwRates*>(plan->d_table);
    a.rates = rates;
    a.b1 = (float)h->beta1; a.rest1 = (float)(1.0 - h->beta1); a.b2 = (float)h->beta2; a.rest2 = (float)(1.0 - h->beta2); a.eps = (float)h->eps;
    const int rc = launch([&] {
        hipLaunchKernelGGL(adamw_prepare_kernel, dim3(1), dim3(1), 0, (hipStream_t)hip_stream, d_step, h->d_lr, h->lr, h->beta1, h->beta2, h->weight_decay, rates);
    });
    if (rc != PCC_OK || plan->n_pieces == 0) return rc;
    // us for 33.5 million elements with 1,024, 2,048 and 4,096 workgroups: 32 bits 205, 207, 206, 8 bits 175, 172, 167
    const uint32_t blocks = std::min<uint32_t>(plan->n_pieces, plan->state_bits == 8 ? 4096 : 1024);
    auto go = [&](auto kernel) { return launch([&] { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kAdamwThreads), 0, (hipStream_t)hip_stream, a); }); };
    auto with_grad = [&](auto copy, auto bits) {
        constexpr int C = decltype(copy)::value, B = decltype(bits)::value;
        return plan->grad_type == PCC_FP32 ? go(adamw_kernel<PCC_FP32, C, B>) : plan->grad_type == PCC_BF16 ? go(adamw_kernel<PCC_BF16, C, B>) : go(adamw_kernel<PCC_FP16, C, B>);
    };
    auto with_copy = [&](auto bits) {
        return plan->copy_type == PCC_BF16 ? with_grad(std::integral_constant<int, PCC_BF16>{}, bits) : with_grad(std::integral_constant<int, PCC_FP16>{}, bits);
    };
    return plan->state_bits == 8 ? with_copy(std::integral_constant<int, 8>{}) : with_copy(std::integral_constant<int, 32>{});
}

}  // extern "C"
