// Launches of the head kernels (adasd_head.cuh).
#include "adasd_head.cuh"
#include "adasd_launch.cuh"
#include "adasd_score_types.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace adasd {
namespace {

// What a call keeps in its scratch.  (Of many rows statistics of the tiles and a piece of the gradient are never needed at once: they share their place.)
struct Layout {
    int n_pad, D8, Dp, tiles;                        // tiles: 256 columns of the vocabulary
    int columns, halves, res_halves;                 // columns of a tile of the statistics; as in HeadTiles
    int piece, splits, planes;                       // columns of a piece; parts that grad_h's sums along them are cut into; planes of G
    long long z_stride;
    size_t h, index, tok, n_active, ticket, zx, coef, res, z, part, big, acc, total;
};

// Tiles of pairs where the rows fill more than one CTA's.
inline bool in_pairs(int n_rows) { return n_rows > kHgM; }

// Columns of a tile of the statistics where a CTA works on its own, its time is that of reading w and there are few tiles: those with which the fullest CTA has
// least to read.  (V = 32000 on 148 SMs: 125 tiles of 256 or 143 of 224.)
int tile_columns(int V, int sm_count) {
    int best = kHgN;
    long long least = -1;
    for (int c = kHgN; c >= 160; c -= 32) {
        const long long tiles = (V + c - 1) / c, t = (tiles + sm_count - 1) / sm_count * (c + 16);
        if (least < 0 || t < least) {
            least = t;
            best = c;
        }
    }
    return best;
}
// Parts that grad_h's sums over a piece are cut into: as many as make the launch end first by this estimate, in steps along K: a step of the products of a
// CTA (0.3 us) against what a part's fp32 sums cost to write and read.  The mean of calls with and without grad_w: one number for both, so that grad_h is
// the same in both to the bit.
int splits_of(int n_rows, int n_pad, int piece, int D, int planes, int m, int sm_count) {
    const double units = sm_count * (double)kHgM / m, steps = piece / (double)kHgK, nt = (D + kHgN - 1) / kHgN, tiles = (double)(n_pad / m) * nt;
    const double w = (piece / (double)m) * nt * ((planes == 2 ? 2 : n_pad / kHgK) + 3);
    const double part = (double)std::max(n_rows, 1) * planes * D * 8.0 / 6.5e6 / 0.3;
    const int fewest = (piece + kHgVocabPart - 1) / kHgVocabPart;
    int best = fewest;
    double least = 0.0;
    const int most = (int)std::max<size_t>(1, std::min<size_t>(128, ((size_t)64 << 20) / ((size_t)n_pad * D * 4)));      // (64 MB)
    for (int s = fewest; s <= most && steps / s >= 4; ++s) {
        const double len = std::ceil(steps / s), alone = std::ceil(tiles * s / units) * len;
        const double t = 0.5 * (alone + std::max((tiles * s * len + w) / units, len)) + s * part;
        if (s == fewest || t < least) {
            least = t;
            best = s;
        }
    }
    return best;
}

// What a logit loses, in the mean, of its size: see the head of adasd_head.cuh.  part: steps of a part.
double sum_loss(int D, int part) {
    const double all = (D + 15) / 16, full = part * (kHgK / 16), parts = std::floor(all / full), rest = all - parts * full;
    return 1.2e-8 * (parts * full * full + rest * rest) / all;
}
constexpr size_t kPieceBytes = (size_t)256 << 20;

Layout layout_of(int n_rows, int V, int D, bool gradient, int sm_count) {
    Layout L;
    const int m = in_pairs(n_rows) ? 2 * kHgM : kHgM;
    L.n_pad = (std::max(n_rows, 1) + m - 1) / m * m;
    L.D8 = (D + 7) / 8 * 8;
    L.Dp = (D + 63) / 64 * 64;
    L.tiles = (V + kHgN - 1) / kHgN;
    L.columns = in_pairs(n_rows) ? kHgN : tile_columns(V, sm_count);
    L.halves = (V + L.columns - 1) / L.columns * 2;
    L.res_halves = (V + kHgHalf - 1) / kHgHalf;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 1023) & ~(size_t)1023;
        return here;
    };
    L.n_active = take(16);
    L.ticket = take(16);
    L.index = take((size_t)L.n_pad * 4);
    L.tok = take((size_t)L.n_pad * 4);
    L.zx = take((size_t)L.n_pad * 4);
    L.coef = take(gradient ? (size_t)L.n_pad * sizeof(HeadCoef) : 0);
    L.h = take((size_t)L.n_pad * L.D8 * 2);
    const size_t part = (size_t)L.n_pad * L.halves * sizeof(float4);
    L.planes = n_rows <= kHgPlaneRows ? 2 : 1;
    L.res = take(gradient && L.planes == 1 ? (size_t)L.n_pad * L.res_halves * sizeof(float) : 0);
    // (up to 128 rows: the logits, for the gradient that is made of them)
    L.z_stride = (V + 63) / 64 * 64;
    L.z = take(gradient && n_rows <= kHgM ? (size_t)n_rows * L.z_stride * sizeof(float) : 0);
    L.piece = L.splits = 0;
    size_t g = 0, acc = 0;
    if (gradient) {
        const long long fit = (long long)(kPieceBytes / (2 * (size_t)L.n_pad)) / kHgN * kHgN;
        L.piece = (int)std::min<long long>((long long)L.tiles * kHgN, std::max<long long>(fit, 2048));
        L.splits = splits_of(n_rows, L.n_pad, L.piece, D, L.planes, m, sm_count);
        g = (size_t)L.n_pad * L.piece * 2;
        acc = (size_t)L.splits * L.n_pad * L.Dp * 4;
    }
    const bool apart = gradient && n_rows <= kHgM;   // (head_g_kernel reads the one while it writes the other)
    L.part = take(apart ? part : 0);
    L.big = take(std::max(apart ? 0 : part, g));
    if (!apart) L.part = L.big;
    L.acc = take(acc);
    L.total = at;
    return L;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}
// Map of a row-major bf16 matrix in boxes of 64 columns.
int make_map(CUtensorMap* map, const void* base, long long rows, long long columns, long long stride, int box_rows) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return ADASD_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? ADASD_OK
               : ADASD_ERR_CUDA;
}

template <int TILE, int CG>
int launch_tiles(const HeadTiles& p, int sm_count, cudaStream_t stream) {
    static std::atomic<bool> allowed[64];
    int dev = 0;
    CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return ADASD_ERR_CUDA;
    if (!allowed[dev].load(std::memory_order_acquire)) {
        if (TILE != TILE_GRADS) {          // (the split of the registers counts on them)
            cudaFuncAttributes fa;
            CUDA_TRY(cudaFuncGetAttributes(&fa, head_tile_kernel<TILE, CG>));
            if (fa.numRegs < kHgLaunchRegs) return ADASD_ERR_CUDA;
        }
        CUDA_TRY(cudaFuncSetAttribute(head_tile_kernel<TILE, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, HeadStage<TILE, CG>::kAll));
        allowed[dev].store(true, std::memory_order_release);
    }
    return launch_pdl(head_tile_kernel<TILE, CG>, sm_count / CG * CG, kHgThreads, HeadStage<TILE, CG>::kAll, CG, stream, p);
}
template <int TILE>
int launch_tiles(const HeadTiles& p, bool pairs, int sm_count, cudaStream_t stream) {
    return pairs ? launch_tiles<TILE, 2>(p, sm_count, stream) : launch_tiles<TILE, 1>(p, sm_count, stream);
}
}  // namespace

size_t head_scratch_need(int n_rows, int V, int D, bool gradient, int sm_count) { return layout_of(n_rows, V, D, gradient, sm_count).total; }

// A call's need does not grow with its rows throughout: up to a tile of them there are logits and statistics apart, and the parts of grad_h and the piece change
// with every pair's tile.  Beyond a tile it hangs on the padded rows and the parts, and of counts with the same padded rows the first has the most parts (what a part
// costs grows with the rows, what it saves does not): one count for each is looked at.
size_t head_scratch_bytes(int n_rows, int V, int D, bool gradient, int sm_count) {
    size_t most = 0;
    for (int n = 0; n <= n_rows; n += n <= kHgM ? 1 : n == kHgM + 1 ? kHgM : 2 * kHgM) most = std::max(most, head_scratch_need(n, V, D, gradient, sm_count));
    return most;
}

int launch_head(const HeadCall& c, cudaStream_t stream) {
    const bool gradient = c.gradient();
    const Layout L = layout_of(c.n_rows, c.V, c.D, gradient, c.sm_count);
    char* s = static_cast<char*>(c.scratch);

    HeadRows r;
    memset(&r, 0, sizeof(r));
    r.c = c;
    r.h = reinterpret_cast<uint16_t*>(s + L.h);
    r.D8 = L.D8;
    r.halves = L.halves;
    r.res_halves = L.res_halves;
    r.planes = L.planes;
    r.res = c.grad_h && L.planes == 1 ? reinterpret_cast<float*>(s + L.res) : nullptr;
    r.index = reinterpret_cast<int32_t*>(s + L.index);
    r.tok = reinterpret_cast<int32_t*>(s + L.tok);
    r.n_active = reinterpret_cast<int32_t*>(s + L.n_active);
    r.zx = reinterpret_cast<float*>(s + L.zx);
    r.coef = gradient ? reinterpret_cast<HeadCoef*>(s + L.coef) : nullptr;
    r.part = reinterpret_cast<const float4*>(s + L.part);
    r.acc = reinterpret_cast<const float*>(s + L.acc);
    r.acc_slot = (long long)L.n_pad * L.Dp;
    r.Dp = L.Dp;
    r.splits = L.splits;
    const double whole = 1.0 + sum_loss(c.D, in_pairs(c.n_rows) ? kHgPart<2> : kHgPart<1>);
    r.c1 = (float)(1.4426950408889634 / (double)c.temperature * whole);
    r.inv_Tz = whole / (double)c.temperature;
    r.inv_T = 1.0 / (double)c.temperature;
    r.rows = c.n_rows <= 2048 ? kHrThreads / 32 : kHrRows;

    HeadTiles t;
    memset(&t, 0, sizeof(t));
    // One tile's rows: nothing is gained by putting the rows that count together.
    const bool as_they_lie = c.n_rows <= kHgM && (reinterpret_cast<uintptr_t>(c.hidden) & 15u) == 0 && c.h_stride % 8 == 0;
    // A CTA on its own brings in no more than the rows there are, in eights.  (Rows beyond a matrix cost a load more than those within: 128 of them for one row
    // made 36 us of 30.)
    const bool pairs = in_pairs(c.n_rows);
    t.h_boxes = c.n_rows > 64 ? 2 : 1;
    t.h_box_rows = ((c.n_rows + t.h_boxes - 1) / t.h_boxes + 7) / 8 * 8;
    const int box_rows = pairs ? 64 : t.h_box_rows;
    // The losses' total by the last row's CTA, unless there are so many that it would take long.
    r.ticket = c.loss && c.n_rows <= 16384 ? reinterpret_cast<uint32_t*>(s + L.ticket) : nullptr;
    if (as_they_lie) {
        r.n_active = nullptr;
        r.index = nullptr;
        r.tok = const_cast<int32_t*>(c.tok);
        if (int rc = make_map(&t.h, c.hidden, c.n_rows, c.D, c.h_stride, box_rows)) return rc;
    } else {
        if (int rc = make_map(&t.h, r.h, L.n_pad, c.D, L.D8, box_rows)) return rc;
        if (int rc = launch_pdl(head_rows_kernel, (c.n_rows + r.rows - 1) / r.rows, kHrThreads, 0, 0, stream, r)) return rc;
    }
    if (int rc = make_map(&t.w, c.weight, c.V, c.D, c.w_stride, pairs ? 64 : L.columns / 4)) return rc;
    t.D = c.D;
    t.V = c.V;
    t.vn = c.V;
    t.n_active = r.n_active;
    t.n_rows = c.n_rows;
    t.c1 = r.c1;
    t.columns = L.columns;
    t.entropy = c.H != nullptr;
    t.part = reinterpret_cast<float4*>(s + L.part);
    t.halves = L.halves;
    t.res_halves = L.res_halves;
    t.planes = L.planes;
    t.res = const_cast<float*>(r.res);
    t.zx = r.zx;
    t.tok = r.tok;
    t.coef = r.coef;
    t.acc = reinterpret_cast<float*>(s + L.acc);
    t.acc_slot = r.acc_slot;
    t.Dp = L.Dp;
    t.splits = r.splits;
    t.want_w = c.grad_w != nullptr;
    t.want_h = c.grad_h != nullptr;
    t.watch = c.op == HEAD_GIVEN;
    t.status = c.status;
    const bool from_logits = as_they_lie && gradient && c.op == HEAD_CE;
    const int rows16 = (c.n_rows + 15) / 16 * 16;
    if (as_they_lie) {
        t.ticket = r.ticket;
        t.rows16 = rows16;
        if (from_logits) {
            t.z = reinterpret_cast<float*>(s + L.z);
            r.z = t.z;
            r.z_stride = t.z_stride = L.z_stride;
            r.g = reinterpret_cast<uint16_t*>(s + L.big);
            r.piece = L.piece;
        }
    }
    if (c.op != HEAD_GIVEN)
        if (int rc = launch_tiles<TILE_STATS>(t, pairs, c.sm_count, stream)) return rc;
    if (!from_logits && (c.op != HEAD_GIVEN || as_they_lie))
        if (int rc = launch_pdl(head_stats_kernel, as_they_lie && gradient ? rows16 : c.n_rows, kHsThreads, 0, 0, stream, r)) return rc;
    if (c.loss && !r.ticket)
        if (int rc = launch_total(c.row_loss, c.n_rows, c.loss, stream)) return rc;
    if (!gradient) return ADASD_OK;

    CUtensorMap g_out{}, gw_out{};                   // (zeros where the call has no such product)
    char* g = s + L.big;
    // (G's tiles have 256 columns; the gradients' products take boxes of 64 rows of both)
    CUtensorMap w_tile = t.w, h_tile = t.h, w_grad = t.w, h_grad = t.h;
    if (!pairs) {
        if (L.columns != kHgN)
            if (int rc = make_map(&w_tile, c.weight, c.V, c.D, c.w_stride, 64)) return rc;
        w_grad = w_tile;
        if (box_rows != 64 || as_they_lie)
            if (int rc = make_map(&h_grad, r.h, L.n_pad, c.D, L.D8, 64)) return rc;
    }
    if (int rc = make_map(&t.g, g, L.n_pad, L.piece, L.piece, 64)) return rc;
    if (L.planes == 2) {
        if (!as_they_lie) t.rows16 = kHgPlaneRows;
        if (int rc = make_map(&t.g_few, g, L.n_pad, L.piece, L.piece, t.rows16)) return rc;
        if (int rc = make_map(&t.h_few, r.h, L.n_pad, c.D, L.D8, t.rows16)) return rc;
    }
    if (!from_logits)
        if (int rc = make_map(&g_out, g, L.n_pad, L.piece, L.piece, 32)) return rc;
    if (c.grad_w)
        if (int rc = make_map(&gw_out, c.grad_w, c.V, c.D, c.gw_stride, 32)) return rc;
    for (int v0 = 0; v0 < c.V; v0 += L.piece) {
        t.v0 = v0;
        t.vn = std::min(L.piece, c.V - v0);
        t.first = v0 == 0;
        t.w = w_tile;
        t.h = h_tile;
        if (from_logits) {
            r.v0 = v0;
            r.vn = t.vn;
            // CTAs: about four for a SM
            const int width = (t.vn + kHgN - 1) / kHgN * kHgN, most = (width + kHxColumns - 1) / kHxColumns;
            const int want = std::max(1, std::min(most, (4 * c.sm_count + rows16 - 1) / rows16));
            r.columns = (most + want - 1) / want * kHxColumns;
            const int parts = (width + r.columns - 1) / r.columns;
            if (int rc = launch_pdl(head_g_kernel, rows16 * parts, kHsThreads, 0, 0, stream, r)) return rc;
        } else {
            t.out = g_out;
            if (int rc = launch_tiles<TILE_G>(t, pairs, c.sm_count, stream)) return rc;
        }
        t.w = w_grad;
        t.h = h_grad;
        t.out = gw_out;
        // (in parts 350 us instead of 341 for 1000 rows of 50257 at dim 1000; no difference from 2048 rows on)
        if (int rc = c.n_rows > kHgRowsPart ? launch_tiles<TILE_LONG, 2>(t, c.sm_count, stream) : launch_tiles<TILE_GRADS>(t, pairs, c.sm_count, stream)) return rc;
    }
    if (!c.grad_h) return ADASD_OK;
    const int columns = kHrThreads / head_groups(r.splits * r.planes) * 8;
    return launch_pdl(head_grad_rows_kernel, c.n_rows * ((c.D + columns - 1) / columns), kHrThreads, 0, 0, stream, r);
}

}  // namespace adasd
