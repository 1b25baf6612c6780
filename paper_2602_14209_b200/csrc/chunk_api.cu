// Host side of the calls on packed chunks of new tokens: rotary positions, cache writes, the 8- and 4-bit caches, chunk attention.
#include <algorithm>
#include <cmath>

#include "chunk.cuh"
#include "chunk_decode.cuh"
#include "chunk_prefill.cuh"
#include "host.cuh"
#include "rope.cuh"

namespace mage {
namespace {

constexpr int kSms = 148;
constexpr int kMaxPos = 1 << 30;                      // positions and tile ends stay below 2^31

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }

// The arrays of a call's cache beside the mage_kv_t: none over 16 bits, codes and scales over 8 or 4.
template <int BITS>
struct Codes {
    chunk::CodeView<BITS> v;
    bool given;                                           // the caller passed a description
};
Codes<16> codes16() { return {{}, true}; }
Codes<8> codes_of(const mage_kv8_t *c) {
    if (!c) return {{}, false};
    return {{static_cast<uint8_t *>(c->k8), static_cast<uint8_t *>(c->v8), c->k_scale, c->v_scale}, true};
}
Codes<4> codes_of(const mage_kv4_t *c) {
    if (!c) return {{}, false};
    return {{static_cast<uint8_t *>(c->k4), static_cast<uint8_t *>(c->v4), static_cast<uint8_t *>(c->k_scale), static_cast<uint8_t *>(c->v_scale)}, true};
}

// The cache description of a chunk call: kv itself, or with the arrays of codes in the place of the 16-bit ones.
template <int BITS>
mage_status chunk_kv(const mage_kv_t *kv, const Codes<BITS> &codes, mage_kv_t *out) {
    if (!kv || !codes.given) return MAGE_ERR_INVALID_ARG;
    *out = *kv;
    if constexpr (BITS == 8) { out->k_cache = codes.v.k8; out->v_cache = codes.v.v8; }
    if constexpr (BITS == 4) { out->k_cache = codes.v.k4; out->v_cache = codes.v.v4; }
    mage_status why = MAGE_OK;
    if (!valid_kv(out, &why)) return why;
    if (out->N_max > kMaxPos) return MAGE_ERR_UNSUPPORTED;
    if (out->flags & MAGE_FLAG_SIMT_KERNELS) return MAGE_ERR_UNSUPPORTED;
    if (!aligned16(out->k_cache) || !aligned16(out->v_cache)) return MAGE_ERR_UNSUPPORTED;
    if constexpr (BITS != 16) {                           // (16 bytes of codes)
        constexpr int kEls = 128 / BITS;
        if (out->N_max > 0 && (!codes.v.k_scale || !codes.v.v_scale)) return MAGE_ERR_INVALID_ARG;
        if (out->page_size == 0 && (out->stride_n % kEls || out->stride_h % kEls || out->stride_p % kEls)) return MAGE_ERR_UNSUPPORTED;
    }
    if constexpr (BITS == 4) {
        if (!aligned16(codes.v.k_scale) || !aligned16(codes.v.v_scale)) return MAGE_ERR_UNSUPPORTED;
    }
    return MAGE_OK;
}
bool valid_chunk(const mage_chunk_t *c) { return c && c->q_start && c->n_tokens >= 0 && c->max_len >= 0 && c->max_len <= c->n_tokens; }
chunk::ChunkView chunk_view(const mage_chunk_t *c) { return {c->q_start, c->n_tokens, c->max_len}; }

// ---- attention of few rows: grid and workspace (pure functions of the description)
struct DecodePlan {
    int rows, grid;                                   // rows of a tile; CTAs
    bool split;                                       // an item may span several CTAs
    size_t off_part, bytes;
};
template <int BITS>
DecodePlan decode_plan(const mage_kv_t *kv, const mage_chunk_t *c) {
    DecodePlan pl;
    constexpr int unit = chunk::Dec<BITS>::kUnit, min_cost = chunk::Dec<BITS>::kMinCost;
    const int64_t G = kv->H_q / kv->H_kv, units = std::max(1, (kv->N_max + unit - 1) / unit);
    pl.rows = c->max_len * G <= 8 ? 8 : 16;
    const int64_t tiles = std::min<int64_t>((int64_t)kv->P * ((c->max_len * G + pl.rows - 1) / pl.rows), c->n_tokens * G / pl.rows + kv->P);
    // all CTAs that fit at once; never more than there can be runs
    const int most = kSms * (pl.rows == 8 ? chunk::Dec<BITS, 1>::kPerSm : chunk::Dec<BITS, 2>::kPerSm);
    const double runs = std::ceil((double)tiles * kv->H_kv * (double)(units + chunk::Dec<BITS>::kItemCost) / min_cost);
    pl.grid = runs < most ? std::max(1, (int)runs) : most;
    pl.split = units > 1;
    pl.off_part = align_up((size_t)pl.grid * sizeof(chunk::Split), 256);
    pl.bytes = pl.off_part + align_up((size_t)pl.grid * 2 * chunk::slot_floats(pl.rows) * sizeof(float), 256);
    return pl;
}

// ---- attention of many rows
struct PrefillPlan {
    int mt_toks, slots, grid;
    size_t off_part, bytes;
};
// Least cost of a run: a key tile.  (100 tokens behind 500, 28 + 4 heads: 19.0 us, with two tiles 21.1, three 22.6; 20 behind 4000: 19.7, 20.0, 22.7;
// 2 x 300 behind nothing: 22.2, 21.3, 22.3.)
constexpr int kPrefillMinCost = chunk::kUnitCost;
PrefillPlan prefill_plan(const mage_kv_t *kv, const mage_chunk_t *c) {
    PrefillPlan pl;
    pl.mt_toks = chunk::kPreTile / (kv->H_q / kv->H_kv);
    pl.slots = c->n_tokens / (2 * pl.mt_toks) + kv->P;
    const double total = (double)pl.slots * kv->H_kv * ((double)std::max(1, (kv->N_max + chunk::kPreTile - 1) / chunk::kPreTile) * chunk::kUnitCost + chunk::kItemCost8);
    pl.grid = total < kSms ? std::max(1, (int)total) : kSms;
    pl.off_part = align_up((size_t)pl.grid * sizeof(chunk::Split), 256);
    pl.bytes = pl.off_part + align_up((size_t)pl.grid * 2 * chunk::kPreSlot * sizeof(float), 256);
    return pl;
}
// Which kernel: rows of a problem per KV head, at most.  Up to 16, one tile of the decoding kernel, it reads a long cache at least as
// fast as the prompt kernel and starts sooner; with a second tile it reads the cache twice.  (us, decoding / prompt kernel, four rows a token.  16
// sequences of 4K to 128K, 16 bits: 4 rows 329 / 327, 16 rows 342 / 333, 32 rows 614 / 339; 8 bits: 179 / 438, 283 / 443, 539 / 451.  One
// sequence of 2048, 16 bits: 9.6 / 13.5, 11.3 / 15.1, 32 rows 11.8 / 15.2; of 16000, 8 bits: 13.6 / 19.2, 19.5 / 20.8, 21.4 / 21.1.)
// Over 4 bits two tiles, although each of them rebuilds every number: four warps an SM that rebuild them once are no faster (16 sequences of 16384, seven rows a token:
// 21 rows 100 / 104, 28 rows 100 / 106, 42 rows 137 / 111; of 1024: 26.6 / 32.8, 28.6 / 34.8, 30.7 / 34.8).
constexpr int kDecodeMaxRows = 16, kDecodeMaxRows4 = 32;
template <int BITS>
bool use_decode(const mage_kv_t *kv, const mage_chunk_t *c) {
    const int64_t G = kv->H_q / kv->H_kv;
    return kv->N_max == 0 || G > chunk::kPreTile || c->max_len * G <= (BITS == 4 ? kDecodeMaxRows4 : kDecodeMaxRows);
}

// The packed queries as (d, G heads of a group, groups, tokens): a box is one d-half of an M-tile's rows.
bool make_queries_map(CUtensorMap *m, const mage_kv_t *kv, const mage_chunk_t *c, const chunk::AttnArgs &at, int toks) {
    tc::EncodeTiledFn fn = tc::encode_fn();
    if (!fn) return false;
    const int G = kv->H_q / kv->H_kv;
    const cuuint64_t any = 16;                            // (the stride of a dimension of one is never used; it must not be 0)
    cuuint64_t dims[4] = {(cuuint64_t)kD, (cuuint64_t)G, (cuuint64_t)kv->H_kv, (cuuint64_t)c->n_tokens};
    cuuint64_t str[3] = {G > 1 ? (cuuint64_t)at.q.sh * 2 : any, kv->H_kv > 1 ? (cuuint64_t)at.q.sh * G * 2 : any, c->n_tokens > 1 ? (cuuint64_t)at.q.st * 2 : any};
    cuuint32_t box[4] = {64, (cuuint32_t)G, 1, (cuuint32_t)toks}, estr[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16 *>(at.q.p), dims, str, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The cache (or its codes, eb = 1) as a rank-4 tensor of 128-byte rows pieces, boxes of box_rows rows, 128-byte swizzle.
bool make_rows_box_map(CUtensorMap *m, const mage_kv_t *kv, const void *base, int eb, int box_rows) {
    tc::EncodeTiledFn fn = tc::encode_fn();
    if (!fn) return false;
    const cuuint64_t e = (cuuint64_t)eb;
    cuuint64_t dims[4], str[3];
    dims[0] = kD;
    if (kv->page_size == 0) {
        dims[1] = kv->N_max; dims[2] = kv->H_kv; dims[3] = kv->P;
        str[0] = kv->stride_n * e;
        str[1] = (kv->H_kv > 1 ? kv->stride_h : kD) * e;      // (the stride of a dimension of one is never used; it must not be 0)
        str[2] = (kv->P > 1 ? kv->stride_p : kD) * e;
    } else {
        dims[1] = kv->page_size; dims[2] = kv->H_kv; dims[3] = kv->num_pages;
        str[0] = kD * e; str[1] = kv->page_size * str[0]; str[2] = kv->H_kv * str[1];
    }
    cuuint32_t box[4] = {eb == 1 ? 128u : 64u, (cuuint32_t)box_rows, 1, 1}, estr[4] = {1, 1, 1, 1};
    return fn(m, eb == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, str, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Attention of prompts over a 4-bit cache: written out in 16 bits first where that pays and the caller's workspace has the room.
// A key tile rebuilt inside the kernel takes a quarter of a row tile's time; written out it costs 84 KB of traffic once.  (us, rebuilt / written out, 28 + 4
// heads.  Row tiles a problem 114, behind 32768: 2061 / 1656;  31 (32 + 8 heads), behind 16384: 606 / 499;  8, behind 4000: 53.9 / 51.5;  4, behind 20000: 83.4 / 81.9, 16
// problems behind 8000: 365 / 346;  2.8, behind 4000: 42.5 / 42.5, 24 problems of 1 to 700 tokens: 114 / 109;  2, behind 20000: 56.1 / 59.1, 16 problems behind
// 16384: 318 / 372;  1: 178 / 256.)
constexpr int kStageHalfTiles = 5;                        // row tiles a problem, on average, in halves
constexpr size_t kStageMost = (size_t)1 << 30;            // bytes: problems are taken at N_max rows each, and large batches are left alone
size_t stage_bytes(const mage_kv_t *kv, const mage_chunk_t *c) {      // of K or V; 0: not staged
    if (use_decode<4>(kv, c) || (int64_t)c->n_tokens < (int64_t)kStageHalfTiles * (chunk::kPreTile / (kv->H_q / kv->H_kv)) * kv->P) return 0;
    const size_t n = (size_t)kv->P * kv->H_kv * kv->N_max * kD * 2;
    return 2 * n <= kStageMost ? align_up(n, 256) : 0;
}

template <int BITS, bool STAGED = false>
mage_status launch_prefill(const mage_kv_t *kv, const Codes<BITS> &codes, const mage_chunk_t *c, const chunk::AttnArgs &at, void *ws, unsigned *status, cudaStream_t st) {
    const PrefillPlan pl = prefill_plan(kv, c);
    chunk::PreMaps maps;
    maps.box_rows = STAGED || kv->page_size == 0 || kv->page_size >= chunk::kPreTile ? chunk::kPreTile : kv->page_size;
    maps.test_stall = (kv->flags & MAGE_FLAG_TEST_STALL) ? 1 : 0;
    if (tc::encode_fn() == nullptr) return MAGE_ERR_CUDA;
    mage_kv_t rows = *kv;                                 // what the tiles are read from
    if constexpr (STAGED) {                               // (kv: the cache of codes; its copy lies behind the workspace's other parts)
        const size_t n = stage_bytes(kv, c);
        uint8_t *copy = static_cast<uint8_t *>(ws) + pl.bytes;
        rows.k_cache = copy; rows.v_cache = copy + n;
        rows.page_size = 0;
        rows.stride_n = kD; rows.stride_h = (int64_t)kv->N_max * kD; rows.stride_p = kv->H_kv * rows.stride_h;
    }
    if (BITS != 4 && (!make_rows_box_map(&maps.k, &rows, rows.k_cache, BITS / 8, maps.box_rows) || !make_rows_box_map(&maps.v, &rows, rows.v_cache, BITS / 8, maps.box_rows)))
        return MAGE_ERR_UNSUPPORTED;
    if (BITS == 8) maps.q = maps.k;                       // (never used: the queries are coded by plain loads)
    else if (!make_queries_map(&maps.q, kv, c, at, pl.mt_toks)) return MAGE_ERR_UNSUPPORTED;
    if (BITS == 4) maps.k = maps.v = maps.q;              // (never used: codes are fetched by cp.async)
    auto kern = chunk::prefill_kernel<BITS, STAGED>;
    constexpr size_t smem = chunk::Pre<BITS>::kSmem;
    static_assert(smem <= 232448, "");
    if (opt_in_smem(kern, smem) != MAGE_OK) return MAGE_ERR_CUDA;
    const chunk::PreGrid pg = {pl.slots, pl.mt_toks, kPrefillMinCost, static_cast<chunk::Split *>(ws), reinterpret_cast<float *>(static_cast<char *>(ws) + pl.off_part)};
    const KvView view = make_view(kv);
    launch_pdl(kern, dim3(pl.grid), dim3(chunk::Pre<BITS>::kThreads), smem, st, maps, view, codes.v, chunk_view(c), at, pg, status);
    if (launch_check() != MAGE_OK) return MAGE_ERR_CUDA;
    if (pl.grid > 1) {
        launch_pdl(chunk::combine_kernel<chunk::kPreRows>, dim3(pl.grid, chunk::kMergeY), dim3(128), 0, st, at, (const chunk::Split *)pg.split, (const float *)pg.part, kv->H_q,
                   kv->H_q / kv->H_kv, pl.mt_toks);
        return launch_check();
    }
    return MAGE_OK;
}
mage_status launch_prefill_staged(const mage_kv_t *kv, const Codes<4> &codes, const mage_chunk_t *c, const chunk::AttnArgs &at, void *ws, unsigned *status, cudaStream_t st) {
    __nv_bfloat16 *copy = reinterpret_cast<__nv_bfloat16 *>(static_cast<uint8_t *>(ws) + prefill_plan(kv, c).bytes);
    launch_pdl(chunk::read_kernel<4, true>, dim3((kv->N_max + 8 * chunk::kStageTurns * chunk::kReadRows - 1) / (8 * chunk::kStageTurns * chunk::kReadRows), kv->P * kv->H_kv), dim3(256), 0, st, make_view(kv), codes.v,
               chunk_view(c), (const int *)nullptr, (const int *)nullptr, 0, kv->N_max, copy, copy + stage_bytes(kv, c) / 2, status);
    if (launch_check() != MAGE_OK) return MAGE_ERR_CUDA;
    return launch_prefill<16, true>(kv, codes16(), c, at, ws, status, st);
}

template <int BITS, int NQ>
mage_status launch_decode(const mage_kv_t *kv, const Codes<BITS> &codes, const mage_chunk_t *c, const chunk::AttnArgs &at, const DecodePlan &pl, void *ws, unsigned *status,
                          cudaStream_t st) {
    auto kern = chunk::decode_kernel<BITS, NQ>;
    constexpr size_t smem = chunk::Dec<BITS, NQ>::kSmem;
    if (opt_in_smem(kern, smem) != MAGE_OK) return MAGE_ERR_CUDA;
    chunk::Split *split = pl.split ? static_cast<chunk::Split *>(ws) : nullptr;
    float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + pl.off_part);
    launch_pdl(kern, dim3(pl.grid), dim3(chunk::kDecWarps * 32), smem, st, make_view(kv), codes.v, chunk_view(c), at, split, part, status);
    if (launch_check() != MAGE_OK) return MAGE_ERR_CUDA;
    if (pl.split && pl.grid > 1) {
        launch_pdl(chunk::combine_kernel<8 * NQ>, dim3(pl.grid, 8 * NQ), dim3(128), 0, st, at, (const chunk::Split *)split, (const float *)part, kv->H_q, kv->H_q / kv->H_kv, 0);
        return launch_check();
    }
    return MAGE_OK;
}

template <int BITS>
mage_status chunk_attn(const mage_kv_t *kv_in, const Codes<BITS> &codes, const mage_chunk_t *c, const void *q, int64_t stride_t, int64_t stride_h,
                       int32_t mask_block, float sm_scale, void *out, float *lse, void *workspace, size_t workspace_bytes, uint32_t *dev_status, void *stream) {
    mage_kv_t kv;
    const mage_status s = chunk_kv(kv_in, codes, &kv);
    if (s != MAGE_OK) return s;
    if (!valid_chunk(c)) return MAGE_ERR_INVALID_ARG;
    if (c->n_tokens == 0) return MAGE_OK;                 // (max_len 0 is a bound like others: ranges that are not empty are reported)
    if (!q || !out || !workspace || mask_block < 0 || !(sm_scale > 0.f) || !std::isfinite(sm_scale * kLog2e) || !stride_ok(stride_t) || !stride_ok(stride_h)) return MAGE_ERR_INVALID_ARG;
    if (BITS == 4 && !std::isfinite(sm_scale * kLog2e * kv4::kUnit)) return MAGE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out)) return MAGE_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return MAGE_ERR_INVALID_ARG;
    if ((int64_t)c->n_tokens * kv.H_q > (int64_t)0x7fffffff) return MAGE_ERR_UNSUPPORTED;
    if (workspace_bytes < mage_chunk_workspace_bytes(kv_in, c)) return MAGE_ERR_WORKSPACE;
    chunk::AttnArgs at;
    at.q = {static_cast<const __nv_bfloat16 *>(q), stride_t, stride_h};
    at.mask_block = mask_block;
    at.scale_log2 = sm_scale * kLog2e;
    at.out = static_cast<__nv_bfloat16 *>(out);
    at.lse = lse;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!use_decode<BITS>(&kv, c)) {
        if constexpr (BITS == 4) {
            const size_t n = stage_bytes(&kv, c);
            if (n && workspace_bytes >= prefill_plan(&kv, c).bytes + 2 * n) return launch_prefill_staged(&kv, codes, c, at, workspace, dev_status, st);
        }
        return launch_prefill<BITS>(&kv, codes, c, at, workspace, dev_status, st);
    }
    const DecodePlan pl = decode_plan<BITS>(&kv, c);
    if (pl.rows == 8) return launch_decode<BITS, 1>(&kv, codes, c, at, pl, workspace, dev_status, st);
    return launch_decode<BITS, 2>(&kv, codes, c, at, pl, workspace, dev_status, st);
}

// rows that share memory cannot be written one by one
bool rows_apart(const mage_kv_t &kv) { return kv.page_size != 0 || ((kv.H_kv == 1 || kv.stride_h >= kD) && (kv.P == 1 || kv.stride_p >= kD)); }

template <int BITS>
mage_status append_chunk(const mage_kv_t *kv_in, const Codes<BITS> &codes, const mage_chunk_t *c, const void *k_new, const void *v_new, int64_t stride_t,
                         int64_t stride_h, uint32_t *dev_status, void *stream) {
    mage_kv_t kv;
    const mage_status s = chunk_kv(kv_in, codes, &kv);
    if (s != MAGE_OK) return s;
    if (!valid_chunk(c)) return MAGE_ERR_INVALID_ARG;
    if (c->n_tokens == 0) return MAGE_OK;                 // (max_len 0 is a bound like others: ranges that are not empty are reported)
    if (!k_new || !v_new || !stride_ok(stride_t) || !stride_ok(stride_h) || kv.N_max < 1) return MAGE_ERR_INVALID_ARG;
    if (!aligned16(k_new) || !aligned16(v_new)) return MAGE_ERR_UNSUPPORTED;
    if (!rows_apart(kv)) return MAGE_ERR_INVALID_ARG;
    const chunk::Strided kn = {static_cast<const __nv_bfloat16 *>(k_new), stride_t, stride_h};
    const __nv_bfloat16 *vn = static_cast<const __nv_bfloat16 *>(v_new);
    // long chunks: four heads' rows per warp, so that 64 bytes per lane are in flight; short ones: one, for the shortest chain (8 bits, 8 heads, one / four:
    // 61 tokens 2.5 / 2.8 us, 300: 2.7 / 2.8, 600: 3.5 / 3.0, 1184: 3.9 / 3.4, 2400: 6.8 / 4.9, 16 prompts of 300 to 2048: 33.9 / 19.4)
    const int rows = (int64_t)c->n_tokens * kv.H_kv >= (int64_t)kSms * 64 ? 4 : 1;
    const dim3 grid((c->n_tokens + 3) / 4, (kv.H_kv + rows - 1) / rows);                  // (H_kv is at most 65535)
    auto kern = rows == 4 ? chunk::append_kernel<BITS, 4> : chunk::append_kernel<BITS, 1>;
    launch_pdl(kern, grid, dim3(128), 0, static_cast<cudaStream_t>(stream), make_view(&kv), codes.v, chunk_view(c), kn, vn, dev_status);
    return launch_check();
}

// What mage_rope and the calls that rotate on the way into the cache check of a rotation alone, and the kernel's part of it.
mage_status rope_args(const mage_rope_t *r, int32_t n_tokens, const int32_t *positions, int64_t pos_stride, rope::Args *a) {
    a->n_tokens = n_tokens; a->rot = r->rot_dim; a->halves = r->halves != 0; a->n_axes = r->n_axes;
    a->mult = r->mult; a->positions = positions; a->pos_stride = pos_stride; a->inv_freq = r->inv_freq;
    for (int i = 0; i < 64; ++i) {
        a->axis[i] = i < r->rot_dim / 2 ? r->axis_of_pair[i] : 0;
        if (a->axis[i] >= r->n_axes) return MAGE_ERR_INVALID_ARG;
    }
    return MAGE_OK;
}
mage_status rope_dims(const mage_rope_t *r) {
    if (!r || r->d < 1 || r->n_axes < 1 || r->rot_dim < 1 || r->rot_dim > r->d) return MAGE_ERR_INVALID_ARG;
    return r->d != kD || r->rot_dim % 16 || r->n_axes > 4 ? MAGE_ERR_UNSUPPORTED : MAGE_OK;
}

template <int BITS>
mage_status rope_append_chunk(const mage_kv_t *kv_in, const Codes<BITS> &codes, const mage_chunk_t *c, const mage_rope_t *r, const int32_t *positions, int64_t pos_stride,
                              const void *q, int64_t q_stride_t, int64_t q_stride_h, void *q_out, int64_t qo_stride_t, int64_t qo_stride_h, const void *k_new,
                              const void *v_new, int64_t stride_t, int64_t stride_h, uint32_t *dev_status, void *stream) {
    mage_kv_t kv;
    mage_status s = chunk_kv(kv_in, codes, &kv);
    if (s != MAGE_OK) return s;
    if (!valid_chunk(c)) return MAGE_ERR_INVALID_ARG;
    if ((s = rope_dims(r)) != MAGE_OK) return s;
    if (c->n_tokens == 0) return MAGE_OK;
    if (!positions || !r->inv_freq || pos_stride < 0 || !std::isfinite(r->mult) || !q || !q_out || !k_new || !v_new || kv.N_max < 1) return MAGE_ERR_INVALID_ARG;
    if (!stride_ok(q_stride_t) || !stride_ok(q_stride_h) || !stride_ok(qo_stride_t) || !stride_ok(qo_stride_h) || !stride_ok(stride_t) || !stride_ok(stride_h)) return MAGE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k_new) || !aligned16(v_new) || kv.H_q > (1 << 20)) return MAGE_ERR_UNSUPPORTED;
    // as mage_rope: heads or tokens that share memory cannot be written one by one, in place means the same elements
    if ((c->n_tokens > 1 && qo_stride_t < kD) || (kv.H_q > 1 && qo_stride_h < kD) || !rows_apart(kv)) return MAGE_ERR_INVALID_ARG;
    if (q == q_out && (q_stride_t != qo_stride_t || q_stride_h != qo_stride_h)) return MAGE_ERR_INVALID_ARG;
    rope::Args a = {};
    a.in[0] = static_cast<const __nv_bfloat16 *>(q); a.in[1] = static_cast<const __nv_bfloat16 *>(k_new);
    a.out[0] = static_cast<__nv_bfloat16 *>(q_out);
    a.st[0] = q_stride_t; a.sh[0] = q_stride_h; a.ost[0] = qo_stride_t; a.osh[0] = qo_stride_h;
    a.st[1] = stride_t; a.sh[1] = stride_h;
    a.heads[0] = kv.H_q; a.heads[1] = kv.H_kv;
    if ((s = rope_args(r, c->n_tokens, positions, pos_stride, &a)) != MAGE_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const __nv_bfloat16 *vn = static_cast<const __nv_bfloat16 *>(v_new);
    // as mage_rope: one token a block for few, two in a smaller block for many, at 64 registers a thread (16 prompts, us, 16 bits / 8 bits and read back: two heads of keys a warp
    // 65.6 / -, one 72.1 / 93.3; with 48 registers 66.8, 70.7 / 94.6; with 80 71.5 / 95.5)
    if (c->n_tokens >= kSms * 8)
        launch_pdl(rope::rope_append_kernel<BITS, 2, 128, BITS == 16 ? 2 : 1, 8>, dim3((c->n_tokens + 1) / 2), dim3(128), 0, st, a, make_view(&kv), codes.v, chunk_view(c), vn,
                   dev_status);
    else
        launch_pdl(rope::rope_append_kernel<BITS, 1, 256, 1, 4>, dim3(c->n_tokens), dim3(256), 0, st, a, make_view(&kv), codes.v, chunk_view(c), vn, dev_status);
    return launch_check();
}

template <int BITS>
mage_status read_rows(const mage_kv_t *kv_in, const Codes<BITS> &codes, const int32_t *indices, const int32_t *k_eff, int32_t row_begin, int32_t n_rows, void *k_out,
                      void *v_out, uint32_t *dev_status, void *stream) {
    mage_kv_t kv;
    const mage_status s = chunk_kv(kv_in, codes, &kv);
    if (s != MAGE_OK) return s;
    if (n_rows < 0 || row_begin < 0 || (indices && (row_begin != 0 || !k_eff))) return MAGE_ERR_INVALID_ARG;
    if (n_rows == 0 || kv.N_max == 0) return MAGE_OK;
    if (!k_out || !v_out) return MAGE_ERR_INVALID_ARG;
    if (!aligned16(k_out) || !aligned16(v_out) || n_rows > kMaxPos || row_begin > kMaxPos) return MAGE_ERR_UNSUPPORTED;
    launch_pdl(chunk::read_kernel<BITS>, dim3((n_rows + 8 * chunk::kReadRows - 1) / (8 * chunk::kReadRows), kv.P * kv.H_kv), dim3(256), 0, static_cast<cudaStream_t>(stream),
               make_view(&kv), codes.v, chunk::ChunkView{}, (const int *)indices, (const int *)k_eff, row_begin, n_rows, static_cast<__nv_bfloat16 *>(k_out), static_cast<__nv_bfloat16 *>(v_out),
               dev_status);
    return launch_check();
}

}  // namespace
}  // namespace mage

using namespace mage;

extern "C" {

mage_status mage_rope(const mage_rope_t *r, int32_t n_tokens, const int32_t *positions, int64_t pos_stride, int32_t H_q, const void *q, int64_t q_stride_t,
                      int64_t q_stride_h, void *q_out, int64_t qo_stride_t, int64_t qo_stride_h, int32_t H_kv, const void *k, int64_t k_stride_t, int64_t k_stride_h,
                      void *k_out, int64_t ko_stride_t, int64_t ko_stride_h, void *stream) {
    if (!r || n_tokens < 0 || H_q < 1 || H_kv < 0) return MAGE_ERR_INVALID_ARG;
    mage_status s = rope_dims(r);
    if (s != MAGE_OK) return s;
    if (n_tokens == 0) return MAGE_OK;
    if (!positions || !r->inv_freq || !q || !q_out || (H_kv > 0 && (!k || !k_out)) || pos_stride < 0 || !std::isfinite(r->mult)) return MAGE_ERR_INVALID_ARG;
    const int64_t strides[8] = {q_stride_t, q_stride_h, qo_stride_t, qo_stride_h, k_stride_t, k_stride_h, ko_stride_t, ko_stride_h};
    for (int i = 0; i < (H_kv > 0 ? 8 : 4); ++i)
        if (!stride_ok(strides[i])) return MAGE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(q_out) || (H_kv > 0 && (!aligned16(k) || !aligned16(k_out)))) return MAGE_ERR_UNSUPPORTED;
    // heads or tokens that share memory cannot be written one by one
    if ((n_tokens > 1 && (qo_stride_t < kD || (H_kv > 0 && ko_stride_t < kD))) || (H_q > 1 && qo_stride_h < kD) || (H_kv > 1 && ko_stride_h < kD)) return MAGE_ERR_INVALID_ARG;
    // in place means the same elements: anything else would read what another thread has written
    if ((q == q_out && (q_stride_t != qo_stride_t || q_stride_h != qo_stride_h)) ||
        (H_kv > 0 && k == k_out && (k_stride_t != ko_stride_t || k_stride_h != ko_stride_h)))
        return MAGE_ERR_INVALID_ARG;
    rope::Args a;
    a.in[0] = static_cast<const __nv_bfloat16 *>(q); a.in[1] = static_cast<const __nv_bfloat16 *>(k);
    a.out[0] = static_cast<__nv_bfloat16 *>(q_out); a.out[1] = static_cast<__nv_bfloat16 *>(k_out);
    a.st[0] = q_stride_t; a.sh[0] = q_stride_h; a.ost[0] = qo_stride_t; a.osh[0] = qo_stride_h;
    a.st[1] = k_stride_t; a.sh[1] = k_stride_h; a.ost[1] = ko_stride_t; a.osh[1] = ko_stride_h;
    a.heads[0] = H_q; a.heads[1] = H_kv;
    if ((int64_t)(H_q + H_kv) > (1 << 20)) return MAGE_ERR_UNSUPPORTED;
    if ((s = rope_args(r, n_tokens, positions, pos_stride, &a)) != MAGE_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // few tokens: one each, so that the call spreads over the SMs; more: two in a smaller block, whose table and exit overlap with other blocks' loads
    // (32 + 8 heads, one / two tokens a block: 148 tokens 2.4 / 3.5 us, 600: 4.7 / 4.5, 1184: 6.1 / 5.4, 2400: 11.1 / 11.2, 8199: 37.6 / 26.7)
    if (n_tokens >= kSms * 8) launch_pdl(rope::rope_kernel<2, 128, 1>, dim3((n_tokens + 1) / 2), dim3(128), 0, st, a);
    else launch_pdl(rope::rope_kernel<1, 256, 2>, dim3(n_tokens), dim3(256), 0, st, a);
    return launch_check();
}

mage_status mage_append_chunk(const mage_kv_t *kv, const mage_chunk_t *chunk, const void *k_new, const void *v_new, int64_t stride_t, int64_t stride_h,
                              uint32_t *dev_status, void *stream) {
    return append_chunk(kv, codes16(), chunk, k_new, v_new, stride_t, stride_h, dev_status, stream);
}
mage_status mage_append_chunk_kv8(const mage_kv_t *kv, const mage_kv8_t *kv8, const mage_chunk_t *chunk, const void *k_new, const void *v_new, int64_t stride_t, int64_t stride_h,
                              uint32_t *dev_status, void *stream) {
    return append_chunk(kv, codes_of(kv8), chunk, k_new, v_new, stride_t, stride_h, dev_status, stream);
}
mage_status mage_append_chunk_kv4(const mage_kv_t *kv, const mage_kv4_t *kv4, const mage_chunk_t *chunk, const void *k_new, const void *v_new, int64_t stride_t, int64_t stride_h,
                              uint32_t *dev_status, void *stream) {
    return append_chunk(kv, codes_of(kv4), chunk, k_new, v_new, stride_t, stride_h, dev_status, stream);
}
mage_status mage_rope_append_chunk(const mage_kv_t *kv, const mage_chunk_t *chunk, const mage_rope_t *rope, const int32_t *positions,
                                       int64_t pos_stride, const void *q, int64_t q_stride_t, int64_t q_stride_h, void *q_out, int64_t qo_stride_t, int64_t qo_stride_h,
                                       const void *k_new, const void *v_new, int64_t stride_t, int64_t stride_h, uint32_t *dev_status, void *stream) {
    return rope_append_chunk(kv, codes16(), chunk, rope, positions, pos_stride, q, q_stride_t, q_stride_h, q_out, qo_stride_t, qo_stride_h, k_new, v_new, stride_t, stride_h, dev_status,
                             stream);
}
mage_status mage_rope_append_chunk_kv8(const mage_kv_t *kv, const mage_kv8_t *kv8, const mage_chunk_t *chunk, const mage_rope_t *rope, const int32_t *positions,
                                       int64_t pos_stride, const void *q, int64_t q_stride_t, int64_t q_stride_h, void *q_out, int64_t qo_stride_t, int64_t qo_stride_h,
                                       const void *k_new, const void *v_new, int64_t stride_t, int64_t stride_h, uint32_t *dev_status, void *stream) {
    return rope_append_chunk(kv, codes_of(kv8), chunk, rope, positions, pos_stride, q, q_stride_t, q_stride_h, q_out, qo_stride_t, qo_stride_h, k_new, v_new, stride_t, stride_h, dev_status,
                             stream);
}
mage_status mage_rope_append_chunk_kv4(const mage_kv_t *kv, const mage_kv4_t *kv4, const mage_chunk_t *chunk, const mage_rope_t *rope, const int32_t *positions,
                                       int64_t pos_stride, const void *q, int64_t q_stride_t, int64_t q_stride_h, void *q_out, int64_t qo_stride_t, int64_t qo_stride_h,
                                       const void *k_new, const void *v_new, int64_t stride_t, int64_t stride_h, uint32_t *dev_status, void *stream) {
    return rope_append_chunk(kv, codes_of(kv4), chunk, rope, positions, pos_stride, q, q_stride_t, q_stride_h, q_out, qo_stride_t, qo_stride_h, k_new, v_new, stride_t, stride_h, dev_status,
                             stream);
}

mage_status mage_kv8_read(const mage_kv_t *kv, const mage_kv8_t *kv8, const int32_t *indices, const int32_t *k_eff, int32_t row_begin, int32_t n_rows, void *k_out,
                          void *v_out, uint32_t *dev_status, void *stream) {
    return read_rows(kv, codes_of(kv8), indices, k_eff, row_begin, n_rows, k_out, v_out, dev_status, stream);
}
mage_status mage_kv4_read(const mage_kv_t *kv, const mage_kv4_t *kv4, const int32_t *indices, const int32_t *k_eff, int32_t row_begin, int32_t n_rows, void *k_out,
                          void *v_out, uint32_t *dev_status, void *stream) {
    return read_rows(kv, codes_of(kv4), indices, k_eff, row_begin, n_rows, k_out, v_out, dev_status, stream);
}

size_t mage_chunk_workspace_bytes_kv4(const mage_kv_t *kv, const mage_chunk_t *chunk) {
    const size_t n = mage_chunk_workspace_bytes(kv, chunk);
    return n ? n + 2 * stage_bytes(kv, chunk) : 0;
}
size_t mage_chunk_workspace_bytes(const mage_kv_t *kv_in, const mage_chunk_t *chunk) {
    if (!kv_in || !chunk || chunk->n_tokens < 0 || chunk->max_len < 0 || chunk->max_len > chunk->n_tokens) return 0;
    mage_kv_t kv = *kv_in;                            // the size is that of every cache type: pointers play no part
    kv.k_cache = kv.v_cache = reinterpret_cast<const void *>(256);
    if (!valid_kv(&kv, nullptr) || kv.N_max > kMaxPos) return 0;
    if ((int64_t)chunk->n_tokens * kv.H_q > (int64_t)0x7fffffff) return 0;
    size_t most = use_decode<4>(&kv, chunk) ? decode_plan<4>(&kv, chunk).bytes : 0;
    if (use_decode<16>(&kv, chunk)) most = std::max({most, decode_plan<16>(&kv, chunk).bytes, decode_plan<8>(&kv, chunk).bytes});
    else most = std::max(most, prefill_plan(&kv, chunk).bytes);
    return most;
}

mage_status mage_chunk_attn(const mage_kv_t *kv, const mage_chunk_t *chunk, const void *q, int64_t stride_t, int64_t stride_h, int32_t mask_block,
                                float sm_scale, void *out, float *lse, void *workspace, size_t workspace_bytes, uint32_t *dev_status, void *stream) {
    return chunk_attn(kv, codes16(), chunk, q, stride_t, stride_h, mask_block, sm_scale, out, lse, workspace, workspace_bytes, dev_status, stream);
}
mage_status mage_chunk_attn_kv8(const mage_kv_t *kv, const mage_kv8_t *kv8, const mage_chunk_t *chunk, const void *q, int64_t stride_t, int64_t stride_h, int32_t mask_block,
                                float sm_scale, void *out, float *lse, void *workspace, size_t workspace_bytes, uint32_t *dev_status, void *stream) {
    return chunk_attn(kv, codes_of(kv8), chunk, q, stride_t, stride_h, mask_block, sm_scale, out, lse, workspace, workspace_bytes, dev_status, stream);
}
mage_status mage_chunk_attn_kv4(const mage_kv_t *kv, const mage_kv4_t *kv4, const mage_chunk_t *chunk, const void *q, int64_t stride_t, int64_t stride_h, int32_t mask_block,
                                float sm_scale, void *out, float *lse, void *workspace, size_t workspace_bytes, uint32_t *dev_status, void *stream) {
    return chunk_attn(kv, codes_of(kv4), chunk, q, stride_t, stride_h, mask_block, sm_scale, out, lse, workspace, workspace_bytes, dev_status, stream);
}

}  // extern "C"
