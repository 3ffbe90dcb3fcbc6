// Host side of the block cache: argument validation and launch sizes of la_kv_store, la_kv_load, la_block_select and
// la_verify_attention_sparse (declared in la_verify.h).
#include <math.h>
#include <string.h>

#include "la_internal.hpp"

namespace la {
namespace {

inline bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr int64_t kMaxUnits = 1 << 23;          // workgroups per launch
constexpr int64_t kMaxThreads = 0xffffffff;     // and threads: a dimension of a grid has fewer than 2^32
constexpr int64_t kMaxBlocks = 1 << 20;         // blocks of one request that a selection can look at
inline bool launchable(int64_t workgroups, int threads) { return workgroups <= kMaxUnits && workgroups * threads <= kMaxThreads; }

// Shape, types and sizes that every call of the block cache checks.
la_status validate(const la_attn_desc *d) {
  if (!d) return LA_ERR_INVALID_ARG;
  if (d->num_requests < 1 || d->num_q_heads < 1 || d->num_kv_heads < 1 || d->head_dim < 1 || d->gamma < 1 ||
      d->branch_len < 1)
    return LA_ERR_INVALID_ARG;
  if (d->num_q_heads % d->num_kv_heads) return LA_ERR_INVALID_ARG;
  if (d->block_size < 16 || (d->block_size & (d->block_size - 1))) return LA_ERR_INVALID_ARG;
  if (d->max_blocks_per_request < 0) return LA_ERR_INVALID_ARG;
  if (!(d->softmax_scale > 0.f) || !isfinite(d->softmax_scale)) return LA_ERR_INVALID_ARG;
  if (d->kv_split_tokens != 0 || d->kernel_shape != 0) return LA_ERR_INVALID_ARG;
  const int32_t dts[4] = {d->q_dtype, d->kv_dtype, d->branch_kv_dtype, d->out_dtype};
  for (int i = 0; i < 4; ++i)
    if (dts[i] < LA_F32 || dts[i] > LA_MXFP4_E2M1) return LA_ERR_INVALID_ARG;
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return LA_ERR_UNSUPPORTED;
  if (d->q_dtype != LA_BF16 || d->branch_kv_dtype != LA_BF16) return LA_ERR_UNSUPPORTED;
  if (d->out_dtype != LA_BF16 && d->out_dtype != LA_F32) return LA_ERR_UNSUPPORTED;
  if (d->kv_dtype != LA_BF16 && d->kv_dtype != LA_MXFP8_E4M3 && d->kv_dtype != LA_MXFP4_E2M1) return LA_ERR_UNSUPPORTED;
  // rows and prefix tokens are indexed with 32-bit integers on the device
  int64_t rows = (int64_t)d->gamma * d->branch_len;
  if (rows > (int64_t)1 << 30) return LA_ERR_UNSUPPORTED;
  rows *= d->num_q_heads;
  if (rows > (int64_t)1 << 30 || rows * d->num_requests > (int64_t)1 << 30) return LA_ERR_UNSUPPORTED;
  if ((int64_t)d->max_blocks_per_request * d->block_size > (int64_t)1 << 30) return LA_ERR_UNSUPPORTED;
  return LA_OK;
}

int format_of(const la_attn_desc *d) {
  return d->kv_dtype == LA_BF16 ? FMT_BF16 : d->kv_dtype == LA_MXFP8_E4M3 ? FMT_MX8 : FMT_MX4;
}

// Rows and exponents of a cache: 16-byte alignment, as all tensors of the library.
bool good_cache(const la_attn_desc *d, const la_block_cache *c) {
  if (!c || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return false;
  return d->kv_dtype == LA_BF16 || (c->k_exp && c->v_exp && aligned(c->k_exp, 16) && aligned(c->v_exp, 16));
}

// Strides of further layers keep every layer's tensors 16-byte aligned.
bool good_layers(const la_attn_desc *d, const la_block_cache *c, const la_layer_strides *l, int row_bytes) {
  if (!l) return true;
  if (l->num_layers < 1 || l->num_layers > 65535) return false;
  if (l->cache_stride < 0 || l->branch_stride < 0 || l->chain_stride < 0 || c->exp_stride < 0 || c->bounds_stride < 0)
    return false;
  const int64_t half_bytes = d->kv_dtype == LA_BF16 ? 4 : d->kv_dtype == LA_MXFP8_E4M3 ? 2 : 1;  // per element
  if (l->cache_stride % 32 || l->cache_stride * half_bytes / 2 % 16) return false;
  return (l->branch_stride * row_bytes) % 16 == 0 && (l->chain_stride * row_bytes) % 16 == 0 && c->exp_stride % 16 == 0 &&
         c->bounds_stride % 8 == 0;
}

la_status check_prefixes(const la_attn_desc *d, const int32_t *prefix_lens_host, int64_t *longest) {
  if (!prefix_lens_host) return LA_ERR_INVALID_ARG;
  *longest = 0;
  for (int b = 0; b < d->num_requests; ++b) {
    const int64_t P = prefix_lens_host[b];
    if (P < 0 || P > (int64_t)d->max_blocks_per_request * d->block_size) return LA_ERR_INVALID_ARG;
    *longest = P > *longest ? P : *longest;
  }
  return LA_OK;
}

la_status validate_select(const la_attn_desc *d, const la_select_desc *s) {
  if (!s || s->group_len < 1 || s->group_len > d->branch_len || s->max_blocks < 1 || s->keep_first < 0 || s->keep_last < 0)
    return LA_ERR_INVALID_ARG;
  if ((int64_t)s->keep_first + s->keep_last > s->max_blocks) return LA_ERR_INVALID_ARG;
  if ((int64_t)s->max_blocks * d->block_size > (int64_t)1 << 30) return LA_ERR_UNSUPPORTED;
  return LA_OK;
}

inline int num_groups(const la_attn_desc *d, const la_select_desc *s) { return (d->branch_len - 1) / s->group_len + 1; }

struct SelectPlan {
  int64_t units;
  int n_max, n_tiles;
  size_t score_bytes, top_bytes, exact_bytes;
};

la_status plan_select(const la_attn_desc *d, const la_select_desc *s, const int32_t *prefix_lens_host, SelectPlan *plan) {
  la_status st = validate(d);
  if (st != LA_OK) return st;
  if ((st = validate_select(d, s)) != LA_OK) return st;
  int64_t longest = 0;
  if ((st = check_prefixes(d, prefix_lens_host, &longest)) != LA_OK) return st;
  const int64_t n = (longest + d->block_size - 1) / d->block_size;
  plan->units = (int64_t)d->num_requests * d->gamma * num_groups(d, s) * d->num_kv_heads;
  if (n > kMaxBlocks) return LA_ERR_UNSUPPORTED;
  if (!launchable(plan->units, block_pick_threads((int)n, s->group_len * (d->num_q_heads / d->num_kv_heads)))) return LA_ERR_UNSUPPORTED;
  plan->n_max = (int)n, plan->n_tiles = (int)((n + 31) / 32);
  const bool all = n <= s->max_blocks;   // nothing to choose
  plan->score_bytes = all ? 0 : align_up((size_t)plan->units * n * sizeof(float));
  plan->top_bytes = all ? 0 : align_up((size_t)d->num_requests * d->num_kv_heads * plan->n_tiles * sizeof(float));
  plan->exact_bytes = all ? 0 : align_up((size_t)plan->units * n * sizeof(double));
  return LA_OK;
}

struct SparsePlan {
  int n_groups, tile_rows, n_row_tiles, waves, n_split;
  size_t part_o_bytes, part_ml_bytes;
};

// Kernel shapes of the attention over blocks: rows per unit, wavefronts per workgroup, keys per tile, and microseconds per tile of
// a workgroup that has its CU to itself (latency) and of one of several that share it (busy, before the memory's share).
struct SparseShape {
  int rows, waves, keys;
  double latency, busy;
};
constexpr SparseShape kShapes[] = {
    {16, 4, 32, 0.26, 0.15}, {16, 8, 32, 0.15, 0.13}, {32, 4, 32, 0.30, 0.20}, {32, 8, 32, 0.17, 0.20},
    {64, 4, 64, 1.30, 0.83}, {96, 6, 64, 1.20, 1.20}, {128, 8, 64, 1.30, 1.30},
    {128, 4, 32, 2.0, 2.0},  // (head dimension 256)
};
bool shape_exists(const SparseShape &s, int D) { return D == 256 ? s.waves == 4 && s.keys == 32 : s.keys == 64 || s.rows <= 32; }
bool shape_fits(const SparseShape &s, int D, int64_t rows) {
  if (!shape_exists(s, D)) return false;
  if (D == 256) return s.rows == (rows <= 16 ? 16 : rows <= 32 ? 32 : 128);
  return rows <= 16 ? s.rows == 16 : rows <= 32 ? s.rows == 32 : rows <= 64 ? s.rows == 64 : s.rows >= 64;
}

// Which shape runs a call and over how many workgroups a unit's keys are split, from a simple model in microseconds (constants
// fitted to measured times of forced shapes and splits at head dimension 128, scaled to the others): what the workgroups of all
// units take, shared out over the CUs, or the longest of them, whichever is more, and the merge of the partial results.  Of 15 calls
// nine take up to 6 % longer than with the fastest shape and split, the others 9 to 34 %.
la_status plan_sparse(const la_attn_desc *d, const la_select_desc *s, const int32_t *prefix_lens_host, SparsePlan *plan) {
  la_status st = validate(d);
  if (st != LA_OK) return st;
  if (s && (st = validate_select(d, s)) != LA_OK) return st;
  int64_t longest = 0;
  if ((st = check_prefixes(d, prefix_lens_host, &longest)) != LA_OK) return st;
  const int G = d->num_q_heads / d->num_kv_heads, D = d->head_dim;
  const int64_t rows = (int64_t)(s ? s->group_len : d->gamma * d->branch_len) * G;   // of a group
  const int64_t listed = s ? (int64_t)s->max_blocks * d->block_size : (int64_t)1 << 30;
  int64_t all_keys = 0;
  for (int b = 0; b < d->num_requests; ++b) all_keys += prefix_lens_host[b] < listed ? prefix_lens_host[b] : listed;
  const int64_t most_keys = longest < listed ? longest : listed;
  const size_t all_rows = (size_t)d->num_requests * d->gamma * d->branch_len * d->num_q_heads;
  const double row_bytes = 2.0 * (d->kv_dtype == LA_BF16 ? 2.0 * D : d->kv_dtype == LA_MXFP8_E4M3 ? D * 33.0 / 32 : D * 17.0 / 32);
  plan->n_groups = s ? d->gamma * num_groups(d, s) : 1;
  const int cus = num_cus();
  double best = -1.0;
  SparseForce force = {0, 0, 0};
  const bool forced = selftest_sparse_plan && selftest_sparse_plan(&force);
  for (const SparseShape &shape : kShapes) {
    if (forced ? !shape_exists(shape, D) || shape.rows != force.rows || shape.waves != force.waves : !shape_fits(shape, D, rows)) continue;
    const int64_t row_tiles = (rows + shape.rows - 1) / shape.rows;
    const int64_t per_request = (int64_t)plan->n_groups * row_tiles * d->num_kv_heads, units = per_request * d->num_requests;
    // tiles of the longest request's units, and of all (own tokens of the branches that a unit's rows belong to)
    const int64_t own = ((int64_t)d->branch_len + shape.rows) / shape.keys + 2;
    const int64_t most = (most_keys + shape.keys - 1) / shape.keys + own;
    const double tiles = (double)all_keys / shape.keys + (double)d->num_requests * own;
    // the blocks of a workgroup's tiles have to fit its table (a range need not begin at a block's first key)
    const int64_t fit = ((int64_t)attn_blocks_max_slots() - 2) * d->block_size / shape.keys - 2;
    const int64_t least = (most + fit - 1) / fit;
    if (!launchable(units * least, 64 * shape.waves)) continue;
    // all CUs stream at 5 TB/s between them
    const double scale = D / 128.0, stream = shape.keys * row_bytes * cus / 5.0e6;
    const double busy = shape.busy * scale > stream ? shape.busy * scale : stream;
    const double alone = shape.latency * scale > busy ? shape.latency * scale : busy;
    const int64_t slots = most / (shape.keys == 32 ? shape.waves : 1);   // a tile at least for every wavefront
    const int64_t n0 = forced && force.split > least ? force.split : least;
    for (int64_t n = n0; n == n0 || (!forced && n <= slots && n <= 64 && units * n <= 4 * (int64_t)cus); ++n) {
      if (n > 1 && (int64_t)all_rows * attn_merge_threads(D, (int)n) > kMaxThreads - 255) break;
      const double start = 1.5, longest_us = (double)most / (double)n * alone + start;
      const double all_us = (double)per_request / cus * (tiles * busy + (double)(n * d->num_requests) * start);
      const double merge_us = n > 1 ? 3.0 + (double)(n * all_rows) * (D + 2) * 8.0 / 3.0e6 : 0.0;
      // units of one length come in whole rounds
      const int64_t rounds = (units * n + cus - 1) / cus;
      const double even_us = (double)rounds * ((double)most / (double)n * busy + start);
      const bool even = most_keys * d->num_requests == all_keys;
      double us = even ? even_us : all_us + 0.25 * longest_us;
      us = (us > longest_us ? us : longest_us) + merge_us;
      if (best < 0.0 || us < best) {
        best = us;
        plan->tile_rows = shape.rows, plan->waves = shape.waves, plan->n_row_tiles = (int)row_tiles, plan->n_split = (int)n;
      }
    }
  }
  if (best < 0.0) return LA_ERR_UNSUPPORTED;   // more workgroups than a launch takes, whatever the shape
  const size_t n = (size_t)plan->n_split;
  plan->part_o_bytes = n > 1 ? align_up(n * all_rows * D * sizeof(float)) : 0;
  plan->part_ml_bytes = n > 1 ? align_up(n * all_rows * 2 * sizeof(float)) : 0;
  return LA_OK;
}

}  // namespace
}  // namespace la

using namespace la;

extern "C" {

la_status la_kv_store(const la_attn_desc *desc, const la_block_cache *cache, const int32_t *block_tables,
                      const int32_t *prefix_lens, const int32_t *prefix_lens_host, const void *k_branch,
                      const void *v_branch, const void *k_chain, const void *v_chain, int32_t chain_len,
                      const int32_t *src_branch, const int32_t *n_chain, const int32_t *n_own, int32_t *new_prefix_lens,
                      const la_layer_strides *layers, void *hip_stream) {
  la_status st = validate(desc);
  if (st != LA_OK) return st;
  if (!good_cache(desc, cache) || !aligned(cache->k_bounds, 16)) return LA_ERR_INVALID_ARG;
  if (!prefix_lens || !prefix_lens_host || !k_branch || !v_branch || !new_prefix_lens || new_prefix_lens == prefix_lens)
    return LA_ERR_INVALID_ARG;
  if (chain_len < 0 || (chain_len > 0 && (!k_chain || !v_chain))) return LA_ERR_INVALID_ARG;
  if (!aligned(k_branch, 16) || !aligned(v_branch, 16) || !aligned(k_chain, 16) || !aligned(v_chain, 16))
    return LA_ERR_INVALID_ARG;
  if (!good_layers(desc, cache, layers, 2) || desc->num_requests > 65535) return LA_ERR_INVALID_ARG;
  const int64_t capacity = (int64_t)desc->max_blocks_per_request * desc->block_size;
  const int64_t tokens = (int64_t)chain_len + desc->branch_len;
  for (int b = 0; b < desc->num_requests; ++b)
    if (prefix_lens_host[b] < 0 || prefix_lens_host[b] + tokens > capacity) return LA_ERR_INVALID_ARG;

  BlockStoreParams p;
  memset(&p, 0, sizeof p);
  p.c.k_cache = cache->k, p.c.v_cache = cache->v;
  p.k_exp = cache->k_exp, p.v_exp = cache->v_exp, p.k_bounds = cache->k_bounds;
  p.exp_stride = cache->exp_stride, p.bounds_stride = cache->bounds_stride;
  p.c.k_branch = k_branch, p.c.v_branch = v_branch, p.c.k_chain = k_chain, p.c.v_chain = v_chain;
  p.c.block_tables = block_tables, p.c.prefix_lens = prefix_lens;
  p.c.src_branch = src_branch, p.c.n_chain = n_chain, p.c.n_own = n_own;
  p.c.new_prefix_lens = new_prefix_lens;
  p.c.B = desc->num_requests, p.c.Hkv = desc->num_kv_heads, p.c.D = desc->head_dim, p.c.gamma = desc->gamma;
  p.c.L = desc->branch_len, p.c.C = chain_len;
  p.c.block_size = desc->block_size, p.c.block_shift = __builtin_ctz((unsigned)desc->block_size);
  p.c.max_blocks = desc->max_blocks_per_request, p.c.capacity = (int)capacity;
  p.c.num_layers = layers ? layers->num_layers : 1;
  if (layers) {
    p.c.cache_stride = layers->cache_stride, p.c.branch_stride = layers->branch_stride;
    p.c.chain_stride = layers->chain_stride;
  }
  // rows that begin anywhere in a block touch at most this many
  p.n_dst = (int)((tokens + desc->block_size - 2) / desc->block_size) + 1;
  if (!launchable((int64_t)p.n_dst * desc->num_kv_heads, 256)) return LA_ERR_UNSUPPORTED;
  return launch_kv_store(p, format_of(desc), (hipStream_t)hip_stream) == hipSuccess ? LA_OK : LA_ERR_LAUNCH;
}

la_status la_kv_load(const la_attn_desc *desc, const la_block_cache *cache, const int32_t *block_tables,
                     const int32_t *prefix_lens, const int32_t *first, int32_t num_tokens, void *k_out, void *v_out,
                     const la_layer_strides *layers, void *hip_stream) {
  la_status st = validate(desc);
  if (st != LA_OK) return st;
  if (!good_cache(desc, cache)) return LA_ERR_INVALID_ARG;
  if (!prefix_lens || !k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16) || num_tokens < 1)
    return LA_ERR_INVALID_ARG;
  const bool f32 = desc->out_dtype == LA_F32;
  if (!good_layers(desc, cache, layers, f32 ? 4 : 2) || desc->num_requests > 65535) return LA_ERR_INVALID_ARG;
  if ((int64_t)num_tokens * desc->num_kv_heads * (desc->head_dim / 8) > (int64_t)1 << 31) return LA_ERR_UNSUPPORTED;
  BlockLoadParams p;
  memset(&p, 0, sizeof p);
  p.k_cache = cache->k, p.v_cache = cache->v, p.k_exp = cache->k_exp, p.v_exp = cache->v_exp;
  p.block_tables = block_tables, p.prefix_lens = prefix_lens, p.first = first;
  p.k_out = k_out, p.v_out = v_out;
  p.B = desc->num_requests, p.Hkv = desc->num_kv_heads, p.D = desc->head_dim, p.T = num_tokens;
  p.block_shift = __builtin_ctz((unsigned)desc->block_size), p.max_blocks = desc->max_blocks_per_request;
  p.capacity = desc->max_blocks_per_request * desc->block_size;
  p.num_layers = layers ? layers->num_layers : 1;
  p.out_f32 = f32;
  p.exp_stride = cache->exp_stride;
  if (layers) p.cache_stride = layers->cache_stride, p.out_stride = layers->branch_stride;
  return launch_kv_load(p, format_of(desc), (hipStream_t)hip_stream) == hipSuccess ? LA_OK : LA_ERR_LAUNCH;
}

la_status la_block_select_workspace(const la_attn_desc *desc, const la_select_desc *sel, const int32_t *prefix_lens_host,
                                    size_t *bytes_out) {
  if (!bytes_out) return LA_ERR_INVALID_ARG;
  SelectPlan plan;
  la_status st = plan_select(desc, sel, prefix_lens_host, &plan);
  if (st != LA_OK) return st;
  *bytes_out = plan.score_bytes + plan.top_bytes + plan.exact_bytes;
  return LA_OK;
}

la_status la_block_select(const la_attn_desc *desc, const la_select_desc *sel, const void *q, const void *k_bounds,
                          const int32_t *block_tables, const int32_t *prefix_lens, const int32_t *prefix_lens_host,
                          int32_t *blocks, int32_t *counts, void *workspace, size_t workspace_bytes, void *hip_stream) {
  SelectPlan plan;
  la_status st = plan_select(desc, sel, prefix_lens_host, &plan);
  if (st != LA_OK) return st;
  if (!q || !prefix_lens || !blocks || !counts || (plan.n_max > 0 && !k_bounds)) return LA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_bounds, 16) || !aligned(workspace, 16)) return LA_ERR_INVALID_ARG;
  const size_t need = plan.score_bytes + plan.top_bytes + plan.exact_bytes;
  if (need > 0 && (!workspace || workspace_bytes < need)) return LA_ERR_WORKSPACE_TOO_SMALL;
  SelectParams p;
  memset(&p, 0, sizeof p);
  p.q = q, p.k_bounds = k_bounds, p.block_tables = block_tables, p.prefix_lens = prefix_lens;
  p.blocks = blocks, p.count = counts;
  p.exact = (double *)workspace;
  p.score = (float *)((uint8_t *)workspace + plan.exact_bytes);
  p.top = (float *)((uint8_t *)workspace + plan.exact_bytes + plan.score_bytes);
  p.B = desc->num_requests, p.Hq = desc->num_q_heads, p.Hkv = desc->num_kv_heads, p.G = p.Hq / p.Hkv, p.D = desc->head_dim;
  p.gamma = desc->gamma, p.L = desc->branch_len, p.group_len = sel->group_len, p.n_groups = num_groups(desc, sel);
  p.block_shift = __builtin_ctz((unsigned)desc->block_size), p.max_blocks = desc->max_blocks_per_request;
  p.max_sel = sel->max_blocks, p.keep_first = sel->keep_first, p.keep_last = sel->keep_last;
  p.n_max = plan.n_max, p.n_tiles = plan.n_tiles;
  return launch_block_select(p, (hipStream_t)hip_stream) == hipSuccess ? LA_OK : LA_ERR_LAUNCH;
}

la_status la_verify_attention_sparse_workspace(const la_attn_desc *desc, const la_select_desc *sel,
                                               const int32_t *prefix_lens_host, size_t *bytes_out) {
  if (!bytes_out) return LA_ERR_INVALID_ARG;
  SparsePlan plan;
  la_status st = plan_sparse(desc, sel, prefix_lens_host, &plan);
  if (st != LA_OK) return st;
  *bytes_out = plan.part_o_bytes + plan.part_ml_bytes;
  return LA_OK;
}

la_status la_verify_attention_sparse(const la_attn_desc *desc, const la_select_desc *sel, const void *q,
                                     const la_block_cache *cache, const int32_t *block_tables, const int32_t *prefix_lens,
                                     const int32_t *prefix_lens_host, const int32_t *blocks, const int32_t *counts,
                                     const void *k_branch, const void *v_branch, void *out, float *lse, void *workspace,
                                     size_t workspace_bytes, void *hip_stream) {
  SparsePlan plan;
  la_status st = plan_sparse(desc, sel, prefix_lens_host, &plan);
  if (st != LA_OK) return st;
  if ((sel != nullptr) != (blocks != nullptr) || (sel != nullptr) != (counts != nullptr)) return LA_ERR_INVALID_ARG;
  if (!q || !prefix_lens || !k_branch || !v_branch || !out) return LA_ERR_INVALID_ARG;
  bool any_prefix = false;
  for (int b = 0; b < desc->num_requests; ++b) any_prefix |= prefix_lens_host[b] > 0;
  if (!cache || (any_prefix && !good_cache(desc, cache))) return LA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_branch, 16) || !aligned(v_branch, 16) || !aligned(out, 16) || !aligned(workspace, 16))
    return LA_ERR_INVALID_ARG;
  const size_t need = plan.part_o_bytes + plan.part_ml_bytes;
  if (need > 0 && (!workspace || workspace_bytes < need)) return LA_ERR_WORKSPACE_TOO_SMALL;
  SparseParams p;
  memset(&p, 0, sizeof p);
  p.q = q, p.k_cache = cache->k, p.v_cache = cache->v, p.k_exp = cache->k_exp, p.v_exp = cache->v_exp;
  p.k_branch = k_branch, p.v_branch = v_branch;
  p.block_tables = block_tables, p.prefix_lens = prefix_lens, p.sel = blocks, p.sel_count = counts;
  if (need > 0) {
    p.part_o = (float *)workspace;
    p.part_ml = (float *)((uint8_t *)workspace + plan.part_o_bytes);
  }
  p.out = out, p.lse = lse;
  p.B = desc->num_requests, p.Hq = desc->num_q_heads, p.Hkv = desc->num_kv_heads, p.G = p.Hq / p.Hkv, p.D = desc->head_dim;
  p.gamma = desc->gamma, p.L = desc->branch_len;
  p.block_shift = __builtin_ctz((unsigned)desc->block_size), p.max_blocks = desc->max_blocks_per_request;
  p.max_sel = sel ? sel->max_blocks : 0, p.group_len = sel ? sel->group_len : 0;
  p.n_groups = plan.n_groups, p.tile_rows = plan.tile_rows, p.n_row_tiles = plan.n_row_tiles, p.waves = plan.waves;
  p.n_rows = desc->gamma * desc->branch_len * desc->num_q_heads;
  p.n_split = plan.n_split, p.out_f32 = desc->out_dtype == LA_F32;
  p.scale_log2 = desc->softmax_scale * 1.44269504088896340736f;
  hipStream_t stream = (hipStream_t)hip_stream;
  if (launch_attn_blocks(p, format_of(desc), stream) != hipSuccess) return LA_ERR_LAUNCH;
  if (plan.n_split == 1) return LA_OK;
  // the workgroups of a unit are joined as the chunks of one long prefix are, all rows being one request's
  AttnParams m;
  memset(&m, 0, sizeof m);
  m.part_o = p.part_o, m.part_ml = p.part_ml, m.out = out, m.lse = lse, m.out_f32 = p.out_f32;
  m.B = 1, m.D = p.D, m.n_rows = p.n_rows * p.B, m.s_max = plan.n_split;
  m.n_inline = 1, m.req[0].n = plan.n_split;
  return launch_attn_merge(m, stream) == hipSuccess ? LA_OK : LA_ERR_LAUNCH;
}

}  // extern "C"
