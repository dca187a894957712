// C entry points of the paged key/value cache: checks, launch shapes and dispatch.  Nothing allocates or synchronises.
#include "../../include/pqcache.h"

#include <algorithm>
#include <cmath>

#include "pqc_paged_kernels.h"

namespace {

using namespace pqc;
using namespace pqc::paged;

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Rows of `row` bytes, `stride` bytes apart.
struct Rows {
  const void* at;
  long long n, row, stride;
};
Rows bytes_at(const void* p, long long bytes) { return Rows{p, 1, bytes, bytes}; }
// Whether any byte of [p, p + bytes) is one of theirs: the first row that ends behind p begins in front of the end, or none does.
bool meets(const void* p, long long bytes, const Rows& r) {
  if (!p || !r.at || bytes <= 0 || r.n <= 0 || r.row <= 0) return false;
  const long long from = (long long)reinterpret_cast<uintptr_t>(p) - (long long)reinterpret_cast<uintptr_t>(r.at);  // p as seen from the first row
  if (from < r.row) return from + bytes > 0;
  if (r.n == 1) return false;
  const long long i = (from - r.row) / r.stride + 1;
  return i < r.n && i * r.stride < from + bytes;
}
template <size_t N>
bool meets_any(const void* p, long long bytes, const Rows (&rows)[N]) {
  for (const Rows& r : rows)
    if (meets(p, bytes, r)) return true;
  return false;
}

// A launch takes fewer than 2^32 work items, workgroups have 256.
constexpr long long kMaxGroups = 1ll << 24;

// Pages of a call from which append lays eight pages' workgroups of one head side by side.  Workgroups go to the eight dies in turn, so that the
// heads of a page then share a die's L2 and its rotation angles, which else every die reads by itself (eight heads, 32768 tokens: 554 MB read, 436
// so, 419 needed).  us without and with it, 32 query heads, 8 KV heads, pages of 64: 4096 tokens (64 pages) 19.9, 19.1, 8192 42.9, 40.0, 32768 161.3,
// 152.4; pages of 256 187.0, 159.9; 2 KV heads 74.7, 73.7.  Fewer pages would be rounded up to workgroups without work.
constexpr int kTogether = 64;

// Workgroups of the kernel of 16 rows over all heads: two per compute unit.  One per compute unit leaves its start and its tiles' ends
// uncovered (48 ragged sequences, 8 heads of 8 query heads, 280 MB: 80.5 us, two 70.4, three 79.9; a single sequence of 131072 tokens 64.9, 59.0,
// 66.9).  kRowsLds, beyond the kernel's own arrays, keeps a third off a compute unit: with room for three the 512 are spread unevenly (8
// sequences of 68224 tokens 233 us, 202 with it).
constexpr int kWorkers = 512;
constexpr size_t kRowsLds = 56 * 1024;
// One per compute unit where there is little to do for each: twice as many have as many more parts to fold.  us with 512 and 256, 8 heads of 4
// query heads, one sequence of 4096 tokens 13.4, 12.8, 6144 15.6, 13.5, 16384 19.5, 18.0, 32768 23.5, 23.5, two of 4096 17.1, 14.4; listed, 4096
// tokens 13.0, 12.0, 6600 14.6, 13.1, 13175 16.4, 15.4.  (This rule and kPartsFolded go by the width of the page table, since the lengths are known
// on the device alone: short sequences under a wide table are planned as long ones.)
constexpr int kFewUnits = 4;
// Items of the kernel of 128 rows that the length of a split aims at.
constexpr int kBlockItems = 480;

// Parts per tile up to which the last workgroup of a tile folds them itself; beyond that a launch of its own with a workgroup per row
// is quicker than one workgroup for all rows.  us, folded by the last and by a launch of its own: 8 heads of 4 query heads,
// 131072 tokens in all, 1 sequence (64 parts) 62.9, 59.4, 2 59.0, 59.5, 4 57.4, 59.8, 32 58.0, 61.8; 4 sequences of 2 heads (64 parts) 34.8,
// 26.1, 16 24.1, 26.8; listed, 13175 tokens each, 2 sequences of 8 query heads (32 parts) 26.0, 21.9, 4 32.7, 33.7.
constexpr int kPartsFolded = 16;

int make_geometry(const pqc_paged_config* c, long long n, Geometry* g) {
  if (!c) return PQC_EINVAL;
  if (c->batch < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads || c->head_dim < 1 || c->page_tokens < 1 ||
      c->n_pages < 1 || c->max_pages < 1 || n < 0)
    return PQC_EINVAL;
  if (c->io_dtype != PQC_F32 && c->io_dtype != PQC_BF16) return PQC_EINVAL;
  if (c->out_dtype != PQC_F32 && c->out_dtype != PQC_BF16) return PQC_EINVAL;
  if (c->cache_dtype != PQC_F32 && c->cache_dtype != PQC_BF16 && c->cache_dtype != PQC_FP8) return PQC_EINVAL;
  if (!std::isfinite(c->softmax_scale)) return PQC_EINVAL;
  if (c->rot_dims < 0 || c->rot_dims > c->head_dim || (c->rot_dims && c->rot_positions < 1)) return PQC_EINVAL;
  if (c->rot_style != PQC_ROT_HALVES && c->rot_style != PQC_ROT_PAIRS) return PQC_EINVAL;
  const int G = c->n_q_heads / c->n_kv_heads, P = c->page_tokens;
  if (c->head_dim != 64 && c->head_dim != 128) return PQC_EUNSUPPORTED;
  if (G > kRows || c->cache_dtype == PQC_F32 || c->rot_dims % 16) return PQC_EUNSUPPORTED;
  if (P < 16 || P > 256 || (P & (P - 1))) return PQC_EUNSUPPORTED;
  if (c->batch > 65535 || c->n_kv_heads > 65535) return PQC_EUNSUPPORTED;
  if ((long long)c->max_pages * P > (1 << 24) || (long long)c->n_pages * c->n_kv_heads * P >= (1ll << 31)) return PQC_EUNSUPPORTED;
  if (n * c->n_q_heads >= (1ll << 31)) return PQC_EUNSUPPORTED;
  g->B = c->batch; g->Hq = c->n_q_heads; g->Hkv = c->n_kv_heads; g->G = G;
  g->P = P;
  g->shift = __builtin_ctz((unsigned)P);
  g->n_pages = c->n_pages; g->max_pages = c->max_pages;
  g->n_q = (int)n;
  g->R = kRows / G;
  g->out_bf16 = c->out_dtype == PQC_BF16;
  const float scale = c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / std::sqrt((float)c->head_dim);
  g->scale_log2e = scale * 1.4426950408889634f;
  g->per_head = g->least = g->items = g->slots = g->workers = g->grain = 0;
  return PQC_OK;
}

// What takes a call: a tile per query token, tiles of 16 rows, or (many queries per sequence) of 128 rows.
// Tiles of 128 rows from 64 rows per sequence on, which is the average: single tokens among prompts take a tile each (8 heads of 4 query heads, bf16
// output; us with tiles of 16 and of 128: one sequence of 17482 tokens, 32 rows 31.5, 42.4, 64 40.1, 42.9, 96 49.6, 44.3, 256 85.7, 51.6; sixteen
// of 4096, 32 rows 48.3, 58.1, 64 70.8, 62.4; with an fp32 output, one more product, 64 rows 40.1, 47.5 and 70.7, 75.1, 256 85.7, 57.4).  Their
// splits are of 512 tokens at least, since each leaves up to 64 KB of partial results (512 queries on themselves: splits of 256 28.8, of 512 22.3).
enum class Tiles { kOne, kRows, kBlock };
Tiles tiles_for(const pqc_paged_config* c, const Geometry& g, const int* offsets) {
  if (!offsets) return Tiles::kOne;
  return (long long)g.n_q * g.G >= 64ll * g.B ? Tiles::kBlock : Tiles::kRows;
}
// The kernel of 16 rows: workers, and units small enough for 32 bits over `tiles` tiles of at most `tokens` tokens.
void plan_rows(Geometry* g, long long tiles, long long tokens) {
  g->workers = std::max(1, kWorkers / g->Hkv);
  if (tiles * (tokens / kGrain) <= kFewUnits * g->workers) g->workers = std::max(1, g->workers / 2);
  g->grain = kGrain;
  while (tiles * (tokens / g->grain + 1 + kTileCost) >= (1ll << 30) - g->workers) g->grain *= 2;
  g->slots = tokens > g->grain ? 2 * g->workers : 0;  // else no border lies inside a tile
}
void plan_attn(Geometry* g, Tiles form) {
  g->R = form == Tiles::kOne ? 1 : (form == Tiles::kRows ? kRows : kBlockRows) / g->G;
  const long long tiles = form == Tiles::kOne ? g->B : std::min<long long>(g->n_q, (long long)g->n_q / g->R + g->B);
  if (form != Tiles::kBlock) {
    plan_rows(g, tiles, (long long)g->max_pages << g->shift);
    return;
  }
  g->per_head = std::max(1, (kBlockItems + g->Hkv - 1) / g->Hkv);
  g->least = 512;
  g->items = (int)tiles + g->per_head;
  g->slots = 2 * g->per_head;
}
void plan_listed(Geometry* g, int n_idx) {
  g->R = 1;
  plan_rows(g, g->B, n_idx);
}
size_t partial_bytes(const Geometry& g, int head_dim) {
  return ((size_t)g.slots * g.Hkv * partial_floats(g.R * g.G, head_dim) * sizeof(float) + 255) / 256 * 256;
}

// Of whichever form takes a call.
size_t attn_bytes(const pqc_paged_config* c, Geometry g) {
  plan_attn(&g, Tiles::kRows);
  const size_t rows = partial_bytes(g, c->head_dim);
  plan_attn(&g, Tiles::kBlock);
  return std::max(rows, partial_bytes(g, c->head_dim));
}

int check_cache(const pqc_paged_config* cfg, const pqc_paged_cache* c) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table || !c->lengths) return PQC_EINVAL;
  if (cfg->cache_dtype == PQC_FP8 && (!c->k_scale || !c->v_scale)) return PQC_EINVAL;
  if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16) || !aligned(c->page_table, 4) || !aligned(c->lengths, 4)) return PQC_EINVAL;
  if (!aligned(c->counters, 4)) return PQC_EINVAL;
  if (cfg->cache_dtype == PQC_FP8 && (!aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))) return PQC_EINVAL;
  return PQC_OK;
}
// Outputs in the pools, or over what says where things lie.
bool over_cache(const void* p, long long bytes, const pqc_paged_config* cfg, const pqc_paged_cache* c) {
  const long long rows = (long long)cfg->n_pages * cfg->n_kv_heads, pool = rows * cfg->page_tokens * cfg->head_dim * (cfg->cache_dtype == PQC_FP8 ? 1 : 2);
  const long long scales = cfg->cache_dtype == PQC_FP8 ? rows * 4 : 0;
  return meets_any(p, bytes, {bytes_at(c->k_pages, pool), bytes_at(c->v_pages, pool), bytes_at(c->k_scale, scales), bytes_at(c->v_scale, scales),
                              bytes_at(c->page_table, (long long)cfg->batch * cfg->max_pages * 4), bytes_at(c->lengths, cfg->batch * 4ll)});
}
// An attention call's output over what it reads or keeps its parts in.
bool out_overlaps(const pqc_paged_config* cfg, const pqc_paged_cache* c, const void* q, long long n, const int* offsets, const int* idx, long long n_idx,
                  const void* out, const void* workspace, long long workspace_bytes) {
  const long long values = n * cfg->n_q_heads * cfg->head_dim, bytes = values * (cfg->out_dtype == PQC_F32 ? 4 : 2);
  return over_cache(out, bytes, cfg, c) ||
         meets_any(out, bytes, {bytes_at(q, values * (cfg->io_dtype == PQC_F32 ? 4 : 2)), bytes_at(offsets, (cfg->batch + 1) * 4ll),
                                bytes_at(idx, (long long)cfg->batch * cfg->n_kv_heads * n_idx * 4), bytes_at(workspace, workspace_bytes)});
}
Cache device_cache(const pqc_paged_cache* c) {
  return Cache{static_cast<unsigned char*>(c->k_pages), static_cast<unsigned char*>(c->v_pages), c->k_scale, c->v_scale, c->page_table, c->lengths, c->counters};
}
int launched() { return hipGetLastError() == hipSuccess ? PQC_OK : PQC_EHIP; }

struct AttnCall {
  const Geometry& g;
  const Cache& c;
  const void* q;
  const int* offsets;
  const int* idx;
  int n_idx;
  void* out;
  float* partials;
  hipStream_t st;
};
template <typename T, class C, int D, bool LISTED>
void launch_rows(const AttnCall& a) {
  const Geometry& g = a.g;
  constexpr size_t lds = kRowsLds - rows_static_lds(D);
  Cache c = a.c;
  const int tokens = LISTED ? a.n_idx : g.max_pages << g.shift;
  if (std::min(g.workers / g.B, tokens / g.grain) > kPartsFolded) c.counters = nullptr;
  hipLaunchKernelGGL((attn_rows_kernel<T, C, D, LISTED>), dim3((unsigned)(g.workers * g.Hkv)), dim3(256), lds, a.st, g, c,
                     static_cast<const T*>(a.q), a.offsets, a.idx, a.n_idx, a.out, a.partials);
  if (g.workers > 1 && g.slots > 0 && !c.counters)
    hipLaunchKernelGGL((attn_fold_kernel<C, D>), dim3((unsigned)g.workers - 1, g.Hkv, g.R * g.G), dim3(256), 0, a.st, g, a.c.lengths,
                       a.offsets,                       LISTED ? a.n_idx : -1, a.partials, a.out);
}
template <typename T, class C, int D>
void launch_block(const AttnCall& a) {
  const Geometry& g = a.g;
  const dim3 grid((unsigned)(g.items * g.Hkv));
  if (g.out_bf16)
    hipLaunchKernelGGL((attn_block_kernel<T, C, D, 2>), grid, dim3(256), 0, a.st, g, a.c, static_cast<const T*>(a.q), a.offsets, a.out, a.partials);
  else
    hipLaunchKernelGGL((attn_block_kernel<T, C, D, 3>), grid, dim3(256), 0, a.st, g, a.c, static_cast<const T*>(a.q), a.offsets, a.out, a.partials);
  if ((g.max_pages << g.shift) <= g.least) return;  // no tile has several splits
  // tiles of several splits have two items at least; few tiles are folded by many workgroups each
  const int tiles = std::min(g.per_head, g.items - g.per_head), by = tiles * g.Hkv <= 128 ? 16 : 4;
  hipLaunchKernelGGL((attn_block_fold_kernel<D>), dim3((unsigned)tiles, g.Hkv, by), dim3(256), 0, a.st, g, a.c.lengths, a.offsets, a.partials, a.out);
}
// f(a query's type, a codec), by the configuration's types
template <class F>
void by_types(const pqc_paged_config* cfg, F f) {
  const bool f32 = cfg->io_dtype == PQC_F32, fp8 = cfg->cache_dtype == PQC_FP8;
  if (f32 && fp8) f(float{}, Fp8{});
  else if (f32) f(float{}, Bf16{});
  else if (fp8) f(bf16_t{}, Fp8{});
  else f(bf16_t{}, Bf16{});
}
int launch_blocks(const pqc_paged_config* cfg, const AttnCall& a) {
  by_types(cfg, [&](auto t, auto c) {
    if (cfg->head_dim == 128)
      launch_block<decltype(t), decltype(c), 128>(a);
    else
      launch_block<decltype(t), decltype(c), 64>(a);
  });
  return launched();
}
template <bool LISTED>
int launch_attn(const pqc_paged_config* cfg, const AttnCall& a) {
  by_types(cfg, [&](auto t, auto c) {
    if (cfg->head_dim == 128)
      launch_rows<decltype(t), decltype(c), 128, LISTED>(a);
    else
      launch_rows<decltype(t), decltype(c), 64, LISTED>(a);
  });
  return launched();
}

template <typename T, bool FP8, int D>
void launch_append(const Geometry& g, const Cache& c, const AppendArgs& a, const int* offsets, hipStream_t st) {
  const unsigned q_groups = a.q ? (unsigned)((g.n_q + a.q_tokens - 1) / a.q_tokens) : 0;
  hipLaunchKernelGGL((append_kernel<T, FP8, D>), dim3((unsigned)a.kv_items * 2 * g.Hkv + q_groups), dim3(256), 0, st, g, c, a, offsets);
}

}  // namespace

extern "C" {

size_t pqc_paged_counter_bytes(const pqc_paged_config* cfg) {
  Geometry g;
  if (make_geometry(cfg, 1, &g) != PQC_OK) return 0;
  return (size_t)std::max(1, kWorkers / g.Hkv) * g.Hkv * sizeof(unsigned);  // of as many workers as any call has
}

size_t pqc_paged_workspace_bytes(const pqc_paged_config* cfg, int32_t n, int32_t n_idx) {
  Geometry g;
  if (n_idx < 0 || make_geometry(cfg, n, &g) != PQC_OK) return 0;
  if (n_idx > 0)
    plan_listed(&g, n_idx);
  else
    return attn_bytes(cfg, g);
  return partial_bytes(g, cfg->head_dim);
}

int pqc_paged_attn(const pqc_paged_config* cfg, const pqc_paged_cache* cache, const void* q, int32_t n, const int32_t* offsets, void* out,
                   void* workspace, size_t workspace_bytes, void* stream) {
  Geometry g;
  int rc = make_geometry(cfg, n, &g);
  if (rc != PQC_OK) return rc;
  rc = check_cache(cfg, cache);
  if (rc != PQC_OK) return rc;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(offsets, 4) || (!offsets && n != g.B)) return PQC_EINVAL;
  const size_t need = attn_bytes(cfg, g);
  const Tiles form = tiles_for(cfg, g, offsets);
  plan_attn(&g, form);
  if ((long long)g.items * g.Hkv >= kMaxGroups) return PQC_EUNSUPPORTED;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return PQC_EWORKSPACE;
  if (n == 0) return PQC_OK;
  if (out_overlaps(cfg, cache, q, n, offsets, nullptr, 0, out, workspace, (long long)need)) return PQC_EINVAL;
  const Cache c = device_cache(cache);
  const AttnCall call{g, c, q, offsets, nullptr, 0, out, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)};
  return form == Tiles::kBlock ? launch_blocks(cfg, call) : launch_attn<false>(cfg, call);
}

int pqc_paged_gather_attn(const pqc_paged_config* cfg, const pqc_paged_cache* cache, const void* q, const int32_t* idx, int32_t n_idx, void* out,
                          void* workspace, size_t workspace_bytes, void* stream) {
  Geometry g;
  int rc = make_geometry(cfg, cfg ? cfg->batch : 0, &g);
  if (rc != PQC_OK) return rc;
  rc = check_cache(cfg, cache);
  if (rc != PQC_OK) return rc;
  if (!q || !out || !idx || n_idx < 1 || !aligned(q, 16) || !aligned(out, 16) || !aligned(idx, 4)) return PQC_EINVAL;
  if (n_idx > (1 << 24)) return PQC_EUNSUPPORTED;
  plan_listed(&g, n_idx);
  const size_t need = partial_bytes(g, cfg->head_dim);
  if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return PQC_EWORKSPACE;
  if (out_overlaps(cfg, cache, q, g.B, nullptr, idx, n_idx, out, workspace, (long long)need)) return PQC_EINVAL;
  const Cache c = device_cache(cache);
  return launch_attn<true>(cfg, AttnCall{g, c, q, nullptr, idx, n_idx, out, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)});
}

int pqc_paged_append(const pqc_paged_config* cfg, const pqc_paged_cache* cache, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                     const void* v, int64_t v_stride, int32_t n, const int32_t* offsets, const int32_t* positions, const float* rotation, void* q_out,
                     void* k_out, void* stream) {
  Geometry g;
  int rc = make_geometry(cfg, n, &g);
  if (rc != PQC_OK) return rc;
  rc = check_cache(cfg, cache);
  if (rc != PQC_OK) return rc;
  const int64_t q_row = (int64_t)g.Hq * cfg->head_dim, kv_row = (int64_t)g.Hkv * cfg->head_dim;
  if (!k || !v || (q && !q_out) || (cfg->rot_dims && !rotation) || (!offsets && n != g.B)) return PQC_EINVAL;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) || !aligned(rotation, 16) ||
      !aligned(offsets, 4) || !aligned(positions, 4))
    return PQC_EINVAL;
  if (k_stride < kv_row || v_stride < kv_row || k_stride % 8 || v_stride % 8 || (q && (q_stride < q_row || q_stride % 8))) return PQC_EINVAL;
  if (n == 0) return PQC_OK;
  AppendArgs a;
  a.q = q; a.k = k; a.v = v;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.positions = positions;
  a.table = rotation;
  a.rot = cfg->rot_dims; a.rot_positions = cfg->rot_positions;
  a.pairs = cfg->rot_style == PQC_ROT_PAIRS;
  a.q_out = q_out; a.k_out = k_out;
  // Query tokens per workgroup: two share a workgroup's heads as soon as there are several workgroups per compute unit (32768 tokens, 32 query
  // heads, 8 KV heads: one 175 us, two 161, four 162, eight 168, 32 197; 4096 tokens 20.3, 19.9, 20.3, 21.6; before pages were put together).
  a.q_tokens = n >= 1024 ? 2 : 1;
  // a sequence of m tokens touches at most 1 + (m + P - 2) / P pages, and no more than m
  long long pages = offsets ? std::min<long long>(n, (long long)n / g.P + 2ll * g.B) : n;
  a.together = pages >= kTogether ? 8 : 1;
  pages = (pages + a.together - 1) / a.together * a.together;
  if (pages * 2 * g.Hkv + (q ? (n + a.q_tokens - 1) / a.q_tokens : 0) >= kMaxGroups) return PQC_EUNSUPPORTED;
  a.kv_items = (int)pages;
  // other workgroups may read an input after a workgroup has stored its part of an output
  const int e = cfg->io_dtype == PQC_F32 ? 4 : 2;
  const Rows in[] = {{q, n, q_row * e, q_stride * e}, {k, n, kv_row * e, k_stride * e}, {v, n, kv_row * e, v_stride * e}, bytes_at(offsets, (g.B + 1) * 4ll),
                     bytes_at(positions, n * 4ll), bytes_at(rotation, (long long)cfg->rot_positions * cfg->rot_dims * 4)};
  const long long q_bytes = q ? n * q_row * e : 0, k_bytes = n * kv_row * e;
  if (meets_any(q_out, q_bytes, in) || meets_any(k_out, k_bytes, in) || meets(k_out, k_bytes, bytes_at(q_out, q_bytes)) || over_cache(q_out, q_bytes, cfg, cache) ||
      over_cache(k_out, k_bytes, cfg, cache))
    return PQC_EINVAL;
  const Cache c = device_cache(cache);
  hipStream_t st = static_cast<hipStream_t>(stream);
  auto by_dim = [&](auto t, auto fp8) {
    if (cfg->head_dim == 128)
      launch_append<decltype(t), decltype(fp8)::value, 128>(g, c, a, offsets, st);
    else
      launch_append<decltype(t), decltype(fp8)::value, 64>(g, c, a, offsets, st);
  };
  const bool f32 = cfg->io_dtype == PQC_F32, fp8 = cfg->cache_dtype == PQC_FP8;
  if (f32 && fp8) by_dim(float{}, std::true_type{});
  else if (f32) by_dim(float{}, std::false_type{});
  else if (fp8) by_dim(bf16_t{}, std::true_type{});
  else by_dim(bf16_t{}, std::false_type{});
  return launched();
}

}  // extern "C"
