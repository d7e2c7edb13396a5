// kvprm_tree_workspace, kvprm_tree_attention: argument checks and the choice of the launch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "rope.h"
#include "tree.h"

using namespace kvprm;

namespace {

constexpr int64_t kLineBytes = (4 * (kTreeSeqs + 2) + 255) / 256 * 256;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct TreePlan {
  bool tc = false, whole = false;
  int ctas = 0, rows = 16, seqs = 0;   // rows: of a partial result; seqs: sequences of a launch
};

int check(const kvprm_cache* c, const kvprm_tree* t, const char* who) {
  if (const int rc = check_cache(c, who)) return rc;
  if (!t) return operator_fail(KVPRM_EINVAL, "%s: no arguments", who);
  if (t->n_seqs < 0 || t->n_tokens < 0 || t->max_blocks < 0 || t->max_len < 0)
    return operator_fail(KVPRM_EINVAL, "%s: n_seqs %d, n_tokens %d, max_blocks %d, max_len %d", who, t->n_seqs, t->n_tokens,
                         t->max_blocks, t->max_len);
  if (t->n_q_heads < 1 || t->n_q_heads > 1024 || t->n_q_heads % c->n_kv_heads != 0)
    return operator_fail(KVPRM_EINVAL, "%s: %d query heads over %d key heads", who, t->n_q_heads, c->n_kv_heads);
  if (t->max_drafts < 1 || t->max_drafts > 1024)
    return operator_fail(KVPRM_EINVAL, "%s: max_drafts %d is not in 1 .. 1024", who, t->max_drafts);
  if (t->mask && t->mask_words < (t->max_drafts + 31) / 32)
    return operator_fail(KVPRM_EINVAL, "%s: %d mask words for %d drafts", who, t->mask_words, t->max_drafts);
  if (!std::isfinite(t->scale)) return operator_fail(KVPRM_EINVAL, "%s: scale is not finite", who);
  return KVPRM_OK;
}

int sm_count(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return operator_fail(KVPRM_ECUDA, "kvprm_tree: no device");
  return KVPRM_OK;
}

// More than 32 rows of a kv head go to the tensor cores (us a call, registers / tensor cores: 8 heads with 24 rows over ragged
// 20,000 bf16 tokens 76 / 78, 8-bit 66 / 89; with 32 over 8 x 32,768 bf16 tokens 187 / 186, 8-bit 155 / 221; 4 heads with 63 over
// 16 x 9,001 8-bit tokens 97 / 80; 2 heads with 42 over ragged 1,000 bf16 tokens 19 / 21, with 126 22 / 21).  CTAs: as many as
// run at once.  Pairs that have a CTA each and few blocks stay whole, for a cut one needs the join (cut / whole: registers, 2 x 8
// heads over 400 tokens 18 / 13, 16 x 4 heads with 28 rows 21 / 15, over 900 22 / 25; tensor cores, 16 x 2 heads with 126 rows
// over ragged 300 8-bit tokens 23 / 18, over 600 21 / 23); where CTAs have several, uneven shares cost more, and fewer do.
int plan(const kvprm_cache& c, const kvprm_tree& t, int sms, TreePlan* out) {
  TreePlan p;
  const int64_t rows = int64_t{t.max_drafts} * (t.n_q_heads / c.n_kv_heads);
  p.tc = rows > 32 && c.n_pages > 0;
  p.rows = p.tc ? 256 : rows > 16 ? 32 : 16;
  const int64_t block = p.tc ? 128 : kTreePage, tiles = ceil_div(rows, p.tc ? 128 : p.rows), lead = 20;
  // the line of a sequence of any length is shorter than this; a launch's stays within 31 bits
  const int64_t depth = ceil_div(int64_t{kTreePage} * t.max_blocks, block) + ceil_div(t.max_drafts, block) + lead;
  const int64_t line = depth * (p.tc ? 4 * ceil_div(tiles, 2) : tiles) * c.n_kv_heads;
  if (line > 0x7FFFFFFF) return operator_fail(KVPRM_ECAPACITY, "kvprm_tree: block tables of %d pages", t.max_blocks);
  p.seqs = static_cast<int>(std::min<int64_t>({t.n_seqs, kTreeSeqs, 0x7FFFFFFF / line}));
  const int64_t len = std::min<int64_t>(t.max_len, int64_t{kTreePage} * t.max_blocks);
  const int64_t pairs = int64_t{p.seqs} * c.n_kv_heads * ceil_div(rows, p.rows);
  const int64_t blocks = ceil_div(len, block) + ceil_div(t.max_drafts, block);
  const int64_t most = int64_t{sms} * (p.tc ? 1 : tree_rows_per_sm(p.rows / 16));
  p.whole = blocks <= (pairs <= most ? (p.tc ? 4 : 32) : (p.tc ? 3 : 16));
  p.ctas = static_cast<int>(std::max<int64_t>(1, std::min(most, p.whole ? pairs : pairs * blocks / (p.tc ? 2 : 8))));
  *out = p;
  return KVPRM_OK;
}

int64_t workspace_bytes(const kvprm_cache& c, const TreePlan& p) {
  return kLineBytes + (p.whole ? 0 : int64_t{2} * p.ctas * p.rows * (4 * c.head_dim + 8));
}

int attend(const kvprm_cache* cache, const kvprm_tree* t, void* workspace, int64_t workspace_size, void* stream, bool fill,
           const char* who) {
  if (const int rc = check(cache, t, who)) return rc;
  if ((t->n_seqs == 0 && !fill) || t->n_tokens == 0) return KVPRM_OK;
  const bool seqs = t->n_seqs > 0;
  if (!t->q || !t->k || !t->v || !t->out || !t->start || (seqs && !t->lens) || (seqs && t->max_blocks > 0 && !t->block_table))
    return operator_fail(KVPRM_EINVAL, "%s: NULL argument", who);
  // (the stride of a dimension of one is nobody's)
  int64_t strides = t->n_tokens > 1 ? t->q_token | t->k_token | t->v_token | t->out_token : 0;
  if (t->n_q_heads > 1) strides |= t->q_head | t->out_head;
  if (cache->n_kv_heads > 1) strides |= t->k_head | t->v_head;
  if (!aligned16(t->q) || !aligned16(t->k) || !aligned16(t->v) || !aligned16(t->out) || (strides & 7) != 0)
    return operator_fail(KVPRM_EINVAL, "%s: rows of q, k, v and out have to be 16-byte aligned", who);
  int sms = 0;
  if (const int rc = sm_count(&sms)) return rc;
  TreePlan p;
  if (const int rc = plan(*cache, *t, sms, &p)) return rc;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return operator_fail(KVPRM_EINVAL, "%s: workspace is NULL or not 256-byte aligned", who);
  if (workspace_size < workspace_bytes(*cache, p))
    return operator_fail(KVPRM_ECAPACITY, "%s: a workspace of %lld bytes, %lld needed", who, static_cast<long long>(workspace_size),
                         static_cast<long long>(workspace_bytes(*cache, p)));
  TreeLaunch a;
  a.t = *t;
  a.pages = static_cast<const uint8_t*>(cache->pages);
  a.exponents = static_cast<const uint8_t*>(cache->exponents);
  a.n_pages = cache->n_pages;
  a.n_kv = cache->n_kv_heads;
  a.group = t->n_q_heads / cache->n_kv_heads;
  a.group_m = a.group > 1 ? static_cast<uint32_t>(((uint64_t{1} << 32) + a.group - 1) / a.group) : 0u;
  a.scale_log2 = t->scale * 1.4426950408889634f;
  a.whole = p.whole;
  a.fill = fill;
  // a chunk with one row tile costs the tensor-core kernel, by what it waits for, 0.75 of one with two (a bf16 cache: memory)
  // or as much (an 8-bit one: its conversion)
  a.weight_full = p.tc ? 4 : 1;
  a.weight_part = !p.tc ? 1 : cache->format == KVPRM_CACHE_E4M3 ? 4 : 3;
  a.line = static_cast<int32_t*>(workspace);
  a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kLineBytes);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + int64_t{2} * p.ctas * p.rows * cache->head_dim);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.seq0 = 0;
  do {   // (once without sequences, which is to fill only)
    a.n_seqs = std::min(p.seqs, t->n_seqs - a.seq0);
    cudaError_t e = p.tc ? launch_tree_tc(a, *cache, p.ctas, st) : launch_tree_rows(a, *cache, p.rows / 16, p.ctas, st);
    if (e == cudaSuccess && !p.whole && seqs) e = launch_tree_join(a, *cache, p.rows, st);
    if (e != cudaSuccess) return operator_fail(KVPRM_ECUDA, "%s: %s", who, cudaGetErrorString(e));
    a.seq0 += p.seqs;
  } while (a.seq0 < t->n_seqs);
  return KVPRM_OK;
}

}  // namespace

extern "C" {

int kvprm_tree_workspace(const kvprm_cache* cache, const kvprm_tree* t, int64_t* bytes) {
  const char* who = "kvprm_tree_workspace";
  if (!bytes) return operator_fail(KVPRM_EINVAL, "%s: bytes is NULL", who);
  if (const int rc = check(cache, t, who)) return rc;
  int sms = 0;
  if (const int rc = sm_count(&sms)) return rc;
  TreePlan p;
  if (const int rc = plan(*cache, *t, sms, &p)) return rc;
  *bytes = workspace_bytes(*cache, p);
  return KVPRM_OK;
}

int kvprm_tree_attention(const kvprm_cache* cache, const kvprm_tree* t, void* workspace, int64_t workspace_bytes,
                         void* stream) {
  return attend(cache, t, workspace, workspace_bytes, stream, false, "kvprm_tree_attention");
}

int kvprm_tree_attention_filled(const kvprm_cache* cache, const kvprm_tree* t, void* workspace, int64_t workspace_bytes,
                                void* stream) {
  return attend(cache, t, workspace, workspace_bytes, stream, true, "kvprm_tree_attention_filled");
}

}  // extern "C"
