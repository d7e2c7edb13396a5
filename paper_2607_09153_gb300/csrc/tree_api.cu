// kvprm_tree_workspace, kvprm_tree_attention: argument checks and the choice of the launch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "rope.h"
#include "tree.h"

using namespace kvprm;

namespace {

constexpr int64_t kTicketBytes = 4 * kTreeTickets;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct TreePlan {
  bool tc = false;
  int ctas = 0, rows = 16;   // rows: of a partial result
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

// More than 16 rows of a kv head go to the tensor cores.  CTAs: as many as run at once, but no more than one per pair
// while pairs are short (a pair in one CTA needs no joining), and a few blocks for each where they are long.
TreePlan plan(const kvprm_cache& c, const kvprm_tree& t, int sms) {
  TreePlan p;
  const int64_t rows = int64_t{t.max_drafts} * (t.n_q_heads / c.n_kv_heads);
  p.tc = rows > 16 && c.n_pages > 0;
  p.rows = p.tc ? 256 : 16;
  const int64_t block = p.tc ? 128 : kTreePage, least = p.tc ? 4 : 16;
  const int64_t len = std::min<int64_t>(t.max_len, int64_t{kTreePage} * t.max_blocks);
  const int64_t pairs = std::min<int64_t>(t.n_seqs, kTreeSeqs) * c.n_kv_heads * ceil_div(rows, p.rows);
  const int64_t blocks = ceil_div(len, block) + ceil_div(t.max_drafts, block);
  const int64_t most = std::min<int64_t>(int64_t{sms} * (p.tc ? 1 : kTreeRows16PerSm), kTreeTickets - 1);
  p.ctas = static_cast<int>(std::max<int64_t>(1, std::min(most, std::max(pairs, pairs * blocks / least))));
  return p;
}

int64_t workspace_bytes(const kvprm_cache& c, const TreePlan& p) {
  return kTicketBytes + int64_t{2} * p.ctas * p.rows * (4 * c.head_dim + 8);
}

}  // namespace

extern "C" {

int kvprm_tree_workspace(const kvprm_cache* cache, const kvprm_tree* t, int64_t* bytes) {
  const char* who = "kvprm_tree_workspace";
  if (!bytes) return operator_fail(KVPRM_EINVAL, "%s: bytes is NULL", who);
  if (const int rc = check(cache, t, who)) return rc;
  int sms = 0;
  if (const int rc = sm_count(&sms)) return rc;
  *bytes = workspace_bytes(*cache, plan(*cache, *t, sms));
  return KVPRM_OK;
}

int kvprm_tree_attention(const kvprm_cache* cache, const kvprm_tree* t, void* workspace, int64_t workspace_size,
                         void* stream) {
  const char* who = "kvprm_tree_attention";
  if (const int rc = check(cache, t, who)) return rc;
  if (t->n_seqs == 0 || t->n_tokens == 0) return KVPRM_OK;
  if (!t->q || !t->k || !t->v || !t->out || !t->lens || !t->start || (t->max_blocks > 0 && !t->block_table))
    return operator_fail(KVPRM_EINVAL, "%s: NULL argument", who);
  if (!aligned16(t->q) || !aligned16(t->k) || !aligned16(t->v) || !aligned16(t->out) ||
      ((t->q_token | t->q_head | t->k_token | t->k_head | t->v_token | t->v_head | t->out_token | t->out_head) & 7) != 0)
    return operator_fail(KVPRM_EINVAL, "%s: rows of q, k, v and out have to be 16-byte aligned", who);
  int sms = 0;
  if (const int rc = sm_count(&sms)) return rc;
  const TreePlan p = plan(*cache, *t, sms);
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
  a.scale_log2 = t->scale * 1.4426950408889634f;
  a.tickets = static_cast<int32_t*>(workspace);
  a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kTicketBytes);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + int64_t{2} * p.ctas * p.rows * cache->head_dim);
  for (a.seq0 = 0; a.seq0 < t->n_seqs; a.seq0 += kTreeSeqs) {
    a.n_seqs = std::min(kTreeSeqs, t->n_seqs - a.seq0);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = p.tc ? launch_tree_tc(a, *cache, p.ctas, st) : launch_tree_rows16(a, *cache, p.ctas, st);
    if (e != cudaSuccess) return operator_fail(KVPRM_ECUDA, "%s: %s", who, cudaGetErrorString(e));
  }
  return KVPRM_OK;
}

}  // extern "C"
