// The second and third kernel of attention behind shared prefixes, as the first one's file starts them.
#pragma once
#include "common.h"
#include "prefix_parts.h"

namespace elasto {

struct PrefixOwnArgs {
  int batch, heads_kv, group, head_dim;
  float scale_log2, down;
  int max_queries, q_rows, max_keys, kv_rows;
  const int* q_start;
  const int* kv_start;
  const int* kv_len;
  const uint16_t* q;
  long long q_row, q_head;
  const uint16_t* v;
  long long v_batch, v_row, v_head;
  uint16_t* out;
  long long out_row, out_head;
  int prefixes, max_prefix;
  const int* seq_start;
  const int* prefix_len;
  const uint16_t* pv;
  long long pv_batch, pv_row, pv_head;
  int hg, nsub, pair, split;
  int prefix_parts, own_split, own_parts;
  int fused;  // prefix_few_kernel joins its rows itself
  PrefixParts parts;
  int blocks;  // of rows, of a sequence and key head
  int join_blocks;  // of rows of a sequence over all heads, for the join
  Divisor by_join;
  Divisor by_split, by_blocks, by_heads_kv, by_group;
  int* status;
};
struct PrefixOwn {
  PrefixOwnArgs a;
  CUtensorMap k, v;
  int64_t units;
  bool bf, many, join_many;  // blocks of 64 rows; the join for many rows
};
elasto_status prefix_own_plan(const elasto_prefix_attention_args& u, const PrefixPlan& p, const PrefixParts& parts, float down, int* status,
                              PrefixOwn* own);
elasto_status prefix_own_launch(const PrefixOwn& own, cudaStream_t s);

}  // namespace elasto
