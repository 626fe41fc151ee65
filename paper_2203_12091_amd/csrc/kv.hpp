// Addresses inside the paged 8-bit cache and the checks of a batch's numbers.
#pragma once

#include "serve.hpp"

namespace fxpq {

// One sequence of a batch as a kernel uses it; ok only when its numbers agree
// with the host's bounds.
struct SeqDev {
  int first;  // row of its first new token in the call's tensors
  int fresh;  // new tokens
  int len;    // tokens in the cache, the new ones included
  bool ok;
};

__device__ inline SeqDev seq_of(const fxpq_kv_batch& b, int s) {
  SeqDev q;
  q.first = b.start[s];
  const int end = b.start[s + 1];
  q.len = b.length[s];
  q.fresh = end - q.first;
  q.ok = q.first >= 0 && end >= q.first && end <= b.tokens && q.fresh <= b.max_new && q.len >= q.fresh &&
         q.len <= b.max_len;
  return q;
}
__device__ inline SeqDev seq_of(const fxpq_kv_batch& b, int page, int s) {
  SeqDev q = seq_of(b, s);
  q.ok = q.ok && (q.len + page - 1) / page <= b.table_ld;
  return q;
}

// The same for a block that works on one sequence: in scalar registers.
__device__ inline SeqDev block_seq(SeqDev q) {
  return SeqDev{__builtin_amdgcn_readfirstlane(q.first), __builtin_amdgcn_readfirstlane(q.fresh),
                __builtin_amdgcn_readfirstlane(q.len), (bool)__builtin_amdgcn_readfirstlane((int)q.ok)};
}

// First byte of token slot `slot` of a page and head: K rows are whole, V rows
// come in 16-token blocks of [dim][16].
__device__ inline int64_t k_offset(const fxpq_kv_cache& c, int page, int head, int slot) {
  return (((int64_t)page * c.heads + head) * c.page + slot) * c.dim;
}
__device__ inline int64_t v_offset(const fxpq_kv_cache& c, int page, int head, int slot, int d) {
  return (((int64_t)page * c.heads + head) * c.page + (slot & ~15)) * c.dim + d * 16 + (slot & 15);
}

// First byte of token slot `slot` of a page of latents.
__device__ inline int64_t latent_offset(const fxpq_latent_cache& c, int page, int slot) {
  return ((int64_t)page * c.page + slot) * (c.latent + c.rope);
}

}  // namespace fxpq
