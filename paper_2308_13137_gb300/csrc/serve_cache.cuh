// Rows of a serving call: which rows of the packed [total_q, ...] arrays belong to a sequence and how
// many tokens its cache holds, with every value that comes from device memory checked.
#pragma once
#include "common.cuh"

struct SeqRows { int row0, nq, len; bool ok; };

__device__ __forceinline__ SeqRows seq_rows(const omq_kv_cache& c, const int32_t* cu_q, int max_q, int total_q, int b) {
  SeqRows s;
  s.len = __ldg(c.kv_len + b);
  if (cu_q) {
    s.row0 = __ldg(cu_q + b);
    const int end = __ldg(cu_q + b + 1);
    s.ok = s.row0 >= 0 && end >= s.row0 && end <= total_q && end - s.row0 <= max_q;
    s.nq = s.ok ? end - s.row0 : 0;
  } else {
    s.row0 = b * max_q;
    s.nq = max_q;
    s.ok = true;
  }
  if (s.len < 0) { s.ok = false; s.len = 0; }
  return s;
}

// checks shared by the calls that take a cache
static inline omq_status kv_check(const omq_kv_cache* c, int32_t total_q, int32_t max_q, const int32_t* cu_q,
                                  int32_t n_heads) {
  OMQ_REQUIRE(c && c->k && c->v && c->k_scale && c->v_scale && c->page_table && c->kv_len, OMQ_ERR_INVALID_ARG);
  OMQ_REQUIRE(c->B > 0 && c->B <= 65535 && c->n_pages > 0 && c->n_kv > 0 && c->max_pages > 0, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(n_heads > 0 && n_heads % c->n_kv == 0 && n_heads <= 1024, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(max_q > 0 && total_q > 0 && max_q <= total_q, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(cu_q || (int64_t)c->B * max_q == total_q, OMQ_ERR_SHAPE);
  OMQ_REQUIRE(omq_aligned16(c->k) && omq_aligned16(c->v) && omq_aligned16(c->k_scale) && omq_aligned16(c->v_scale) &&
                  omq_aligned16(c->page_table) && omq_aligned16(c->kv_len) && omq_aligned16(cu_q),
              OMQ_ERR_ALIGN);
  return OMQ_OK;
}
