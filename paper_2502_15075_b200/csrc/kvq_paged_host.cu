// C-ABI of the paged cache: argument checks and dispatch.
#include <math.h>

#include "kvq_debug.h"
#include "kvq_paged.cuh"

using namespace kvq;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool paged_width(int b) { return b == 2 || b == 4 || b == 8; }

constexpr int kMaxBatch = 1024;

// The configurations that a paged cache may have.
int paged_geom(const kvq_config* cfg, Geom* g) {
  const int rc = make_geom(cfg, g);
  if (rc != KVQ_OK) return rc;
  if (g->k_axis != 0 || g->R != 0 || !paged_width(g->kb) || !paged_width(g->vb) || g->B > kMaxBatch) return KVQ_ERR_UNSUPPORTED;
  return KVQ_OK;
}

int paged_args(const Geom& g, const kvq_paged_cache* c, const int32_t* cu, int32_t n_rows, Paged* p) {
  if (!c || !c->pages || !c->block_table || !c->seq_len || !c->status || !cu) return KVQ_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->table_stride < g.n_pages || n_rows < 0) return KVQ_ERR_INVALID_ARG;
  if (!aligned16(c->pages)) return KVQ_ERR_MISALIGNED;
  *p = Paged{static_cast<uint8_t*>(c->pages), c->block_table, c->table_stride, c->seq_len, cu, reinterpret_cast<uint32_t*>(c->status),
             c->n_pages, n_rows, 0, 0, 0, 0};
  return KVQ_OK;
}

// Rows of `D` 16-bit elements at 16-byte boundaries (a stride that is never taken does not matter).
int rows_ok(const Geom& g, const void* x, int64_t row, int64_t head, int heads, int n_rows) {
  if ((n_rows > 1 && row < g.D) || (heads > 1 && head < g.D)) return KVQ_ERR_INVALID_ARG;
  return !aligned16(x) || (n_rows > 1 && row % 8) || (heads > 1 && head % 8) ? KVQ_ERR_MISALIGNED : KVQ_OK;
}

// The workspace begins with the decode kernel's count words, one per stream, whichever kernel serves the call; the last ones end at a multiple of 16.
size_t count_words_bytes(const Geom& g) { return ((size_t)g.B * g.Hkv * 8 + 15) & ~(size_t)15; }
size_t paged_workspace_bytes(const Geom& g) {
  const size_t decode = paged_decode_workspace_bytes(g), chunk = paged_chunk_workspace_bytes(g);
  return count_words_bytes(g) + (decode > chunk ? decode : chunk);
}

// The most rows of a sequence that an attention call can have: max_rows may be any bound, but no sequence has more rows than tokens.
int32_t bounded_rows(const Geom& g, int32_t max_rows) { return max_rows < g.capacity ? max_rows : g.capacity; }

// What an attention call announces.
void set_rows(Geom* g, Paged* p, int32_t max_rows, int32_t window, int32_t sinks) {
  g->rows = p->max_rows = bounded_rows(*g, max_rows);
  p->window = window;
  p->sinks = sinks;
}

int attention_with(const DecodeDebug& dbg, const kvq_config* cfg, const kvq_paged_cache* cache, const void* q, const int32_t* cu, int32_t n_rows,
                   int32_t max_rows, int32_t window, int32_t sinks, void* out, int32_t out_dtype, float softmax_scale,
                   void* workspace, size_t workspace_bytes, void* cuda_stream) {
  Geom g;
  Paged p;
  int rc = paged_geom(cfg, &g);
  if (rc == KVQ_OK) rc = paged_args(g, cache, cu, n_rows, &p);
  if (rc != KVQ_OK) return rc;
  if (max_rows < 1 || window < 0 || sinks < 0) return KVQ_ERR_INVALID_ARG;
  if (n_rows == 0) return KVQ_OK;
  if (!q || !out || !workspace) return KVQ_ERR_INVALID_ARG;
  if (out_dtype != KVQ_FP16 && out_dtype != KVQ_BF16 && out_dtype != KVQ_FP32) return KVQ_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return KVQ_ERR_MISALIGNED;
  set_rows(&g, &p, max_rows, window, sinks);
  if (workspace_bytes < paged_workspace_bytes(g)) return KVQ_ERR_WORKSPACE_TOO_SMALL;
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)g.D);
  const float c1 = scale * 1.4426950408889634f;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto launch = paged_decode_serves(g, p) ? launch_paged_decode : launch_paged_chunk;
  return launch(g, p, q, out, out_dtype, c1, reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + count_words_bytes(g)), dbg, stream);
}

}  // namespace

extern "C" {

int kvq_paged_append(const kvq_config* cfg, const kvq_paged_cache* cache, const void* k, const void* v, int64_t kv_stride_row,
                     int64_t kv_stride_head, const int32_t* cu, int32_t n_rows, const kvq_rope* rope, const void* q,
                     int64_t q_stride_row, int64_t q_stride_head, void* q_out, void* cuda_stream) {
  Geom g;
  Paged p;
  int rc = paged_geom(cfg, &g);
  if (rc == KVQ_OK) rc = paged_args(g, cache, cu, n_rows, &p);
  if (rc != KVQ_OK) return rc;
  if (n_rows == 0) return KVQ_OK;
  if (!k || !v || (q == nullptr) != (q_out == nullptr) || (q && !rope)) return KVQ_ERR_INVALID_ARG;
  rc = rows_ok(g, k, kv_stride_row, kv_stride_head, g.Hkv, n_rows);
  if (rc == KVQ_OK && !aligned16(v)) rc = KVQ_ERR_MISALIGNED;
  if (rc == KVQ_OK && q) rc = rows_ok(g, q, q_stride_row, q_stride_head, g.Hq, n_rows);
  if (rc == KVQ_OK && !aligned16(q_out)) rc = KVQ_ERR_MISALIGNED;
  if (rc != KVQ_OK) return rc;
  // in place only row by row: anything else would be read after it was overwritten
  if (q && q == q_out && ((g.Hq > 1 && q_stride_head != g.D) || (n_rows > 1 && q_stride_row != (int64_t)g.Hq * g.D))) return KVQ_ERR_INVALID_ARG;
  RopeArgs r{nullptr, nullptr, 0, 0, 0};
  if (rope) {
    if (!rope->cos || !rope->sin || rope->n_positions < 1 || rope->rotary_dim < 16 || rope->rotary_dim > g.D || rope->rotary_dim % 16 ||
        (rope->interleaved != 0 && rope->interleaved != 1))
      return KVQ_ERR_INVALID_ARG;
    if (!aligned16(rope->cos) || !aligned16(rope->sin)) return KVQ_ERR_MISALIGNED;
    r = RopeArgs{rope->cos, rope->sin, rope->n_positions, rope->rotary_dim / 2, rope->interleaved};
  }
  return launch_paged_append(g, p, k, v, kv_stride_row, kv_stride_head, r, q, q_stride_row, q_stride_head, q_out,
                             static_cast<cudaStream_t>(cuda_stream));
}

int kvq_paged_workspace_bytes(const kvq_config* cfg, int32_t max_rows, size_t* out) {
  Geom g;
  const int rc = paged_geom(cfg, &g);
  if (rc != KVQ_OK) return rc;
  if (!out || max_rows < 1) return KVQ_ERR_INVALID_ARG;
  g.rows = bounded_rows(g, max_rows);
  *out = paged_workspace_bytes(g);
  return KVQ_OK;
}

int kvq_paged_attention(const kvq_config* cfg, const kvq_paged_cache* cache, const void* q, const int32_t* cu, int32_t n_rows,
                        int32_t max_rows, int32_t window, int32_t sinks, void* out, int32_t out_dtype, float softmax_scale,
                        void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return attention_with(DecodeDebug{}, cfg, cache, q, cu, n_rows, max_rows, window, sinks, out, out_dtype, softmax_scale, workspace,
                        workspace_bytes, cuda_stream);
}

int kvq_debug_paged_stall(const kvq_config* cfg, const kvq_paged_cache* cache, const void* q, const int32_t* cu, int32_t n_rows,
                          int32_t max_rows, int32_t window, int32_t sinks, void* out, int32_t out_dtype, void* workspace,
                          size_t workspace_bytes, int64_t skip_page, uint32_t wait_us, void* cuda_stream) {
  if (wait_us == 0 || wait_us > 100000u) return KVQ_ERR_INVALID_ARG;      // the hook never waits longer than 0.1 s
  DecodeDebug dbg;
  dbg.skip_page = skip_page;
  dbg.wait_us = wait_us;
  return attention_with(dbg, cfg, cache, q, cu, n_rows, max_rows, window, sinks, out, out_dtype, 0.0f, workspace, workspace_bytes,
                        cuda_stream);
}

int kvq_debug_paged_launches(const kvq_config* cfg, int32_t max_rows, int32_t window, int32_t sinks, int32_t* launches) {
  Geom g;
  const int rc = paged_geom(cfg, &g);
  if (rc != KVQ_OK) return rc;
  if (!launches || max_rows < 1 || window < 0 || sinks < 0) return KVQ_ERR_INVALID_ARG;
  Paged p{};
  set_rows(&g, &p, max_rows, window, sinks);
  *launches = paged_decode_launches(g, p);
  return KVQ_OK;
}

int kvq_paged_dequantize(const kvq_config* cfg, const kvq_paged_cache* cache, const int32_t* cu, int32_t n_rows, void* k_out,
                         void* v_out, void* cuda_stream) {
  Geom g;
  Paged p;
  int rc = paged_geom(cfg, &g);
  if (rc == KVQ_OK) rc = paged_args(g, cache, cu, n_rows, &p);
  if (rc != KVQ_OK) return rc;
  if (!aligned16(k_out) || !aligned16(v_out)) return KVQ_ERR_MISALIGNED;
  if (n_rows == 0 || (!k_out && !v_out)) return KVQ_OK;
  return launch_paged_dequantize(g, p, k_out, v_out, static_cast<cudaStream_t>(cuda_stream));
}

int kvq_paged_check_status(const kvq_paged_cache* cache, void* cuda_stream) {
  if (!cache || !cache->status) return KVQ_ERR_INVALID_ARG;
  kvq_cache c = {};
  c.status = cache->status;
  return kvq_check_status(&c, cuda_stream);
}

}  // extern "C"
