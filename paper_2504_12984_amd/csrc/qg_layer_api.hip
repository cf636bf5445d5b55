// C entry points of include/qg_layer.h: argument checks, then one launch.
#include <cmath>

#include "qg_layer.h"

using namespace qg;

namespace {

bool multiple(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool act_ok(int act) { return act == QG_F16 || act == QG_BF16; }

// 0: int8, 1: e4m3, -1: no cache type
int kv_kind(const qg_wtype& t) {
  if (t.kind == QG_INT && t.bits == 8 && t.ebits == 0 && t.mbits == 0) return 0;
  if (t.kind == QG_FLOAT && t.bits == 8 && t.ebits == 4 && t.mbits == 3) return 1;
  return -1;
}

constexpr int64_t MOST_ROWS = 1 << 24;

// What the three cache calls have in common.
int check_kv(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, const qg_wtype& type,
             int64_t num_blocks, const int32_t* row_start, const int32_t* kv_len, const int32_t* block_table, int64_t table_width,
             int64_t batch, int64_t rows, int64_t max_rows, int kv_heads, int head_dim, int act, KvParams* p) {
  if (!act_ok(act) || kv_heads < 1 || kv_heads > 65536 || head_dim < 1) return QG_EINVAL;
  const int kind = kv_kind(type);
  if (kind < 0) return wt_index(type) == -1 ? QG_EINVAL : QG_EUNSUPPORTED;       // a weight type, but not one of a cache
  if (head_dim != 64 && head_dim != 128) return QG_EUNSUPPORTED;
  if (batch < 0 || batch > MOST_ROWS || rows < 0 || rows > MOST_ROWS || max_rows < 0) return QG_EINVAL;
  if (num_blocks < 1 || num_blocks > INT32_MAX || table_width < 1 || table_width > INT32_MAX) return QG_EINVAL;
  if (batch == 0 || rows == 0 || max_rows == 0) return QG_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !row_start || !kv_len || !block_table) return QG_EINVAL;
  if (!multiple(k_cache, 16) || !multiple(v_cache, 16) || !multiple(k_scale, 4) || !multiple(v_scale, 4) ||
      !multiple(row_start, 4) || !multiple(kv_len, 4) || !multiple(block_table, 4)) return QG_EINVAL;
  p->k_cache = const_cast<uint8_t*>(static_cast<const uint8_t*>(k_cache));
  p->v_cache = const_cast<uint8_t*>(static_cast<const uint8_t*>(v_cache));
  p->k_scale = const_cast<float*>(k_scale);
  p->v_scale = const_cast<float*>(v_scale);
  p->row_start = row_start; p->kv_len = kv_len; p->table = block_table;
  p->width = table_width; p->num_blocks = num_blocks;
  p->batch = (int)batch; p->rows = (int)rows; p->max_rows = (int)(max_rows < rows ? max_rows : rows);
  p->kv_heads = kv_heads; p->bf16 = act == QG_BF16; p->e4m3 = kind;
  return QG_OK;
}

int rows_to_8_bits(RowsParams& p, bool norm, int act, int64_t M, int64_t N, int8_t* A8, float* a_scale, void* stream) {
  p.A8 = A8; p.a_scale = a_scale; p.M = M; p.N = (int)N; p.bf16 = act == QG_BF16;
  // wide: every row that is there starts at a multiple of 16 bytes
  p.wide = N % 8 == 0 && multiple(p.x, 16) && p.x_stride % 8 == 0 && multiple(A8, 8) &&
           (!p.y || (multiple(p.y, 16) && p.y_stride % 8 == 0)) && (!p.w || multiple(p.w, 16)) &&
           (!p.sum || (multiple(p.sum, 16) && p.sum_stride % 8 == 0));
  hipStream_t st = static_cast<hipStream_t>(stream);
  return norm ? layer_norm_launch(p, st) : layer_gate_launch(p, st);
}

}  // namespace

extern "C" {

int qg_rmsnorm_a8(const void* x, const void* residual, const void* weight, float eps, int act, int64_t M, int64_t N,
                  int64_t x_stride, int64_t residual_stride, int8_t* A8, float* a_scale, void* sum_out, int64_t sum_stride,
                  void* stream) {
  if (!act_ok(act) || M < 0 || M > MOST_ROWS || N < 1 || N > MOST_ROWS || !(eps >= 0.0f)) return QG_EINVAL;
  if (x_stride < N || (residual && residual_stride < N) || (sum_out && sum_stride < N)) return QG_EINVAL;
  if (M == 0) return QG_OK;
  if (!x || !weight || !A8 || !a_scale) return QG_EINVAL;
  if (!multiple(x, 2) || !multiple(residual, 2) || !multiple(weight, 2) || !multiple(sum_out, 2) || !multiple(a_scale, 4)) return QG_EINVAL;
  RowsParams p = {};
  p.x = static_cast<const uint16_t*>(x); p.x_stride = x_stride;
  p.y = static_cast<const uint16_t*>(residual); p.y_stride = residual ? residual_stride : 0;
  p.w = static_cast<const uint16_t*>(weight);
  p.sum = static_cast<uint16_t*>(sum_out); p.sum_stride = sum_out ? sum_stride : 0;
  p.eps = eps;
  return rows_to_8_bits(p, true, act, M, N, A8, a_scale, stream);
}

int qg_silu_a8(const void* gate, const void* up, int act, int64_t M, int64_t N, int64_t gate_stride, int64_t up_stride,
               int8_t* A8, float* a_scale, void* stream) {
  if (!act_ok(act) || M < 0 || M > MOST_ROWS || N < 1 || N > MOST_ROWS) return QG_EINVAL;
  if (gate_stride < N || up_stride < N) return QG_EINVAL;
  if (M == 0) return QG_OK;
  if (!gate || !up || !A8 || !a_scale) return QG_EINVAL;
  if (!multiple(gate, 2) || !multiple(up, 2) || !multiple(a_scale, 4)) return QG_EINVAL;
  RowsParams p = {};
  p.x = static_cast<const uint16_t*>(gate); p.x_stride = gate_stride;
  p.y = static_cast<const uint16_t*>(up); p.y_stride = up_stride;
  return rows_to_8_bits(p, false, act, M, N, A8, a_scale, stream);
}

int qg_kv_append(const void* q, const void* k, const void* v, int act, int64_t q_stride, int64_t k_stride, int64_t v_stride,
                 const float* cos, const float* sin, int64_t positions, int rot_dim, int neighbours,
                 const int32_t* row_start, const int32_t* kv_len, const int32_t* block_table, int64_t table_width,
                 int64_t batch, int64_t rows, int64_t max_rows, int q_heads, int kv_heads, int head_dim, qg_wtype type,
                 int64_t num_blocks, void* k_cache, void* v_cache, float* k_scale, float* v_scale, void* q_out, void* stream) {
  KvParams p = {};
  const int rc = check_kv(k_cache, v_cache, k_scale, v_scale, type, num_blocks, row_start, kv_len, block_table, table_width, batch,
                          rows, max_rows, kv_heads, head_dim, act, &p);
  if (rc != QG_OK) return rc;
  if (!cos != !sin || rot_dim < 0 || rot_dim > head_dim || rot_dim % 2) return QG_EINVAL;
  if (cos && positions < 1) return QG_EINVAL;
  if (q && (q_heads < 1 || q_heads > 65536 || q_stride < (int64_t)q_heads * head_dim)) return QG_EINVAL;
  if (k_stride < (int64_t)kv_heads * head_dim || v_stride < (int64_t)kv_heads * head_dim) return QG_EINVAL;
  if (p.batch == 0) return QG_OK;                                  // nothing to append
  if (!k || !v || (q && !q_out)) return QG_EINVAL;
  if (!multiple(q, 2) || !multiple(k, 2) || !multiple(v, 2) || !multiple(cos, 4) || !multiple(sin, 4) || !multiple(q_out, 16)) return QG_EINVAL;
  p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.rot = cos ? rot_dim : 0;
  p.cos = p.rot ? cos : nullptr; p.sin = p.rot ? sin : nullptr;
  p.positions = positions; p.neighbours = neighbours != 0;
  p.q_heads = q ? q_heads : 0;
  p.q_out = static_cast<uint16_t*>(q_out);
  p.wide = (!q || (multiple(q, 16) && q_stride % 8 == 0)) && multiple(k, 16) && k_stride % 8 == 0 && multiple(v, 16) && v_stride % 8 == 0 &&
           (!p.rot || (p.rot % (p.neighbours ? 16 : 32) == 0 && multiple(cos, 16) && multiple(sin, 16)));
  return kv_append_launch(p, head_dim, static_cast<hipStream_t>(stream));
}

int qg_kv_attention(const void* q, int act, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scale,
                    const float* v_scale, qg_wtype type, int64_t num_blocks, const int32_t* row_start, const int32_t* kv_len,
                    const int32_t* block_table, int64_t table_width, int64_t batch, int64_t rows, int64_t max_rows, int64_t max_kv,
                    int q_heads, int kv_heads, int head_dim, float scale, int causal, int64_t window, void* out, void* stream) {
  KvParams p = {};
  const int rc = check_kv(k_cache, v_cache, k_scale, v_scale, type, num_blocks, row_start, kv_len, block_table, table_width, batch,
                          rows, max_rows, kv_heads, head_dim, act, &p);
  if (rc != QG_OK) return rc;
  if (q_heads < 1 || q_heads > 65536 || q_heads % kv_heads || q_stride < (int64_t)q_heads * head_dim) return QG_EINVAL;
  if (!(scale > 0.0f) || std::isinf(scale) || window < 0 || max_kv < 0) return QG_EINVAL;
  if (p.batch == 0) return QG_OK;
  if (!q || !out || !multiple(q, 2) || !multiple(out, 16)) return QG_EINVAL;
  // the workspace is kept by stream: one handle value names a different stream in every thread
  if (static_cast<hipStream_t>(stream) == hipStreamPerThread) {
    layer_error("hipStreamPerThread is not accepted: pass a stream of your own");
    return QG_EINVAL;
  }
  p.q = static_cast<const uint16_t*>(q); p.q_stride = q_stride; p.q_heads = q_heads;
  p.wide = multiple(q, 16) && q_stride % 8 == 0;
  p.out = static_cast<uint16_t*>(out);
  p.factor = scale * 1.44269504088896340736f;
  p.causal = causal != 0;
  p.window = (int)(window < INT32_MAX ? window : 0);               // as many tokens as there can be: no window
  const int64_t room = table_width * QG_KV_BLOCK;
  return kv_attention_launch(p, head_dim, max_kv == 0 || max_kv > room ? room : max_kv, static_cast<hipStream_t>(stream));
}

int qg_kv_dequant(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, qg_wtype type,
                  int64_t num_blocks, const int32_t* row_start, const int32_t* kv_len, const int32_t* block_table,
                  int64_t table_width, int64_t batch, int64_t rows, int64_t max_rows, int kv_heads, int head_dim, int act,
                  void* k_out, void* v_out, void* stream) {
  KvParams p = {};
  const int rc = check_kv(k_cache, v_cache, k_scale, v_scale, type, num_blocks, row_start, kv_len, block_table, table_width, batch,
                          rows, max_rows, kv_heads, head_dim, act, &p);
  if (rc != QG_OK) return rc;
  if (p.batch == 0) return QG_OK;
  if (!k_out || !v_out || !multiple(k_out, 16) || !multiple(v_out, 16)) return QG_EINVAL;
  p.k_out = static_cast<uint16_t*>(k_out); p.v_out = static_cast<uint16_t*>(v_out);
  return kv_dequant_launch(p, head_dim, static_cast<hipStream_t>(stream));
}

}  // extern "C"
