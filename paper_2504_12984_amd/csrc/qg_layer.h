// Shared definitions of the kernels between a layer's products (interface: include/qg_layer.h).
#pragma once
#include "../../include/qg_layer.h"
#include "qg_common.h"

namespace qg {

// ---- the 8-bit rule ------------------------------------------------------------------------
constexpr float SCALE_FLOOR = 0x1p-40f;

// Magnitudes travel as the bits of |x|: as unsigned integers they order as the numbers do, infinities above all numbers
// and NaN above those, so one integer maximum also says that something was not finite.
constexpr uint32_t NOT_FINITE = 0x7f800000u;
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(uint32_t amax, float qmax) {
  if (amax >= NOT_FINITE) return __builtin_nanf("");
  return fmaxf(__builtin_bit_cast(float, amax) / qmax, SCALE_FLOOR);
}

// Four numbers, already divided by their scale, as int8 codes (two's complement) / as e4m3 codes in the bytes of a register.
__device__ __forceinline__ uint32_t codes_i8(float a, float b, float c, float d) {
  const auto code = [](float x) { return (uint32_t)(int)fminf(fmaxf(rintf(x), -127.0f), 127.0f); };
  const uint32_t lo = __builtin_amdgcn_perm(code(b), code(a), 0x0c0c0400u), hi = __builtin_amdgcn_perm(code(d), code(c), 0x04000c0cu);
  return lo | hi;
}
__device__ __forceinline__ uint32_t codes_e4m3(float a, float b, float c, float d) {
  const auto in = [](float x) { return fminf(fmaxf(x, -448.0f), 448.0f); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), w, true);
  return (uint32_t)w;
}

// ---- 16-bit inputs ---------------------------------------------------------------------------
template <bool BF16>
__device__ __forceinline__ float act_to_f32(uint16_t u) {
  if constexpr (BF16) return __builtin_bit_cast(float, (uint32_t)u << 16);
  else                return (float)__builtin_bit_cast(_Float16, u);
}
template <bool BF16>
__device__ __forceinline__ uint16_t f32_to_act(float x) {
  if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  else                return __builtin_bit_cast(uint16_t, (_Float16)x);
}
// The two halves of a register.
template <bool BF16>
__device__ __forceinline__ void unpack2(uint32_t u, float* lo, float* hi) {
  if constexpr (BF16) {
    *lo = __builtin_bit_cast(float, u << 16);
    *hi = __builtin_bit_cast(float, u & 0xffff0000u);
  } else {
    *lo = act_to_f32<false>((uint16_t)u);
    *hi = act_to_f32<false>((uint16_t)(u >> 16));
  }
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return (uint32_t)f32_to_act<BF16>(lo) | ((uint32_t)f32_to_act<BF16>(hi) << 16);
}
template <bool BF16>
__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8]) {
  unpack2<BF16>(u.x, &x[0], &x[1]); unpack2<BF16>(u.y, &x[2], &x[3]);
  unpack2<BF16>(u.z, &x[4], &x[5]); unpack2<BF16>(u.w, &x[6], &x[7]);
}
template <bool BF16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
}

// ---- rows to 8 bits --------------------------------------------------------------------------
struct RowsParams {
  const uint16_t* x;        // norm: x;         gate: gate
  const uint16_t* y;        // norm: residual;  gate: up
  const uint16_t* w;        // norm: weight
  uint16_t* sum;            // norm: x + residual, or null
  int8_t* A8;
  float* a_scale;
  int64_t x_stride, y_stride, sum_stride;
  int64_t M;
  int N;
  float eps;
  int bf16;
  int wide;                 // everything may be read and written 8 elements at a time
};

// ---- the paged cache -------------------------------------------------------------------------
constexpr int KV_BLOCK = QG_KV_BLOCK;
// Byte of (token, dimension) inside a (block, head), see include/qg_layer.h.
template <int D>
__host__ __device__ constexpr int key_byte(int token, int d) {
  return (((token / 16 * (D / 64) + d / 64) * 4 + d % 64 / 16) * 16 + token % 16) * 16 + d % 16;
}
__host__ __device__ constexpr int value_byte(int token, int d) {
  return ((d / 16 * 4 + token % 16 / 4) * 16 + d % 16) * 16 + token / 16 * 4 + token % 4;
}

struct KvParams {
  uint8_t* k_cache; uint8_t* v_cache;
  float* k_scale; float* v_scale;
  const int32_t* row_start; const int32_t* kv_len; const int32_t* table;
  int64_t width;                       // of the table
  int64_t num_blocks;
  int batch, rows, max_rows;
  int q_heads, kv_heads;
  int bf16, e4m3;
  // append
  const uint16_t* q; const uint16_t* k; const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;
  const float* cos; const float* sin;
  int64_t positions;
  int rot, neighbours;
  int wide;                            // rows, and the rotation's pairs, may be read 16 elements at a time
  uint16_t* q_out;
  // dequant
  uint16_t* k_out; uint16_t* v_out;
  // attention (q, q_stride above)
  uint16_t* out;
  float factor;                        // scale * log2(e)
  int causal;
  int window;                          // 0: none
  int splits;                          // blocks to a part; or shares of a head's tiles,
  int least;                           // and what one of them costs at least
  int stride;                          // of the arrival counters
  float* partial; unsigned* tickets;
};

// First row, rows and tokens of sequence b, kept inside what the arrays hold.
struct Sequence { int first, rows, before, length; };
__device__ __forceinline__ Sequence sequence(const KvParams& p, int b) {
  Sequence s;
  const int start = p.row_start[b], end = p.row_start[b + 1];
  s.first = max(start, 0);
  s.rows = min(min(end, p.rows) - s.first, p.max_rows);
  // the rows are the last ones of kv_len, whatever part of them is served
  s.length = p.kv_len[b];
  s.before = s.length - (end - start);
  return s;
}

// Threads of one grid dimension stay below 2^32.
constexpr int64_t MOST_GROUPS = (1 << 22) - 1;          // of at most 1024

int layer_norm_launch(const RowsParams&, hipStream_t);
int layer_gate_launch(const RowsParams&, hipStream_t);
int kv_append_launch(const KvParams&, int head_dim, hipStream_t);
int kv_dequant_launch(const KvParams&, int head_dim, hipStream_t);
int kv_attention_launch(KvParams&, int head_dim, int64_t max_kv, hipStream_t);

// qg_api.hip: the workspace of split-K calls, and the text of the last error.
int layer_workspace(size_t partial_bytes, size_t counters, hipStream_t, float** partial, unsigned** tickets);
size_t layer_workspace_bytes();
void layer_error(const char* text);
int layer_knob(int i);                 // experiment overrides, see include/qgemm_tuning.h

}  // namespace qg
