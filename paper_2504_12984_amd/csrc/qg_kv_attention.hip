// Attention over the paged 8-bit cache.
//
//   s_t = scale q . k_t,   out = sum_t exp(s_t) v_t / sum_t exp(s_t)      over the tokens t that a row sees
//
// Both kernels compute transposed: scores^T = K Q^T and out^T = V^T P^T with the 16x16x32 matrix instruction, so that a
// lane holds scores of ONE row of q (column i = lane % 16) and the softmax needs no lane but the three others of that
// column.  The four scores that lane 16 b + i gets of a 16-token tile are tokens 4 b .. 4 b + 3; a cache block stores its
// values' tokens in the order that makes these registers the operand of the second product as they are.
//
// Codes become fp16 exactly (int8 through 1024 + u, e4m3 by the hardware's convert).  The scales are applied where they
// cost nothing: the keys' with the softmax's factor, and the values' in the exponent,
//   P'_t = exp2(s_t log2(e) + log2(vs) - m),   out = sum P'_t code_t / sum_blocks (sum_t P'_t) / vs,
// so a block's scale is one addition to the exponent's constant and one multiplication of a row sum, and P', whose largest
// is near 1, is what the fp16 operand can hold best.
// The reference m is not the running maximum itself but is only moved when that exceeds it by 8 (P' up to 256): rescaling
// the accumulators becomes rare.
#include "qg_layer.h"

namespace qg {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr float MOVE_BY = 8.0f;
constexpr float NONE = -__builtin_inff();

// Eight codes -> fp16, exactly.
template <bool E4M3>
__device__ __forceinline__ half8 numbers(uint32_t w0, uint32_t w1) {
  half2v r[4];
  if constexpr (E4M3) {
    r[0] = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, false));
    r[1] = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, true));
    r[2] = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, false));
    r[3] = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, true));
  } else {
    // bytes u under the exponent of 1024 are 1024 + u; the codes are u - 128
    const half2v off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    r[0] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w0, 0x04010400u)) + off;
    r[1] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w0, 0x04030402u)) + off;
    r[2] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w1, 0x04010400u)) + off;
    r[3] = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w1, 0x04030402u)) + off;
  }
  return half8{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

// Over the four lanes of a column (i, 16 + i, 32 + i, 48 + i), in all of them: swaps of rows of lanes, no trip through LDS.
// (The results' elements are copied before their bits are cast: a cast of an element itself reads the first one.)
template <class F>
__device__ __forceinline__ float over_column(float x, F f) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  u = __builtin_bit_cast(uint32_t, f(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
  const auto b = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t b0 = b[0], b1 = b[1];
  return f(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
__device__ __forceinline__ float column_max(float x) { return over_column(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float column_sum(float x) { return over_column(x, [](float a, float b) { return a + b; }); }

// Codes that one workgroup reads, once: past the caches.  (Not so where several workgroups read them, for different rows.)
template <bool SHARED>
__device__ __forceinline__ uint4 stream16(const uint4* at) {
  if constexpr (SHARED) return *at;
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u4*>(at)));
}

// What one block brings.
struct BlockScales { float k, v; bool there; };

// The tokens that a row sees are lo .. hi - 1.
struct Seen { int lo, hi; };
__device__ __forceinline__ Seen seen(const KvParams& p, int pos, int length) {
  Seen s;
  s.hi = p.causal ? min(pos + 1, length) : length;
  s.lo = p.window ? max(pos - p.window + 1, 0) : 0;
  return s;
}

// Rows of q as the matrix instruction's column operand: lane 16 b + i holds dimensions 64 c + 16 b + 8 e + 0..7 of row i.
// Returns what the row was divided by.
template <int D, bool BF16>
__device__ __forceinline__ float load_q(const uint16_t* row, bool wide, int b, half8 (&q)[D / 32]) {
  float x[D / 32][8];
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int at = 64 * c + 16 * b + 8 * e;
      float (&y)[8] = x[2 * c + e];
      if (!row) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = 0.0f;
      } else if (wide) {
        unpack8<BF16>(*reinterpret_cast<const uint4*>(row + at), y);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = act_to_f32<BF16>(row[at + k]);
      }
    }
  float by = 1.0f, inv = 1.0f;
  if constexpr (BF16) {
    // bf16 numbers reach beyond fp16's: the row's largest is brought to 1 .. 2 (a power of two: nothing is lost down to
    // 2^-14 of it, and 2^-25 of it below)
    uint32_t amax = 0u;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) amax = max(amax, magnitude(x[j][k]));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
    // (exponents 1 .. 253, so that both factors are normal numbers)
    const uint32_t e = min(max(amax >> 23, 1u), 253u);
    if (amax < NOT_FINITE) { by = __builtin_bit_cast(float, e << 23); inv = __builtin_bit_cast(float, (254u - e) << 23); }
  }
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
#pragma unroll
    for (int k = 0; k < 8; ++k) q[j][k] = (_Float16)(x[j][k] * inv);
  return by;
}

// One tile of 16 rows against the 64 tokens of a block: from score registers to the operand of the second product.
// `acc` are the products of q and codes, f the factor of the scores, moved: the factor that the accumulators have to be
// multiplied by (1: none).
struct RowState { float m, l; };
template <bool EDGE>
__device__ __forceinline__ float softmax_step(float4v (&acc)[4], half8 (&P)[2], RowState& st, float f, float lv, float ivs, int token0, Seen see) {
  // token0: the first token of the lane, 64 * block + 4 b
  if constexpr (EDGE) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int token = token0 + 16 * t + r;
        if (token < see.lo || token >= see.hi) acc[t][r] = NONE;
      }
  }
  float top = NONE;
#pragma unroll
  for (int t = 0; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(acc[t][0], acc[t][1]), fmaxf(acc[t][2], acc[t][3])));
  top = column_max(top);
  top = fmaf(top, f, lv);                                    // NaN (a scale, a score) never moves the reference
  float alpha = 1.0f;
  if (top > st.m + MOVE_BY) {
    alpha = st.m == NONE ? 0.0f : __builtin_amdgcn_exp2f(st.m - top);
    st.m = top;
    st.l *= alpha;
  }
  const float c = lv - (st.m == NONE ? 0.0f : st.m);
  float sum = 0.0f;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float e = __builtin_amdgcn_exp2f(fmaf(acc[t][r], f, c));
      if constexpr (EDGE) {
        const int token = token0 + 16 * t + r;
        if (token < see.lo || token >= see.hi) e = 0.0f;     // also where the block's scales are NaN
      }
      sum += e;
      P[t / 2][4 * (t % 2) + r] = (_Float16)e;
    }
  st.l += sum == 0.0f ? 0.0f : sum * ivs;
  return alpha;
}

__device__ __forceinline__ uint32_t bytes_below(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

constexpr int STREAM_WAVES = 8;
// Partial results of one unit and part: O [16 T][D], then the references and the sums of the 16 T rows.
template <int D, int T>
constexpr int PART = 16 * T * (D + 2);

// Few rows per sequence: the cache is streamed once.  A workgroup takes 16 T rows (query heads of one key/value head,
// consecutive tokens) and a part of the blocks they see; its wavefronts take every fourth block each, all by themselves,
// and meet at the end.  Bound: HBM, 2 D bytes a token and head.
template <int D, bool BF16, bool E4M3, int T, bool SHARED>
__global__ __launch_bounds__(64 * STREAM_WAVES, 2) void stream_kernel(KvParams p) {
  constexpr int BYTES = KV_BLOCK * D, LOADS = BYTES / 1024, STREAM_ROWS = 16 * T;
  __shared__ __attribute__((aligned(16))) float o_sh[STREAM_WAVES][STREAM_ROWS][D + 4];
  __shared__ float m_sh[STREAM_WAVES][STREAM_ROWS], l_sh[STREAM_WAVES][STREAM_ROWS];
  __shared__ unsigned last;
  const int tid = threadIdx.x, l = tid & 63, i = l & 15, b4 = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = p.kv_heads, G = p.q_heads / H, units = p.batch * H;
  const int unit = blockIdx.x % units, tile = blockIdx.x / units, b = unit / H, h = unit % H;
  const Sequence s = sequence(p, b);
  const int rows = s.rows * G, r0 = tile * STREAM_ROWS;
  if (r0 >= rows) return;
  const int length = (int)min((int64_t)max(s.length, 0), p.width * KV_BLOCK);
  // what all rows of the tile see together (from, upto), and what every one of them sees (lo, hi)
  const int pos0 = s.before + r0 / G, pos1 = s.before + (min(r0 + STREAM_ROWS, rows) - 1) / G;
  const Seen see0 = seen(p, pos0, length), see1 = seen(p, pos1, length);
  const int from = see0.lo, upto = see1.hi, lo = see1.lo, hi = see0.hi;
  const int first = from / KV_BLOCK, count = upto > from ? (upto - 1) / KV_BLOCK - first + 1 : 0;
  // p.splits: blocks to a part; more where the cache is longer than the call said, so that the grid's parts cover it
  const int each = max(p.splits, (int)((count + gridDim.y - 1) / gridDim.y));
  const int parts = max((count + each - 1) / each, 1);
  const int part = blockIdx.y;
  if (part >= parts) return;
  const int begin = first + part * each, end = min(begin + each, first + count);

  half8 q[T][D / 32];
  float cs[T];
  Seen see[T];
  RowState st[T];
  float4v o[T][D / 16];
#pragma unroll
  for (int n = 0; n < T; ++n) {
    const int row = r0 + 16 * n + i;
    const bool valid = row < rows;
    see[n] = seen(p, s.before + row / G, length);
    if (!valid) see[n].lo = see[n].hi = 0;
    const uint16_t* q_row = valid ? p.q + (int64_t)(s.first + row / G) * p.q_stride + (h * G + row % G) * D : nullptr;
    cs[n] = load_q<D, BF16>(q_row, p.wide, b4, q[n]) * p.factor;
    st[n] = {NONE, 0.0f};
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[n][d] = float4v{0, 0, 0, 0};
  }

  const int32_t* table = p.table + (int64_t)b * p.width;
  uint4 K[LOADS], V[LOADS];
  BlockScales bs;
  int64_t base;
  const auto find = [&](uint32_t id) {
    bs.there = id < (uint64_t)p.num_blocks;
    base = bs.there ? (int64_t)id * H + h : 0;
    bs.k = p.k_scale[base]; bs.v = p.v_scale[base];
  };
  const auto load_k = [&]() {
    const uint4* at = reinterpret_cast<const uint4*>(p.k_cache + base * BYTES) + l;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) K[j] = stream16<SHARED>(at + 64 * j);
  };
  const auto load_v = [&]() {
    const uint4* at = reinterpret_cast<const uint4*>(p.v_cache + base * BYTES) + l;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) V[j] = stream16<SHARED>(at + 64 * j);
  };
  int block = begin + wave;
  // where a block lies is read a turn ahead of its codes, its scales with them
  uint32_t next_id = 0;
  if (block < end) {
    find((uint32_t)table[block]);
    next_id = (uint32_t)table[min(block + STREAM_WAVES, end - 1)];
    load_k();
    __builtin_amdgcn_sched_barrier(0);       // keys first, here as in the loop: its waits count on the order
    load_v();
  }
  while (block < end) {
    const int next = block + STREAM_WAVES;
    const BlockScales now = bs;
    float4v acc[T][4];
#pragma unroll
    for (int n = 0; n < T; ++n)
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[n][t] = float4v{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint4 w = K[t * (D / 64) + c / 2];
        const half8 a = c % 2 ? numbers<E4M3>(w.z, w.w) : numbers<E4M3>(w.x, w.y);
#pragma unroll
        for (int n = 0; n < T; ++n) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[n][c], acc[n][t], 0, 0, 0);
      }
    // the next block's keys are on their way while this one's scores are worked on
    if (next < end) {
      find(next_id);
      next_id = (uint32_t)table[min(next + STREAM_WAVES, end - 1)];
      load_k();
    }
    const float vs = now.v < SCALE_FLOOR ? SCALE_FLOOR : now.v;
    const float lv = __builtin_amdgcn_logf(vs), ivs = 1.0f / vs;
    const int token0 = block * KV_BLOCK + 4 * b4;
    const bool edge = !now.there || block * KV_BLOCK < lo || block * KV_BLOCK + KV_BLOCK > hi;
    half8 P[T][2];
    float alpha[T];
    if (edge) {
#pragma unroll
      for (int n = 0; n < T; ++n) alpha[n] = softmax_step<true>(acc[n], P[n], st[n], cs[n] * now.k, lv, ivs, token0, now.there ? see[n] : Seen{0, 0});
      // bytes of tokens that are not there may be anything, also NaN
      if constexpr (E4M3) {
        uint32_t keep[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) keep[t] = now.there ? bytes_below(length - (token0 + 16 * t)) : 0u;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) { V[j].x &= keep[0]; V[j].y &= keep[1]; V[j].z &= keep[2]; V[j].w &= keep[3]; }
      }
    } else {
#pragma unroll
      for (int n = 0; n < T; ++n) alpha[n] = softmax_step<false>(acc[n], P[n], st[n], cs[n] * now.k, lv, ivs, token0, see[n]);
    }
#pragma unroll
    for (int n = 0; n < T; ++n)
      if (__ballot(alpha[n] != 1.0f)) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[n][d] *= alpha[n];
      }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        const half8 a = k ? numbers<E4M3>(V[d].z, V[d].w) : numbers<E4M3>(V[d].x, V[d].y);
#pragma unroll
        for (int n = 0; n < T; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, P[n][k], o[n][d], 0, 0, 0);
      }
    if (next < end) load_v();
    block = next;
  }

  // the wavefronts meet
#pragma unroll
  for (int n = 0; n < T; ++n) {
    const float sum = column_sum(st[n].l);
    if (b4 == 0) { m_sh[wave][16 * n + i] = st[n].m; l_sh[wave][16 * n + i] = sum; }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<float4v*>(&o_sh[wave][16 * n + i][16 * d + 4 * b4]) = o[n][d];
  }
  __syncthreads();
  constexpr int EACH = 4 * STREAM_WAVES / T, PER = D / EACH;    // threads to a row, dimensions a thread
  const int mine = tid / EACH, d0 = (tid % EACH) * PER, my_row = r0 + mine;
  float M = NONE, L = 0.0f, x[PER];
#pragma unroll
  for (int w = 0; w < STREAM_WAVES; ++w) M = fmaxf(M, m_sh[w][mine]);
#pragma unroll
  for (int e = 0; e < PER; ++e) x[e] = 0.0f;
#pragma unroll
  for (int w = 0; w < STREAM_WAVES; ++w) {
    const float a = M == NONE ? 1.0f : __builtin_amdgcn_exp2f(m_sh[w][mine] - M);
    L = fmaf(a, l_sh[w][mine], L);
#pragma unroll
    for (int e = 0; e < PER; ++e) x[e] = fmaf(a, o_sh[w][mine][d0 + e], x[e]);
  }
  if (parts > 1) {
    // parts meet in the workspace: device-scope relaxed stores are out when they are waited for, and the last one to come
    // adds all parts up in their order
    float* to = p.partial + ((int64_t)blockIdx.x * gridDim.y + part) * PART<D, T>;
    if (my_row < rows) {
#pragma unroll
      for (int e = 0; e < PER; e += 2) {
        const uint64_t two = __builtin_bit_cast(uint32_t, x[e]) | (uint64_t)__builtin_bit_cast(uint32_t, x[e + 1]) << 32;
        __hip_atomic_store(reinterpret_cast<unsigned long long*>(to + mine * D + d0 + e), two, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      if (tid % EACH == 0) {
        __hip_atomic_store(to + STREAM_ROWS * D + mine, M, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(to + STREAM_ROWS * D + STREAM_ROWS + mine, L, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    unsigned* ticket = p.tickets + (int64_t)blockIdx.x * p.tiles;            // p.tiles: distance of counters
    if (tid == 0) last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(parts - 1);
    __syncthreads();
    if (!last) return;
    if (tid == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (my_row >= rows) return;
    const float* of = p.partial + (int64_t)blockIdx.x * gridDim.y * PART<D, T>;
    const auto stat = [&](int k, int which) {
      return __hip_atomic_load(of + k * PART<D, T> + STREAM_ROWS * (D + which) + mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    // A turn to AHEAD parts, all of whose loads are under way together.  (The last turn's loads past the end read
    // the last part again and count for nothing.)
    constexpr int AHEAD = 8;
    M = NONE;
    L = 0.0f;
#pragma unroll
    for (int e = 0; e < PER; ++e) x[e] = 0.0f;
    for (int k0 = 0; k0 < parts; k0 += AHEAD) {
      float m[AHEAD], sum[AHEAD];
      uint64_t two[AHEAD][PER / 2];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int part_k = min(k0 + k, parts - 1);
        m[k] = stat(part_k, 0);
        sum[k] = stat(part_k, 1);
#pragma unroll
        for (int e = 0; e < PER / 2; ++e)
          two[k][e] = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(of + part_k * PART<D, T> + mine * D + d0 + 2 * e), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      float top = M;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) top = fmaxf(top, m[k]);
      const float back = top == NONE ? 1.0f : __builtin_amdgcn_exp2f(M - top);
      M = top;
      L *= back;
#pragma unroll
      for (int e = 0; e < PER; ++e) x[e] *= back;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        float a = M == NONE ? 1.0f : __builtin_amdgcn_exp2f(m[k] - M);
        if (k0 + k >= parts) { a = 0.0f; sum[k] = 0.0f; }
        L = fmaf(a, sum[k], L);
#pragma unroll
        for (int e = 0; e < PER / 2; ++e) {
          const uint64_t u = k0 + k < parts ? two[k][e] : 0;
          x[2 * e] = fmaf(a, __builtin_bit_cast(float, (uint32_t)u), x[2 * e]);
          x[2 * e + 1] = fmaf(a, __builtin_bit_cast(float, (uint32_t)(u >> 32)), x[2 * e + 1]);
        }
      }
    }
  }
  if (my_row >= rows) return;
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  uint32_t w[PER / 2 > 0 ? PER / 2 : 1];
#pragma unroll
  for (int e = 0; e < PER; e += 2) w[e / 2] = pack2<BF16>(x[e] * inv, x[e + 1] * inv);
  uint16_t* out = p.out + ((int64_t)(s.first + my_row / G) * p.q_heads + h * G + my_row % G) * D + d0;
  if constexpr (PER == 8)      *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
  else if constexpr (PER == 4) *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
  else                         *reinterpret_cast<uint32_t*>(out) = w[0];
}

// Many rows per sequence: bound by the matrix instruction and the softmax's vector work.  A workgroup takes 256 rows (the
// query heads of one key/value head for 256 / heads consecutive tokens), 32 to a wavefront; a block's codes are
// converted once for all of them, into LDS in the order in which lanes read operands.
constexpr int TILE_WAVES = 8, TILE_QT = 2, TILE_ROWS = TILE_WAVES * TILE_QT * 16;
template <int D, bool BF16, bool E4M3>
__global__ __launch_bounds__(64 * TILE_WAVES) void tile_kernel(KvParams p) {
  constexpr int BYTES = KV_BLOCK * D, PIECES = BYTES / 16, FRAGS = BYTES * 2 / 1024;
  constexpr int PER = 2 * PIECES / (64 * TILE_WAVES);                 // 16-byte pieces of codes a thread converts
  __shared__ uint4 lds[2][2][FRAGS * 64];                             // stage, keys / values
  const int tid = threadIdx.x, l = tid & 63, i = l & 15, b4 = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int H = p.kv_heads, G = p.q_heads / H;
  const int h = blockIdx.x % H, b = blockIdx.x / H % p.batch;
  const int tile = p.tiles - 1 - (int)(blockIdx.x / H / p.batch);      // rows that see most start first
  const Sequence s = sequence(p, b);
  const int rows = s.rows * G, r0 = tile * TILE_ROWS;
  if (r0 >= rows) return;
  const int length = (int)min((int64_t)max(s.length, 0), p.width * KV_BLOCK);
  const auto place = [&](int row) { return s.before + min(row, rows - 1) / G; };
  const int from = seen(p, place(r0), length).lo, upto = seen(p, place(r0 + TILE_ROWS - 1), length).hi;
  const int first = from / KV_BLOCK, end = upto > from ? (upto - 1) / KV_BLOCK + 1 : first;
  // the wavefront's own rows: seen by some of them, by all of them
  const int w0 = r0 + wave * TILE_QT * 16;
  const Seen seeA = seen(p, place(w0), length), seeZ = seen(p, place(w0 + TILE_QT * 16 - 1), length);
  const int w_from = seeA.lo, w_upto = w0 < rows ? seeZ.hi : 0, lo = seeZ.lo, hi = seeA.hi;

  half8 q[TILE_QT][D / 32];
  float cs[TILE_QT];
  Seen see[TILE_QT];
  RowState st[TILE_QT];
  float4v o[TILE_QT][D / 16];
#pragma unroll
  for (int t = 0; t < TILE_QT; ++t) {
    const int row = w0 + 16 * t + i;
    const bool valid = row < rows;
    see[t] = seen(p, s.before + row / G, length);
    if (!valid) see[t].lo = see[t].hi = 0;
    const uint16_t* q_row = valid ? p.q + (int64_t)(s.first + row / G) * p.q_stride + (h * G + row % G) * D : nullptr;
    cs[t] = load_q<D, BF16>(q_row, p.wide, b4, q[t]) * p.factor;
    st[t] = {NONE, 0.0f};
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[t][d] = float4v{0, 0, 0, 0};
  }

  const int32_t* table = p.table + (int64_t)b * p.width;
  uint4 raw[PER];
  BlockScales bs = {0.0f, 0.0f, false};
  const auto fetch = [&](int block) {
    const uint32_t id = (uint32_t)table[block];
    bs.there = id < (uint64_t)p.num_blocks;
    const int64_t base = bs.there ? (int64_t)id * H + h : 0;
    const float k = p.k_scale[base], v = p.v_scale[base];
    bs.k = k; bs.v = v < SCALE_FLOOR ? SCALE_FLOOR : v;
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int piece = tid + n * 64 * TILE_WAVES;
      raw[n] = reinterpret_cast<const uint4*>((piece < PIECES ? p.k_cache : p.v_cache) + base * BYTES)[piece % PIECES];
    }
  };
  const auto stage = [&](int block, int at) {
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int piece = (tid + n * 64 * TILE_WAVES) % PIECES, which = (tid + n * 64 * TILE_WAVES) / PIECES;
      uint4 c = raw[n];
      if (E4M3 && which == 1 && (!bs.there || block * KV_BLOCK + KV_BLOCK > length)) {
        const int token0 = block * KV_BLOCK + 4 * (piece % 64 / 16), upto = bs.there ? length : 0;
        c.x &= bytes_below(upto - token0); c.y &= bytes_below(upto - token0 - 16);
        c.z &= bytes_below(upto - token0 - 32); c.w &= bytes_below(upto - token0 - 48);
      }
      uint4* to = &lds[at][which][piece / 64 * 128 + piece % 64];
      to[0] = __builtin_bit_cast(uint4, numbers<E4M3>(c.x, c.y));
      to[64] = __builtin_bit_cast(uint4, numbers<E4M3>(c.z, c.w));
    }
  };
  BlockScales now = bs;
  if (first < end) { fetch(first); stage(first, 0); now = bs; }
  __syncthreads();
  for (int block = first, at = 0; block < end; ++block, at ^= 1) {
    if (block + 1 < end) fetch(block + 1);
    const int t0 = block * KV_BLOCK;
    if (t0 < w_upto && t0 + KV_BLOCK > w_from) {
      const uint4* kf = &lds[at][0][l];
      const uint4* vf = &lds[at][1][l];
      float4v acc[TILE_QT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int n = 0; n < TILE_QT; ++n) acc[n][t] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const half8 a = __builtin_bit_cast(half8, kf[(t * (D / 32) + c) * 64]);
#pragma unroll
          for (int n = 0; n < TILE_QT; ++n) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[n][c], acc[n][t], 0, 0, 0);
        }
      }
      const float lv = __builtin_amdgcn_logf(now.v), ivs = 1.0f / now.v;
      const bool edge = !now.there || t0 < lo || t0 + KV_BLOCK > hi;
      half8 P[TILE_QT][2];
      float alpha[TILE_QT];
#pragma unroll
      for (int n = 0; n < TILE_QT; ++n) {
        if (edge) alpha[n] = softmax_step<true>(acc[n], P[n], st[n], cs[n] * now.k, lv, ivs, t0 + 4 * b4, now.there ? see[n] : Seen{0, 0});
        else      alpha[n] = softmax_step<false>(acc[n], P[n], st[n], cs[n] * now.k, lv, ivs, t0 + 4 * b4, see[n]);
      }
#pragma unroll
      for (int n = 0; n < TILE_QT; ++n)
        if (__ballot(alpha[n] != 1.0f)) {
#pragma unroll
          for (int d = 0; d < D / 16; ++d) o[n][d] *= alpha[n];
        }
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const half8 a = __builtin_bit_cast(half8, vf[(2 * d + k) * 64]);
#pragma unroll
          for (int n = 0; n < TILE_QT; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, P[n][k], o[n][d], 0, 0, 0);
        }
    }
    if (block + 1 < end) { stage(block + 1, at ^ 1); now = bs; }
    __syncthreads();
  }
#pragma unroll
  for (int n = 0; n < TILE_QT; ++n) {
    const int row = w0 + 16 * n + i;
    const float L = column_sum(st[n].l);
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    if (row >= rows) continue;
    uint16_t* out = p.out + ((int64_t)(s.first + row / G) * p.q_heads + h * G + row % G) * D + 4 * b4;
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
      *reinterpret_cast<uint2*>(out + 16 * d) = make_uint2(pack2<BF16>(o[n][d][0] * inv, o[n][d][1] * inv), pack2<BF16>(o[n][d][2] * inv, o[n][d][3] * inv));
  }
}

// How long a part is.  Workgroups read at some 40 GB/s each, so as many as there are CUs stream the cache at its rate, and more
// only add partial results; parts of less than four blocks do not pay for their meeting, and parts of at most 128 keep one
// long sequence among short ones from being the last one left.  One row tile, 64 heads over 8, us:
//   1 x 131071 tokens (8 units): 32 / 64 / 128 blocks 55 / 48 / 53;    64 x 1000 .. 8000 (512 units): 108.. for 128, 114 for 64, 119 for 32
//   8 x 500 .. 4000 (64 units):  8 / 16 / 32 blocks 17 / 13 / 17;      1 x 1000 (8 units): 4 / 8 / 16 blocks 7.6 / 8.8 / 8.8
template <int D, bool BF16, bool E4M3, int T>
static int launch_stream(KvParams& p, int64_t max_tile_rows, int64_t max_kv, hipStream_t st) {
  const int64_t tiles = (max_tile_rows + 16 * T - 1) / (16 * T), units = tiles * p.kv_heads * p.batch;
  if (units > MOST_GROUPS) return QG_EUNSUPPORTED;
  const int64_t blocks = std::max<int64_t>((max_kv + KV_BLOCK - 1) / KV_BLOCK, 1);
  const size_t part = PART<D, T> * sizeof(float);
  int64_t chunk = std::clamp<int64_t>((units * blocks + 255) / 256, 4, 128);
  while (chunk < blocks && (size_t)units * ((blocks + chunk - 1) / chunk) * part > layer_workspace_bytes()) chunk *= 2;
  int64_t parts = (blocks + chunk - 1) / chunk;
  p.tiles = ticket_stride(units);
  if (parts > 1 && (parts > 65535 || p.tiles * units > WS_TICKETS ||
                    layer_workspace((size_t)units * parts * part, (size_t)(units * p.tiles), st, &p.partial, &p.tickets) != QG_OK)) {
    parts = 1;
    chunk = blocks;
  }
  p.splits = (int)std::min<int64_t>(chunk, INT32_MAX / KV_BLOCK);
  const dim3 grid((unsigned)units, (unsigned)parts), threads(64 * STREAM_WAVES);
  if (tiles > 1) hipLaunchKernelGGL((stream_kernel<D, BF16, E4M3, T, true>), grid, threads, 0, st, p);
  else           hipLaunchKernelGGL((stream_kernel<D, BF16, E4M3, T, false>), grid, threads, 0, st, p);
  return hipGetLastError() == hipSuccess ? QG_OK : QG_EHIP;
}

template <int D, bool BF16, bool E4M3>
static int launch_attention(KvParams& p, int64_t max_kv, hipStream_t st) {
  const int G = p.q_heads / p.kv_heads;
  const int64_t max_tile_rows = (int64_t)p.max_rows * G;
  if (max_tile_rows > 64) {
    const int64_t tiles = (max_tile_rows + TILE_ROWS - 1) / TILE_ROWS, grid = tiles * p.kv_heads * p.batch;
    if (grid > MOST_GROUPS) return QG_EUNSUPPORTED;
    p.tiles = (int)tiles;
    hipLaunchKernelGGL((tile_kernel<D, BF16, E4M3>), dim3((unsigned)grid), dim3(64 * TILE_WAVES), 0, st, p);
    return hipGetLastError() == hipSuccess ? QG_OK : QG_EHIP;
  }
  return max_tile_rows <= 16 ? launch_stream<D, BF16, E4M3, 1>(p, max_tile_rows, max_kv, st)
                             : launch_stream<D, BF16, E4M3, 2>(p, max_tile_rows, max_kv, st);
}

int kv_attention_launch(KvParams& p, int head_dim, int64_t max_kv, hipStream_t st) {
  const int which = (head_dim == 128 ? 4 : 0) + (p.bf16 ? 2 : 0) + (p.e4m3 ? 1 : 0);
  switch (which) {
    case 0: return launch_attention<64, false, false>(p, max_kv, st);
    case 1: return launch_attention<64, false, true>(p, max_kv, st);
    case 2: return launch_attention<64, true, false>(p, max_kv, st);
    case 3: return launch_attention<64, true, true>(p, max_kv, st);
    case 4: return launch_attention<128, false, false>(p, max_kv, st);
    case 5: return launch_attention<128, false, true>(p, max_kv, st);
    case 6: return launch_attention<128, true, false>(p, max_kv, st);
    default: return launch_attention<128, true, true>(p, max_kv, st);
  }
}

}  // namespace qg
