// Row operators of the paged key/value cache: norms of queries and keys with the
// position rotation in the same pass, appending to the pages, and the gather back
// into one contiguous prefix per request.  All are bound by memory: every value is
// read once and written once, 16 bytes a lane.  Norms of 7,800 tokens of 40 heads of 128:
// 37 us (4.3 TB/s; a large copy moves 5.4), in 32 bits 70 (4.6); append of 14,600 tokens of
// 8 + 8 heads: 24 us (4.9), in 32 bits 51 (4.7), to 8 bits 28 (3.2); gather of the 18-layer prefix of
// eight requests: 44 us (5.2); single tokens 4 to 5 us.
//
// A head's row of D values is the work of D / 16 lanes: lane c holds values
// 8 c .. 8 c + 7 and their partners at + D / 2, so that a pair rotates inside a lane
// and the sum of squares takes log2(D / 16) cross-lane steps.  The cosines depend on
// the token only: a block computes them once for its tokens, into LDS, and every
// head of those tokens reads them (with 40 heads the 128 sincos of a token would
// otherwise be 5,120).
#include "common.hpp"
#include "errors.hpp"
#include "paged.hpp"

#include <type_traits>

namespace phyai {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 2;       // tokens of a block

// eight consecutive values
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// e4m3 codes, to the nearest, ties to even; what lies beyond 448 becomes 448, NaN stays.
// 0 is 0 over a scale of 0 too, which a head of zeros has by its largest magnitude.
__device__ __forceinline__ float sat_fp8(float x) { return x != x ? x : fminf(fmaxf(x, -448.f), 448.f); }
__device__ __forceinline__ void store8_fp8(uint8_t* p, const float (&v)[8], float scale) {
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = sat_fp8(v[i] == 0.f ? v[i] : v[i] / scale);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], w[i], false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], w[i], true);
  }
  *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

// cos and sin of position * freq turns.  The product modulo one turn is exact in
// 64 bits; its upper 32, as a signed fraction of a turn rounded to float32 (2^-26 of a
// turn at most), is what the sine takes.
__device__ __forceinline__ float2 turn(uint64_t freq, int pos) {
  const uint64_t p = freq * static_cast<uint64_t>(pos);
  const float half_turns = static_cast<float>(static_cast<int32_t>(p >> 32)) * 0x1p-31f;
  float s, c;
  sincospif(half_turns, &s, &c);
  return make_float2(c, s);
}

// The (cos, sin) of a block's tokens, the first of which stands at pos0.
template <int D>
__device__ __forceinline__ void fill_angles(float2 (&cs)[kMaxTokens][D / 2], const RopeFreq& freq, int tokens, int pos0) {
  for (int x = threadIdx.x; x < tokens * (D / 2); x += kThreads) {
    const int t = x / (D / 2), i = x % (D / 2);
    cs[t][i] = turn(freq.f[i], pos0 + t);
  }
  __syncthreads();
}

// Pairs of a lane rotated: (a, b) -> (a cos - b sin, b cos + a sin).
__device__ __forceinline__ void rotate8(float (&a)[8], float (&b)[8], const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = a[i], y = b[i];
    a[i] = x * cs[i].x - y * cs[i].y;
    b[i] = y * cs[i].x + x * cs[i].y;
  }
}

// Sum over the L lanes of a row (4, 8 or 16), in every one of them.
template <int L>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f32<0xB1>(v);                       // lane ^ 1
  v += dpp_f32<0x4E>(v);                       // lane ^ 2
  if constexpr (L >= 8) v += dpp_f32<0x141>(v);
  if constexpr (L >= 16) v += dpp_f32<0x140>(v);
  return v;
}

// Where a block stands: request b, tokens i0 .. i0 + n - 1 of it.
struct BlockTokens {
  int b, i0, n, past;
};
__device__ __forceinline__ bool block_tokens(BlockTokens& t, const int32_t* new_len, const int32_t* past_len, int M, int per,
                                             int64_t cap, int32_t* status) {
  const int groups = (M + per - 1) / per;
  t.b = blockIdx.x / groups;
  t.i0 = blockIdx.x % groups * per;
  const RowSpan s = row_span(new_len ? new_len[t.b] : M, past_len ? past_len[t.b] : 0, M, cap);
  if (!s.ok) {
    if (status && threadIdx.x == 0) atomicOr(status, PAGED_BAD_LENGTH);
    return false;
  }
  t.past = s.past + t.i0;
  t.n = min(per, s.n - t.i0);
  return t.n > 0;
}

// y = x / sqrt(mean x^2 + eps) (1 + gain), rotated.  A row is read whole before it is
// written, by the same lanes, so the output may be the input.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRopeArgs a) {
  constexpr int L = D / 16;
  __shared__ float2 cs[kMaxTokens][D / 2];
  BlockTokens t;
  if (!block_tokens(t, a.new_len, a.past_len, a.M, a.tokens_per_block, INT32_MAX, a.status)) return;
  const int heads = a.q.n + a.k.n, rows = t.n * heads;
  const int c = threadIdx.x % L;
  auto at = [&](const HeadRows& h, int tok, int head) {
    return static_cast<T*>(h.p) + t.b * h.b + (t.i0 + tok) * h.t + head * h.h + 8 * c;
  };
  auto load = [&](int r, float (&x)[8], float (&y)[8]) {
    const int tok = r / heads, head = r % heads;
    const T* p = head < a.q.n ? at(a.q, tok, head) : at(a.k, tok, head - a.q.n);
    load8(p, x);
    load8(p + D / 2, y);
  };
  // the first rows are requested before the angles are computed, the next ones before
  // the present ones are worked on
  float x[8], y[8];
  int r = threadIdx.x / L;
  if (r < rows) load(r, x, y);
  if (a.rope) fill_angles<D>(cs, a.freq, t.n, t.past);
  for (; r < rows; r += kThreads / L) {
    float nx[8], ny[8];
    const int rn = r + kThreads / L;
    if (rn < rows) load(rn, nx, ny);
    const int tok = r / heads, head = r % heads;
    const bool is_q = head < a.q.n;
    if (a.norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], fmaf(y[i], y[i], ss));
      const float inv = 1.0f / sqrtf(row_sum<L>(ss) * (1.0f / D) + a.eps);
      const float* gain = is_q ? a.q_gain : a.k_gain;
      float ga[8], gb[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) ga[i] = gb[i] = 0.f;
      if (gain) {
        load8(gain + 8 * c, ga);
        load8(gain + D / 2 + 8 * c, gb);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = x[i] * inv * (1.0f + ga[i]);
        y[i] = y[i] * inv * (1.0f + gb[i]);
      }
    }
    if (a.rope) rotate8(x, y, &cs[tok][8 * c]);
    T* p = is_q ? at(a.q_out, tok, head) : at(a.k_out, tok, head - a.q.n);
    store8(p, x);
    store8(p + D / 2, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = nx[i];
      y[i] = ny[i];
    }
  }
}

template <typename CT>
__device__ __forceinline__ void store8_pool(char* p, const float (&v)[8], float scale) {
  if constexpr (std::is_same<CT, uint8_t>::value) store8_fp8(reinterpret_cast<uint8_t*>(p), v, scale);
  else store8(reinterpret_cast<CT*>(p), v);
}

// The rows of a token: its key heads (rotated), then its value heads.
template <typename T, typename CT, int D>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedAppendArgs a) {
  constexpr int L = D / 16;
  __shared__ float2 cs[kMaxTokens][D / 2];
  BlockTokens t;
  const int64_t cap = (int64_t)a.pool.max_pages << a.pool.page_shift;
  if (!block_tokens(t, a.new_len, a.past_len, a.M, a.tokens_per_block, cap, a.status)) return;
  const int nkv = a.k.n, rows = t.n * 2 * nkv;
  const int c = threadIdx.x % L;
  if (a.rope) fill_angles<D>(cs, a.freq, t.n, t.past);
  for (int r = threadIdx.x / L; r < rows; r += kThreads / L) {
    const int tok = r / (2 * nkv), hh = r % (2 * nkv);
    const bool is_k = hh < nkv;
    const int head = is_k ? hh : hh - nkv;
    const HeadRows& h = is_k ? a.k : a.v;
    const T* p = static_cast<const T*>(h.p) + t.b * h.b + (t.i0 + tok) * h.t + head * h.h + 8 * c;
    float x[8], y[8];
    load8(p, x);
    load8(p + D / 2, y);
    const int64_t pos = t.past + tok;
    const int page = a.pool.table[(int64_t)t.b * a.pool.table_stride + (pos >> a.pool.page_shift)];
    if (!page_ok(page, a.pool.n_pages)) {
      if (a.status && c == 0) atomicOr(a.status, PAGED_BAD_PAGE);
      continue;
    }
    if (is_k && a.rope) rotate8(x, y, &cs[tok][8 * c]);
    float scale = 1.f;
    if constexpr (std::is_same<CT, uint8_t>::value) scale = is_k ? a.pool.k_scale[head] : a.pool.v_scale[head];
    char* dst = (is_k ? a.pool.k : a.pool.v) + page_row_offset(a.pool, page, pos, head) + 8 * c * (int)sizeof(CT);
    store8_pool<CT>(dst, x, scale);
    store8_pool<CT>(dst + (D / 2) * (int)sizeof(CT), y, scale);
  }
}

// One lane writes 8 values of [layers][2][B][rows][nkv * D]; rows behind a request's
// length are zero, rows of an unusable page or length NaN.
template <typename CT, typename T>
__global__ __launch_bounds__(kThreads) void paged_gather_kernel(PagedGatherArgs a) {
  const int CPH = a.D / 8;                     // chunks of a head
  const int64_t per_row = (int64_t)a.nkv * CPH;
  const int64_t chunks = (int64_t)a.rows * per_row;
  // slab: (layer, K or V, request)
  const int slab = blockIdx.y;
  const int b = slab % a.B, which = slab / a.B % 2, layer = slab / a.B / 2;
  int n = a.kv_len[b];
  bool bad = n < 0 || n > a.rows || n > ((int64_t)a.pool.max_pages << a.pool.page_shift);
  if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, PAGED_BAD_LENGTH);
  const char* pool = (which ? a.pool.v : a.pool.k) + layer * a.pool.layer_bytes;
  T* out = static_cast<T*>(a.out) + (int64_t)slab * chunks * 8;
  for (int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x; x < chunks; x += (int64_t)gridDim.x * kThreads) {
    const int row = static_cast<int>(x / per_row), rest = static_cast<int>(x % per_row);
    const int head = rest / CPH, c = rest % CPH;
    float v[8];
    const float fill = bad ? __builtin_nanf("") : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fill;
    if (!bad && row < n) {
      const int page = a.pool.table[(int64_t)b * a.pool.table_stride + (row >> a.pool.page_shift)];
      if (page_ok(page, a.pool.n_pages)) {
        const char* p = pool + page_row_offset(a.pool, page, row, head) + 8 * c * (int)sizeof(CT);
        if constexpr (sizeof(CT) == 1) {
          const uint2 w = *reinterpret_cast<const uint2*>(p);
          const float scale = which ? a.pool.v_scale[head] : a.pool.k_scale[head];
          const uint32_t u[4] = {fp8x2_to_bf16x2<false>(w.x), fp8x2_to_bf16x2<true>(w.x), fp8x2_to_bf16x2<false>(w.y),
                                 fp8x2_to_bf16x2<true>(w.y)};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16) * scale;
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u) * scale;
          }
        } else {
          load8(reinterpret_cast<const CT*>(p), v);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_nanf("");
        if (a.status) atomicOr(a.status, PAGED_BAD_PAGE);
      }
    }
    store8(out + 8 * x, v);
  }
}

template <typename F>
void by_dim(int D, F&& f) {
  switch (D) {
    case 64: f(std::integral_constant<int, 64>{}); break;
    case 128: f(std::integral_constant<int, 128>{}); break;
    default: f(std::integral_constant<int, 256>{}); break;
  }
}

// Tokens of a block: two, once that still leaves four blocks for every CU, else one, for
// the shortest path.  Norms of 7,800 tokens of 40 heads of 128, blocks of 1, 2, 3, 4, 8
// tokens: 37.8, 37.7, 38.5, 40.9, 39.7 us; append of 14,600 tokens of 8 + 8 heads: 27.3, 23.4,
// 24.9, 24.8, 29.2 us.
int tokens_per_block(int B, int M) { return (int64_t)B * ((M + kMaxTokens - 1) / kMaxTokens) >= 1024 ? kMaxTokens : 1; }

}  // namespace

void norm_rope(const NormRopeArgs& a_in, int D, int kind, hipStream_t s) {
  NormRopeArgs a = a_in;
  a.tokens_per_block = tokens_per_block(a.B, a.M);
  const int grid = a.B * ((a.M + a.tokens_per_block - 1) / a.tokens_per_block);
  by_dim(D, [&](auto d) {
    constexpr int kD = decltype(d)::value;
    if (kind == PAGED_F32) norm_rope_kernel<float, kD><<<grid, kThreads, 0, s>>>(a);
    else norm_rope_kernel<bf16_t, kD><<<grid, kThreads, 0, s>>>(a);
  });
}

void paged_append(const PagedAppendArgs& a_in, int D, int pool_kind, hipStream_t s) {
  PagedAppendArgs a = a_in;
  a.tokens_per_block = tokens_per_block(a.B, a.M);
  const int grid = a.B * ((a.M + a.tokens_per_block - 1) / a.tokens_per_block);
  by_dim(D, [&](auto d) {
    constexpr int kD = decltype(d)::value;
    if (pool_kind == PAGED_F32) paged_append_kernel<float, float, kD><<<grid, kThreads, 0, s>>>(a);
    else if (pool_kind == PAGED_BF16) paged_append_kernel<bf16_t, bf16_t, kD><<<grid, kThreads, 0, s>>>(a);
    else paged_append_kernel<bf16_t, uint8_t, kD><<<grid, kThreads, 0, s>>>(a);
  });
}

void paged_gather(const PagedGatherArgs& a, int pool_kind, hipStream_t s) {
  const int64_t chunks = (int64_t)a.rows * a.nkv * (a.D / 8);
  const int64_t want = (chunks + kThreads - 1) / kThreads;
  const dim3 grid(static_cast<unsigned>(want > 1024 ? 1024 : want), static_cast<unsigned>(a.layers * 2 * a.B));
  if (pool_kind == PAGED_F32) paged_gather_kernel<float, float><<<grid, kThreads, 0, s>>>(a);
  else if (pool_kind == PAGED_BF16) paged_gather_kernel<bf16_t, bf16_t><<<grid, kThreads, 0, s>>>(a);
  else paged_gather_kernel<uint8_t, bf16_t><<<grid, kThreads, 0, s>>>(a);
}

}  // namespace phyai
