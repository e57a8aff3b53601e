// Attention of a chunk of new tokens, or of single tokens, over a paged
// key/value cache.
//
// o_r = sum_j p_rj v_j, p_r = softmax_j(scale q_r . k_j) over the keys that row r
// sees.  The query heads that share a K/V head are folded into the rows (row =
// token * G + head of the group), so a K/V row is read once for all of them.
//
// MFMA formulation: S^T = K Q^T and O^T = V^T P^T on 32x32 tiles.  A query row is
// always an MFMA column (lane % 32), its softmax state lives in lanes l and l ^ 32,
// and the probabilities leave the S^T accumulators in the order in which the
// P.V product takes them: accumulator v of lane half h is key 8 (v / 4) + 4 h + v % 4
// of the 32, and the V^T operand is read in that same order.  V rows lie
// token-major in their pages; the transposing LDS read hands each lane four keys of
// one column.
//
// Three shapes of block:
//   rows   four waves x 32 query rows that share K/V tiles, the next tile under way in a
//          second buffer: chunks.  Bound by the matrix cores and what goes on beside them:
//          4,096 rows of 32 heads over 8,192 keys of 128, causal, take 416 .. 449 us from card
//          to card, 477 under a slower trace (864 .. 991 TFLOP/s; the library's product of
//          8,192^3 reaches 1,398 .. 1,450), the matrix cores busy 49 % of the cycles, the LDS
//          25 %, with 0.5 % of those in conflict; with keys of 64: 260 us, with 8-bit keys of
//          128: 454.  At head_dim 256 a CU has one wave a SIMD, and the scores run a tile
//          ahead so that products and exponentials overlap inside the wave.  In 32 bits 1,024
//          rows of 16 heads over 2,048 keys of 128 take 150 us (86 TFLOP/s; the library's
//          32-bit product 154).
//   pairs  the same of bf16 at head_dim 256 with tiles of 32 keys: registers and LDS of two
//          blocks a CU, whose waves overlap each other instead.  2,048 rows of 8 heads over
//          8,192 keys: 155 us, the rows shape 170.
//   keys   one wave on 32 rows, one tile of K and of V in LDS, many waves a CU: few
//          rows, which are bound by reading K/V: 64 requests of one token over 600 .. 4,000
//          keys 124 .. 130 us (4.6 to 4.9 TB/s; a large copy moves 5.4, a read alone 6.5),
//          131,072 keys in 8 bits 167 .. 185 us (5.0 to 5.6 TB/s), one request over 817 keys
//          12 us, of which the two launches are about seven.
// Each may split the keys over blocks; a second kernel joins the splits (25 us for 64
// splits of 128 rows with one wave a row, 6.5 with four).
#include "common.hpp"
#include "errors.hpp"
#include "paged.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace phyai {

namespace {

typedef __attribute__((address_space(3))) void lds_void;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int s32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// LDS by byte address
template <typename V>
__device__ __forceinline__ V lds_at(uint32_t addr) {
  return *reinterpret_cast<__attribute__((address_space(3))) const V*>(addr);
}

constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes per lane from base + off into LDS at (wave-uniform) lds + 16 * lane.
// `base` is wave-uniform.  Completion is awaited with dma_wait.
__device__ __forceinline__ void dma16(const char* base, uint32_t off, uint32_t lds) {
  // the halves are cast to 32 unsigned bits before they are widened: readfirstlane
  // returns an int, whose sign would spread over the upper half
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  const uint32_t p_lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p));
  const uint32_t p_hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(p >> 32));
  const uint64_t sp = static_cast<uint64_t>(p_hi) << 32 | p_lo;
  lds = __builtin_amdgcn_readfirstlane(lds);
  // a vector instruction may have written the base just before: five wait states to
  // the load that reads it, which the compiler does not count inside asm
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(lds), "v"(off), "s"(sp) : "memory", "m0");
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Barrier without the fence of __syncthreads(): the caller's LDS accesses are
// complete (lgkmcnt 0), loads into LDS have been awaited before.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The larger value, NaN if either is (one v_maximum3_f32 for two of them; fmaxf would
// quiet every input first).  Left to the compiler and not written as asm: it counts
// the wait states between a matrix instruction and the first reader of its result.
__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float max3(float a, float b, float c) { return max2(max2(a, b), c); }
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// LDS tiles hold rows of RB bytes in 16-byte chunks, chunk c of row r at
// c ^ swz(r), so that the lanes of one fragment read fall in different banks:
//   K   16 lanes read 16 consecutive rows at one chunk
//   V   bf16: 32 lanes, which the LDS serves at once, read 64 bytes of each of 4
//       rows, so rows 0 .. 3 differ in the bits above those 64 bytes; f32: 32 lanes
//       read 128 bytes of one row, the other half of the row 4 further on
//       8-bit codes: 32 lanes read 32 bytes of each of 8 rows (0 .. 3 and 8 .. 11)
template <int RB>
__device__ __forceinline__ int k_swz(int r) { return RB >= 256 ? (r & 15) : RB >= 128 ? ((r >> 1) & 7) : ((r >> 2) & 3); }
template <int VS, int RB>
__device__ __forceinline__ int v_swz(int r) {
  if (VS == 4) return 8 * ((r >> 2) & 1);
  if (VS == 2) return RB >= 256 ? 4 * (r & 3) + 2 * ((r >> 2) & 1) : 4 * ((r >> 1) & 1) + 2 * ((r >> 2) & 1);
  const int far = (r >> 3) & 1;
  return RB >= 256 ? 2 * (r & 3) + 8 * far : RB >= 128 ? 2 * ((r >> 1) & 1) + 4 * far : 2 * far;
}

// Order of one MFMA loop whose operands come from LDS: PD reads ahead, then each
// MFMA followed by the reads of a later one (RPM reads per MFMA).
template <int N, int RPM, int PD>
__device__ __forceinline__ void mfma_pipeline() {
#pragma unroll
  for (int i = 0; i < PD; ++i) __builtin_amdgcn_sched_group_barrier(0x100, RPM, 0);
#pragma unroll
  for (int i = 0; i < N - PD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, RPM, 0);
  }
#pragma unroll
  for (int i = 0; i < PD; ++i) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
}

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// The 18 wait states between a 32-bit product and the first reader of its result.  The
// compiler counts them too, but not where the reader is the copy out of an accumulator
// register that opens the block after a branch (two 32-bit kernels read the last of
// sixteen scores 4 states after the product).
__device__ __forceinline__ void mfma_settle() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3");
  __builtin_amdgcn_sched_barrier(0);
}

// What a block of one kind looks like.  CT: element of the pool, T: of the rows
// and of the products.
enum Block { kRows, kKeys, kPairs };

template <typename CT, typename T, int D, Block BLK>
struct Shape {
  static constexpr bool KEYS = BLK == kKeys;
  static constexpr int ES = sizeof(T);
  static constexpr bool kFp8 = sizeof(CT) == 1;
  // An 8-bit pool's codes go into LDS as they are where one wave works on a tile, and
  // are widened when the fragments are read; four waves would each widen all of them, so
  // there the tile is widened once, on its way through registers.
  static constexpr bool kCodes = kFp8 && KEYS, kRegs = kFp8 && !KEYS;
  static constexpr int VS = kCodes ? 1 : ES;            // bytes of a value in LDS
  static constexpr int RB = D * VS;                     // bytes of an LDS row
  static constexpr int OB = D * ES;                     // bytes of a row of q and out
  static constexpr int CPR = OB / 16;                   // chunks of it
  static constexpr int KT = (ES == 2 && BLK == kRows) ? 64 : 32;   // keys of a tile
  static constexpr int TILE = KT * RB;                  // bytes of a K or V tile
  static constexpr int NW = KEYS ? 1 : 4;
  static constexpr int ROWS = 32 * NW;                  // query rows of a block
  static constexpr int BUFS = KEYS ? 1 : 2;             // buffers of K and of V
  static constexpr int LDS = 2 * BUFS * TILE;
  // rows: the scores run a tile ahead
  static constexpr bool kAhead = BLK == kRows && ES == 2 && D == 256;
  // waves of a SIMD asked for, and with them blocks of a CU
  static constexpr int PER_SIMD = KEYS ? (OB <= 128 ? 4 : OB <= 256 ? (kCodes ? 3 : 2) : 1) : (LDS <= 64 * 1024 ? 2 : 1);
  static constexpr int LDS_BLOCKS = 160 * 1024 / LDS;
  static constexpr int PER_CU = LDS_BLOCKS < 4 * PER_SIMD / NW ? LDS_BLOCKS : 4 * PER_SIMD / NW;
};

template <typename CT, typename T, int D, Block BLK, int NT = 64 * Shape<CT, T, D, BLK>::NW,
          int PER_SIMD = Shape<CT, T, D, BLK>::PER_SIMD>
__global__ __launch_bounds__(NT, PER_SIMD) void paged_attn_kernel(PagedAttnArgs a) {
  using S = Shape<CT, T, D, BLK>;
  constexpr bool KEYS = S::KEYS;
  constexpr int ES = S::ES, VS = S::VS, RB = S::RB, OB = S::OB, CPR = S::CPR, KT = S::KT, KB = KT / 32, TILE = S::TILE, NW = S::NW;
  constexpr int V_AT = S::BUFS * TILE;                  // LDS: [K, V][buffer][TILE]
  constexpr int ROWS = S::ROWS, NQ = OB / 32;           // chunk pairs of a row
  // aligned so that the two buffers of a tile differ in one address bit
  __shared__ __attribute__((aligned(2 * TILE))) char sm[S::LDS];
  __shared__ int s_bad;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int lr = lane % 32, hl = lane / 32;
  const int G = a.G;

  // Blocks are dealt to the 8 XCDs in turn; each XCD takes a run of (request, K/V
  // head, split) groups, whose keys its L2 then holds.  Inside a group the tiles
  // alternate between the last (under a causal mask the longest) and the first,
  // so that any part of a group is about as much work.
  const int total = a.B * a.nkv * a.n_split * a.n_tiles;
  const int per_xcd = (total + 7) / 8;
  const int wid = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (wid >= total) return;
  const int gi = wid / a.n_tiles, tp = wid % a.n_tiles;
  const int rt = (tp & 1) ? tp / 2 : a.n_tiles - 1 - tp / 2;
  const int grp = gi / a.n_split, split = gi % a.n_split;
  const int b = grp / a.nkv, kvh = grp % a.nkv;

  // readfirstlane: the compiler keeps what it loads as vectors, and everything that
  // follows from the lengths would be vector arithmetic and divergent branches
  int kv = __builtin_amdgcn_readfirstlane(a.kv_len[b]);
  const RowSpan span = row_span(a.new_len ? __builtin_amdgcn_readfirstlane(a.new_len[b]) : a.M, 0, a.M, a.M);
  bool bad = !span.ok || kv < 0 || kv > a.max_kv;
  if (bad) {
    kv = 0;
    if (a.status && threadIdx.x == 0) atomicOr(a.status, PAGED_BAD_LENGTH);
  }
  const int n = span.n, rows = n * G;
  if (rt * ROWS >= rows) return;

  if constexpr (!KEYS) {
    if (threadIdx.x == 0) s_bad = 0;
    __syncthreads();
  }

  // this lane's query row and the keys it sees; a lane behind the last row works on
  // zeros and sees what the others see
  const int wrow = rt * ROWS + wave * 32;
  const int row = wrow + lr;
  const bool valid = row < rows;
  const int tok = valid ? row / G : n - 1;
  const int qhead = kvh * G + (valid ? row % G : 0);
  const int hi = seen_end(tok, n, kv, a.causal), lo = seen_begin(tok, n, kv, a.window);

  // keys of the block and of this split
  const int tok0 = (rt * ROWS) / G, tok1 = min(n - 1, (rt * ROWS + ROWS - 1) / G);
  const int bl = seen_begin(tok0, n, kv, a.window) / KT * KT, bh = seen_end(tok1, n, kv, a.causal);
  int kbeg = bl, kend = bh;
  if (a.n_split > 1) {
    kbeg = bl + split * a.split_keys;
    kend = min(bh, kbeg + a.split_keys);
  }

  const int64_t grow = (int64_t)grp * a.M * G;          // first row of (request, K/V head) in the workspace
  if (a.n_split > 1 && kbeg >= kend && !bad) {
    // no key of this split is seen: a weight of 0, which the join does not follow
    if (valid && hl == 0) a.ml[(grow + row) * a.n_split + split] = make_float2(-INFINITY, 0.f);
    return;
  }

  // Q^T operand: chunk 2 s + h of the row; with codes in LDS, where a lane reads 16 of a
  // key at once, chunk 4 (s / 2) + 2 h + s % 2
  uint4 qf[NQ];
  {
    const char* qp = static_cast<const char*>(a.q.p) + (b * a.q.b + tok * a.q.t + qhead * a.q.h) * ES +
                     (S::kCodes ? 32 : 16) * hl;
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
      qf[s] = make_uint4(0, 0, 0, 0);
      if (valid) qf[s] = *reinterpret_cast<const uint4*>(qp + (S::kCodes ? 64 * (s / 2) + 16 * (s % 2) : 32 * s));
    }
  }

  const float ks = S::kFp8 ? a.pool.k_scale[kvh] : 1.f;
  const float vs = S::kFp8 ? a.pool.v_scale[kvh] : 1.f;
  const float sl2 = fmaxf(a.scale * ks * kLog2e, 1e-37f);  // not 0: a hidden key's -inf stays -inf

  // ---- loading ----
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)sm));
  const int psm = (1 << a.pool.page_shift) - 1;
  const int32_t* table = a.pool.table + (int64_t)b * a.pool.table_stride;
  const char* kpool = a.pool.k + kvh * a.pool.head_bytes;
  const char* vpool = a.pool.v + kvh * a.pool.head_bytes;
  const int last_page = (kend - 1) >> a.pool.page_shift;
  // The first page that a row of the block sees.  The first tile may begin before it: the
  // program may have given those pages back, so their numbers are not judged, and where
  // there is none, page 0 is read in its place (no row sees what it holds).
  const int first_page = seen_begin(tok0, n, kv, a.window) >> a.pool.page_shift;
  // 64 entries of the table from `pbase` on, one per lane; the numbers are checked here
  int pbase = 0, pages = 0;
  auto load_pages = [&](int from) {
    pbase = from;
    const int i = from + lane;
    int id = 0;
    if (i <= last_page && i < a.pool.max_pages) id = table[i];
    const bool out = !page_ok(id, a.pool.n_pages);
    if (__ballot(out && i >= first_page)) {
      bad = true;
      if (a.status && lane == 0) atomicOr(a.status, PAGED_BAD_PAGE);
    }
    pages = out ? 0 : id;
  };
  // where the page of a key starts, from the pool's start (page numbers are not negative
  // here: unsigned products take half the instructions)
  auto page_at = [&](int key) {
    const uint32_t page = __builtin_amdgcn_readlane(pages, (key >> a.pool.page_shift) - pbase);
    return page * static_cast<uint64_t>(a.pool.page_bytes);
  };

  constexpr int GB = S::kFp8 ? D : OB;                  // bytes of a row in its page
  constexpr int LPR = GB / 16;                          // lanes of a row
  constexpr int RPI = kWave / LPR;                      // rows of one load instruction
  constexpr int NLD = KT / RPI / NW;                    // load instructions of a wave, per operand
  static_assert(KT % RPI == 0 && KT / RPI % NW == 0 && NLD >= 1, "whole loads");
  static_assert(RPI <= 16, "the rows of one load lie in one page");
  // Row first_row(i) + lane / LPR, chunk lane % LPR.  A lane's place in its row is
  // chunk ^ swizzle; what of the swizzle depends on i is a constant, since
  // first_row(i) and lane / LPR share no bits.
  const int lrow = lane / LPR, wrow0 = wave * RPI;
  auto row_of = [&](int i) { return NW * i * RPI; };   // first_row(i) - wrow0
  const uint32_t lane_row = static_cast<uint32_t>(lrow) * a.pool.token_bytes;
  const uint32_t kc = 16 * ((lane % LPR) ^ (S::kRegs ? 0 : k_swz<RB>(wrow0 + lrow)));
  const uint32_t vc = 16 * ((lane % LPR) ^ (S::kRegs ? 0 : v_swz<VS, RB>(wrow0 + lrow)));
  uint4 kr[S::kRegs ? NLD : 1], vr[S::kRegs ? NLD : 1];
  // The window holds the pages of keys from .. to (fewer than 64 pages), `from` and later
  // ones being all that is still needed.
  auto cover = [&](int from, int to) {
    if ((min(to, kend) - 1) >> a.pool.page_shift >= pbase + kWave) load_pages(from >> a.pool.page_shift);
  };
  const int big_page = a.pool.page_shift >= (KT == 64 ? 6 : 5);   // a page holds whole tiles
  const uint32_t token_bytes = a.pool.token_bytes;
  auto load = [&](bool is_v, uint32_t buf, int i, const char* p, uint32_t row_off) {
    const uint32_t off = row_off + (is_v ? vc ^ (S::kRegs ? 0 : 16 * v_swz<VS, RB>(row_of(i)))
                                         : kc ^ (S::kRegs ? 0 : 16 * k_swz<RB>(row_of(i))));
    if constexpr (S::kRegs) (is_v ? vr : kr)[i] = *reinterpret_cast<const uint4*>(p + off);
    else dma16(p, off, lds0 + buf + (is_v ? V_AT : 0) + (wrow0 + row_of(i)) * RB);
  };
  auto issue = [&](bool is_v, uint32_t buf, int k0) {
    const char* pool = is_v ? vpool : kpool;
    if (k0 + KT > kend) {
      // the range ends inside the tile: lanes behind it read its last key again
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const int key = k0 + wrow0 + row_of(i);
        load(is_v, buf, i, pool + page_at(min(key, kend - 1)),
             static_cast<uint32_t>(min(key + lrow, kend - 1) & psm) * token_bytes);
      }
    } else if (big_page) {
      const char* p = pool + page_at(k0) + static_cast<uint32_t>((k0 & psm) + wrow0) * token_bytes;
#pragma unroll
      for (int i = 0; i < NLD; ++i) load(is_v, buf, i, p + row_of(i) * token_bytes, lane_row);
    } else {
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const int key = k0 + wrow0 + row_of(i);
        load(is_v, buf, i, pool + page_at(key) + static_cast<uint32_t>(key & psm) * token_bytes, lane_row);
      }
    }
  };
  // what was issued last for K or V is complete and in LDS
  auto commit = [&](bool is_v, uint32_t buf) {
    if constexpr (S::kRegs) {
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const int r = wrow0 + row_of(i) + lrow, c = 2 * (lane % LPR);
        const int sw = is_v ? v_swz<VS, RB>(r) : k_swz<RB>(r);
        const uint4 w = (is_v ? vr : kr)[i];
        char* row = sm + buf + (is_v ? V_AT : 0) + r * RB;
        *reinterpret_cast<bf16x8*>(row + 16 * (c ^ sw)) = fp8x8_to_bf16x8(w.x, w.y);
        *reinterpret_cast<bf16x8*>(row + 16 * ((c + 1) ^ sw)) = fp8x8_to_bf16x8(w.z, w.w);
      }
    } else {
      dma_wait();
    }
  };

  // ---- one tile ----
  f32x16 o[D / 32];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[i][v] = 0.f;

  // Fragment addresses: chunk 2 s + h of K row lr is at k_at ^ 32 s, the V^T operand
  // of dims 32 db + lr in the key order of the accumulators at v_at ^ (64 db) (bf16,
  // four keys a read) or v_at ^ (128 db) (f32, one key), plus whole rows.
  // codes: eight keys a read, at v_at ^ (32 db)
  const int i16 = lane % 16, half16 = (lane / 16) % 2;
  const int vr0 = S::kCodes ? 8 * (i16 / 8) + 4 * hl + i16 / 2 % 4 : ES == 2 ? 4 * hl + i16 / 4 : 4 * hl;
  const uint32_t k_at = lds0 + lr * RB + 16 * (hl ^ k_swz<RB>(lr));
  const uint32_t v_at =
      lds0 + V_AT + vr0 * RB +
      (S::kCodes ? 16 * (half16 ^ v_swz<VS, RB>(vr0)) + 8 * (i16 & 1)
       : ES == 2 ? 16 * ((2 * half16 + (i16 % 4) / 2) ^ v_swz<VS, RB>(vr0)) + 8 * (i16 & 1)
                 : 16 * ((lr / 4) ^ v_swz<VS, RB>(vr0)) + 4 * (lr % 4));
  auto v_bf16 = [&](uint32_t at, int t, int db) {
    if constexpr (S::kCodes) {
      const s32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
          reinterpret_cast<__attribute__((address_space(3))) s32x2*>((at ^ (32u * db)) + 16 * t * RB));
      return fp8x8_to_bf16x8(w.x, w.y);
    } else {
      union { s16x4 h[2]; bf16x8 v; } f;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        f.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<__attribute__((address_space(3))) s16x4*>((at ^ (64u * db)) + (16 * t + 8 * j) * RB));
      return f.v;
    }
  };
  auto v_f32 = [&](uint32_t at, int kb, int v, int db) {
    return lds_at<float>((at ^ (128u * db)) + (32 * kb + 8 * (v / 4) + v % 4) * RB);
  };

  // S^T of one tile
  auto scores = [&](f32x16 (&st)[KB], uint32_t buf) {
    const uint32_t ka = k_at ^ buf;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) st[kb][v] = 0.f;
#pragma unroll
    for (int s = 0; s < NQ; s += S::kCodes ? 2 : 1)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const u32x4 kv4 = lds_at<u32x4>((ka ^ (S::kCodes ? 16u * s : 32u * s)) + 32 * kb * RB);
        const uint4 kf = make_uint4(kv4.x, kv4.y, kv4.z, kv4.w);
        if constexpr (S::kCodes) {
          st[kb] = mfma32x32x16(fp8x8_to_bf16x8(kf.x, kf.y), as_bf16x8(qf[s]), st[kb]);
          st[kb] = mfma32x32x16(fp8x8_to_bf16x8(kf.z, kf.w), as_bf16x8(qf[s + 1]), st[kb]);
        } else if constexpr (ES == 2) {
          st[kb] = mfma32x32x16(as_bf16x8(kf), as_bf16x8(qf[s]), st[kb]);
        } else {
          st[kb] = mfma_f32(__uint_as_float(kf.x), __uint_as_float(qf[s].x), st[kb]);
          st[kb] = mfma_f32(__uint_as_float(kf.y), __uint_as_float(qf[s].y), st[kb]);
          st[kb] = mfma_f32(__uint_as_float(kf.z), __uint_as_float(qf[s].z), st[kb]);
          st[kb] = mfma_f32(__uint_as_float(kf.w), __uint_as_float(qf[s].w), st[kb]);
        }
      }
    if constexpr (ES == 4) mfma_settle();
  };
  // this lane's largest score (its half of the tile's keys)
  auto half_max = [&](const f32x16 (&st)[KB]) {
    float mx[2 * KB];
#pragma unroll
    for (int c = 0; c < 2 * KB; ++c) {
      const f32x16& x = st[c >> 1];
      const int f = 8 * (c & 1);
      float m = max3(x[f], x[f + 1], x[f + 2]);
      m = max3(m, x[f + 3], x[f + 4]);
      m = max3(m, x[f + 5], x[f + 6]);
      mx[c] = max2(m, x[f + 7]);
    }
    if constexpr (KB == 2) return max3(max2(mx[0], mx[1]), mx[2], mx[3]);
    else return max2(mx[0], mx[1]);
  };
  // hidden keys get -inf, only in tiles where a row of the wave has any
  auto hide = [&](f32x16 (&st)[KB], float& tmax, int k0) {
    if (__ballot(k0 < lo || k0 + KT > hi) == 0) return;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = k0 + 32 * kb + 8 * (v / 4) + 4 * hl + v % 4;
        st[kb][v] = key >= lo && key < hi ? st[kb][v] : -INFINITY;
      }
    tmax = half_max(st);
  };
  // The reference m moves only when a tile's maximum exceeds it by more than 8
  // (powers of two: p stays below 2^8), so the accumulators are rescaled a few
  // times per key range and not at every tile.
  auto rescale = [&](float half) {
    const float tmax = pair_max(half) * sl2;
    if (__ballot(tmax > m_run + 8.f)) {
      const float m_new = fmaxf(m_run, tmax);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] *= alpha;
      m_run = m_new;
    }
  };
  // P^T of one tile as the B operand, and its sum into l.  The matrix cores take 16-bit
  // operands here, so beside bf16 values p is rounded to bf16 (half a step, 2^-8 of it); a
  // second term for the rest would double the products of V.  l sums the p that are not
  // rounded.  Over hundreds of keys the roundings average out: the output's own rounding is 1.7e-3
  // of its size, and this adds up to 0.04e-3 (four requests of 816 rows over 816 keys).
  auto weights = [&](f32x16 (&st)[KB], bf16x8 (&pf)[2 * KB]) {
    const float m_use = m_run == -INFINITY ? 0.f : m_run;   // nothing seen yet: every p is 0
    float ps[2 * KB];
#pragma unroll
    for (int t = 0; t < 2 * KB; ++t) {
      float pv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pv[j] = __builtin_amdgcn_exp2f(fmaf(st[t >> 1][8 * (t & 1) + j], sl2, -m_use));
        if constexpr (ES == 4) st[t >> 1][8 * (t & 1) + j] = pv[j];
      }
      ps[t] = ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
      if constexpr (ES == 2) {
        uint4 w;
        w.x = pack_bf16x2(pv[0], pv[1]);
        w.y = pack_bf16x2(pv[2], pv[3]);
        w.z = pack_bf16x2(pv[4], pv[5]);
        w.w = pack_bf16x2(pv[6], pv[7]);
        pf[t] = as_bf16x8(w);
      }
    }
    if constexpr (KB == 2) l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
    else l_run += ps[0] + ps[1];
  };
  // O^T += V^T P^T
  auto values = [&](const f32x16 (&st)[KB], const bf16x8 (&pf)[2 * KB], uint32_t buf) {
    const uint32_t tv = v_at ^ buf;
    if constexpr (ES == 2) {
#pragma unroll
      for (int t = 0; t < 2 * KB; ++t)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) o[db] = mfma32x32x16(v_bf16(tv, t, db), pf[t], o[db]);
    } else {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
#pragma unroll
          for (int db = 0; db < D / 32; ++db) o[db] = mfma_f32(v_f32(tv, kb, v, db), st[kb][v], o[db]);
    }
  };

  // Scores of the next tile and values of this one, written out in the order in which
  // they are to issue, one product after another: N1 of K Q^T, then N2 of V^T P^T, each
  // with the LDS reads of the product PD further on and its share of the exponentials.
  // The P of a group of 16 keys is ready when the first product that takes it comes.
  // Left to itself the compiler puts the N1 products first and all vector work beside
  // the N2 (head_dim 128, 4,096 rows over 8,192 keys: 485 us).
  auto scores_and_values = [&](f32x16 (&next)[KB], const f32x16 (&st)[KB], uint32_t buf) {
    constexpr int DB = D / 32, N1 = KB * NQ, N2 = 2 * KB * DB, N = N1 + N2, NE = 16 * KB, SPAN = N - DB, PD = 4;
    const uint32_t ka = k_at ^ buf ^ TILE, tv = v_at ^ buf;
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    bf16x8 frag[PD], pf[2 * KB];
    float pv[8], ps[2 * KB];
    auto read = [&](int i) {
      if (i < N1) {
        const u32x4 w = lds_at<u32x4>((ka ^ (32u * (i / KB))) + 32 * (i % KB) * RB);
        frag[i % PD] = __builtin_bit_cast(bf16x8, w);
      } else if (i < N) {
        frag[i % PD] = v_bf16(tv, (i - N1) / DB, (i - N1) % DB);
      }
    };
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) next[kb][v] = 0.f;
#pragma unroll
    for (int i = 0; i < PD; ++i) read(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i < N1) next[i % KB] = mfma32x32x16(frag[i % PD], as_bf16x8(qf[i / KB]), next[i % KB]);
      else o[(i - N1) % DB] = mfma32x32x16(frag[i % PD], pf[(i - N1) / DB], o[(i - N1) % DB]);
      read(i + PD);
      const int e0 = i * NE / SPAN, e1 = (i + 1) * NE / SPAN;
#pragma unroll
      for (int e = e0; e < e1 && e < NE; ++e) {
        const int t = e / 8, j = e % 8;
        pv[j] = __builtin_amdgcn_exp2f(fmaf(st[t >> 1][8 * (t & 1) + j], sl2, -m_use));
        if (j == 7) {
          ps[t] = ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
          pf[t] = as_bf16x8(make_uint4(pack_bf16x2(pv[0], pv[1]), pack_bf16x2(pv[2], pv[3]), pack_bf16x2(pv[4], pv[5]),
                                       pack_bf16x2(pv[6], pv[7])));
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (KB == 2) l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
    else l_run += ps[0] + ps[1];
  };

  // ---- the key range ----
  if constexpr (KEYS) {
    // One buffer each: K's is refilled once the scores are computed, V's once the values
    // are, so a wave has most of a tile in flight at any time, and many waves fit a CU.
    if (kbeg < kend) {
      auto wait = [&](bool last) {                      // all loads but the youngest tile's
        if (last) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NLD) : "memory");
      };
      // other lanes read what a lane wrote, and loads overwrite what lanes have read: LDS
      // operations of a wave complete in order, the compiler has to keep that order
      auto fence = [&] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
      load_pages(kbeg >> a.pool.page_shift);
      issue(false, 0, kbeg);
      issue(true, 0, kbeg);
      wait(false);
      for (int k0 = kbeg;; k0 += KT) {
        const bool more = k0 + KT < kend;
        f32x16 st[KB];
        bf16x8 pf[2 * KB];
        scores(st, 0);
        if constexpr (VS == 2) mfma_pipeline<KB * NQ, 1, 4>();
        fence();
        if (more) {
          cover(k0 + KT, k0 + 2 * KT);
          issue(false, 0, k0 + KT);
        }
        float half = half_max(st);
        hide(st, half, k0);
        rescale(half);
        weights(st, pf);
        wait(!more);
        values(st, pf, 0);
        if constexpr (VS == 2) mfma_pipeline<2 * KB * (D / 32), 2, 2>();
        if (!more) break;
        fence();
        issue(true, 0, k0 + KT);
        wait(false);
      }
    }
  } else if constexpr (!S::kAhead) {
    if (kbeg < kend) {
      // two buffers: the next tile is under way while this one is worked on
      uint32_t buf = 0;
      load_pages(kbeg >> a.pool.page_shift);
      issue(false, 0, kbeg);
      issue(true, 0, kbeg);
      commit(false, 0);
      commit(true, 0);
      lds_barrier();
      for (int k0 = kbeg;; k0 += KT, buf ^= TILE) {
        const bool more = k0 + KT < kend;
        if (more) {
          cover(k0 + KT, k0 + 2 * KT);
          issue(false, buf ^ TILE, k0 + KT);
          issue(true, buf ^ TILE, k0 + KT);
        }
        f32x16 st[KB];
        bf16x8 pf[2 * KB];
        scores(st, buf);
        if constexpr (ES == 2) mfma_pipeline<KB * NQ, 1, 4>();
        float half = half_max(st);
        hide(st, half, k0);
        rescale(half);
        weights(st, pf);
        values(st, pf, buf);
        if constexpr (ES == 2) mfma_pipeline<2 * KB * (D / 32), 2, 2>();
        if (!more) break;
        commit(false, buf ^ TILE);
        commit(true, buf ^ TILE);
        lds_barrier();
      }
    }
  } else {
    if (kbeg < kend) {
      // The scores of tile t + 1 are computed beside the exponentials of tile t, so that
      // the matrix cores work while the vector units do: K runs a tile ahead of V.
      // K(t) and V(t) lie in buffer t % 2; step t reads K(t + 1) and V(t) and loads
      // K(t + 2) and V(t + 1), whose buffers the step before was the last to read.
      f32x16 st[KB];
      bf16x8 pf[2 * KB];
      load_pages(kbeg >> a.pool.page_shift);
      issue(false, 0, kbeg);
      issue(true, 0, kbeg);
      commit(false, 0);
      commit(true, 0);
      if (kbeg + KT < kend) {
        issue(false, TILE, kbeg + KT);
        commit(false, TILE);
      }
      lds_barrier();
      scores(st, 0);
      float half = half_max(st);
      hide(st, half, kbeg);
      lds_barrier();
      uint32_t buf = 0;
      int k0 = kbeg;
      for (; k0 + KT < kend; k0 += KT, buf ^= TILE) {
        const bool more = k0 + 2 * KT < kend;
        cover(k0 + KT, k0 + 3 * KT);
        if (more) issue(false, buf, k0 + 2 * KT);
        issue(true, buf ^ TILE, k0 + KT);
        rescale(half);
        f32x16 next[KB];
        scores_and_values(next, st, buf);
        half = half_max(next);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) st[kb] = next[kb];
        hide(st, half, k0 + KT);
        if (more) commit(false, buf);
        commit(true, buf ^ TILE);
        lds_barrier();
      }
      rescale(half);
      weights(st, pf);
      values(st, pf, buf);
    }
  }
  l_run = pair_sum(l_run);

  // A hidden key's weight is 0, and 0 times an infinite or NaN value is NaN: where a row
  // came out NaN although its weights are numbers, and a key that it does not see but
  // its block does holds such a value, it is computed once more over the keys that it
  // sees and no other, with the maximum m and sum l found above.  The last key stands
  // again, hidden, behind the end of a last tile that is not full.
  float nan = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) nan += o[i][v];
  const uint64_t nan_lanes = __ballot(valid && nan != nan && l_run == l_run);
  const uint32_t nan_rows = static_cast<uint32_t>(nan_lanes) | static_cast<uint32_t>(nan_lanes >> 32);
  auto repair = [&](int rr, float m, float l) {
    constexpr int E = D / kWave, U = 8;
    const int t = rr / G;
    const int64_t head = kvh * G + rr % G;
    auto elem = [](const char* p, int e) {
      if constexpr (S::kFp8) return __uint_as_float(fp8x2_to_bf16x2<false>(reinterpret_cast<const uint8_t*>(p)[e]) << 16);
      else return ActIO<T>::load(reinterpret_cast<const T*>(p) + e);
    };
    // this lane's part of a key's row; the pages were checked when they were loaded
    auto row_at = [&](int key) {
      const int id = table[key >> a.pool.page_shift];
      return page_row_offset(a.pool, page_ok(id, a.pool.n_pages) ? id : 0, key, kvh) + (int64_t)E * lane * sizeof(CT);
    };
    const int first = max(kbeg, seen_begin(t, n, kv, a.window)), end = min(kend, seen_end(t, n, kv, a.causal));
    bool hidden = false;                                // at most a tile and the block's rows on either side
    const int behind = (kend - kbeg) % KT ? min(end, kend - 1) : end;
    for (int key = kbeg; key < kend; ++key) {
      if (key == first && first < end) key = behind;
      if (key >= kend) break;
      const int64_t at = row_at(key);
#pragma unroll
      for (int e = 0; e < E; ++e) hidden |= !(fabsf(elem(a.pool.v + at, e)) < INFINITY);
    }
    if (__ballot(hidden) == 0) return;
    const T* qp = static_cast<const T*>(a.q.p) + b * a.q.b + t * a.q.t + head * a.q.h + E * lane;
    float q[E], acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[e] = ActIO<T>::load(qp + e);
      acc[e] = 0.f;
    }
    for (int k0 = first; k0 < end; k0 += U) {
      float s[U], v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = row_at(min(k0 + u, end - 1));
        s[u] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          s[u] = fmaf(q[e], elem(a.pool.k + at, e), s[u]);
          v[u][e] = elem(a.pool.v + at, e);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float p = __builtin_amdgcn_exp2f(fmaf(wave_sum(s[u]), sl2, -m));
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = k0 + u < end ? fmaf(p, v[u][e], acc[e]) : acc[e];
      }
    }
    if (a.n_split == 1) {
      T* op = static_cast<T*>(a.out.p) + b * a.out.b + t * a.out.t + head * a.out.h + E * lane;
#pragma unroll
      for (int e = 0; e < E; ++e) ActIO<T>::store(op + e, l == 0.f ? 0.f : acc[e] * (vs / l));
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) a.part[((grow + rr) * a.n_split + split) * D + E * lane + e] = acc[e];
    }
  };

  // ---- out ----
  // an unusable page or length makes the block's rows NaN
  if constexpr (!KEYS) {
    if (bad && lane == 0) s_bad = 1;
    __syncthreads();
    bad = __builtin_amdgcn_readfirstlane(s_bad) != 0;
  }
  if (bad) {
    m_run = 0.f;
    l_run = __builtin_nanf("");
  }
  if (a.n_split > 1) {
    if (valid) {
      const int64_t at = (grow + row) * a.n_split + split;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          *reinterpret_cast<float4*>(a.part + at * D + 32 * db + 8 * u + 4 * hl) =
              make_float4(o[db][4 * u], o[db][4 * u + 1], o[db][4 * u + 2], o[db][4 * u + 3]);
      if (hl == 0) a.ml[at] = make_float2(m_run, l_run);
    }
  } else {
    // whole rows through LDS, so that a store instruction covers 1 KiB of them
    const float inv = l_run == 0.f ? 0.f : vs / l_run;
    char* stage = sm + wave * 32 * OB;
    static_assert(S::LDS >= NW * 32 * OB, "the output is staged in the tiles");
    constexpr int SW = CPR < 16 ? CPR - 1 : 15;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float v4[4] = {o[db][4 * u] * inv, o[db][4 * u + 1] * inv, o[db][4 * u + 2] * inv, o[db][4 * u + 3] * inv};
        const int byte = (32 * db + 8 * u + 4 * hl) * ES;
        ActIO<T>::store4(reinterpret_cast<T*>(stage + lr * OB + 16 * ((byte / 16) ^ (lr & SW)) + byte % 16), v4);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int RPS = kWave / CPR > 0 ? kWave / CPR : 1;
#pragma unroll
    for (int i = 0; i < 32 / RPS; ++i) {
      const int r = RPS * i + lane / CPR, c = lane % CPR;
      const int rr = wrow + r;
      if (rr < rows) {
        const uint4 w = *reinterpret_cast<const uint4*>(stage + r * OB + 16 * (c ^ (r & SW)));
        char* op = reinterpret_cast<char*>(static_cast<T*>(a.out.p) + b * a.out.b + (rr / G) * a.out.t +
                                           (kvh * G + rr % G) * a.out.h);
        *reinterpret_cast<uint4*>(op + 16 * c) = w;
      }
    }
  }
  if (nan_rows && !bad) {
    dma_wait();                                         // the rows above are written
    for (uint32_t left = nan_rows; left; left &= left - 1) {
      const int r = __builtin_ctz(left);
      repair(wrow + r, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m_run), r)),
             __int_as_float(__builtin_amdgcn_readlane(__float_as_int(l_run), r)));
    }
  }
}

// Joins the splits of a row: o = sum_s w_s o_s / sum_s w_s l_s, w_s = 2^(m_s - max m).
// W waves take the splits of a row in turn, eight loads under way each, and add up in
// LDS in a fixed order.  Splits without a key have l = 0 and are not taken.
template <typename T, int D, int W>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a, bool fp8) {
  constexpr int E = D / kWave;
  __shared__ float part_sum[W > 1 ? W : 1][D];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int MG = a.M * a.G, wr = wave % W;
  const int64_t gr = (int64_t)blockIdx.x * (4 / W) + wave / W;
  if (gr >= (int64_t)a.B * a.nkv * MG) return;
  const int grp = static_cast<int>(gr / MG), row = static_cast<int>(gr % MG);
  const int b = grp / a.nkv, kvh = grp % a.nkv;
  // requested together: every split's (m, l), and the length
  float2 x = make_float2(-INFINITY, 0.f);
  if (lane < a.n_split) x = a.ml[gr * a.n_split + lane];
  const RowSpan span = row_span(a.new_len ? a.new_len[b] : a.M, 0, a.M, a.M);
  if (row >= span.n * a.G) return;
  const float l = x.y;
  float mm = l == 0.f ? -INFINITY : x.x;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) mm = fmaxf(mm, __shfl_xor(mm, s, kWave));
  const float w = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(x.x - mm);
  const float total = wave_sum(l == 0.f ? 0.f : w * l);
  const uint64_t live = __ballot(l != 0.f);
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  const float* part = a.part + gr * a.n_split * D + E * lane;
  for (int s0 = 8 * wr; s0 < a.n_split; s0 += 8 * W) {
    if ((live >> s0 & 0xff) == 0) continue;
    float v[8][E];
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = part[(int64_t)min(s0 + k, a.n_split - 1) * D + e];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float ws = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), (s0 + k) & 63));
      const bool take = s0 + k < a.n_split && (live >> (s0 + k) & 1);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(ws, take ? v[k][e] : 0.f, acc[e]);
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) part_sum[wr][E * lane + e] = acc[e];
    __syncthreads();
    if (wr > 0) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      acc[e] = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) acc[e] += part_sum[k][E * lane + e];
    }
  }
  const float inv = total == 0.f ? 0.f : (fp8 ? a.pool.v_scale[kvh] : 1.f) / total;
  T* op = static_cast<T*>(a.out.p) + b * a.out.b + (row / a.G) * a.out.t + (kvh * a.G + row % a.G) * a.out.h + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) ActIO<T>::store(op + e, acc[e] * inv);
}

// Which shape: of few rows the keys shape, whose waves each stream keys of their own, of
// more the rows shape, whose four waves share a tile.  Figures in us, keys | rows shape:
//   bf16, head_dim 128, 32 requests over 4,096 keys, 8 K/V heads: 4 rows 114 | 110, 8 rows
//     120 | 115, 16 rows 129 | 118, 32 rows 146 | 121; 64 ragged requests of 4 rows 128 | 144, of 8
//     rows of 256: 41 | 56; eight requests: 4 rows 30.9 | 31.3, 16 rows 35.8 | 32.6; one request:
//     4 rows 12.1 | 12.4, 32 rows 14.4 | 15.3.
//   8 bits, the same: 4 rows 64 | 78, 8 rows 69 | 79, 16 rows 78 | 80, 32 rows 93 | 83.
//   32 bits, bound by its products, of which the rows shape does those of 128 rows
//     whatever there are: 64 requests of 4 rows 179 | 520, 4 requests over 2,048 keys of 32
//     rows 25 | 30, of 64 rows 29 | 33, of 128 rows 39 | 39.  At head_dim 256 a wave's rows,
//     accumulators and a tile exceed its registers: 4 rows 61 | 48, 64 requests 1,134 | 1,085;
//     there is no keys shape for it.
// Rows or pairs: where the CUs have about one block each and more would come only of a split,
// the rows shape (816 rows of four requests of 8 heads over 816 keys: 41 us, pairs 55, 57
// split in two); else pairs (four requests over 4,096 keys, 32, 64, 96, 128 rows: 15.6, 17.9,
// 20.5, 23.2 us, the rows shape 17.5, 21.1, 23.9, 26.9).  The plan's cost decides.  Widening
// 8-bit codes takes registers that a second wave does not leave.
template <typename CT, typename T, int D>
constexpr bool kHasPairs = sizeof(CT) == 2 && D == 256;
template <typename CT, typename T, int D>
constexpr int kKeysRows = sizeof(T) == 4 ? (D == 256 ? 0 : 64) : sizeof(CT) == 1 ? 16 : 8;

template <typename CT, typename T, int D, Block BLK>
void launch(const PagedAttnArgs& a, hipStream_t s) {
  const int64_t total = (int64_t)a.B * a.nkv * a.n_split * a.n_tiles;
  const int grid = static_cast<int>((total + 7) / 8 * 8);
  paged_attn_kernel<CT, T, D, BLK><<<grid, 64 * Shape<CT, T, D, BLK>::NW, 0, s>>>(a);
  if (a.n_split > 1) {
    const int64_t rows = (int64_t)a.B * a.nkv * a.M * a.G;
    if (a.n_split <= 8) paged_join_kernel<T, D, 1><<<static_cast<int>((rows + 3) / 4), 256, 0, s>>>(a, sizeof(CT) == 1);
    else paged_join_kernel<T, D, 4><<<static_cast<int>(rows), 256, 0, s>>>(a, sizeof(CT) == 1);
  }
}

template <typename CT, typename T, int D>
void launch_shape(const PagedAttnArgs& a, hipStream_t s) {
  if constexpr (kKeysRows<CT, T, D> > 0)
    if (a.M * a.G <= kKeysRows<CT, T, D>) return launch<CT, T, D, kKeys>(a, s);
  if constexpr (kHasPairs<CT, T, D>)
    if (a.pairs) return launch<CT, T, D, kPairs>(a, s);
  launch<CT, T, D, kRows>(a, s);
}

// What a launch costs without a window, in us where kRows and kPairs are compared.
template <typename CT, typename T, int D, Block BLK>
double plan(PagedAttnArgs& a) {
  using S = Shape<CT, T, D, BLK>;
  constexpr bool KEYS = S::KEYS;
  // us of a tile with every slot of a CU taken, measured; a block of pairs alone on its CU
  // takes 1.95
  constexpr double kTile = kHasPairs<CT, T, D> ? (BLK == kPairs ? 2.4 : 2.8)
                                               : 2.2 * S::KT / 64 * D / 128 * (sizeof(T) == 4 ? 16 : 1);
  a.n_tiles = (a.M * a.G + S::ROWS - 1) / S::ROWS;
  const int64_t base = (int64_t)a.B * a.nkv * a.n_tiles;
  const int64_t slots = 256 * S::PER_CU;
  // Splits are of equal length, so that a launch over ragged requests is made of equal
  // blocks.  A block costs its tiles plus two or three to start and finish, joining two.
  //   rows: bound by the blocks' own work, a launch costs whole rounds of blocks over the
  //     chip (4,096 rows over 8,192 keys, two rounds unsplit: 432 us, two splits 498; 64
  //     rows of eight requests: 86 us unsplit, 64, 66, 60, 76 with 2, 3, 4, 8 splits).
  //   keys: bound by memory, of which a few waves a CU are enough; what costs is the half
  //     round in which some blocks have ended, and of ragged requests many have nothing
  //     to do (64 tokens over 600 .. 4,000 keys: 195 us unsplit, 148 with one round of
  //     four splits, 132 .. 139 with 5 to 24; all of 2,300 keys: 120 unsplit, 128 .. 138).
  //     The parts of a split are written and read at 4.7 TB/s.
  double least = 1e300;
  auto choose = [&](int steps, int most) {
    int best = 1;
    least = 1e300;
    for (int n = 1; n <= std::min(most, steps); ++n) {
      const int per = (steps + n - 1) / n;
      if ((steps + per - 1) / per != n) continue;       // the last splits would be empty
      const double rounds = static_cast<double>(base) * n / slots;
      const double parts = KEYS || n == 1 ? 0.0 : base * n * (S::ROWS * D * 8 / 4.7e6) / kTile;
      const double alone = BLK == kPairs && base * n <= 256 ? 1.95 / 2.4 : 1.0;
      const double cost = (KEYS ? (std::max(1.0, rounds) + 0.5) * (per + 3) : std::ceil(rounds) * (per + 2) * alone) +
                          (n > 1 ? 2 : 0) + parts;
      if (cost < least) {
        least = cost;
        best = n;
      }
      if (base * n >= 4 * slots) break;
    }
    return best;
  };
  // the longest range of a block; the workspace is sized without the window
  const int steps = std::max(1, (a.max_kv + S::KT - 1) / S::KT);
  a.n_split = choose(steps, 64);
  const double us = least * kTile;
  int span = steps;
  if (a.window > 0) {
    const int64_t keys = (int64_t)a.window + (S::ROWS - 1) / a.G + 1;
    span = static_cast<int>(std::min<int64_t>(steps, (keys + S::KT - 1) / S::KT + 1));
    a.n_split = choose(span, a.n_split);
  }
  a.split_keys = (span + a.n_split - 1) / a.n_split * S::KT;
  return us;
}

template <typename CT, typename T, int D>
void plan_shape(PagedAttnArgs& a) {
  if constexpr (kKeysRows<CT, T, D> > 0)
    if (a.M * a.G <= kKeysRows<CT, T, D>) {
      plan<CT, T, D, kKeys>(a);
      return;
    }
  const double us = plan<CT, T, D, kRows>(a);
  if constexpr (kHasPairs<CT, T, D>) {
    // compared without the window, which the size of the workspace does not know
    PagedAttnArgs p = a;
    p.pairs = 1;
    if (plan<CT, T, D, kPairs>(p) < us) a = p;
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

}  // namespace

int64_t paged_attention_plan(PagedAttnArgs& a, int D, int pool_kind) {
  by_dim(D, [&](auto d) {
    constexpr int kD = decltype(d)::value;
    if (pool_kind == PAGED_F32) plan_shape<float, float, kD>(a);
    else if (pool_kind == PAGED_BF16) plan_shape<bf16_t, bf16_t, kD>(a);
    else plan_shape<uint8_t, bf16_t, kD>(a);
  });
  if (a.n_split == 1) return 0;
  return (int64_t)a.B * a.nkv * a.M * a.G * a.n_split * (D + 2);
}

void paged_attention(const PagedAttnArgs& a, int D, int pool_kind, hipStream_t s) {
  by_dim(D, [&](auto d) {
    constexpr int kD = decltype(d)::value;
    if (pool_kind == PAGED_F32) launch_shape<float, float, kD>(a, s);
    else if (pool_kind == PAGED_BF16) launch_shape<bf16_t, bf16_t, kD>(a, s);
    else launch_shape<uint8_t, bf16_t, kD>(a, s);
  });
}

}  // namespace phyai
