// Attention of whole prompts (the S_q > 1 arm of Sec. 3.3): causal, packed sequences of different lengths, grouped
// heads, fp16 or bf16, on the matrix cores.
//
// A row is one (token, query head) pair; the rows of a sequence that share a KV head are numbered token by token,
// token * gqa + head, and a block takes 64 to 256 consecutive ones (so that the heads of a group share every tile of
// K and V, and a block's rows span few tokens: little is computed that the causal mask throws away, and a short
// sequence fills its blocks).  A wave has 32 rows; at head_dim 512 four waves share 32.  Block n works on the n-th
// block of rows from the end (the longest rows of keys first: what is left for the last compute units is short).
//
// Scores are computed transposed, S^T = K Q^T (32 keys x 32 rows to an instruction, A = K, B = Q): a lane then
// holds 16 keys of ONE row, the softmax's maxima and sums stay in the lane up to one exchange between the wave's
// halves, and the accumulator's layout is that of the B operand of O^T = V^T P^T up to the order of the keys, which
// both operands may share in any order.  The A operand V^T comes out of the row-major tile by the transposing LDS
// read.  Online softmax (Alg. 1) over tiles of keys.
//
// The weights are rounded to the inputs' type because the matrix instruction's operands are that type; their sum takes
// the rounded ones, so that a row's weights still sum to one.  Everything else is 32 bits up to the output's rounding.
//
// Floor: 4 D (attended pairs) H_q operations on the matrix cores; the bytes (q, k, v and out once) are a tenth of that from
// about 1500 tokens on.  A 32x32x16 product is 32 clocks of a SIMD, and the 16 exponentials, 16 multiply-adds, 8
// conversions and 8 sums per 32 keys x 32 rows and lane are 8 (exp) or 4 clocks each when one wave issues them, half that when two do:
// at head_dim 128 as much as the half of its 16 products, which is why each kernel below is arranged around having the two at
// the same time.
#include <cfloat>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "tq_internal.h"

namespace tq {
namespace {

typedef float float16v __attribute__((ext_vector_type(16)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

struct PrefillParams {
  const uint16_t* q;          // rows of q_stride elements per token, head h at h * D
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;              // [n_tokens][n_q_heads][D]
  const int32_t* cu_seqlens;  // [n_seqs + 1]
  int64_t q_stride, k_stride, v_stride;
  int32_t n_tokens, n_seqs, n_q_heads, n_kv_heads, gqa, window;
  int32_t slots;              // row tiles per KV head that the grid has room for
  uint32_t q_flip;            // 0x80008000 for a negative scale: q with the other sign
  float scale_log2;           // |attn_scale| * log2(e)
};

// what differs between the two types: the instruction, and the rounding of the weights and the output
template <bool BF16>
struct Type;
template <>
struct Type<false> {
  typedef _Float16 vec8 __attribute__((ext_vector_type(8)));
  typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float16v mfma(vec8 a, vec8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Type<true> {
  typedef __bf16 vec8 __attribute__((ext_vector_type(8)));
  typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ float16v mfma(vec8 a, vec8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {     // round to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{a, b}, typename Type<BF16>::vec2));
}

// acc + both of the weights in w, as rounded
template <bool BF16>
__device__ __forceinline__ float add2(uint32_t w, float acc) {
  if constexpr (BF16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Type<true>::vec2, w), Type<true>::vec2{1.0f, 1.0f}, acc, false);
  else return __builtin_amdgcn_fdot2(__builtin_bit_cast(Type<false>::vec2, w), Type<false>::vec2{(_Float16)1.0f, (_Float16)1.0f}, acc, false);
}

// Where piece c (16 bytes) of row r lies in an LDS tile.  The score product's operand is read with one row to a lane, the
// same piece of 32 rows at a time: any 8 consecutive rows have to differ in the banks.  The transposing reads take
// 64 bytes of four consecutive rows: there the rows have to differ above those 64 bytes.
__device__ __forceinline__ int k_piece(int r, int c) { return c ^ (r & 15); }
__device__ __forceinline__ int v_piece(int r, int c) { return c ^ ((r & 3) << 2); }

// Direct global -> LDS load of 16 bytes per lane: lane l's bytes land at m0 + 16 l.  Written as asm so that the compiler does not
// wait for the loads at every later LDS read: wait_loads and a barrier stand in front of the tile's first one.  (M0
// cannot be named as a clobber; the compiler keeps no value live in it across other instructions.)
__device__ __forceinline__ void dma16(const void* sbase, uint32_t voff, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(voff), "s"(sbase), "s"(m0) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void block_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// V^T as the A operand of 16 keys and 32 dims, out of a row-major tile: lane: dim lane % 32, keys 4 hi + 0..3 and 8 + 4 hi + 0..3 (the
// order in which the scores' accumulator leaves a lane's weights).  The transposing read hands lane i of 16 the i-th of 16 dims that
// four lanes' addresses name for each of four keys.
template <int ROWB>
__device__ __forceinline__ uint32_t v_read(int lane, int d) {    // the lane's offset in a tile, for dims 32 d ...
  const int r = 4 * (lane >> 5) + (lane & 15) / 4;
  return r * ROWB + v_piece(r, d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2) * 16 + (lane & 1) * 8;
}
template <bool BF16, int ROWB>
__device__ __forceinline__ typename Type<BF16>::vec8 v_operand(const char* at) {
  typedef __attribute__((address_space(3))) short4v* lds_ptr;
  const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at));
  const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 8 * ROWB)));
  return __builtin_bit_cast(typename Type<BF16>::vec8, uint4v{x[0], x[1], y[0], y[1]});
}

// The same value, which the compiler does not know: what is worked out from it stays where it is used, instead of in registers across the
// loop.  (Neighbouring LDS offsets of a lane's reads differ in bits that no row's arrangement carries out of: an exclusive or leads
// from one to the next.)
__device__ __forceinline__ uint32_t fresh(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// For the scheduler: AHEAD LDS reads, then TIMES matrix instructions with READS reads behind each.  Left alone it puts every read
// right in front of its use.
template <int AHEAD>
__device__ __forceinline__ void order_reads() { __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0); }
template <int TIMES, int READS>
__device__ __forceinline__ void order_products() {
#pragma unroll
  for (int i = 0; i < TIMES; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
}

// Eight dims of a lane's row, 16 i + 8 hi .. of 32, divided by its sum: the wave's halves exchange what they hold of 16.
template <bool BF16>
__device__ __forceinline__ uint4v eight_dims(const float16v& o, int i, float inv) {
  uint32_t x[2], y[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t a = pack2<BF16>(o[8 * i + 2 * j] * inv, o[8 * i + 2 * j + 1] * inv);
    const uint32_t b = pack2<BF16>(o[8 * i + 4 + 2 * j] * inv, o[8 * i + 4 + 2 * j + 1] * inv);
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    x[j] = r[0];
    y[j] = r[1];
  }
  return uint4v{x[0], x[1], y[0], y[1]};
}
// A lane's row of the output, straight to memory.
template <bool BF16, int DT>
__device__ __forceinline__ void store_row(uint16_t* dst, const float16v (&o)[DT], float inv, int hi) {
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4v*>(dst + d * 32 + 16 * i + 8 * hi) = eight_dims<BF16>(o[d], i, inv);
}

// The 32 rows of a wave, from row0 on (past the sequence's last row: that one again).
struct WaveRows {
  int first;                  // the first row's token
  int rel0, rel_last, gqa;    // rows counted from that token's first
  float inv_gqa;
  __device__ __forceinline__ WaveRows(const PrefillParams& p, int row0, int n_rows) {
    gqa = p.gqa;
    const int r0 = min(row0, n_rows - 1);
    first = r0 / gqa;
    rel0 = r0 - first * gqa;
    rel_last = n_rows - 1 - first * gqa;
    inv_gqa = __builtin_amdgcn_rcpf((float)gqa);
  }
  // Row i of the 32, counted from the first token's first, and its token, counted from the first.  (The quotient keeps 1 / (2 gqa) off the next integer.  Its
  // error is 2^-22 of it; it is below 33, and below 2 from gqa = 32 on, and gqa is at most 2^17: rows of 2^24 elements hold no more heads.)
  __device__ __forceinline__ void at(int i, int& rel, int& token) const {
    rel = min(rel0 + i, rel_last);
    token = (int)(((float)rel + 0.5f) * inv_gqa);
  }
  // Bytes from the first token's first row of the KV head to row i, where tokens are `stride` elements apart (fewer than 2^24: 33 of them are
  // inside 32 bits).
  template <int D>
  __device__ __forceinline__ uint32_t bytes(int i, int64_t stride) const {
    int rel, token;
    at(i, rel, token);
    return (uint32_t)rel * (D * 2) + (uint32_t)token * ((uint32_t)stride - (uint32_t)(gqa * D)) * 2;
  }
};

// Queries come, and the output leaves, by way of LDS ([32 rows][D] per wave, pieces as in a tile of K): both sides of memory then see whole
// rows, where a lane's own row would be 32 bytes of 32 rows to an instruction.  us per call, a lane's own rows / by way of LDS: head_dim 128,
// 64 heads over 8, 24 prompts of 17 to 2048 tokens 323 / 314, 32 of 512 242 / 237, 2048 79 / 76, 173 7.8 / 7.8.  At head_dim 256 the output alone, in blocks of
// eight waves: windows of 256 in two prompts of 8192 287 / 272, of 1024 623 / 611; in the small grids of blocks of four waves it costs 0.5 us
// (54 tokens 8.2 / 8.8), and for the queries' addresses there are no registers.
template <int D>
__device__ __forceinline__ void load_queries(const PrefillParams& p, const WaveRows& w, int begin, int kv, uint32_t to) {
  constexpr int CH = D / 8;
  const int lane = threadIdx.x & 63;
  const uint16_t* const base = p.q + (int64_t)(begin + w.first) * p.q_stride + (int64_t)kv * p.gqa * D;
#pragma unroll
  for (int u = 0; u < CH / 2; ++u) {
    const int r = (u * 64 + lane) / CH, c = (u * 64 + lane) % CH;
    dma16(base, w.bytes<D>(r, p.q_stride) + k_piece(r, c) * 16, to + u * 1024);
  }
}
template <bool BF16, int D>
__device__ __forceinline__ void store_rows(const PrefillParams& p, const WaveRows& w, int begin, int kv, int n_left, char* lds, const float16v (&o)[D / 32],
                                           float inv) {
  constexpr int CH = D / 8;
  const int lane = threadIdx.x & 63, c32 = lane & 31, hi = lane >> 5;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<uint4v*>(lds + c32 * (D * 2) + k_piece(c32, d * 4 + 2 * i + hi) * 16) = eight_dims<BF16>(o[d], i, inv);
  char* const base = reinterpret_cast<char*>(p.out + ((int64_t)(begin + w.first) * p.n_q_heads + kv * p.gqa) * D);
#pragma unroll
  for (int u = 0; u < CH / 2; ++u) {
    const int r = (u * 64 + lane) / CH, c = (u * 64 + lane) % CH;
    const uint4v x = *reinterpret_cast<const uint4v*>(lds + r * (D * 2) + k_piece(r, c) * 16);
    if (r < n_left) *reinterpret_cast<uint4v*>(base + w.bytes<D>(r, (int64_t)p.n_q_heads * D) + c * 16) = x;
  }
}

// The rows of a slot: `ROWS` consecutive ones of one sequence.
struct Rows {
  int begin, len;             // the sequence's tokens
  int tile_row, n_rows;       // the first row (outside of [0, n_rows): nothing to do), and all rows per KV head of the sequence
  int t_lo, t_hi;             // first and last of the rows' tokens
};
__device__ __forceinline__ Rows find_rows(const PrefillParams& p, int slot, int rows) {
  // Where the row tiles of sequence b start in the list of all: one per sequence is lost at most, none overlap.  (All tokens have fewer
  // than 2^31 - 256 rows per KV head: a launch has fewer than 2^23 blocks.)
  auto token = [&](int i) { return min(max(p.cu_seqlens[i], 0), p.n_tokens); };
  auto base = [&](int at, int b) { return at * p.gqa / rows + b; };
  // the last sequence that starts at or before the slot: 64 candidates at a time
  const int lane = threadIdx.x & 63;
  int b = 0, n = p.n_seqs, begin, end, first_slot;
  for (;;) {
    const int step = (n + 63) >> 6, i = b + min(lane * step, n - 1);
    const int at = token(i), next = token(i + 1);               // (the end counts in the last round, where candidates are neighbours)
    const int slot_of = base(at, i);
    const int last = 63 - __clzll((long long)(__ballot(lane * step < n && slot_of <= slot) | 1));
    b += last * step;
    n = min(step, n - last * step);
    begin = __builtin_amdgcn_readlane(at, last);
    end = __builtin_amdgcn_readlane(next, last);
    first_slot = __builtin_amdgcn_readlane(slot_of, last);
    if (step == 1) break;
  }
  Rows r;
  r.begin = begin;
  r.len = max(end, begin) - begin;
  r.tile_row = (slot - first_slot) * rows;
  r.n_rows = r.len * p.gqa;
  r.t_lo = r.tile_row / p.gqa;
  r.t_hi = min(r.tile_row + rows - 1, r.n_rows - 1) / p.gqa;
  return r;
}

// ---- head_dim 256: 64 KB of LDS hold two tiles of K and of V, 32 keys each.  A row's output (128 registers) and queries (64) leave no room for a
// second unit of scores in flight as at head_dim 128; eight waves take turns instead (see below).  Measured: two sequences of 5003 tokens, 32
// heads over 16, window 1024: 357 us, 840 TFLOP/s, 0.73 of a large product of the library; 8192 tokens without a window 910 us, 1210 TFLOP/s, at
// the power limit.  What bounds it: a tile takes 3630 clocks where its products alone take 2048 (a barrier and the first LDS reads
// of every turn), and a block, alone on its compute unit, has about 10 us of start and end (queries 128 KB, output 128 KB) beside 1.7 us per
// tile.  (Not kept: loads by the waves in their arithmetic turn, and queries by way of LDS, which both spilled registers; both
// kinds of work in one wave as at 128, likewise; a lane's own row of the output straight to memory, see store_rows.)
template <int NW_>
struct Cfg256 {
  static constexpr int D = 256, NW = NW_, ROWS = NW * 32, BN = 32;
  static constexpr int KS = D / 16, DT = D / 32, CH = D / 8, ROWB = D * 2, TILE = BN * ROWB, LPW = TILE / 1024 / NW;
  static constexpr int SMEM = NW == 8 ? ROWS * ROWB : 4 * TILE;     // two tiles of K, two of V; the output
};

template <int NW, bool BF16>
__global__ __launch_bounds__(NW * 64, 2) void prefill256_kernel(PrefillParams p) {
  using C = Cfg256<NW>;
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  constexpr int D = C::D;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  const int kv = blockIdx.x % p.n_kv_heads;
  const Rows rows = find_rows(p, p.slots - 1 - (int)(blockIdx.x / p.n_kv_heads), C::ROWS);      // long rows of keys first
  if (rows.tile_row < 0 || rows.tile_row >= rows.n_rows) return;
  const int begin = rows.begin, len = rows.len;

  const int first = p.window > 0 ? max(0, rows.t_lo - p.window + 1) : 0;
  const int n_tiles = (rows.t_hi - first) / C::BN + 1;
  const char* const kb = reinterpret_cast<const char*>(p.k + begin * p.k_stride + (int64_t)kv * D);
  const char* const vb = reinterpret_cast<const char*>(p.v + begin * p.v_stride + (int64_t)kv * D);
  const uint32_t k_row = (uint32_t)p.k_stride * 2, v_row = (uint32_t)p.v_stride * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  // Load i of a tile fills the tile's i-th 1024 bytes; its lane fetches the piece that belongs at the lane's place.
  // Rows past the sequence's last token repeat it (finite values that weights of zero meet).
  auto issue = [&](const char* base, uint32_t row_bytes, auto piece, int tile, uint32_t to) {
    const int k0 = first + tile * C::BN;
    base += (int64_t)k0 * row_bytes;
    const int last = len - 1 - k0;
#pragma unroll
    for (int u = 0; u < C::LPW; ++u) {
      const int i = u * C::NW + wave;                               // 1 KB pieces go around the waves
      const int r = i * 64 / C::CH + lane / C::CH, c = (i * 64 + lane) % C::CH;
      dma16(base, (uint32_t)min(r, last) * row_bytes + piece(r, c) * 16, to + i * 1024);
    }
  };
  auto issue_k = [&](int tile) { issue(kb, k_row, k_piece, tile, lds0 + (tile & 1) * C::TILE); };
  auto issue_v = [&](int tile) { issue(vb, v_row, v_piece, tile, lds0 + (2 + (tile & 1)) * C::TILE); };
  issue_k(0);

  // this lane's row
  const int row = rows.tile_row + wave * 32 + c32, my_row = min(row, rows.n_rows - 1);
  const int token = my_row / p.gqa, head = kv * p.gqa + my_row - token * p.gqa;
  vec8 q[C::KS];
  {
    const uint16_t* const src = p.q + (begin + token) * p.q_stride + (int64_t)head * D + hi * 8;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      uint4v x = *reinterpret_cast<const uint4v*>(src + s * 16);
      x ^= p.q_flip;
      q[s] = __builtin_bit_cast(vec8, x);
    }
  }
  float16v o[C::DT];
#pragma unroll
  for (int d = 0; d < C::DT; ++d) o[d] = float16v{};
  float m = -INFINITY, l = 0.0f;                      // log2 units; l: this lane's half of the keys
  const int w_lo = __builtin_amdgcn_readfirstlane(token);                         // the wave's tokens
  const int w_hi = __builtin_amdgcn_readlane(token, 31);
  const int oldest = p.window > 0 ? token - p.window + 1 : 0;

  const uint32_t k_at0 = c32 * C::ROWB + k_piece(c32, hi) * 16, v_at0 = 2 * C::TILE + v_read<C::ROWB>(lane, 0);   // LDS offsets of this lane's reads

  // tiles that some row of this wave attends
  const int t_first = p.window > 0 ? max(0, w_lo - p.window + 1 - first) / C::BN : 0, t_last = (w_hi - first) / C::BN;

  float16v s;
  uint32_t w[8];
  auto score = [&](int tile) {                        // S^T of a tile
    const char* const k_lds = smem + (tile & 1) * C::TILE;
    const uint32_t k_at = fresh(k_at0);
    s = float16v{};
#pragma unroll
    for (int i = 0; i < C::KS; ++i) s = T::mfma(*reinterpret_cast<const vec8*>(k_lds + (k_at ^ ((i & 7) * 32)) + (i >> 3) * 256), q[i], s);
  };
  auto weigh = [&](int tile) {                        // masks, maximum, weights
    const int k0 = first + tile * C::BN;
    if (k0 + C::BN - 1 > w_lo || (p.window > 0 && k0 <= w_hi - p.window)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + 8 * (i / 4) + 4 * hi + i % 4;
        s[i] = key > token || key < oldest ? -INFINITY : s[i];
      }
    }
    float top = s[0], x, y;
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    swap32(top, x, y);
    top = fmaxf(x, y) * p.scale_log2;
    // The reference may lag behind the maximum by a factor of 2^8 in the weights, which neither the types nor the sums
    // mind: most tiles then leave the accumulators as they are.
    if (__any(top > m + 8.0f)) {
      const float m_new = fmaxf(m, top);
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < C::DT; ++d) o[d] *= alpha;
    }
    const float ref = m == -INFINITY ? 0.0f : m;      // (no key of this row yet)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[2 * i], p.scale_log2, -ref));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], p.scale_log2, -ref));
      w[i] = pack2<BF16>(p0, p1);
      l = add2<BF16>(w[i], l);
    }
  };
  auto accumulate = [&](int tile) {
    const char* const v_lds = smem + (tile & 1) * C::TILE;
    const uint32_t v_at = fresh(v_at0);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const vec8 pb = __builtin_bit_cast(vec8, uint4v{w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]});
#pragma unroll
      for (int d = 0; d < C::DT; ++d)
        o[d] = T::mfma(v_operand<BF16, C::ROWB>(v_lds + (v_at ^ ((d & 3) * 64)) + h * 16 * C::ROWB + (d >> 2) * 256), pb, o[d]);
    }
  };

  // Blocks of eight waves: the two waves of a SIMD take turns.  While one is at its matrix instructions (the weights of tile t - 1
  // meet V, tile t meets the queries), the other works out its weights; left alone they run in step, and the two kinds of work one after the
  // other.  Turns are barriers; waves 0 to 3 have their matrix turn for tile t in turn 2 t, waves 4 to 7 in turn 2 t + 1.  K of tile t is in use
  // in those two turns and V in the two after; at the start of turn 2 t the next loads begin, and they have two turns.  Blocks of four waves
  // have nobody to take turns with, and a barrier only where the loads want one.
  const int off = NW == 8 ? wave >> 2 : 0;
  auto turn = [&](int i) {
    const bool loads = (i & 1) == 0;
    if (NW == 4 && !loads) return;
    if (loads) wait_loads();
    block_barrier();
    if (loads) {
      const int t = i >> 1;
      if (t + 1 < n_tiles) issue_k(t + 1);
      if (t < n_tiles) issue_v(t);
    }
  };
  int i = 0;
  while (i < 2 * t_first + off) turn(i++);
  turn(i++);
  score(t_first);
  turn(i++);
  weigh(t_first);
  if (t_first < t_last) {
    int t = t_first;
    do {
      turn(i);
      if constexpr (NW == 8) __builtin_amdgcn_s_setprio(1);       // (in front of the other's arithmetic: 8192 tokens 916 / 908 us)
      accumulate(t);
      score(t + 1);
      order_reads<6>();
      order_products<13, 2>();
      order_products<16, 1>();
      order_products<3, 0>();
      if constexpr (NW == 8) __builtin_amdgcn_s_setprio(0);
      turn(i + 1);
      ++t;
      i += 2;
      weigh(t);
    } while (t < t_last);
  }
  turn(i++);
  accumulate(t_last);
  while (i < 2 * n_tiles + 2) turn(i++);

  float l0, l1;
  swap32(l, l0, l1);
  const float inv = 1.0f / (l0 + l1);                 // (a row has at least its own token)
  if constexpr (NW == 8) {
    block_barrier();                                  // (everybody has done with the tiles)
    const int row0 = rows.tile_row + wave * 32;
    store_rows<BF16, D>(p, WaveRows(p, row0, rows.n_rows), begin, kv, rows.n_rows - row0, smem + wave * (32 * C::ROWB), o, inv);
  } else if (row < rows.n_rows) {
    store_row<BF16, C::DT>(p.out + ((int64_t)(begin + token) * p.n_q_heads + head) * D, o, inv, hi);
  }
}

// ---- head_dim 128
// Work goes in units of 32 keys, two to a tile.  Of three neighbouring units one is scored, one is weighed and one is accumulated
// at the same time (step): the three have no dependence on each other, so that the arithmetic of the second fills the issue slots
// between the matrix instructions of the others.
// Measured, 64 heads over 8: 16384 tokens 4.0 ms, 1100 TFLOP/s (a large product of the library: 1154); matrix cores at work 67 % of the
// time at 1.4 GHz, to which the card's power limit brings the clock (an earlier version at 54 % ran at 1.8 GHz in nearly the same time); 24 sequences of 17 to
// 2048 tokens (bf16) 316 us, 43 % at 1.95 GHz: there a block's 41 thousand clocks are 1400 of look-up, 3300 until its queries are there, 2600
// to the first weights, 2900 per tile, 3400 for the masked tile, 2100 for the end, 2800 to store, and 2300 until the next block has begun.  173 tokens
// 8.4 us, of which 5 are latency: look-up of the rows, queries, first tile, and the units one after the other.
// (Not kept, all slower: 64 rows to a wave, where past 256 registers the accumulators are copied; turns as at 256; three tiles ahead with
// eight waves to a block; an order for the scheduler with the arithmetic's instructions between the products.)
struct Cfg128 {
  static constexpr int D = 128, NW = 4, ROWS = NW * 32, BN = 64;     // two blocks to a compute unit
  static constexpr int KS = D / 16, DT = D / 32, CH = D / 8, ROWB = D * 2, TILE = BN * ROWB, LPW = TILE / 1024 / NW;
  static constexpr int SMEM = 4 * TILE;              // two tiles of K, two of V
};
// A row's sum of weights from which its reference is brought up to the maximum again.  (fp16 weights are infinite, and so is the
// sum, from 2^16; both formats keep their precision below.)
constexpr float kMuch = 0x1p20f;

template <bool BF16>
__global__ __launch_bounds__(Cfg128::NW * 64, 2) void prefill128_kernel(PrefillParams p) {
  using C = Cfg128;
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  constexpr int D = C::D, NW = C::NW;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  const int kv = blockIdx.x % p.n_kv_heads;
  const Rows rows = find_rows(p, p.slots - 1 - (int)(blockIdx.x / p.n_kv_heads), C::ROWS);      // long rows of keys first
  if (rows.tile_row < 0 || rows.tile_row >= rows.n_rows) return;
  const int begin = rows.begin, len = rows.len;

  const int first = p.window > 0 ? max(0, rows.t_lo - p.window + 1) : 0;
  const int n_tiles = (rows.t_hi - first) / C::BN + 1;
  const uint32_t k_row = (uint32_t)p.k_stride * 2, v_row = (uint32_t)p.v_stride * 2;
  const char* const kb = reinterpret_cast<const char*>(p.k + (int64_t)(begin + first) * p.k_stride + (int64_t)kv * D);
  const char* const vb = reinterpret_cast<const char*>(p.v + (int64_t)(begin + first) * p.v_stride + (int64_t)kv * D);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  // Load u of this wave fills 1024 bytes of a tile; a lane fetches the piece that belongs at its place.  Offsets in a whole tile, and
  // in the last one, where rows past the sequence's last token repeat it (finite values that weights of zero meet).
  uint32_t k_off[2][C::LPW], v_off[2][C::LPW];
  {
    const int last = min(C::BN - 1, len - 1 - first - (n_tiles - 1) * C::BN);
#pragma unroll
    for (int u = 0; u < C::LPW; ++u) {
      const int i = u * NW + wave;                                  // 1 KB pieces go around the waves
      const int r = i * 64 / C::CH + lane / C::CH, c = (i * 64 + lane) % C::CH;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        k_off[e][u] = (uint32_t)(e ? min(r, last) : r) * k_row + k_piece(r, c) * 16;
        v_off[e][u] = (uint32_t)(e ? min(r, last) : r) * v_row + v_piece(r, c) * 16;
      }
    }
  }
  auto load_k = [&](int t) {
    if (t >= n_tiles) return;
#pragma unroll
    for (int u = 0; u < C::LPW; ++u)
      dma16(kb + (int64_t)(t * C::BN) * k_row, t == n_tiles - 1 ? k_off[1][u] : k_off[0][u], lds0 + (t & 1) * C::TILE + (u * NW + wave) * 1024);
  };
  auto load_v = [&](int t) {
    if (t >= n_tiles) return;
#pragma unroll
    for (int u = 0; u < C::LPW; ++u)
      dma16(vb + (int64_t)(t * C::BN) * v_row, t == n_tiles - 1 ? v_off[1][u] : v_off[0][u], lds0 + (2 + (t & 1)) * C::TILE + (u * NW + wave) * 1024);
  };
  const int row0 = rows.tile_row + wave * 32;
  const WaveRows mine(p, row0, rows.n_rows);
  const int q_at = 2 * C::TILE + wave * (32 * C::ROWB);            // (the tiles of V come later)
  load_queries<D>(p, mine, begin, kv, lds0 + q_at);
  load_k(0);

  // this lane's row, and its queries
  int rel, token;
  mine.at(c32, rel, token);
  token += mine.first;
  vec8 q[C::KS];
  wait_loads();
#pragma unroll
  for (int s = 0; s < C::KS; ++s) {
    uint4v x = *reinterpret_cast<const uint4v*>(smem + q_at + c32 * C::ROWB + k_piece(c32, 2 * s + hi) * 16);
    x ^= p.q_flip;
    q[s] = __builtin_bit_cast(vec8, x);
  }
  float16v o[C::DT];
#pragma unroll
  for (int d = 0; d < C::DT; ++d) o[d] = float16v{};
  float m = -INFINITY, l = 0.0f;                      // log2 units; l: this lane's half of the keys
  const int w_lo = __builtin_amdgcn_readfirstlane(token), w_hi = __builtin_amdgcn_readlane(token, 31);   // the wave's tokens

  uint32_t k_at[8], v_at[4];                          // LDS offsets of this lane's reads
#pragma unroll
  for (int i = 0; i < 8; ++i) k_at[i] = c32 * C::ROWB + k_piece(c32, 2 * i + hi) * 16;
#pragma unroll
  for (int d = 0; d < 4; ++d) v_at[d] = 2 * C::TILE + v_read<C::ROWB>(lane, d);

  // Units that some row of this wave attends; the one by which every row has met a key; the last that no row's own token cuts short
  const int u_first = p.window > 0 ? max(0, w_lo - p.window + 1 - first) / 32 : 0, u_last = (w_hi - first) / 32;
  const int u_all = p.window > 0 ? max(0, w_hi - p.window + 1 - first) / 32 : 0;
  const int u_whole = (w_lo - 31 - first) >> 5;
  auto active = [&](int u) { return u >= u_first && u <= u_last; };

  typedef uint32_t Weights[8];
  auto score = [&](float16v& s, int u) {              // S^T of a unit
    const char* const k_lds = smem + ((u >> 1) & 1) * C::TILE + (u & 1) * (32 * C::ROWB);
    s = float16v{};
#pragma unroll
    for (int i = 0; i < C::KS; ++i) s = T::mfma(*reinterpret_cast<const vec8*>(k_lds + k_at[i]), q[i], s);
  };
  auto mask = [&](float16v& s, int u) {               // (key 8 (i / 4) + 4 hi + i % 4 of the unit)
    const int from = first + u * 32 + 4 * hi, newest = token - from;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 > newest ? -INFINITY : s[i];
    if (p.window > 0) {
      const int oldest = newest - p.window + 1;       // (where this wraps, newest < 0 and all of the unit is masked already)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 < oldest ? -INFINITY : s[i];
    }
  };
  auto top_of = [&](const float16v& s) {              // the row's largest score
    float top = s[0], x, y;
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    swap32(top, x, y);
    return fmaxf(x, y) * p.scale_log2;
  };
  auto refer = [&](float top) {                       // the reference becomes the maximum
    if (!__any(top > m)) return;
    const float m_new = fmaxf(m, top);
    const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int d = 0; d < C::DT; ++d) o[d] *= alpha;
  };
  auto weigh = [&](const float16v& s, Weights& w) {
    const float ref = m == -INFINITY ? 0.0f : m;      // (no key of this row yet)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[2 * i], p.scale_log2, -ref));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], p.scale_log2, -ref));
      w[i] = pack2<BF16>(p0, p1);
      l = add2<BF16>(w[i], l);
    }
  };
  auto accumulate = [&](const Weights& w, int u) {
    const char* const v_lds = smem + ((u >> 1) & 1) * C::TILE + (u & 1) * (32 * C::ROWB);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const vec8 pb = __builtin_bit_cast(vec8, uint4v{w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]});
#pragma unroll
      for (int d = 0; d < C::DT; ++d) o[d] = T::mfma(v_operand<BF16, C::ROWB>(v_lds + v_at[d] + h * 16 * C::ROWB), pb, o[d]);
    }
  };
  // Score, weigh and accumulate three units in a row.  The reference stays what it is (a maximum is 8 instructions and an exchange that
  // all wait for each other) unless the weights show that it lags too far behind.
  auto step = [&](auto masked, float16v& scored, const float16v& weighed, Weights& w, const Weights& wa, int ua) {
    const float l_before = l;
    __builtin_amdgcn_s_setprio(1);                    // (while it lasts the SIMD's other wave, of another block, waits its turn: us per call
    score(scored, ua + 2);                            //  2048 tokens 78.2 / 75.7, 4096 of 32 heads over 32 136 / 132)
    weigh(weighed, w);
    accumulate(wa, ua);
    if constexpr (masked) mask(scored, ua + 2);
    order_reads<6>();
    order_products<8, 1>();
    order_products<5, 2>();
    order_products<3, 0>();
    __builtin_amdgcn_s_setprio(0);
    if (__any(!(l < kMuch))) {
      float x, y;
      swap32(l, x, y);
      const float over = !(fmaxf(x, y) < kMuch) ? m + 9.0f : -INFINITY;      // (of the row: both halves of the wave)
      l = l_before;
      refer(fmaxf(top_of(weighed), over));
      weigh(weighed, w);
    }
  };
  float16v s0, s1;
  Weights w0, w1;
  // Before tile t: unit 2 t is weighed (w0), unit 2 t + 1 scored (s1).  K of tile t + 1 and V of tile t are here, and the loads of K of
  // tile t + 2 and V of tile t + 1 take the place of what has served.
  int tile = -1;
  auto sync = [&]() {
    wait_loads();
    block_barrier();
    load_v(tile + 1);
  };
  auto slow = [&]() {
    sync();
    load_k(tile + 2);
    if (active(2 * tile)) accumulate(w0, 2 * tile);
    if (active(2 * tile + 1)) {
      refer(top_of(s1));
      weigh(s1, w1);
      accumulate(w1, 2 * tile + 1);
    }
    if (active(2 * tile + 2)) {
      score(s0, 2 * tile + 2);
      mask(s0, 2 * tile + 2);
      refer(top_of(s0));
      weigh(s0, w0);
    }
    if (active(2 * tile + 3)) {
      score(s1, 2 * tile + 3);
      mask(s1, 2 * tile + 3);
    }
    ++tile;
  };
  // From unit u_all on every row has a reference, and none of its window's start cuts a unit behind that one.
  if (u_all == 0) {
    sync();
    load_k(1);
    score(s0, 0);
    score(s1, 1);
    if (u_whole < 1 || p.window > 0) {
      mask(s0, 0);
      mask(s1, 1);
    }
    m = fmaxf(top_of(s0), top_of(s1));
    weigh(s0, w0);
    tile = 0;
  } else {
    while (tile < min((u_all + 1) >> 1, n_tiles)) slow();
  }
  if (2 * tile + 3 <= u_whole) {
    do {
      sync();
      step(std::false_type{}, s0, s1, w1, w0, 2 * tile);
      load_k(tile + 2);                               // (all loads at once take the waves longer to send off)
      step(std::false_type{}, s1, s0, w0, w1, 2 * tile + 1);
      ++tile;
    } while (2 * tile + 3 <= u_whole);
  }
  for (; 2 * tile + 2 <= u_last; ++tile) {
    sync();
    step(std::true_type{}, s0, s1, w1, w0, 2 * tile);
    load_k(tile + 2);
    step(std::true_type{}, s1, s0, w0, w1, 2 * tile + 1);
  }
  while (tile < n_tiles) slow();
  wait_loads();                                    // (none may arrive after the block's end)
  float l0, l1;
  swap32(l, l0, l1);
  const float inv = 1.0f / (l0 + l1);                 // (a row has at least its own token)
  // (Behind the last tile's barrier nobody reads K any more.)
  store_rows<BF16, D>(p, mine, begin, kv, rows.n_rows - row0, smem + wave * (32 * C::ROWB), o, inv);
}

// ---- head_dim 512: a wave can hold neither 32 rows of the output (256 registers) next to their queries (128) at two waves to a
// SIMD, so teams of four waves share 32 rows.  Of a tile of 64 keys a wave scores 16 (all 512 dims; 16x16 instructions, A = K,
// B = Q), the weights go through LDS, and it accumulates 128 of the 512 dims over all 64 (32x32 instructions).  K and V have one tile each in
// LDS: the next K loads while the weights meet V, the next V while K is scored.  The team's maximum is only exchanged where a score
// passes the one in use by 8 (log2): the waves vote through LDS.
// Measured, 32 heads over one: 4099 tokens (bf16) 600 to 615 us, 900 TFLOP/s; 1024 tokens 57 us.  Matrix cores at work 39 % of the time.  What
// bounds it is the chain of phases, which all eight waves go through in step, with one block to a compute unit: of about 5500 clocks per tile
// the scores take 1800 (their products alone 1024), softmax 530, the barrier behind it 550, the loads' issue 690, the output 1300 (1024).  LDS moves
// 416 KB in that time, 3300 clocks' worth.  (Not kept: four operands read ahead, which spilled registers; K loaded by one team and V by the
// other, 673 us; the next K's loads spread over the products; 64 rows x 64 dims to a wave's output, which reads 32 KB less from LDS, 617 us.)
struct Cfg512 {
  static constexpr int D = 512, TEAMS = 2, NW = 4 * TEAMS, ROWS = 32 * TEAMS, BN = 64;
  static constexpr int ROWB = D * 2, TILE = BN * ROWB;
  static constexpr int P_TEAM = 32 * BN * 2;         // weights of a team: [32 rows][64 keys]
  static constexpr int P_AT = 2 * TILE, M_AT = P_AT + TEAMS * P_TEAM, FLAG_AT = M_AT + NW * 32 * 4;   // M: 32 row maxima (or sums) per wave
  static constexpr int SMEM = FLAG_AT + 16;
};
template <bool BF16>
__device__ __forceinline__ float4v mfma16(typename Type<BF16>::vec8 a, typename Type<BF16>::vec8 b, float4v c) {
  if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

template <bool BF16>
__global__ __launch_bounds__(Cfg512::NW * 64, 2) void prefill512_kernel(PrefillParams p) {
  using C = Cfg512;
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5, c16 = lane & 15, quarter = lane >> 4;
  const int team = wave >> 2, part = wave & 3;
  const int kv = blockIdx.x % p.n_kv_heads;
  const Rows rows = find_rows(p, p.slots - 1 - (int)(blockIdx.x / p.n_kv_heads), C::ROWS);
  if (rows.tile_row < 0 || rows.tile_row >= rows.n_rows) return;
  const int begin = rows.begin, len = rows.len;
  const int row0 = rows.tile_row + team * 32;                           // the team's first row
  auto row_at = [&](int i) { return min(row0 + i, rows.n_rows - 1); };

  const int first = p.window > 0 ? max(0, rows.t_lo - p.window + 1) : 0;
  const int n_tiles = (rows.t_hi - first) / C::BN + 1;
  const char* const kb = reinterpret_cast<const char*>(p.k + begin * p.k_stride + (int64_t)kv * C::D);
  const char* const vb = reinterpret_cast<const char*>(p.v + begin * p.v_stride + (int64_t)kv * C::D);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // A load is a row; rows past the sequence's last token repeat it.
  auto load_k = [&](int tile, int u) {
    const int r = u * C::NW + wave;
    dma16(kb + (int64_t)min(first + tile * C::BN + r, len - 1) * (p.k_stride * 2), k_piece(r, lane) * 16, lds0 + r * C::ROWB);
  };
  auto load_v = [&](int tile, int u) {
    const int r = u * C::NW + wave;
    dma16(vb + (int64_t)min(first + tile * C::BN + r, len - 1) * (p.v_stride * 2), v_piece(r, lane) * 16, lds0 + C::TILE + r * C::ROWB);
  };
  constexpr int LPW = C::BN / C::NW;
#pragma unroll
  for (int u = 0; u < LPW; ++u) load_k(0, u);

  vec8 q[2][16];                                     // rows c16 and c16 + 16
  int token[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = row_at(16 * g + c16);
    token[g] = row / p.gqa;
    const int head = kv * p.gqa + row - token[g] * p.gqa;
    const uint16_t* const src = p.q + (begin + token[g]) * p.q_stride + (int64_t)head * C::D + quarter * 8;
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      uint4v x = *reinterpret_cast<const uint4v*>(src + s * 32);
      x ^= p.q_flip;
      q[g][s] = __builtin_bit_cast(vec8, x);
    }
  }
  const int t_first = __builtin_amdgcn_readfirstlane(token[0]), t_last = __builtin_amdgcn_readlane(token[1], 15);
  float16v o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) o[d] = float16v{};
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
  float m_out = -INFINITY;                           // the same maximum, of the output's row c32

  // LDS offsets of this lane's reads and writes
  const uint32_t k_at0 = (16 * part + c16) * C::ROWB + k_piece(c16, quarter) * 16;
  const uint32_t v_at0 = C::TILE + (8 * hi + (lane & 15) / 4) * C::ROWB + v_piece((lane & 15) / 4, ((lane >> 4) & 1) * 2 + (lane & 3) / 2) * 16 +
                         (lane & 1) * 8 + part * 256;
  char* const p_lds = smem + C::P_AT + team * C::P_TEAM;                // weights of a row: eight pieces of eight keys
  auto p_at = [&](int row, int piece) { return row * 128 + (piece ^ ((row >> 1) & 7)) * 16; };   // (two rows to a turn of the banks)
  const uint32_t p_wr0 = p_at(c16, 2 * part + (quarter >> 1)) + (quarter & 1) * 8, p_rd0 = p_at(c32, hi);
  float* const maxima = reinterpret_cast<float*>(smem + C::M_AT) + team * 128;   // [part][row]
  typedef __attribute__((address_space(3))) volatile int lds_int;        // (a generic pointer's accesses would wait for the tile loads)
  lds_int* const flags = (lds_int*)(smem + C::FLAG_AT);
  if (threadIdx.x < 2) flags[threadIdx.x] = 0;

  for (int tile = 0; tile < n_tiles; ++tile) {
    wait_loads();
    block_barrier();                                 // K is here; everybody has done with V
    if (threadIdx.x == 0) flags[(tile + 1) & 1] = 0;
    const int k0 = first + tile * C::BN;
    float4v s[2] = {float4v{}, float4v{}};
    constexpr int kFrags = 2;                        // operands read ahead of their use (four do not fit into the registers)
    vec8 a[2][kFrags];
    const uint32_t k_at = fresh(k_at0);
#pragma unroll
    for (int i = 0; i < kFrags; ++i) a[0][i] = *reinterpret_cast<const vec8*>(smem + (k_at ^ ((i & 3) * 64)) + (i >> 2) * 256);
#pragma unroll
    for (int j = 0; j < 16 / kFrags; ++j) {
#pragma unroll
      for (int u = 0; u < LPW * kFrags / 16; ++u) load_v(tile, j * (LPW * kFrags / 16) + u);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kFrags; ++i) {
        const int n = (j + 1) * kFrags + i;
        if (n < 16) a[(j + 1) & 1][i] = *reinterpret_cast<const vec8*>(smem + (k_at ^ ((n & 3) * 64)) + (n >> 2) * 256);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kFrags; ++i)
#pragma unroll
        for (int g = 0; g < 2; ++g) s[g] = mfma16<BF16>(a[j & 1][i], q[g][j * kFrags + i], s[g]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (k0 + C::BN - 1 > t_first || (p.window > 0 && k0 <= t_last - p.window)) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int oldest = p.window > 0 ? token[g] - p.window + 1 : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = k0 + 16 * part + 4 * quarter + i;
          s[g][i] = key > token[g] || key < oldest ? -INFINITY : s[g][i];
        }
      }
    }
    auto weigh = [&]() {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float ref = m[g] == -INFINITY ? 0.0f : m[g];        // (no key of this row yet)
        uint2v w;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          w[i] = pack2<BF16>(__builtin_amdgcn_exp2f(fmaf(s[g][2 * i], p.scale_log2, -ref)),
                             __builtin_amdgcn_exp2f(fmaf(s[g][2 * i + 1], p.scale_log2, -ref)));
        *reinterpret_cast<uint2v*>(p_lds + p_wr0 + g * 2048) = w;
      }
    };
    float top[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) top[g] = fmaxf(fmaxf(s[g][0], s[g][1]), fmaxf(s[g][2], s[g][3])) * p.scale_log2;
    if (__any(top[0] > m[0] + 8.0f || top[1] > m[1] + 8.0f)) {
      if (lane == 0) flags[tile & 1] = 1;
    } else {
      weigh();
    }
    wait_loads();
    block_barrier();                                 // V and the weights are here; everybody has done with K
    if (__builtin_amdgcn_readfirstlane(flags[tile & 1])) {      // (the same answer for the whole block)
      const int at16 = fresh(c16), at32 = fresh(c32);
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        top[g] = blocks_max(top[g]);
        if (quarter == 0) maxima[part * 32 + 16 * g + at16] = top[g];
      }
      block_barrier();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float m_new = m[g];
#pragma unroll
        for (int w = 0; w < 4; ++w) m_new = fmaxf(m_new, maxima[w * 32 + 16 * g + at16]);
        l[g] *= m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[g] - m_new);
        m[g] = m_new;
      }
      float m_new = m_out;
#pragma unroll
      for (int w = 0; w < 4; ++w) m_new = fmaxf(m_new, maxima[w * 32 + at32]);
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_out - m_new);
      m_out = m_new;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= alpha;
      weigh();
      block_barrier();
    }
#pragma unroll
    for (int u = 0; u < LPW; ++u) load_k(min(tile + 1, n_tiles - 1), u);      // (once too often: no branch between here and the products)
#pragma unroll
    for (int g = 0; g < 2; ++g) {                    // (a wave's own weights, as they lie in LDS)
      const uint2v w = *reinterpret_cast<const uint2v*>(p_lds + p_wr0 + g * 2048);
      l[g] = add2<BF16>(w[1], add2<BF16>(w[0], l[g]));
    }
    const uint32_t v_at = fresh(v_at0), p_rd = fresh(p_rd0);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const vec8 pb = *reinterpret_cast<const vec8*>(p_lds + (p_rd ^ (n * 32)));
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        typedef __attribute__((address_space(3))) short4v* lds_ptr;
        const char* const at = smem + (v_at ^ (d * 64)) + n * 16 * C::ROWB;
        const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at));
        const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * C::ROWB)));
        o[d] = T::mfma(__builtin_bit_cast(vec8, uint4v{x[0], x[1], y[0], y[1]}), pb, o[d]);
      }
    }
    order_reads<3 + 8>();
    order_products<12, 2>();
    order_products<4, 0>();
  }
  wait_loads();                                       // (none may arrive after the block's end)
  block_barrier();
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float sum = blocks_sum(l[g]);
    if (quarter == 0) maxima[part * 32 + 16 * g + c16] = sum;
  }
  block_barrier();
  const float inv = 1.0f / (maxima[c32] + maxima[32 + c32] + maxima[64 + c32] + maxima[96 + c32]);
  const int row = row_at(c32);
  const int tok = row / p.gqa, head = kv * p.gqa + row - tok * p.gqa;
  if (row0 + c32 < rows.n_rows)
    store_row<BF16, 4>(p.out + ((int64_t)(begin + tok) * p.n_q_heads + head) * C::D + part * 128, o, inv, hi);
}

// head_dim 256: eight waves to a block, which load a tile for twice the rows, where that leaves every compute unit a block and a half at
// least; else four.  us per call, eight / four, 32 heads over 16, by blocks of eight waves: 54 tokens (16 over 8, 8 blocks) 9.3 / 8.2, 500 (64)
// 32.3 / 28.5, 8 of 300 (304) 42.1 / 34.2, 2048 (256) 108.3 / 104.8, 4 of 1000 (500) 97.9 / 97.4, 4000 (500) 265 / 272, 4000 of 32 over 4
// (500) 251 / 266, 8192 (1024) 940 / 997.
bool wide256(const tq_packed_qkv& x) { return (int64_t)x.n_tokens * x.n_q_heads / Cfg256<8>::ROWS >= 384; }
int block_rows(const tq_packed_qkv& x) {
  return x.head_dim == 128 ? Cfg128::ROWS : x.head_dim == 512 ? Cfg512::ROWS : wide256(x) ? Cfg256<8>::ROWS : Cfg256<4>::ROWS;
}

// Launch with so much LDS (over 64 KB: the function has to be told, once per device).
template <int ID>
hipError_t launch_kernel(void (*kernel)(PrefillParams), const PrefillParams& p, int threads, int lds, hipStream_t s) {
  if (lds > 65536) {
    static std::once_flag configured[64];
    static hipError_t outcome[64];
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    std::call_once(configured[dev], [&] {
      outcome[dev] = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    });
    if (outcome[dev] != hipSuccess) return outcome[dev];
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.slots * (unsigned)p.n_kv_heads), dim3(threads), lds, s, p);
  return hipGetLastError();
}
template <bool BF16>
hipError_t launch(const tq_packed_qkv& x, const PrefillParams& p, hipStream_t s) {
  switch (x.head_dim) {
    case 128: return launch_kernel<128 + BF16>(prefill128_kernel<BF16>, p, Cfg128::NW * 64, Cfg128::SMEM, s);
    case 256:
      return wide256(x) ? launch_kernel<256 + BF16>(prefill256_kernel<8, BF16>, p, 8 * 64, Cfg256<8>::SMEM, s)
                        : launch_kernel<258 + BF16>(prefill256_kernel<4, BF16>, p, 4 * 64, Cfg256<4>::SMEM, s);
    case 512: return launch_kernel<512 + BF16>(prefill512_kernel<BF16>, p, Cfg512::NW * 64, Cfg512::SMEM, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

int prefill_block_rows(const tq_packed_qkv& x) { return block_rows(x); }

int64_t prefill_blocks(const tq_packed_qkv& x, int n_seqs) {
  const int64_t slots = (int64_t)x.n_tokens * (x.n_q_heads / x.n_kv_heads) / block_rows(x) + n_seqs;
  return slots * x.n_kv_heads;
}

hipError_t launch_prefill(const tq_packed_qkv& x, const int32_t* cu_seqlens, int n_seqs, float attn_scale, int window, void* out,
                          hipStream_t s) {
  PrefillParams p;
  p.q = static_cast<const uint16_t*>(x.q);
  p.k = static_cast<const uint16_t*>(x.k);
  p.v = static_cast<const uint16_t*>(x.v);
  p.out = static_cast<uint16_t*>(out);
  p.cu_seqlens = cu_seqlens;
  p.q_stride = x.q_stride;
  p.k_stride = x.k_stride;
  p.v_stride = x.v_stride;
  p.n_tokens = x.n_tokens;
  p.n_seqs = n_seqs;
  p.n_q_heads = x.n_q_heads;
  p.n_kv_heads = x.n_kv_heads;
  p.gqa = x.n_q_heads / x.n_kv_heads;
  p.window = window;
  p.slots = (int)(prefill_blocks(x, n_seqs) / x.n_kv_heads);
  p.q_flip = attn_scale < 0 ? 0x80008000u : 0u;
  // (a scale of zero: so small a one that all weights come out as 1, as they should, and that a masked score stays -inf)
  p.scale_log2 = attn_scale == 0.0f ? FLT_MIN : std::fabs(attn_scale) * 1.4426950408889634f;
  return x.dtype == TQ_DTYPE_BF16 ? launch<true>(x, p, s) : launch<false>(x, p, s);
}

}  // namespace tq
