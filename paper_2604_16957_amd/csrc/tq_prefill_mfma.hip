// Attention of whole prompts (the S_q > 1 arm of Sec. 3.3): causal, packed sequences of different lengths, grouped
// heads, fp16 or bf16, on the matrix cores.
//
// A row is one (token, query head) pair; the rows of a sequence that share a KV head are numbered token by token,
// token * gqa + head, and a block takes kRows consecutive ones (so that the heads of a group share every tile of
// K and V, and a block's rows span few tokens: little is computed that the causal mask throws away, and a short
// sequence fills its blocks).  One wave has 32 rows.
//
// Scores are computed transposed, S^T = K Q^T (32 keys x 32 rows to an instruction, A = K, B = Q): a lane then
// holds 16 keys of ONE row, the softmax's maxima and sums stay in the lane up to one exchange between the wave's
// halves, and the accumulator's layout is that of the B operand of O^T = V^T P^T up to the order of the keys, which
// both operands may share in any order.  The A operand V^T comes out of the row-major tile by the transposing LDS
// read.  Online softmax (Alg. 1) over tiles of keys.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <mutex>

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

template <int D>
struct PrefillCfg {
  // Eight waves, two to a SIMD, share the tiles: one wave's softmax runs beside the other's matrix instructions.  TFLOP/s, 16384 tokens,
  // 64 heads over 8, d = 128, fp16: eight waves of 32 rows 1023, two blocks of four (which load every tile twice as often) 716, four waves of 64
  // rows, one to a SIMD, 858.  d = 256, 32 over 16, 8192 tokens, bf16: tiles of 32 keys 1097, of 64 (which spills) 961.
  static constexpr int NW = 8;                       // waves per block
  static constexpr int RG = 1;                       // groups of 32 rows per wave
  static constexpr int ROWS = NW * RG * 32;
  static constexpr int BN = D == 128 ? 64 : 32;      // keys per tile
  static constexpr int KS = D / 16;                  // k-steps of the score product
  static constexpr int DT = D / 32;                  // 32-dim tiles of the output
  static constexpr int CH = D / 8;                   // 16-byte pieces of a row
  static constexpr int ROWB = D * 2;
  static constexpr int TILE = BN * ROWB;
  static constexpr int LPW = TILE / 1024 / NW;       // 1 KB loads per wave and tile, of K and of V
  static constexpr int SMEM = 4 * TILE;              // K and V, two tiles each
};

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

// where the row tiles of sequence b start in the list of all (one per sequence is lost at most, none overlap)
__device__ __forceinline__ int slot_base(const PrefillParams& p, int b, int rows) {
  const int at = min(max(p.cu_seqlens[b], 0), p.n_tokens);
  return (int)((int64_t)at * p.gqa / rows) + b;
}

// The rows of a slot: `ROWS` consecutive ones of one sequence.
struct Rows {
  int begin, len;             // the sequence's tokens
  int64_t tile_row, n_rows;   // the first row (outside of [0, n_rows): nothing to do), and all rows per KV head of the sequence
  int t_lo, t_hi;             // first and last of the rows' tokens
};
__device__ __forceinline__ Rows find_rows(const PrefillParams& p, int slot, int rows) {
  const int lane = threadIdx.x & 63;
  // the last sequence that starts at or before the slot: 64 candidates at a time
  int b = 0;
  for (int n = p.n_seqs; n > 1;) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool before = i < n && slot_base(p, b + i, rows) <= slot;
    const int last = 63 - __clzll((long long)(__ballot(before) | 1));
    b += last * step;
    n = min(step, n - last * step);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  Rows r;
  r.begin = min(max(p.cu_seqlens[b], 0), p.n_tokens);
  r.len = min(max(p.cu_seqlens[b + 1], r.begin), p.n_tokens) - r.begin;
  r.tile_row = (int64_t)(slot - slot_base(p, b, rows)) * rows;
  r.n_rows = (int64_t)r.len * p.gqa;
  r.t_lo = (int)(r.tile_row / p.gqa);
  r.t_hi = (int)(min(r.tile_row + rows - 1, r.n_rows - 1) / p.gqa);
  return r;
}

template <int D, bool BF16>
__global__ __launch_bounds__(PrefillCfg<D>::NW * 64) void prefill_mfma_kernel(PrefillParams p) {
  using C = PrefillCfg<D>;
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  constexpr int RG = C::RG, NB = C::BN / 32;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  const int kv = blockIdx.x % p.n_kv_heads;
  const Rows rows = find_rows(p, p.slots - 1 - (int)(blockIdx.x / p.n_kv_heads), C::ROWS);      // long rows of keys first
  if (rows.tile_row < 0 || rows.tile_row >= rows.n_rows) return;
  const int begin = rows.begin, len = rows.len, t_lo = rows.t_lo, t_hi = rows.t_hi;
  const int64_t tile_row = rows.tile_row, n_rows = rows.n_rows;
  const int first = p.window > 0 ? max(0, t_lo - p.window + 1) : 0;
  const int n_tiles = (t_hi - first) / C::BN + 1;
  const char* const kb = reinterpret_cast<const char*>(p.k + begin * p.k_stride + (int64_t)kv * D);
  const char* const vb = reinterpret_cast<const char*>(p.v + begin * p.v_stride + (int64_t)kv * D);
  const uint32_t k_row = (uint32_t)p.k_stride * 2, v_row = (uint32_t)p.v_stride * 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  // Load i of a tile fills the tile's i-th 1024 bytes; its lane fetches the piece that belongs at the lane's place.
  // Rows past the sequence's last token repeat it (finite values that weights of zero meet).
  auto issue = [&](int tile) {
    const int k0 = first + tile * C::BN;
    const uint32_t to = lds0 + (tile & 1) * (2 * C::TILE);
    const char* const ks = kb + (int64_t)k0 * k_row;
    const char* const vs = vb + (int64_t)k0 * v_row;
    const int last = len - 1 - k0;
#pragma unroll
    for (int u = 0; u < C::LPW; ++u) {
      const int i = u * C::NW + wave;                               // 1 KB pieces go around the waves
      const int r = i * 64 / C::CH + lane / C::CH, c = (i * 64 + lane) % C::CH;
      const int rr = min(r, last);
      dma16(ks, (uint32_t)rr * k_row + k_piece(r, c) * 16, to + i * 1024);
      dma16(vs, (uint32_t)rr * v_row + v_piece(r, c) * 16, to + C::TILE + i * 1024);
    }
  };
  issue(0);

  // this lane's rows
  int token[RG], head[RG];
  bool mine[RG];
  vec8 q[RG][C::KS];
  float16v o[RG][C::DT];
  float m[RG], l[RG];                                 // log2 units; l: this lane's half of the keys
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    const int64_t row = tile_row + (wave * RG + g) * 32 + c32, my_row = min(row, n_rows - 1);
    mine[g] = row < n_rows;
    token[g] = (int)(my_row / p.gqa);
    head[g] = kv * p.gqa + (int)(my_row - (int64_t)token[g] * p.gqa);
    const uint16_t* const src = p.q + (begin + token[g]) * p.q_stride + (int64_t)head[g] * D + hi * 8;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      uint4v x = *reinterpret_cast<const uint4v*>(src + s * 16);
      x ^= p.q_flip;
      q[g][s] = __builtin_bit_cast(vec8, x);
    }
#pragma unroll
    for (int d = 0; d < C::DT; ++d) o[g][d] = float16v{};
    m[g] = -INFINITY;
    l[g] = 0.0f;
  }
  const int w_lo = __builtin_amdgcn_readfirstlane(token[0]);                      // the wave's tokens
  const int w_hi = __builtin_amdgcn_readlane(token[RG - 1], 31);

  uint32_t k_at[8], v_at[4];                          // LDS offsets of this lane's reads (more pieces, rows: a constant further)
#pragma unroll
  for (int i = 0; i < 8; ++i) k_at[i] = c32 * C::ROWB + k_piece(c32, 2 * i + hi) * 16;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    // Lane: dim 32 d + lane % 32, keys 4 hi + 0..3 and 8 + 4 hi + 0..3 of 16.  The transposing read hands lane i of 16 the i-th
    // of 16 dims that four lanes' addresses name for each of four keys.
    const int r = 4 * hi + (lane & 15) / 4;
    v_at[d] = r * C::ROWB + v_piece(r, d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2) * 16 + (lane & 1) * 8;
  }

  for (int tile = 0; tile < n_tiles; ++tile) {
    wait_loads();
    block_barrier();
    if (tile + 1 < n_tiles) issue(tile + 1);
    const int k0 = first + tile * C::BN;
    if (k0 > w_hi || (p.window > 0 && k0 + C::BN - 1 <= w_lo - p.window)) continue;     // nothing here for this wave
    const char* const k_lds = smem + (tile & 1) * (2 * C::TILE);
    const char* const v_lds = k_lds + C::TILE;
    float16v s[RG][NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int g = 0; g < RG; ++g) s[g][n] = float16v{};
#pragma unroll
      for (int i = 0; i < C::KS; ++i) {
        const vec8 a = *reinterpret_cast<const vec8*>(k_lds + k_at[i & 7] + (n * 32 * C::ROWB + (i >> 3) * 256));
#pragma unroll
        for (int g = 0; g < RG; ++g) s[g][n] = T::mfma(a, q[g][i], s[g][n]);
      }
    }
    if (k0 + C::BN - 1 > w_lo || (p.window > 0 && k0 <= w_hi - p.window)) {
#pragma unroll
      for (int g = 0; g < RG; ++g) {
        const int oldest = p.window > 0 ? token[g] - p.window + 1 : 0;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = k0 + n * 32 + 8 * (i / 4) + 4 * hi + i % 4;
            s[g][n][i] = key > token[g] || key < oldest ? -INFINITY : s[g][n][i];
          }
      }
    }
    uint32_t w[RG][NB][8];
#pragma unroll
    for (int g = 0; g < RG; ++g) {
      float top = s[g][0][0];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[g][n][i]);
      float a, z;
      swap32(top, a, z);
      top = fmaxf(a, z) * p.scale_log2;
      // The reference may lag behind the maximum by a factor of 2^8 in the weights, which neither the types nor the
      // sums mind: most tiles then leave the accumulators as they are.
      if (__any(top > m[g] + 8.0f)) {
        const float m_new = fmaxf(m[g], top);
        const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[g] - m_new);
        m[g] = m_new;
        l[g] *= alpha;
#pragma unroll
        for (int d = 0; d < C::DT; ++d) o[g][d] *= alpha;
      }
      const float ref = m[g] == -INFINITY ? 0.0f : m[g];        // (no key of this row yet)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[g][n][2 * i], p.scale_log2, -ref));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[g][n][2 * i + 1], p.scale_log2, -ref));
          w[g][n][i] = pack2<BF16>(p0, p1);
          l[g] = add2<BF16>(w[g][n][i], l[g]);
        }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int d = 0; d < C::DT; ++d) {
          typedef __attribute__((address_space(3))) short4v* lds_ptr;
          const char* const at = v_lds + v_at[d & 3] + ((n * 32 + h * 16) * C::ROWB + (d >> 2) * 256);
          const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at));
          const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 8 * C::ROWB)));
          const vec8 a = __builtin_bit_cast(vec8, uint4v{x[0], x[1], y[0], y[1]});
#pragma unroll
          for (int g = 0; g < RG; ++g) {
            const vec8 pb = __builtin_bit_cast(vec8, uint4v{w[g][n][4 * h], w[g][n][4 * h + 1], w[g][n][4 * h + 2], w[g][n][4 * h + 3]});
            o[g][d] = T::mfma(a, pb, o[g][d]);
          }
        }
  }
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    float l0, l1;
    swap32(l[g], l0, l1);
    const float inv = 1.0f / (l0 + l1);                 // (a row has at least its own token)
    if (!mine[g]) continue;
    uint16_t* const dst = p.out + ((int64_t)(begin + token[g]) * p.n_q_heads + head[g]) * D;
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2v x = {pack2<BF16>(o[g][d][4 * i] * inv, o[g][d][4 * i + 1] * inv), pack2<BF16>(o[g][d][4 * i + 2] * inv, o[g][d][4 * i + 3] * inv)};
        *reinterpret_cast<uint2v*>(dst + d * 32 + 8 * i + 4 * hi) = x;
      }
  }
}

// ---- head_dim 512: a wave can hold neither 32 rows of the output (256 registers) next to their queries (128) at two waves to a
// SIMD, so teams of four waves share 32 rows.  Of a tile of 64 keys a wave scores 16 (all 512 dims; 16x16 instructions, A = K,
// B = Q), the weights go through LDS, and it accumulates 128 of the 512 dims over all 64 (32x32 instructions).  K and V have one tile each in
// LDS: the next K loads while the weights meet V, the next V while K is scored.  The team's maximum is only exchanged where a score
// passes the one in use by 8 (log2): the waves vote through LDS.
struct TeamCfg {
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
__global__ __launch_bounds__(TeamCfg::NW * 64, 2) void prefill_team_kernel(PrefillParams p) {
  using C = TeamCfg;
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
  const int64_t row0 = rows.tile_row + team * 32;                       // the team's first row
  auto row_at = [&](int i) { return min(row0 + i, rows.n_rows - 1); };

  const int first = p.window > 0 ? max(0, rows.t_lo - p.window + 1) : 0;
  const int n_tiles = (rows.t_hi - first) / C::BN + 1;
  const char* const kb = reinterpret_cast<const char*>(p.k + begin * p.k_stride + (int64_t)kv * C::D);
  const char* const vb = reinterpret_cast<const char*>(p.v + begin * p.v_stride + (int64_t)kv * C::D);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  // A load is a row; rows past the sequence's last token repeat it.
  auto issue_k = [&](int tile) {
#pragma unroll
    for (int u = 0; u < C::BN / C::NW; ++u) {
      const int r = u * C::NW + wave;
      dma16(kb + (int64_t)min(first + tile * C::BN + r, len - 1) * (p.k_stride * 2), k_piece(r, lane) * 16, lds0 + r * C::ROWB);
    }
  };
  auto issue_v = [&](int tile) {
#pragma unroll
    for (int u = 0; u < C::BN / C::NW; ++u) {
      const int r = u * C::NW + wave;
      dma16(vb + (int64_t)min(first + tile * C::BN + r, len - 1) * (p.v_stride * 2), v_piece(r, lane) * 16, lds0 + C::TILE + r * C::ROWB);
    }
  };
  issue_k(0);

  vec8 q[2][16];                                     // rows c16 and c16 + 16
  int token[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int64_t row = row_at(16 * g + c16);
    token[g] = (int)(row / p.gqa);
    const int head = kv * p.gqa + (int)(row - (int64_t)token[g] * p.gqa);
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

  uint32_t k_at[4], v_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = (16 * part + c16) * C::ROWB + k_piece(c16, 4 * i + quarter) * 16;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int r = 8 * hi + (lane & 15) / 4;
    v_at[d] = C::TILE + r * C::ROWB + v_piece(r, d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2) * 16 + (lane & 1) * 8 + part * 256;
  }
  // weights of a row: eight pieces of eight keys, which differ in the banks from row to row
  char* const p_lds = smem + C::P_AT + team * C::P_TEAM;
  auto p_at = [&](int row, int piece) { return row * 128 + (piece ^ (row & 7)) * 16; };
  uint32_t p_wr[2], p_rd[4];
#pragma unroll
  for (int g = 0; g < 2; ++g) p_wr[g] = p_at(16 * g + c16, 2 * part + (quarter >> 1)) + (quarter & 1) * 8;
#pragma unroll
  for (int s = 0; s < 4; ++s) p_rd[s] = p_at(c32, 2 * s + hi);
  float* const maxima = reinterpret_cast<float*>(smem + C::M_AT) + team * 128;   // [part][row]
  volatile int* const flags = reinterpret_cast<volatile int*>(smem + C::FLAG_AT);
  if (threadIdx.x < 2) flags[threadIdx.x] = 0;

  for (int tile = 0; tile < n_tiles; ++tile) {
    wait_loads();
    block_barrier();                                 // K is here; everybody has done with V
    issue_v(tile);
    if (threadIdx.x == 0) flags[(tile + 1) & 1] = 0;
    const int k0 = first + tile * C::BN;
    float4v s[2] = {float4v{}, float4v{}};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const vec8 a = *reinterpret_cast<const vec8*>(smem + k_at[i & 3] + (i >> 2) * 256);
      s[0] = mfma16<BF16>(a, q[0][i], s[0]);
      s[1] = mfma16<BF16>(a, q[1][i], s[1]);
    }
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
        *reinterpret_cast<uint2v*>(p_lds + p_wr[g]) = w;
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
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        top[g] = blocks_max(top[g]);
        if (quarter == 0) maxima[part * 32 + 16 * g + c16] = top[g];
      }
      block_barrier();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float m_new = m[g];
#pragma unroll
        for (int w = 0; w < 4; ++w) m_new = fmaxf(m_new, maxima[w * 32 + 16 * g + c16]);
        l[g] *= m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[g] - m_new);
        m[g] = m_new;
      }
      float m_new = m_out;
#pragma unroll
      for (int w = 0; w < 4; ++w) m_new = fmaxf(m_new, maxima[w * 32 + c32]);
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m_out - m_new);
      m_out = m_new;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= alpha;
      weigh();
      block_barrier();
    }
    if (tile + 1 < n_tiles) issue_k(tile + 1);
#pragma unroll
    for (int g = 0; g < 2; ++g) {                    // (a wave's own weights, as they lie in LDS)
      const uint2v w = *reinterpret_cast<const uint2v*>(p_lds + p_wr[g]);
      l[g] = add2<BF16>(w[1], add2<BF16>(w[0], l[g]));
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const vec8 pb = *reinterpret_cast<const vec8*>(p_lds + p_rd[n]);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        typedef __attribute__((address_space(3))) short4v* lds_ptr;
        const char* const at = smem + v_at[d] + n * 16 * C::ROWB;
        const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at));
        const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * C::ROWB)));
        o[d] = T::mfma(__builtin_bit_cast(vec8, uint4v{x[0], x[1], y[0], y[1]}), pb, o[d]);
      }
    }
  }
  block_barrier();
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float sum = blocks_sum(l[g]);
    if (quarter == 0) maxima[part * 32 + 16 * g + c16] = sum;
  }
  block_barrier();
  if (row0 + c32 < rows.n_rows) {
    const float inv = 1.0f / (maxima[c32] + maxima[32 + c32] + maxima[64 + c32] + maxima[96 + c32]);
    const int64_t row = row0 + c32;
    const int tok = (int)(row / p.gqa), head = kv * p.gqa + (int)(row - (int64_t)tok * p.gqa);
    uint16_t* const dst = p.out + ((int64_t)(begin + tok) * p.n_q_heads + head) * C::D + part * 128;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2v x = {pack2<BF16>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack2<BF16>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
        *reinterpret_cast<uint2v*>(dst + d * 32 + 8 * i + 4 * hi) = x;
      }
  }
}

int block_rows(int head_dim) {
  return head_dim == 128 ? PrefillCfg<128>::ROWS : head_dim == 256 ? PrefillCfg<256>::ROWS : TeamCfg::ROWS;
}

// Launch with so much LDS (over 64 KB: the function has to be told, once per device).
template <int ID>
hipError_t launch_kernel(void (*kernel)(PrefillParams), const PrefillParams& p, int threads, int lds, hipStream_t s) {
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
  hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)p.slots * p.n_kv_heads)), dim3(threads), lds, s, p);
  return hipGetLastError();
}
template <int D, bool BF16>
hipError_t launch(const PrefillParams& p, hipStream_t s) {
  if constexpr (D == 512) return launch_kernel<D + BF16>(prefill_team_kernel<BF16>, p, TeamCfg::NW * 64, TeamCfg::SMEM, s);
  else return launch_kernel<D + BF16>(prefill_mfma_kernel<D, BF16>, p, PrefillCfg<D>::NW * 64, PrefillCfg<D>::SMEM, s);
}

}  // namespace

int64_t prefill_blocks(const tq_packed_qkv& x, int n_seqs) {
  const int64_t slots = (int64_t)x.n_tokens * (x.n_q_heads / x.n_kv_heads) / block_rows(x.head_dim) + n_seqs;
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
  const bool bf16 = x.dtype == TQ_DTYPE_BF16;
  switch (x.head_dim) {
    case 128: return bf16 ? launch<128, true>(p, s) : launch<128, false>(p, s);
    case 256: return bf16 ? launch<256, true>(p, s) : launch<256, false>(p, s);
    case 512: return bf16 ? launch<512, true>(p, s) : launch<512, false>(p, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace tq
