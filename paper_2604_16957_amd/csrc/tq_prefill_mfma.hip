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

#include "tq_internal.h"

namespace tq {
namespace {

typedef float float16v __attribute__((ext_vector_type(16)));
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

template <int D>
struct PrefillCfg {
  static constexpr int NW = 4;                       // waves per block
  static constexpr int ROWS = NW * 32;
  static constexpr int BN = D == 512 ? 32 : 64;      // keys per tile
  static constexpr int KS = D / 16;                  // k-steps of the score product
  static constexpr int DT = D / 32;                  // 32-dim tiles of the output
  static constexpr int CH = D / 8;                   // 16-byte pieces of a row
  static constexpr int TILE = BN * D * 2;
  static constexpr int SMEM = 2 * TILE;
};

// Where piece c (16 bytes) of row r lies in an LDS tile.  The score product's operand is read with one row to a lane, the
// same piece of 32 rows at a time: any 8 consecutive rows have to differ in the banks.  The transposing reads take
// 64 bytes of four consecutive rows: there the rows have to differ above those 64 bytes.
__device__ __forceinline__ int k_piece(int r, int c) { return c ^ (r & 15); }
__device__ __forceinline__ int v_piece(int r, int c) { return c ^ ((r & 3) << 2); }

// where the row tiles of sequence b start in the list of all (one per sequence is lost at most, none overlap)
__device__ __forceinline__ int slot_base(const PrefillParams& p, int b, int rows) {
  const int at = min(max(p.cu_seqlens[b], 0), p.n_tokens);
  return (int)((int64_t)at * p.gqa / rows) + b;
}

template <int D, bool BF16>
__global__ __launch_bounds__(PrefillCfg<D>::NW * 64) void prefill_mfma_kernel(PrefillParams p) {
  using C = PrefillCfg<D>;
  using T = Type<BF16>;
  using vec8 = typename T::vec8;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hi = lane >> 5;
  const int kv = blockIdx.x % p.n_kv_heads;
  const int slot = p.slots - 1 - (int)(blockIdx.x / p.n_kv_heads);      // long rows of keys first

  // the last sequence that starts at or before the slot: 64 candidates at a time
  int b = 0;
  for (int n = p.n_seqs; n > 1;) {
    const int step = (n + 63) >> 6, i = lane * step;
    const bool before = i < n && slot_base(p, b + i, C::ROWS) <= slot;
    const int last = 63 - __clzll((long long)(__ballot(before) | 1));
    b += last * step;
    n = min(step, n - last * step);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int begin = min(max(p.cu_seqlens[b], 0), p.n_tokens);
  const int len = min(max(p.cu_seqlens[b + 1], begin), p.n_tokens) - begin;
  const int64_t tile_row = (int64_t)(slot - slot_base(p, b, C::ROWS)) * C::ROWS;
  const int64_t n_rows = (int64_t)len * p.gqa;
  if (tile_row < 0 || tile_row >= n_rows) return;

  // this lane's row
  const int64_t my_row = min(tile_row + wave * 32 + c32, n_rows - 1);
  const bool mine = tile_row + wave * 32 + c32 < n_rows;
  const int token = (int)(my_row / p.gqa), head = kv * p.gqa + (int)(my_row - (int64_t)token * p.gqa);
  const int t_lo = (int)(tile_row / p.gqa), t_hi = (int)(min(tile_row + C::ROWS - 1, n_rows - 1) / p.gqa);   // the block's tokens
  const int w_lo = __builtin_amdgcn_readfirstlane(token);
  const int w_hi = __builtin_amdgcn_readlane(token, 31);                                                      // the wave's

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

  const int first = p.window > 0 ? max(0, t_lo - p.window + 1) : 0;
  const uint16_t* const kb = p.k + begin * p.k_stride + (int64_t)kv * D;
  const uint16_t* const vb = p.v + begin * p.v_stride + (int64_t)kv * D;
  char* const k_lds = smem;
  char* const v_lds = smem + C::TILE;

  for (int k0 = first; k0 <= t_hi; k0 += C::BN) {
    __syncthreads();
    // rows past the sequence's last token repeat it (finite values that weights of zero meet)
    for (int i = threadIdx.x; i < C::BN * C::CH; i += C::NW * 64) {
      const int r = i / C::CH, c = i % C::CH, t = min(k0 + r, len - 1);
      *reinterpret_cast<uint4v*>(k_lds + (r * C::CH + k_piece(r, c)) * 16) = *reinterpret_cast<const uint4v*>(kb + t * p.k_stride + c * 8);
      *reinterpret_cast<uint4v*>(v_lds + (r * C::CH + v_piece(r, c)) * 16) = *reinterpret_cast<const uint4v*>(vb + t * p.v_stride + c * 8);
    }
    __syncthreads();
    if (k0 > w_hi || (p.window > 0 && k0 + C::BN - 1 <= w_lo - p.window)) continue;     // nothing here for this wave
    float16v s[C::BN / 32];
#pragma unroll
    for (int n = 0; n < C::BN / 32; ++n) {
      s[n] = float16v{};
#pragma unroll
      for (int i = 0; i < C::KS; ++i) {
        const int r = n * 32 + c32;
        const vec8 a = *reinterpret_cast<const vec8*>(k_lds + (r * C::CH + k_piece(r, 2 * i + hi)) * 16);
        s[n] = T::mfma(a, q[i], s[n]);
      }
    }
    if (k0 + C::BN - 1 > w_lo || (p.window > 0 && k0 <= w_hi - p.window)) {
      const int oldest = p.window > 0 ? token - p.window + 1 : 0;
#pragma unroll
      for (int n = 0; n < C::BN / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = k0 + n * 32 + 8 * (i / 4) + 4 * hi + i % 4;
          s[n][i] = key > token || key < oldest ? -INFINITY : s[n][i];
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < C::BN / 32; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
    float a, z;
    swap32(top, a, z);
    const float m_new = fmaxf(m, fmaxf(a, z) * p.scale_log2);
    const float ref = m_new == -INFINITY ? 0.0f : m_new;        // (no key of this row yet)
    const float alpha = exp2f(m - ref);
    m = m_new;
    uint32_t w[C::BN / 32][8];
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < C::BN / 32; ++n)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p0 = exp2f(fmaf(s[n][2 * i], p.scale_log2, -ref)), p1 = exp2f(fmaf(s[n][2 * i + 1], p.scale_log2, -ref));
        w[n][i] = pack2<BF16>(p0, p1);
        const auto r = __builtin_bit_cast(typename T::vec2, w[n][i]);
        sum += (float)r[0] + (float)r[1];
      }
    l = l * alpha + sum;
#pragma unroll
    for (int d = 0; d < C::DT; ++d) o[d] *= alpha;
#pragma unroll
    for (int n = 0; n < C::BN / 32; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const vec8 pb = __builtin_bit_cast(vec8, uint4v{w[n][4 * h], w[n][4 * h + 1], w[n][4 * h + 2], w[n][4 * h + 3]});
#pragma unroll
        for (int d = 0; d < C::DT; ++d) {
          // Lane: dim 32 d + lane % 32, keys 4 hi + 0..3 and 8 + 4 hi + 0..3 of these 16.  The transposing read hands lane i of 16
          // the i-th of 16 dims that four lanes' addresses name for each of four keys.
          const int r = n * 32 + h * 16 + 4 * hi + (lane & 15) / 4;
          const int c = d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2;
          typedef __attribute__((address_space(3))) short4v* lds_ptr;
          const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(v_lds + (r * C::CH + v_piece(r, c)) * 16 + (lane & 1) * 8));
          const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(v_lds + ((r + 8) * C::CH + v_piece(r + 8, c)) * 16 + (lane & 1) * 8));
          const uint2v xu = __builtin_bit_cast(uint2v, x), yu = __builtin_bit_cast(uint2v, y);
          o[d] = T::mfma(__builtin_bit_cast(vec8, uint4v{xu[0], xu[1], yu[0], yu[1]}), pb, o[d]);
        }
      }
  }
  float l0, l1;
  swap32(l, l0, l1);
  const float inv = 1.0f / (l0 + l1);                 // (a row has at least its own token)
  if (mine) {
    uint16_t* const dst = p.out + ((int64_t)(begin + token) * p.n_q_heads + head) * D;
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2v x = {pack2<BF16>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack2<BF16>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
        *reinterpret_cast<uint2v*>(dst + d * 32 + 8 * i + 4 * hi) = x;
      }
  }
}

template <int D>
int rows_of_block() { return PrefillCfg<D>::ROWS; }
int block_rows(int head_dim) { return head_dim == 128 ? rows_of_block<128>() : head_dim == 256 ? rows_of_block<256>() : rows_of_block<512>(); }

template <int D, bool BF16>
hipError_t launch(const PrefillParams& p, hipStream_t s) {
  using C = PrefillCfg<D>;
  const auto kernel = prefill_mfma_kernel<D, BF16>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)p.slots * p.n_kv_heads)), dim3(C::NW * 64), C::SMEM, s, p);
  return hipGetLastError();
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
