// One 32-token cache block against tiles of query rows on the matrix cores: the pieces that the workgroup-level attention kernels are
// made of (verify_attn_wide over a sequence's own cache, the kernels over paged caches).  bf16 and INT8 caches.
//
// Matrix-core mapping (32 x 32, c = lane % 32, h = lane / 32):
//   S^T[32 tokens x 32 rows] = K Q^T: row c of operand A is token wide_token(c) of the block (bits 3 and 4 of c exchanged), step ks
//     takes head elements 8 (2 ks + h) .. + 7 (INT8: 16 (2 ks + h) .. + 15); a lane then holds, for query row c, the tokens
//     16 ((i >> 2) & 1) + 8 (i >> 3) + 4 h + (i & 3), i = 0 .. 15,
//   which is, eight by eight, the token order of the cache's V chunks, so that the probabilities are operand B of
//   O^T[32 head elements x 32 rows] += V^T P^T as they are.
#pragma once
#include <type_traits>

#include "bass_common.h"

namespace bass {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(16))) int i32x16;

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// 128-bit variants through raw buffer accesses with the device-scope cache policy (sc1); the
// buffer descriptor also bounds the access: offsets beyond `bytes` read zero / are dropped.
constexpr int kAuxDeviceScope = 16;  // sc1

// base and bytes are wave-uniform by construction; saying so keeps the descriptor in scalar
// registers (otherwise every access is wrapped in a loop over distinct descriptors).
__device__ inline __amdgpu_buffer_rsrc_t dev_buffer(const float* base, unsigned bytes) {
  const unsigned long long a = (unsigned long long)base;
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a);
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
  float* ub = (float*)(((unsigned long long)hi << 32) | lo);
  return __builtin_amdgcn_make_buffer_rsrc(ub, 0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

__device__ inline void store_dev4(__amdgpu_buffer_rsrc_t rs, unsigned byte_off, f32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs, (int)byte_off, 0, kAuxDeviceScope);
}

__device__ inline f32x4 load_dev4(__amdgpu_buffer_rsrc_t rs, unsigned byte_off) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)byte_off, 0, kAuxDeviceScope));
}

constexpr int kAuxNonTemporal = 2;  // nt
constexpr float kMaxSlack = 8.f;  // log2 units: how far a row's scores may exceed its reference maximum before that is moved

// Reductions over the four lanes l, l + 16, l + 32, l + 48 (the lanes that share a query row in the
// matrix-core result layout) with gfx950's lane-swap instructions: v_permlane32_swap of a value with
// itself leaves (low half, low half) and (high half, high half), v_permlane16_swap (rows 0 and 2 twice)
// and (rows 1 and 3 twice) -- two VALU operations per step instead of two trips through the LDS crossbar.
__device__ inline float rows4_max(float v) {
  const u32x2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u32x2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ inline float rows4_sum(float v) {
  const u32x2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const u32x2 b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// eight INT8 codes (two words) -> eight bf16 (exact: |code| <= 127)
__device__ inline uint4 codes_to_bf16(uint32_t lo, uint32_t hi) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = (__bf16)(float)(int)(int8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
  return __builtin_bit_cast(uint4, o);
}

// NT tiles of 32 query rows, or (NT = 0) one of 16.  A lane belongs to row lane % kRows of a tile; h = lane / kRows.
template <int D, bool kI8, int NT>
struct Wide {
  static constexpr bool kSmall = NT == 0;
  static constexpr int kTiles = kSmall ? 1 : NT, kRows = kSmall ? 16 : 32, kLanes = 64 / kRows;  // lanes of a row
  static constexpr int kAllRows = kRows * kTiles;
  static constexpr int kBlkVec = kI8 ? 2 * D + 8 : 4 * D;   // uint4 per block and tensor
  static constexpr int kChunks = D / (kI8 ? 32 : 16);       // 16-byte chunks per lane, block and tensor
  static constexpr int kQuerySteps = D / (kLanes * (kI8 ? 16 : 8));  // operands of a score tile's queries
  static constexpr int kScores = kSmall ? 8 : 16;           // scores of a lane per block and tile
  static constexpr int kProbs = kScores / 8;                // operands of the V product
  static constexpr int kAcc = D / kRows;                    // accumulators per tile ...
  static constexpr int kQuads = kSmall ? 1 : 4;             // ... of this many quads of head elements each
  typedef typename std::conditional<kSmall, f32x4, f32x16>::type Acc;

  // Token of the block that a lane's score i belongs to; eight by eight these are the tokens of the cache's V chunks.
  __device__ static int token(int i, int h) {
    return kSmall ? 16 * (i >> 2) + 4 * h + (i & 3) : 16 * ((i >> 2) & 1) + 8 * (i >> 3) + 4 * h + (i & 3);
  }
  // Chunk x of K: this lane's token and which 16 bytes of its row.  (32 rows: bits 3 and 4 of the row exchanged.)
  __device__ static int k_token(int x, int c) {
    return kSmall ? 16 * (x / (kChunks / 2)) + c : (c & 7) | ((c & 8) << 1) | ((c & 16) >> 1);
  }
  __device__ static int k_part(int x, int h) { return kSmall ? 4 * (x % (kChunks / 2)) + h : 2 * x + h; }
  // First head element of a lane's fragment f of V chunk x (INT8 chunks hold two fragments)
  __device__ static int v_elem(int x, int f, int c) {
    return kSmall ? (kI8 ? 32 * x + 16 * f + c : 16 * x + c) : kI8 ? 64 * (x >> 1) + 32 * (c >> 4) + 16 * f + (c & 15) : 32 * (x >> 1) + c;
  }
  // First of the four head elements of quad q of accumulator a
  __device__ static int elem(int a, int q, int h) {
    return kSmall ? 16 * a + 4 * h : kI8 ? 64 * (a >> 1) + 32 * (q >> 1) + 16 * (a & 1) + 8 * (q & 1) + 4 * h : 32 * a + 8 * q + 4 * h;
  }
  // Where a lane's chunks lie in a block (uint4): a lane offset and a step per chunk.
  __device__ static int k_lane(int lane) {
    const int c = lane & 31, t = k_token(0, c);
    return kSmall ? lane : (t >> 4) * (32 * kChunks) + (lane >> 5) * 16 + (t & 15);
  }
  __device__ static int v_lane(int lane) { return kSmall ? lane : ((lane >> 4) & 1) * 64 + (lane >> 5) * 16 + (lane & 15); }
  __device__ static constexpr int k_step(int x) { return kSmall ? 64 * x : (x >> 1) * 64 + (x & 1) * 32; }
  __device__ static constexpr int v_step(int x) { return kSmall ? 64 * x : (x >> 1) * 128 + (x & 1) * 32; }

  __device__ static float row_max(float v) {  // over the lanes of a row
    if constexpr (kSmall) return rows4_max(v);
    const u32x2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  }
  __device__ static float row_sum(float v) {
    if constexpr (kSmall) return rows4_sum(v);
    const u32x2 a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
};

// A block on its way to its wavefront, and (INT8) one scale: lane l < 32 the K scale of token l, lane l >= 32 the V scale of
// token l - 32.
template <int D, bool kI8>
struct WideBlock {
  static constexpr int kChunks = D / (kI8 ? 32 : 16);
  u32x4 k[kChunks], v[kChunks];
  float scale;
};

template <int D, bool kI8, int NT>
struct WideQueries {
  using G = Wide<D, kI8, NT>;
  u32x4 q[G::kTiles][G::kQuerySteps];  // operand B of the score tiles
  float row_scale[G::kTiles];          // INT8: row scale * |softmax scale| * log2(e)
  int lim[G::kTiles];                  // last token visible to the row
};

template <int D, bool kI8, int NT>
struct WideState {
  using G = Wide<D, kI8, NT>;
  typename G::Acc acc[G::kTiles][G::kAcc];
  float m[G::kTiles], l[G::kTiles];  // running maximum (log2 units; the same in all lanes of a row), this lane's share of the sum
};

// Scores of a block in log2 units.  INT8: integer products times the product of the token's and the row's scale, which is in range
// where the scales and the integers one after the other need not be.
template <int D, bool kI8, int NT>
__device__ inline void wide_scores(const WideBlock<D, kI8>& r, const WideQueries<D, kI8, NT>& q, float abs_scale_log2, int h, const float* scales,
                                   float (&s)[Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kScores]) {
  using G = Wide<D, kI8, NT>;
  constexpr int n = G::kQuerySteps;
#pragma unroll
  for (int nt = 0; nt < G::kTiles; ++nt) {
    if constexpr (G::kSmall) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if constexpr (kI8) {
          i32x4 z = {0, 0, 0, 0};
#pragma unroll
          for (int x = 0; x < n; ++x)
            z = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, r.k[t * n + x]), __builtin_bit_cast(i32x4, q.q[nt][x]), z, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][4 * t + i] = (float)z[i];
        } else {
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int x = 0; x < n; ++x)
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.k[t * n + x]), __builtin_bit_cast(bf16x8, q.q[nt][x]), z, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[nt][4 * t + i] = z[i];
        }
      }
    } else if constexpr (kI8) {
      i32x16 z = {0};
#pragma unroll
      for (int x = 0; x < n; ++x)
        z = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, r.k[x]), __builtin_bit_cast(i32x4, q.q[nt][x]), z, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[nt][i] = (float)z[i];
    } else {
      f32x16 z = {0.f};
#pragma unroll
      for (int x = 0; x < n; ++x)
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, r.k[x]), __builtin_bit_cast(bf16x8, q.q[nt][x]), z, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[nt][i] = z[i];
    }
    // A rounded product, as the maximum is: fused with the subtraction of the maximum, the largest probability would not be 1 but 2 to
    // the power of what the rounding took from the maximum, which costs precision from 2^10 on and is not finite from 2^31 on.
#pragma unroll
    for (int y = 0; y < G::kScores / 4; ++y) {
#pragma clang fp contract(off)
      f32x4 scale = {abs_scale_log2, abs_scale_log2, abs_scale_log2, abs_scale_log2};
      if constexpr (kI8) scale = *(const f32x4*)&scales[G::token(4 * y, h)] * q.row_scale[nt];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nt][4 * y + e] *= scale[e];
    }
  }
}

// A block that reaches beyond ctx_len: causal limits; and stale cache rows may hold anything, NaN included: they are zero in V
// (bf16), so that 0 * garbage cannot reach the accumulator.  In place and apart from the step itself: two instances of the step,
// with and without masks, would make the compiler merge their register tuples and spill hundreds of them.
template <int D, bool kI8, int NT>
__device__ inline void mask_wide(WideBlock<D, kI8>& r, float (&s)[Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kScores],
                                 const WideQueries<D, kI8, NT>& q, int tok0, int n_valid, int h) {
  using G = Wide<D, kI8, NT>;
#pragma unroll
  for (int nt = 0; nt < G::kTiles; ++nt)
#pragma unroll
    for (int i = 0; i < G::kScores; ++i)
      if (tok0 + G::token(i, h) > q.lim[nt]) s[nt][i] = -INFINITY;
  if constexpr (!kI8) {
#pragma unroll
    for (int y = 0; y < G::kProbs; ++y)
#pragma unroll
      for (int wd = 0; wd < 4; ++wd) {
        const int t_lo = tok0 + G::token(8 * y + 2 * wd, h);
        const uint32_t keep = (t_lo < n_valid ? 0x0000FFFFu : 0u) | (t_lo + 1 < n_valid ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int x = y; x < G::kChunks; x += G::kProbs) r.v[x][wd] &= keep;
      }
  }
}

// Online softmax of a block: scores -> probabilities as operand B of the V product (INT8: times the tokens' V scales), running
// maximum and sum.  16 rows: with few shares per unit the rounding of the probabilities to bf16 would cost precision (kNarrowUnits); their
// 24 bits are cut into three operands of 8 and all multiplied.  No part is negative, and none is
// zero where the probability is not, so that an infinite element of V stays infinite in every product: the second and third are at
// least 2^-133, the smallest bf16, which the matrix instruction takes as it is (a probability is 0 or at least 2^-126; together they are
// off by at most 2^-132, 2^-22 of a probability of 2^-110).  (Two parts leave 2^-17: 3.6e-6 instead of 2.3e-6 with a rounded first part,
// whose remainder may be negative.)
template <int D, bool kI8, int NT>
__device__ inline void wide_softmax(const float (&s)[Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kScores], WideState<D, kI8, NT>& st, int h, const float* scales,
                                    bf16x8 (&pf)[Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kProbs],
                                    bf16x8 (&pr)[2][Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kProbs]) {
  using G = Wide<D, kI8, NT>;
  auto cut = [](float z) { return __uint_as_float(__float_as_uint(z) & 0xFFFF0000u); };
#pragma unroll
  for (int nt = 0; nt < G::kTiles; ++nt) {
    float mx = s[nt][0];
#pragma unroll
    for (int i = 1; i < G::kScores; ++i) mx = fmaxf(mx, s[nt][i]);
    mx = G::row_max(mx);
    // The reference maximum of a row moves only when a block exceeds it by more than kMaxSlack (log2 units).
    const float m_old = st.m[nt];
    const bool grow = mx > m_old + kMaxSlack;
    if (__any(grow)) {
      const float m_new = grow ? mx : m_old;
      const float alpha = __builtin_amdgcn_exp2f(m_old - (m_new == -INFINITY ? 0.f : m_new));
      st.l[nt] *= alpha;
#pragma unroll
      for (int a = 0; a < G::kAcc; ++a) st.acc[nt][a] *= alpha;
      st.m[nt] = m_new;
    }
    const float m_use = st.m[nt] == -INFINITY ? 0.f : st.m[nt];  // rows without a visible token yet
    float psum = 0.f;
#pragma unroll
    for (int y = 0; y < G::kScores / 4; ++y) {
      f32x4 vs = {1.f, 1.f, 1.f, 1.f};
      if constexpr (kI8) vs = *(const f32x4*)&scales[32 + G::token(4 * y, h)];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * y + e;
        const float pj = __builtin_amdgcn_exp2f(s[nt][i] - m_use);
        psum += pj;
        const float z = kI8 ? pj * vs[e] : pj;
        if constexpr (G::kSmall) {
          const float a = cut(z), b = cut(z - a), least = fminf(z, 0x1p-133f);
          pf[nt][i >> 3][i & 7] = (__bf16)a;
          pr[0][nt][i >> 3][i & 7] = (__bf16)fmaxf(b, least);
          pr[1][nt][i >> 3][i & 7] = (__bf16)fmaxf(z - a - b, least);
        } else {
          pf[nt][i >> 3][i & 7] = (__bf16)z;
        }
      }
    }
    st.l[nt] += psum;
  }
}

template <int D, bool kI8, int NT>
__device__ inline void wide_values(const WideBlock<D, kI8>& r, const bf16x8 (&pf)[Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kProbs],
                                   const bf16x8 (&pr)[2][Wide<D, kI8, NT>::kTiles][Wide<D, kI8, NT>::kProbs], WideState<D, kI8, NT>& st) {
  using G = Wide<D, kI8, NT>;
  constexpr int kFrags = kI8 ? 2 : 1;  // V fragments of a chunk
#pragma unroll
  for (int x = 0; x < G::kChunks; ++x)
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      bf16x8 v;
      if constexpr (kI8) v = __builtin_bit_cast(bf16x8, codes_to_bf16(r.v[x][2 * f], r.v[x][2 * f + 1]));
      else v = __builtin_bit_cast(bf16x8, r.v[x]);
#pragma unroll
      for (int nt = 0; nt < G::kTiles; ++nt) {
        typename G::Acc& acc = st.acc[nt][kFrags * (x / G::kProbs) + f];
        if constexpr (G::kSmall) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pr[1][nt][0], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pr[0][nt][0], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[nt][0], acc, 0, 0, 0);
        } else {
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[nt][x & 1], acc, 0, 0, 0);
        }
      }
    }
}

}  // namespace bass
