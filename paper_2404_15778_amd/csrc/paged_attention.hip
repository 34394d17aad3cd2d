// Attention over paged caches with shared prefixes: bass_paged_verify_attention.
//
// A run's query tokens (paged_plan.h) see its blocks through one table.  Over a run of P, for a query row q:
//   m = max_j s_j,  l = sum_j 2^(s_j - m),  a = sum_j 2^(s_j - m) v_j,   s_j = q k_j * scale * log2(e)   (one pass, 32 bits)
// and a row's result over the runs and workgroups that have a part of its tokens: M = max m, O = sum 2^(m - M) a / sum 2^(m - M) l.
// A prefix's blocks are so read once for the query rows of all sequences that begin with it.
//
// paged_attn: a workgroup of four wavefronts per share of the list.  Up to 64 query rows: the wavefronts take a unit's blocks in turn, each with the
// state of all of the unit's rows, NT tiles of 32 (wide_tiles.h), and merge their states through LDS at the end of the unit; in short runs each has a kv
// head of its own.  More rows: every wavefront has rows of its own, and they go through the blocks together.
// paged_merge: joins the partial results and writes O, lse and the zeros of unused rows.
//
// Precision: 32 bits but for the operands of the V product and O.  Probabilities are bf16 there, one matrix instruction for each (a second and third part, as
// the kernels for few rows of caches per sequence multiply them, would be two and three: in tiles these instructions are half of the work), and over INT8 pools
// they are rounded behind the product with the token's scale.  Error of O against 64 bits 1.8e-3 - 2.4e-3, 1.65e-3 with 32 bits everywhere and O in bf16.
//
// us per layer, attention + merge.  Few rows: bound by the trips to memory of a launch, one behind the other (8 answers of up to 7 tokens to a prompt of 1500, 32 heads:
// 14 + 4 for 37 MB), and in long contexts by memory (16 sequences of up to 8192 tokens: 21 + 4 for 88 MB, 4.2 TB/s).  Tiles: 3 prefixes of up to 8000 tokens, 32
// sequences of 5 tokens, 64/8 heads: 42 + 7 (16 GFLOP; every workgroup has but a few blocks between the 6 us that a tile's beginning takes and the
// 3 of its end); a prefix of 16 384, 64 sequences of 8, 32/8 heads: 160 - 180 + 11 (137 GFLOP, 0.8 PFLOP/s): issue of matrix and softmax instructions from one
// wavefront per SIMD, at the clock that the card's power leaves.  INT8, a prefix of 4096, 24 sequences of one token, 64/8 heads: 26 + 6, the same bounds.  Tiles of up to 128
// rows: 16 sequences of 6 behind 32 768 tokens, 32 heads: 114 + 7 (555 MB, 4.9 TB/s).
// The same with heads of 64: answers 10 + 4, ragged 13 + 4, prompts 29 + 6, document 120 + 7, INT8 prompt 19 + 5; over INT8 pools, heads of 128: answers 15 + 4, ragged 19 + 4
// (half the bytes: the trips are the same, and a block's conversions), prompts 45 + 8, document 190 + 10.
#include "paged_plan.h"
#include "wide_tiles.h"

namespace bass {

struct PagedParams {
  int B, kmax, Hq, Hkv, g, blocks_per_page, n_pages, max_pages;
  unsigned g_magic;  // ceil(2^20 / g): r / g == (r * g_magic) >> 20 for r < 2048, g <= 64
  float scale_log2;
  int32_t signature;
  const uint16_t* Q;
  const uint4 *Kp, *Vp;
  const int32_t* tables;
  const PagedHeader* header;
  const PagedShare* shares;
  const PagedRun* runs;
  const PagedSeq* seqs;
  const int32_t* tokens;
  uint16_t* O;
  float* lse;
  float* part_acc;  // [partial row][D]
  float* part_ml;   // [partial row][2]: running maximum (log2 units), sum
  int32_t* status;
};

// What a workgroup has of one unit.
struct PagedSegment {
  PagedRun run;
  int kvh, tile;       // (first) kv head
  int first, n;        // blocks
  int tok, n_tok;      // query tokens: entries of the token list or, in a run of one sequence, tokens
  bool solo;           // its result is the final one
};

__device__ inline PagedRun uniform_run(const PagedRun* at) {
  const i32x4 a = ((const i32x4*)at)[0], b = ((const i32x4*)at)[1], c = ((const i32x4*)at)[2];
  const i32x4 d = ((const i32x4*)at)[3];
  return PagedRun{uniform(a[0]), uniform(a[1]), uniform(a[2]), uniform(a[3]), uniform(b[0]), uniform(b[1]), uniform(b[2]), uniform(b[3]),
                  uniform(c[0]), uniform(c[1]), uniform(c[2]), uniform(c[3]),
                  uniform(d[0]), uniform(d[1]), {0, 0}};
}

__device__ inline PagedSegment paged_segment(const PagedRun& r, int unit, int off, int entries) {
  PagedSegment s;
  s.run = r;
  const int at = unit / r.n_tiles;
  s.kvh = at * r.heads;
  s.tile = unit - at * r.n_tiles;
  const int from = r.block_at(off);
  s.first = r.first + from;
  s.n = (entries < r.n_blk * r.cost - off ? r.block_at(off + entries) : r.n_blk) - from;
  s.tok = r.tok + s.tile * r.tile_tok;
  s.n_tok = min(r.tile_tok, r.n_tok - s.tile * r.tile_tok);
  s.solo = r.whole && s.n == r.n_blk;
  return s;
}

__device__ inline int row_of(const PagedParams& p, int r) { return (int)(((unsigned)r * p.g_magic) >> 20); }  // query token of a tile's row

// Query tokens of a lane's rows (any for a row that does not exist), as rows of [B * kmax].  Requested in front of everything else: in a shared run the
// queries wait for them.
template <int NT>
struct QueryTokens {
  int tok[NT];
};
template <int NT>
__device__ inline QueryTokens<NT> query_tokens(const PagedParams& p, const PagedSegment& s, int row0) {
  QueryTokens<NT> q;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int t = row_of(p, row0 + 32 * nt), at = s.tok + (t < s.n_tok ? t : 0);
    q.tok[nt] = s.run.L < 0 ? p.tokens[at] : at;
  }
  return q;
}

// Operand B of the score tiles.  A lane's row is c of each tile, and its two lanes (h) have the row's 16-byte chunks in turn.  A negative softmax
// scale is moved into the queries (exact), and so is a zero; the factor that is left is positive.  INT8: quantized per row, with 127 (1 / amax), as the header
// says, for the 127 / amax of cached rows and of the kernels for caches per sequence: no quicker, but what this operator's results have been since it was
// there.  The codes are the same but where x 127 / amax is a half to within its roundings: one element in 4.5 % of rows of 128, in 2.3 % of rows of 64.
template <int D, bool kI8, int NT>
__device__ inline void load_paged_queries(const PagedParams& p, const PagedSegment& s, const QueryTokens<NT>& tokens, int kvh, int c, int h,
                                          WideQueries<D, kI8, NT>& q) {
  using G = Wide<D, kI8, NT>;
  const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = 32 * nt + c, t = row_of(p, row);
    const bool live = t < s.n_tok && p.scale_log2 != 0.f;
    const int hg = row - t * p.g;
    const u32x4* src = (const u32x4*)(p.Q + ((size_t)tokens.tok[nt] * p.Hq + kvh * p.g + hg) * D);
    q.lim[nt] = s.run.L < 0 ? 0x7fffffff : s.run.L + (t < s.n_tok ? t : 0);
    const uint32_t keep = live ? 0xFFFFFFFFu : 0u;
    if constexpr (kI8) {
      u32x4 raw[2 * G::kQuerySteps];
      float amax = 0.f;
#pragma unroll
      for (int x = 0; x < 2 * G::kQuerySteps; ++x) {
        raw[x] = (src[2 * (2 * (x >> 1) + h) + (x & 1)] ^ flip) & keep;
        amax = fmaxf(amax, amax8(__builtin_bit_cast(uint4, raw[x])));
      }
      amax = G::row_max(amax);
      const float scale = amax / 127.0f * fabsf(p.scale_log2);
      const float inv = amax > 0.f && scale != 0.f ? 1.0f / amax * 127.0f : 0.f;  // a division and a product, each rounded
      q.row_scale[nt] = scale != 0.f ? scale : 1.f;
#pragma unroll
      for (int x = 0; x < G::kQuerySteps; ++x) {
        const uint2 lo = quantize8(__builtin_bit_cast(uint4, raw[2 * x]), inv), hi = quantize8(__builtin_bit_cast(uint4, raw[2 * x + 1]), inv);
        q.q[nt][x] = u32x4{lo.x, lo.y, hi.x, hi.y};
      }
    } else {
#pragma unroll
      for (int x = 0; x < G::kQuerySteps; ++x) q.q[nt][x] = (src[2 * x + h] ^ flip) & keep;
    }
  }
}

__device__ inline uint2 to_bf16(f32x4 v) {  // round to nearest even
  typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
  return __builtin_bit_cast(uint2, __builtin_convertvector(v, bf16x4));
}

// Page numbers of the blocks that a wavefront takes, 64 at a time: lane l holds the block (counted over the pool's pages) of turn base + l.
struct PageWindow {
  int base;
  int now, next;
};

template <int D, bool kI8, int NT>
struct PagedExchange {
  using G = Wide<D, kI8, NT>;
  f32x4 acc[NT * G::kAcc][kPagedWaves - 1][4][64];
  float m[kPagedWaves][NT][32], l[kPagedWaves][NT][32];
  __align__(16) float scales[kPagedWaves][kI8 ? 64 : 4];
};

// kHeads: a wavefront has a kv head of its own and all of the blocks (run.heads).
template <int D, bool kI8, int NT, bool kHeads>
__device__ inline void paged_unit(const PagedParams& p, const PagedSegment& s, int wg, PagedExchange<D, kI8, NT>& lds) {
  using G = Wide<D, kI8, NT>;
  using Block = WideBlock<D, kI8>;
  constexpr int W = kPagedWaves, kAccs = NT * G::kAcc, kBlkVec = G::kBlkVec;
  constexpr int R = 2;  // blocks a wavefront has in its registers or on the way there
  constexpr int kStride = kHeads ? 1 : W;
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
  const int kvh = s.kvh + (kHeads ? wv : 0), first_mine = kHeads ? 0 : wv;
  if (kHeads && kvh >= p.Hkv) return;
  const int n_mine = (s.n - first_mine + kStride - 1) / kStride;  // turns of this wavefront: block s.first + first_mine + kStride t
  const int32_t* table = p.tables + (size_t)s.run.row * p.max_pages;
  int bad = 0;
  auto pool_blocks = [&](int t0) {  // of turns t0 + lane
    const int t = min(t0 + lane, max(n_mine - 1, 0)), blk = s.first + min(first_mine + kStride * t, s.n - 1);
    const int at = blk / p.blocks_per_page;
    int page = table[at];
    if (page < 0 || page >= p.n_pages) {
      page = 0;
      bad = 1;
    }
    return page * p.blocks_per_page + (blk - at * p.blocks_per_page);
  };
  const QueryTokens<NT> tokens = query_tokens<NT>(p, s, c);
  PageWindow win{0, pool_blocks(0), 0};
  const int k_lane = 16 * G::k_lane(lane), v_lane = 16 * G::v_lane(lane);
  // One past the end goes through a buffer descriptor of size zero and touches nothing: all fetches are unconditional (exact wait counts).
  auto block_at = [&](int t) {
    const int blk = t - win.base < 64 ? __builtin_amdgcn_readlane(win.now, (t - win.base) & 63) : __builtin_amdgcn_readlane(win.next, (t - win.base) & 63);
    return pool_block(blk, p.blocks_per_page, p.Hkv, kvh) * kBlkVec;
  };
  auto fetch_k = [&](Block& r, int t) {
    const size_t off = block_at(t);
    const __amdgpu_buffer_rsrc_t at = dev_buffer((const float*)(p.Kp + off), t < n_mine ? 16u * kBlkVec : 0u);
#pragma unroll
    for (int x = 0; x < Block::kChunks; ++x) r.k[x] = __builtin_amdgcn_raw_buffer_load_b128(at, k_lane, 16 * G::k_step(x), kAuxNonTemporal);
    if constexpr (kI8) r.scale = ((const float*)((lane < 32 ? p.Kp : p.Vp) + off + 2 * D))[lane % 32];
  };
  auto fetch_v = [&](Block& r, int t) {
    const __amdgpu_buffer_rsrc_t at = dev_buffer((const float*)(p.Vp + block_at(t)), t < n_mine ? 16u * kBlkVec : 0u);
#pragma unroll
    for (int x = 0; x < Block::kChunks; ++x) r.v[x] = __builtin_amdgcn_raw_buffer_load_b128(at, v_lane, 16 * G::v_step(x), kAuxNonTemporal);
  };
  Block ring[R];
#pragma unroll
  for (int x = 0; x < R; ++x) {
    fetch_k(ring[x], x);
    fetch_v(ring[x], x);
  }
  WideQueries<D, kI8, NT> q;
  load_paged_queries<D, kI8, NT>(p, s, tokens, kvh, c, h, q);
  WideState<D, kI8, NT> st;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    st.m[nt] = -INFINITY;
    st.l[nt] = 0.f;
#pragma unroll
    for (int a = 0; a < G::kAcc; ++a)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.acc[nt][a][i] = 0.f;
  }
  const float abs_scale = p.scale_log2 == 0.f ? 1.f : fabsf(p.scale_log2);
  const int n_valid = s.run.L < 0 ? 0x7fffffff : s.run.L + s.run.n_tok;  // tokens of the sequence
  const int n_plain = s.run.L < 0 ? 0x7fffffff : s.run.L + 1;            // tokens that every row sees
  auto step = [&](Block& r, int t) {
    const int tok0 = (s.first + first_mine + kStride * t) * kBlockTokens;
    float* sc = lds.scales[wv];
    if constexpr (kI8) {
      sc[lane] = (lane >= 32 && tok0 + lane - 32 >= n_valid) ? 0.f : r.scale;  // stale tokens may carry any V scale
      __builtin_amdgcn_wave_barrier();  // a wavefront's LDS accesses stay in order
    }
    float z[NT][G::kScores];
    wide_scores<D, kI8, NT>(r, q, abs_scale, h, sc, z);
    fetch_k(r, t + R);
    if (tok0 + kBlockTokens > n_plain) mask_wide<D, kI8, NT>(r, z, q, tok0, n_valid, h);
    bf16x8 pf[NT][G::kProbs], pr[2][NT][G::kProbs];
    wide_softmax<D, kI8, NT>(z, st, h, sc, pf, pr);
    if constexpr (kI8) __builtin_amdgcn_wave_barrier();
    wide_values<D, kI8, NT>(r, pf, pr, st);
    fetch_v(r, t + R);
  };
  for (int t = 0; t < n_mine; t += R) {
    if (t - win.base == 64) {  // on to the next window
      win.base = t;
      win.now = win.next;
    }
    if (t - win.base == 32 && t + 32 < n_mine) win.next = pool_blocks(t + 32);
#pragma unroll
    for (int x = 0; x < R; ++x) {
      if (x > 0 && t + x >= n_mine) break;
      step(ring[x], t + x);
    }
  }
  if (bad && p.status) atomicOr(p.status, BASS_STATUS_PAGE_CLAMPED);

  const size_t base = partial_row(s.run, p.g, kvh, s.tile, wg);
  // A quad of head elements of row `row` (valid), and with the first one the row's maximum and sum: the result, or a partial one.
  auto deliver = [&](int row, int d, f32x4 v, bool first, float M, float sum, float inv) {
    if (s.solo) {
      const int t = row_of(p, row);
      const size_t orow = (size_t)(s.tok + t) * p.Hq + kvh * p.g + (row - t * p.g);
      *(uint2*)(p.O + orow * D + d) = to_bf16(v * inv);
      if (first && p.lse) p.lse[orow] = (M + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    } else {
      *(f32x4*)(p.part_acc + (base + row) * D + d) = v;
      if (first) *(float2*)(p.part_ml + (base + row) * 2) = make_float2(M, sum);
    }
  };
  auto quad = [&](int x, int y) {
    const typename G::Acc& a = st.acc[x / G::kAcc][x % G::kAcc];
    return f32x4{a[4 * y], a[4 * y + 1], a[4 * y + 2], a[4 * y + 3]};
  };
  if constexpr (kHeads) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float sum = G::row_sum(st.l[nt]), inv = __builtin_amdgcn_rcpf(sum);
      const int row = 32 * nt + c;
      if (row < s.n_tok * p.g) {
#pragma unroll
        for (int a = 0; a < G::kAcc; ++a)
#pragma unroll
          for (int y = 0; y < 4; ++y) deliver(row, G::elem(a, y, h), quad(nt * G::kAcc + a, y), a == 0 && y == 0 && h == 0, st.m[nt], sum, inv);
      }
    }
    return;
  }
  // The four states: M = max m_w, weights 2^(m_w - M) (a wavefront that saw no visible token has m = -inf and weight 0).
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = G::row_sum(st.l[nt]);
    if (h == 0) {
      lds.m[wv][nt][c] = st.m[nt];
      lds.l[wv][nt][c] = l;
    }
  }
  __syncthreads();
  float M[NT], sum[NT], mine[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    M[nt] = -INFINITY;
    sum[nt] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) M[nt] = fmaxf(M[nt], lds.m[w][nt][c]);
    const float Mf = M[nt] == -INFINITY ? 0.f : M[nt];
#pragma unroll
    for (int w = 0; w < W; ++w) sum[nt] += lds.l[w][nt][c] * __builtin_amdgcn_exp2f(lds.m[w][nt][c] - Mf);
    mine[nt] = __builtin_amdgcn_exp2f(st.m[nt] - Mf);
  }
#pragma unroll
  for (int x = 0; x < kAccs; ++x) {
    const int owner = x % W;
    st.acc[x / G::kAcc][x % G::kAcc] *= mine[x / G::kAcc];
    if (wv != owner) {
#pragma unroll
      for (int y = 0; y < 4; ++y) lds.acc[x][wv < owner ? wv : wv - 1][y][lane] = quad(x, y);
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kAccs; ++x) {
    const int nt = x / G::kAcc, a = x % G::kAcc;
    if (wv != x % W) continue;
    const int row = 32 * nt + c;
    const float inv = __builtin_amdgcn_rcpf(sum[nt]);
    f32x4 v[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      v[y] = quad(x, y);
#pragma unroll
      for (int w = 0; w < W - 1; ++w) v[y] += lds.acc[x][w][y][lane];
    }
    if (row < s.n_tok * p.g) {
#pragma unroll
      for (int y = 0; y < 4; ++y) deliver(row, G::elem(a, y, h), v[y], a == 0 && y == 0 && h == 0, M[nt], sum[nt], inv);
    }
  }
}

// ---------------------------------------------------------------------------------------
// Many query rows (a shared prefix): a wavefront has 32 NT rows of its own, 128 NT in all, and all four go through the blocks together.  A block
// is fetched once for the workgroup, into registers two or four blocks ahead, and from there into LDS one block ahead, in the operand order
// that it has in the pool (INT8: V as bf16, so that the codes are widened once and not by every wavefront).  Every wavefront reads the whole block
// from LDS, 16 KB for 16 NT matrix instructions; with NT = 2 that is half of what LDS can deliver in their time.
// Every token of a shared run is visible to every row: there are no masks.
// ---------------------------------------------------------------------------------------
template <int D, bool kI8>
struct TileBlocks {
  u32x4 k[2][kBlockTokens * D * (kI8 ? 1 : 2) / 16];
  u32x4 v[2][kBlockTokens * D * 2 / 16];
  __align__(16) float scales[kI8 ? 4 : 1][64];  // of K, then of V; four blocks
};

template <int D, bool kI8, int NT>
__device__ inline void paged_tile(const PagedParams& p, const PagedSegment& s, int wg, TileBlocks<D, kI8>& lds) {
  using G = Wide<D, kI8, NT>;
  using F = Wide<D, false, NT>;  // V in LDS is bf16
  constexpr int kVec = kBlockTokens * D * (kI8 ? 1 : 2) / 16;  // chunks of codes or elements per block and tensor
  constexpr int kLoads = (kVec + 255) / 256;
  static_assert(kVec == 128 || kVec == 256 || kVec == 512, "heads of 64 and 128");
  constexpr int kPool = G::kBlkVec;
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6), c = lane & 31, h = lane >> 5;
  const int32_t* table = p.tables + (size_t)s.run.row * p.max_pages;
  int bad = 0;
  // Block t0 + lane as the pool counts them (past the end: the last one), in two steps: its page's number is on its way meanwhile.
  auto block_of_lane = [&](int t0) { return s.first + min(t0 + lane, s.n - 1); };
  auto request = [&](int t0) { return table[block_of_lane(t0) / p.blocks_per_page]; };
  auto arrived = [&](int page, int t0) {
    if (page < 0 || page >= p.n_pages) {
      page = 0;
      bad = 1;
    }
    const int blk = block_of_lane(t0);
    return (page * p.Hkv + s.kvh) * p.blocks_per_page + (blk - blk / p.blocks_per_page * p.blocks_per_page);
  };
  // This wavefront's rows: from row 32 NT wv of the tile on.  Rows that do not exist have zero queries and are not stored.
  const int row0 = 32 * NT * wv, rows = s.n_tok * p.g;
  const QueryTokens<NT> tokens = query_tokens<NT>(p, s, row0 + c);
  // Blocks on their way in registers, of K and of V.  Two cover the way from memory, but for bf16 blocks under 128 rows: a workgroup wants 16 KB in 0.6 us
  // there (a prompt of 32 768 tokens, 16 sequences of 6, 32 heads: 114 instead of 120 us with four; INT8 115 either way).
  constexpr int S = NT == 1 && !kI8 ? 4 : 2, kAhead = 2 + S;  // turn t asks for block t + kAhead of K and for the one before it of V
  const int start_blocks = arrived(request(0), 0);    // lane l: block l
  int now = arrived(request(kAhead), kAhead);         // lane l: the block that turn 64 w + l asks for
  // Whole rounds of 256 chunks (INT8 heads of 64: half of the threads have one).
  constexpr bool kHalf = kVec < 256;
  const int mine = kHalf ? tid & (kVec - 1) : tid;
  struct Stage {
    u32x4 a, b;
    float scale;
  } k0, k1, k2, k3, v0, v1, v2, v3;
  auto start_block = [&](int t) { return __builtin_amdgcn_readlane(start_blocks, t); };
  auto fetch = [&](Stage& r, const uint4* pool, int blk) {
    const u32x4* at = (const u32x4*)(pool + (size_t)blk * kPool) + mine;
    r.a = at[0];
    if constexpr (kLoads == 2) r.b = at[256];
  };
  auto fetch_k = [&](Stage& r, int blk) {
    fetch(r, p.Kp, blk);
    if constexpr (kI8) r.scale = ((const float*)((lane < 32 ? p.Kp : p.Vp) + (size_t)blk * kPool + 2 * D))[lane % 32];
  };
  auto commit_k = [&](const Stage& r, int t) {
    u32x4* to = lds.k[t & 1];
    if (!kHalf || tid < kVec) to[mine] = r.a;
    if constexpr (kLoads == 2) to[256 + mine] = r.b;
    if constexpr (kI8) {
      if (tid < 64) lds.scales[t & 3][tid] = r.scale;
    }
  };
  auto commit_v = [&](const Stage& r, int t) {
    u32x4* to = lds.v[t & 1];
    if constexpr (kI8) {  // chunk (d / 32, lane): head elements d % 32 and 16 + d % 32 of eight tokens
      if (!kHalf || tid < kVec) {
        to[128 * (mine / 64) + mine % 64] = __builtin_bit_cast(u32x4, codes_to_bf16(r.a[0], r.a[1]));
        to[128 * (mine / 64) + 64 + mine % 64] = __builtin_bit_cast(u32x4, codes_to_bf16(r.a[2], r.a[3]));
      }
    } else {
      to[mine] = r.a;
      if constexpr (kLoads == 2) to[256 + mine] = r.b;
    }
  };
  fetch_k(k0, start_block(0));
  fetch_k(k1, start_block(1));
  fetch(v0, p.Vp, start_block(0));
  WideQueries<D, kI8, NT> q;
  load_paged_queries<D, kI8, NT>(p, s, tokens, s.kvh, row0 + c, h, q);
  // The queries stay in accumulation registers, where matrix instructions take an operand from as they are: the others' room is needed.
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int x = 0; x < G::kQuerySteps; ++x) asm volatile("" : "+a"(q.q[nt][x]));
  typedef typename std::conditional<kI8, i32x16, f32x16>::type Scores;
  f32x16 acc[NT][F::kAcc];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    l[nt] = 0.f;
#pragma unroll
    for (int a = 0; a < F::kAcc; ++a)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[nt][a][i] = 0.f;
  }
  // bf16 scores stay as the products give them; the factor to log2 units (positive: load_paged_queries) is applied to their difference from
  // the row's reference maximum, which loses nothing however large they are.  INT8 scores get the scales of row and token, multiplied first.
  const float factor = kI8 ? 1.f : p.scale_log2 == 0.f ? 1.f : fabsf(p.scale_log2);
  const int k_lane = G::k_lane(lane), v_lane = F::v_lane(lane);
  constexpr int kSteps = G::kQuerySteps, kFrags = D / 16;
  u32x4 kf[kSteps], vf[kFrags];  // operands of the block at hand: K of block t + 1, V of block t
  Scores z[NT];
  float e[NT][16];
  bf16x8 pf[NT][2];
  auto read_k = [&](int x, int t) { kf[x] = lds.k[t & 1][k_lane + G::k_step(x)]; };
  auto read_v = [&](int x, int t) { vf[x] = lds.v[t & 1][v_lane + F::v_step(x)]; };
  auto score = [&](int nt, int x) {
    if (x == 0) z[nt] = Scores{};
    if constexpr (kI8) z[nt] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, kf[x]), __builtin_bit_cast(i32x4, q.q[nt][x]), z[nt], 0, 0, 0);
    else z[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[x]), __builtin_bit_cast(bf16x8, q.q[nt][x]), z[nt], 0, 0, 0);
  };
  auto value = [&](int nt, int x) {
    acc[nt][x >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[x]), pf[nt][x & 1], acc[nt][x >> 1], 0, 0, 0);
  };
  // INT8: scales of a lane's 16 tokens, of K of block t + 1 and of V, read ahead of their use as the operands are.
  float ks[kI8 ? 16 : 1], vs[kI8 ? 16 : 1];
  auto read_scales = [&](float* to, int y, int t, int first) {
    if constexpr (kI8) {
      const f32x4 four = *(const f32x4*)&lds.scales[t & 3][first + G::token(4 * y, h)];
#pragma unroll
      for (int i = 0; i < 4; ++i) to[4 * y + i] = four[i];
    }
  };
  // Softmax of a tile of rows, element by element (16 of a lane), so that it can be laid between matrix instructions.
  float mx[NT], sum[NT], m_use[NT], arg[NT][16];
  // Score i as a number.  INT8: times the scales of token and row, multiplied first.
  auto take = [&](int nt, int i) {
    if constexpr (kI8) e[nt][i] = (float)z[nt][i] * (ks[i] * q.row_scale[nt]);
    else e[nt][i] = z[nt][i];
    mx[nt] = i == 0 ? e[nt][0] : fmaxf(mx[nt], e[nt][i]);
  };
  // The row's reference maximum moves when a block exceeds it by more than kMaxSlack.
  auto settle = [&](int nt) {
    mx[nt] = F::row_max(mx[nt]);
    const bool grow = (mx[nt] - m[nt]) * factor > kMaxSlack;  // from -inf: infinite
    if (__any(grow)) {
      const float m_new = grow ? mx[nt] : m[nt];
      const float alpha = grow ? __builtin_amdgcn_exp2f((m[nt] - m_new) * factor) : 1.f;
      l[nt] *= alpha;
#pragma unroll
      for (int a = 0; a < F::kAcc; ++a) acc[nt][a] *= alpha;
      m[nt] = m_new;
    }
    m_use[nt] = m[nt] == -INFINITY ? 0.f : m[nt];  // no score above -inf yet
    sum[nt] = 0.f;
  };
  // Probability i in three steps, one behind the other: argument, exponential, sum and operand.
  auto soft = [&](int nt, int i) {
    if (i < 16) arg[nt][i] = kI8 ? e[nt][i] - m_use[nt] : (e[nt][i] - m_use[nt]) * factor;
    if (i >= 1 && i < 17) e[nt][i - 1] = __builtin_amdgcn_exp2f(arg[nt][i - 1]);
    if (i >= 2 && i < 18) {
      const int j = i - 2;
      sum[nt] += e[nt][j];
      if (j & 1) {
        if constexpr (kI8) {
          pf[nt][j >> 3][(j & 7) - 1] = (__bf16)(e[nt][j - 1] * vs[j - 1]);
          pf[nt][j >> 3][j & 7] = (__bf16)(e[nt][j] * vs[j]);
        } else {
          pf[nt][j >> 3][(j & 7) - 1] = (__bf16)e[nt][j - 1];
          pf[nt][j >> 3][j & 7] = (__bf16)e[nt][j];
        }
      }
    }
  };
  auto finish = [&](int nt, bool counts) {
    l[nt] += counts ? sum[nt] : 0.f;
    asm volatile("" : "+v"(pf[nt][0]), "+v"(pf[nt][1]), "+v"(l[nt]));  // in front of the branch of settle(), not where it is needed
  };
  // Two tiles of rows go through the blocks half a block apart, so that the matrix instructions of one stand beside the softmax of the
  // other: turn t is  [scores of A, block t + 1; values of A, block t | probabilities of B, block t], then
  // [scores of B, block t + 1; values of B, block t | probabilities of A, block t + 1].  Operands are read from LDS eight matrix instructions ahead, V in
  // the first half and K in the second, behind their last use.  The last turn's scores are of the last block again, and their probabilities are not counted.
  // A wavefront has its SIMD for itself: what is to run beside a matrix instruction has to stand right behind it, and the compiler, left to
  // itself, gathers the matrix instructions and lets the rest wait (a prefix of 16 384 tokens, 64 sequences of 8 tokens, 32/8 heads of 128: 189 instead of 169 us).
  constexpr int kHalf16 = kSteps + kFrags;  // matrix instructions of a half turn
  int v_blk = 0;                            // block t + kAhead - 1
  auto half_turn = [&](auto tile_m, auto tile_s, bool counts, auto beside) {
    constexpr int nm = decltype(tile_m)::value, ns = decltype(tile_s)::value;
#pragma unroll
    for (int x = 0; x < kHalf16; ++x) {
      if (x < kSteps) score(nm, x);
      else value(nm, x - kSteps);
#pragma unroll
      for (int i = x * 18 / kHalf16; i < (x + 1) * 18 / kHalf16; ++i) soft(ns, i);
      if (x > kSteps) {
        constexpr int n = kFrags - 1;
        const int y = x - kSteps - 1;
#pragma unroll
        for (int i = y * 16 / n; i < (y + 1) * 16 / n; ++i) take(nm, i);
      }
      beside(x);
      __builtin_amdgcn_sched_barrier(0);
    }
    finish(ns, counts);
    settle(nm);
  };
  auto turn = [&](int t, Stage& k_stage, Stage& v_stage) {
    const int k_blk = __builtin_amdgcn_readlane(now, t & 63);
    if constexpr (NT == 2) {
      half_turn(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{}, true, [&](int x) {
        if (x < kFrags) read_v(x, t);
        if (x < 4) read_scales(ks, x, t + 1, 0);
        if (x == 1) commit_k(k_stage, t + 2);
        if (x == 2) commit_v(v_stage, t + 1);
        if (x == 4) fetch_k(k_stage, k_blk);
        if (x == 5) fetch(v_stage, p.Vp, v_blk);
      });
      __syncthreads();
      half_turn(std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{}, t + 1 < s.n, [&](int x) {
        if (x == 0) {
#pragma unroll
          for (int y = 0; y < 4; ++y) read_scales(vs, y, t + 1, 32);
        }
        if (x < kSteps) read_k(x, t + 2);
      });
    } else {
      // One tile: the scores of block t + 1 beside the probabilities of block t, then the values of block t beside the maximum of block t + 1.
#pragma unroll
      for (int x = 0; x < kSteps; ++x) {
        score(0, x);
#pragma unroll
        for (int i = x * 18 / kSteps; i < (x + 1) * 18 / kSteps; ++i) soft(0, i);
#pragma unroll
        for (int i = x * kFrags / kSteps; i < (x + 1) * kFrags / kSteps; ++i) read_v(i, t);
        if (x == 0) {
#pragma unroll
          for (int y = 0; y < 4; ++y) read_scales(ks, y, t + 1, 0);
          commit_k(k_stage, t + 2);
          fetch_k(k_stage, k_blk);
        }
        if (x == 1) {
          commit_v(v_stage, t + 1);
          fetch(v_stage, p.Vp, v_blk);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      finish(0, true);
      __syncthreads();
#pragma unroll
      for (int x = 0; x < kFrags; ++x) {
        value(0, x);
#pragma unroll
        for (int i = x * 16 / kFrags; i < (x + 1) * 16 / kFrags; ++i) take(0, i);
        if (x == 0) {
#pragma unroll
          for (int y = 0; y < 4; ++y) read_scales(vs, y, t + 1, 32);
        }
        if (x < kSteps) read_k(x, t + 2);
        __builtin_amdgcn_sched_barrier(0);
      }
      settle(0);
    }
    v_blk = k_blk;
  };
  commit_k(k0, 0);
  commit_k(k1, 1);
  commit_v(v0, 0);
  fetch_k(k0, start_block(2));  // in the order of the turns: the wait counts of the loop's entry and of its end are the same
  fetch(v0, p.Vp, start_block(1));
  fetch_k(k1, start_block(3));
  fetch(v1, p.Vp, start_block(2));
  if constexpr (S == 4) {
    fetch_k(k2, start_block(4));
    fetch(v2, p.Vp, start_block(3));
    fetch_k(k3, start_block(5));
    fetch(v3, p.Vp, start_block(4));
  }
  v_blk = start_block(kAhead - 1);
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kSteps; ++x) {
    read_k(x, 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) score(nt, x);
    read_k(x, 1);
  }
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    read_scales(ks, y, 0, 0);
    read_scales(vs, y, 0, 32);
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 16; ++i) take(nt, i);
    settle(nt);
  }
  if constexpr (NT == 2) {
#pragma unroll
    for (int i = 0; i < 18; ++i) soft(0, i);
    finish(0, true);
  }
  __syncthreads();  // before the first turn writes over block 0
  // Windows of 64 turns.  The inner loop has no loads but those of the stages and no way out between its S turns, so that its wait counts are exact.
  int t = 0;
  for (int end = 64;; end += 64) {
    const int page = request(end + kAhead);
    for (const int stop = min(end, s.n) - (S - 1); t < stop; t += S) {
      turn(t, k0, v0);
      turn(t + 1, k1, v1);
      if constexpr (S == 4) {
        turn(t + 2, k2, v2);
        turn(t + 3, k3, v3);
      }
    }
    if (end >= s.n) break;
    now = arrived(page, end + kAhead);
  }
  if (t < s.n) turn(t, k0, v0);
  if constexpr (S == 4) {
    if (t + 1 < s.n) turn(t + 1, k1, v1);
    if (t + 2 < s.n) turn(t + 2, k2, v2);
  }
  if (bad && p.status) atomicOr(p.status, BASS_STATUS_PAGE_CLAMPED);
  const size_t base = partial_row(s.run, p.g, s.kvh, s.tile, wg);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = row0 + 32 * nt + c;
    const float all = F::row_sum(l[nt]);
    if (row < rows) {
      if (h == 0) *(float2*)(p.part_ml + (base + row) * 2) = make_float2(m[nt] * factor, all);
#pragma unroll
      for (int a = 0; a < F::kAcc; ++a)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          *(f32x4*)(p.part_acc + (base + row) * D + F::elem(a, y, h)) = f32x4{acc[nt][a][4 * y], acc[nt][a][4 * y + 1], acc[nt][a][4 * y + 2], acc[nt][a][4 * y + 3]};
    }
  }
}

template <int D, bool kI8>
__global__ __launch_bounds__(64 * kPagedWaves, 1) void paged_attn(PagedParams p) {
  __shared__ union {
    PagedExchange<D, kI8, 1> one;
    PagedExchange<D, kI8, 2> two;
    TileBlocks<D, kI8> tile;
  } lds;
  const PagedShare* rec = p.shares + blockIdx.x;
  if (uniform(rec->signature) != p.signature) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, BASS_STATUS_PLAN_MISMATCH);
    return;
  }
  int entries = uniform(rec->entries), run_no = uniform(rec->run), unit = uniform(rec->unit), off = uniform(rec->off);
  if (entries <= 0) return;
  PagedRun run = uniform_run(&rec->first);
  for (;;) {
    const PagedSegment s = paged_segment(run, unit, off, entries);
    if (s.n > 0) {
      const int rows = s.n_tok * p.g;
      if (is_tile(run.L < 0, run.tile_tok * p.g)) {
        if (run.tile_tok * p.g <= kTileRows / 2) paged_tile<D, kI8, 1>(p, s, blockIdx.x, lds.tile);
        else paged_tile<D, kI8, 2>(p, s, blockIdx.x, lds.tile);
      } else if (rows <= 32) {
        if (run.heads > 1) paged_unit<D, kI8, 1, true>(p, s, blockIdx.x, lds.one);
        else paged_unit<D, kI8, 1, false>(p, s, blockIdx.x, lds.one);
      } else {
        if (run.heads > 1) paged_unit<D, kI8, 2, true>(p, s, blockIdx.x, lds.two);
        else paged_unit<D, kI8, 2, false>(p, s, blockIdx.x, lds.two);
      }
    }
    entries -= run.entries() - off;
    if (entries <= 0) break;
    off = 0;
    if (++unit == (p.Hkv + run.heads - 1) / run.heads * run.n_tiles) {
      unit = 0;
      run = uniform_run(p.runs + ++run_no);
    }
    __syncthreads();  // the exchange is free again, whichever of its two forms is next
  }
}

// ---------------------------------------------------------------------------------------
// Merge.  A workgroup per query token and 1024 / D of its heads, D / 4 threads per output row, four head elements each.  A row's partial results lie
// wherever a workgroup ended inside its unit, of the shared run and of its own; kMergeRound of them are on their way at a time, because each
// round is a trip to memory.  Latency: header and sequence, then the partial results.
// ---------------------------------------------------------------------------------------
constexpr int kMergeRound = 8;

template <int D>
__global__ __launch_bounds__(256) void paged_merge(PagedParams p, int head_groups) {
  constexpr int kLanes = D / 4, kRows = 256 / kLanes;
  static_assert(kRows == kMergeElems / D, "merge_groups counts the workgroups");
  const int tok = blockIdx.x / head_groups, b = tok / p.kmax, i = tok - b * p.kmax;
  const int hq = (int)(blockIdx.x % head_groups) * kRows + threadIdx.x / kLanes, q4 = threadIdx.x % kLanes;
  const PagedHeader* header = p.header;
  const PagedSeq* seq = p.seqs + b;
  const int signature = uniform(header->signature), nq = uniform(seq->nq), pos = uniform(seq->pos);
  const PagedSplit split{uniform(header->per), uniform(header->rem), uniform(header->total)};
  const PagedRun own = uniform_run(&seq->own), shared = uniform_run(&seq->shared);
  if (signature != p.signature || hq >= p.Hq) return;
  const size_t orow = (size_t)tok * p.Hq + hq;
  uint16_t* out = p.O + orow * D + 4 * q4;
  if (i >= nq) {
    *(uint2*)out = make_uint2(0u, 0u);
    if (p.lse && q4 == 0) p.lse[orow] = 0.f;
    return;
  }
  const int kvh = hq / p.g, hg = hq - kvh * p.g;
  // Partial results of a run: n of them from workgroup w0 on, kSlotRows rows apart.
  auto parts = [&](const PagedRun& r, int tile, int row, int& n) {
    const int start = r.start + (kvh / r.heads * r.n_tiles + tile) * r.entries();
    const int w0 = split.owner(start);
    n = split.owner(start + (r.n_blk - 1) * r.cost) - w0 + 1;
    return partial_row(r, p.g, kvh, tile, w0) + row;
  };
  int n_own, n_shared = 0;
  const size_t at_own = parts(own, 0, i * p.g + hg, n_own);
  if (own.whole && n_own == 1) return;  // written by the workgroup that has it all
  size_t at_shared = 0;
  if (shared.n_blk > 0) {
    const int at = pos + i, tile = at / shared.tile_tok;
    at_shared = parts(shared, tile, (at - tile * shared.tile_tok) * p.g + hg, n_shared);
  }
  float M = -INFINITY, L = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int n = n_own + n_shared;
  for (int x0 = 0; x0 < n; x0 += kMergeRound) {
    float2 ml[kMergeRound];
    f32x4 a[kMergeRound];
#pragma unroll
    for (int x = 0; x < kMergeRound; ++x) {  // past the end: the last one again, with weight 0 (rounds of two for two were no quicker)
      const int y = min(x0 + x, n - 1);
      const size_t at = y < n_own ? at_own + (size_t)y * kSlotRows : at_shared + (size_t)(y - n_own) * kSlotRows;
      ml[x] = *(const float2*)(p.part_ml + at * 2);
      a[x] = *(const f32x4*)(p.part_acc + at * D + 4 * q4);
    }
    const float M_old = M;
#pragma unroll
    for (int x = 0; x < kMergeRound; ++x) M = fmaxf(M, ml[x].x);
    const float Mf = M == -INFINITY ? 0.f : M, alpha = __builtin_amdgcn_exp2f(M_old - Mf);
    L *= alpha;
    acc *= alpha;
#pragma unroll
    for (int x = 0; x < kMergeRound; ++x)
      if (x0 + x < n) {
        const float wgt = __builtin_amdgcn_exp2f(ml[x].x - Mf);
        L += ml[x].y * wgt;
        acc += a[x] * wgt;
      }
  }
  const float inv = __builtin_amdgcn_rcpf(L);
  *(uint2*)out = to_bf16(acc * inv);
  if (p.lse && q4 == 0) p.lse[orow] = (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

}  // namespace bass

extern "C" size_t bass_paged_attention_workspace_bytes(const bass_paged_desc* d) {
  if (bass::check_paged_attention(d) != BASS_OK) return 0;
  return bass::partial_rows(d) * (d->D + 2) * sizeof(float);
}

extern "C" int bass_paged_verify_attention(const bass_paged_desc* d, const void* Q, const void* Kpool, const void* Vpool, const int32_t* tables,
                                           const void* plan, void* O, float* lse, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                           void* stream) {
  using namespace bass;
  const int rc = check_paged_attention(d);
  if (rc != BASS_OK) return rc;
  if (!Q || !Kpool || !Vpool || !tables || !plan || !O || !workspace) return BASS_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(Kpool) || !aligned16(Vpool) || !aligned16(plan) || !aligned16(O) || !aligned16(workspace)) return BASS_ERR_INVALID_ARG;
  if (workspace_bytes < bass_paged_attention_workspace_bytes(d)) return BASS_ERR_WORKSPACE_TOO_SMALL;
  const PagedLayout l = paged_layout(d);
  const char* at = (const char*)plan;
  const int g = d->Hq / d->Hkv;
  PagedParams p{d->B, d->kmax, d->Hq, d->Hkv, g, d->page_tokens / kBlockTokens, d->n_pages, d->max_pages, ((1u << 20) + g - 1) / g,
                d->scale * 1.4426950408889634f, paged_signature(d), (const uint16_t*)Q, (const uint4*)Kpool, (const uint4*)Vpool, tables,
                (const PagedHeader*)at, (const PagedShare*)(at + l.shares), (const PagedRun*)(at + l.runs), (const PagedSeq*)(at + l.seqs),
                (const int32_t*)(at + l.tokens), (uint16_t*)O, lse, (float*)workspace, (float*)workspace + partial_rows(d) * d->D, dev_status};
  hipStream_t s = (hipStream_t)stream;
  const bool int8 = d->dtype == BASS_DTYPE_INT8KV;
  const dim3 grid(kPagedShares), block(64 * kPagedWaves);
  const dim3 merge_grid((unsigned)merge_groups(d));
  const int head_groups = (int)(merge_groups(d) / ((int64_t)d->B * d->kmax));
  if (d->D == 128) {
    if (int8) hipLaunchKernelGGL((paged_attn<128, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((paged_attn<128, false>), grid, block, 0, s, p);
    hipLaunchKernelGGL(paged_merge<128>, merge_grid, dim3(256), 0, s, p, head_groups);
  } else {
    if (int8) hipLaunchKernelGGL((paged_attn<64, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((paged_attn<64, false>), grid, block, 0, s, p);
    hipLaunchKernelGGL(paged_merge<64>, merge_grid, dim3(256), 0, s, p, head_groups);
  }
  return launch_status();
}
