// Planning of a step's attention over paged caches: bass_paged_attention_plan.
//
// One workgroup, everything but the results in LDS.  Phases: lengths; the prefixes' sequences, query tokens and common blocks; prefix sums over
// the runs (shared ones first); the shared runs' token lists, in the order of the sequences; one record per workgroup of the attention launch.
#include "paged_plan.h"

namespace bass {

// Small batches (sequences and prefixes together) go to a workgroup of 256 threads and keep the runs in LDS too: 16 wavefronts more to start and
// to wait for at every barrier, and a second look at the runs in memory, take 2 - 3 us of 8.
constexpr int kSmallBatch = 256;

struct PagedPlanParams {
  int B, kmax, g, Hkv, most_tokens, n_prefixes;
  bool int8;
  int32_t signature;
  const int32_t *ctx_len, *draft_len, *prefix_of, *prefix_len;
  PagedHeader* header;
  PagedShare* shares;
  PagedRun* runs;
  PagedSeq* seqs;
  int32_t* tokens;
  int32_t* status;
};

// Exclusive prefix sums of four numbers at once over the workgroup, and their totals; all threads call.
struct Four {
  int v[4];
};
template <int T>
__device__ inline Four scan_four(Four x, Four* lds, Four& total) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  Four s = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = __shfl_up(s.v[i], o);
      if (lane >= o) s.v[i] += t;
    }
  __syncthreads();
  if (lane == 63) lds[wv] = s;
  __syncthreads();
  total = Four{{0, 0, 0, 0}};
#pragma unroll
  for (int w = 0; w < T / 64; ++w)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (w < wv) s.v[i] += lds[w].v[i];
      total.v[i] += lds[w].v[i];
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) s.v[i] -= x.v[i];
  return s;
}

// T threads; at most N sequences and N prefixes.
template <int T, int N>
__global__ __launch_bounds__(T) void paged_plan_kernel(PagedPlanParams p) {
  constexpr bool kRunsInLds = N <= kSmallBatch;
  __shared__ Four sums[T / 64];
  __shared__ PagedRun lds_runs[kRunsInLds ? N : 1];
  __shared__ int seq_L[N], seq_n[N], seq_g[N];
  // of each prefix: least ctx_len, then common blocks; query tokens, then their first place in the list; sequences, then its run; first sequence
  __shared__ int pre_L[N], pre_tok[N], pre_row[N], pre_n[N];
  __shared__ int starts[2 * N], live, saved_all;  // live: sequences with query tokens, and tiles of shared runs
  const int tid = threadIdx.x;
  // the first sequence of every thread, requested with the prefixes' lengths: one trip to memory
  const bool has = tid < p.B;
  const int my_L = has ? p.ctx_len[tid] : 0, my_n = has ? p.draft_len[tid] : 0, my_x = has && p.prefix_of ? p.prefix_of[tid] : -1;
  if (tid == 0) live = saved_all = 0;
  for (int x = tid; x < p.n_prefixes; x += T) {
    pre_L[x] = p.prefix_len[x];
    pre_tok[x] = pre_n[x] = 0;
    pre_row[x] = 1 << 30;
  }
  __syncthreads();
  int bad = 0;
  for (int b = tid; b < p.B; b += T) {
    int L = b == tid ? my_L : p.ctx_len[b], n = b == tid ? my_n : p.draft_len[b];
    if (clamp_lengths(L, n, p.kmax, p.most_tokens)) bad = BASS_STATUS_LEN_CLAMPED;
    int x = b == tid ? my_x : p.prefix_of ? p.prefix_of[b] : -1;
    if (x >= p.n_prefixes) bad = BASS_STATUS_LEN_CLAMPED;
    if (x < 0 || x >= p.n_prefixes || n == 0) x = -1;
    seq_L[b] = L;
    seq_n[b] = n;
    seq_g[b] = x;
    if (n > 0) atomicAdd(&live, 1);
    if (x >= 0) {
      atomicMin(&pre_L[x], L);
      atomicAdd(&pre_tok[x], n);
      atomicMin(&pre_row[x], b);
      atomicAdd(&pre_n[x], 1);
    }
  }
  if (bad && p.status) atomicOr(p.status, bad);
  __syncthreads();
  // Common blocks of a prefix's sequences; 0: they go by themselves.  And the tiles of their query tokens.
  auto tiles_of = [&](int tokens, int& tile_tok) {
    const int n = (tokens * p.g + kTileRows - 1) / kTileRows;
    tile_tok = min((tokens + n - 1) / n, kTileRows / p.g);
    return (tokens + tile_tok - 1) / tile_tok;
  };
  auto saved_by = [&](int x, int& blocks, bool& tile) {
    blocks = pre_n[x] >= 2 ? max(pre_L[x], 0) / kBlockTokens : 0;
    if (blocks == 0) return 0;
    int tile_tok;
    const int tiles = tiles_of(pre_tok[x], tile_tok);
    tile = is_tile(true, tile_tok * p.g);
    return saved_by_sharing(pre_n[x], pre_tok[x], tiles, tile_tok, blocks, p.g, p.Hkv, p.int8);
  };
  int blocks;
  bool tile = false;
  for (int x = tid; x < p.n_prefixes; x += T) atomicAdd(&saved_all, saved_by(x, blocks, tile));
  __syncthreads();
  for (int x = tid; x < p.n_prefixes; x += T) {
    const int saved = saved_by(x, blocks, tile);
    pre_L[x] = worth_sharing(saved, saved_all, tile) ? blocks : 0;
    int tile_tok;
    if (pre_L[x] > 0) atomicAdd(&live, tiles_of(pre_tok[x], tile_tok));
  }
  __syncthreads();
  const int units_all = live * p.Hkv;  // with a unit for every kv head

  // Two passes where there are prefixes: the first finds how long the list is by the plain costs.
  int n_runs = 0, entries = 0, rows = 0, listed = 0, per = 0;
  const int items = p.n_prefixes + p.B;
  for (int pass = p.n_prefixes > 0 ? 0 : 1; pass < 2; ++pass) {
    per = min(entries / kPagedShares, 1 << 20);
    n_runs = entries = rows = listed = 0;
    for (int x0 = 0; x0 < items; x0 += T) {
      const int x = x0 + tid, b = x - p.n_prefixes;
      PagedRun r{};
      int units = 0, list = 0;
      if (x < p.n_prefixes) {
        r.n_blk = pre_L[x];
        if (r.n_blk > 0) {
          r.row = pre_row[x];
          r.n_tok = list = pre_tok[x];
          r.n_tiles = tiles_of(r.n_tok, r.tile_tok);
          r.L = -1;
        }
      } else if (x < items && seq_n[b] > 0) {
        r.row = b;
        r.tok = b * p.kmax;
        r.n_tok = r.tile_tok = seq_n[b];
        r.n_tiles = 1;
        r.L = seq_L[b];
        const int shared = seq_g[b] >= 0 ? pre_L[seq_g[b]] : 0;
        r.first = shared;
        r.n_blk = num_blocks(seq_L[b] + seq_n[b]) - shared;
        r.whole = shared == 0;
      }
      const bool shared_run = r.L < 0;
      const int tile_rows = r.tile_tok * p.g;
      const bool tile = is_tile(shared_run, tile_rows);
      if (r.n_tok > 0) {
        r.heads = p.Hkv > 1 && !tile && r.n_blk <= head_blocks(units_all, tile_rows) ? kPagedWaves : 1;
        units = r.n_tiles * ((p.Hkv + r.heads - 1) / r.heads);
      }
      r.cost = block_cost(shared_run, tile_rows, r.heads, p.int8);
      if (pass == 1 && tile) r.cost = tile_cost(r.cost, per);
      r.pad = unit_pad(shared_run, tile_rows, r.heads);
      Four total;
      const Four before = scan_four<T>(Four{{units > 0, units * r.entries(), units > 0 ? r.n_tok * p.g * p.Hkv : 0, list}}, sums, total);
      const int at = n_runs + before.v[0], place = listed + before.v[3];
      r.start = entries + before.v[1];
      r.row_base = rows + before.v[2];
      n_runs += total.v[0];
      entries += total.v[1];
      rows += total.v[2];
      listed += total.v[3];
      if (pass == 0) continue;
      if (x < p.n_prefixes) {
        r.tok = place;
        pre_n[x] = units > 0 ? at : -1;
        pre_tok[x] = place;
      }
      if (units > 0) {
        p.runs[at] = r;
        if constexpr (kRunsInLds) lds_runs[at] = r;
        starts[at] = r.start;
      }
      if (x >= p.n_prefixes && x < items) p.seqs[b] = PagedSeq{seq_n[b], 0, {0, 0}, r, PagedRun{}};
    }
  }
  __syncthreads();

  // Token lists of the shared runs: a sequence's tokens stand behind those of the sequences before it.  Every member looks at all sequences since its prefix's
  // first, 256 or 1024 members at a time: the whole launch takes 11 us with 64 sequences, 20 with 240, 24 with 300, 60 with 1000, 517 with 4096 of one prefix, once for a
  // step's layers.
  for (int b = tid; b < p.B; b += T) {
    const int x = seq_g[b];
    if (x < 0 || pre_n[x] < 0) continue;
    int pos = 0;
#pragma unroll 8
    for (int o = pre_row[x]; o < b; ++o) pos += seq_g[o] == x ? seq_n[o] : 0;
    for (int i = 0; i < seq_n[b]; ++i) p.tokens[pre_tok[x] + pos + i] = b * p.kmax + i;
    if constexpr (kRunsInLds) p.seqs[b].shared = lds_runs[pre_n[x]];
    else p.seqs[b].shared = p.runs[pre_n[x]];
    p.seqs[b].pos = pos;
  }

  // Few entries go to fewer workgroups, so that each of a workgroup's four wavefronts has a block or two.
  const int used = min(kPagedShares, max(1, entries / kLeastEntries));
  const PagedSplit split{entries / used, entries % used, entries};
  if (tid == 0) {
    PagedHeader h{};
    h.signature = p.signature;
    h.n_runs = n_runs;
    h.total = entries;
    h.per = split.per;
    h.rem = split.rem;
    h.used = used;
    *p.header = h;
  }
  for (int w = tid; w < kPagedShares; w += T) {
    PagedShare s{};
    s.signature = p.signature;
    const int x0 = w < used ? split.first(w) : entries, x1 = w < used ? split.first(w + 1) : entries;
    s.entries = x1 - x0;
    if (s.entries > 0) {
      int lo = 0, hi = n_runs - 1;  // the last run that starts at x0 or before
      while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (starts[m] <= x0) lo = m;
        else hi = m - 1;
      }
      s.run = lo;
      if constexpr (kRunsInLds) s.first = lds_runs[lo];
      else s.first = p.runs[lo];
      s.unit = (x0 - s.first.start) / s.first.entries();
      s.off = (x0 - s.first.start) % s.first.entries();
    }
    p.shares[w] = s;
  }
}

}  // namespace bass

extern "C" size_t bass_paged_attention_plan_bytes(const bass_paged_desc* d) {
  return bass::check_paged_attention(d) == BASS_OK ? bass::paged_layout(d).bytes : 0;
}

extern "C" int bass_paged_attention_plan(const bass_paged_desc* d, const int32_t* ctx_len, const int32_t* draft_len, const int32_t* prefix_of,
                                         const int32_t* prefix_len, int32_t n_prefixes, void* plan, size_t plan_bytes, int32_t* dev_status,
                                         void* stream) {
  using namespace bass;
  const int rc = check_paged_attention(d);
  if (rc != BASS_OK) return rc;
  if (!ctx_len || !draft_len || !plan || !aligned16(plan) || n_prefixes < 0) return BASS_ERR_INVALID_ARG;
  if ((prefix_of == nullptr) != (n_prefixes == 0) || (prefix_of == nullptr) != (prefix_len == nullptr)) return BASS_ERR_INVALID_ARG;
  if (n_prefixes > kMaxPagedBatch) return BASS_ERR_UNSUPPORTED;
  const PagedLayout l = paged_layout(d);
  if (plan_bytes < l.bytes) return BASS_ERR_WORKSPACE_TOO_SMALL;
  char* at = (char*)plan;
  PagedPlanParams p{d->B, d->kmax, d->Hq / d->Hkv, d->Hkv, d->max_pages * d->page_tokens, n_prefixes,
                     d->dtype == BASS_DTYPE_INT8KV, paged_signature(d),
                    ctx_len, draft_len, prefix_of, prefix_len, (PagedHeader*)at, (PagedShare*)(at + l.shares), (PagedRun*)(at + l.runs),
                    (PagedSeq*)(at + l.seqs), (int32_t*)(at + l.tokens), dev_status};
  // a batch of N sequences and prefixes has at most N runs
  if (d->B + n_prefixes <= kSmallBatch) hipLaunchKernelGGL((paged_plan_kernel<256, kSmallBatch>), dim3(1), dim3(256), 0, (hipStream_t)stream, p);
  else hipLaunchKernelGGL((paged_plan_kernel<1024, kMaxPagedBatch>), dim3(1), dim3(1024), 0, (hipStream_t)stream, p);
  return launch_status();
}
