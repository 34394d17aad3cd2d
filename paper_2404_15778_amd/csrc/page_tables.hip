// Page tables and slots of libbass built on the GPU from the rows' lengths: bass_page_tables.
//
// State: refs[page] = rows that hold the page.  A call is three steps, each a launch, because every one needs the whole result of the
// one before:
//   page_rows    a wavefront per row: shared pages are copied from the tables as they were and counted, pages that are given back
//                are counted down; what the row keeps (mid) and wants.  refs changes by integer atomics, whose order is irrelevant.
//   page_counts  free pages (refs = 0) of each tile of 4096; one more workgroup: prefix sums of what the rows want
//   page_assign  the k-th free page, in the order of the numbers, belongs to the row whose wants cover k.  A workgroup per tile ranks its
//                free pages; a wavefront per row writes what needs no new page.
// Bytes: refs twice, and the tables only where they change.  What bounds it is latency: three dependent launches, 4.3 + 6.4 + 7.4 us for 1000 rows
// and 250 000 pages (1 MB of refs: 0.3 us of the memory's time).  Slots of longer rows (page_slots): 2.6 us for 1000 rows of 64 tokens, 3.3 for 8 of 2000.
#include <algorithm>

#include "paged.h"

namespace bass {

constexpr int kTilePages = 4096, kTileThreads = 256, kTilePer = kTilePages / kTileThreads;
// Slots of newly taken pages are written by the thread that finds the page, token by token, while a row has few new tokens; longer
// prompts get a launch of their own with a thread per token.
constexpr int kInlineSlots = 32;
constexpr int kLdsRows = 4096;  // of so many rows the prefix sums are searched in LDS
// Small pools and few rows: all of it by one workgroup in one launch.  16 rows, 1024 pages: 8.9 us, against 3.2 + 2.7 + 5.4 and two gaps.
constexpr int kSmallPages = 16384, kSmallRows = 64, kSmallSlots = 8192, kSmallThreads = 1024, kSmallPer = kSmallPages / kSmallThreads;

struct PageParams {
  int rows, max_pages, page_tokens, n_pages, kmax, tiles;
  const int32_t *length, *share_from, *share_len, *ctx_len, *n_new;
  int32_t *held, *tables, *refs, *slots;
  int32_t *mid, *want, *start, *count;  // workspace: [rows], [rows], [rows + 1], [tiles]
  int32_t* status;
};

__device__ inline void raise(int32_t* status, int bits) {
  if (bits && status) atomicOr(status, bits);
}

__device__ inline int pages_needed(const PageParams& p, int r, int& bad) {
  int n = p.length[r];
  const int most = p.max_pages * p.page_tokens;
  if (n < 0) { n = 0; bad |= BASS_STATUS_LEN_CLAMPED; }
  if (n > most) { n = most; bad |= BASS_STATUS_LEN_CLAMPED; }
  return num_pages(n, p.page_tokens);
}
__device__ inline int pages_held(const PageParams& p, int r) { return min(max(p.held[r], 0), p.max_pages); }

// First step of row r, by one wavefront: pages shared and given back are counted; returns what the row keeps, and what it wants.
__device__ inline int share_and_release(const PageParams& p, int r, int lane, int& want) {
  int bad = 0;
  const int need = pages_needed(p, r, bad);
  int held = pages_held(p, r);
  int32_t* mine = p.tables + (size_t)r * p.max_pages;
  if (p.share_from && held == 0 && need > 0) {
    const int src = p.share_from[r];
    if (src >= p.rows || src == r) bad |= BASS_STATUS_LEN_CLAMPED;
    else if (src >= 0) {
      held = min(min(max(p.share_len[r], 0) / p.page_tokens, pages_held(p, src)), need);
      const int32_t* theirs = p.tables + (size_t)src * p.max_pages;
      for (int j = lane; j < held; j += 64) {
        int page = theirs[j];
        if (page < 0 || page >= p.n_pages) { page = -1; bad |= BASS_STATUS_PAGE_CLAMPED; }
        else atomicAdd(p.refs + page, 1);
        mine[j] = page;
      }
    }
  }
  for (int j = need + lane; j < held; j += 64) {
    const int page = mine[j];
    if (page < 0 || page >= p.n_pages) bad |= BASS_STATUS_PAGE_CLAMPED;
    else atomicSub(p.refs + page, 1);
  }
  raise(p.status, bad);
  const int mid = min(held, need);
  want = need - mid;
  return mid;
}

__global__ __launch_bounds__(256) void page_rows(PageParams p) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= p.rows) return;
  int want;
  const int mid = share_and_release(p, r, lane, want);
  if (lane == 0) {
    p.mid[r] = mid;
    p.want[r] = want;
  }
}

// Inclusive prefix sum over a workgroup of N threads and its total; all threads call.
template <int N>
__device__ inline int scan_threads(int v, int* lds, int& total) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(x, o);
    if (lane >= o) x += t;
  }
  __syncthreads();  // lds may still be read
  if (lane == 63) lds[wv] = x;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int i = 0; i < N / 64; ++i) {
    if (i < wv) x += lds[i];
    total += lds[i];
  }
  return x;
}
__device__ inline int scan256(int v, int* lds, int& total) { return scan_threads<256>(v, lds, total); }

__global__ __launch_bounds__(kTileThreads) void page_counts(PageParams p) {
  __shared__ int lds[4];
  const int tid = threadIdx.x;
  int total;
  if ((int)blockIdx.x < p.tiles) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kTilePer; ++i) {
      const int page = blockIdx.x * kTilePages + i * kTileThreads + tid;
      if (page < p.n_pages && p.refs[page] == 0) ++n;
    }
    scan256(n, lds, total);
    if (tid == 0) p.count[blockIdx.x] = total;
  } else {
    const int per = (p.rows + kTileThreads - 1) / kTileThreads, r0 = min(tid * per, p.rows), r1 = min(r0 + per, p.rows);
    int mine = 0;
    for (int r = r0; r < r1; ++r) mine += p.want[r];
    int before = scan256(mine, lds, total) - mine;
    for (int r = r0; r < r1; ++r) {
      p.start[r] = before;
      before += p.want[r];
    }
    if (tid == 0) p.start[p.rows] = total;
  }
}

// Free pages of all tiles, and of those in front of tile t; all threads of the workgroup call.
__device__ inline int free_pages(const PageParams& p, int t, int* lds, int& before) {
  int all = 0, front = 0;
  for (int i = threadIdx.x; i < p.tiles; i += kTileThreads) {
    const int c = p.count[i];
    all += c;
    if (i < t) front += c;
  }
  int total;
  scan256(front, lds, before);
  scan256(all, lds, total);
  return total;
}

__device__ inline int new_tokens(const PageParams& p, int r, int& bad) {
  const int n = p.n_new[r];
  if (n < 0 || n > p.kmax) bad |= BASS_STATUS_LEN_CLAMPED;
  return min(max(n, 0), p.kmax);
}

// The row that the k-th free page goes to: the last one whose wants start at k or before (rows that want nothing start where the next does).
__device__ inline int row_of_rank(const int32_t* start, int rows, int k) {
  int lo = 0, hi = rows - 1;
  while (lo < hi) {
    const int m = (lo + hi + 1) >> 1;
    if (start[m] <= k) lo = m;
    else hi = m - 1;
  }
  return lo;
}

__global__ __launch_bounds__(kTileThreads) void page_assign(PageParams p) {
  __shared__ int lds[4], found[kTilePages], starts[kLdsRows + 1];
  const int tid = threadIdx.x, tile = blockIdx.x;
  int before;
  const int free_all = free_pages(p, tile, lds, before);
  const bool inline_slots = p.slots && p.kmax <= kInlineSlots;
  if (tile < p.tiles) {
    const int wanted = p.start[p.rows];
    if (before >= wanted) return;  // the tiles in front have enough
    const bool in_lds = p.rows <= kLdsRows;
    if (in_lds)
      for (int r = tid; r <= p.rows; r += kTileThreads) starts[r] = p.start[r];
    unsigned mask = 0;
#pragma unroll
    for (int i = 0; i < kTilePer; ++i) {
      const int page = tile * kTilePages + tid * kTilePer + i;
      if (page < p.n_pages && p.refs[page] == 0) mask |= 1u << i;
    }
    int total;
    int at = scan256(__popc(mask), lds, total) - __popc(mask);
    for (; mask; mask &= mask - 1) found[at++] = tile * kTilePages + tid * kTilePer + __builtin_ctz(mask);
    __syncthreads();
    // a thread per page: neighbours go to the same row or the next, and a thread has one chain of loads per page
    for (int x = tid; x < min(total, wanted - before); x += kTileThreads) {
      const int k = before + x;
      const int r = in_lds ? row_of_rank(starts, p.rows, k) : row_of_rank(p.start, p.rows, k);
      const int from = in_lds ? starts[r] : p.start[r], to = in_lds ? starts[r + 1] : p.start[r + 1];
      if (to > free_all) break;  // too few for this row, and for those behind it
      const int page = found[x], j = p.mid[r] + k - from;
      p.tables[(size_t)r * p.max_pages + j] = page;
      p.refs[page] = 1;
      if (inline_slots) {  // the new tokens of page j, if there are any
        int bad = 0;
        const int64_t off = (int64_t)p.ctx_len[r] - (int64_t)j * p.page_tokens;
        const int n = new_tokens(p, r, bad), i0 = (int)min(max(-off, (int64_t)0), (int64_t)n), i1 = (int)min((int64_t)n, p.page_tokens - off);
        for (int i = i0; i < i1; ++i) p.slots[(size_t)r * p.kmax + i] = page * p.page_tokens + (int)off + i;
      }
    }
    return;
  }
  const int r = (tile - p.tiles) * 4 + (tid >> 6), lane = tid & 63;
  if (r >= p.rows) return;
  int bad = 0;
  const int need = pages_needed(p, r, bad), mid = p.mid[r], want = p.want[r];
  const bool gets = want == 0 || p.start[r] + want <= free_all;
  const int held = pages_held(p, r);
  int32_t* mine = p.tables + (size_t)r * p.max_pages;
  for (int j = need + lane; j < held; j += 64) mine[j] = -1;
  if (!gets) bad |= BASS_STATUS_NO_PAGES;
  if (lane == 0) p.held[r] = mid + (gets ? want : 0);
  if (inline_slots) {
    const int n = new_tokens(p, r, bad), L = p.ctx_len[r];
    if (n > 0 && L < 0) bad |= BASS_STATUS_LEN_CLAMPED;
    for (int i = lane; i < p.kmax; i += 64) {
      const int64_t tok = (int64_t)L + i, j = tok / p.page_tokens;
      int slot = -1;
      if (i < n && tok >= 0) {
        if (j < mid) {
          const int page = mine[j];
          if (page >= 0 && page < p.n_pages) slot = page * p.page_tokens + (int)(tok - j * p.page_tokens);
          else bad |= BASS_STATUS_PAGE_CLAMPED;
        } else if (gets && j < mid + want) continue;  // the workgroup that finds the page writes this one
      }
      p.slots[(size_t)r * p.kmax + i] = slot;
    }
  }
  raise(p.status, bad);
}

// Slots of long rows, a thread per token, once the tables are complete.
__global__ __launch_bounds__(256) void page_slots(PageParams p) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)p.rows * p.kmax) return;
  const int r = (int)(at / p.kmax), i = (int)(at - (int64_t)r * p.kmax);
  int bad = 0, slot = -1;
  const int n = new_tokens(p, r, bad);
  const int64_t tok = (int64_t)p.ctx_len[r] + i, j = tok / p.page_tokens;
  if (i < n) {
    if (tok < 0) bad |= BASS_STATUS_LEN_CLAMPED;
    else if (j < pages_held(p, r)) {
      const int page = p.tables[(size_t)r * p.max_pages + j];
      if (page >= 0 && page < p.n_pages) slot = page * p.page_tokens + (int)(tok - j * p.page_tokens);
      else bad |= BASS_STATUS_PAGE_CLAMPED;
    }
  }
  p.slots[at] = slot;
  raise(p.status, bad);
}

// The three steps by one workgroup.  The rows' results and the free pages that they get stay in LDS, so that slots need no second look at
// the tables.
__global__ __launch_bounds__(kSmallThreads) void page_tables_small(PageParams p) {
  __shared__ int lds[kSmallThreads / 64], mid[kSmallRows], want[kSmallRows], start[kSmallRows + 1], found[kSmallPages];
  const int tid = threadIdx.x, lane = tid & 63;
  for (int r = tid >> 6; r < p.rows; r += kSmallThreads / 64) {
    int w;
    const int m = share_and_release(p, r, lane, w);
    if (lane == 0) {
      mid[r] = m;
      want[r] = w;
    }
  }
  __threadfence();  // the counts have reached the level that they are read from below
  int total;
  const int per = (p.n_pages + kSmallThreads - 1) / kSmallThreads;
  __syncthreads();
  const int mine = tid < p.rows ? want[tid] : 0;
  const int incl = scan_threads<kSmallThreads>(mine, lds, total);
  if (tid < p.rows) start[tid] = incl - mine;
  if (tid == 0) start[p.rows] = total;
  const int wanted = total;
  unsigned mask = 0;
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i) {
    const int page = tid * per + i;
    if (i < per && page < p.n_pages && __hip_atomic_load(p.refs + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0) mask |= 1u << i;
  }
  int at = scan_threads<kSmallThreads>(__popc(mask), lds, total) - __popc(mask);
  for (; mask && at < wanted; mask &= mask - 1) found[at++] = tid * per + __builtin_ctz(mask);
  const int free_all = total;
  __syncthreads();
  for (int k = tid; k < min(wanted, free_all); k += kSmallThreads) {
    const int r = row_of_rank(start, p.rows, k);
    if (start[r + 1] > free_all) break;
    p.tables[(size_t)r * p.max_pages + mid[r] + k - start[r]] = found[k];
    p.refs[found[k]] = 1;
  }
  if (p.slots) {
    for (int x = tid; x < p.rows * p.kmax; x += kSmallThreads) {
      const int r = x / p.kmax, i = x - r * p.kmax;
      int bad = 0, slot = -1;
      const int n = new_tokens(p, r, bad);
      const int64_t tok = (int64_t)p.ctx_len[r] + i;
      if (i < n) {
        if (tok < 0) bad |= BASS_STATUS_LEN_CLAMPED;
        else {
          const int64_t j = tok / p.page_tokens;
          int page = -2;  // none
          if (j < mid[r]) page = p.tables[(size_t)r * p.max_pages + j];
          else if (j < mid[r] + want[r] && start[r + 1] <= free_all) page = found[start[r] + (int)j - mid[r]];
          if (page >= 0 && page < p.n_pages) slot = page * p.page_tokens + (int)(tok - j * p.page_tokens);
          else if (page != -2) bad |= BASS_STATUS_PAGE_CLAMPED;
        }
      }
      p.slots[x] = slot;
      raise(p.status, bad);
    }
  }
  for (int r = tid >> 6; r < p.rows; r += kSmallThreads / 64) {
    int bad = 0;
    const int need = pages_needed(p, r, bad), held = pages_held(p, r);
    const bool gets = want[r] == 0 || start[r + 1] <= free_all;
    for (int j = need + lane; j < held; j += 64) p.tables[(size_t)r * p.max_pages + j] = -1;
    if (!gets) bad |= BASS_STATUS_NO_PAGES;
    if (lane == 0) p.held[r] = mid[r] + (gets ? want[r] : 0);
    raise(p.status, bad);
  }
}

static int tiles_of(int n_pages) { return (n_pages + kTilePages - 1) / kTilePages; }

}  // namespace bass

extern "C" size_t bass_page_tables_workspace_bytes(int32_t rows, int32_t n_pages) {
  if (rows <= 0 || n_pages <= 0) return 0;
  return (4 * (3 * (size_t)rows + 1 + bass::tiles_of(n_pages)) + 15) / 16 * 16;
}

extern "C" int bass_page_tables(int32_t rows, int32_t max_pages, int32_t page_tokens, int32_t n_pages, const int32_t* length,
                                const int32_t* share_from, const int32_t* share_len, int32_t* held, int32_t* tables, int32_t* refs,
                                int32_t kmax, const int32_t* ctx_len, const int32_t* n_new, int32_t* slots, void* workspace,
                                size_t workspace_bytes, int32_t* dev_status, void* stream) {
  using namespace bass;
  if (rows <= 0 || max_pages <= 0 || page_tokens <= 0 || n_pages <= 0 || kmax < 0) return BASS_ERR_INVALID_ARG;
  if (!length || !held || !tables || !refs || !workspace || !aligned16(workspace)) return BASS_ERR_INVALID_ARG;
  if ((share_from == nullptr) != (share_len == nullptr)) return BASS_ERR_INVALID_ARG;
  if (slots && (!ctx_len || !n_new || kmax == 0)) return BASS_ERR_INVALID_ARG;
  if (page_tokens % kBlockTokens != 0 || kmax > 65535) return BASS_ERR_UNSUPPORTED;
  if ((int64_t)rows * max_pages >= (1ll << 31) || (int64_t)n_pages * page_tokens >= (1ll << 31) || (int64_t)max_pages * page_tokens >= (1ll << 31))
    return BASS_ERR_UNSUPPORTED;
  const int64_t slot_groups = ((int64_t)rows * kmax + 255) / 256, row_groups = ((int64_t)rows + 3) / 4;
  const int tiles = tiles_of(n_pages);
  if (!grid_fits(slot_groups) || !grid_fits(tiles + row_groups)) return BASS_ERR_UNSUPPORTED;
  if (workspace_bytes < bass_page_tables_workspace_bytes(rows, n_pages)) return BASS_ERR_WORKSPACE_TOO_SMALL;
  int32_t* ws = (int32_t*)workspace;
  PageParams p{rows, max_pages, page_tokens, n_pages, kmax, tiles, length, share_from, share_len, ctx_len, n_new,
               held, tables, refs, slots, ws, ws + rows, ws + 2 * (size_t)rows, ws + 3 * (size_t)rows + 1, dev_status};
  hipStream_t s = (hipStream_t)stream;
  if (rows <= kSmallRows && n_pages <= kSmallPages && (int64_t)rows * kmax <= kSmallSlots) {
    hipLaunchKernelGGL(page_tables_small, dim3(1), dim3(kSmallThreads), 0, s, p);
    return launch_status();
  }
  hipLaunchKernelGGL(page_rows, dim3((unsigned)row_groups), dim3(256), 0, s, p);
  hipLaunchKernelGGL(page_counts, dim3(tiles + 1), dim3(kTileThreads), 0, s, p);
  hipLaunchKernelGGL(page_assign, dim3((unsigned)(tiles + row_groups)), dim3(kTileThreads), 0, s, p);
  if (slots && kmax > kInlineSlots) hipLaunchKernelGGL(page_slots, dim3((unsigned)slot_groups), dim3(256), 0, s, p);
  return launch_status();
}
