// Writer and reader of paged caches: bass_page_pool_bytes, bass_paged_append (by slot), bass_paged_gather, bass_paged_gather_int8 (by table).
//
// One workgroup per (sequence, kv head, block of 32 tokens): the rows of a block's tokens, D / 8 chunks of 16 bytes each, against the
// block's chunks, which mix its tokens (V turns them: eight tokens of one head element per chunk).  The turn is made in LDS, so that both sides
// are whole 16-byte chunks of consecutive addresses wherever the rows cover the block.  Bound by memory; every byte moves once.
// us, append / gather, 8 sequences of 2000 tokens from an odd place on, 32 heads: bf16, heads of 128 105 / 101 (524 MB read and written), of 64 43 / 35; INT8 81 / 51 (397 / 270 MB)
// and 34 / 26.  A step's 6 tokens: 4.0 and 3.6, INT8 5.2 and 4.3;
// 24 windows of 64 tokens, 8 heads: 4.4 and 3.8, INT8 4.3 and 3.9.
#include "paged.h"

namespace bass {

struct PagedRows {
  int B, kmax, Hkv, page_tokens, blocks_per_page, n_pages, max_pages, windows;
  void *Kp, *Vp;       // pools
  void *Kr, *Vr;       // rows [B, kmax, Hkv, D]: source of an append, destination of a gather
  float *Ks, *Vs;      // INT8 gather: scales [B, kmax, Hkv]
  const int32_t *slots;                  // append [B, kmax]
  const int32_t *tables, *start, *count; // gather [B, max_pages], [B], [B]
  int32_t* status;
};

// Token slot j (0 .. 7) of a V chunk of lane group grp
__device__ inline int chunk_token(int grp, int j) { return j < 4 ? 4 * grp + j : 16 + 4 * grp + (j - 4); }

// ---------------------------------------------------------------------------------------
// Append.  The rows of a sequence are looked at through windows of 32 that begin where its first row's slot lies in its block:
// consecutive tokens fill blocks one after the other, so that a window's rows are one block's (`together`).  Slots that are not so -- any
// map is allowed -- are written row by row.
// ---------------------------------------------------------------------------------------
template <int D, bool kI8>
__global__ __launch_bounds__(256) void paged_append(PagedRows p) {
  constexpr int CPR = D / 8, kTurns = kBlockTokens * CPR / 256;  // 8-element chunks per row; per thread and tensor
  constexpr int kElem = kI8 ? 1 : 2;
  constexpr int kPitch = D * kElem + 16;  // 16 bytes apart in the banks
  __shared__ __align__(16) uint8_t kt[kI8 ? kBlockTokens * kPitch : 16], vt[kBlockTokens * kPitch];
  __shared__ float kscale[kBlockTokens], vscale[kBlockTokens];
  const int tid = threadIdx.x;
  const int kvh = blockIdx.x % p.Hkv, window = blockIdx.x / p.Hkv % p.windows, b = blockIdx.x / p.Hkv / p.windows;
  const int32_t* slots = p.slots + (size_t)b * p.kmax;
  const int head = max(slots[0], 0) % kBlockTokens;
  // every wavefront looks at the window's 32 slots by itself
  const int i0 = window * kBlockTokens - head, w_lane = tid & 31, i_lane = i0 + w_lane;
  int slot = i_lane >= 0 && i_lane < p.kmax ? slots[i_lane] : -1;
  if (slot >= p.n_pages * p.page_tokens) {
    if (kvh == 0 && tid < 32 && p.status) atomicOr(p.status, BASS_STATUS_PAGE_CLAMPED);
    slot = -1;
  }
  const uint32_t mask = (uint32_t)__ballot(slot >= 0);
  if (mask == 0) return;
  const int blk_lane = slot / kBlockTokens;
  const int blk = __builtin_amdgcn_readlane(blk_lane, __builtin_ctz(mask));
  const bool together = __all(slot < 0 || (blk_lane == blk && slot % kBlockTokens == w_lane));

  uint4 k[kTurns], v[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int c = tid + 256 * i, w = c / CPR, ck = c % CPR;
    k[i] = v[i] = make_uint4(0, 0, 0, 0);
    if (mask >> w & 1) {
      const size_t src = (((size_t)b * p.kmax + (i0 + w)) * p.Hkv + kvh) * D + 8 * ck;
      k[i] = *(const uint4*)((const uint16_t*)p.Kr + src);
      v[i] = *(const uint4*)((const uint16_t*)p.Vr + src);
    }
  }
  constexpr size_t kBytes = kI8 ? (size_t)kBlockTokens * (D + 4) : (size_t)kBlockTokens * D * 2;
  uint8_t* kc = (uint8_t*)p.Kp + pool_block(blk, p.blocks_per_page, p.Hkv, kvh) * kBytes;
  uint8_t* vc = (uint8_t*)p.Vp + pool_block(blk, p.blocks_per_page, p.Hkv, kvh) * kBytes;
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int c = tid + 256 * i, w = c / CPR, ck = c % CPR;
    uint8_t *kw = kc, *vw = vc;
    int at = w;
    if (!together && (mask >> w & 1)) {
      const int s = slots[i0 + w];
      at = s % kBlockTokens;
      const size_t off = pool_block(s / kBlockTokens, p.blocks_per_page, p.Hkv, kvh) * kBytes;
      kw = (uint8_t*)p.Kp + off;
      vw = (uint8_t*)p.Vp + off;
    }
    if constexpr (kI8) {  // the quantizer of bass_kv_append: a row's D / 8 threads are consecutive lanes
      float ka = amax8(k[i]), va = amax8(v[i]);
#pragma unroll
      for (int s = CPR >> 1; s >= 1; s >>= 1) {
        ka = fmaxf(ka, __shfl_xor(ka, s));
        va = fmaxf(va, __shfl_xor(va, s));
      }
      const uint2 kq = quantize8(k[i], ka > 0.f ? 127.0f / ka : 0.f), vq = quantize8(v[i], va > 0.f ? 127.0f / va : 0.f);
      if (together) {
        *(uint2*)&kt[w * kPitch + 8 * ck] = kq;
        *(uint2*)&vt[w * kPitch + 8 * ck] = vq;
        if (ck == 0) {
          kscale[w] = ka / 127.0f;
          vscale[w] = va / 127.0f;
        }
      } else if (mask >> w & 1) {
        *(uint2*)(kw + i8_k_offset(D, at, 8 * ck)) = kq;
#pragma unroll
        for (int e = 0; e < 8; ++e) vw[i8_v_offset(D, at, 8 * ck + e)] = (uint8_t)((e < 4 ? vq.x : vq.y) >> (8 * (e & 3)));
        if (ck == 0) {
          ((float*)(kw + (size_t)kBlockTokens * D))[at] = ka / 127.0f;
          ((float*)(vw + (size_t)kBlockTokens * D))[at] = va / 127.0f;
        }
      }
    } else if (mask >> w & 1) {
      *(uint4*)(kw + 2 * k_elem_offset(D, at, 8 * ck)) = k[i];  // 8 consecutive head elements are one chunk
      if (together) {
        *(uint4*)&vt[w * kPitch + 16 * ck] = v[i];
      } else {
        const uint32_t e[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
        for (int j = 0; j < 8; ++j) ((uint16_t*)vw)[v_elem_offset(D, at, 8 * ck + j)] = (uint16_t)(e[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
  if (!together) return;
  __syncthreads();
  if constexpr (kI8) {
    for (int c = tid; c < 2 * D; c += 256) {  // the block's 16-byte chunks of codes
      const int l = c % 64, grp = l >> 4, r = l & 15;
      const int tile = c / 64 / (D / 64), ks = c / 64 % (D / 64);  // K: token 16 tile + r, head elements 64 ks + 16 grp ..
      if (mask >> (16 * tile + r) & 1) *(uint4*)(kc + 16 * c) = *(const uint4*)&kt[(16 * tile + r) * kPitch + 64 * ks + 16 * grp];
      const int d = 32 * (c / 64) + r;  // V: head elements d and d + 16 of eight tokens
#pragma unroll
      for (int q = 0; q < 4; ++q) {  // four consecutive tokens of a head element, or single ones
        const int w = chunk_token(grp, 4 * (q & 1));
        uint8_t e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = vt[(w + i) * kPitch + d + 16 * (q >> 1)];
        uint8_t* dst = vc + 16 * c + 4 * q;
        if ((mask >> w & 15) == 15) {
          *(uint32_t*)dst = e[0] | (uint32_t)e[1] << 8 | (uint32_t)e[2] << 16 | (uint32_t)e[3] << 24;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (mask >> (w + i) & 1) dst[i] = e[i];
        }
      }
    }
    if (tid < kBlockTokens && (mask >> tid & 1)) {
      ((float*)(kc + (size_t)kBlockTokens * D))[tid] = kscale[tid];
      ((float*)(vc + (size_t)kBlockTokens * D))[tid] = vscale[tid];
    }
  } else {
    for (int c = tid; c < (D / 16) * 64; c += 256) {
      const int mt = c / 64, l = c % 64, grp = l >> 4, dr = l & 15;
      uint16_t e[8];
      uint32_t live = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int w = chunk_token(grp, j);
        e[j] = *(const uint16_t*)&vt[w * kPitch + 2 * (16 * mt + dr)];
        live |= (mask >> w & 1) << j;
      }
      uint16_t* dst = (uint16_t*)vc + (size_t)c * 8;
      if (live == 255) {
        *(uint4*)dst = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (live >> j & 1) dst[j] = e[j];
      }
    }
  }
}

// ---------------------------------------------------------------------------------------
// Gather, codes and scales of INT8 pools or bf16 rows: a workgroup per block that the asked tokens touch.
// ---------------------------------------------------------------------------------------
template <int D, bool kI8>
__global__ __launch_bounds__(256) void paged_gather(PagedRows p) {
  constexpr int kElem = kI8 ? 1 : 2, kPitch = D * kElem + 16;
  constexpr int kChunks = kBlockTokens * D * kElem / 16 / 256;  // 16-byte chunks per thread and tensor (INT8 heads of 64: half of the threads)
  __shared__ __align__(16) uint8_t kt[kBlockTokens * kPitch], vt[kBlockTokens * kPitch];
  const int tid = threadIdx.x;
  const int kvh = blockIdx.x % p.Hkv, window = blockIdx.x / p.Hkv % p.windows, b = blockIdx.x / p.Hkv / p.windows;
  int n = p.count[b];
  bool bad = n < 0 || n > p.kmax;
  n = min(max(n, 0), p.kmax);
  const int64_t off = p.start[b], most = (int64_t)p.max_pages * p.page_tokens;
  const int64_t lo = max(off, (int64_t)0), hi = min(off + n, most);  // tokens that the table can have
  if (n > 0 && (off < 0 || off + n > most)) bad = true;
  if (bad && window == 0 && kvh == 0 && tid == 0 && p.status) atomicOr(p.status, BASS_STATUS_LEN_CLAMPED);
  if (hi <= lo) return;
  const int first = ((int)(lo / kBlockTokens) + window) * kBlockTokens;  // first token of this block: below 2^31
  const int t0 = max((int)lo, first), t1 = (int)min(hi, (int64_t)first + kBlockTokens);
  if (t1 <= t0) return;
  const int page = p.tables[(size_t)b * p.max_pages + first / p.page_tokens];
  if (page < 0 || page >= p.n_pages) {
    if (kvh == 0 && tid == 0 && p.status) atomicOr(p.status, BASS_STATUS_PAGE_CLAMPED);
    return;
  }
  constexpr size_t kBytes = kI8 ? (size_t)kBlockTokens * (D + 4) : (size_t)kBlockTokens * D * 2;
  const size_t at = (((size_t)page * p.Hkv + kvh) * p.blocks_per_page + first % p.page_tokens / kBlockTokens) * kBytes;
  const uint8_t *kc = (const uint8_t*)p.Kp + at, *vc = (const uint8_t*)p.Vp + at;
  constexpr int kTurns = kChunks > 0 ? kChunks : 1;
  constexpr int kUsed = kChunks > 0 ? 256 : kBlockTokens * D * kElem / 16;
  uint4 k[kTurns], v[kTurns];
  if (tid < kUsed) {
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      k[i] = ((const uint4*)kc)[tid + 256 * i];
      v[i] = ((const uint4*)vc)[tid + 256 * i];
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int c = tid + 256 * i, l = c % 64, grp = l >> 4, r = l & 15;
      constexpr int kSteps = D * kElem / 64;  // 64 bytes of a row per step of the K order
      const int tile = c / 64 / kSteps, t = c / 64 % kSteps;
      *(uint4*)&kt[(16 * tile + r) * kPitch + 64 * t + 16 * grp] = k[i];
      const uint32_t e[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      if constexpr (kI8) {
        const int d = 32 * (c / 64) + r;
#pragma unroll
        for (int x = 0; x < 16; ++x) vt[chunk_token(grp, x & 7) * kPitch + d + 16 * (x >> 3)] = (uint8_t)(e[x >> 2] >> (8 * (x & 3)));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) *(uint16_t*)&vt[chunk_token(grp, j) * kPitch + 2 * (16 * (c / 64) + r)] = (uint16_t)(e[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
  __syncthreads();
  constexpr int kPieces = D * kElem / 16;  // 16-byte pieces of a row
  for (int c = tid; c < kBlockTokens * kPieces; c += 256) {
    const int w = c / kPieces, ck = c % kPieces, tok = first + w;
    if (tok >= t0 && tok < t1) {
      const size_t row = ((size_t)b * p.kmax + (size_t)(tok - off)) * p.Hkv + kvh;
      *(uint4*)((uint8_t*)p.Kr + row * D * kElem + 16 * ck) = *(const uint4*)&kt[w * kPitch + 16 * ck];
      *(uint4*)((uint8_t*)p.Vr + row * D * kElem + 16 * ck) = *(const uint4*)&vt[w * kPitch + 16 * ck];
    }
  }
  if constexpr (kI8) {
    const int tok = first + tid;
    if (tid < kBlockTokens && tok >= t0 && tok < t1) {
      const size_t row = ((size_t)b * p.kmax + (size_t)(tok - off)) * p.Hkv + kvh;
      p.Ks[row] = ((const float*)(kc + (size_t)kBlockTokens * D))[tid];
      p.Vs[row] = ((const float*)(vc + (size_t)kBlockTokens * D))[tid];
    }
  }
}

static int launch_paged_rows(const bass_paged_desc* d, bool gather, PagedRows p, void* stream) {
  // the blocks that kmax consecutive tokens can touch
  p.windows = (int)(((int64_t)d->kmax + kBlockTokens - 2) / kBlockTokens + 1);
  const int64_t per_sequence = (int64_t)p.windows * d->Hkv;  // by itself first: the product with B may need more than 64 bits
  if (!grid_fits(per_sequence) || !grid_fits(d->B * per_sequence)) return BASS_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(d->B * per_sequence)), block(256);
  hipStream_t s = (hipStream_t)stream;
  const bool int8 = d->dtype == BASS_DTYPE_INT8KV;
#define BASS_LAUNCH(kernel)                                                            \
  if (d->D == 128) {                                                                   \
    if (int8) hipLaunchKernelGGL((kernel<128, true>), grid, block, 0, s, p);           \
    else hipLaunchKernelGGL((kernel<128, false>), grid, block, 0, s, p);               \
  } else {                                                                             \
    if (int8) hipLaunchKernelGGL((kernel<64, true>), grid, block, 0, s, p);            \
    else hipLaunchKernelGGL((kernel<64, false>), grid, block, 0, s, p);                \
  }
  if (gather) { BASS_LAUNCH(paged_gather) } else { BASS_LAUNCH(paged_append) }
#undef BASS_LAUNCH
  return launch_status();
}

static PagedRows paged_rows(const bass_paged_desc* d, void* Kp, void* Vp, void* Kr, void* Vr, int32_t* status) {
  PagedRows p{};
  p.B = d->B; p.kmax = d->kmax; p.Hkv = d->Hkv;
  p.page_tokens = d->page_tokens; p.blocks_per_page = d->page_tokens / kBlockTokens;
  p.n_pages = d->n_pages; p.max_pages = d->max_pages;
  p.Kp = Kp; p.Vp = Vp; p.Kr = Kr; p.Vr = Vr; p.status = status;
  return p;
}

static int gather_paged(const bass_paged_desc* d, bool int8, const void* Kpool, const void* Vpool, void* K_out, void* V_out, float* Ks, float* Vs,
                        const int32_t* tables, const int32_t* start, const int32_t* n, int32_t* status, void* stream) {
  const int rc = check_paged(d);
  if (rc != BASS_OK) return rc;
  if (int8 != (d->dtype == BASS_DTYPE_INT8KV)) return BASS_ERR_UNSUPPORTED;
  if (!Kpool || !Vpool || !K_out || !V_out || !tables || !start || !n || (int8 && (!Ks || !Vs))) return BASS_ERR_INVALID_ARG;
  if (!aligned16(Kpool) || !aligned16(Vpool) || !aligned16(K_out) || !aligned16(V_out)) return BASS_ERR_INVALID_ARG;
  PagedRows p = paged_rows(d, (void*)Kpool, (void*)Vpool, K_out, V_out, status);
  p.Ks = Ks; p.Vs = Vs; p.tables = tables; p.start = start; p.count = n;
  return launch_paged_rows(d, true, p, stream);
}

}  // namespace bass

extern "C" size_t bass_page_pool_bytes(const bass_paged_desc* d) {
  if (bass::check_paged(d) != BASS_OK) return 0;
  return (size_t)d->n_pages * d->Hkv * (d->page_tokens / bass::kBlockTokens) * bass::page_block_bytes(d);
}

extern "C" int bass_paged_append(const bass_paged_desc* d, void* Kpool, void* Vpool, const void* K_new, const void* V_new,
                                 const int32_t* slots, int32_t* dev_status, void* stream) {
  using namespace bass;
  const int rc = check_paged(d);
  if (rc != BASS_OK) return rc;
  if (!Kpool || !Vpool || !K_new || !V_new || !slots) return BASS_ERR_INVALID_ARG;
  if (!aligned16(Kpool) || !aligned16(Vpool) || !aligned16(K_new) || !aligned16(V_new)) return BASS_ERR_INVALID_ARG;
  PagedRows p = paged_rows(d, Kpool, Vpool, (void*)K_new, (void*)V_new, dev_status);
  p.slots = slots;
  return launch_paged_rows(d, false, p, stream);
}

extern "C" int bass_paged_gather(const bass_paged_desc* d, const void* Kpool, const void* Vpool, void* K_out, void* V_out,
                                 const int32_t* tables, const int32_t* start, const int32_t* n, int32_t* dev_status, void* stream) {
  return bass::gather_paged(d, false, Kpool, Vpool, K_out, V_out, nullptr, nullptr, tables, start, n, dev_status, stream);
}

extern "C" int bass_paged_gather_int8(const bass_paged_desc* d, const void* Kpool, const void* Vpool, int8_t* K_codes, int8_t* V_codes,
                                      float* K_scales, float* V_scales, const int32_t* tables, const int32_t* start, const int32_t* n,
                                      int32_t* dev_status, void* stream) {
  return bass::gather_paged(d, true, Kpool, Vpool, K_codes, V_codes, K_scales, V_scales, tables, start, n, dev_status, stream);
}
