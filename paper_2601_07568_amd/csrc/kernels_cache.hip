// Pages of long caches mapped on the device, and the cache in 4 bits: block tables, slot maps, what is stored and read back.
#include "common.h"

namespace dllm {

#define WSC(c, field, type) ((type*)((c)->ws + (c)->map.field))

// ==========================================================================================
// Block tables (dllm_plan_pages).  needed(b, p): the entry holds a position that is still read.
struct PlanArgs {
  int B, max_pages, pt, n_pages, keep_head;
  const int32_t *length, *first;
  int32_t *table, *stack, *n_free, *granted, *status;
  int32_t *rel, *need, *hdr;      // workspace: pages given back and missing per sequence, then their prefix sums; hdr[0] pages that were
                                  // free, hdr[1] free once everything given back has been pushed
};

struct PlanRow { int n_head, lo, hi; bool ok; };   // entries [0, n_head) and [lo, hi) are needed
__device__ inline PlanRow plan_row(const PlanArgs& a, int b) {
  const int len = a.length[b], f = a.first ? a.first[b] : 0;
  PlanRow r;
  r.ok = len >= 0 && (int64_t)len <= (int64_t)a.max_pages * a.pt && f >= 0;
  r.n_head = r.ok ? (min(a.keep_head, len) + a.pt - 1) / a.pt : 0;
  r.lo = r.ok ? min(f, len) / a.pt : 0;
  r.hi = r.ok ? (len + a.pt - 1) / a.pt : 0;
  return r;
}
__device__ inline bool plan_needed(const PlanRow& r, int p) { return p < r.n_head || (p >= r.lo && p < r.hi); }

// One wave: pages that sequence b gives back (those of the pool) and entries it misses; need -1: a row that is left alone.
__device__ inline void plan_count(const PlanArgs& a, int b, int lane) {
  const PlanRow r = plan_row(a, b);
  int rel = 0, need = 0;
  for (int p = lane; p < a.max_pages && r.ok; p += 64) {
    const int e = a.table[(int64_t)b * a.max_pages + p];
    const bool n = plan_needed(r, p);
    rel += e >= 0 && e < a.n_pages && !n;
    need += e < 0 && n;
  }
  for (int o = 32; o > 0; o >>= 1) { rel += __shfl_xor(rel, o, 64); need += __shfl_xor(need, o, 64); }
  if (lane == 0) {
    a.rel[b] = rel;
    a.need[b] = r.ok ? need : -1;
    if (!r.ok) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
  }
}
// One workgroup of 1024: exclusive prefix sums of rel and, for the granted, of need (-1: not granted); the stack's size.
__device__ inline void plan_scan(const PlanArgs& a, int tid) {
  __shared__ int32_t w_rel[16];
  __shared__ int64_t w_need[16];
  __shared__ int32_t s_rel;
  __shared__ int64_t s_need;
  const int lane = tid & 63, w = tid >> 6;
  const int nf_in = a.n_free[0], nf = min(max(nf_in, 0), a.n_pages);
  if (tid == 0) { s_rel = 0; s_need = 0; }
  __syncthreads();
  // pages given back first: the grants depend on their number
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + tid, v = b < a.B ? a.rel[b] : 0;
    int x = v;
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(x, o, 64); if (lane >= o) x += y; }
    if (lane == 63) w_rel[w] = x;
    __syncthreads();
    int before = s_rel;
    for (int i = 0; i < w; ++i) before += w_rel[i];
    if (b < a.B) a.rel[b] = before + x - v;
    __syncthreads();
    if (tid == 1023) s_rel = before + x;
    __syncthreads();
  }
  const int64_t sum = (int64_t)nf + s_rel;
  const int top = (int)(sum < a.n_pages ? sum : a.n_pages);
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + tid, v = b < a.B ? a.need[b] : 0;
    int64_t x = v > 0 ? v : 0;
    for (int o = 1; o < 64; o <<= 1) { const int64_t y = __shfl_up(x, o, 64); if (lane >= o) x += y; }
    if (lane == 63) w_need[w] = x;
    __syncthreads();
    int64_t upto = s_need + x;
    for (int i = 0; i < w; ++i) upto += w_need[i];
    const bool ok = v == 0 || (v > 0 && upto <= top);
    if (b < a.B) {
      a.need[b] = ok ? (int32_t)(v == 0 ? 0 : upto - v) : -1;
      if (a.granted) a.granted[b] = ok ? 1 : 0;
    }
    __syncthreads();
    if (tid == 1023) s_need = upto;
    __syncthreads();
  }
  if (tid == 0) {
    a.hdr[0] = nf;
    a.hdr[1] = top;
    if (nf != nf_in) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
    if (sum > top) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
  }
}
// One wave: what sequence b gives back goes onto the stack.
__device__ inline void plan_release(const PlanArgs& a, int b, int lane) {
  const PlanRow r = plan_row(a, b);
  if (!r.ok) return;
  int at = a.hdr[0] + a.rel[b];
  bool bad = false;
  for (int p0 = 0; p0 < a.max_pages; p0 += 64) {
    const int p = p0 + lane;
    int32_t* const e = a.table + (int64_t)b * a.max_pages + p;
    const int v = p < a.max_pages ? *e : -1;
    const bool gone = v >= 0 && !plan_needed(r, p), push = gone && v < a.n_pages;
    const uint64_t m = __builtin_amdgcn_ballot_w64(push);
    const int slot = at + __popcll(m & ((1ull << lane) - 1));
    if (push && slot < a.n_pages) a.stack[slot] = v;
    if (gone) *e = -1;
    bad |= gone && !push;
    at += __popcll(m);
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
}
// One wave: the missing entries of sequence b pop their pages.
__device__ inline void plan_take(const PlanArgs& a, int b, int lane) {
  const PlanRow r = plan_row(a, b);
  const int first = a.need[b];
  if (!r.ok || first < 0) return;
  int at = a.hdr[1] - 1 - first;
  bool bad = false;
  for (int p0 = 0; p0 < r.hi; p0 += 64) {                 // (no needed entry behind hi: n_head <= hi)
    const int p = p0 + lane;
    int32_t* const e = a.table + (int64_t)b * a.max_pages + p;
    const bool miss = p < r.hi && plan_needed(r, p) && *e < 0;
    const uint64_t m = __builtin_amdgcn_ballot_w64(miss);
    if (miss) {
      const int page = a.stack[at - __popcll(m & ((1ull << lane) - 1))];
      const bool ok = page >= 0 && page < a.n_pages;
      *e = ok ? page : -1;
      bad |= !ok;
    }
    at -= __popcll(m);
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
  // the last granted sequence's end is the new top
  if (lane == 0) atomicMin(a.n_free, at + 1);
}

__global__ __launch_bounds__(256) void k_plan_count(const PlanArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b < a.B) plan_count(a, b, threadIdx.x & 63);
}
__global__ __launch_bounds__(1024) void k_plan_scan(const PlanArgs a) {
  plan_scan(a, threadIdx.x);
  __syncthreads();
  if (threadIdx.x == 0) a.n_free[0] = a.hdr[1];           // plan_take lowers it to what is left
}
__global__ __launch_bounds__(256) void k_plan_release(const PlanArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b < a.B) plan_release(a, b, threadIdx.x & 63);
}
__global__ __launch_bounds__(256) void k_plan_take(const PlanArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b < a.B) plan_take(a, b, threadIdx.x & 63);
}

hipError_t launch_plan_pages(dllm_ctx* c, hipStream_t s, int n_pages, int B, int keep_head, const int32_t* length, const int32_t* first,
                             int32_t* table, int32_t* stack, int32_t* n_free, int32_t* granted) {
  PlanArgs a;
  a.B = B; a.max_pages = c->cfg.max_pages_per_seq; a.pt = c->cfg.page_tokens; a.n_pages = n_pages; a.keep_head = keep_head;
  a.length = length; a.first = first; a.table = table; a.stack = stack; a.n_free = n_free; a.granted = granted;
  a.status = WSC(c, status, int32_t);
  a.hdr = WSC(c, plan, int32_t);
  a.rel = a.hdr + 4;
  a.need = a.rel + c->cfg.max_batch;
  const int wgs = (B + 3) / 4;
  k_plan_count<<<wgs, 256, 0, s>>>(a);
  k_plan_scan<<<1, 1024, 0, s>>>(a);
  k_plan_release<<<wgs, 256, 0, s>>>(a);
  k_plan_take<<<wgs, 256, 0, s>>>(a);
  return hipGetLastError();
}

// ==========================================================================================
// Slot maps (dllm_slot_map).
struct SlotArgs {
  int B, max_pages, pt, n_pages, capacity;
  const int32_t *start, *end, *table;
  int32_t *cu, *slots, *status;
};
// positions of sequence b that are listed: [lo, hi)
__device__ inline void slot_range(const SlotArgs& a, int b, int& lo, int& hi, bool& bad) {
  const int64_t most = (int64_t)a.max_pages * a.pt;
  const int s = a.start[b], e = a.end[b];
  lo = (int)(s < 0 ? 0 : (s > most ? most : s));
  hi = (int)(e < 0 ? 0 : (e > most ? most : e));
  bad = lo != s || hi != e;
  if (hi < lo) hi = lo;
}
__global__ __launch_bounds__(1024) void k_slot_scan(const SlotArgs a) {
  __shared__ int32_t w_n[16];
  __shared__ int32_t s_n;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  if (tid == 0) s_n = 0;
  __syncthreads();
  bool bad = false;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + tid;
    int v = 0;
    if (b < a.B) {
      int lo, hi;
      bool x;
      slot_range(a, b, lo, hi, x);
      bad |= x;
      v = hi - lo;
    }
    int x = v;
    for (int o = 1; o < 64; o <<= 1) { const int y = __shfl_up(x, o, 64); if (lane >= o) x += y; }
    if (lane == 63) w_n[w] = x;
    __syncthreads();
    int before = s_n;
    for (int i = 0; i < w; ++i) before += w_n[i];
    if (b < a.B) a.cu[b] = before + x - v;
    __syncthreads();
    if (tid == 1023) s_n = before + x;
    __syncthreads();
  }
  if (tid == 0) {
    a.cu[a.B] = s_n;
    if (s_n > a.capacity) bad = true;
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
}
__global__ __launch_bounds__(256) void k_slot_fill(const SlotArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.capacity) return;
  int32_t out = -1;
  if (i < a.cu[a.B]) {
    int lo = 0, hi = a.B;                                  // the last sequence that starts at or before i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] <= i) lo = mid; else hi = mid;
    }
    int p0, p1;
    bool bad;
    slot_range(a, lo, p0, p1, bad);
    const int pos = p0 + (int)(i - a.cu[lo]), pi = pos / a.pt;
    const int page = a.table[(int64_t)lo * a.max_pages + pi];
    if (page >= 0 && page < a.n_pages) out = page * a.pt + (pos - pi * a.pt);
  }
  a.slots[i] = out;
}

hipError_t launch_slot_map(dllm_ctx* c, hipStream_t s, int n_pages, int B, int capacity, const int32_t* start, const int32_t* end,
                           const int32_t* table, int32_t* cu, int32_t* slots) {
  SlotArgs a;
  a.B = B; a.max_pages = c->cfg.max_pages_per_seq; a.pt = c->cfg.page_tokens; a.n_pages = n_pages; a.capacity = capacity;
  a.start = start; a.end = end; a.table = table; a.cu = cu; a.slots = slots;
  a.status = WSC(c, status, int32_t);
  k_slot_scan<<<1, 1024, 0, s>>>(a);
  k_slot_fill<<<(unsigned)(((int64_t)capacity + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

// ==========================================================================================
// The cache in 4 bits.  One workgroup moves 32 positions of one kv head of one layer: a thread per 32 values that share a scale
// (one key's 32 channels, one channel's 32 positions), head_dim threads of each kind.
struct Kv4Args {
  int n_tokens, pt, n_pages, n_pages4, hkv;
  char* kv;              // the pool of dllm_create
  uint8_t* kv4;
  int64_t slab;          // elements of a K or V slab of it
  const int32_t *src, *dst;
  int32_t* status;
};

// 2^(byte - 127), byte in 1 .. 254
__device__ __forceinline__ float pow2_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// 32 bfloat16 values -> 16 bytes of codes and the scale byte
__device__ inline uint4 kv4_quantise(const bf16_t (&x)[32], uint32_t& byte, bool& odd) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint32_t m = x[i] & 0x7fffu;
    if (m >= 0x7f80u) odd = true;
    else top = m > top ? m : top;
  }
  // max = (1 + m/128) 2^(e-127): 7 * 2^(e-129) holds it up to m = 96, twice that always does
  const int e = (int)(top >> 7) - 2 + ((top & 127u) > 96u ? 1 : 0);
  byte = (uint32_t)(e < 7 ? 7 : (e > 252 ? 252 : e));   // (6 * 2^125 is still a number)
  const float s = pow2_of(byte);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = x[i + j], m = b & 0x7fffu;
      f[j] = bf16_to_f32((bf16_t)(m > 0x7f80u ? 0u : b));                   // NaN -> 0
      if (m == 0x7f80u) f[j] = b & 0x8000u ? -6.f * s : 6.f * s;            // infinity: the largest value
    }
    // round to nearest, ties to the even code, values beyond 6 become 6
    uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0], f[1], s, 0);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, f[2], f[3], s, 1);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, f[4], f[5], s, 2);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, f[6], f[7], s, 3);
    w[i >> 3] = v;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DH>
__global__ __launch_bounds__(2 * DH) void k_kv4_store(const Kv4Args a) {
  __shared__ int32_t s_src[32];
  __shared__ int s_ok, s_run;
  const int tid = threadIdx.x, grp = blockIdx.x, h = blockIdx.y, layer = blockIdx.z;
  const int n_slots = a.n_pages * a.pt, n_slots4 = a.n_pages4 * a.pt;       // (below 2^31, checked by the call)
  if (tid < 64) {
    const int i = tid & 31;
    const int d0 = a.dst[(int64_t)grp * 32], d = a.dst[(int64_t)grp * 32 + i], s = a.src[(int64_t)grp * 32 + i];
    const bool none = __builtin_amdgcn_ballot_w64(d != -1) == 0;
    const bool good = d0 >= 0 && d0 < n_slots4 && (d0 & 31) == 0 && d == d0 + i && s >= 0 && s < n_slots;
    const bool all = __builtin_amdgcn_ballot_w64(!good) == 0;
    // the 32 positions one behind the other in a page, from a multiple of 8 on: 16-byte reads of V
    const int s0 = a.src[(int64_t)grp * 32];
    const bool run = __builtin_amdgcn_ballot_w64(!(s == s0 + i && s0 % a.pt + i < a.pt)) == 0 && s0 % 8 == 0 && a.pt % 8 == 0;
    if (tid < 32) s_src[i] = s;
    if (tid == 0) {
      s_ok = all;
      s_run = run;
      if (!all && !none && h == 0 && layer == 0) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
    }
  }
  __syncthreads();
  if (!s_ok) return;
  const int d0 = a.dst[(int64_t)grp * 32], page4 = d0 / a.pt, g4 = (d0 - page4 * a.pt) >> 5;
  const int64_t rec_at = (((int64_t)layer * a.n_pages4 + page4) * a.hkv + h) * (a.pt >> 5) + g4;
  uint8_t* const rec = a.kv4 + rec_at * 34 * DH;
  bf16_t x[32];
  if (tid < DH) {                                           // one key's 32 channels
    constexpr int NG = DH / 32;
    const int key = tid / NG, cb = tid % NG, s = s_src[key], page = s / a.pt;
    const bf16_t* p = (const bf16_t*)a.kv + (2 * layer) * a.slab + (((int64_t)page * a.hkv + h) * a.pt + (s - page * a.pt)) * DH + cb * 32;
#pragma unroll
    for (int i = 0; i < 4; ++i) *(uint4*)(x + 8 * i) = *(const uint4*)(p + 8 * i);
    uint32_t byte;
    bool odd = false;
    const uint4 w = kv4_quantise(x, byte, odd);
    *(uint4*)(rec + key * (DH / 2) + cb * 16) = w;
    rec[32 * DH + ((((key >> 4) << 2) + (key & 3)) * NG + cb) * 4 + ((key >> 2) & 3)] = (uint8_t)byte;
    if (odd) atomicOr(a.status, DLLM_STATUS_NOT_FINITE);
  } else {                                                  // one channel's 32 positions
    const int ch = tid - DH;
    const bf16_t* slab = (const bf16_t*)a.kv + (2 * layer + 1) * a.slab;
    if (s_run) {
      const int s = s_src[0], page = s / a.pt;
      const bf16_t* p = slab + (((int64_t)page * a.hkv + h) * DH + ch) * a.pt + (s - page * a.pt);
#pragma unroll
      for (int i = 0; i < 4; ++i) *(uint4*)(x + 8 * i) = *(const uint4*)(p + 8 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int s = s_src[i], page = s / a.pt;
        x[i] = slab[(((int64_t)page * a.hkv + h) * DH + ch) * a.pt + (s - page * a.pt)];
      }
    }
    uint32_t byte;
    bool odd = false;
    const uint4 w = kv4_quantise(x, byte, odd);
    *(uint4*)(rec + 16 * DH + ch * 16) = w;
    rec[33 * DH + (ch & 15) * (DH / 16) + (ch >> 4)] = (uint8_t)byte;
    if (odd) atomicOr(a.status, DLLM_STATUS_NOT_FINITE);
  }
}

// the value of a code under a scale, as bfloat16 (exact)
__device__ __forceinline__ bf16_t kv4_value(uint32_t code, uint32_t byte) {
  // 0, 1/2, 1, 3/2, 2, 3, 4, 6 in eighths of their binade: (code & 1) is the mantissa bit, codes 0 and 1 have none
  const uint32_t m = code & 7u;
  const float f = (float)(m < 2 ? m : (2u + (m & 1u)) << ((m >> 1) - 1)) * 0.5f * pow2_of(byte);
  return f32_to_bf16(code & 8u ? -f : f);
}

template <int DH>
__global__ __launch_bounds__(2 * DH) void k_kv4_load(const Kv4Args a) {
  constexpr int NG = DH / 32;
  __shared__ int32_t s_src[32], s_dst[32];
  const int tid = threadIdx.x, h = blockIdx.y, layer = blockIdx.z;
  const int64_t i0 = (int64_t)blockIdx.x * 32;
  const int n_slots = a.n_pages * a.pt, n_slots4 = a.n_pages4 * a.pt;
  if (tid < 32) {
    int s = -1, d = -1;
    if (i0 + tid < a.n_tokens) { s = a.src[i0 + tid]; d = a.dst[i0 + tid]; }
    const bool ok = s >= 0 && s < n_slots4 && d >= 0 && d < n_slots;
    if (!ok && !(s == -1 && d == -1) && h == 0 && layer == 0) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
    s_src[tid] = ok ? s : -1;
    s_dst[tid] = d;
  }
  __syncthreads();
  auto record = [&](int s) -> const uint8_t* {
    const int page = s / a.pt, g = (s - page * a.pt) >> 5;
    return a.kv4 + ((((int64_t)layer * a.n_pages4 + page) * a.hkv + h) * (a.pt >> 5) + g) * 34 * DH;
  };
  if (tid < DH) {
    const int i = tid / NG, cb = tid % NG, s = s_src[i];
    if (s < 0) return;
    const uint8_t* rec = record(s);
    const int key = s & 31, d = s_dst[i], page = d / a.pt;
    const uint4 w = *(const uint4*)(rec + key * (DH / 2) + cb * 16);
    const uint32_t byte = rec[32 * DH + ((((key >> 4) << 2) + (key & 3)) * NG + cb) * 4 + ((key >> 2) & 3)];
    bf16_t* p = (bf16_t*)a.kv + (2 * layer) * a.slab + (((int64_t)page * a.hkv + h) * a.pt + (d - page * a.pt)) * DH + cb * 32;
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
    bf16_t x[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) x[e] = kv4_value(ww[e >> 3] >> (4 * (e & 7)) & 15u, byte);
#pragma unroll
    for (int e = 0; e < 4; ++e) *(uint4*)(p + 8 * e) = *(const uint4*)(x + 8 * e);
  } else {
    const int ch = tid - DH;
    bf16_t* slab = (bf16_t*)a.kv + (2 * layer + 1) * a.slab;
    for (int i = 0; i < 32; ++i) {
      const int s = s_src[i];
      if (s < 0) continue;
      const uint8_t* rec = record(s);
      const int d = s_dst[i], page = d / a.pt;
      const uint32_t code = rec[16 * DH + ch * 16 + ((s & 31) >> 1)] >> (4 * (s & 1)) & 15u;
      slab[(((int64_t)page * a.hkv + h) * DH + ch) * a.pt + (d - page * a.pt)] = kv4_value(code, rec[33 * DH + (ch & 15) * (DH / 16) + (ch >> 4)]);
    }
  }
}

static Kv4Args kv4_args(dllm_ctx* c, int n_tokens, const int32_t* src, const int32_t* dst) {
  Kv4Args a;
  a.n_tokens = n_tokens; a.pt = c->cfg.page_tokens; a.n_pages = c->cfg.n_pages; a.n_pages4 = c->n_pages4; a.hkv = c->cfg.n_kv_heads;
  a.kv = c->kv_pool; a.kv4 = c->kv4_pool;
  a.slab = (int64_t)kv_slab_elems(c->cfg);
  a.src = src; a.dst = dst;
  a.status = WSC(c, status, int32_t);
  return a;
}

hipError_t launch_kv4_store(dllm_ctx* c, hipStream_t s, int n_tokens, const int32_t* src, const int32_t* dst) {
  if (c->cfg.n_layers == 0) return hipSuccess;
  const Kv4Args a = kv4_args(c, n_tokens, src, dst);
  const dim3 grid(n_tokens / 32, c->cfg.n_kv_heads, c->cfg.n_layers);
  if (c->cfg.head_dim == 128) k_kv4_store<128><<<grid, 256, 0, s>>>(a);
  else k_kv4_store<64><<<grid, 128, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv4_load(dllm_ctx* c, hipStream_t s, int n_tokens, const int32_t* src, const int32_t* dst) {
  if (c->cfg.n_layers == 0) return hipSuccess;
  const Kv4Args a = kv4_args(c, n_tokens, src, dst);
  const dim3 grid((n_tokens + 31) / 32, c->cfg.n_kv_heads, c->cfg.n_layers);
  if (c->cfg.head_dim == 128) k_kv4_load<128><<<grid, 256, 0, s>>>(a);
  else k_kv4_load<64><<<grid, 128, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dllm
