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
  int32_t *rel, *need, *hdr;      // workspace: pages that sequences give back (~n: and wrong entries) and miss (-1: a row that is left
                                  // alone); hdr[0] pages that were free, hdr[1] free once everything given back has been pushed
};

struct PlanRow { int n_head, lo, hi; bool ok; };   // entries [0, n_head) and [lo, hi) are needed
__device__ inline PlanRow plan_row(const PlanArgs& a, int b) {
  const int len = a.length[b], f = a.first ? a.first[b] : 0;
  auto pages = [&](int n) { return n > 0 ? (n - 1) / a.pt + 1 : 0; };
  PlanRow r;
  r.ok = len >= 0 && (int64_t)len <= (int64_t)a.max_pages * a.pt && f >= 0;
  r.n_head = r.ok ? pages(min(a.keep_head, len)) : 0;
  r.lo = r.ok ? min(f, len) / a.pt : 0;
  r.hi = r.ok ? pages(len) : 0;
  return r;
}
__device__ inline bool plan_needed(const PlanRow& r, int p) { return p < r.n_head || (p >= r.lo && p < r.hi); }

// Entries p0 .. p0 + PLAN_ROW - 1 of a row, requested together (-1 from `end` on): the walks below would wait for each 64 otherwise.
constexpr int PLAN_ROW = 512;
__device__ inline void plan_row_entries(const PlanArgs& a, int b, int p0, int lane, int end, int32_t (&e)[PLAN_ROW / 64]) {
  const int32_t* const row = a.table + (int64_t)b * a.max_pages;
#pragma unroll
  for (int i = 0; i < PLAN_ROW / 64; ++i) {
    const int p = p0 + i * 64 + lane;
    e[i] = row[min(p, a.max_pages - 1)];
    if (p >= end) e[i] = -1;
  }
}
__device__ inline int plan_given(int rel) { return rel < 0 ? ~rel : rel; }

// One wave: pages that sequence b gives back and entries it misses.
__device__ inline void plan_count(const PlanArgs& a, int b, int lane) {
  const PlanRow r = plan_row(a, b);
  int rel = 0, need = 0;
  bool wrong = false;
  for (int p0 = 0; p0 < a.max_pages && r.ok; p0 += PLAN_ROW) {
    int32_t e[PLAN_ROW / 64];
    plan_row_entries(a, b, p0, lane, a.max_pages, e);
#pragma unroll
    for (int i = 0; i < PLAN_ROW / 64; ++i) {
      const int p = p0 + i * 64 + lane;
      if (p0 + i * 64 >= a.max_pages) break;
      const bool in = p < a.max_pages, n = plan_needed(r, p);
      rel += in && e[i] >= 0 && e[i] < a.n_pages && !n;
      wrong |= in && e[i] >= a.n_pages && !n;
      need += in && e[i] < 0 && n;
    }
  }
  for (int o = 32; o > 0; o >>= 1) { rel += __shfl_xor(rel, o, 64); need += __shfl_xor(need, o, 64); }
  const bool any = __builtin_amdgcn_ballot_w64(wrong) != 0;
  if (lane == 0) {
    a.rel[b] = any ? ~rel : rel;
    a.need[b] = r.ok ? need : -1;
    if (!r.ok) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
  }
}
// Sums over a workgroup of NT threads; every thread gets the total and the sum of the threads before it.
template <int NT, typename T>
__device__ inline T block_scan(T v, int tid, T* sm, T& total) {
  const int lane = tid & 63, w = tid >> 6;
  T x = v;
  for (int o = 1; o < 64; o <<= 1) { const T y = __shfl_up(x, o, 64); if (lane >= o) x += y; }
  __syncthreads();
  if (lane == 63) sm[w] = x;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) { if (i < w) before += sm[i]; total += sm[i]; }
  return before + x - v;
}
// Pages that are free before the call, and once everything given back is on the stack.
__device__ inline int plan_free(const PlanArgs& a, bool report) {
  const int n = a.n_free[0], nf = min(max(n, 0), a.n_pages);
  if (report && nf != n) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
  return nf;
}
__device__ inline int plan_top(const PlanArgs& a, int nf, int64_t rel, bool report) {
  const int64_t sum = nf + rel;
  if (report && sum > a.n_pages) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
  return (int)(sum < a.n_pages ? sum : a.n_pages);
}
// What the grants say of sequence b, which misses `need` entries where those before it miss `before`: the first place from the
// top that its pages are popped from, -1: it gets nothing.
__device__ inline int plan_grant(int need, int64_t before, int top) {
  return need < 0 ? -1 : (need == 0 ? 0 : (before + need <= top ? (int)before : -1));
}
// One wave: what sequence b gives back goes onto the stack.  e: the first entries of the row.
__device__ inline void plan_release(const PlanArgs& a, const PlanRow& r, int b, int lane, int at, int32_t (&e)[PLAN_ROW / 64]) {
  if (!r.ok) return;
  bool bad = false;
  for (int p0 = 0; p0 < a.max_pages; p0 += PLAN_ROW) {
    if (p0 > 0) plan_row_entries(a, b, p0, lane, a.max_pages, e);
#pragma unroll
    for (int i = 0; i < PLAN_ROW / 64; ++i) {
      const int p = p0 + i * 64 + lane;
      if (p0 + i * 64 >= a.max_pages) break;
      const bool gone = e[i] >= 0 && !plan_needed(r, p), push = gone && e[i] < a.n_pages;
      const uint64_t m = __builtin_amdgcn_ballot_w64(push);
      const int slot = at + __popcll(m & ((1ull << lane) - 1));
      if (push && slot < a.n_pages) a.stack[slot] = e[i];
      if (gone) a.table[(int64_t)b * a.max_pages + p] = -1;
      bad |= gone && !push;
      at += __popcll(m);
    }
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
}
// One wave: the missing entries of sequence b pop their pages, from place `at` on downwards.  e: the first entries of the row.
__device__ inline void plan_take(const PlanArgs& a, const PlanRow& r, int b, int lane, int at, int32_t (&e)[PLAN_ROW / 64]) {
  bool bad = false;
  for (int p0 = 0; p0 < r.hi; p0 += PLAN_ROW) {           // (no needed entry behind hi: n_head <= hi)
    int32_t page[PLAN_ROW / 64];
    if (p0 > 0) plan_row_entries(a, b, p0, lane, a.max_pages, e);
    uint32_t miss = 0;
#pragma unroll
    for (int i = 0; i < PLAN_ROW / 64; ++i) {
      const int p = p0 + i * 64 + lane;
      page[i] = 0;
      if (p0 + i * 64 >= r.hi) continue;
      const bool x = p < r.hi && plan_needed(r, p) && e[i] < 0;
      const uint64_t m = __builtin_amdgcn_ballot_w64(x);
      page[i] = x ? a.stack[at - __popcll(m & ((1ull << lane) - 1))] : 0;
      miss |= (uint32_t)x << i;
      at -= __popcll(m);
    }
#pragma unroll
    for (int i = 0; i < PLAN_ROW / 64; ++i)
      if (miss >> i & 1) {
        const bool ok = page[i] >= 0 && page[i] < a.n_pages;
        a.table[(int64_t)b * a.max_pages + p0 + i * 64 + lane] = ok ? page[i] : -1;
        bad |= !ok;
      }
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
}

// Small batches, one launch: a workgroup with a wave a sequence counts, sums, pushes and pops, a barrier between (what the waves write
// for each other goes through the L1 that they share).  us in a graph, this / three launches: 8 rows of 40 entries 3.7 / 7.6, 16 of 64
// 5.7 / 8.6, 16 of 512 7.3 / 9.9; two rows a wave: 32 of 64 10.2 / 9.3, 32 of 512 16.8 / 10.9.
constexpr int PLAN_ONE_MAX = 16;
static bool plan_one(int B, int max_pages) { return B <= PLAN_ONE_MAX && max_pages <= PLAN_ROW; }
__global__ __launch_bounds__(1024) void k_plan_one(const PlanArgs a) {
  __shared__ int32_t s_rel[PLAN_ONE_MAX], s_need[PLAN_ONE_MAX], s_push[PLAN_ONE_MAX], s_pop[PLAN_ONE_MAX];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  PlanArgs l = a;
  l.rel = s_rel;
  l.need = s_need;
  if (w < a.B) plan_count(l, w, lane);
  __syncthreads();
  if (w == 0) {                                            // a lane a sequence
    const int nf = plan_free(a, lane == 0);
    const int rel = lane < a.B ? plan_given(s_rel[lane]) : 0, need = lane < a.B ? s_need[lane] : 0;
    int64_t r = rel, n = max(need, 0);
    for (int o = 1; o < PLAN_ONE_MAX; o <<= 1) {
      const int64_t x = __shfl_up(r, o, 64), y = __shfl_up(n, o, 64);
      if (lane >= o) { r += x; n += y; }
    }
    const int top = plan_top(a, nf, __shfl(r, PLAN_ONE_MAX - 1, 64), lane == 0);
    const int at = plan_grant(need, n - max(need, 0), top);
    if (lane < a.B) {
      s_push[lane] = (int32_t)min((int64_t)a.n_pages, nf + r - rel);
      s_pop[lane] = need > 0 && at >= 0 ? top - 1 - at : -1;
      if (a.granted) a.granted[lane] = at >= 0 ? 1 : 0;
    }
    // what is left: below the last granted sequence's pages
    int left = (int)(lane < a.B && at >= 0 && need > 0 ? top - n : top);
    for (int o = 32; o > 0; o >>= 1) left = min(left, __shfl_xor(left, o, 64));
    if (lane == 0) a.n_free[0] = left;
  }
  __syncthreads();
  if (w < a.B && s_rel[w] != 0) {
    int32_t e[PLAN_ROW / 64];
    plan_row_entries(l, w, 0, lane, a.max_pages, e);
    plan_release(l, plan_row(l, w), w, lane, s_push[w], e);
  }
  __syncthreads();
  if (w < a.B && s_pop[w] >= 0) {
    int32_t e[PLAN_ROW / 64];
    plan_row_entries(l, w, 0, lane, a.max_pages, e);
    plan_take(l, plan_row(l, w), w, lane, s_pop[w], e);
  }
}

// Large batches.  Every workgroup adds up by itself what the sequences before its four give back (miss).
__global__ __launch_bounds__(256) void k_plan_count(const PlanArgs a) {
  const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.hdr[0] = plan_free(a, true);
  if (b < a.B) plan_count(a, b, threadIdx.x & 63);
}
template <typename F>
__device__ inline int64_t plan_sum(F v, int b0, int B, int64_t* sm, int64_t& total) {
  int64_t x = 0, y = 0, before;
  for (int i = threadIdx.x; i < B; i += 256) {
    const int n = v(i);
    y += n;
    x += i < b0 ? n : 0;
  }
  block_scan<256>(x, threadIdx.x, sm, before);
  block_scan<256>(y, threadIdx.x, sm, total);
  return before;
}
__global__ __launch_bounds__(256) void k_plan_release(const PlanArgs a) {
  __shared__ int64_t sm[4];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, b0 = blockIdx.x * 4, b = b0 + w;
  const int nf = a.hdr[0];
  const int row = min(b, a.B - 1), rel = a.rel[row];           // (as in k_plan_take)
  const PlanRow r = plan_row(a, row);
  int32_t e[PLAN_ROW / 64];
  plan_row_entries(a, row, 0, lane, a.max_pages, e);
  int64_t total;
  auto given = [&](int i) { return plan_given(a.rel[i]); };
  int64_t before = plan_sum(given, b0, a.B, sm, total);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.n_free[0] = a.hdr[1] = plan_top(a, nf, total, true);   // plan_take lowers it to what is left
  if (b >= a.B || rel == 0) return;
  for (int i = b0; i < b; ++i) before += given(i);
  plan_release(a, r, b, lane, (int)min((int64_t)a.n_pages, nf + before), e);
}
__global__ __launch_bounds__(256) void k_plan_take(const PlanArgs a) {
  __shared__ int64_t sm[4];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, b0 = blockIdx.x * 4, b = b0 + w;
  const int top = a.hdr[1];
  // (the row travels while the sums are made)
  const int row = min(b, a.B - 1), need = a.need[row];
  const PlanRow r = plan_row(a, row);
  int32_t e[PLAN_ROW / 64];
  plan_row_entries(a, row, 0, lane, a.max_pages, e);
  int64_t total;
  auto missing = [&](int i) { return max(a.need[i], 0); };
  int64_t before = plan_sum(missing, b0, a.B, sm, total);
  const bool all = total <= top;                                // everything is granted: what is left is known without the others
  if (all && blockIdx.x == 0 && threadIdx.x == 0) a.n_free[0] = (int32_t)(top - total);
  if (b >= a.B) return;
  for (int i = b0; i < b; ++i) before += missing(i);
  const int at = plan_grant(need, before, top);
  if (lane == 0 && a.granted) a.granted[b] = at >= 0 ? 1 : 0;
  if (at < 0 || need == 0) return;
  if (!all && lane == 0) atomicMin(a.n_free, (int32_t)(top - before - need));   // (one address: 500 of them take 3 us)
  plan_take(a, r, b, lane, top - 1 - at, e);
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
  if (plan_one(B, a.max_pages)) {
    k_plan_one<<<1, 1024, 0, s>>>(a);
    return hipGetLastError();
  }
  const int wgs = (B + 3) / 4;
  k_plan_count<<<wgs, 256, 0, s>>>(a);
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
// Where the sequences' positions start in the list, by one workgroup: for more sequences than k_slot_map adds up by itself.
__global__ __launch_bounds__(1024) void k_slot_scan(const SlotArgs a) {
  __shared__ int32_t sm[16];
  const int tid = threadIdx.x;
  bool bad = false;
  int32_t at = 0;
  for (int b0 = 0; b0 < a.B; b0 += 1024) {
    const int b = b0 + tid;
    int lo = 0, hi = 0;
    bool x = false;
    if (b < a.B) slot_range(a, b, lo, hi, x);
    bad |= x;
    int32_t total;
    const int32_t before = block_scan<1024>(hi - lo, tid, sm, total);
    if (b < a.B) a.cu[b] = at + before;
    at += total;
  }
  if (tid == 0) {
    a.cu[a.B] = at;
    if (at > a.capacity) bad = true;
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
}
// A workgroup fills 2048 entries, 4 a thread and pass; up to SLOT_ONE sequences it also adds their lengths up (into LDS; workgroup 0
// writes cu), so that the call is one launch.
constexpr int SLOT_ONE = 4096, SLOT_WG = 2048;
__global__ __launch_bounds__(256) void k_slot_map(const SlotArgs a, int own_scan, int wide) {
  __shared__ int32_t s_cu[SLOT_ONE + 1], s_lo[SLOT_ONE], sm[4];
  const int tid = threadIdx.x;
  if (own_scan) {
    const int per = (a.B + 255) / 256;
    bool bad = false;
    int32_t sum = 0, total;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      int lo, hi;
      bool x;
      if (b < a.B) { slot_range(a, b, lo, hi, x); bad |= x; sum += hi - lo; s_cu[b] = hi - lo; s_lo[b] = lo; }
    }
    int32_t at = block_scan<256>(sum, tid, sm, total);
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < a.B) {
        const int n = s_cu[b];
        s_cu[b] = at;
        if (blockIdx.x == 0) a.cu[b] = at;
        at += n;
      }
    }
    if (tid == 0) {
      s_cu[a.B] = total;
      if (blockIdx.x == 0) { a.cu[a.B] = total; if (total > a.capacity) bad = true; }
    }
    if (bad && blockIdx.x == 0) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
    __syncthreads();
  }
  const int32_t* const cu = own_scan ? s_cu : a.cu;
  const int n = cu[a.B];
  auto start_of = [&](int b) { return own_scan ? s_lo[b] : (int)min((int64_t)max(a.start[b], 0), (int64_t)a.max_pages * a.pt); };
  for (int pass = 0; pass < SLOT_WG / 1024; ++pass) {
    const int64_t i0 = (int64_t)blockIdx.x * SLOT_WG + pass * 1024 + tid * 4;
    if (i0 >= a.capacity) return;
    int4 out = make_int4(-1, -1, -1, -1);
    if (i0 < n) {
      int b = 0, end = a.B;                                // the last sequence that starts at or before i0
      while (end - b > 1) {
        const int mid = (b + end) >> 1;
        if (cu[mid] <= i0) b = mid; else end = mid;
      }
      int first = cu[b], lo = start_of(b), page = -1, pi = -1;
      int32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t i = i0 + e;
        o[e] = -1;
        if (i < n) {
          while (cu[b + 1] <= i) {
            ++b;
            first = cu[b];
            lo = start_of(b);
            pi = -1;
          }
          const int pos = lo + (int)(i - first), p = pos / a.pt;
          if (p != pi) { page = a.table[(int64_t)b * a.max_pages + p]; pi = p; }
          if (page >= 0 && page < a.n_pages) o[e] = page * a.pt + (pos - p * a.pt);
        }
      }
      out = make_int4(o[0], o[1], o[2], o[3]);
    }
    if (wide && i0 + 4 <= a.capacity) *(int4*)(a.slots + i0) = out;
    else {
      const int32_t o[4] = {out.x, out.y, out.z, out.w};
      for (int e = 0; e < 4; ++e) if (i0 + e < a.capacity) a.slots[i0 + e] = o[e];
    }
  }
}

hipError_t launch_slot_map(dllm_ctx* c, hipStream_t s, int n_pages, int B, int capacity, const int32_t* start, const int32_t* end,
                           const int32_t* table, int32_t* cu, int32_t* slots) {
  SlotArgs a;
  a.B = B; a.max_pages = c->cfg.max_pages_per_seq; a.pt = c->cfg.page_tokens; a.n_pages = n_pages; a.capacity = capacity;
  a.start = start; a.end = end; a.table = table; a.cu = cu; a.slots = slots;
  a.status = WSC(c, status, int32_t);
  const int own_scan = B <= SLOT_ONE;
  if (!own_scan) k_slot_scan<<<1, 1024, 0, s>>>(a);
  k_slot_map<<<(unsigned)(((int64_t)capacity + SLOT_WG - 1) / SLOT_WG), 256, 0, s>>>(a, own_scan, ((uintptr_t)slots & 15) == 0);
  return hipGetLastError();
}

// ==========================================================================================
// The cache in 4 bits.  One workgroup moves 32 positions of one kv head of one layer: 2 * head_dim units of 32 values that share a
// scale (one key's 32 channels, one channel's 32 positions), four lanes a unit with 8 values (16 bytes of bfloat16, 4 of codes) each, so
// that neighbouring lanes touch neighbouring bytes on both sides.  Bound: HBM, 4 bytes a value pair of K and V on one side and 1.06 on
// the other: 8 layers of 16 sequences of 2048 positions, 4 key heads of 128, 603 MB each way: load 114 us (5.3 TB/s), store 128 .. 150 (with
// float arithmetic for the scale and a byte store a scale 150 .. 180).
struct Kv4Args {
  int n_tokens, pt, n_pages, n_pages4, hkv;
  char* kv;              // the pool of dllm_create
  uint8_t* kv4;
  int64_t slab;          // elements of a K or V slab of it
  const int32_t *src, *dst;
  int32_t* status;
};
// byte of a record: scale of the 32 channels cb of a key, of a channel
template <int DH> __device__ __forceinline__ int kv4_k_scale(int key, int cb) {
  return 32 * DH + ((((key >> 4) << 2) + (key & 3)) * (DH / 32) + cb) * 4 + ((key >> 2) & 3);
}
template <int DH> __device__ __forceinline__ int kv4_v_scale(int ch) { return 33 * DH + (ch & 15) * (DH / 16) + (ch >> 4); }

// 2^(byte - 127), byte in 1 .. 254
__device__ __forceinline__ float pow2_of(uint32_t byte) { return __uint_as_float(byte << 23); }

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
// largest of a value and those of the other lanes of its four
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));     // lanes 1 0 3 2
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));  // lanes 2 3 0 1
}
// a lane's 8 of a unit's 32 bfloat16 values -> their codes and the unit's scale byte
__device__ __forceinline__ uint32_t kv4_quantise(uint32_t (&x)[4], uint32_t& byte, bool& odd) {
  auto largest = [](const uint32_t (&y)[4]) -> uint32_t {       // magnitudes order like their bits
    u16x2 m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __builtin_bit_cast(u16x2, y[i] & 0x7fff7fffu);
    const u16x2 t = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), __builtin_elementwise_max(m[2], m[3]));
    return max((uint32_t)t[0], (uint32_t)t[1]);
  };
  uint32_t top = largest(x);
  const bool wrong = top >= 0x7f80u, any = __builtin_amdgcn_ballot_w64(wrong) != 0;
  auto part = [](uint32_t w, int i) -> uint32_t { return w >> (16 * i) & 0xffffu; };
  if (any) {
    uint32_t y[4];                                              // the finite values, 0 for the others
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = 0;
      for (int h = 0; h < 2; ++h) if ((part(x[i], h) & 0x7fffu) < 0x7f80u) y[i] |= x[i] & (0xffffu << (16 * h));
    }
    top = largest(y);
    odd |= wrong;
  }
  top = quad_max(top);
  // max = (1 + m/128) 2^(e-127): 7 * 2^(e-129) holds it up to m = 96, twice that always does
  const int e = (int)(top >> 7) - 2 + ((top & 127u) > 96u ? 1 : 0);
  byte = (uint32_t)(e < 7 ? 7 : (e > 252 ? 252 : e));   // (6 * 2^125 is still a number)
  const float s = pow2_of(byte);
  if (any) {                                            // NaN -> 0, infinity -> the largest value, 6 s
    const uint32_t six = __float_as_uint(6.f * s) >> 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      for (int h = 0; h < 2; ++h) {
        const uint32_t v = part(x[i], h), m = v & 0x7fffu;
        if (m >= 0x7f80u) x[i] = (x[i] & ~(0xffffu << (16 * h))) | (m > 0x7f80u ? 0u : (v & 0x8000u) | six) << (16 * h);
      }
  }
  // round to nearest, ties to the even code, values beyond 6 become 6
  uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2_t, x[0]), s, 0);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2_t, x[1]), s, 1);
  v = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2_t, x[2]), s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(v, __builtin_bit_cast(bf16x2_t, x[3]), s, 3);
}
// the values of 8 codes under a scale, as bfloat16 (exact)
__device__ __forceinline__ uint4 kv4_values(uint32_t codes, uint32_t byte) {
  const float s = pow2_of(byte);
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3)));
}
// The 32 lanes' slots are one behind the other in a page, the first a multiple of 8 (asked by both halves of a wave): V of a
// channel is then 16-byte pieces.
__device__ __forceinline__ bool slots_run(int s, int i, int pt) {
  const int s0 = __shfl(s, 0, 64);
  return s0 >= 0 && __builtin_amdgcn_ballot_w64(!(s == s0 + i && s0 % pt + i < pt)) == 0 && s0 % 8 == 0;
}

// Group of a workgroup: two that are side by side in a page, 64 bytes of V each of a 128-byte line, on one XCD (workgroups go round
// over the eight), whose L2 then has the line for both.
__device__ __forceinline__ int kv4_group() {
  const int i = blockIdx.x, n = gridDim.x & ~15;
  return i < n ? (i & ~15) + (i & 7) * 2 + ((i >> 3) & 1) : i;
}

template <int DH>
__global__ __launch_bounds__(256) void k_kv4_store(const Kv4Args a) {
  constexpr int NG = DH / 32, IT = DH / 32;               // 16-byte pieces of K, of V: 4 * DH each
  __shared__ int32_t s_src[32];
  __shared__ int s_ok, s_run, s_dst;
  __shared__ uint32_t s_scale[DH / 2];                    // of K, of V: 32 * DH on in the record
  const int tid = threadIdx.x, grp = kv4_group(), h = blockIdx.y, layer = blockIdx.z;
  const int n_slots = a.n_pages * a.pt, n_slots4 = a.n_pages4 * a.pt;       // (below 2^31, checked by the call)
  if (tid < 64) {
    const int i = tid & 31;
    const int d = a.dst[(int64_t)grp * 32 + i], s = a.src[(int64_t)grp * 32 + i], d0 = __shfl(d, 0, 64);
    const bool none = __builtin_amdgcn_ballot_w64(d != -1) == 0;
    const bool good = d0 >= 0 && d0 < n_slots4 && (d0 & 31) == 0 && d == d0 + i && s >= 0 && s < n_slots;
    const bool all = __builtin_amdgcn_ballot_w64(!good) == 0, run = slots_run(s, i, a.pt);
    if (tid < 32) s_src[i] = s;
    if (tid == 0) {
      s_ok = all;
      s_run = run;
      s_dst = d0;
      if (!all && !none && h == 0 && layer == 0) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
    }
  }
  __syncthreads();
  if (!s_ok) return;
  const int d0 = s_dst, page4 = d0 / a.pt, g4 = (d0 - page4 * a.pt) >> 5;
  uint8_t* const rec = a.kv4 + ((((int64_t)layer * a.n_pages4 + page4) * a.hkv + h) * (a.pt >> 5) + g4) * 34 * DH;
  const bf16_t* const ks = (const bf16_t*)a.kv + (2 * (int64_t)layer) * a.slab;
  const bf16_t* const vs = ks + a.slab;
  bool odd = false;
  uint32_t x[IT][4], byte;
  const bool run = s_run;
  const int s0 = s_src[0], page0 = s0 / a.pt;
  const int64_t ph0 = (int64_t)page0 * a.hkv + h;
#pragma unroll
  for (int it = 0; it < IT; ++it) {                       // IT / 2 rounds of K (DH 64: one), then of V
    const int item = it * 256 + tid, u = item >> 2, part = item & 3;
    if (u < DH) {
      const int key = u / NG, cb = u % NG, s = s_src[key], page = s / a.pt;
      *(uint4*)x[it] = *(const uint4*)(ks + (((int64_t)page * a.hkv + h) * a.pt + (s - page * a.pt)) * DH + cb * 32 + part * 8);
    } else if (run) {
      *(uint4*)x[it] = *(const uint4*)(vs + (ph0 * DH + (u - DH)) * a.pt + (s0 - page0 * a.pt) + part * 8);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int s = s_src[part * 8 + e], page = s / a.pt;
        const uint32_t v = vs[(((int64_t)page * a.hkv + h) * DH + (u - DH)) * a.pt + (s - page * a.pt)];
        x[it][e >> 1] = e & 1 ? x[it][e >> 1] | v << 16 : v;
      }
    }
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int item = it * 256 + tid, u = item >> 2, part = item & 3;
    const uint32_t w = kv4_quantise(x[it], byte, odd);
    *(uint32_t*)(rec + u * 16 + part * 4) = w;            // (K and V codes: 16 bytes a unit, one behind the other)
    if (part == 0) ((uint8_t*)s_scale)[(u < DH ? kv4_k_scale<DH>(u / NG, u % NG) : kv4_v_scale<DH>(u - DH)) - 32 * DH] = (uint8_t)byte;
  }
  __syncthreads();
  if (tid < DH / 2) *(uint32_t*)(rec + 32 * DH + tid * 4) = s_scale[tid];
  if (odd) atomicOr(a.status, DLLM_STATUS_NOT_FINITE);
}

template <int DH>
__global__ __launch_bounds__(256) void k_kv4_load(const Kv4Args a) {
  constexpr int NG = DH / 32, IT = DH / 32;
  __shared__ int32_t s_src[32], s_dst[32];
  __shared__ int s_run;
  const int tid = threadIdx.x, h = blockIdx.y, layer = blockIdx.z;
  const int64_t i0 = (int64_t)kv4_group() * 32;
  const int n_slots = a.n_pages * a.pt, n_slots4 = a.n_pages4 * a.pt;
  if (tid < 64) {
    const int i = tid & 31;
    int s = -1, d = -1;
    if (i0 + i < a.n_tokens) { s = a.src[i0 + i]; d = a.dst[i0 + i]; }
    const bool ok = s >= 0 && s < n_slots4 && d >= 0 && d < n_slots;
    const bool all = __builtin_amdgcn_ballot_w64(!ok) == 0;
    const bool run = slots_run(s, i, a.pt) && slots_run(d, i, a.pt) && (__shfl(s, 0, 64) & 31) == 0;   // a whole record to a run
    if (!ok && !(s == -1 && d == -1) && h == 0 && layer == 0) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
    if (tid < 32) { s_src[i] = ok ? s : -1; s_dst[i] = d; }
    if (tid == 0) s_run = all && run;
  }
  __syncthreads();
  auto record = [&](int s) -> const uint8_t* {
    const int page = s / a.pt, g = (s - page * a.pt) >> 5;
    return a.kv4 + ((((int64_t)layer * a.n_pages4 + page) * a.hkv + h) * (a.pt >> 5) + g) * 34 * DH;
  };
  bf16_t* const ks = (bf16_t*)a.kv + (2 * (int64_t)layer) * a.slab;
  bf16_t* const vs = ks + a.slab;
  auto k_row = [&](int d, int cb, int part) -> bf16_t* {
    const int page = d / a.pt;
    return ks + (((int64_t)page * a.hkv + h) * a.pt + (d - page * a.pt)) * DH + cb * 32 + part * 8;
  };
  auto v_at = [&](int d, int ch) -> bf16_t* {
    const int page = d / a.pt;
    return vs + (((int64_t)page * a.hkv + h) * DH + ch) * a.pt + (d - page * a.pt);
  };
  if (s_run) {
    const uint8_t* const rec = record(s_src[0]);
    uint32_t w[IT], byte[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int item = it * 256 + tid, u = item >> 2, part = item & 3;
      w[it] = *(const uint32_t*)(rec + u * 16 + part * 4);
      byte[it] = rec[u < DH ? kv4_k_scale<DH>(u / NG, u % NG) : kv4_v_scale<DH>(u - DH)];
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int item = it * 256 + tid, u = item >> 2, part = item & 3;
      *(uint4*)(u < DH ? k_row(s_dst[u / NG], u % NG, part) : v_at(s_dst[0], u - DH) + part * 8) = kv4_values(w[it], byte[it]);
    }
    return;
  }
  for (int it = 0; it < IT; ++it) {
    const int item = it * 256 + tid, u = item >> 2, part = item & 3;
    if (u < DH) {
      const int i = u / NG, cb = u % NG, s = s_src[i];
      if (s < 0) continue;
      const uint8_t* rec = record(s);
      const int key = s & 31;
      *(uint4*)k_row(s_dst[i], cb, part) = kv4_values(*(const uint32_t*)(rec + (key * NG + cb) * 16 + part * 4), rec[kv4_k_scale<DH>(key, cb)]);
    } else {
      const int ch = u - DH;
      for (int e = 0; e < 8; ++e) {
        const int s = s_src[part * 8 + e];
        if (s < 0) continue;
        const uint8_t* rec = record(s);
        const uint32_t code = rec[16 * DH + ch * 16 + ((s & 31) >> 1)] >> (4 * (s & 1)) & 15u;
        *v_at(s_dst[part * 8 + e], ch) = (bf16_t)kv4_values(code, rec[kv4_v_scale<DH>(ch)]).x;
      }
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
  else k_kv4_store<64><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv4_load(dllm_ctx* c, hipStream_t s, int n_tokens, const int32_t* src, const int32_t* dst) {
  if (c->cfg.n_layers == 0) return hipSuccess;
  const Kv4Args a = kv4_args(c, n_tokens, src, dst);
  const dim3 grid((n_tokens - 1) / 32 + 1, c->cfg.n_kv_heads, c->cfg.n_layers);
  if (c->cfg.head_dim == 128) k_kv4_load<128><<<grid, 256, 0, s>>>(a);
  else k_kv4_load<64><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dllm
