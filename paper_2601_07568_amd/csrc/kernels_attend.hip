// Attention of a step's rows over parts of the cache: first positions and a window, keys in 4 bits and in the model's type.
#include "mfma_common.h"

namespace dllm {

struct AttendArgs {
  const void* q;            // [B, Q, Hq, dh] rotated
  void* o;                  // as q, or in fragment order (out_mt > 0)
  int out_mt;
  const int32_t *prefix_len, *q_valid, *table, *table4, *len4;
  const void *k, *v;        // slabs of the layer
  const uint8_t* kv4;       // records of the layer
  int B, Q, Hq, Hkv, max_prefix, window, n_sink;
  int pt, max_pages, n_pages, n_pages4;
  int32_t* status;
};

// The keys of sequence b: n_q rows at positions pl .. pl + n_q - 1 read keys [0, kv_len), those below n4 in 4 bits.
struct AttendSeq { int pl, n_q, kv_len, n4; bool bad; };
__device__ __forceinline__ AttendSeq attend_seq(const AttendArgs& a, int b) {
  AttendSeq s;
  const int p = a.prefix_len[b], qv = a.q_valid ? a.q_valid[b] : a.Q;
  s.pl = min(max(p, 0), a.max_prefix);
  s.bad = s.pl != p;
  s.n_q = qv < 0 ? 0 : min(qv, a.Q);
  s.kv_len = s.pl + s.n_q;
  s.n4 = 0;
  if (a.len4) {
    const int n = a.len4[b];
    s.n4 = min(max(n, 0), s.pl) & ~31;
    s.bad |= s.n4 != n;
  }
  return s;
}

// Any shape, both types, any page size: one workgroup per row and query head, 256 keys at a time, a thread a key for the scores and
// a thread a channel for the sums.
template <typename T>
__global__ __launch_bounds__(256) void k_attend_any(const AttendArgs a, int dh) {
  __shared__ float qs[128], sc[256], red[8], part[256];
  __shared__ int64_t at_v[256];      // element of the key's V row in the slab, the byte of its record in 4 bits, -1: not addressable
  const int b = blockIdx.x / a.Q, j = blockIdx.x - b * a.Q, h = blockIdx.y, tid = threadIdx.x;
  const AttendSeq s = attend_seq(a, b);
  if (s.bad && tid == 0 && j == 0 && h == 0) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
  if (j >= s.n_q) return;
  const int64_t row = (int64_t)blockIdx.x * a.Hq + h;
  const int kvh = h / (a.Hq / a.Hkv), p = s.pl + j;
  const int lo = a.window > 0 ? max(0, p - a.window + 1) : 0, n_head = min(a.n_sink, lo), n = n_head + s.kv_len - lo;
  if (tid < dh) qs[tid] = Elem<T>::load((const T*)a.q + row * dh + tid);
  __syncthreads();
  const float scale = 1.0f / sqrtf((float)dh);
  const int groups = 256 / dh, grp = tid / dh, ch = tid - grp * dh;
  const int64_t rec_bytes = 34 * dh;
  auto code = [](uint32_t c) -> float {      // value of a 4-bit code
    const uint32_t m = c & 7u;
    const float f = (float)(m < 2 ? m : (2u + (m & 1u)) << ((m >> 1) - 1)) * 0.5f;
    return c & 8u ? -f : f;
  };
  auto pow2 = [](uint32_t byte) -> float { return __uint_as_float(byte << 23); };
  float m = -DEV_INF, l = 0.f, acc = 0.f;
  bool bad = false;
  for (int c0 = 0; c0 < n; c0 += 256) {
    const int i = c0 + tid, key = i < n_head ? i : lo + (i - n_head);
    float x = -DEV_INF;
    int64_t at = -1;
    if (i < n) {
      const bool four = key < s.n4;
      const int pi = key / a.pt, slot = key - pi * a.pt;
      const int page = pi < a.max_pages ? (four ? a.table4 : a.table)[(int64_t)b * a.max_pages + pi] : -1;
      if (page < 0 || page >= (four ? a.n_pages4 : a.n_pages)) bad = true;
      else if (four) {
        at = (((int64_t)page * a.Hkv + kvh) * (a.pt >> 5) + (slot >> 5)) * rec_bytes;
        const uint8_t* rec = a.kv4 + at;
        const int kk = slot & 31;
        float sum = 0.f;
        for (int cb = 0; cb < dh / 32; ++cb) {
          const uint32_t byte = rec[32 * dh + ((((kk >> 4) << 2) + (kk & 3)) * (dh / 32) + cb) * 4 + ((kk >> 2) & 3)];
          float d = 0.f;
          for (int e = 0; e < 32; e += 2) {
            const uint32_t w = rec[kk * (dh / 2) + cb * 16 + e / 2];
            d = fmaf(qs[cb * 32 + e], code(w & 15u), d);
            d = fmaf(qs[cb * 32 + e + 1], code(w >> 4), d);
          }
          sum = fmaf(d, pow2(byte), sum);
        }
        x = sum * scale;
      } else {
        const int64_t ph = (int64_t)page * a.Hkv + kvh;
        const T* kr = (const T*)a.k + (ph * a.pt + slot) * dh;
        float sum = 0.f;
        for (int e = 0; e < dh; ++e) sum = fmaf(qs[e], Elem<T>::load(kr + e), sum);
        x = sum * scale;
        at = ph * dh * a.pt + slot;
      }
    }
    // largest score of the chunk
    float mx = x;
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
    __syncthreads();                                      // (the chunk before has been read)
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    at_v[tid] = at;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float base = m_new > -DEV_INF ? m_new : 0.f;
    const float e = at >= 0 ? expf(x - base) : 0.f;       // (a score that is NaN stays NaN)
    sc[tid] = e;
    float sum = e;
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
    __syncthreads();
    const float alpha = expf(m - base);
    l = l * alpha + (red[4] + red[5] + red[6] + red[7]);
    acc *= alpha;
    for (int u = grp; u < min(256, n - c0); u += groups) {
      const int64_t av = at_v[u];
      if (av < 0) continue;
      const int ku = c0 + u < n_head ? c0 + u : lo + (c0 + u - n_head);
      float v;
      if (ku < s.n4) {
        const uint8_t* rec = a.kv4 + av;
        const int kk = ku & 31;
        v = code(rec[16 * dh + ch * 16 + (kk >> 1)] >> (4 * (kk & 1)) & 15u) * pow2(rec[33 * dh + (ch & 15) * (dh / 16) + (ch >> 4)]);
      } else {
        v = Elem<T>::load((const T*)a.v + av + (int64_t)ch * a.pt);
      }
      acc = fmaf(sc[u], v, acc);
    }
    m = m_new;
  }
  __syncthreads();
  part[tid] = acc;
  __syncthreads();
  if (tid < dh) {
    float sum = 0.f;
    for (int g = 0; g < groups; ++g) sum += part[g * dh + tid];
    const int64_t at = a.out_mt > 0 ? frag_offset((int)blockIdx.x, h * dh + tid, a.out_mt) : row * dh + tid;
    Elem<T>::store((T*)a.o + at, sum / l);                // a row without a finite score: 0 / 0
  }
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
}

hipError_t launch_attend(dllm_ctx* c, hipStream_t s, const StepGeom& g, int layer, const void* q, void* o, int out_mt) {
  const dllm_config& f = c->cfg;
  const KVView kv = pool_view(c, g, layer);
  AttendArgs a;
  a.q = q; a.o = o; a.out_mt = out_mt;
  a.prefix_len = g.prefix_len; a.q_valid = g.q_valid; a.table = g.block_table;
  a.table4 = g.view->table4; a.len4 = g.view->len4;
  a.k = kv.k; a.v = kv.v;
  a.kv4 = c->kv4_pool ? c->kv4_pool + (int64_t)layer * c->n_pages4 * f.n_kv_heads * (f.page_tokens / 32) * 34 * f.head_dim : nullptr;
  a.B = g.B; a.Q = g.Q; a.Hq = f.n_q_heads; a.Hkv = f.n_kv_heads; a.max_prefix = g.max_kv - g.Q;
  a.window = g.view->window; a.n_sink = g.view->n_sink;
  a.pt = f.page_tokens; a.max_pages = f.max_pages_per_seq; a.n_pages = f.n_pages; a.n_pages4 = c->n_pages4;
  a.status = WSM(c, status, int32_t);
  if (f.dtype == DLLM_BF16) k_attend_any<bf16_t><<<dim3(g.T, f.n_q_heads), 256, 0, s>>>(a, f.head_dim);
  else k_attend_any<float><<<dim3(g.T, f.n_q_heads), 256, 0, s>>>(a, f.head_dim);
  return hipGetLastError();
}

}  // namespace dllm
