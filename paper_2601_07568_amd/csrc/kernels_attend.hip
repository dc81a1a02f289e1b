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
  uint32_t pt_inv;          // key / pt = the high word of key * pt_inv (k_attend)
  int32_t* status;
  // k_attend
  int lds_q;                // where a workgroup's LDS has its queries
  int n_rg, kspl;           // row groups of a (sequence, key head); waves of a workgroup, along the keys of its row group
  int n_parts;              // workgroups along the keys; > 1: partial results, merged by k_attend_merge
  float scale_log2;         // log2(e) / sqrt(dh)
  float *part_o, *part_ml;  // [rows, n_parts, dh], [rows, n_parts, 2]
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
// a thread a channel for the sums.  Bound by the scores' scalar loads of K (32 sequences of 32 rows of 28/4 heads over 8192 keys in 4 bits:
// 59 ms): for page sizes that the kernels below do not take, and to check them.
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

// ==========================================================================================
// bfloat16 models with pages of a multiple of 8 tokens.
//
// One wave owns 16 * QT rows (head in group, token) of a (sequence, kv head) and walks blocks of keys: 128 of them in 4 bits, then 32
// in bfloat16.  Both kinds compute S^T = K Q^T and O^T = V^T P^T with K rows and V^T rows (channels) as the first operand of a
// 16-row matrix instruction, so that a query's scores, statistics and sums stay in the lanes of its column and the scores' layout is
// the second product's operand as it stands (K rows are handed out to match).
//
// 4 bits: v_mfma_scale_f32_16x16x128 multiplies the codes as they lie in memory, with the power of two of every 32 values along k as the
// instruction's own scale; nothing is unpacked.  Its other operand is e4m3: a query row (scaled by a power of two) enters as hi + lo / 16, two
// e4m3 values that together hold the 8 significant bits of a bfloat16 exactly (but for channels 2^14 below the row's largest, whose
// error is 2^-21 of that one); a probability enters the same way, which rounds it to 8 bits (relative 2^-8 at most, 2^-10 on average).
// Operand layouts (lane l, c = l % 16, g = l / 16): the 4-bit operand holds row c, k = 32g .. +31; the e4m3 one column c, bytes 0-15: k =
// 16g .. +15, bytes 16-31: k = 64 + 16g .. +15; the scale of the block of k 32x .. +31 is taken from lane group x.  D holds column c,
// rows 4g .. 4g+3.  So row 4a + i of score tile t is given key 64 (t/4) + 16a + 4 (t%4) + i, and tile t's four scores are bytes 4t ..
// 4t+3 of the second product's operand.  With 64 channels k holds them twice, against hi and lo of the query.
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef const int32_t __attribute__((address_space(4)))* const_i32;   // what a launch only reads, by scalar loads

template <int SEL>
__device__ __forceinline__ f32x4 mfma4(u32x4 a, i32x8 b, f32x4 c, uint32_t scale_a, uint32_t scale_b) {
  const i32x8 av = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, b, c, 4, 0, SEL, (int)scale_a, 0, (int)scale_b);
}
__device__ __forceinline__ f32x4 mfma4_sel(int sel, u32x4 a, i32x8 b, f32x4 c, uint32_t scale_a, uint32_t scale_b) {
  switch (sel) {   // (a constant once the loops are unrolled)
    case 0: return mfma4<0>(a, b, c, scale_a, scale_b);
    case 1: return mfma4<1>(a, b, c, scale_a, scale_b);
    case 2: return mfma4<2>(a, b, c, scale_a, scale_b);
    default: return mfma4<3>(a, b, c, scale_a, scale_b);
  }
}
// four floats -> four e4m3 (hi) and what they leave out, times 16, in e4m3 (lo)
__device__ __forceinline__ void e4m3_pair(float x0, float x1, float x2, float x3, int& hi, int& lo) {
  int h;                                                        // (any register: the two conversions fill a half each)
  s16x2 l;
  asm volatile("" : "=v"(h), "=v"(l));
  h = __builtin_amdgcn_cvt_pk_fp8_f32(x0, x1, h, false);
  h = __builtin_amdgcn_cvt_pk_fp8_f32(x2, x3, h, true);
  const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8(h, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(h, true);
  l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, x0 - a[0], x1 - a[1], 0.0625f, false);
  l = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(l, x2 - b[0], x3 - b[1], 0.0625f, true);
  hi = h;
  lo = __builtin_bit_cast(int, l);
}

// Probabilities are kept 2^P_SHIFT times too large, and the running maximum follows the scores only when one exceeds it by more than
// P_SLACK: with 16 rows a tile some row's maximum moves in nearly every block, which would rescale all sums each time.  The largest
// probability is then 2^8, near the top of e4m3 (448); what lo resolves is 2^-13, 2^-17 of a row's largest at least.
constexpr float P_SHIFT = 4.0f, P_SLACK = 4.0f;

// Online softmax of one query tile's NT score tiles, in two steps: the maximum (log2 units after scale_log2), to which all sums are
// brought where it moves, then the probabilities in the scores' place.  A row that has seen no key but masked ones keeps the maximum
// -inf and weights 0.
template <int NT, int DT, int QT>
__device__ __forceinline__ void attend_max(const f32x4 (&s)[NT], int t, float scale_log2, float (&m_run)[QT], float (&l_run)[QT],
                                           f32x4 (&oacc)[DT][QT]) {
  float mx = s[0][0];
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[x][i]);
  mx = rows_max(mx) * scale_log2;
  // (a first finite score always moves it: -inf + P_SLACK)
  if (__builtin_amdgcn_ballot_w64(mx > m_run[t] + P_SLACK) != 0) {
    const float m_new = fmaxf(m_run[t], mx);
    const float alpha = m_new > -DEV_INF ? __builtin_amdgcn_exp2f(m_run[t] - m_new) : 1.f;
    l_run[t] *= alpha;
#pragma unroll
    for (int d = 0; d < DT; ++d) oacc[d][t] = oacc[d][t] * alpha;
    m_run[t] = m_new;
  }
}
template <int NT>
__device__ __forceinline__ void attend_exp(f32x4 (&s)[NT], float scale_log2, float m, float& l) {
  const float off = P_SHIFT - (m > -DEV_INF ? m : 0.f);
  float p0 = 0.f, p1 = 0.f;
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[x][i] = __builtin_amdgcn_exp2f(fmaf(s[x][i], scale_log2, off));
      if (i & 1) p1 += s[x][i];
      else p0 += s[x][i];
    }
  l += p0 + p1;
}

// What a workgroup of k_attend / k_attend_f32 works on: row group rg (16 * QT rows) of (sequence b, kv head kvh), part `part` of the keys.
struct AttendRows {
  AttendSeq sq;
  int b, kvh, rg, part, R;      // R: rows of the (sequence, kv head)
  int lo, lo_all, n_head;       // its rows read keys [0, n_head) and from lo on; all of them those below n_sink and from lo_all on
  bool none;                    // nothing to do
};
template <int QT>
__device__ __forceinline__ AttendRows attend_rows(const AttendArgs& a) {
  AttendRows v;
  // the row groups of a part one behind the other on one XCD (workgroups go round over the eight), whose L2 then holds its keys for them
  const int xi = blockIdx.x >> 3, u = (xi / a.n_rg << 3) + (blockIdx.x & 7), seq = u / a.n_parts;
  v.rg = xi % a.n_rg;
  v.part = u - seq * a.n_parts;
  v.none = seq >= a.B * a.Hkv;
  v.b = v.none ? 0 : seq / a.Hkv;
  v.kvh = seq - v.b * a.Hkv;
  v.sq = attend_seq(a, v.b);
  v.R = v.sq.n_q * (a.Hq / a.Hkv);
  v.none |= v.rg * 16 * QT >= v.R;
  v.lo = v.lo_all = v.n_head = 0;
  if (a.window > 0 && !v.none) {
    const int n_q = v.sq.n_q, r0 = v.rg * 16 * QT, r1 = min(r0 + 16 * QT, v.R) - 1;
    const bool one = r0 / n_q == r1 / n_q;
    v.lo = max(0, v.sq.pl + (one ? r0 % n_q : 0) - a.window + 1);
    v.lo_all = max(0, v.sq.pl + (one ? r1 % n_q : n_q - 1) - a.window + 1);
    v.n_head = min(a.n_sink, v.lo);
  }
  return v;
}
// row (token * Hq + head) of the lane's query in tile t (of the last one beyond the end), and the position above which it reads keys
__device__ __forceinline__ int attend_row(const AttendArgs& a, const AttendRows& v, int r, int& wlo) {
  const int rr = min(r, v.R - 1), hg = rr / v.sq.n_q, j = rr - hg * v.sq.n_q;
  wlo = a.window > 0 ? max(-1, v.sq.pl + j - a.window) : -1;   // (differences with keys stay in 32 bits)
  return (v.b * a.Q + j) * a.Hq + v.kvh * (a.Hq / a.Hkv) + hg;
}
__device__ __forceinline__ void attend_report(const AttendArgs& a, const AttendRows& v, bool bad) {
  if (bad) atomicOr(a.status, DLLM_STATUS_BAD_PAGE);
  if (v.sq.bad && threadIdx.x == 0 && v.rg == 0 && v.part == 0 && v.kvh == 0) atomicOr(a.status, DLLM_STATUS_BAD_LENGTH);
}

__device__ __forceinline__ void attend_put(const AttendArgs& a, int64_t row, int ch, int dh, f32x4 v, bf16_t*) {
  const int tok = (int)(row / a.Hq), head = (int)(row - (int64_t)tok * a.Hq);
  const int64_t at = a.out_mt > 0 ? frag_offset(tok, head * dh + ch, a.out_mt) : row * dh + ch;
  *(uint2*)((bf16_t*)a.o + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}
__device__ __forceinline__ void attend_put(const AttendArgs& a, int64_t row, int ch, int dh, f32x4 v, float*) {
  *(f32x4*)((float*)a.o + row * dh + ch) = v;
}

// The end of a workgroup: the waves bring their sums to a common maximum and hand each other slices of the channels through LDS; then
// the output, or this part's share of it.  The lane holds query column c, channels 16 d + 4g + i.
template <typename T, int DH, int QT>
__device__ __forceinline__ void attend_finish(const AttendArgs& a, const AttendRows& v, int lane, int w, unsigned char* smem, const int (&row_in)[QT],
                                              f32x4 (&oacc)[DH / 16][QT], const float (&m_run)[QT], const float (&l_run)[QT]) {
  constexpr int DT = DH / 16;
  const int c = lane & 15, g = lane >> 4;
  float l_red[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float l = l_run[t];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    l_red[t] = l;
  }
  auto store = [&](int d, int t, f32x4 x, float m, float l) {
    if (v.rg * 16 * QT + t * 16 + c >= v.R) return;
    const int64_t ro = row_in[t];
    const int ch = d * 16 + 4 * g;
    if (a.n_parts > 1) {
      const int64_t slot = ro * a.n_parts + v.part;
      *(f32x4*)(a.part_o + slot * DH + ch) = x;
      if (d == 0 && g == 0) { a.part_ml[slot * 2] = m; a.part_ml[slot * 2 + 1] = l; }
      return;
    }
    const float inv = 1.0f / l;                                 // (no finite score: 0 / 0)
    attend_put(a, ro, ch, DH, x * inv, (T*)nullptr);
  };
  if (a.kspl == 1) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int d = 0; d < DT; ++d) store(d, t, oacc[d][t], m_run[t], l_red[t]);
    return;
  }
  const int KS = a.kspl;                                        // 2 or 4
  float* sm_m = (float*)smem;                                   // [KS][QT][16] maxima, then sums
  float* sm_l = sm_m + KS * QT * 16;
  f32x4* sm_o = (f32x4*)(smem + 4 * QT * 32 * sizeof(float));   // [DT * QT][KS - 1][64]
  if (g == 0) {
#pragma unroll
    for (int t = 0; t < QT; ++t) { sm_m[(w * QT + t) * 16 + c] = m_run[t]; sm_l[(w * QT + t) * 16 + c] = l_red[t]; }
  }
  __syncthreads();
  float m_all[QT], l_all[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    float mx = -DEV_INF;
    for (int k = 0; k < KS; ++k) mx = fmaxf(mx, sm_m[(k * QT + t) * 16 + c]);
    const float base = mx > -DEV_INF ? mx : 0.f;
    float ls = 0.f;
    for (int k = 0; k < KS; ++k) ls = fmaf(sm_l[(k * QT + t) * 16 + c], __builtin_amdgcn_exp2f(sm_m[(k * QT + t) * 16 + c] - base), ls);
    m_all[t] = mx;
    l_all[t] = ls;
    const float f = __builtin_amdgcn_exp2f(m_run[t] - base);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      oacc[d][t] = oacc[d][t] * f;
      const int u = d * QT + t, own = u & (KS - 1);
      if (own != w) sm_o[(u * (KS - 1) + ((w - own - 1) & (KS - 1))) * 64 + lane] = oacc[d][t];
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const int u = d * QT + t;
      if ((u & (KS - 1)) != w) continue;
      f32x4 x = oacc[d][t];
      for (int k = 0; k < KS - 1; ++k) x = x + sm_o[(u * (KS - 1) + k) * 64 + lane];
      store(d, t, x, m_all[t], l_all[t]);                       // (a part's statistics go with channel tile 0)
    }
}

// Bound, many rows: the matrix pipe (64 scaled products a block of 128 keys and 32 rows, 42 % busy) and the vector pipe beside it (65 %;
// 16 exponentials and two conversions each of 8 values a lane and tile) at two waves a SIMD: 32 sequences of 32 rows of 28/4 heads over up to 8192 keys
// in 4 bits 130 us in a row of calls (0.86 PFLOP/s; 152 with the running maximum followed at once and the sums by vector instructions, 137
// before the queries went to LDS and the tiles took turns).  Few rows: reading the records (32 single tokens of 32/32 heads, windows of 4096 of
// 32768 keys: 107 us, 5.5 TB/s).  In bfloat16: 16 KB a block of 32 keys and wave from the L2, which many row groups of a key head
// read again and again (16 x 64 rows of 28/4 heads, windows of 2048: 137 us, the staged kernel 74).
template <int DH, int QT>
__global__ __launch_bounds__(256, 2) void k_attend(const AttendArgs a) {
  constexpr int KK = DH / 32, DT = DH / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const AttendRows v = attend_rows<QT>(a);
  if (v.none) { attend_report(a, v, false); return; }
  const int b = v.b, kvh = v.kvh, kv_len = v.sq.kv_len, n4 = v.sq.n4, lo = v.lo, lo_all = v.lo_all, n_head = v.n_head;
  const int U = a.n_parts * a.kspl, unit = v.part * a.kspl + w;
  int row_in[QT], wlo[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) row_in[t] = attend_row(a, v, v.rg * 16 * QT + t * 16 + c, wlo[t]);
  auto read_all = [&](int k0, int k1) { return (bool)((k1 <= a.n_sink) | (k0 >= lo_all)); };     // every row reads keys k0 .. k1 - 1
  auto read_any = [&](int k0, int k1) { return (bool)((k0 < n_head) | (k1 > lo)); };             // some row may

  f32x4 oacc[DT][QT];
  float m_run[QT], l_run[QT];                 // l_run: the lane's share of the sum
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m_run[t] = -DEV_INF;
    l_run[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) oacc[d][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool bad = false;
  const bf16_t* const q = (const bf16_t*)a.q;

  // ---- keys in 4 bits, blocks of 128: those of the head, then those from lo on
  const int first = min(lo, n4) >> 7, n_b = lo < n4 ? ((n4 + 127) >> 7) - first : 0;
  int n_a = (min(n_head, n4) + 127) >> 7;
  if (n_b > 0) n_a = min(n_a, first);
  const int n_blk4 = n_a + n_b;
  // Their queries as e4m3 pairs, in LDS for all waves: as registers that live through the loop they would not fit.
  u32x4* const sm_q = (u32x4*)(smem + a.lds_q);                // [QT][4: hi, hi, lo, lo (64 channels: hi, lo)][64]
  uint32_t* const sm_qs = (uint32_t*)(sm_q + QT * 4 * 64);      // [QT][64] scale bytes: hi, lo in the next byte (64 channels: the lane's own)
  if (n_blk4 > 0) {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (t % a.kspl != w) continue;
      const bf16_t* p = q + (int64_t)row_in[t] * DH + 16 * g;
      uint32_t x[DH / 8];
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) {
        const u32x4 u = *(const u32x4*)(p + 64 * i), v = *(const u32x4*)(p + 64 * i + 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[8 * i + e] = u[e]; x[8 * i + 4 + e] = v[e]; }
      }
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
      top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
      const uint32_t e = max(top >> 7, 12u);                    // the largest channel goes to 2^7 .. 2^8
      const float f = __uint_as_float((261u - e) << 23);
      u32x4 h[DH / 64], l[DH / 64];
#pragma unroll
      for (int i = 0; i < DH / 16; ++i) {
        int hi, lo;
        e4m3_pair(__uint_as_float(x[2 * i] << 16) * f, __uint_as_float(x[2 * i] & 0xffff0000u) * f, __uint_as_float(x[2 * i + 1] << 16) * f,
                  __uint_as_float(x[2 * i + 1] & 0xffff0000u) * f, hi, lo);
        h[i >> 2][i & 3] = (uint32_t)hi;
        l[i >> 2][i & 3] = (uint32_t)lo;
      }
#pragma unroll
      for (int i = 0; i < DH / 64; ++i) {
        sm_q[(t * 4 + i) * 64 + lane] = h[i];
        sm_q[(t * 4 + DH / 64 + i) * 64 + lane] = l[i];
      }
      sm_qs[t * 64 + lane] = DH == 128 ? (e - 7) | (e - 11) << 8 : (g < 2 ? e - 7 : e - 11);
    }
    __syncthreads();
  }
  if (unit < n_blk4) {
    const int gpp = a.pt >> 5;                                  // groups of 32 a page
    const const_i32 table = (const_i32)(uintptr_t)(a.table4 + (int64_t)b * a.max_pages);
    const int gch = DH == 128 ? g : g & 1;
    int k_off = (16 * ((c >> 2) & 1) + (c & 3)) * (DH / 2) + gch * 16, ks_off = 32 * DH + (((c >> 2) & 1) * 4 + (c & 3)) * (DH / 8) + gch * 4;
    int v_off = 16 * DH + c * 16, vs_off = 33 * DH + c * (DH / 16);
    // A block's four records (scalar work): their bases, and which of them hold no key that is read or cannot be addressed - anything
    // may lie there.  Table entries are asked for a block ahead.
    struct Ent { int e0, e1, e2, e3; };
    struct Recs { int k0, k1, v; uint32_t dead; };              // the lane's records: K of the first 64 keys, of the others, V
    auto key_of = [&](int i) { const int j = min(i, n_blk4 - 1); return (j < n_a ? j : first + (j - n_a)) << 7; };
    auto page_of = [&](int key) { return (int)__umulhi((uint32_t)key, a.pt_inv); };
    auto entry = [&](int key) { return table[min(page_of(key), a.max_pages - 1)]; };
    auto entries = [&](int k0) { return Ent{entry(k0), entry(k0 + 32), entry(k0 + 64), entry(k0 + 96)}; };
    auto records = [&](int k0, const Ent& x) {
      Recs r;
      int e0 = x.e0, e1 = x.e1, e2 = x.e2, e3 = x.e3;
      r.dead = 0;
      const uint32_t top = max(max((uint32_t)e0, (uint32_t)e1), max((uint32_t)e2, (uint32_t)e3));
      if (top >= (uint32_t)a.n_pages4 || k0 + 128 > n4 || !(k0 + 128 <= n_head || k0 >= lo)) {
        auto look = [&](int j, int& e) {
          const int key = k0 + 32 * j;
          const bool ok = (page_of(key) < a.max_pages) & ((uint32_t)e < (uint32_t)a.n_pages4), want = (key < n4) & read_any(key, key + 32);
          bad |= want & !ok;
          r.dead |= (uint32_t)!(want & ok) << j;
          if (!ok) e = 0;
        };
        look(0, e0);
        look(1, e1);
        look(2, e2);
        look(3, e3);
      }
      auto rec = [&](int j, int e) { const int key = k0 + 32 * j; return (e * a.Hkv + kvh) * gpp + ((key - page_of(key) * a.pt) >> 5); };
      const int r0 = rec(0, e0), r1 = rec(1, e1), r2 = rec(2, e2), r3 = rec(3, e3);
      r.k0 = c & 8 ? r1 : r0;
      r.k1 = c & 8 ? r3 : r2;
      const int va = g & 1 ? r1 : r0, vb = g & 1 ? r3 : r2;
      r.v = g & 2 ? vb : va;
      return r;
    };
    u32x4 kf[8], vf[DT];
    uint32_t ks[2], vs[DT / 4];
    auto load_k = [&](const Recs& r) {
      asm volatile("" : "+v"(k_off), "+v"(ks_off));             // (else the sums with the pool's address live through the loop)
      const uint8_t *p0 = a.kv4 + (int64_t)r.k0 * (34 * DH), *p1 = a.kv4 + (int64_t)r.k1 * (34 * DH);
      ks[0] = *(const uint32_t*)(p0 + ks_off);
      ks[1] = *(const uint32_t*)(p1 + ks_off);
#pragma unroll
      for (int t = 0; t < 8; ++t) kf[t] = *(const u32x4*)((t < 4 ? p0 : p1) + k_off + (t & 3) * 4 * (DH / 2));
    };
    auto load_v = [&](const Recs& r) {
      asm volatile("" : "+v"(v_off), "+v"(vs_off));
      const uint8_t* p = a.kv4 + (int64_t)r.v * (34 * DH);
#pragma unroll
      for (int d = 0; d < DT / 4; ++d) vs[d] = *(const uint32_t*)(p + vs_off + d * 4);
#pragma unroll
      for (int d = 0; d < DT; ++d) vf[d] = *(const u32x4*)(p + v_off + d * 256);
    };
    // The loads of a block's K are issued when the block before has its scores, those of V behind its second product: they travel
    // while the wave, and the SIMD's other one, work on what lies between.
    int k0 = key_of(unit);
    Recs cur = records(k0, entries(k0));
    Ent ahead = entries(key_of(unit + U));
    __builtin_amdgcn_sched_barrier(0);
    load_k(cur);
    __builtin_amdgcn_sched_barrier(0);
    load_v(cur);
    __builtin_amdgcn_sched_barrier(0);
    for (int i = unit; i < n_blk4; i += U) {
      asm volatile("" ::: "memory");                            // (the queries are read again for every block)
      // Matrix instructions of one query tile beside the vector instructions of the other: scores of tile 1 while tile 0's become
      // probabilities, V^T P^T of tile 0 while tile 1's do.
      f32x4 s[QT][8];
      i32x8 ph[QT], pl[QT];
      auto query = [&](int x, int part) {
        const u32x4 u = sm_q[(x * 4 + 2 * part) * 64 + lane], v = sm_q[(x * 4 + 2 * part + 1) * 64 + lane];
        return i32x8{(int)u[0], (int)u[1], (int)u[2], (int)u[3], (int)v[0], (int)v[1], (int)v[2], (int)v[3]};
      };
      // a product of the scores of tile x: n < 8 query hi with K tile n, behind it (128 channels) query lo with tile n - 8
      uint32_t qs = 0;
      i32x8 qh, ql;
      auto ask_query = [&](int x) {
        qs = sm_qs[x * 64 + lane];
        qh = query(x, 0);
        if constexpr (DH == 128) ql = query(x, 1);
      };
      auto score = [&](int x, int n) {
        const int t = n & 7;
        s[x][t] = n < 8 ? mfma4_sel(t & 3, kf[t], qh, f32x4{0.f, 0.f, 0.f, 0.f}, ks[t >> 2], qs)
                        : mfma4_sel(t & 3, kf[t], ql, s[x][t], ks[t >> 2], qs >> 8);
      };
      const bool some = cur.dead != 0 || !read_all(k0, k0 + 128);
      auto mask = [&](int x) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const bool gone = (cur.dead >> (2 * (t >> 2) + (g >> 1))) & 1;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int at = 64 * (t >> 2) + 4 * (t & 3) + e;     // key = k0 + 16 g + at
            const bool see = (bool)((at < a.n_sink - k0 - 16 * g) | (at > wlo[x] - k0 - 16 * g)) & !gone;
            s[x][t][e] = see ? s[x][t][e] : -DEV_INF;
          }
        }
      };
      float off = 0.f;
      auto weight_scale = [&](int x) { off = P_SHIFT - (m_run[x] > -DEV_INF ? m_run[x] : 0.f); };
      auto weight = [&](int x, int t) {                         // score tile t becomes four bytes of the second product's operands
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[x][t][e], a.scale_log2, off));
        l_run[x] += (p[0] + p[1]) + (p[2] + p[3]);
        int h, l;
        e4m3_pair(p[0], p[1], p[2], p[3], h, l);
        asm volatile("" : "+v"(h), "+v"(l), "+v"(l_run[x]));    // (computed here, not where it is used)
        ph[x][t] = h;
        pl[x][t] = l;
      };
      auto output = [&](int x, int n) {                         // n < DT: P hi with channel tile n, behind it P lo with tile n - DT
        const int d = n % DT;
        oacc[d][x] = n < DT ? mfma4_sel(d & 3, vf[d], ph[x], oacc[d][x], vs[d >> 2], 127) : mfma4_sel(d & 3, vf[d], pl[x], oacc[d][x], vs[d >> 2], 123);
      };
      constexpr int NS = DH == 128 ? 16 : 8, NO = 2 * DT;       // products of a query tile's scores, of its outputs
      ask_query(0);
#pragma unroll
      for (int n = 0; n < NS; ++n) score(0, n);
      const int k1 = key_of(i + U);
      const Recs nxt = records(k1, ahead);
      ahead = entries(key_of(i + 2 * U));
      if (some) {
        mask(0);
        const bool gone = (cur.dead >> g) & 1;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[d][e] = gone ? 0u : vf[d][e];
#pragma unroll
        for (int d = 0; d < DT / 4; ++d) vs[d] = gone ? 0x7f7f7f7fu : vs[d];
      }
      attend_max<8, DT, QT>(s[0], 0, a.scale_log2, m_run, l_run, oacc);
      weight_scale(0);
      if constexpr (QT == 2) {
        ask_query(1);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int n = t * NS / 8; n < (t + 1) * NS / 8; ++n) score(1, n);
          weight(0, t);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (some) mask(1);
        attend_max<8, DT, QT>(s[1], 1, a.scale_log2, m_run, l_run, oacc);
        __builtin_amdgcn_sched_barrier(0);
        load_k(nxt);                                            // (behind the last block: that one again)
        weight_scale(1);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int n = t * NO / 8; n < (t + 1) * NO / 8; ++n) output(0, n);
          weight(1, t);
        }
        __builtin_amdgcn_sched_barrier(0);
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) weight(0, t);
        __builtin_amdgcn_sched_barrier(0);
        load_k(nxt);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int n = 0; n < NO; ++n) output(QT - 1, n);
      __builtin_amdgcn_sched_barrier(0);
      load_v(nxt);
      __builtin_amdgcn_sched_barrier(0);
      cur = nxt;
      k0 = k1;
    }
  }

  // ---- keys in bfloat16, blocks of 32; the units go on behind the ones that took the last blocks of 128
  const int f16 = n4 >> 5;
  const int sB = max(lo, n4) >> 5, n_b16 = ((kv_len + 31) >> 5) - sB;
  const int n_a16 = min(max(0, ((n_head + 31) >> 5) - f16), sB - f16), n_blk = n_a16 + n_b16;
  int i = unit - n_blk4 % U;
  if (i < 0) i += U;
  if (i < n_blk) {
    const bf16_t *kslab = (const bf16_t*)a.k, *vslab = (const bf16_t*)a.v;
    const const_i32 table = (const_i32)(uintptr_t)(a.table + (int64_t)b * a.max_pages);
    u32x4 qf[QT][KK];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[t][kk] = *(const u32x4*)(q + (int64_t)row_in[t] * DH + kk * 32 + g * 8);
    // A block's four pieces of 8 keys, each in one page: where the lane's piece of K and of V lies in the slabs, and which of them have
    // no key that is read or cannot be addressed.
    struct Ent { int e0, e1, e2, e3; };
    struct Pcs { int64_t k, v; uint32_t dead; };
    auto key_of = [&](int i) { const int j = min(i, n_blk - 1); return (j < n_a16 ? f16 + j : sB + (j - n_a16)) << 5; };
    auto page_of = [&](int key) { return (int)__umulhi((uint32_t)key, a.pt_inv); };
    auto entry = [&](int key) { return table[min(page_of(key), a.max_pages - 1)]; };
    auto entries = [&](int k0) { return Ent{entry(k0), entry(k0 + 8), entry(k0 + 16), entry(k0 + 24)}; };
    auto piece = [&](int key, int page, uint32_t bit, uint32_t& dead, int64_t& v) -> int64_t {
      const int pi = page_of(key), slot = key - pi * a.pt;
      const bool ok = (pi < a.max_pages) & ((uint32_t)page < (uint32_t)a.n_pages), want = (key < kv_len) & read_any(key, key + 8);
      bad |= want & !ok;
      dead |= want & ok ? 0u : bit;
      const int64_t rows = ((int64_t)(ok ? page : 0) * a.Hkv + kvh) * a.pt;
      v = rows * DH + slot;
      return (rows + slot) * DH;
    };
    auto pieces = [&](int k0, const Ent& x) {
      Pcs r;
      uint32_t dead = 0;
      int64_t v0, v1, v2, v3;
      const int64_t r0 = piece(k0, x.e0, 1, dead, v0), r1 = piece(k0 + 8, x.e1, 2, dead, v1), r2 = piece(k0 + 16, x.e2, 4, dead, v2),
                    r3 = piece(k0 + 24, x.e3, 8, dead, v3);
      const int64_t ka = c & 4 ? r1 : r0, kb = c & 4 ? r3 : r2, va = g & 1 ? v1 : v0, vb = g & 1 ? v3 : v2;
      r.k = c & 8 ? kb : ka;
      r.v = g & 2 ? vb : va;
      r.dead = dead;
      return r;
    };
    u32x4 kf[2][KK], vf[DT];
    // key 8 (c / 4) + c % 4 + 4 tt of the block is row c of score tile tt
    auto load_k = [&](const Pcs& r) {
      const bf16_t* kp = kslab + (r.k + (c & 3) * DH + g * 8);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) kf[tt][kk] = *(const u32x4*)(kp + tt * 4 * DH + kk * 32);
    };
    auto load_v = [&](const Pcs& r) {
      const bf16_t* vp = vslab + (r.v + c * a.pt);
#pragma unroll
      for (int d = 0; d < DT; ++d) vf[d] = *(const u32x4*)(vp + (int64_t)d * 16 * a.pt);
    };
    auto zero_keys = [&](u32x4 (&v)[DT], auto gone) {            // V of the lane's keys 8g + e for which gone(e)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t m = (gone(2 * e) ? 0u : 0xffffu) | (gone(2 * e + 1) ? 0u : 0xffff0000u);
#pragma unroll
        for (int d = 0; d < DT; ++d) v[d][e] &= m;
      }
    };
    int k0 = key_of(i);
    Pcs cur = pieces(k0, entries(k0));
    Ent ahead = entries(key_of(i + U));
    __builtin_amdgcn_sched_barrier(0);
    load_k(cur);
    __builtin_amdgcn_sched_barrier(0);
    load_v(cur);
    __builtin_amdgcn_sched_barrier(0);
    for (; i < n_blk; i += U) {
      f32x4 s[QT][2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) acc = mfma16(kf[tt][kk], qf[t][kk], acc);
          s[t][tt] = acc;
        }
      const int k1 = key_of(i + U);
      const Pcs nxt = pieces(k1, ahead);
      ahead = entries(key_of(i + 2 * U));
      bool apart = false;                                       // some rows do not read a value that is not finite
      const bool all = read_all(k0, k0 + 32);
      if (cur.dead != 0 || k0 + 32 > kv_len || !all) {
        const bool gone = (cur.dead >> g) & 1;
        const int end = gone ? 0 : kv_len - k0 - 8 * g;         // the lane's keys 8g + e, e < end, are there
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = 4 * tt + e;
              const bool see = (bool)((at < a.n_sink - k0 - 8 * g) | (at > wlo[t] - k0 - 8 * g)) & (at < end);
              s[t][tt][e] = see ? s[t][tt][e] : -DEV_INF;
            }
        zero_keys(vf, [&](int e) { return e >= end; });
        if (!all) {
          uint32_t odd = 0;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t v = vf[d][e];
              odd |= (uint32_t)((v & 0x7f80u) == 0x7f80u) | (uint32_t)((v & 0x7f800000u) == 0x7f800000u);
            }
          apart = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
        }
      }
#pragma unroll
      for (int t = 0; t < QT; ++t) attend_max<2, DT, QT>(s[t], t, a.scale_log2, m_run, l_run, oacc);
#pragma unroll
      for (int t = 0; t < QT; ++t) attend_exp<2>(s[t], a.scale_log2, m_run[t], l_run[t]);
      u32x4 ph[QT], pl[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = s[t][e >> 1][(e & 1) * 2], p1 = s[t][e >> 1][(e & 1) * 2 + 1];
          const uint32_t h = pack_bf16x2(p0, p1);
          ph[t][e] = h;
          pl[t][e] = pack_bf16x2(p0 - __uint_as_float(h << 16), p1 - __uint_as_float(h & 0xffff0000u));
        }
      __builtin_amdgcn_sched_barrier(0);
      load_k(nxt);
      __builtin_amdgcn_sched_barrier(0);
      if (apart) {
        // 0 * NaN is NaN: what is not finite is taken out of V and added to the rows that read it.  Two products count, per channel
        // and row, the values that are +infinity or NaN and those that are -infinity or NaN.
        u32x4 see[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int hd = a.n_sink - k0 - 8 * g, wl = wlo[t] - k0 - 8 * g;
            see[t][e] = ((2 * e < hd) | (2 * e > wl) ? 0x3f80u : 0u) | ((2 * e + 1 < hd) | (2 * e + 1 > wl) ? 0x3f800000u : 0u);
          }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          u32x4 pos, neg;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pos[e] = neg[e] = 0;
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              const uint32_t v = (vf[d][e] >> (16 * hi)) & 0xffffu, m = v & 0x7fffu, one = 0x3f80u << (16 * hi);
              pos[e] |= (m > 0x7f80u) | (v == 0x7f80u) ? one : 0u;
              neg[e] |= (m > 0x7f80u) | (v == 0xff80u) ? one : 0u;
              vf[d][e] &= m >= 0x7f80u ? ~(0xffffu << (16 * hi)) : 0xffffffffu;
            }
          }
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            const f32x4 np = mfma16(pos, see[t], f32x4{0.f, 0.f, 0.f, 0.f}), nn = mfma16(neg, see[t], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (np[e] > 0.f) oacc[d][t][e] += DEV_INF;
              if (nn[e] > 0.f) oacc[d][t][e] -= DEV_INF;        // (both: NaN)
            }
          }
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
#pragma unroll
        for (int t = 0; t < QT; ++t) oacc[d][t] = mfma16(vf[d], ph[t], oacc[d][t]);
#pragma unroll
        for (int t = 0; t < QT; ++t) oacc[d][t] = mfma16(vf[d], pl[t], oacc[d][t]);
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v(nxt);
      __builtin_amdgcn_sched_barrier(0);
      cur = nxt;
      k0 = k1;
    }
  }

  attend_finish<bf16_t, DH, QT>(a, v, lane, w, smem, row_in, oacc, m_run, l_run);
  attend_report(a, v, bad && lane == 0);
}

// ==========================================================================================
// Float models with pages of a multiple of 4 tokens: the same walk in blocks of 32 keys, 16 rows a wave, on the float matrix
// instruction.  v_mfma_f32_16x16x4 (lane l, c = l % 16, g = l / 16): the first operand is row c, k = g, the second column c, k = g,
// one float each; D is column c, rows 4g .. 4g+3.  k = g of score step (kk, e) is channel 16 kk + 4g + e, so that a lane's share of a row
// of K or Q is 16-byte pieces; the scores of keys 4g + i are then step i of V^T P^T as they stand, and V^T's share keys 4g .. 4g+3.
// Bound by a wave's chain of matrix instructions (64 channels: 64 of them a block, 0.9 us) and the latency of its loads.  Windows of 300
// .. 4096 keys of 4 heads of 64 channels, 1 .. 32 sequences of 1 .. 96 rows: 11 .. 63 us where k_attend_any takes 190 .. 430.
template <int DH>
__global__ __launch_bounds__(256, 2) void k_attend_f32(const AttendArgs a) {
  constexpr int KK = DH / 16, DT = DH / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const AttendRows v = attend_rows<1>(a);
  if (v.none) { attend_report(a, v, false); return; }
  const int kv_len = v.sq.kv_len, lo = v.lo, lo_all = v.lo_all, n_head = v.n_head;
  const int U = a.n_parts * a.kspl, unit = v.part * a.kspl + w;
  int row_in[1], wlo;
  row_in[0] = attend_row(a, v, v.rg * 16 + c, wlo);
  auto read_all = [&](int k0, int k1) { return (bool)((k1 <= a.n_sink) | (k0 >= lo_all)); };
  auto read_any = [&](int k0, int k1) { return (bool)((k0 < n_head) | (k1 > lo)); };
  f32x4 oacc[DT][1], qf[KK];
  float m_run[1] = {-DEV_INF}, l_run[1] = {0.f};
  bool bad = false;
#pragma unroll
  for (int d = 0; d < DT; ++d) oacc[d][0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *(const f32x4*)((const float*)a.q + (int64_t)row_in[0] * DH + 16 * kk + 4 * g);
  const int sB = lo >> 5, n_a = min((n_head + 31) >> 5, sB), n_blk = n_a + ((kv_len + 31) >> 5) - sB;
  const const_i32 table = (const_i32)(uintptr_t)(a.table + (int64_t)v.b * a.max_pages);
  auto page_of = [&](int key) { return (int)__umulhi((uint32_t)key, a.pt_inv); };
  auto mm = [&](float x, float y, f32x4 z) { return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, z, 0, 0, 0); };
  auto first_of = [&](int i) { return (i < n_a ? i : sB + (i - n_a)) << 5; };
  int ek[2], ev[2];                                             // table entries of the block's K and V, requested a block ahead
  auto entries = [&](int k0) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      ek[u] = table[min(page_of(k0 + 16 * u + c), a.max_pages - 1)];
      ev[u] = table[min(page_of(k0 + 16 * u + 4 * g), a.max_pages - 1)];
    }
  };
  if (unit < n_blk) entries(first_of(unit));
  for (int i = unit; i < n_blk; i += U) {
    const int k0 = first_of(i);
    // K row k0 + 16 u + c, V^T columns k0 + 16 u + 4g .. +3 of half u; dead: none of these four keys is read, or they cannot be addressed
    f32x4 kf[2][KK], vf[2][DT];
    bool dead[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int key_k = k0 + 16 * u + c, key_v = k0 + 16 * u + 4 * g, pk = page_of(key_k), pv = page_of(key_v);
      const bool okk = (pk < a.max_pages) & ((uint32_t)ek[u] < (uint32_t)a.n_pages), okv = (pv < a.max_pages) & ((uint32_t)ev[u] < (uint32_t)a.n_pages);
      const bool want = (key_v < kv_len) & read_any(key_v, key_v + 4);
      bad |= want & !okv;
      dead[u] = !(want & okv);
      const float* kp = (const float*)a.k + ((((int64_t)(okk ? ek[u] : 0) * a.Hkv + v.kvh) * a.pt + (key_k - pk * a.pt)) * DH + 4 * g);
      const float* vp = (const float*)a.v + ((((int64_t)(okv ? ev[u] : 0) * a.Hkv + v.kvh) * DH + c) * a.pt + (key_v - pv * a.pt));
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[u][kk] = *(const f32x4*)(kp + 16 * kk);
#pragma unroll
      for (int d = 0; d < DT; ++d) vf[u][d] = *(const f32x4*)(vp + (int64_t)d * 16 * a.pt);
    }
    if (i + U < n_blk) entries(first_of(i + U));
    f32x4 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;                   // (two sums: half the chain)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        x = mm(kf[u][kk][0], qf[kk][0], x);
        y = mm(kf[u][kk][1], qf[kk][1], y);
        x = mm(kf[u][kk][2], qf[kk][2], x);
        y = mm(kf[u][kk][3], qf[kk][3], y);
      }
      s[u] = x + y;
    }
    const bool all = read_all(k0, k0 + 32);
    auto is = [&](int u, int e) { return (k0 + 16 * u + 4 * g + e < kv_len) & !dead[u]; };                  // a key there is
    auto mine = [&](int u, int e) {                                                                        // ... that the lane's row reads
      const int key = k0 + 16 * u + 4 * g + e;
      return is(u, e) & ((key < a.n_sink) | (key > wlo));
    };
    if (__builtin_amdgcn_ballot_w64(dead[0] | dead[1]) != 0 || k0 + 32 > kv_len || !all) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[u][e] = mine(u, e) ? s[u][e] : -DEV_INF;
#pragma unroll
          for (int d = 0; d < DT; ++d) vf[u][d][e] = is(u, e) ? vf[u][d][e] : 0.f;
        }
    }
    attend_max<2, DT, 1>(s, 0, a.scale_log2, m_run, l_run, oacc);
    if (!all) {
      // 0 * NaN is NaN: what is not finite is taken out of V and added to the rows that read it (their number, by products)
      bool odd = false;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= !(fabsf(vf[u][d][e]) < DEV_INF);
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          f32x4 np = {0.f, 0.f, 0.f, 0.f}, nn = np;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float x = vf[u][d][e], see = mine(u, e) ? 1.f : 0.f;
              np = mm(x != x || x == DEV_INF ? 1.f : 0.f, see, np);
              nn = mm(x != x || x == -DEV_INF ? 1.f : 0.f, see, nn);
              vf[u][d][e] = fabsf(x) < DEV_INF ? x : 0.f;
            }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (np[e] > 0.f) oacc[d][0][e] += DEV_INF;
            if (nn[e] > 0.f) oacc[d][0][e] -= DEV_INF;
          }
        }
      }
    }
    attend_exp<2>(s, a.scale_log2, m_run[0], l_run[0]);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int d = 0; d < DT; ++d) oacc[d][0] = mm(vf[u][d][e], s[u][e], oacc[d][0]);
  }
  attend_finish<float, DH, 1>(a, v, lane, w, smem, row_in, oacc, m_run, l_run);
  attend_report(a, v, bad);
}

// Partial results of a row: four channels a lane, eight parts requested together.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_attend_merge(const AttendArgs a, int64_t n_rows) {
  constexpr int LR = DH / 4;
  const int64_t row = (int64_t)blockIdx.x * (256 / LR) + threadIdx.x / LR;
  if (row >= n_rows) return;
  const int ch = threadIdx.x % LR * 4;
  const int tok = (int)(row / a.Hq), b = tok / a.Q;
  const int qv = a.q_valid ? a.q_valid[b] : a.Q;
  if (tok - b * a.Q >= qv) return;                               // (no partials of rows that are not part of the call)
  const float2* ml = (const float2*)a.part_ml + row * a.n_parts;
  const float* po = a.part_o + row * a.n_parts * DH + ch;
  float mx = -DEV_INF, den = 0.f;
  f32x4 num = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < a.n_parts; p0 += 8) {
    float2 x[8];
    f32x4 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = min(p0 + i, a.n_parts - 1);
      x[i] = ml[p];
      o[i] = *(const f32x4*)(po + (int64_t)p * DH);
    }
    float m = mx;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, x[i].x);
    const float base = m > -DEV_INF ? m : 0.f, r = __builtin_amdgcn_exp2f(mx - base);
    den *= r;
    num = num * r;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p0 + i < a.n_parts) {
        const float f = __builtin_amdgcn_exp2f(x[i].x - base);
        den = fmaf(x[i].y, f, den);
        num = num + o[i] * f;
      }
    mx = m;
  }
  attend_put(a, row, ch, DH, num * (1.0f / den), (T*)nullptr);
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
  a.pt_inv = 0;
  a.status = WSM(c, status, int32_t);
  // (the division by multiplication is exact for positions below 2^32 / page_tokens, for any with a page size of a power of two)
  const bool pow2 = (f.page_tokens & (f.page_tokens - 1)) == 0;
  const bool records_fit = !a.len4 || (int64_t)c->n_pages4 * f.n_kv_heads * (f.page_tokens / 32) < ((int64_t)1 << 31);   // (numbered in 31 bits)
  const bool bf16 = f.dtype == DLLM_BF16;
  if (c->kernel_mode == 0 && f.page_tokens % (bf16 ? 8 : 4) == 0 && records_fit &&
      (pow2 || (int64_t)f.max_pages_per_seq * f.page_tokens < (((int64_t)1 << 32) - 1) / f.page_tokens - 256)) {
    a.pt_inv = (uint32_t)((((uint64_t)1 << 32) + f.page_tokens - 1) / f.page_tokens);
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)f.head_dim);
    // float models have no buffer for partial results: theirs lie where the feed-forward product keeps its results (g, u, h), idle here
    const int64_t part_rows = bf16 ? c->map.attn_rows : (int64_t)((c->map.rope_cos - c->map.g) / 4) / (f.head_dim + 2);
    a.part_o = bf16 ? WSM(c, attn_part, float) : WSM(c, g, float);
    a.part_ml = a.part_o + part_rows * f.head_dim;
    const AttendPlan p = attend_plan(device_cus(), f.n_q_heads, f.n_kv_heads, g.B, g.Q, g.max_kv, a.window, a.n_sink, a.len4 != nullptr, bf16, part_rows);
    AttnPlan staged;
    a.n_parts = attn_win_parts(c, g, p, &staged);
    hipError_t e;
    if (a.n_parts > 0) {
      e = launch_attn_win(c, s, g, kv, staged, q, o, out_mt);
    } else {
      a.n_rg = p.n_rg; a.kspl = p.kspl; a.n_parts = p.n_parts;
      const unsigned grid = (unsigned)(((int64_t)g.B * f.n_kv_heads * p.n_parts + 7) / 8 * 8 * p.n_rg);
      const int threads = 64 * p.kspl;
      a.lds_q = p.kspl == 1 ? 0 : 4 * p.qt * 32 * 4 + (f.head_dim / 16) * p.qt * (p.kspl - 1) * 1024;   // (merging: statistics, sums)
      const size_t lds = a.lds_q + (a.len4 ? p.qt * (4 * 1024 + 256) : 0);
      if (!bf16) {
        if (f.head_dim == 128) k_attend_f32<128><<<grid, threads, lds, s>>>(a);
        else k_attend_f32<64><<<grid, threads, lds, s>>>(a);
      } else if (f.head_dim == 128) {
        if (p.qt == 1) k_attend<128, 1><<<grid, threads, lds, s>>>(a);
        else k_attend<128, 2><<<grid, threads, lds, s>>>(a);
      } else {
        if (p.qt == 1) k_attend<64, 1><<<grid, threads, lds, s>>>(a);
        else k_attend<64, 2><<<grid, threads, lds, s>>>(a);
      }
      e = hipGetLastError();
    }
    if (e != hipSuccess || a.n_parts == 1) return e;
    const int64_t rows = (int64_t)g.T * f.n_q_heads;
    const unsigned n = (unsigned)((rows + 1024 / f.head_dim - 1) / (1024 / f.head_dim));
    if (f.head_dim == 128) {
      if (bf16) k_attend_merge<bf16_t, 128><<<n, 256, 0, s>>>(a, rows);
      else k_attend_merge<float, 128><<<n, 256, 0, s>>>(a, rows);
    } else {
      if (bf16) k_attend_merge<bf16_t, 64><<<n, 256, 0, s>>>(a, rows);
      else k_attend_merge<float, 64><<<n, 256, 0, s>>>(a, rows);
    }
    return hipGetLastError();
  }
  if (f.dtype == DLLM_BF16) k_attend_any<bf16_t><<<dim3(g.T, f.n_q_heads), 256, 0, s>>>(a, f.head_dim);
  else k_attend_any<float><<<dim3(g.T, f.n_q_heads), 256, 0, s>>>(a, f.head_dim);
  return hipGetLastError();
}

}  // namespace dllm
