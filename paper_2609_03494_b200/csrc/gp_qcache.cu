// gp_qcache_append and gp_qcache_select: what goes into the 8-bit cache, and which of its pages a row looks at.
#include "gp_qcache.cuh"

namespace {

// ================================================================================================ append
struct QcRows {                // gp_qrows
  const unsigned short *k, *v, *q;
  unsigned short* q_out;
  long long k_stride, v_stride, q_stride, qo_stride;
  const int* positions;
  const float *qw, *kw;
  double eps;
  int Hq, f16, rope;
};
struct QcFreq { double over_pi[64]; };      // theta^(-2i/d) / pi: angles in units of pi

constexpr int QA_THREADS = 256;
constexpr int QA_WARPS = QA_THREADS / 32;
constexpr int QA_QROWS = 16;                   // rows whose queries a block takes

// A magnitude as an integer of the same order, as far as the exponent of a scale needs it: the high word of the double and whether anything follows
// (32 bits take one instruction to reduce over a warp).
__device__ __forceinline__ uint32_t qc_size(double x) { return (uint32_t)__double2hiint(x) * 2u + min((uint32_t)__double2loint(x), 1u); }
constexpr uint32_t QC_FAR64 = (1023u + 127u) << 21;             // size of 2^127: from here on fp32 may not hold the number
// the same of two 16-bit numbers in one register; QC_INF16: sizes that are not finite begin here
__device__ __forceinline__ uint32_t qc_sizes(uint32_t two) { return two & 0x7fff7fffu; }
template <bool F16> constexpr uint32_t QC_INF16 = F16 ? 0x7c00u : 0x7f80u;
// least e with amax <= 448 * 2^e = 0.875 * 2^(e + 9), from the exponent field over its bias and whether the mantissa is above 1.75
__device__ __forceinline__ int qc_exponent(uint32_t size, int exponent, bool above) {
  return size == 0 ? QC_E_MIN : min(max(exponent - 8 + (above ? 1 : 0), QC_E_MIN), QC_E_MAX);
}
__device__ __forceinline__ int qc_exponent64(uint32_t size) { return qc_exponent(size, (int)(size >> 21) - 1023, (size & 0x1fffff) > 0x180000); }
__device__ __forceinline__ int qc_exponent32(uint32_t size) { return qc_exponent(size, (int)(size >> 23) - 127, (size & 0x7fffff) > 0x600000); }
__device__ __forceinline__ int qc_scale_exponent(float s) {      // of a scale that is there; anything else is brought into the range
  return min(max((int)((__float_as_uint(s) >> 23) & 255) - 127, QC_E_MIN), QC_E_MAX);
}
__device__ __forceinline__ float pow2f(int e) {                  // 2^e, 0 below the normal numbers
  return e < -126 ? 0.f : __uint_as_float((uint32_t)(e + 127) << 23);
}
// 1 / sqrt(x) in fp64: Newton's iteration on y^-2 - x from the fp32 result, twice (2^-22, 2^-44, beyond fp64)
__device__ __forceinline__ double qc_rsqrt(double x) {
  const float f = (float)x;
  if (!(f > 1e-30f && f < 1e30f)) return 1.0 / sqrt(x);
  double y = rsqrtf(f);
  y = y * fma(-0.5 * x * y, y, 1.5);
  return y * fma(-0.5 * x * y, y, 1.5);
}
// eight 16-bit elements, two at a time
template <bool F16>
__device__ __forceinline__ void qc_elems8(const uint4& w, float* x) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) { const float2 t = qc_elems(v[e], F16); x[2 * e] = t.x; x[2 * e + 1] = t.y; }
}
// two fp32 numbers at a time
__device__ __forceinline__ uint64_t pack2(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpack2(uint64_t x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
// four numbers to e4m3, known to be finite
__device__ __forceinline__ uint32_t qc_codes_finite(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}

// Which sequence job `at` is of, where each has as many as `count` says, and its number there: false if there is none.  Every thread of the block adds up a
// run of sequences.
template <typename Count>
__device__ __forceinline__ bool qc_find(const QcDev& c, int at, Count count, int* seq, int* nth) {
  __shared__ int s_upto[QA_THREADS], s_warp[QA_WARPS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, run = (c.n_seq + QA_THREADS - 1) / QA_THREADS;
  int upto = 0;
  for (int s = tid * run; s < min((tid + 1) * run, c.n_seq); ++s) upto += count(qc_seq(c, s));
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  for (int w = 0; w < warp; ++w) upto += s_warp[w];
  s_upto[tid] = upto;
  __syncthreads();
  if (at >= s_upto[QA_THREADS - 1]) return false;
  int lo = 0, hi = QA_THREADS - 1;                    // the run: first with s_upto > at
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (s_upto[mid] > at) hi = mid;
    else lo = mid + 1;
  }
  int s = lo * run, before = lo ? s_upto[lo - 1] : 0;
  for (int n; at >= before + (n = count(qc_seq(c, s))); ++s) before += n;
  *seq = s; *nth = at - before;
  return true;
}
// pages that a sequence's rows touch; stretches of QA_QROWS rows that it has
__device__ __forceinline__ int qc_pages(const QcDev& c, const QcSeq& q) {
  const int first = max(q.slot0, 0), end = min(q.slot0 + q.rows, c.limit);
  return first < end ? ((end - 1) >> c.page_log) - (first >> c.page_log) + 1 : 0;
}
__device__ __forceinline__ int qc_stretches(const QcSeq& q) { return (q.rows + QA_QROWS - 1) / QA_QROWS; }

// Queries of up to 16 rows of a sequence, for a part of the heads.
template <int D, bool F16>
__device__ __forceinline__ void qc_append_queries(const QcDev& c, const QcRows& r, const QcFreq& freq, int at, int places, int groups, int heads_per, float2* tab) {
  constexpr int LPR = D / 16, RPW = 32 / LPR, HALF = D / 2;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lr = lane % LPR, sub = lane / LPR;
  const int q0 = at % groups * heads_per, q1 = min(q0 + heads_per, r.Hq); at /= groups;
  int place = at % max(places, 1), s = at / max(places, 1);
  if (places == 0 && !qc_find(c, at, [](const QcSeq& q) { return qc_stretches(q); }, &s, &place)) return;
  const QcSeq q = qc_seq(c, s);
  const int i0 = max(place * QA_QROWS, -q.slot0), i1 = min(min((place + 1) * QA_QROWS, q.rows), c.limit - q.slot0);      // rows that lie in a slot
  const int nt = i1 - i0;
  if (nt <= 0) return;
  const int row0 = q.r0 + i0, slot = q.slot0 + i0;
  if (r.rope) {
    for (int i = tid; i < nt * HALF; i += QA_THREADS) {
      const int t = i / HALF;
      const double g = (r.positions ? r.positions[row0 + t] : slot + t) * freq.over_pi[i % HALF];
      float sn, cs;
      sincospif((float)(g - 2.0 * rint(0.5 * g)), &sn, &cs);
      tab[t * HALF + i % 8 * LPR + i % HALF / 8] = make_float2(cs, sn);
    }
    __syncthreads();
  }
  const int per = max(1, QA_WARPS / nt);              // warps a token has
  float w0[8], w1[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) { w0[e] = r.qw ? r.qw[lr * 8 + e] : 1.f; w1[e] = r.qw ? r.qw[HALF + lr * 8 + e] : 1.f; }
  for (int t = warp / per; t < nt; t += QA_WARPS / per) {
    uint64_t ca[4], sa[4], cb[4], sb[4];              // first half = inv (ca x + sa y), second = inv (cb y + sb x), two at a time
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float2 i = make_float2(1.f, 0.f), j = i;
      if (r.rope) { i = tab[t * HALF + 2 * e * LPR + lr]; j = tab[t * HALF + (2 * e + 1) * LPR + lr]; }
      ca[e] = pack2(w0[2 * e] * i.x, w0[2 * e + 1] * j.x);
      sa[e] = pack2(-w1[2 * e] * i.y, -w1[2 * e + 1] * j.y);
      cb[e] = pack2(w1[2 * e] * i.x, w1[2 * e + 1] * j.x);
      sb[e] = pack2(w0[2 * e] * i.y, w0[2 * e + 1] * j.y);
    }
    const unsigned short* src = r.q + (size_t)(row0 + t) * r.q_stride + lr * 8;
    unsigned short* dst = r.q_out + (size_t)(row0 + t) * r.qo_stride + lr * 8;
    auto load = [&](int h, uint4* w) {
      w[0] = w[1] = make_uint4(0, 0, 0, 0);
      if (h < q1) {
        w[0] = *reinterpret_cast<const uint4*>(src + h * D);
        w[1] = *reinterpret_cast<const uint4*>(src + h * D + HALF);
      }
    };
    int h = q0 + warp % per * RPW + sub;
    uint4 now[2], then[2];
    load(h, now);
    for (; h - sub < q1; h += per * RPW) {
      load(h + per * RPW, then);
      float x[8], y[8], inv = 1.f;
      qc_elems8<F16>(now[0], x);
      qc_elems8<F16>(now[1], y);
      if (r.qw) {
        uint64_t ss = 0;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const uint64_t xx = pack2(x[e], x[e + 1]), yy = pack2(y[e], y[e + 1]);
          ss = fma2(xx, xx, ss);
          ss = fma2(yy, yy, ss);
        }
        float s0, s1;
        unpack2(ss, s0, s1);
        s0 += s1;
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
        inv = 1.f / sqrtf(s0 * (1.f / D) + (float)r.eps);
      }
      const uint64_t inv2 = pack2(inv, inv);
      uint32_t o0[4], o1[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint64_t xx = pack2(x[2 * e], x[2 * e + 1]), yy = pack2(y[2 * e], y[2 * e + 1]);
        float u0, u1, v0, v1;
        unpack2(mul2(inv2, fma2(ca[e], xx, mul2(sa[e], yy))), u0, u1);
        unpack2(mul2(inv2, fma2(cb[e], yy, mul2(sb[e], xx))), v0, v1);
        o0[e] = qc_pack(u0, u1, F16);
        o1[e] = qc_pack(v0, v1, F16);
      }
      if (h < q1) {
        *reinterpret_cast<uint4*>(dst + h * D) = make_uint4(o0[0], o0[1], o0[2], o0[3]);
        *reinterpret_cast<uint4*>(dst + h * D + HALF) = make_uint4(o1[0], o1[1], o1[2], o1[3]);
      }
      now[0] = then[0]; now[1] = then[1];
    }
  }
}

// A thread block takes the new rows of one page, for a part of the KV heads; the last blocks of the grid take queries.
//
// Keys and values: a team of TEAM warps takes a KV head at a time.  A row lies in D / 16 lanes (eight elements of its first half and eight of its
// second, so that a lane has both elements of the pairs it rotates), a team takes TEAM * 512 / D rows in a pass and keeps up to PASSES passes in
// registers until the largest magnitude of all of them is known.  Keys are computed in fp64: their largest magnitude decides an integer, and against a
// definition in 64 bits only 64 bits decide it alike.  The angles of the block's tokens are computed once for all heads (TABLE).  Values need no
// arithmetic before their maximum.
// Queries decide nothing: fp32, with angles reduced in fp64.  A warp takes a token and all of the block's query heads (where there are fewer tokens than
// warps, a part of them), with the weights and the angles multiplied out once: x' = inv (a x + b y).
// Measured (16 800 rows of seven prompts, 32 and 8 heads, d = 128, normalised and rotated): 101 us, of which queries 46 for 275 MB, at the copy rate, and keys and
// values 55 (37 with neither normalisation nor rotation), bound by their instructions, 39 an element.  256 single tokens, pages of 16 / 64 / 256: 9.9 / 12.0 /
// 27.8 us, one chain of loads and fp64 a block, and the keys that a page holds read for its bounds (2 / 8 / 33 MB).
template <int D, bool F16, int TEAM, int PASSES, bool TABLE>
__global__ void __launch_bounds__(QA_THREADS, PASSES == 1 ? 3 : PASSES == 2 ? 2 : 1)
qc_append_kernel(const __grid_constant__ QcDev c, const __grid_constant__ QcRows r, const __grid_constant__ QcFreq freq, int places, int groups, int heads_per,
                 int kv_blocks, int q_places, int q_groups, int q_heads_per) {
  constexpr int LPR = D / 16;                         // lanes per row
  constexpr int RPW = 32 / LPR;                       // rows of a warp in a pass
  constexpr int HALF = D / 2;
  constexpr int TEAMS = QA_WARPS / TEAM;
  extern __shared__ __align__(16) uint8_t qa_smem[];
  __shared__ uint32_t s_size[2][QA_WARPS];
  __shared__ uint32_t s_bnd[TEAM > 1 ? QA_WARPS : 1][2][TEAM > 1 ? HALF : 1];
  double2* tab = reinterpret_cast<double2*>(qa_smem); // [new rows][8][LPR] cos, sin of a lane's eighth e of the pairs: what lanes read together lies together
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lr = lane % LPR, sub = lane / LPR;
  if ((int)blockIdx.x >= kv_blocks) {
    qc_append_queries<D, F16>(c, r, freq, blockIdx.x - kv_blocks, q_places, q_groups, q_heads_per, reinterpret_cast<float2*>(qa_smem));
    return;
  }
  const int team = warp / TEAM, tw = warp % TEAM;
  int at = blockIdx.x;
  const int grp = at % groups; at /= groups;
  int place = at % max(places, 1), s = at / max(places, 1);
  if (places == 0 && !qc_find(c, at, [&](const QcSeq& q) { return qc_pages(c, q); }, &s, &place)) return;
  const QcSeq q = qc_seq(c, s);
  const int first = max(q.slot0, 0), end = min(q.slot0 + q.rows, c.limit);        // slots the batch fills
  const int lp = (first >> c.page_log) + place;
  const int a = max(first, lp << c.page_log), z = min(end, (lp + 1) << c.page_log);
  if (a >= z) return;
  const int nt = z - a, kept = a & (c.page - 1);      // new rows; rows the page holds already
  const int row0 = q.r0 + a - q.slot0;                // batch row of the first new one
  const int pid = qc_page(c, s, lp);
  if (pid < 0) return;
  auto team_sync = [&]() {
    if (TEAM == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(TEAM * 32) : "memory");
  };
  auto turns = [&](int t, int i) {                    // of token t's pair i, in units of pi
    const int p = r.positions ? r.positions[row0 + t] : a + t;
    return p * freq.over_pi[i];
  };
  const int h0 = grp * heads_per, h1 = min(h0 + heads_per, c.Hkv);
  auto h2 = [](uint32_t w) { return *reinterpret_cast<__half2*>(&w); };
  auto u2 = [](__half2 w) { return *reinterpret_cast<uint32_t*>(&w); };
  // a head's keys are asked for as soon as those of the head before have been taken over, its values as those of the one before have been written
  uint4 kraw[PASSES][2], vraw[PASSES][2];
  auto ask = [&](const unsigned short* from, long long stride, int h, uint4 (*raw)[2]) {
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
      const int t = (u * TEAM + tw) * RPW + sub;
      raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
      if (t < nt && h < h1) {
        const unsigned short* src = from + (size_t)(row0 + t) * stride + h * D + lr * 8;
        raw[u][0] = *reinterpret_cast<const uint4*>(src);
        raw[u][1] = *reinterpret_cast<const uint4*>(src + HALF);
      }
    }
  };
  ask(r.k, r.k_stride, h0 + team, kraw);
  ask(r.v, r.v_stride, h0 + team, vraw);
  if (TABLE && r.rope) {
    for (int i = tid; i < nt * HALF; i += QA_THREADS) {
      double2 cs;
      sincospi(turns(i / HALF, i % HALF), &cs.y, &cs.x);
      tab[i / HALF * HALF + i % 8 * LPR + i % HALF / 8] = cs;
    }
    __syncthreads();
  }
  for (int h = h0 + team; h < h1; h += TEAMS) {
    const size_t unit = (size_t)pid * c.Hkv + h;
    float2 old_scale = make_float2(1.f, 1.f);
    if (kept) {
      old_scale = *reinterpret_cast<const float2*>(c.scales + unit * 2);
      if (c.bounds)                                   // keys that are there already: wanted for the bounds, behind this head's arithmetic
        if (tw == 0 && lane == 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(c.codes + unit * 2 * c.page * D), "r"(kept * D) : "memory");
    }
    auto key_rows = [&](int u, int t, double* y) {    // a row's part, normalised and rotated
      float f[16];
      qc_elems8<F16>(kraw[u][0], f);
      qc_elems8<F16>(kraw[u][1], f + 8);
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = f[e];
      if (r.kw) {
        double s0 = 0.0, s1 = 0.0;
#pragma unroll
        for (int e = 0; e < 16; e += 2) { s0 = fma(y[e], y[e], s0); s1 = fma(y[e + 1], y[e + 1], s1); }
        s0 += s1;
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
        const double inv = qc_rsqrt(s0 * (1.0 / D) + r.eps);
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] *= inv * (double)r.kw[lr * 8 + (e & 7) + (e >> 3) * HALF];
      }
      if (r.rope && t < nt) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          double2 cs;
          if (TABLE) cs = tab[t * HALF + e * LPR + lr];
          else sincospi(turns(t, lr * 8 + e), &cs.y, &cs.x);
          const double p = y[e], m = y[e + 8];
          y[e] = p * cs.x - m * cs.y;
          y[e + 8] = m * cs.x + p * cs.y;
        }
      }
    };
    float x[PASSES][16];
    uint32_t ksize = 0, vsize = 0;
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        for (uint32_t w : {vraw[u][hf].x, vraw[u][hf].y, vraw[u][hf].z, vraw[u][hf].w}) vsize = __vmaxu2(vsize, qc_sizes(w));
      double y[16];
      key_rows(u, (u * TEAM + tw) * RPW + sub, y);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ksize = max(ksize, qc_size(y[e]));
        x[u][e] = (float)y[e];
      }
    }
    vsize = max(vsize & 0xffff, vsize >> 16);
    const bool odd = __any_sync(0xffffffffu, ksize >= QC_FAR64 || vsize >= QC_INF16<F16>);      // something may not be finite: all over, more carefully
    if (odd) {
      ksize = vsize = 0;
#pragma unroll
      for (int u = 0; u < PASSES; ++u) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
          for (uint32_t w : {vraw[u][hf].x, vraw[u][hf].y, vraw[u][hf].z, vraw[u][hf].w})
            for (uint32_t one : {qc_sizes(w) & 0xffff, qc_sizes(w) >> 16}) if (one < QC_INF16<F16>) vsize = max(vsize, one);
        double y[16];
        key_rows(u, (u * TEAM + tw) * RPW + sub, y);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float f = (float)y[e];
          if (fabs(y[e]) < INFINITY) {
            ksize = max(ksize, qc_size(y[e]));
            if (!(fabsf(f) < INFINITY)) f = copysignf(3.402823466e38f, f);      // finite in 64 bits, but not in 32: the largest that 32 hold
          }
          x[u][e] = f;
        }
      }
    }
    vsize = __float_as_uint(F16 ? __half2float(__ushort_as_half((unsigned short)vsize)) : __uint_as_float(vsize << 16));
    ask(r.k, r.k_stride, h + TEAMS, kraw);
    // the team's largest magnitudes
    ksize = __reduce_max_sync(0xffffffffu, ksize);
    vsize = __reduce_max_sync(0xffffffffu, vsize);
    if (TEAM > 1) {
      if (lane == 0) { s_size[0][warp] = ksize; s_size[1][warp] = vsize; }
      team_sync();
#pragma unroll
      for (int o = 0; o < TEAM; ++o) { ksize = max(ksize, s_size[0][team * TEAM + o]); vsize = max(vsize, s_size[1][team * TEAM + o]); }
      if (!c.bounds || kept) team_sync();             // (the words are written again, and rows may be rounded again, behind a meeting of the team)
    }
    int ek = qc_exponent64(ksize), ev = qc_exponent32(vsize);
    const int ek0 = qc_scale_exponent(old_scale.x), ev0 = qc_scale_exponent(old_scale.y);
    if (kept) { ek = max(ek, ek0); ev = max(ev, ev0); }
    uint8_t* kdst = c.codes + unit * 2 * c.page * D;
    uint8_t* vdst = kdst + (size_t)c.page * D;
    if (kept && (ek != ek0 || ev != ev0)) {           // rows that are there already, rounded to the new scale
      for (int i = tw * 32 + lane; i < 2 * kept * (D / 16); i += TEAM * 32) {
        const bool isv = i >= kept * (D / 16);
        const int by = isv ? ev0 - ev : ek0 - ek;
        if (by == 0) continue;
        uint4* p = reinterpret_cast<uint4*>(isv ? vdst : kdst) + (isv ? i - kept * (D / 16) : i);
        uint4 w = *p;
        const float m = pow2f(by);
        for (uint32_t* e : {&w.x, &w.y, &w.z, &w.w}) {
          const float2 lo = qc_half2(e4m3x2_to_f16x2(*e)), hi = qc_half2(e4m3x2_hi_to_f16x2(*e));
          *e = qc_codes(lo.x * m, lo.y * m, hi.x * m, hi.y * m);
        }
        *p = w;
      }
    }
    // codes of the new rows; bounds from the codes, as pairs of fp16
    const uint32_t PINF2 = 0x7c007c00u, NINF2 = 0xfc00fc00u;
    uint32_t lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { lo[e] = PINF2; hi[e] = NINF2; }
    auto bound = [&](int e, uint32_t w) {
      lo[e] = u2(__hmin2(h2(lo[e]), h2(w)));
      hi[e] = u2(__hmax2(h2(hi[e]), h2(w)));
    };
    auto numbers = [&](uint32_t w) { return w & __heq2_mask(h2(w), h2(w)); };      // NaN counts as 0
    if (c.bounds && kept) {                           // rows that are there already, from their codes: the old bounds may hold rows that were taken back since
      if (ek != ek0) team_sync();
#pragma unroll 4
      for (int t = tw * RPW + sub; t < kept; t += TEAM * RPW) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const uint2 w = *reinterpret_cast<const uint2*>(kdst + (size_t)t * D + lr * 8 + hf * HALF);
          bound(hf * 4, numbers(e4m3x2_to_f16x2(w.x))); bound(hf * 4 + 1, numbers(e4m3x2_hi_to_f16x2(w.x)));
          bound(hf * 4 + 2, numbers(e4m3x2_to_f16x2(w.y))); bound(hf * 4 + 3, numbers(e4m3x2_hi_to_f16x2(w.y)));
        }
      }
    }
    const float km = pow2f(-ek), vm = pow2f(-ev);
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
      const int t = (u * TEAM + tw) * RPW + sub;
      if (t < nt) {
        const size_t off = (size_t)(kept + t) * D + lr * 8;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float* y = x[u] + hf * 8;
          uint2 w;
          if (odd) {
            w.x = qc_codes(y[0] * km, y[1] * km, y[2] * km, y[3] * km);
            w.y = qc_codes(y[4] * km, y[5] * km, y[6] * km, y[7] * km);
          } else {
            w.x = qc_codes_finite(y[0] * km, y[1] * km, y[2] * km, y[3] * km);
            w.y = qc_codes_finite(y[4] * km, y[5] * km, y[6] * km, y[7] * km);
          }
          *reinterpret_cast<uint2*>(kdst + off + hf * HALF) = w;
          const uint32_t num[4] = {e4m3x2_to_f16x2(w.x), e4m3x2_hi_to_f16x2(w.x), e4m3x2_to_f16x2(w.y), e4m3x2_hi_to_f16x2(w.y)};
#pragma unroll
          for (int e = 0; e < 4; ++e) bound(hf * 4 + e, odd ? numbers(num[e]) : num[e]);
          float g[8];
          qc_elems8<F16>(vraw[u][hf], g);
          if (odd) {
            w.x = qc_codes(g[0] * vm, g[1] * vm, g[2] * vm, g[3] * vm);
            w.y = qc_codes(g[4] * vm, g[5] * vm, g[6] * vm, g[7] * vm);
          } else {
            w.x = qc_codes_finite(g[0] * vm, g[1] * vm, g[2] * vm, g[3] * vm);
            w.y = qc_codes_finite(g[4] * vm, g[5] * vm, g[6] * vm, g[7] * vm);
          }
          *reinterpret_cast<uint2*>(vdst + off + hf * HALF) = w;
        }
      }
    }
    ask(r.v, r.v_stride, h + TEAMS, vraw);
    if (tw == 0 && lane == 0) *reinterpret_cast<float2*>(c.scales + unit * 2) = make_float2(pow2f(ek), pow2f(ev));
    if (!c.bounds) continue;
#pragma unroll
    for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] = u2(__hmin2(h2(lo[e]), h2(__shfl_xor_sync(0xffffffffu, lo[e], o))));
        hi[e] = u2(__hmax2(h2(hi[e]), h2(__shfl_xor_sync(0xffffffffu, hi[e], o))));
      }
    if (TEAM > 1) {
      if (sub == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int pair = lr * 4 + (e & 3) + (e >> 2) * (HALF / 2);
          s_bnd[warp][0][pair] = lo[e];
          s_bnd[warp][1][pair] = hi[e];
        }
      }
      team_sync();
      if (tw == 0 && sub == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int pair = lr * 4 + (e & 3) + (e >> 2) * (HALF / 2);
#pragma unroll
          for (int o = 1; o < TEAM; ++o) {
            lo[e] = u2(__hmin2(h2(lo[e]), h2(s_bnd[team * TEAM + o][0][pair])));
            hi[e] = u2(__hmax2(h2(hi[e]), h2(s_bnd[team * TEAM + o][1][pair])));
          }
        }
      }
      team_sync();
    }
    if (tw == 0 && sub == 0) {
      uint8_t* b = c.bounds + unit * 2 * D + lr * 8;
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t w0 = side ? hi[hf * 4 + e * 2] : lo[hf * 4 + e * 2], w1 = side ? hi[hf * 4 + e * 2 + 1] : lo[hf * 4 + e * 2 + 1];
            reinterpret_cast<uint32_t*>(b + side * D + hf * HALF)[e] = f16x4_to_e4m3x4(w0, w1);
          }
    }
  }
}

// ================================================================================================ select
constexpr int QS_THREADS = 128;              // of a scoring block
constexpr int QS_SEL_THREADS = 256;
constexpr int QS_BITS = 9;                   // of a key that a step of the descent looks at
constexpr int QS_CAP = 8192;                 // scores of a unit that the selection keeps in shared memory
constexpr int QS_CLOSE = 256;                // pages close to the border that are ranked in shared memory
constexpr double QS_UP = 0x1p860, QS_DOWN = 0x1p156;      // QS_UP * QS_DOWN = 2^1016
constexpr float QS_ERR = 0x1p-14f * 448.f;   // error of a first score, of its scale times the sum of the weights' magnitudes (see there)

// The integers that come out of the selection are those of scores in fp64; but only near the border does it take fp64 to know on which side a page lies.
// So the tensor cores compute a first score with a bound on its error (a third of the time of fp64 throughout, which is bound by turning codes into
// doubles: 52 us for 48 rows over 1375 pages and 8 heads), and the selection takes pages in fp64 only where those bounds leave it open.

// sum of max(q, 0) and of min(q, 0) over the group, of one channel
__device__ __forceinline__ double2 qs_weights(const unsigned short* q, int G, int D, bool f16) {      // (low's, high's)
  double2 w = make_double2(0.0, 0.0);
  for (int g = 0; g < G; ++g) {
    const double x = qc_elem(q[(size_t)g * D], f16);
    w.y += fmax(x, 0.0); w.x += fmin(x, 0.0);
  }
  return w;
}

// First scores of `chunk` pages for one (row, KV head): both kinds of sums are one product of the page's 2 d codes with the weights
// [sum of min(q, 0), sum of max(q, 0)], whatever the group.  Pages are the rows of the products, codes fp16 (exact), the weights two columns: fp16, and
// what that leaves times 2^11.  A lane reads 16 codes of a page at a time; the weights are read in the order in which four lanes then have them.
// Error, with S the sum of magnitudes of all a page's terms (at most 448 times the scale times the weights' sum of magnitudes): a product adds 16 exact terms to
// an fp32 sum and may cut each of the 17 off at 2^-23 of the largest, so each of the 2 d / 16 <= 16 products is off by less than 17 * 2^-23 of S (the sum so far may be
// nearly all of S from the first product on), together by 2^-14.9 S.  The other column is off alike and counts 2^-11 of it; a weight in two parts is off by 2^-22 of
// itself, the last addition and multiplication by 2^-23 each.  QS_ERR, 2^-14, is nearly twice the sum of these.  Both numbers are kept times 2^-30 (and the weights' power
// of two), where fp32 holds them for every scale.
template <int D>
__global__ void __launch_bounds__(QS_THREADS)
qc_score_kernel(const __grid_constant__ QcDev c, const unsigned short* __restrict__ q, long long q_stride, int Hq, int f16, int keep, int first, int recent,
                float2* __restrict__ scores, int chunks, int chunk, int key_stride) {
  constexpr int LD = 2 * D / 64;                      // 16-byte pieces of a page that a lane reads
  constexpr int STEP = QS_THREADS / 32 * 16;          // pages of the block in a round
  __shared__ __align__(16) __half s_w[2][2 * D];
  __shared__ int s_seq;
  __shared__ float s_max[QS_THREADS / 32], s_sum[QS_THREADS / 32];
  const int part = blockIdx.x % chunks, unit = blockIdx.x / chunks, row = unit / c.Hkv, h = unit % c.Hkv, G = Hq / c.Hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = lane & 3;
  const int s = qc_seq_of_row(c, row, &s_seq);
  gp_pdl_launch_dependents();
  if (s < 0) return;
  const QcSeq sq = qc_seq(c, s);
  const int vis = min(sq.slot0 + row - sq.r0 + 1, c.limit);
  const int m = vis > 0 ? (vis + c.page - 1) >> c.page_log : 0;
  const int p0 = max(part * chunk, first), p1 = min((part + 1) * chunk, m - recent);
  if (m <= keep || p0 >= p1) return;
  const int* table = c.table + (size_t)s * c.stride;
  const size_t page_bytes = (size_t)c.Hkv * 2 * D;
  const uint8_t* src = c.bounds + (size_t)h * 2 * D + quad * 16;
  int p = p0 + warp * 16 + (lane >> 2);               // this lane's pages: p and p + 8
  auto id_of = [&](int at) {
    const int id = at < p1 ? table[at] : -1;
    return (unsigned)id < (unsigned)c.n_pages ? id : -1;
  };
  int id[2] = {id_of(p), id_of(p + 8)};
  // weights: thread i has channel i of both kinds
  float mx = 0.f, sum = 0.f;
  double2 w = make_double2(0.0, 0.0);
  if (tid < D) {
    w = qs_weights(q + (size_t)row * q_stride + (size_t)h * G * D + tid, G, D, f16 != 0);
    mx = fmaxf((float)-w.x, (float)w.y);
    sum = (float)(w.y - w.x);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
  }
  if (lane == 0) { s_max[warp] = mx; s_sum[warp] = sum; }
  __syncthreads();
  mx = 0.f; sum = 0.f;
#pragma unroll
  for (int i = 0; i < QS_THREADS / 32; ++i) { mx = fmaxf(mx, s_max[i]); sum += s_sum[i]; }
  const int up = min(14 - max((int)(__float_as_uint(mx) >> 23) - 127, -100), 114);      // 2^up brings the largest to 2^14 .. 2^15
  const double mul = __hiloint2double((1023 + up) << 20, 0);
  if (tid < D) {
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const double x = (side ? w.y : w.x) * mul;
      const __half hi = __float2half_rn((float)x);
      s_w[0][side * D + tid] = hi;
      s_w[1][side * D + tid] = __float2half_rn((float)((x - (double)__half2float(hi)) * 2048.0));
    }
  }
  const float err = sum * __uint_as_float((uint32_t)(127 + up) << 23) * QS_ERR;
  uint4 x[2][LD];
  float sc[2];
  auto fetch = [&](const int* of) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint8_t* from = src + (size_t)max(of[k], 0) * page_bytes;
#pragma unroll
      for (int i = 0; i < LD; ++i) x[k][i] = *reinterpret_cast<const uint4*>(from + i * 64);
      sc[k] = of[k] >= 0 ? c.scales[((size_t)of[k] * c.Hkv + h) * 2] : -1.f;
    }
  };
  fetch(id);
  int next[2] = {id_of(p + STEP), id_of(p + STEP + 8)};
  __syncthreads();
  uint32_t b[LD * 4][2];                              // column lane / 4: the weights, what they leave, nothing
#pragma unroll
  for (int i = 0; i < LD * 4; ++i) {
    b[i][0] = b[i][1] = 0;
    if (lane < 8) {
      const uint2 v = *reinterpret_cast<const uint2*>(&s_w[lane >> 2][(i >> 2) * 64 + quad * 16 + (i & 3) * 4]);
      b[i][0] = v.x; b[i][1] = v.y;
    }
  }
  for (; p - (lane >> 2) < p1; p += STEP) {
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const uint32_t r0[4] = {x[0][i].x, x[0][i].y, x[0][i].z, x[0][i].w}, r1[4] = {x[1][i].x, x[1][i].y, x[1][i].z, x[1][i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        mma_f16(acc, e4m3x2_to_f16x2(r0[e]), e4m3x2_to_f16x2(r1[e]), e4m3x2_hi_to_f16x2(r0[e]), e4m3x2_hi_to_f16x2(r1[e]), b[i * 4 + e][0], b[i * 4 + e][1]);
    }
    const float s0 = sc[0], s1 = sc[1];
    const int at = p;
    fetch(next);
    next[0] = id_of(p + 2 * STEP); next[1] = id_of(p + 2 * STEP + 8);
    if (quad == 0) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int pg = at + 8 * k;
        if (pg >= p1) continue;
        const float scale = (k ? s1 : s0) * 0x1p-30f;
        if (scale < 0.f && c.status) atomicOr(c.status, GP_E_BOUNDS);
        // (a page that is not there: below everything, and known to be)
        scores[(size_t)unit * key_stride + pg] = scale < 0.f ? make_float2(-INFINITY, 0.f)
                                                             : make_float2(fmaf(acc[2 * k + 1], 0x1p-11f, acc[2 * k]) * scale, fmaxf(err * scale, 1e-36f));
      }
    }
  }
}

// a score as an integer of the same order; what is not a number is lowest
__device__ __forceinline__ unsigned long long qc_key(double x) {
  if (!(x == x)) return 0ull;
  const unsigned long long b = (unsigned long long)__double_as_longlong(x + 0.0);
  return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t qc_key(float x) {      // (as minus infinity)
  if (!(x == x)) return 0x007fffffu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float qc_unkey(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

struct QsShared {
  int hist[1 << QS_BITS];
  int seq, bin, left, count, page[QS_CLOSE];
  unsigned long long lo[QS_SEL_THREADS / 32], hi[QS_SEL_THREADS / 32], sum[QS_SEL_THREADS / 32], key[QS_CLOSE];
  float err[QS_SEL_THREADS / 32];
};
// What the threads before this one have of a sum, and what all have.
__device__ __forceinline__ unsigned long long qs_scan(QsShared& sh, unsigned long long mine, unsigned long long* all = nullptr) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  unsigned long long upto = mine, total = 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  __syncthreads();
  if (lane == 31) sh.sum[warp] = upto;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QS_SEL_THREADS / 32; ++w) {
    if (w < warp) upto += sh.sum[w];
    total += sh.sum[w];
  }
  if (all) *all = total;
  return upto - mine;
}
// The want-th highest of n keys (1 <= want <= n): a radix descent from the first bit in which they differ, 9 bits at a time (11, with 2048 bins to
// clear and scan: 45.6 us a call of 48 rows against 43.5).  *thr: its known bits, *known:
// which those are, returns how many of the keys equal to it there are wanted.  hist is zero before and after.
template <typename K, typename Get>
__device__ __forceinline__ int qs_descend(QsShared& sh, int n, int want, Get get, K* thr_out, K* known_out) {
  constexpr int BINS = 1 << QS_BITS, PER = BINS / QS_SEL_THREADS, W = sizeof(K) * 8;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  K lo = ~(K)0, hi = 0;
  for (int i = tid; i < n; i += QS_SEL_THREADS) {
    const K k = get(i);
    lo = min(lo, k); hi = max(hi, k);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  __syncthreads();
  if (lane == 0) { sh.lo[warp] = lo; sh.hi[warp] = hi; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QS_SEL_THREADS / 32; ++w) { lo = min(lo, (K)sh.lo[w]); hi = max(hi, (K)sh.hi[w]); }
  K thr = lo, known = ~(K)0;
  int left = want;
  const K diff = lo ^ hi;
  if (diff) {
    int top = 64 - __clzll((unsigned long long)diff);      // bits below this one differ
    known = top == W ? (K)0 : (K)(~(K)0 << top);
    thr = hi & known;
    while (top > 0) {
      const int bits = min(QS_BITS, top), sh2 = top - bits;
      for (int i = tid; i < n; i += QS_SEL_THREADS) {
        const K x = get(i);
        if ((x & known) == thr) atomicAdd(&sh.hist[(int)(x >> sh2) & ((1 << bits) - 1)], 1);
      }
      __syncthreads();
      int cnt[PER], sum = 0;                          // bins from above
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        cnt[e] = sh.hist[BINS - 1 - (tid * PER + e)];
        sum += cnt[e];
      }
      int before = (int)qs_scan(sh, (unsigned long long)sum);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int b = BINS - 1 - (tid * PER + e);
        if (before < left && before + cnt[e] >= left) { sh.bin = b; sh.left = left - before; sh.count = cnt[e]; }
        before += cnt[e];
        sh.hist[b] = 0;
      }
      __syncthreads();
      thr |= (K)sh.bin << sh2;
      known |= (K)((1 << bits) - 1) << sh2;
      left = sh.left;
      top = sh2;
      if (sh.count == left) break;                    // the whole bin is wanted
    }
  }
  *thr_out = thr; *known_out = known;
  return left;
}

// One block per (row, KV head): the pages whose first score is above the border by more than the errors, and as many of those closer to it as are
// wanted, by their scores in fp64; in ascending order (a thread takes a run of pages, one scan says where each run's go).
template <int D>
__global__ void __launch_bounds__(QS_SEL_THREADS)
qc_select_kernel(const __grid_constant__ QcDev c, const unsigned short* __restrict__ q, long long q_stride, int Hq, int f16, int keep, int first, int recent,
                 float2* scores, int key_stride, int* __restrict__ pages) {
  extern __shared__ uint32_t s_key[];
  __shared__ QsShared sh;
  __shared__ __align__(16) double s_w[2 * D];
  const int unit = blockIdx.x, row = unit / c.Hkv, h = unit % c.Hkv, G = Hq / c.Hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int s = qc_seq_of_row(c, row, &sh.seq);
  gp_pdl_launch_dependents();
  if (s < 0) { gp_pdl_wait(); return; }
  const QcSeq sq = qc_seq(c, s);
  const int vis = min(sq.slot0 + row - sq.r0 + 1, c.limit);
  const int m = vis > 0 ? (vis + c.page - 1) >> c.page_log : 0;
  int* out = pages + (size_t)unit * keep;
  if (m <= keep) {
    for (int i = tid; i < keep; i += QS_SEL_THREADS) out[i] = i < m ? i : -1;
    gp_pdl_wait();                                    // no block ends before the kernel in front of it
    return;
  }
  for (int i = tid; i < first; i += QS_SEL_THREADS) out[i] = i;
  for (int i = tid; i < recent; i += QS_SEL_THREADS) out[keep - recent + i] = m - recent + i;
  const int want = keep - first - recent, n = m - first - recent;        // want < n
  for (int i = tid; i < 1 << QS_BITS; i += QS_SEL_THREADS) sh.hist[i] = 0;
  gp_pdl_wait();
  if (want == 0) return;
  float2* src = scores + (size_t)unit * key_stride + first;
  const bool near = n <= QS_CAP;
  float err = 0.f;
  for (int i = tid; i < n; i += QS_SEL_THREADS) {
    const float2 x = __ldcg(src + i);
    if (near) s_key[i] = qc_key(x.x);
    err = fmaxf(err, x.y);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) err = fmaxf(err, __shfl_xor_sync(0xffffffffu, err, o));
  if (lane == 0) sh.err[warp] = err;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QS_SEL_THREADS / 32; ++w) err = fmaxf(err, sh.err[w]);
  auto key = [&](int i) { return near ? s_key[i] : qc_key(__ldcg(src + i).x); };
  uint32_t thr, known;
  int left = qs_descend<uint32_t>(sh, n, want, key, &thr, &known);
  // The want-th highest first score lies between the least and the greatest key with these bits; a page further than two errors from there is decided.
  const float far = 2.0001f * err;
  // (All keys lie between those of the two infinities.)  above: certain, below: certainly not.  Where a bound on the errors is not finite (the weights of a group's
  // queries may pass what fp32 holds, and queries may be infinite) the first scores say nothing: all pages are close.
  const bool told = far < INFINITY;
  const uint32_t above = told ? qc_key(qc_unkey(min(thr | ~known, 0xff800000u)) + far) : ~0u, below = told ? qc_key(qc_unkey(max(thr, 0x007fffffu)) - far) : 0u;
  const int run = (n + QS_SEL_THREADS - 1) / QS_SEL_THREADS, i0 = min(tid * run, n), i1 = min(i0 + run, n);
  int gt = 0, eq = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t x = key(i);
    gt += x > above; eq += x <= above && x >= below;
  }
  unsigned long long all, ahead = qs_scan(sh, (unsigned long long)gt << 32 | (unsigned)eq, &all);
  const int close = (int)(unsigned)all;
  left = want - (int)(all >> 32);                     // pages wanted of the close ones
  if (close == left) {                                // all of them
    int at = first + (int)(ahead >> 32) + (int)(unsigned)ahead;
    for (int i = i0; i < i1; ++i)
      if (key(i) >= below) out[at++] = first + i;
    return;
  }
  for (int i = tid; i < D; i += QS_SEL_THREADS) {
    const double2 w = qs_weights(q + (size_t)row * q_stride + (size_t)h * G * D + i, G, D, f16 != 0);
    s_w[i] = w.x * QS_UP;
    s_w[i + D] = w.y * QS_UP;
  }
  // a page's score in fp64, by a warp.  A code's sign and its seven other bits, put where a double has its sign and the low end of its exponent, are that
  // number times 2^-1016 (codes without an exponent included: a subnormal double)
  auto exact = [&](int page) {
    const int id = c.table[(size_t)s * c.stride + page];
    if ((unsigned)id >= (unsigned)c.n_pages) return 0ull;
    const size_t u = (size_t)id * c.Hkv + h;
    const uint32_t* b = reinterpret_cast<const uint32_t*>(c.bounds + u * 2 * D);
    double acc = 0.0;
#pragma unroll
    for (int i = 0; i < 2 * D / 128; ++i) {
      const uint32_t word = b[i * 32 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc = fma(__hiloint2double(((int)(word << (24 - 8 * e)) >> 7) & 0x80fe0000, 0), s_w[(i * 32 + lane) * 4 + e], acc);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    return qc_key(acc * QS_DOWN * (double)c.scales[u * 2]);
  };
  if (close <= QS_CLOSE) {
    int at = (int)(unsigned)ahead;                    // the close pages, in their order
    for (int i = i0; i < i1; ++i) {
      const uint32_t x = key(i);
      if (x <= above && x >= below) sh.page[at++] = i;
    }
    __syncthreads();
    for (int i = warp; i < close; i += QS_SEL_THREADS / 32) {
      const unsigned long long k = exact(first + sh.page[i]);
      if (lane == 0) sh.key[i] = k;
    }
    __syncthreads();
    bool taken = false;
    if (tid < close) {                                // one that fewer than `left` are ahead of
      const unsigned long long mine = sh.key[tid];
      int better = 0;
      for (int i = 0; i < close; ++i) better += sh.key[i] > mine || (sh.key[i] == mine && i < tid);
      taken = better < left;
    }
    __syncthreads();
    if (tid < close) sh.key[tid] = taken;
    __syncthreads();
    // places: certain pages and taken ones before this thread's run
    int mine = 0, nth = (int)(unsigned)ahead;
    for (int i = nth; i < nth + eq; ++i) mine += (int)sh.key[i];
    at = first + (int)(ahead >> 32) + (int)qs_scan(sh, (unsigned long long)mine);
    for (int i = i0; i < i1; ++i) {
      const uint32_t x = key(i);
      if (x > above) out[at++] = first + i;
      else if (x >= below && sh.key[nth++]) out[at++] = first + i;
    }
    return;
  }
  // many close pages (equal ones, or one of a scale far above the others'): 64-bit keys in the scores' place, all ones for the certain pages
  unsigned long long* keys = reinterpret_cast<unsigned long long*>(src);
  __syncthreads();
  for (int i = warp; i < n; i += QS_SEL_THREADS / 32) {
    const uint32_t x = key(i);
    unsigned long long k = x > above ? ~0ull : 0ull;
    if (x <= above && x >= below) k = max(exact(first + i), 1ull);
    __syncwarp();
    if (lane == 0) __stcg(keys + i, k);
  }
  __threadfence_block();
  __syncthreads();
  auto key64 = [&](int i) { return __ldcg(keys + i); };
  unsigned long long thr64, known64;
  left = qs_descend<unsigned long long>(sh, n, want, key64, &thr64, &known64);
  gt = eq = 0;
  for (int i = i0; i < i1; ++i) {
    const unsigned long long x = key64(i) & known64;
    gt += x > thr64; eq += x == thr64;
  }
  ahead = qs_scan(sh, (unsigned long long)gt << 32 | (unsigned)eq);
  int eqs = (int)(unsigned)ahead, at = first + (int)(ahead >> 32) + min(eqs, left);
  for (int i = i0; i < i1; ++i) {
    const unsigned long long x = key64(i) & known64;
    if (x > thr64) out[at++] = first + i;
    else if (x == thr64 && eqs++ < left) out[at++] = first + i;
  }
}

template <int D>
struct QcAppendPlan {
  using K = void (*)(const QcDev, const QcRows, const QcFreq, int, int, int, int, int, int, int);
  K kern;
  int teams, table_rows;
};
// By the new rows a page can receive: few (single tokens, short drafts) leave a warp a head to itself, so that a block's eight warps take
// eight heads at once; up to 16 or 32 rows four warps; beyond that all eight warps share a head.  Above 64 rows a table of angles does not fit
// beside others on an SM; each lane then computes its own.
template <int D, bool F16>
QcAppendPlan<D> qc_append_plan(int rows) {
  constexpr int RPW = 512 / D;
  if (rows <= RPW) return {qc_append_kernel<D, F16, 1, 1, true>, 8, RPW};
  if (rows <= 4 * RPW) return {qc_append_kernel<D, F16, 4, 1, true>, 2, 4 * RPW};
  if (rows <= 64) return {qc_append_kernel<D, F16, 8, 8 / RPW, true>, 1, 64};
  if (rows <= 128) return {qc_append_kernel<D, F16, 8, 16 / RPW, false>, 1, 0};
  return {qc_append_kernel<D, F16, 8, 32 / RPW, false>, 1, 0};
}

template <int D>
int qc_append(const QcDev& c, const QcRows& r, const QcFreq& f, cudaStream_t s) {
  const int rows = c.page < c.max_rows ? c.page : c.max_rows;
  const QcAppendPlan<D> plan = r.f16 ? qc_append_plan<D, true>(rows) : qc_append_plan<D, false>(rows);
  // Jobs: pages that max_rows new tokens can touch, for every sequence; where that is far more than all the rows together can (one long chunk among single
  // tokens), as many as they can, and a block looks for its own (256 sequences, one of 2048 rows: 36 us; 110 with a block for every page and sequence)
  long long places = ((long long)c.max_rows + c.page - 2) / c.page + 1, q_places = ((long long)c.max_rows + QA_QROWS - 1) / QA_QROWS;
  long long jobs = places * c.n_seq, q_jobs = q_places * c.n_seq;
  const long long most = (long long)c.n_rows / c.page + 2 * (long long)c.n_seq, q_most = (long long)c.n_rows / QA_QROWS + c.n_seq;
  if (jobs > 4 * most) { jobs = most; places = 0; }
  if (q_jobs > 4 * q_most) { q_jobs = q_most; q_places = 0; }
  if (!r.q) q_jobs = 0;
  // heads of a page together share the table of angles and keep a block's warps busy; apart where that leaves SMs without a block (256 single tokens, 8
  // heads, pages of 16: 9.9 us; 12.1 with two blocks an SM, i.e. four heads a block)
  int heads_per = c.Hkv;
  while (heads_per > 1 && jobs * ((c.Hkv + heads_per - 1) / heads_per) < 148) heads_per = (heads_per + 1) / 2;
  const int groups = (c.Hkv + heads_per - 1) / heads_per;
  const long long kv = jobs * groups;
  int q_heads = r.Hq;
  while (q_heads > 512 / D && q_jobs * ((r.Hq + q_heads - 1) / q_heads) < 296) q_heads = (q_heads + 1) / 2;
  const int q_groups = r.q ? (r.Hq + q_heads - 1) / q_heads : 1;
  const long long qb = q_jobs * q_groups;
  if (kv + qb > 0x7fffffff) return GP_ERR_INVALID;
  size_t smem = r.rope ? (size_t)plan.table_rows * (D / 2) * sizeof(double2) : 0;
  const size_t q_smem = r.rope && r.q ? (size_t)(c.max_rows < QA_QROWS ? c.max_rows : QA_QROWS) * (D / 2) * sizeof(float2) : 0;
  if (q_smem > smem) smem = q_smem;
  if (smem > 32 * 1024 && cudaFuncSetAttribute(plan.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return GP_ERR_CUDA;
  plan.kern<<<(unsigned)(kv + qb), QA_THREADS, smem, s>>>(c, r, f, (int)places, groups, heads_per, (int)kv, (int)q_places, q_groups, q_heads);
  return cudaGetLastError() == cudaSuccess ? GP_OK : GP_ERR_CUDA;
}

}  // namespace

extern "C" int gp_qcache_append(const gp_qcache* cache, const gp_qbatch* batch, const gp_qrows* rows, void* stream) {
  QcDev c;
  const int st = qc_check(cache, batch, &c);
  if (st != GP_OK) return st;
  if (!rows || (!qc_empty(c) && (!rows->k || !rows->v)) || (rows->type != GP_TYPE_BF16 && rows->type != GP_TYPE_F16)) return GP_ERR_INVALID;
  const int64_t need = (int64_t)c.Hkv * cache->head_dim;
  if (qc_misaligned(rows->k, 16) || qc_misaligned(rows->v, 16) || rows->k_stride < need || rows->v_stride < need || rows->k_stride % 8 || rows->v_stride % 8)
    return GP_ERR_INVALID;
  if (qc_misaligned(rows->positions, 4) || qc_misaligned(rows->q_weight, 4) || qc_misaligned(rows->k_weight, 4)) return GP_ERR_INVALID;
  if (!(rows->eps >= 0.0) || !(rows->rope_theta >= 0.0) || isinf(rows->eps) || isinf(rows->rope_theta)) return GP_ERR_INVALID;
  if (rows->q) {
    if (!qc_check_q(cache, rows->q, rows->q_stride, rows->n_q_heads, rows->type)) return GP_ERR_INVALID;
    if (!rows->q_out || qc_misaligned(rows->q_out, 16) || rows->q_out_stride < (int64_t)rows->n_q_heads * cache->head_dim || rows->q_out_stride % 8)
      return GP_ERR_INVALID;
    if (rows->q_out == rows->q && rows->q_out_stride != rows->q_stride) return GP_ERR_INVALID;
  }
  if (qc_empty(c)) return GP_OK;
  QcRows r;
  r.k = static_cast<const unsigned short*>(rows->k); r.v = static_cast<const unsigned short*>(rows->v);
  r.q = static_cast<const unsigned short*>(rows->q); r.q_out = static_cast<unsigned short*>(rows->q_out);
  r.k_stride = rows->k_stride; r.v_stride = rows->v_stride; r.q_stride = rows->q_stride; r.qo_stride = rows->q_out_stride;
  r.positions = rows->positions;
  r.qw = rows->q_weight; r.kw = rows->k_weight;
  r.eps = rows->eps;
  r.Hq = rows->n_q_heads;
  r.f16 = rows->type == GP_TYPE_F16;
  r.rope = rows->rope_theta > 0.0;
  const int half = cache->head_dim / 2;
  static thread_local struct { QcFreq f; double theta; int half; } last = {};      // 64 powers take 2 us: kept for the next call with this base
  if (r.rope && (last.theta != rows->rope_theta || last.half != half)) {
    for (int i = 0; i < 64; ++i) last.f.over_pi[i] = i < half ? pow(rows->rope_theta, -(double)i / half) / M_PI : 0.0;
    last.theta = rows->rope_theta; last.half = half;
  }
  const QcFreq& f = last.f;
  QcDevice dev(cache->device);
  if (!dev.ok) return GP_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return cache->head_dim == 128 ? qc_append<128>(c, r, f, s) : qc_append<64>(c, r, f, s);
}

extern "C" size_t gp_qcache_select_bytes(const gp_qcache* cache, const gp_qbatch* batch) {
  QcDev c;
  if (qc_check(cache, batch, &c) != GP_OK || qc_empty(c)) return 0;
  return (size_t)c.n_rows * c.Hkv * (((size_t)c.limit + c.page - 1) / c.page) * 8;
}

extern "C" int gp_qcache_select(const gp_qcache* cache, const gp_qbatch* batch, const void* q, int64_t q_stride, int32_t n_q_heads, int32_t type,
                                int32_t keep, int32_t first, int32_t recent, int32_t* pages, void* work, size_t work_bytes, void* stream) {
  QcDev c;
  const int st = qc_check(cache, batch, &c);
  if (st != GP_OK) return st;
  if (!qc_check_q(cache, q, q_stride, n_q_heads, type) || !cache->bounds) return GP_ERR_INVALID;
  if (keep < 1 || first < 0 || recent < 1 || (int64_t)first + recent > keep || (!qc_empty(c) && (!q || !pages)) || qc_misaligned(pages, 4)) return GP_ERR_INVALID;
  const size_t need = gp_qcache_select_bytes(cache, batch);
  if (need && (!work || qc_misaligned(work, 16) || work_bytes < need)) return GP_ERR_INVALID;
  if (qc_empty(c)) return GP_OK;
  const long long units = (long long)c.n_rows * c.Hkv;
  const int stride = (int)(((long long)c.limit + c.page - 1) / c.page);
  // a block prepares its weights for as many pages as leave the GPU two rounds of blocks (eight an SM), 128 at least
  long long chunk = ((long long)stride * units / (2 * 148 * 8) + 127) / 128 * 128;
  if (chunk < 128) chunk = 128;
  const long long chunks = stride > keep ? (stride + chunk - 1) / chunk : 0;
  if (units * (chunks ? chunks : 1) > 0x7fffffff) return GP_ERR_INVALID;
  QcDevice dev(cache->device);
  if (!dev.ok) return GP_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  float2* scores = static_cast<float2*>(work);
  const unsigned short* qp = static_cast<const unsigned short*>(q);
  const int f16 = type == GP_TYPE_F16;
  if (chunks) {
    auto score = cache->head_dim == 128 ? qc_score_kernel<128> : qc_score_kernel<64>;
    score<<<(unsigned)(units * chunks), QS_THREADS, 0, s>>>(c, qp, q_stride, n_q_heads, f16, keep, first, recent, scores, (int)chunks, (int)chunk, stride);
    if (cudaGetLastError() != cudaSuccess) return GP_ERR_CUDA;
  }
  auto select = cache->head_dim == 128 ? qc_select_kernel<128> : qc_select_kernel<64>;
  const size_t smem = (size_t)(stride < QS_CAP ? stride : QS_CAP) * 4;
  if (smem > 16 * 1024 && cudaFuncSetAttribute(select, cudaFuncAttributeMaxDynamicSharedMemorySize, QS_CAP * 4) != cudaSuccess) return GP_ERR_CUDA;
  return gp_launch(select, (int)units, QS_SEL_THREADS, smem, s, chunks > 0, c, qp, (long long)q_stride, (int)n_q_heads, f16, (int)keep, (int)first, (int)recent, scores,
                   stride, static_cast<int*>(pages)) == cudaSuccess ? GP_OK : GP_ERR_CUDA;
}
