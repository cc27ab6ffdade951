// What the two attention kernels of the 8-bit cache share: arguments, units of work, how blocks' parts of a result are joined.
#pragma once
#include "gp_qcache.cuh"

constexpr int QT_WARPS = 4;
constexpr int QT_THREADS = QT_WARPS * 32;

// A sequence goes to the kernel for few rows (gp_qattn.cu) up to this many columns (row, query head of the group), beyond it to the one for many
// (gp_qprompt.cu), whose tiles have 256.  3000 tokens, 8 KV heads, us: d = 64, 16 sequences, with 32 / 48 / 64 columns 39 / 55 / 57 in the former, 60 in
// the latter (64 sequences: 103 / 179 / 187 and 177; one of 12 000 tokens: 29 and 34); d = 128 with 16 / 24 / 32 / 48 columns 38 / 52 / 75 / 78 and
// 68 / 69 / 70 / 71 (64 sequences: 95 / 139 / 246 / 256 and 202; one: 25 / 30 / 34 / 34 and 36).
constexpr int qt_few(int d) { return d == 64 ? 64 : 24; }

constexpr float QT_NONE = -3.3e38f;            // a maximum of nothing

// A part of a column's result: D sums of weighted values, m, the sum of weights l, e (and a word that nobody reads).  With logits s to base 2, weights are 2^(s - m) and the
// values' sums are held times 2^-e, so that no sum on the way passes what fp32 holds where the result does not: what is meant is 2^m l and 2^(m + e) o.
// e is a whole number.
__host__ __device__ constexpr int qt_part(int d) { return d + 4; }

struct QtArgs {
  const unsigned short* q;
  long long q_stride;
  int Hq, G, f16;
  const int* pages; int n_list;                // nullptr: all pages
  void* out; int out_type;
  int4* joins;                                 // [blocks][2] what qt_merge_kernel has to do
  float* part;                                 // [blocks][2][columns][qt_part(D)]
  int few;                                     // qt_few
  unsigned by_g;                               // qt_row
  int rows_tile;                               // rows whose columns (row, query head of the group) a thread block has together
  long long patience;                          // cycles after which a wait gives up
  int withhold;                                // gp_qcache_test_withhold
};
constexpr long long QT_PATIENCE = 1ll << 32;   // 2 s

__device__ __forceinline__ float qt_exp2(float x) {      // 2^x to 2^-22 relative; 0 below 2^-126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void qt_store(void* out, int type, size_t i, float x) {
  if (type == GP_TYPE_F32) static_cast<float*>(out)[i] = x;
  else if (type == GP_TYPE_F16) static_cast<__half*>(out)[i] = __float2half_rn(x);
  else static_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(x);
}

struct QtUnit {
  int seq, h, row0, rows, cols, slot0;         // of the tile: first batch row, rows, columns, slot of the first row
  int t0, t1;                                  // tokens of the stretch (with a list: places of the list times the page size)
  int total;                                   // granules of the unit, on the line behind QT_UNIT more
};
// the row of column `col` (of 256 at most) in its tile: col / G by a multiplication, exact for col * (G - 1) < 2^16
__device__ __forceinline__ int qt_row(const QtArgs& a, int col) { return (int)((unsigned)col * a.by_g >> 16); }
__host__ __device__ inline unsigned qt_by_g(int G) { return (65536u + G - 1) / G; }
// tokens that column `col` of a unit sees
__device__ __forceinline__ int qt_visible(const QcDev& c, const QtArgs& a, const QtUnit& u, int col) {
  return min(u.slot0 + qt_row(a, col) + 1, c.limit);
}
// where column `col`'s query, or result, lies: its number among the call's (row, query head)
__device__ __forceinline__ size_t qt_query(const QtArgs& a, const QtUnit& u, int col) {
  const int r = qt_row(a, col);
  return (size_t)(u.row0 + r) * a.Hq + u.h * a.G + (col - r * a.G);
}
// A warp per (block of the kernel before, column): joins the parts of the unit that ended in that block's stretch, if it began before.  (A block per
// column cost the kernel for many rows 38 000 blocks, nearly all without work.)
template <int D, int COLS, int SLOTS>      // SLOTS: partial results a block has room for
__global__ void __launch_bounds__(128)
qt_merge_kernel(const __grid_constant__ QtArgs a) {
  constexpr int ST = qt_part(D), PER = D / 64;               // pairs of elements a lane
  const int lane = threadIdx.x & 31, at = blockIdx.x * 4 + (threadIdx.x >> 5), col = at % COLS, b = at / COLS;
  gp_pdl_wait();
  const int4 j = __ldcg(a.joins + b * 2);              // columns, the first part, the next block, the last block
  if (col >= j.x) return;
  const int4 u = __ldcg(a.joins + b * 2 + 1);
  const int n_parts = j.w - j.z + 2;
  auto part = [&](int s) { return a.part + ((size_t)(s == 0 ? j.y : (j.z + s - 1) * SLOTS) * COLS + col) * ST; };
  float m = QT_NONE, top = -INFINITY, l = 0.f;         // of the parts so far; o is held times 2^-top beside 2^-m
  float2 o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = make_float2(0.f, 0.f);
  for (int s0 = 0; s0 < n_parts; s0 += 32) {           // 32 parts at a time
    float4 x = make_float4(QT_NONE, 0.f, 0.f, 0.f);
    if (s0 + lane < n_parts) x = __ldcg(reinterpret_cast<const float4*>(part(s0 + lane) + D));
    float mx = x.x;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
    const float to = fmaxf(m, mx), at = x.x - to + x.z;
    float tx = at;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) tx = fmaxf(tx, __shfl_xor_sync(0xffffffffu, tx, off));
    const float was = top + (m - to), now = fmaxf(was, tx), corr = exp2f(was - now);
    float add = exp2f(x.x - to) * x.y;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) add += __shfl_xor_sync(0xffffffffu, add, off);
    l = l * exp2f(m - to) + add;
    m = to; top = now;
    const float w = exp2f(at - now);
#pragma unroll
    for (int e = 0; e < PER; ++e) { o[e].x *= corr; o[e].y *= corr; }
    const int n = min(32, n_parts - s0);
#pragma unroll 8
    for (int s = 0; s < n; ++s) {
      const float ws = __shfl_sync(0xffffffffu, w, s);
      const float2* p = reinterpret_cast<const float2*>(part(s0 + s));
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const float2 y = __ldcg(p + e * 32 + lane);
        o[e].x += ws * y.x; o[e].y += ws * y.y;
      }
    }
  }
  const int row = qt_row(a, col);
  const size_t rh = ((size_t)(u.x + row) * a.Hq + u.y * a.G + (col - row * a.G)) * D;
  const float inv = l != 0.f ? 1.f / l : 0.f, scale = exp2f(top);      // (a NaN sum is not 0)
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const size_t i = rh + (e * 32 + lane) * 2;
    const float x = o[e].x * inv * scale, y = o[e].y * inv * scale;
    if (a.out_type == GP_TYPE_F32) *reinterpret_cast<float2*>(static_cast<float*>(a.out) + i) = make_float2(x, y);
    else *reinterpret_cast<uint32_t*>(static_cast<unsigned short*>(a.out) + i) = qc_pack(x, y, a.out_type == GP_TYPE_F16);
  }
}
