// gp_qcache_attention: attention of a packed batch's rows over the 8-bit cache, over all pages or over a list of them per row and KV head.
#include "gp_qcache.cuh"

namespace {

constexpr int QT_WARPS = 4;
constexpr int QT_THREADS = QT_WARPS * 32;
constexpr int QT_STAGES = 4;                   // stages of a warp's ring
constexpr int QT_STAGE_BYTES = 4096;           // keys and values of 16 tokens of 128 elements, of 32 of 64
constexpr int QT_CTAS = 888;                   // thread blocks a launch is cut into where there is that much work
constexpr int QT_MIN_SPLIT = 256;              // tokens of the longest sequence below which splits are not cut further
constexpr float QT_LIFT = 15.f;                // weights are carried times 2^15, where fp16 reaches 2^-39 of the largest

struct QtArgs {
  const unsigned short* q;
  long long q_stride;
  int Hq, G, f16;
  const int* pages; int n_list;                // nullptr: all pages
  void* out; int out_type;
  float* part;                                 // [n_rows * Hq][n_split][D + 2], n_split > 1
  int n_split, col_tiles;                      // col_tiles: tiles of columns (row, head) that max_rows rows have
};

// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col)
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t qt_transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void qt_cp_async16(uint32_t dst_smem, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst_smem), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void qt_store(void* out, int type, size_t i, float x) {
  if (type == GP_TYPE_F32) static_cast<float*>(out)[i] = x;
  else if (type == GP_TYPE_F16) static_cast<__half*>(out)[i] = __float2half_rn(x);
  else static_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(x);
}

// One unit of work: the columns (row, query head of the group) of one KV head that a thread block has together, and the tokens of its split.
struct QtUnit {
  int seq, h, row0, cols, col0;                // batch row of the sequence's first; columns; number of the first one
  int slot0;                                   // slot of the sequence's first row
  int t0, t1;                                  // tokens of the split (with a list: places of the list times the page size)
};
// tokens that column `col` of a unit sees
__device__ __forceinline__ int qt_visible(const QcDev& c, const QtUnit& u, int G, int col) {
  return min(u.slot0 + (u.col0 + col) / G + 1, c.limit);
}

// The unit's result, or its split's partial one, from its warps' (warps x columns x (D + 2) floats in shared memory).
template <int D>
__device__ __forceinline__ void qt_write(const QtArgs& a, const QtUnit& u, int split, const float* s_part, int warps, int cols_stride) {
  constexpr int ST = D + 2;
  for (int i = threadIdx.x; i < u.cols * D; i += QT_THREADS) {
    const int col = i / D, e = i % D;
    float M = -INFINITY;
    for (int w = 0; w < warps; ++w) M = fmaxf(M, s_part[(size_t)(w * cols_stride + col) * ST + D]);
    float o = 0.f, l = 0.f;
    for (int w = 0; w < warps; ++w) {
      const float* p = s_part + (size_t)(w * cols_stride + col) * ST;
      const float wt = M == -INFINITY ? 0.f : exp2f(p[D] - M);
      o += wt * p[e];
      l += wt * p[D + 1];
    }
    const int cc = u.col0 + col;
    const size_t rh = (size_t)(u.row0 + cc / a.G) * a.Hq + u.h * a.G + cc % a.G;
    if (a.n_split == 1) {
      qt_store(a.out, a.out_type, rh * D + e, l != 0.f ? o / l : 0.f);      // (a NaN sum is not 0)
    } else {
      float* dst = a.part + (rh * a.n_split + split) * ST;
      dst[e] = o;
      if (e == 0) { dst[D] = M; dst[D + 1] = l; }
    }
  }
}

// The unit in plain arithmetic, a warp a token and column after column: for a result that is not finite where rows see different tokens (a
// NaN value that one row sees must not reach another through a weight of zero).
template <int D>
__device__ __noinline__ void qt_plain(const QcDev& c, const QtArgs& a, const QtUnit& u, int split, float* smem) {
  constexpr int PER = D / 32, ST = D + 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float scale = 1.4426950408889634f * rsqrtf((float)D);
  for (int col = 0; col < u.cols; ++col) {
    const int cc = u.col0 + col, row = u.row0 + cc / a.G, head = u.h * a.G + cc % a.G, vis = qt_visible(c, u, a.G, col);
    float q[PER], o[PER], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) { q[e] = qc_elem(a.q[(size_t)row * a.q_stride + (size_t)head * D + lane + 32 * e], a.f16); o[e] = 0.f; }
    for (int t = u.t0 + warp; t < min(u.t1, vis); t += QT_WARPS) {
      const int id = qc_page(c, u.seq, t >> c.page_log);
      if (id < 0) continue;
      const size_t unit = (size_t)id * c.Hkv + u.h;
      const uint8_t* kp = c.codes + (unit * 2 * c.page + (t & (c.page - 1))) * D;
      const uint8_t* vp = kp + (size_t)c.page * D;
      const float2 sc = *reinterpret_cast<const float2*>(c.scales + unit * 2);
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < PER; ++e) s += q[e] * (qc_half2(e4m3x2_to_f16x2(kp[lane + 32 * e])).x * sc.x);
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      s *= scale;
      const float mn = fmaxf(m, s), corr = m == mn ? 1.f : exp2f(m - mn), p = exp2f(s - mn);
      l = l * corr + p;
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] = o[e] * corr + p * (qc_half2(e4m3x2_to_f16x2(vp[lane + 32 * e])).x * sc.y);
      m = mn;
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) smem[warp * ST + lane + 32 * e] = o[e];
    if (lane == 0) { smem[warp * ST + D] = m; smem[warp * ST + D + 1] = l; }
    __syncthreads();
    QtUnit one = u;
    one.col0 = cc; one.cols = 1;
    qt_write<D>(a, one, split, smem, QT_WARPS, 1);
    __syncthreads();
  }
}

// One thread block per (split, KV head, tile of columns).  A column is a (row, query head of the group); NT tiles of eight columns share the
// keys and values that the block brings in.  Tokens are the rows of the products, as in the dense entry point:
//   S^T [16 tokens x 8 columns] = K x Q^T, O^T [16 of d x 8 columns] += V^T x P^T
// e4m3 codes are exact in fp16, and so are the products' factors: a query is brought to a largest magnitude of 2^14 by a power of two (what is
// 2^-28 of the row's largest or more keeps all its bits), the scales of pages are multiplied into fp32 results: a tile of 16 tokens lies in
// one page, so one scale for S and one for the tile's part of O.  Weights are fp32 times 2^15, carried as two fp16 terms (22 bits and more).
// No sum grows over tiles inside the tensor core.
// Keys: ldmatrix gives a lane four consecutive codes of a token, which are its elements of both halves of a k step when the queries are
// read in the same order.  Values: ldmatrix.trans moves pairs of codes, i.e. two channels of two tokens in a register; a byte permutation
// puts them in pairs of tokens, and the two channels go to rows r and r + 8 of the product.
template <int D, int NT, bool LIST>
__global__ void __launch_bounds__(QT_THREADS)
qt_split_kernel(const QcDev c, const QtArgs a) {
  constexpr int TILES = QT_STAGE_BYTES / (32 * D);      // tiles of 16 tokens in a stage
  constexpr int CH = D / 16;                            // 16-byte pieces of a token's codes
  constexpr int ST = D + 2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int split = blockIdx.x % a.n_split;
  QtUnit u;
  {
    int at = blockIdx.x / a.n_split;
    u.h = at % c.Hkv; at /= c.Hkv;
    const int tile = at % a.col_tiles;
    u.seq = at / a.col_tiles;
    const QcSeq q = qc_seq(c, u.seq);
    u.row0 = q.r0; u.slot0 = q.slot0;
    u.col0 = tile * (LIST ? a.G : NT * 8);
    u.cols = min(LIST ? a.G : NT * 8, q.rows * a.G - u.col0);
  }
  if (LIST) gp_pdl_wait();                              // the list may come from the kernel before
  gp_pdl_launch_dependents();
  if (u.cols <= 0) return;
  const int row_first = u.row0 + u.col0 / a.G;
  const int* list = LIST ? a.pages + ((size_t)row_first * c.Hkv + u.h) * a.n_list : nullptr;
  const int vis = max(qt_visible(c, u, a.G, u.cols - 1), 0);             // of the last column: the most
  {
    const int len = LIST ? a.n_list << c.page_log : vis;
    const int chunk = ((len + a.n_split - 1) / a.n_split + 15) / 16 * 16;
    u.t0 = min(len, split * chunk); u.t1 = min(len, u.t0 + chunk);
  }

  // this warp's tiles: tile j of the warp covers tokens u.t0 + 16 * ((j / TILES * QT_WARPS + warp) * TILES + j % TILES)
  const int n_tiles = (u.t1 - u.t0 + 15) >> 4;
  const int n_stages = (n_tiles + TILES - 1) / TILES;
  auto tile_token = [&](int j) { return u.t0 + 16 * (((j / TILES) * QT_WARPS + warp) * TILES + j % TILES); };
  // page and scales of 32 of the warp's tiles, a lane each; the next 32 are fetched while these are worked on
  struct Where { int id, tok, left; float ks, vs; };      // page (-1: none), its row of the tile, tokens that any column sees
  auto look = [&](int j) {
    Where w;
    w.id = -1; w.tok = 0; w.left = 0; w.ks = w.vs = 0.f;
    const int t = tile_token(j);
    if (t < u.t1) {
      int lp = t >> c.page_log;
      if (LIST) { lp = list[lp]; if (lp < 0 || lp > (vis - 1) >> c.page_log) lp = -1; }
      const int slot = (lp << c.page_log) + (t & (c.page - 1));
      if (lp >= 0 && slot < vis) {
        w.id = qc_page(c, u.seq, lp);
        w.tok = slot;
        w.left = LIST ? vis - slot : min(vis, u.t1) - slot;
      }
    }
    return w;
  };
  auto look_scales = [&](Where& w) {
    if (w.id >= 0) {
      const float2 s = *reinterpret_cast<const float2*>(c.scales + ((size_t)w.id * c.Hkv + u.h) * 2);
      w.ks = s.x; w.vs = s.y;
    }
  };
  Where cur = look(lane), nxt;
  look_scales(cur);
  nxt = look(32 + lane);
  look_scales(nxt);

  uint8_t* ring = smem + warp * QT_STAGES * QT_STAGE_BYTES;
  auto fetch = [&](int i, int batch) {                  // stage i of the warp
    if (i * QT_WARPS + warp < n_stages) {
#pragma unroll
      for (int k = 0; k < TILES; ++k) {
        const int j = i * TILES + k;
        const int id = __shfl_sync(0xffffffffu, (j >> 5) == batch ? cur.id : nxt.id, j & 31);
        const int tok = __shfl_sync(0xffffffffu, (j >> 5) == batch ? cur.tok : nxt.tok, j & 31);
        const int left = __shfl_sync(0xffffffffu, (j >> 5) == batch ? cur.left : nxt.left, j & 31);
        const uint8_t* src = c.codes + ((((size_t)max(id, 0) * c.Hkv + u.h) * 2) * c.page + (tok & (c.page - 1))) * D;
        const uint32_t dst = smem_u32(ring + (i % QT_STAGES) * QT_STAGE_BYTES + k * 32 * D);
#pragma unroll
        for (int e = 0; e < 2 * CH / 2; ++e) {
          const int piece = (e * 32 + lane) % (16 * CH), t = piece / CH, pc = piece % CH;
          const bool isv = e >= CH / 2;
          const int sw = D == 128 ? t & 7 : (t >> 1) & 3;
          qt_cp_async16(dst + (isv ? 16 * D : 0) + t * D + ((pc ^ sw) << 4), src + (isv ? (size_t)c.page * D : 0) + t * D + pc * 16, t < left ? 16 : 0);
        }
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < QT_STAGES - 1; ++i) fetch(i, 0);

  // queries: column n = lane / 4 of each tile, codes 4 (lane % 4) .. + 3 of every 16
  uint32_t qb[NT][CH][2];
  float qs[NT][2];                                      // what S is multiplied with, of columns 2 (lane % 4), + 1
  const float norm = 1.4426950408889634f * rsqrtf((float)D);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int col = n * 8 + (lane >> 2), cc = u.col0 + col;
    float mx = 0.f;
    uint2 raw[CH];
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      raw[j] = make_uint2(0, 0);
      if (col < u.cols)
        raw[j] = *reinterpret_cast<const uint2*>(a.q + (size_t)(u.row0 + cc / a.G) * a.q_stride + (size_t)(u.h * a.G + cc % a.G) * D + j * 16 + (lane & 3) * 4);
      const float2 x = qc_elems(raw[j].x, a.f16), y = qc_elems(raw[j].y, a.f16);
      mx = fmaxf(mx, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(y.x), fabsf(y.y))));
    }
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    // 2^up brings the largest magnitude to 2^14 .. 2^15 (a row of zeros, and what is tiny, stays in range)
    const int ex = max((int)(__float_as_uint(mx) >> 23) - 127, -100);
    const int up = min(14 - ex, 114);
    const float mul0 = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const float2 x = qc_elems(raw[j].x, a.f16), y = qc_elems(raw[j].y, a.f16);
      __half2 h0 = __floats2half2_rn(x.x * mul0, x.y * mul0), h1 = __floats2half2_rn(y.x * mul0, y.y * mul0);
      qb[n][j][0] = *reinterpret_cast<uint32_t*>(&h0);
      qb[n][j][1] = *reinterpret_cast<uint32_t*>(&h1);
    }
    const float down = norm * __uint_as_float((uint32_t)(127 - up) << 23);
    qs[n][0] = __shfl_sync(0xffffffffu, down, (lane & 3) * 8);
    qs[n][1] = __shfl_sync(0xffffffffu, down, (lane & 3) * 8 + 4);
  }
  int see[NT][2];                                       // tokens that the lane's columns see
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) see[n][e] = qt_visible(c, u, a.G, n * 8 + (lane & 3) * 2 + e);

  float o[NT][CH][4];
  float m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int j = 0; j < CH; ++j) o[n][j][0] = o[n][j][1] = o[n][j][2] = o[n][j][3] = 0.f;
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
  }

  const int mi = lane >> 3, mr = lane & 7;              // ldmatrix: matrix and row this lane addresses
  int batch = 0;
  for (int i = 0; i * QT_WARPS + warp < n_stages; ++i) {
    if (((i * TILES) >> 5) != batch) {                  // 32 tiles on: `nxt` holds these, ask for the ones behind
      ++batch;
      cur = nxt;
      nxt = look((batch + 1) * 32 + lane);
      look_scales(nxt);
    }
    fetch(i + QT_STAGES - 1, batch);
    cp_async_wait<QT_STAGES - 1>();
    __syncwarp();
#pragma unroll
    for (int k = 0; k < TILES; ++k) {
      const int j = i * TILES + k;
      const int left = __shfl_sync(0xffffffffu, cur.left, j & 31);
      if (left <= 0 || __shfl_sync(0xffffffffu, cur.id, j & 31) < 0) continue;
      const int tok = __shfl_sync(0xffffffffu, cur.tok, j & 31);
      const float ks = __shfl_sync(0xffffffffu, cur.ks, j & 31), vs = __shfl_sync(0xffffffffu, cur.vs, j & 31);
      const uint32_t kt = smem_u32(ring + (i % QT_STAGES) * QT_STAGE_BYTES + k * 32 * D), vt = kt + 16 * D;
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
      {
        const int t = mr + (mi & 1) * 8;
        const int sw = D == 128 ? t & 7 : (t >> 1) & 3;
#pragma unroll
        for (int p = 0; p < CH / 2; ++p) {
          uint32_t r0, r1, r2, r3;                      // pieces 2p, 2p + 1 of tokens 0..7 and 8..15
          ldsm_x4(kt + t * D + (((2 * p + (mi >> 1)) ^ sw) << 4), r0, r1, r2, r3);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t x = half ? r2 : r0, y = half ? r3 : r1;
            const uint32_t a0 = e4m3x2_to_f16x2(x), a2 = e4m3x2_hi_to_f16x2(x), a1 = e4m3x2_to_f16x2(y), a3 = e4m3x2_hi_to_f16x2(y);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(s[n], a0, a1, a2, a3, qb[n][2 * p + half][0], qb[n][2 * p + half][1]);
          }
        }
      }
      uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int t = tok + (lane >> 2);
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tt = t + (e >> 1) * 8;
          const bool seen = tt < see[n][e & 1] && tt - tok < left;
          s[n][e] = seen ? s[n][e] * (ks * qs[n][e & 1]) : -INFINITY;
          mx[e & 1] = fmaxf(mx[e & 1], s[n][e]);
        }
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
          mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], off));
          mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], off));
        }
        float base[2], corr[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float mn = fmaxf(m[n][e], mx[e]);
          base[e] = mn == -INFINITY ? 0.f : mn - QT_LIFT;      // nothing seen yet: weights of zero
          corr[e] = m[n][e] == mn ? 1.f : exp2f(m[n][e] - mn);
          m[n][e] = mn;
        }
        if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
          l[n][0] *= corr[0]; l[n][1] *= corr[1];
#pragma unroll
          for (int jj = 0; jj < CH; ++jj) { o[n][jj][0] *= corr[0]; o[n][jj][1] *= corr[1]; o[n][jj][2] *= corr[0]; o[n][jj][3] *= corr[1]; }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const float p0 = exp2f(s[n][2 * half] - base[0]), p1 = exp2f(s[n][2 * half + 1] - base[1]);
          l[n][0] += p0; l[n][1] += p1;
          const __half2 h = __floats2half2_rn(p0, p1);
          const float2 hf = __half22float2(h);
          const __half2 r = __floats2half2_rn(p0 - hf.x, p1 - hf.y);
          hi[n][half] = qt_transpose8x8(*reinterpret_cast<const uint32_t*>(&h));
          lo[n][half] = qt_transpose8x8(*reinterpret_cast<const uint32_t*>(&r));
        }
      }
      {
        const int t = mr + (mi & 1) * 8;
        const int sw = D == 128 ? t & 7 : (t >> 1) & 3;
#pragma unroll
        for (int p = 0; p < CH / 2; ++p) {
          uint32_t r0, r1, r2, r3;                      // pieces 2p, 2p + 1 of tokens 0..7 and 8..15, transposed in pairs of channels
          ldsm_x4_t(vt + t * D + (((2 * p + (mi >> 1)) ^ sw) << 4), r0, r1, r2, r3);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t x = __byte_perm(half ? r2 : r0, 0, 0x3120), y = __byte_perm(half ? r3 : r1, 0, 0x3120);
            const uint32_t a0 = e4m3x2_to_f16x2(x), a1 = e4m3x2_hi_to_f16x2(x), a2 = e4m3x2_to_f16x2(y), a3 = e4m3x2_hi_to_f16x2(y);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float d[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(d, a0, a1, a2, a3, lo[n][0], lo[n][1]);
              mma_f16(d, a0, a1, a2, a3, hi[n][0], hi[n][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[n][2 * p + half][e] = fmaf(d[e], vs, o[n][2 * p + half][e]);
            }
          }
        }
      }
    }
    __syncwarp();                                       // the stage has been read: it may be fetched into
  }
  cp_async_wait<0>();
  bool bad = false;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) {
      l[n][0] += __shfl_xor_sync(0xffffffffu, l[n][0], off);
      l[n][1] += __shfl_xor_sync(0xffffffffu, l[n][1], off);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) bad |= !(fabsf(o[n][j][e]) < INFINITY) && n * 8 + (lane & 3) * 2 + (e & 1) < u.cols;
  }
  const bool one_row = LIST || u.col0 / a.G == (u.col0 + u.cols - 1) / a.G;
  if (__syncthreads_or(!one_row && bad)) {
    qt_plain<D>(c, a, u, split, reinterpret_cast<float*>(smem));
    return;
  }
  float* s_part = reinterpret_cast<float*>(smem);       // [warps][NT * 8][D + 2]
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int col = n * 8 + (lane & 3) * 2, r = lane >> 2;
    float* p0 = s_part + (size_t)(warp * NT * 8 + col) * ST;
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) p0[(e & 1) * ST + j * 16 + 2 * r + (e >> 1)] = o[n][j][e];
    if (r == 0) {
      p0[D] = m[n][0]; p0[D + 1] = l[n][0];
      p0[ST + D] = m[n][1]; p0[ST + D + 1] = l[n][1];
    }
  }
  __syncthreads();
  qt_write<D>(a, u, split, s_part, QT_WARPS, NT * 8);
}

// One block per (row, query head): merges the splits.
template <int D>
__global__ void __launch_bounds__(D)
qt_merge_kernel(const QcDev c, const QtArgs a) {
  __shared__ float s_w[256], s_l[256], s_red[D / 32];
  constexpr int ST = D + 2;
  const int tid = threadIdx.x, head = blockIdx.x % a.Hq, i = blockIdx.x / a.Hq % c.max_rows, seq = blockIdx.x / a.Hq / c.max_rows;
  const QcSeq q = qc_seq(c, seq);
  gp_pdl_wait();
  if (i >= q.rows) return;
  const size_t rh = (size_t)(q.r0 + i) * a.Hq + head;
  const float* base = a.part + rh * a.n_split * ST;
  float M = -INFINITY;
  for (int s = tid; s < a.n_split; s += D) M = fmaxf(M, __ldcg(base + (size_t)s * ST + D));
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
  if ((tid & 31) == 0) s_red[tid >> 5] = M;
  __syncthreads();
  for (int w = 0; w < D / 32; ++w) M = fmaxf(M, s_red[w]);
  float o = 0.f, l = 0.f;
  for (int s0 = 0; s0 < a.n_split; s0 += 256) {
    const int n = min(256, a.n_split - s0);
    __syncthreads();
    for (int s = tid; s < n; s += D) {
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(base + (size_t)(s0 + s) * ST + D));
      s_w[s] = M == -INFINITY ? 0.f : exp2f(ml.x - M);
      s_l[s] = ml.y;
    }
    __syncthreads();
#pragma unroll 8
    for (int s = 0; s < n; ++s) {
      o += s_w[s] * __ldcg(base + (size_t)(s0 + s) * ST + tid);
      l += s_w[s] * s_l[s];
    }
  }
  qt_store(a.out, a.out_type, rh * D + tid, l != 0.f ? o / l : 0.f);
}

// How a call is cut up, by sizes alone.
struct QtPlan { int nt, col_tiles, n_split; long long blocks; };
QtPlan qt_plan(const QcDev& c, int G, int n_list, bool list) {
  QtPlan p;
  if (list) { p.nt = 1; p.col_tiles = c.max_rows; }
  else {
    const long long cols = (long long)c.max_rows * G;
    p.nt = cols <= 8 ? 1 : cols <= 16 ? 2 : 4;
    p.col_tiles = (int)((cols + p.nt * 8 - 1) / (p.nt * 8));
  }
  const long long units = (long long)c.n_seq * p.col_tiles * c.Hkv;
  const long long len = list ? (long long)n_list << c.page_log : c.limit;
  long long splits = units > 0 ? (QT_CTAS + units - 1) / units : 1;
  const long long most = (len + QT_MIN_SPLIT - 1) / QT_MIN_SPLIT;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  p.n_split = (int)splits;
  p.blocks = units * splits;
  return p;
}
size_t qt_bytes(const QcDev& c, const QtPlan& p, int Hq, int d) {
  return p.n_split > 1 ? (size_t)c.n_rows * Hq * p.n_split * (d + 2) * sizeof(float) : 0;
}

template <int D, int NT, bool LIST>
int qt_launch(const QcDev& c, const QtArgs& a, const QtPlan& p, cudaStream_t s) {
  auto kern = qt_split_kernel<D, NT, LIST>;
  size_t smem = QT_WARPS * QT_STAGES * QT_STAGE_BYTES;
  const size_t merge = (size_t)QT_WARPS * NT * 8 * (D + 2) * sizeof(float);
  if (merge > smem) smem = merge;
  smem += 128;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return GP_ERR_CUDA;
  if (gp_launch(kern, (int)p.blocks, QT_THREADS, smem, s, LIST, c, a) != cudaSuccess) return GP_ERR_CUDA;
  if (p.n_split > 1 && gp_launch(qt_merge_kernel<D>, c.n_seq * c.max_rows * a.Hq, D, 0, s, true, c, a) != cudaSuccess) return GP_ERR_CUDA;
  return GP_OK;
}
template <int D>
int qt_dispatch(const QcDev& c, const QtArgs& a, const QtPlan& p, cudaStream_t s) {
  if (a.pages) return qt_launch<D, 1, true>(c, a, p, s);
  if (p.nt == 1) return qt_launch<D, 1, false>(c, a, p, s);
  if (p.nt == 2) return qt_launch<D, 2, false>(c, a, p, s);
  return qt_launch<D, 4, false>(c, a, p, s);
}

}  // namespace

extern "C" size_t gp_qcache_attention_bytes(const gp_qcache* cache, const gp_qbatch* batch, int32_t n_q_heads, int32_t n_list) {
  QcDev c;
  if (qc_check(cache, batch, &c) != GP_OK || n_q_heads < 1 || n_q_heads % c.Hkv || n_q_heads / c.Hkv > 8 || n_list < 0) return 0;
  if (qc_empty(c)) return 0;
  return qt_bytes(c, qt_plan(c, n_q_heads / c.Hkv, n_list, n_list > 0), n_q_heads, cache->head_dim);
}

extern "C" int gp_qcache_attention(const gp_qcache* cache, const gp_qbatch* batch, const void* q, int64_t q_stride, int32_t n_q_heads, int32_t type,
                                   const int32_t* pages, int32_t n_list, void* out, int32_t out_type, void* work, size_t work_bytes, void* stream) {
  QcDev c;
  const int st = qc_check(cache, batch, &c);
  if (st != GP_OK) return st;
  if (!qc_check_q(cache, q, q_stride, n_q_heads, type) || qc_misaligned(out, 16) || (!qc_empty(c) && (!q || !out))) return GP_ERR_INVALID;
  if (out_type != GP_TYPE_BF16 && out_type != GP_TYPE_F16 && out_type != GP_TYPE_F32) return GP_ERR_INVALID;
  if (pages ? n_list < 1 || qc_misaligned(pages, 4) || (long long)n_list * c.page > 0x7fffff00 : n_list != 0) return GP_ERR_INVALID;
  if (qc_empty(c)) return GP_OK;
  QtArgs a;
  a.q = static_cast<const unsigned short*>(q);
  a.q_stride = q_stride;
  a.Hq = n_q_heads; a.G = n_q_heads / c.Hkv; a.f16 = type == GP_TYPE_F16;
  a.pages = pages; a.n_list = n_list;
  a.out = out; a.out_type = out_type;
  const QtPlan p = qt_plan(c, a.G, n_list, pages != nullptr);
  const size_t need = qt_bytes(c, p, n_q_heads, cache->head_dim);
  if (need && (!work || qc_misaligned(work, 16) || work_bytes < need)) return GP_ERR_INVALID;
  if (p.blocks > 0x7fffffff || (long long)c.n_seq * c.max_rows * n_q_heads > 0x7fffffff) return GP_ERR_INVALID;
  a.part = static_cast<float*>(work);
  a.n_split = p.n_split; a.col_tiles = p.col_tiles;
  QcDevice dev(cache->device);
  if (!dev.ok) return GP_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return cache->head_dim == 128 ? qt_dispatch<128>(c, a, p, s) : qt_dispatch<64>(c, a, p, s);
}
