// gp_qcache_attention: attention of a packed batch's rows over the 8-bit cache, over all pages or over a list of them per row and KV head.
#include <cuda.h>
#include <cudaTypedefs.h>

#include "gp_qprompt.cuh"

namespace {

__host__ __device__ constexpr int qt_stages(int d) { return d == 64 ? 4 : 2; }      // stages of a warp's ring: 16 KB
constexpr int QT_TILES = 2;                    // tiles of 16 tokens in a stage
constexpr int QT_GRANULE = QT_WARPS * QT_TILES * 16;
constexpr int QT_MIN_SHARE = 2;                // granules a thread block takes at least
constexpr int QT_UNIT = 2;                     // what a unit costs beside its granules, in granules (its queries, the way to its first page, its end)
constexpr float QT_LIFT = 8.f;                 // weights are carried times 2^8 ...
constexpr float QT_SLACK = 7.f;                // ... while no logit is further above the maximum they refer to than this (base 2)

constexpr int qt_resident(int nt, int d) { return nt * d <= 192 ? 3 : 2; }      // blocks of an SM that the registers allow

__device__ __forceinline__ uint32_t qt_transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// 16 rows of codes (of one page) to shared memory, completion counted on an mbarrier
__device__ __forceinline__ void qt_tma_rows(uint32_t dst_smem, const CUtensorMap* map, int row, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst_smem), "l"(map),
               "r"(0), "r"(row), "r"(page), "r"(bar)
               : "memory");
}
// Joins the parts of a column that a block's warps have.  s_part: [warps][cols_stride] parts; nan (or null): per channel the least row that sees a value that is no number.
template <int D>
__device__ __forceinline__ void qt_write(const QtArgs& a, const QtUnit& u, const float* s_part, int cols_stride, const int* nan, float* part) {
  constexpr int ST = qt_part(D);
  for (int i = threadIdx.x; i < u.cols * D; i += QT_THREADS) {
    const int col = i / D, e = i % D;
    auto p = [&](int w) { return s_part + (size_t)(w * cols_stride + col) * ST; };
    float m = QT_NONE, top = -INFINITY;
#pragma unroll
    for (int w = 0; w < QT_WARPS; ++w) m = fmaxf(m, p(w)[D]);
#pragma unroll
    for (int w = 0; w < QT_WARPS; ++w) top = fmaxf(top, p(w)[D] - m + p(w)[D + 2]);
    float o = 0.f, l = 0.f;
#pragma unroll
    for (int w = 0; w < QT_WARPS; ++w) {
      o += exp2f(p(w)[D] - m + p(w)[D + 2] - top) * p(w)[e];
      l += exp2f(p(w)[D] - m) * p(w)[D + 1];
    }
    if (nan && nan[e] <= qt_row(a, col)) o = __int_as_float(0x7fffffff);
    if (!part) {
      qt_store(a.out, a.out_type, qt_query(a, u, col) * D + e, l != 0.f ? o / l * exp2f(top) : 0.f);      // (a NaN sum is not 0)
    } else {
      float* dst = part + (size_t)col * ST;
      dst[e] = o;
      if (e == 0) *reinterpret_cast<float4*>(dst + D) = make_float4(m, l, top, 0.f);
    }
  }
}

// The work of a call is one line of granules (the tokens that a block's warps take at a time): sequence by sequence, KV head by KV head, tile of
// rows by tile of rows.  Every thread block takes the same stretch of it, whatever the lengths: none waits for a long sequence at the end, and
// only the first and the last unit of a stretch can be shared with other blocks, so two partial results per block are all there is.
template <bool LIST>
__device__ __forceinline__ int qt_granules(const QcDev& c, const QtArgs& a, const QcSeq& q, int tile) {      // of one unit
  if (LIST) return ((a.n_list << c.page_log) + QT_GRANULE - 1) / QT_GRANULE;
  const int last = min((tile + 1) * a.rows_tile, q.rows);
  return max((min(q.slot0 + last, c.limit) + QT_GRANULE - 1) / QT_GRANULE, 1);      // (1: a unit without tokens is still written)
}
template <bool LIST>
__device__ __forceinline__ long long qt_head_granules(const QcDev& c, const QtArgs& a, const QcSeq& q) {     // of one KV head of a sequence
  if (LIST) return (long long)q.rows * (qt_granules<LIST>(c, a, q, 0) + QT_UNIT);
  if (q.rows * a.G > a.few) return 0;                  // the other kernel's
  long long g = 0;
  for (int t = 0; t * a.rows_tile < q.rows; ++t) g += qt_granules<LIST>(c, a, q, t) + QT_UNIT;
  return g;
}

// A column is a (row, query head of the group); NT tiles of eight columns share the keys and values that a block brings in.  Tokens are the rows
// of the products, as in the dense entry point:
//   S^T [16 tokens x 8 columns] = K x Q^T, O^T [16 of d x 8 columns] += V^T x P^T
// e4m3 codes are exact in fp16, and so are the products' factors: a query is brought to a largest magnitude of 2^14 by a power of two (what is
// 2^-28 of the row's largest or more keeps all its bits), the scales of pages are multiplied into fp32 results: a tile of 16 tokens lies in
// one page, so one scale for S and one for the tile's part of O.  Weights are computed in fp32 and rounded to fp16: once for 16-bit results
// (2^-11 of a weight at most, an eighth of a bf16 result's own rounding), as two terms (22 bits) for fp32 ones (TERMS).  Sums of weights are fp32.
// No sum grows over tiles inside the tensor core.
// The maximum that weights refer to is only brought up to date when a logit passes it by 2^7: until then a tile needs no exchange between
// lanes.  Weights times 2^8 then stay below 2^15, and fp16 reaches down to 2^-32 of the largest; a token that the maximum was taken from has 2^8, so one
// that outweighs all others loses nothing to fp16.
// O is held times 2^-e, with 2^e the largest scale of the values of the 32 tiles that a warp looks up at a time and of those before: no sum on the way passes what
// fp32 holds (weights of 2^15 times values of 448 * 2^119 would), and a tile's own factor is at most 1.
// Keys: ldmatrix gives a lane four consecutive codes of a token, which are its elements of both halves of a k step when the queries are
// read in the same order.  Values: ldmatrix.trans moves pairs of codes, i.e. two channels of two tokens in a register; a byte permutation
// puts them in pairs of tokens, and the two channels go to rows r and r + 8 of the product.
// Values that are no numbers: a weight of 0 would carry them to rows that do not see them.  Where the rows of a tile see different tokens, the codes of tokens that
// not all of them see are looked at in shared memory; a NaN counts as 0 there, and at the end the least row that sees one is found per channel.
// A warp brings its own tiles in, two at a time by TMA, into its own stages: nothing in the loop waits for another warp.
// What bounds it (with the join): memory where sequences are long (three of 60 001 to 131 071 tokens, 8 KV heads, groups of 8, d = 128: 123 us, 5.8 TB/s); where
// they are short, the start and end of a block's units (64 of 60 to 4000 tokens, groups of 4: 52 us, 5.1 TB/s); with many columns, instructions (five rows of 48
// sequences, 20 columns, d = 64: 70 us for 146 MB).
template <int D, int NT, int TERMS, bool LIST>
__global__ void __launch_bounds__(QT_THREADS, qt_resident(NT, D))
qt_split_kernel(const __grid_constant__ QcDev c, const __grid_constant__ QtArgs a, const __grid_constant__ CUtensorMap map) {
  constexpr int CH = D / 16;                            // 16-byte pieces of a token's codes
  constexpr int ST = qt_part(D);
  constexpr int ROWS = 16 * D;                          // bytes of a tile's keys, or values
  constexpr int STAGE = QT_TILES * 2 * ROWS, STAGES = qt_stages(D);
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_upto[QT_THREADS], s_warp[QT_WARPS];
  __shared__ __align__(8) uint64_t s_bar[QT_WARPS][STAGES];
  __shared__ int s_nan[D], s_found;
  __shared__ uint32_t s_top[QT_WARPS];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);      // (the swizzle goes by the address)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid < QT_WARPS * STAGES) mbar_init(&s_bar[0][0] + tid, 1);
  if (tid < D) s_nan[tid] = 0x7fffffff;
  if (tid == 0) s_found = 0;
  fence_mbar_init();
  if (LIST) gp_pdl_wait();                              // the list may come from the kernel before
  gp_pdl_launch_dependents();

  // this block's stretch: each thread adds up a run of sequences
  const int run = (c.n_seq + QT_THREADS - 1) / QT_THREADS;
  long long mine = 0;
  for (int s = tid * run; s < min((tid + 1) * run, c.n_seq); ++s) mine += c.Hkv * qt_head_granules<LIST>(c, a, qc_seq(c, s));
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  long long all = 0;
#pragma unroll
  for (int w = 0; w < QT_WARPS; ++w) {
    if (w < warp) upto += s_warp[w];
    all += s_warp[w];
  }
  s_upto[tid] = upto;
  __syncthreads();
  const long long share = max((all + gridDim.x - 1) / gridDim.x, (long long)QT_MIN_SHARE);
  const long long x0 = blockIdx.x * share, x1 = min(all, x0 + share);
  if (tid == 0) a.joins[blockIdx.x * 2] = make_int4(0, 0, 0, 0);
  if (x0 >= x1) return;
  int lo = 0, hi = QT_THREADS - 1;                      // the run that x0 lies in: first with s_upto > x0
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (s_upto[mid] > x0) hi = mid;
    else lo = mid + 1;
  }
  int seq = lo * run;
  long long xs = lo ? s_upto[lo - 1] : 0;               // where sequence `seq` begins
  QcSeq sq = qc_seq(c, seq);
  long long per_head = qt_head_granules<LIST>(c, a, sq);
  const float norm = 1.4426950408889634f * rsqrtf((float)D);
  const uint32_t ring = smem_u32(smem) + warp * STAGES * STAGE;
  uint32_t phases = 0;                                  // parity of each stage's barrier
  bool gave_up = false;

  for (long long x = x0; x < x1;) {
    while (x >= xs + per_head * c.Hkv) {
      xs += per_head * c.Hkv;
      sq = qc_seq(c, ++seq);
      per_head = qt_head_granules<LIST>(c, a, sq);
    }
    QtUnit u;
    u.seq = seq;
    u.h = (int)((x - xs) / per_head);
    long long xu = xs + u.h * per_head;                 // where the unit begins
    int tile = 0;
    if (LIST) {
      u.total = qt_granules<LIST>(c, a, sq, 0);
      tile = (int)((x - xu) / (u.total + QT_UNIT));
      xu += (long long)tile * (u.total + QT_UNIT);
    } else {
      while (x >= xu + (u.total = qt_granules<LIST>(c, a, sq, tile)) + QT_UNIT) { xu += u.total + QT_UNIT; ++tile; }
    }
    u.row0 = sq.r0 + tile * a.rows_tile;
    u.rows = min(a.rows_tile, sq.rows - tile * a.rows_tile);
    u.cols = u.rows * a.G;
    u.slot0 = sq.slot0 + tile * a.rows_tile;
    const bool begins = x == x0;
    xu += QT_UNIT;                                      // where its granules begin
    const int g0 = (int)max(0ll, x - xu), g1 = (int)min((long long)u.total, x1 - xu);
    if (g1 <= 0) break;                                 // the stretch ends before them
    const bool whole = g0 == 0 && g1 == u.total;
    float* part = whole ? nullptr : a.part + (size_t)(blockIdx.x * 2 + (begins ? 0 : 1)) * (NT * 8) * ST;
    if (g0 > 0 && g1 == u.total && tid == 0) {          // the unit began before this block and ends here: its parts are to be joined
      const int from = (int)(xu / share);
      a.joins[blockIdx.x * 2] = make_int4(u.cols, from * 2 + (xu - QT_UNIT <= from * share ? 0 : 1), from + 1, blockIdx.x);
      a.joins[blockIdx.x * 2 + 1] = make_int4(u.row0, u.h, 0, 0);
    }
    x = xu + g1;
    const int* list = LIST ? a.pages + ((size_t)u.row0 * c.Hkv + u.h) * a.n_list : nullptr;
    const int vis = max(qt_visible(c, a, u, u.cols - 1), 0);           // of the last column: the most
    const int vis0 = qt_visible(c, a, u, 0);                           // of the first: the least
    u.t0 = g0 * QT_GRANULE;
    u.t1 = min(LIST ? a.n_list << c.page_log : vis, g1 * QT_GRANULE);

    // this warp's tiles: tile j of the warp covers tokens u.t0 + 16 * ((j / QT_TILES * QT_WARPS + warp) * QT_TILES + j % QT_TILES)
    const int n_stages = gave_up ? 0 : (u.t1 - u.t0 + 16 * QT_TILES - 1) / (16 * QT_TILES);
    auto tile_token = [&](int j) { return u.t0 + 16 * (((j / QT_TILES) * QT_WARPS + warp) * QT_TILES + j % QT_TILES); };
    // page and scales of 32 of the warp's tiles, a lane each; the next 32 are fetched while these are worked on
    struct Where { int id, tok, left; float ks, vs; };      // page (-1: none), first slot of the tile, slots from it on that some column sees
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
          w.left = w.id >= 0 ? vis - slot : 0;
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
    // scales of values of 32 more tiles times 2^-e, with `was` the 2^e so far; what O is to be multiplied with
    auto scaled = [&](Where& w, uint32_t was) {
      const uint32_t top = max(was, __reduce_max_sync(0xffffffffu, __float_as_uint(w.vs)));
      w.vs *= 1.f / __uint_as_float(top);
      __syncwarp();
      if (lane == 0) s_top[warp] = top;
      __syncwarp();
      return __uint_as_float(was) / __uint_as_float(top);
    };
    Where cur = look(lane), nxt;
    nxt.id = -1; nxt.tok = nxt.left = 0; nxt.ks = nxt.vs = 0.f;
    if (n_stages * QT_TILES > 32 * QT_WARPS) nxt = look(32 + lane);
    look_scales(cur);
    look_scales(nxt);

    const bool hold = a.withhold & 1 && u.seq == 0 && u.h == 0 && tile == 0 && g0 == 0 && warp == 0;
    auto fetch = [&](int i, int batch) {                // stage i of the warp: lanes 0 .. 3 bring keys and values of its tiles
      if (i * QT_WARPS + warp >= n_stages) return;
      const int j = i * QT_TILES + ((lane >> 1) & (QT_TILES - 1));
      const bool now = (i * QT_TILES >> 5) == batch;
      const int id = __shfl_sync(0xffffffffu, now ? cur.id : nxt.id, j & 31);
      const int tok = __shfl_sync(0xffffffffu, now ? cur.tok : nxt.tok, j & 31);
      const int left = __shfl_sync(0xffffffffu, now ? cur.left : nxt.left, j & 31);
      const bool mine = lane < 2 * QT_TILES && left > 0;
      const uint32_t bar = smem_u32(&s_bar[warp][i % STAGES]);
      const int n = __popc(__ballot_sync(0xffffffffu, mine));
      if (lane == 0) mbar_expect_tx(&s_bar[warp][i % STAGES], n * ROWS + (hold && i == 0 ? 16 : 0));
      __syncwarp();
      if (mine) qt_tma_rows(ring + (i % STAGES) * STAGE + lane * ROWS, &map, (u.h * 2 + (lane & 1)) * c.page + (tok & (c.page - 1)), id, bar);
    };
    auto arrived = [&](int i) {                         // a bounded wait of the warp for stage i
      uint64_t* bar = &s_bar[warp][i % STAGES];
      const uint32_t parity = (phases >> (i % STAGES)) & 1;
      phases ^= 1u << (i % STAGES);
      if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
      const long long since = clock64();
      while (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)))
        if (__any_sync(0xffffffffu, clock64() - since > a.patience)) return false;
      return true;
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(i, 0);

    // queries: column n = lane / 4 of each tile, codes 4 (lane % 4) .. + 3 of every 16
    uint32_t qb[NT][CH][2];
    float qs[NT][2];                                    // what S is multiplied with, of columns 2 (lane % 4), + 1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int col = n * 8 + (lane >> 2);
      float mx = 0.f;
      uint2 raw[CH];
      const int r = qt_row(a, col);
      const unsigned short* from = a.q + (size_t)(u.row0 + r) * a.q_stride + (size_t)(u.h * a.G + col - r * a.G) * D + (lane & 3) * 4;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        raw[j] = make_uint2(0, 0);
        if (col < u.cols)
          raw[j] = *reinterpret_cast<const uint2*>(from + j * 16);
      }
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const float2 x2 = qc_elems(raw[j].x, a.f16), y2 = qc_elems(raw[j].y, a.f16);
        mx = fmaxf(mx, fmaxf(fmaxf(fabsf(x2.x), fabsf(x2.y)), fmaxf(fabsf(y2.x), fabsf(y2.y))));
      }
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      // 2^up brings the largest magnitude to 2^14 .. 2^15 (a row of zeros, and what is tiny, stays in range)
      const int ex = max((int)(__float_as_uint(mx) >> 23) - 127, -100);
      const int up = min(14 - ex, 114);
      const float mul0 = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const float2 x2 = qc_elems(raw[j].x, a.f16), y2 = qc_elems(raw[j].y, a.f16);
        __half2 h0 = __floats2half2_rn(x2.x * mul0, x2.y * mul0), h1 = __floats2half2_rn(y2.x * mul0, y2.y * mul0);
        qb[n][j][0] = *reinterpret_cast<uint32_t*>(&h0);
        qb[n][j][1] = *reinterpret_cast<uint32_t*>(&h1);
      }
      const float down = norm * __uint_as_float((uint32_t)(127 - up) << 23);
      qs[n][0] = __shfl_sync(0xffffffffu, down, (lane & 3) * 8);
      qs[n][1] = __shfl_sync(0xffffffffu, down, (lane & 3) * 8 + 4);
    }

    float o[NT][CH][4];
    float m[NT][2], l[NT][2];                           // m: less the lift; l: of the lane's tokens
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < CH; ++j) o[n][j][0] = o[n][j][1] = o[n][j][2] = o[n][j][3] = 0.f;
      m[n][0] = m[n][1] = QT_NONE;
      l[n][0] = l[n][1] = 0.f;
    }

    const int mi = lane >> 3, mr = lane & 7;            // ldmatrix: matrix and row this lane addresses
    const int lt = mr + (mi & 1) * 8, lsw = D == 128 ? lt & 7 : (lt >> 1) & 3;
    int batch = 0;
    scaled(cur, (uint32_t)(QC_E_MIN + 127) << 23);      // (here: copies and queries are asked for before the scales have come)
    for (int i = 0; i * QT_WARPS + warp < n_stages; ++i) {
      if ((i * QT_TILES >> 5) != batch) {               // 32 tiles on: `nxt` holds these, ask for the ones behind
        ++batch;
        cur = nxt;
        const float by = scaled(cur, s_top[warp]);
        if (by != 1.f) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < CH; ++j) { o[n][j][0] *= by; o[n][j][1] *= by; o[n][j][2] *= by; o[n][j][3] *= by; }
        }
        nxt = look((batch + 1) * 32 + lane);
        look_scales(nxt);
      }
      fetch(i + STAGES - 1, batch);
      if (!arrived(i)) {                                // nothing more is asked for; what has been is waited for before the memory is anything else's
        gave_up = true;
        for (int k = i + 1; k < i + STAGES && k * QT_WARPS + warp < n_stages; ++k) arrived(k);
        break;
      }
      const uint32_t stage = ring + (i % STAGES) * STAGE;
      int left[QT_TILES], tok[QT_TILES];
      float kf[QT_TILES], vs[QT_TILES];                 // scales of keys and values
      int most = 0, end = 0;
#pragma unroll
      for (int k = 0; k < QT_TILES; ++k) {
        const int j = (i * QT_TILES + k) & 31;
        left[k] = __shfl_sync(0xffffffffu, cur.left, j);
        kf[k] = __shfl_sync(0xffffffffu, cur.ks, j);
        vs[k] = __shfl_sync(0xffffffffu, cur.vs, j);
        tok[k] = left[k] > 0 ? __shfl_sync(0xffffffffu, cur.tok, j) : 0x40000000;      // (a tile that is not there is seen by nobody)
        most = max(most, left[k]); end = max(end, tok[k]);
      }
      if (most <= 0) { __syncwarp(); continue; }
      const bool ragged = end + 16 > vis0;              // some column does not see all of the stage
      if (ragged) {
#pragma unroll
        for (int k = 0; k < QT_TILES; ++k) {
          // rows behind the sequence, and tiles that are not there: whatever an earlier owner or tile left, NaN too
          for (int r = max(left[k], 0) * (D / 16) + lane; r < D; r += 32)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(stage + (k * 2 + 1) * ROWS + r * 16), "r"(0) : "memory");
          // rows that some column does not see
          for (int r = max(vis0 - tok[k], 0) * (D / 16) + lane; r < min(left[k], 16) * (D / 16); r += 32) {
            const uint32_t at = stage + (k * 2 + 1) * ROWS + r * 16;
            uint32_t w[4], any = 0;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t bad = __vcmpeq4(w[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
              w[e] &= ~bad; any |= bad;
            }
            if (any) {
              s_found = 1;
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
            }
          }
        }
        fence_proxy_async();                            // the next copy into the stage comes behind these stores
        __syncwarp();
      }
      float s[QT_TILES][NT][4];
      auto factor = [&](int k, int n, int e) { return fmaxf(kf[k] * qs[n][e], 1.2e-38f); };      // (above 0: a masked logit stays what it is)
      // (d = 64: no branch on what a tile holds lies between the tiles of a stage, so that one's instructions fill the other's waits, 73 -> 70 us for five
      // rows of 48 sequences; d = 128 has no registers for both, 122 -> 126 us for three long sequences)
#pragma unroll
      for (int k = 0; k < QT_TILES; ++k) {
        if (D == 128 && left[k] <= 0) continue;
#pragma unroll
        for (int p = 0; p < CH / 2; ++p) {
          uint32_t r0, r1, r2, r3;                      // pieces 2p, 2p + 1 of tokens 0..7 and 8..15
          ldsm_x4(stage + k * 2 * ROWS + lt * D + (((2 * p + (mi >> 1)) ^ lsw) << 4), r0, r1, r2, r3);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t xx = half ? r2 : r0, yy = half ? r3 : r1;
            const uint32_t a0 = e4m3x2_to_f16x2(xx), a2 = e4m3x2_hi_to_f16x2(xx), a1 = e4m3x2_to_f16x2(yy), a3 = e4m3x2_hi_to_f16x2(yy);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              if (p == 0 && half == 0) mma_f16_first(s[k][n], a0, a1, a2, a3, qb[n][0][0], qb[n][0][1]);
              else mma_f16(s[k][n], a0, a1, a2, a3, qb[n][2 * p + half][0], qb[n][2 * p + half][1]);
            }
          }
        }
      }
      if (ragged) {
#pragma unroll
        for (int k = 0; k < QT_TILES; ++k) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (tok[k] + (lane >> 2) + (e >> 1) * 8 >= qt_visible(c, a, u, n * 8 + (lane & 3) * 2 + (e & 1))) s[k][n][e] = -INFINITY;
        }
      }
      bool over = false;
#pragma unroll
      for (int k = 0; k < QT_TILES; ++k)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          over |= fmaf(fmaxf(s[k][n][0], s[k][n][2]), factor(k, n, 0), -m[n][0]) > QT_LIFT + QT_SLACK ||
                  fmaf(fmaxf(s[k][n][1], s[k][n][3]), factor(k, n, 1), -m[n][1]) > QT_LIFT + QT_SLACK;
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int k = 0; k < QT_TILES; ++k) {
            mx[0] = fmaxf(mx[0], fmaxf(s[k][n][0], s[k][n][2]) * factor(k, n, 0));
            mx[1] = fmaxf(mx[1], fmaxf(s[k][n][1], s[k][n][3]) * factor(k, n, 1));
          }
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) {
            mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], off));
            mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], off));
          }
          float corr[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float mn = fmaxf(m[n][e], mx[e] - QT_LIFT);
            corr[e] = m[n][e] == mn ? 1.f : qt_exp2(m[n][e] - mn);
            m[n][e] = mn;
          }
          l[n][0] *= corr[0]; l[n][1] *= corr[1];
#pragma unroll
          for (int jj = 0; jj < CH; ++jj) { o[n][jj][0] *= corr[0]; o[n][jj][1] *= corr[1]; o[n][jj][2] *= corr[0]; o[n][jj][3] *= corr[1]; }
        }
      }
#pragma unroll
      for (int k = 0; k < QT_TILES; ++k) {
        if (D == 128 && left[k] <= 0) continue;
        uint32_t pb[NT][TERMS][2];                      // B fragments of P^T: tokens 0..7 and 8..15
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float f0 = factor(k, n, 0), f1 = factor(k, n, 1);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float p0 = qt_exp2(fmaf(s[k][n][2 * half], f0, -m[n][0])), p1 = qt_exp2(fmaf(s[k][n][2 * half + 1], f1, -m[n][1]));
            l[n][0] += p0; l[n][1] += p1;
            const __half2 h = __floats2half2_rn(p0, p1);
            pb[n][0][half] = qt_transpose8x8(*reinterpret_cast<const uint32_t*>(&h));
            if (TERMS == 2) {
              const float2 hf = __half22float2(h);
              const __half2 r = __floats2half2_rn(p0 - hf.x, p1 - hf.y);
              pb[n][TERMS - 1][half] = qt_transpose8x8(*reinterpret_cast<const uint32_t*>(&r));
            }
          }
        }
#pragma unroll
        for (int p = 0; p < CH / 2; ++p) {
          uint32_t r0, r1, r2, r3;                      // pieces 2p, 2p + 1 of tokens 0..7 and 8..15, transposed in pairs of channels
          ldsm_x4_t(stage + (k * 2 + 1) * ROWS + lt * D + (((2 * p + (mi >> 1)) ^ lsw) << 4), r0, r1, r2, r3);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t xx = __byte_perm(half ? r2 : r0, 0, 0x3120), yy = __byte_perm(half ? r3 : r1, 0, 0x3120);
            const uint32_t a0 = e4m3x2_to_f16x2(xx), a1 = e4m3x2_hi_to_f16x2(xx), a2 = e4m3x2_to_f16x2(yy), a3 = e4m3x2_hi_to_f16x2(yy);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float d[4];
              mma_f16_first(d, a0, a1, a2, a3, pb[n][TERMS - 1][0], pb[n][TERMS - 1][1]);
              if (TERMS == 2) mma_f16(d, a0, a1, a2, a3, pb[n][0][0], pb[n][0][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[n][2 * p + half][e] = fmaf(d[e], vs[k], o[n][2 * p + half][e]);
            }
          }
        }
      }
      __syncwarp();                                     // the stage has been read: it may be fetched into
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) {
        l[n][0] += __shfl_xor_sync(0xffffffffu, l[n][0], off);
        l[n][1] += __shfl_xor_sync(0xffffffffu, l[n][1], off);
      }
    }
    __syncthreads();
    const bool nans = s_found != 0;
    float* s_part = reinterpret_cast<float*>(smem);     // [warps][NT * 8] parts
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
        p0[D + 2] = p0[ST + D + 2] = (float)((int)(s_top[warp] >> 23) - 127);
      }
    }
    if (nans)                                           // once more, from the cache: which channels, which rows
      for (int i = tid; i < (u.t1 - max(u.t0, vis0)) * (D / 4); i += QT_THREADS) {
        const int t = max(u.t0, vis0) + i / (D / 4), id = qc_page(c, seq, t >> c.page_log);
        if (id < 0) continue;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(c.codes + (((size_t)id * c.Hkv + u.h) * 2 * c.page + c.page + (t & (c.page - 1))) * D + i % (D / 4) * 4);
        for (int e = 0; e < 4; ++e)
          if ((w >> (8 * e) & 0x7f) == 0x7f) atomicMin(&s_nan[i % (D / 4) * 4 + e], t + 1 - vis0);
      }
    __syncthreads();
    qt_write<D>(a, u, s_part, NT * 8, nans ? s_nan : nullptr, part);
    fence_proxy_async();
    __syncthreads();                                    // the memory is the ring's again
    if (nans) {
      if (tid < D) s_nan[tid] = 0x7fffffff;
      if (tid == 0) s_found = 0;
      __syncthreads();
    }
  }
  if (gave_up && c.status) atomicOr(c.status, GP_E_SPIN);
}

// The codes as TMA sees them: [pages][rows of a page: KV head, keys | values, token][d], 16 rows at a time, swizzled so that ldmatrix meets no
// bank twice.  Encoded anew for every call (host work of a fraction of a microsecond).
bool qt_map(const gp_qcache* c, CUtensorMap* map) {
  static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult got;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &got) != cudaSuccess || got != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  if (!encode) return false;
  const cuuint64_t rows = (cuuint64_t)c->n_kv_heads * 2 * c->page_size, d = (cuuint64_t)c->head_dim;
  const cuuint64_t dims[3] = {d, rows, (cuuint64_t)c->n_pages}, strides[2] = {d, rows * d};
  const cuuint32_t box[3] = {(cuuint32_t)d, 16, 1}, step[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, c->codes, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a call is cut up, by sizes alone.
struct QtPlan { int nt, blocks; };
QtPlan qt_plan(const QcDev& c, int G, int d, int n_list, bool list) {
  QtPlan p;
  const bool all = (long long)c.max_rows * G <= qt_few(d);                     // sequences of more rows are the other kernel's
  const int rows = list ? 1 : all ? c.max_rows : qt_few(d) / G;
  const long long cols = (long long)rows * G;
  // Tiles of columns by what a sequence may have; beside sequences of many rows most have one row (255 of them beside one of 2048 rows: 272 us with single
  // tiles, 380 with as many as 48 columns want).
  p.nt = cols <= 8 || !all ? 1 : cols <= 16 ? 2 : cols <= 24 ? 3 : 4;
  if (list) p.nt = 1;
  const int rows_tile = list ? 1 : p.nt * 8 / G;
  const long long units = (long long)c.n_seq * ((list ? c.max_rows : rows) + rows_tile - 1) / rows_tile * c.Hkv;
  const long long len = list ? (long long)n_list << c.page_log : c.limit;
  const long long most = units * ((len + QT_GRANULE - 1) / QT_GRANULE + 1 + QT_UNIT);          // granules, more than there can be
  const long long wave = 148 * qt_resident(p.nt, d);
  const long long blocks = (most + QT_MIN_SHARE - 1) / QT_MIN_SHARE;
  p.blocks = (int)(blocks < wave ? blocks : wave);
  return p;
}
size_t qt_joins_bytes(const QtPlan& p) { return (size_t)p.blocks * 2 * sizeof(int4); }
size_t qt_bytes(const QtPlan& p, int d) { return qt_joins_bytes(p) + (size_t)p.blocks * 2 * p.nt * 8 * qt_part(d) * sizeof(float); }

template <int D, int NT, int TERMS, bool LIST>
int qt_launch(const QcDev& c, const QtArgs& a, const CUtensorMap& map, const QtPlan& p, cudaStream_t s) {
  auto kern = qt_split_kernel<D, NT, TERMS, LIST>;
  size_t smem = QT_WARPS * qt_stages(D) * QT_TILES * 32 * D;
  const size_t merge = (size_t)QT_WARPS * NT * 8 * qt_part(D) * sizeof(float);
  if (merge > smem) smem = merge;
  smem += 1024;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return GP_ERR_CUDA;
  if (gp_launch(kern, p.blocks, QT_THREADS, smem, s, LIST, c, a, map) != cudaSuccess) return GP_ERR_CUDA;
  if (p.blocks > 1 && gp_launch(qt_merge_kernel<D, NT * 8, 2>, p.blocks * NT * 2, 128, 0, s, true, a) != cudaSuccess) return GP_ERR_CUDA;
  return GP_OK;
}
template <int D, int TERMS>
int qt_dispatch(const QcDev& c, const QtArgs& a, const CUtensorMap& map, const QtPlan& p, cudaStream_t s) {
  if (a.pages) return qt_launch<D, 1, TERMS, true>(c, a, map, p, s);
  switch (p.nt) {
    case 1: return qt_launch<D, 1, TERMS, false>(c, a, map, p, s);
    case 2: return qt_launch<D, 2, TERMS, false>(c, a, map, p, s);
    case 3: return qt_launch<D, 3, TERMS, false>(c, a, map, p, s);
    default: return qt_launch<64, 4, TERMS, false>(c, a, map, p, s);
  }
}

// Which of the two kernels a call has work for: that for many rows where a sequence may have them; that for few unless all have as many.
struct QtBoth { bool few, many; QtPlan few_plan; QpPlan many_plan; size_t few_bytes, bytes; };
QtBoth qt_both(const QcDev& c, int G, int d, int n_list) {
  QtBoth b = {};
  const bool list = n_list > 0;
  b.many = !list && (long long)c.max_rows * G > qt_few(d);
  b.few = !b.many || (c.n_seq > 1 && c.n_rows < (long long)c.n_seq * c.max_rows);
  if (b.few) { b.few_plan = qt_plan(c, G, d, n_list, list); b.few_bytes = (qt_bytes(b.few_plan, d) + 15) / 16 * 16; }
  b.bytes = b.few_bytes;
  if (b.many) { b.many_plan = qp_plan(c, G); b.bytes += qp_bytes(b.many_plan, d); }
  return b;
}

}  // namespace

static thread_local struct { long long patience; int withhold; } qt_test = {QT_PATIENCE, 0};

extern "C" int gp_qcache_test_withhold(int32_t what, int64_t cycles) {
  if (what < 0 || what > 3 || cycles < 0) return GP_ERR_INVALID;
  qt_test = {cycles > 0 ? cycles : QT_PATIENCE, what};
  return GP_OK;
}

extern "C" size_t gp_qcache_attention_bytes(const gp_qcache* cache, const gp_qbatch* batch, int32_t n_q_heads, int32_t n_list) {
  QcDev c;
  if (qc_check(cache, batch, &c) != GP_OK || n_q_heads < 1 || n_q_heads % c.Hkv || n_q_heads / c.Hkv > 8 || n_list < 0) return 0;
  return qc_empty(c) ? 0 : qt_both(c, n_q_heads / c.Hkv, cache->head_dim, n_list).bytes;
}

extern "C" int gp_qcache_attention(const gp_qcache* cache, const gp_qbatch* batch, const void* q, int64_t q_stride, int32_t n_q_heads, int32_t type,
                                   const int32_t* pages, int32_t n_list, void* out, int32_t out_type, void* work, size_t work_bytes, void* stream) {
  QcDev c;
  const int st = qc_check(cache, batch, &c);
  if (st != GP_OK) return st;
  if (!qc_check_q(cache, q, q_stride, n_q_heads, type) || qc_misaligned(out, 16) || (!qc_empty(c) && (!q || !out))) return GP_ERR_INVALID;
  if (out_type != GP_TYPE_BF16 && out_type != GP_TYPE_F16 && out_type != GP_TYPE_F32) return GP_ERR_INVALID;
  if (pages ? n_list < 1 || qc_misaligned(pages, 4) || (long long)n_list * c.page > QC_MAX_LEN : n_list != 0) return GP_ERR_INVALID;
  if (qc_empty(c)) return GP_OK;
  QtArgs a;
  a.q = static_cast<const unsigned short*>(q);
  a.q_stride = q_stride;
  a.Hq = n_q_heads; a.G = n_q_heads / c.Hkv; a.by_g = qt_by_g(a.G); a.f16 = type == GP_TYPE_F16;
  a.pages = pages; a.n_list = n_list;
  a.out = out; a.out_type = out_type;
  const int d = cache->head_dim;
  a.few = qt_few(d);
  a.patience = qt_test.patience; a.withhold = qt_test.withhold;
  const QtBoth b = qt_both(c, a.G, d, n_list);
  if (!work || qc_misaligned(work, 16) || work_bytes < b.bytes) return GP_ERR_INVALID;
  QcDevice dev(cache->device);
  if (!dev.ok) return GP_ERR_CUDA;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (b.few) {
    const QtPlan& p = b.few_plan;
    a.joins = static_cast<int4*>(work);
    a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(work) + qt_joins_bytes(p));
    a.rows_tile = pages ? 1 : p.nt * 8 / a.G;
    CUtensorMap map;
    if (!qt_map(cache, &map)) return GP_ERR_CUDA;
    const int got = d == 128 ? (out_type == GP_TYPE_F32 ? qt_dispatch<128, 2>(c, a, map, p, s) : qt_dispatch<128, 1>(c, a, map, p, s))
                             : (out_type == GP_TYPE_F32 ? qt_dispatch<64, 2>(c, a, map, p, s) : qt_dispatch<64, 1>(c, a, map, p, s));
    if (got != GP_OK) return got;
  }
  a.few = b.few ? qt_few(d) : 0;                        // (alone, it takes sequences of few rows too)
  return b.many ? qp_launch(c, a, b.many_plan, d, static_cast<uint8_t*>(work) + b.few_bytes, s) : GP_OK;
}
