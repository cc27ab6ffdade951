// Attention over the 8-bit cache for many rows of a sequence at once (chunks of prompts): both products on the fifth-generation tensor cores.
#include "gp_qprompt.cuh"

namespace {

constexpr int QP_M = 128;                      // columns (row, query head of the group) of a half of a block's tile: the rows of a product
constexpr int QP_COLS = 2 * QP_M;
constexpr int QP_N = 128;                      // tokens of a step
constexpr int QP_SOFT = 256, QP_CONV = 128;    // threads that turn logits into weights, a column each; that turn codes into fp16
constexpr int QP_THREADS = QP_SOFT + QP_CONV;
constexpr int QP_ISSUER = 11;                  // warp whose first lane issues the products
constexpr int QP_UNIT = 256;                   // what a unit costs beside its tokens, in tokens
constexpr float QP_SLACK = 7.f;                // a row's maximum is brought up to date when something passes it by 2^7
constexpr float QP_LIFT = 8.f;
constexpr int QP_BLOCK = QP_N * 128;           // bytes of 64 fp16 channels of 128 rows

__device__ __forceinline__ uint64_t qp_desc(uint32_t addr, uint32_t lbo) {      // shared-memory matrix, 128-byte swizzle, groups of 8 rows 1024 bytes apart
  return (uint64_t)((addr >> 4) & 0x3fff) | (uint64_t)((lbo >> 4) & 0x3fff) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ void qp_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
               "r"((uint32_t)add)
               : "memory");
}
__device__ __forceinline__ void qp_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {      // A in tensor memory
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
               "r"((uint32_t)add)
               : "memory");
}
__device__ __forceinline__ void qp_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void qp_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// two fp32 numbers at a time
__device__ __forceinline__ uint64_t qp_pack2(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void qp_unpack2(uint64_t x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t qp_fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t qp_add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float qp_max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ void qp_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void qp_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void qp_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void qp_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 / 16 columns of the warp's 32 lanes
__device__ __forceinline__ void qp_ld32(uint32_t t, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(t));
}
__device__ __forceinline__ void qp_st32(uint32_t t, const float* x) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(x);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(t),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void qp_st16(uint32_t t, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(t), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}

struct QpShared {
  // per half of the tile and, for what a step's place in the two-deep rings depends on, per parity of the step
  uint64_t q_full[2], k_full[2], v_full[2], s_full[2][2], p_full[2], o_full[2][2], sc_full[4];
  uint32_t tmem;
  int dead;                                    // a wait ran out: all others end at once
  int nan[2];                                  // the last piece of work (its number, by parity) with a value that is no number where rows see different tokens
  float ks[4][8], ev[4][8];                    // per step (four at a time) and group of 16 tokens: scale of the keys (-1: no such page), exponent of that of the values
  long long upto[QP_THREADS], warp[QP_THREADS / 32];
  float plain[2][QT_WARPS * 130];
};
// A bounded wait for a phase of a barrier.
__device__ __forceinline__ void qp_wait(QpShared& sh, uint64_t* bar, uint32_t parity) {
  for (unsigned spin = 0; !mbar_try_wait(bar, parity); ++spin)
    if (spin > GP_SPIN_LIMIT || *reinterpret_cast<volatile int*>(&sh.dead)) { *reinterpret_cast<volatile int*>(&sh.dead) = 1; break; }
}

// The line of work (as in the other kernel): sequence by sequence, KV head by KV head, tile of rows by tile of rows, measured in tokens.  Tile t of
// a sequence has s + R (t + 1) + QP_UNIT of it, with R the rows of a tile and s the slot of the sequence's first row, so T tiles have
__device__ __forceinline__ long long qp_line(const QcSeq& q, int R, long long T) {
  return T * (max(q.slot0, 0) + QP_UNIT) + R * (T * (T + 1) / 2);
}
__device__ __forceinline__ long long qp_head_line(const QcSeq& q, int R) { return qp_line(q, R, (q.rows + R - 1) / R); }

struct QpPiece {                               // a stretch of a unit
  QtUnit u;                                    // of all of the tile
  int n_steps;
  bool whole, begins;                          // all of the unit; at the start of the block's stretch
};
// Walks along a block's stretch of the line; every thread does.
struct QpWalk {
  long long x, x0, x1, share, xs, per_head;
  int seq;
  QcSeq sq;
  __device__ __forceinline__ bool start(const QcDev& c, int R, QpShared& sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (c.n_seq + QP_THREADS - 1) / QP_THREADS;
    long long up = 0;
    for (int s = tid * run; s < min((tid + 1) * run, c.n_seq); ++s) up += c.Hkv * qp_head_line(qc_seq(c, s), R);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += y;
    }
    if (lane == 31) sh.warp[warp] = up;
    __syncthreads();
    long long all = 0;
    for (int w = 0; w < QP_THREADS / 32; ++w) {
      if (w < warp) up += sh.warp[w];
      all += sh.warp[w];
    }
    sh.upto[tid] = up;
    __syncthreads();
    share = max((all + gridDim.x - 1) / gridDim.x, 4ll * QP_N);
    x = x0 = blockIdx.x * share;
    x1 = min(all, x0 + share);
    if (x0 >= x1) return false;
    int lo = 0, hi = QP_THREADS - 1;                    // the run that x0 lies in: first with upto > x0
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (sh.upto[mid] > x0) hi = mid;
      else lo = mid + 1;
    }
    seq = lo * run;
    xs = lo ? sh.upto[lo - 1] : 0;
    sq = qc_seq(c, seq);
    per_head = qp_head_line(sq, R);
    return true;
  }
  __device__ __forceinline__ bool next(const QcDev& c, const QtArgs& a, int R, QpPiece& p, int4* join) {      // join[0], [1]: what is to be joined at its end
    for (;;) {
      if (x >= x1) return false;
      while (x >= xs + per_head * c.Hkv) {
        xs += per_head * c.Hkv;
        sq = qc_seq(c, ++seq);
        per_head = qp_head_line(sq, R);
      }
      QtUnit& u = p.u;
      u.seq = seq;
      u.h = (int)((x - xs) / per_head);
      const long long xh = xs + u.h * per_head;
      // the tile: the root of R T^2 / 2 + (s + QP_UNIT + R / 2) T = x - xh, put right by whole numbers
      const double b = max(sq.slot0, 0) + QP_UNIT + 0.5 * R;
      long long T = (long long)((sqrt(b * b + 2.0 * R * (double)(x - xh)) - b) / R);
      while (T > 0 && qp_line(sq, R, T) > x - xh) --T;
      while (qp_line(sq, R, T + 1) <= x - xh) ++T;
      const long long xu = xh + qp_line(sq, R, T), xe = xh + qp_line(sq, R, T + 1);
      u.row0 = sq.r0 + (int)T * R;
      u.rows = min(R, sq.rows - (int)T * R);
      u.cols = u.rows * a.G;
      u.slot0 = sq.slot0 + (int)T * R;
      const int vis = max(min(u.slot0 + u.rows, c.limit), 0);
      u.total = max((vis + QP_N - 1) / QP_N, 1);        // (1: a unit without tokens is still written)
      // step k lies at xu + k QP_N
      const int g0 = (int)min((x - xu + QP_N - 1) / QP_N, (long long)u.total), g1 = (int)min((min(x1, xe) - xu + QP_N - 1) / QP_N, (long long)u.total);
      p.begins = x == x0;
      x = min(x1, xe);
      if (g0 >= g1) continue;                           // a stretch of the unit's end that holds no step
      p.whole = g0 == 0 && g1 == u.total;
      u.t0 = g0 * QP_N;
      u.t1 = min(vis, g1 * QP_N);
      p.n_steps = (max(u.t1 - u.t0, 0) + QP_N - 1) / QP_N;
      if (g0 > 0 && g1 == u.total) {                    // the unit began before this block and ends here
        const int from = (int)(xu / share);
        join[0] = make_int4(u.cols, from * 2 + (xu == from * share ? 0 : 1), from + 1, blockIdx.x);
        join[1] = make_int4(u.row0, u.h, 0, 0);
      }
      return true;
    }
  }
};

// A block takes tiles of up to 256 columns (row, query head of the group) of one (sequence, KV head), in two halves A and B, and a stretch of their
// tokens, 128 at a step.  Per half:
//   S [128 columns x 128 tokens] = Q K^T      (tcgen05, fp16 in shared memory, S in tensor memory)
//   P = weights of S                           (four warps, a thread a column; fp16, over S in tensor memory)
//   O [128 columns x d] += P V                 (tcgen05, P from tensor memory, V in shared memory)
// While one half's weights are computed, the other's products run.  Four more warps bring codes in and write them to shared memory as fp16, which
// holds them exactly and unscaled: K and V in the same image (a token's channels along a row, 64 a swizzled 128 bytes), which the first product
// reads with the channels, the second with the tokens as inner dimension; one of their threads issues the products.  Two steps of K and V are there.
// Scales of pages cost nothing per element: 16 columns of S lie in one page, so the keys' scale joins the factor of the logits and the exponent of
// the values' scale the constant that is added before the exponential: p' = 2^(s + ev - M), M the running maximum of s + ev.  O is then a plain
// sum of p' times codes.  The sum of weights L is taken of p' 2^(E - ev) group by group, with E (an exponent of about the size of the largest ev so far)
// keeping it in range; out = 2^E O / L.
// What bounds it: 2 x 128 x 128 exponentials a step and SM (16 a cycle) against 2 x 128 x 128 x 2 d multiply-adds (4096 a cycle): with d = 128 the same.
template <int D, int TERMS>
__global__ void __launch_bounds__(QP_THREADS, 1)
qp_kernel(const __grid_constant__ QcDev c, const __grid_constant__ QtArgs a) {
  constexpr int CH = D / 16, ST = D + 2;
  constexpr int OPERAND = D / 64 * QP_BLOCK;            // bytes of a half's Q, of a step's K or V in shared memory
  // tensor memory: S (and P over it) and O of each half; the second terms of the weights over the S columns that P leaves free
  constexpr uint32_t T_S = 0, T_O = 256;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) QpShared sh;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = base, k_smem = base + 2 * OPERAND, v_smem = base + 4 * OPERAND;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int RT = QP_M / a.G, R = 2 * RT;                // rows of a half, of a tile

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], 4);
      mbar_init(&sh.k_full[i], 4);
      mbar_init(&sh.v_full[i], 4);
      mbar_init(&sh.p_full[i], 4);
      for (int e = 0; e < 2; ++e) { mbar_init(&sh.s_full[i][e], 1); mbar_init(&sh.o_full[i][e], 1); }
      sh.nan[i] = -1;
    }
    for (int i = 0; i < 4; ++i) mbar_init(&sh.sc_full[i], 1);
    sh.dead = 0;
    fence_mbar_init();
    a.joins[blockIdx.x * 2] = make_int4(0, 0, 0, 0);
  }
  if (warp == QP_ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  qp_fence_before();
  QpWalk walk;
  const bool any = walk.start(c, R, sh);                // (meets twice)
  qp_fence_after();
  gp_pdl_launch_dependents();
  const uint32_t tmem = sh.tmem;
  int n = 0;                                            // steps before the piece
  QpPiece p;

  if (!any) {
  } else if (warp >= 8) {                               // ---- codes to fp16, products
    const int ct = tid - QP_SOFT, cw = warp - 8;
    constexpr int TPI = QP_CONV / CH;                   // tokens of a round
    constexpr int IT = QP_N / TPI;
    const int ch = ct % CH, tt = ct / CH;               // piece of 16 channels; token in the round
    const uint32_t idesc = 1u << 4 | (QP_M / 16u) << 24, qk = idesc | (QP_N / 8u) << 17, pv = idesc | 1u << 16 | (D / 8u) << 17;
    const bool issuer = warp == QP_ISSUER && lane == 0;
    int4 join[2];
    join[0].x = 0;
    for (int piece = 0; walk.next(c, a, R, p, join); ++piece) {
      const QtUnit& u = p.u;
      const bool has_b = u.cols > RT * a.G;
      const int vis0 = qt_visible(c, u, a.G, 0);        // of the first row: the least
      // lanes 0 .. 7: page of a group of 16 tokens of a step
      auto page_of = [&](int j) {
        const int t = u.t0 + j * QP_N + lane * 16;
        return lane < 8 && t < u.t1 ? qc_page(c, u.seq, t >> c.page_log) : -1;
      };
      auto load = [&](uint4* r, int j, int ids, int kv) {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          const int t = i * TPI + tt, at = u.t0 + j * QP_N + t;
          const int id = __shfl_sync(0xffffffffu, ids, t >> 4);
          r[i] = make_uint4(0, 0, 0, 0);
          if (id >= 0 && at < u.t1)
            r[i] = __ldg(reinterpret_cast<const uint4*>(c.codes + ((((size_t)id * c.Hkv + u.h) * 2 + kv) * c.page + (at & (c.page - 1))) * D + ch * 16));
        }
      };
      auto store = [&](const uint4* r, uint32_t dst) {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          const int t = i * TPI + tt;
          const uint32_t row = dst + (ch >> 2) * QP_BLOCK + t * 128;
          const int c0 = (ch & 3) * 2, flip = (ch >> 2) & 1;    // the two halves of 128 channels write their pieces in opposite order: no bank twice
          const uint4 x = r[i];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int hf = e ^ flip;
            const uint32_t w0 = hf ? x.z : x.x, w1 = hf ? x.w : x.y;
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + (((c0 + hf) ^ (t & 7)) << 4)), "r"(e4m3x2_to_f16x2(w0)),
                         "r"(e4m3x2_hi_to_f16x2(w0)), "r"(e4m3x2_to_f16x2(w1)), "r"(e4m3x2_hi_to_f16x2(w1))
                         : "memory");
          }
        }
      };
      auto issue_qk = [&](int half, int s) {            // step s (of all)
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k >> 2) * QP_BLOCK + (k & 3) * 32;
          if (half == 0 || has_b)
            qp_mma_ss(tmem + T_S + half * 128, qp_desc(q_smem + half * OPERAND + off, 16), qp_desc(k_smem + (s & 1) * OPERAND + off, 16), qk, k > 0);
        }
        qp_commit(&sh.s_full[half][s & 1]);
      };
      auto issue_pv = [&](int half, int s, bool first) {
        qp_wait(sh, &sh.p_full[half], s & 1);
        qp_fence_after();
        if (half == 0 || has_b) {
#pragma unroll
          for (int t = 0; t < TERMS; ++t)
#pragma unroll
            for (int k = 0; k < QP_N / 16; ++k)
              qp_mma_ts(tmem + T_O + half * 128, tmem + T_S + half * 128 + t * 64 + k * 8, qp_desc(v_smem + (s & 1) * OPERAND + k * 2048, QP_BLOCK), pv,
                        !first || t > 0 || k > 0);
        }
        qp_commit(&sh.o_full[half][s & 1]);
      };
      uint4 kr[IT], vr[IT];
      int ids = page_of(0), ids1 = page_of(1);
      load(kr, 0, ids, 0);
      load(vr, 0, ids, 1);
      for (int j = 0; j < p.n_steps; ++j) {
        const int s = n + j;
        const int ids2 = page_of(j + 2);
        if (s >= 2) {                                   // both halves' products have read the keys that were here
          qp_wait(sh, &sh.s_full[0][s & 1], ((s - 2) >> 1) & 1);
          qp_wait(sh, &sh.s_full[1][s & 1], ((s - 2) >> 1) & 1);
        }
        if (cw == 0) {
          float2 sc = make_float2(-1.f, 1.f);
          if (ids >= 0) sc = *reinterpret_cast<const float2*>(c.scales + ((size_t)ids * c.Hkv + u.h) * 2);
          if (lane < 8) { sh.ks[s & 3][lane] = sc.x; sh.ev[s & 3][lane] = (float)((int)((__float_as_uint(sc.y) >> 23) & 255) - 127); }
          __syncwarp();
          if (lane == 0) qp_arrive(&sh.sc_full[s & 3]);
        }
        store(kr, k_smem + (s & 1) * OPERAND);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) qp_arrive(&sh.k_full[s & 1]);
        load(kr, j + 1, ids1, 0);
        if (u.t0 + (j + 1) * QP_N > vis0) {             // rows see different tokens of the step
          bool nan = false;
#pragma unroll
          for (int i = 0; i < IT; ++i)
            nan |= (__vcmpeq4(vr[i].x & 0x7f7f7f7f, 0x7f7f7f7f) | __vcmpeq4(vr[i].y & 0x7f7f7f7f, 0x7f7f7f7f) | __vcmpeq4(vr[i].z & 0x7f7f7f7f, 0x7f7f7f7f) |
                    __vcmpeq4(vr[i].w & 0x7f7f7f7f, 0x7f7f7f7f)) != 0;
          if (nan) *reinterpret_cast<volatile int*>(&sh.nan[piece & 1]) = piece;
        }
        if (s >= 2) {
          qp_wait(sh, &sh.o_full[0][s & 1], ((s - 2) >> 1) & 1);
          qp_wait(sh, &sh.o_full[1][s & 1], ((s - 2) >> 1) & 1);
        }
        store(vr, v_smem + (s & 1) * OPERAND);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) qp_arrive(&sh.v_full[s & 1]);
        load(vr, j + 1, ids1, 1);
        if (issuer) {                                   // the products of the step before and, behind each half's, the next logits
          if (j == 0) qp_wait(sh, &sh.q_full[0], piece & 1);
          else { qp_wait(sh, &sh.v_full[(s - 1) & 1], ((s - 1) >> 1) & 1); issue_pv(0, s - 1, j == 1); }
          qp_wait(sh, &sh.k_full[s & 1], (s >> 1) & 1);
          qp_fence_after();
          issue_qk(0, s);
          if (j == 0) qp_wait(sh, &sh.q_full[1], piece & 1);
          else issue_pv(1, s - 1, j == 1);
          issue_qk(1, s);
        }
        __syncwarp();
        ids = ids1; ids1 = ids2;
      }
      n += p.n_steps;
      if (issuer && p.n_steps > 0) {
        qp_wait(sh, &sh.v_full[(n - 1) & 1], ((n - 1) >> 1) & 1);
        issue_pv(0, n - 1, p.n_steps == 1);
        issue_pv(1, n - 1, p.n_steps == 1);
      }
      __syncwarp();
    }
    if (tid == QP_SOFT && join[0].x > 0) { a.joins[blockIdx.x * 2] = join[0]; a.joins[blockIdx.x * 2 + 1] = join[1]; }
  } else {                                              // ---- weights: a thread a column
    const int half = warp >> 2, t128 = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + T_S + half * 128, t_o = tmem + lanes + T_O + half * 128;
    int4 join[2];
    for (int piece = 0; walk.next(c, a, R, p, join); ++piece) {
      QtUnit u = p.u;                                   // of this half
      u.row0 += half * RT; u.slot0 += half * RT;
      u.rows = max(min(RT, u.rows - half * RT), 0);
      u.cols = u.rows * a.G;
      const bool used = u.cols > 0, real = t128 < u.cols;
      const int my = min(t128, max(u.cols - 1, 0));
      const int row = u.row0 + my / a.G, head = u.h * a.G + my % a.G;
      const int see = real ? qt_visible(c, u, a.G, t128) : 0x7fffffff;
      float qs = 0.f;                                   // what S is multiplied with
      if (used) {
        const unsigned short* src = a.q + (size_t)row * a.q_stride + (size_t)head * D;
        float mx = 0.f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(src + i * 8);
          for (uint32_t e : {w.x, w.y, w.z, w.w}) { const float2 x = qc_elems(e, a.f16); mx = fmaxf(mx, fmaxf(fabsf(x.x), fabsf(x.y))); }
        }
        const int ex = max((int)(__float_as_uint(mx) >> 23) - 127, -100), up = min(14 - ex, 114);    // largest magnitude to 2^14 .. 2^15, as in the other kernel
        const float mul = __uint_as_float((uint32_t)(127 + up) << 23);
        qs = 1.4426950408889634f * rsqrtf((float)D) * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          uint4 w = *reinterpret_cast<const uint4*>(src + i * 8);
          for (uint32_t* e : {&w.x, &w.y, &w.z, &w.w}) {
            const float2 x = qc_elems(*e, a.f16);
            const __half2 h = __floats2half2_rn(real ? x.x * mul : 0.f, real ? x.y * mul : 0.f);
            *e = *reinterpret_cast<const uint32_t*>(&h);
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_smem + half * OPERAND + (i >> 3) * QP_BLOCK + t128 * 128 + (((i & 7) ^ (t128 & 7)) << 4)),
                       "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w)
                       : "memory");
        }
        fence_proxy_async();
      }
      __syncwarp();
      if (lane == 0) qp_arrive(&sh.q_full[half]);
      float M = -INFINITY, L = 0.f;                     // M: less the lift
      float E = 0.f;                                    // set at the first step
      for (int j = 0; j < p.n_steps; ++j) {
        const int s = n + j;
        qp_wait(sh, &sh.sc_full[s & 3], (s >> 2) & 1);
        qp_wait(sh, &sh.s_full[half][s & 1], (s >> 1) & 1);
        qp_fence_after();
        if (used) {
          const float *ksp = sh.ks[s & 3], *evp = sh.ev[s & 3];
          const int t0 = u.t0 + j * QP_N;
          float top = -1000.f;
          bool gone = false;
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            if (ksp[g] < 0.f) gone = true;
            else top = fmaxf(top, evp[g]);
          }
          const bool masked = __any_sync(0xffffffffu, t0 + QP_N > see) || gone;      // some row does not see all of the step
          auto mask = [&](float* x, int at) {           // 32 columns
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = t0 + at + e < see && ksp[at / 16 + (e >> 4)] >= 0.f ? x[e] : -INFINITY;
          };
          auto factor = [&](int g) { return fmaxf(ksp[g] * qs, 1.2e-38f); };
          float mx = -INFINITY;                         // the largest s + ev of the step
          auto top_of = [&](const float* x, int g) {    // of 16 columns
            float m0 = qp_max3(x[0], x[1], x[2]), m1 = qp_max3(x[3], x[4], x[5]);
            m0 = qp_max3(m0, x[6], x[7]); m1 = qp_max3(m1, x[8], x[9]);
            m0 = qp_max3(m0, x[10], x[11]); m1 = qp_max3(m1, x[12], x[13]);
            m0 = qp_max3(m0, x[14], x[15]);
            mx = fmaxf(mx, fmaf(fmaxf(m0, m1), factor(g), evp[g]));
          };
          float x0[32], x1[32];
          qp_ld32(t_s + 96, x0);
          qp_ld32(t_s + 64, x1);
          qp_wait_ld();
          if (masked) { mask(x0, 96); mask(x1, 64); }
          top_of(x0, 6); top_of(x0 + 16, 7); top_of(x1, 4); top_of(x1 + 16, 5);
          qp_ld32(t_s + 32, x1);
          qp_ld32(t_s, x0);
          qp_wait_ld();
          if (masked) { mask(x1, 32); mask(x0, 0); }
          top_of(x1, 2); top_of(x1 + 16, 3); top_of(x0, 0); top_of(x0 + 16, 1);
          // maximum and E
          float dE = 0.f;
          if (top > -1000.f) {
            if (j == 0) E = top;
            else if (top > E + 40.f) { dE = top - E; E = top; }
          }
          const bool over = mx > M + (QP_LIFT + QP_SLACK);
          if (__any_sync(0xffffffffu, over || dE != 0.f)) {
            float corr = 1.f;
            if (over) {
              const float to = mx - QP_LIFT, by = M - to;      // (-infinity at first)
              corr = qt_exp2(by);
              L = L > 0.f ? L * qt_exp2(fminf(dE + by, 100.f)) : L * corr;
              M = to;
            } else if (dE != 0.f) {
              L *= qt_exp2(fminf(dE, 100.f));
            }
            if (j > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
              qp_wait(sh, &sh.o_full[half][(s - 1) & 1], ((s - 1) >> 1) & 1);      // all of O is there
              qp_fence_after();
#pragma unroll 1
              for (int g = 0; g < D / 32; ++g) {
                float o[32];
                qp_ld32(t_o + g * 32, o);
                qp_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] *= corr;
                qp_st32(t_o + g * 32, o);
              }
            }
          }
          const float zero = M == -INFINITY ? 0.f : M;
          auto weigh = [&](const float* x, int at) {    // weights of 32 columns to tensor memory
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const int g = at / 16 + hf;
              const float f1 = factor(g), b1 = evp[g] - zero;
              const uint64_t f = qp_pack2(f1, f1), b = qp_pack2(b1, b1);
              uint64_t sum = 0;
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                float p0, p1;
                qp_unpack2(qp_fma2(qp_pack2(x[hf * 16 + e], x[hf * 16 + e + 1]), f, b), p0, p1);
                p0 = qt_exp2(p0); p1 = qt_exp2(p1);
                sum = qp_add2(sum, qp_pack2(p0, p1));
                const __half2 h = __floats2half2_rn(p0, p1);
                hi[hf * 8 + e / 2] = *reinterpret_cast<const uint32_t*>(&h);
                if (TERMS == 2) {
                  const float2 b2 = __half22float2(h);
                  const __half2 r = __floats2half2_rn(p0 - b2.x, p1 - b2.y);
                  lo[hf * 8 + e / 2] = *reinterpret_cast<const uint32_t*>(&r);
                }
              }
              float s0, s1;
              qp_unpack2(sum, s0, s1);
              L = fmaf(s0 + s1, qt_exp2(fminf(E - evp[g], 100.f)), L);
            }
            qp_st16(t_s + at / 2, hi);
            if (TERMS == 2) qp_st16(t_s + 64 + at / 2, lo);
          };
          if (TERMS == 1) {
            weigh(x0, 0);
            qp_ld32(t_s + 64, x0);                      // (tokens 64 .. 127 lie where no weight has been written yet)
            weigh(x1, 32);
            qp_wait_ld();
            qp_ld32(t_s + 96, x1);
            if (masked) mask(x0, 64);
            weigh(x0, 64);
            qp_wait_ld();
            if (masked) mask(x1, 96);
            weigh(x1, 96);
          } else {                                      // second terms are written over those columns: all of them are read before
            float x2[32], x3[32];
            qp_ld32(t_s + 64, x2);
            qp_ld32(t_s + 96, x3);
            qp_wait_ld();
            if (masked) { mask(x2, 64); mask(x3, 96); }
            weigh(x0, 0);
            weigh(x1, 32);
            weigh(x2, 64);
            weigh(x3, 96);
          }
          qp_wait_st();
        }
        qp_fence_before();
        __syncwarp();
        if (lane == 0) qp_arrive(&sh.p_full[half]);
      }
      n += p.n_steps;
      if (p.n_steps > 0) {
        qp_wait(sh, &sh.o_full[half][(n - 1) & 1], ((n - 1) >> 1) & 1);
        qp_fence_after();
      }
      if (!used) continue;
      // out = 2^E O / L; a part of a result: 2^E O, M - E, L
      const float scale = exp2f(E), inv = L != 0.f ? scale / L : 0.f;      // (a NaN sum is not 0)
      float* parts = p.whole ? nullptr : a.part + (size_t)(blockIdx.x * 2 + (p.begins ? 0 : 1)) * QP_COLS * ST + (size_t)half * RT * a.G * ST;
      const size_t rh = ((size_t)row * a.Hq + head) * D;
      float* part = parts + (size_t)t128 * ST;
#pragma unroll 1
      for (int g = 0; g < D / 32; ++g) {
        float o[32];
        __syncwarp();
        if (p.n_steps > 0) {
          qp_ld32(t_o + g * 32, o);
          qp_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (!real) {
        } else if (parts) {
#pragma unroll
          for (int e = 0; e < 32; e += 2) *reinterpret_cast<float2*>(part + g * 32 + e) = make_float2(o[e] * scale, o[e + 1] * scale);
        } else if (a.out_type == GP_TYPE_F32) {
          float4* dst = reinterpret_cast<float4*>(static_cast<float*>(a.out) + rh + g * 32);
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[e] = make_float4(o[4 * e] * inv, o[4 * e + 1] * inv, o[4 * e + 2] * inv, o[4 * e + 3] * inv);
        } else {
          const bool f16 = a.out_type == GP_TYPE_F16;
          uint4* dst = reinterpret_cast<uint4*>(static_cast<unsigned short*>(a.out) + rh + g * 32);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dst[e] = make_uint4(qc_pack(o[8 * e] * inv, o[8 * e + 1] * inv, f16), qc_pack(o[8 * e + 2] * inv, o[8 * e + 3] * inv, f16),
                                qc_pack(o[8 * e + 4] * inv, o[8 * e + 5] * inv, f16), qc_pack(o[8 * e + 6] * inv, o[8 * e + 7] * inv, f16));
        }
      }
      if (parts && real) { part[D] = M == -INFINITY ? M : M - E; part[D + 1] = L; }
      if (*reinterpret_cast<volatile int*>(&sh.nan[piece & 1]) == piece)      // some row may have met another's NaN: all of the half in plain arithmetic
        qt_plain<D>(c, a, u, sh.plain[half], parts, 1 + half);
    }
  }
  qp_fence_before();
  __syncthreads();
  if (warp == QP_ISSUER) {
    qp_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  if (tid == 0 && sh.dead && c.status) atomicOr(c.status, GP_E_SPIN);
}

template <int D, int TERMS>
int qp_run(const QcDev& c, const QtArgs& a, const QpPlan& p, cudaStream_t s) {
  auto kern = qp_kernel<D, TERMS>;
  const size_t smem = 6 * (D / 64) * QP_BLOCK + 1024;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return GP_ERR_CUDA;
  if (gp_launch(kern, p.blocks, QP_THREADS, smem, s, false, c, a) != cudaSuccess) return GP_ERR_CUDA;
  if (p.blocks > 1 && gp_launch(qt_merge_kernel<D, QP_COLS, 2>, p.blocks * QP_COLS, D, 0, s, true, a) != cudaSuccess) return GP_ERR_CUDA;
  return GP_OK;
}

}  // namespace

QpPlan qp_plan(const QcDev& c, int G) {
  const int R = QP_COLS / G / 2 * 2;
  const long long units = (long long)c.n_seq * ((c.max_rows + R - 1) / R) * c.Hkv;
  const long long most = units * ((long long)c.limit + R + QP_UNIT);             // of the line, more than there can be
  const long long blocks = (most + 4 * QP_N - 1) / (4 * QP_N);
  QpPlan p;
  p.blocks = (int)(blocks < 148 ? blocks : 148);                                 // a block has an SM's tensor memory
  return p;
}
size_t qp_bytes(const QpPlan& p, int d) { return (size_t)p.blocks * 2 * (sizeof(int4) + (size_t)QP_COLS * (d + 2) * sizeof(float)); }
int qp_launch(const QcDev& c, QtArgs a, const QpPlan& p, int d, void* work, cudaStream_t s) {
  a.joins = static_cast<int4*>(work);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(work) + (size_t)p.blocks * 2 * sizeof(int4));
  if (d == 128) return a.out_type == GP_TYPE_F32 ? qp_run<128, 2>(c, a, p, s) : qp_run<128, 1>(c, a, p, s);
  return a.out_type == GP_TYPE_F32 ? qp_run<64, 2>(c, a, p, s) : qp_run<64, 1>(c, a, p, s);
}
