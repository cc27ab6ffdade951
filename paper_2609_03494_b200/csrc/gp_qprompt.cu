// Attention over the 8-bit cache for many rows of a sequence at once (chunks of prompts): both products on the fifth-generation tensor cores.
#include "gp_qprompt.cuh"

namespace {

constexpr int QP_M = 128;                      // columns (row, query head of the group) of a block: the rows of its products
constexpr int QP_N = 128;                      // tokens of a step
constexpr int QP_SOFT = 128, QP_CONV = 128;    // threads that turn logits into weights, a row each; that turn codes into fp16
constexpr int QP_THREADS = QP_SOFT + QP_CONV;
constexpr int QP_ISSUER = 7;                   // warp whose first lane issues the products
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
  uint64_t q_full, k_full, v_full, s_full, p_full, o_full;
  uint32_t tmem;
  int dead;                                    // a wait ran out: all others end at once
  int nan;                                     // a value that is no number where rows see different tokens
  float ks[2][8], ev[2][8];                    // per step (two at a time) and group of 16 tokens: scale of the keys (-1: no such page), exponent of that of the values
};
// A bounded wait for a phase of a barrier.
__device__ __forceinline__ void qp_wait(QpShared& sh, uint64_t* bar, uint32_t parity) {
  for (unsigned spin = 0; !mbar_try_wait(bar, parity); ++spin)
    if (spin > GP_SPIN_LIMIT || *reinterpret_cast<volatile int*>(&sh.dead)) { *reinterpret_cast<volatile int*>(&sh.dead) = 1; break; }
}

// A block takes up to 128 columns (row, query head of the group) of one (sequence, KV head) and a stretch of its tokens, 128 at a step:
//   S [128 columns x 128 tokens] = Q K^T      (tcgen05, fp16 in shared memory, S in tensor memory)
//   P = weights of S                           (four warps, a thread a column; fp16, over S in tensor memory)
//   O [128 columns x d] += P V                 (tcgen05, P from tensor memory, V in shared memory)
// Four more warps bring codes in and write them to shared memory as fp16, which holds them exactly and unscaled: K and V in the same image (a
// token's channels along a row, 64 a swizzled 128 bytes), which the first product reads with the channels, the second with the tokens as inner
// dimension; one of their threads issues the products.  Two blocks fill an SM's tensor memory and take turns: while one computes weights, the other's
// products run.
// Scales of pages cost nothing per element: 16 columns of S lie in one page, so the keys' scale joins the factor of the logits and the exponent of
// the values' scale the constant that is added before the exponential: p' = 2^(s + ev - M), M the running maximum of s + ev.  O is then a plain
// sum of p' times codes.  The sum of weights L is taken of p' 2^(E - ev) group by group, with E (an exponent of about the size of the largest ev so far)
// keeping it in range; out = 2^E O / L.
// What bounds it: 128 x 128 exponentials a step and SM (16 a cycle) against 128 x 128 x 2 d multiply-adds (4096 a cycle), with d = 128 the same.
template <int D, int TERMS>
__global__ void __launch_bounds__(QP_THREADS, TERMS == 1 ? 2 : 1)
qp_kernel(const __grid_constant__ QcDev c, const __grid_constant__ QtArgs a, int tiles, int n_split) {
  constexpr int CH = D / 16, ST = D + 2;
  constexpr int OPERAND = D / 64 * QP_BLOCK;            // bytes of Q, K or V in shared memory
  constexpr uint32_t COLS = TERMS == 1 ? 256 : 512;
  constexpr uint32_t T_S = 0, T_O = 128, T_P = TERMS == 1 ? 0 : 256;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) QpShared sh;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = base, k_smem = base + OPERAND, v_smem = base + 2 * OPERAND;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  QtUnit u;
  int split, n_steps, step0;
  {
    int at = blockIdx.x;
    split = at % n_split; at /= n_split;
    u.h = at % c.Hkv; at /= c.Hkv;
    u.seq = at % c.n_seq;
    const QcSeq sq = qc_seq(c, u.seq);
    const int n_tiles = (sq.rows + a.rows_tile - 1) / a.rows_tile;
    const int tile = n_tiles - 1 - at / c.n_seq;        // the last rows, which see the most, first
    if (tile < 0) {
      if (tid == 0 && n_split > 1) a.joins[blockIdx.x * 2] = make_int4(0, 0, 0, 0);
      return;
    }
    u.row0 = sq.r0 + tile * a.rows_tile;
    u.rows = min(a.rows_tile, sq.rows - tile * a.rows_tile);
    u.cols = u.rows * a.G;
    u.slot0 = sq.slot0 + tile * a.rows_tile;
  }
  const int vis_all = max(qt_visible(c, u, a.G, u.cols - 1), 0);
  {
    const int all = (vis_all + QP_N - 1) / QP_N, per = (all + n_split - 1) / n_split;
    step0 = min(all, split * per);
    n_steps = min(all, step0 + per) - step0;
    u.t0 = step0 * QP_N;
    u.t1 = min(vis_all, u.t0 + n_steps * QP_N);
  }
  if (tid == 0 && n_split > 1) {
    const int b0 = blockIdx.x - split;
    a.joins[blockIdx.x * 2] = split ? make_int4(0, 0, 0, 0) : make_int4(u.cols, b0, b0 + 1, b0 + n_split - 1);
    a.joins[blockIdx.x * 2 + 1] = make_int4(u.row0, u.h, 0, 0);
  }
  if (tid == 0) {
    mbar_init(&sh.q_full, QP_SOFT / 32);
    mbar_init(&sh.k_full, QP_CONV / 32);
    mbar_init(&sh.v_full, QP_CONV / 32);
    mbar_init(&sh.s_full, 2);                           // the product, and the step's scales
    mbar_init(&sh.p_full, QP_SOFT / 32);
    mbar_init(&sh.o_full, 1);
    sh.dead = 0; sh.nan = 0;
    fence_mbar_init();
  }
  if (warp == QP_ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  qp_fence_before();
  __syncthreads();
  qp_fence_after();
  gp_pdl_launch_dependents();
  const uint32_t tmem = sh.tmem;

  if (warp >= 4) {                                      // ---- codes to fp16, products
    const int ct = tid - QP_SOFT, cw = warp - 4;
    constexpr int TPI = QP_CONV / CH;                   // tokens of a round
    constexpr int IT = QP_N / TPI;
    const int ch = ct % CH, tt = ct / CH;               // piece of 16 channels; token in the round
    const int vis0 = qt_visible(c, u, a.G, 0);          // of the first row: the least
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
        const int c0 = (ch & 3) * 2, flip = (ch >> 2) & 1;      // the two halves of 128 channels write their pieces in opposite order: no bank twice
        const uint4 x = r[i];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int hf = e ^ flip;
          const uint32_t w0 = hf ? x.z : x.x, w1 = hf ? x.w : x.y;
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + (((c0 + hf) ^ (t & 7)) << 4)), "r"(e4m3x2_to_f16x2(w0)), "r"(e4m3x2_hi_to_f16x2(w0)),
                       "r"(e4m3x2_to_f16x2(w1)), "r"(e4m3x2_hi_to_f16x2(w1))
                       : "memory");
        }
      }
    };
    const uint32_t idesc = 1u << 4 | (QP_M / 16u) << 24, qk = idesc | (QP_N / 8u) << 17, pv = idesc | 1u << 16 | (D / 8u) << 17;
    auto issue_qk = [&](int j) {
      qp_wait(sh, &sh.k_full, j & 1);
      qp_fence_after();
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t off = (k >> 2) * QP_BLOCK + (k & 3) * 32;
        qp_mma_ss(tmem + T_S, qp_desc(q_smem + off, 16), qp_desc(k_smem + off, 16), qk, k > 0);
      }
      qp_commit(&sh.s_full);
    };
    auto issue_pv = [&](int j) {
      qp_wait(sh, &sh.v_full, j & 1);
      qp_wait(sh, &sh.p_full, j & 1);
      qp_fence_after();
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int k = 0; k < QP_N / 16; ++k)
          qp_mma_ts(tmem + T_O, tmem + T_P + t * 64 + k * 8, qp_desc(v_smem + k * 2048, QP_BLOCK), pv, j > 0 || t > 0 || k > 0);
      qp_commit(&sh.o_full);
    };
    auto put_k = [&](const uint4* r, int j, int ids) {
      if (cw == 0) {
        float2 sc = make_float2(-1.f, 1.f);
        if (ids >= 0) sc = *reinterpret_cast<const float2*>(c.scales + ((size_t)ids * c.Hkv + u.h) * 2);
        if (lane < 8) { sh.ks[j & 1][lane] = sc.x; sh.ev[j & 1][lane] = (float)((int)((__float_as_uint(sc.y) >> 23) & 255) - 127); }
        __syncwarp();
        if (lane == 0) qp_arrive(&sh.s_full);
      }
      store(r, k_smem);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) qp_arrive(&sh.k_full);
    };
    auto put_v = [&](const uint4* r, int j) {
      if (u.t0 + (j + 1) * QP_N > vis0) {               // rows see different tokens of the step
        bool nan = false;
#pragma unroll
        for (int i = 0; i < IT; ++i)
          nan |= (__vcmpeq4(r[i].x & 0x7f7f7f7f, 0x7f7f7f7f) | __vcmpeq4(r[i].y & 0x7f7f7f7f, 0x7f7f7f7f) | __vcmpeq4(r[i].z & 0x7f7f7f7f, 0x7f7f7f7f) |
                  __vcmpeq4(r[i].w & 0x7f7f7f7f, 0x7f7f7f7f)) != 0;
        if (nan) *reinterpret_cast<volatile int*>(&sh.nan) = 1;
      }
      store(r, v_smem);
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) qp_arrive(&sh.v_full);
    };
    const bool issuer = warp == QP_ISSUER && lane == 0;
    uint4 kr[IT], vr[IT];
    if (n_steps > 0) {
      int ids = page_of(0), ids1 = page_of(1);
      load(kr, 0, ids, 0);
      load(vr, 0, ids, 1);
      put_k(kr, 0, ids);
      load(kr, 1, ids1, 0);
      if (issuer) { qp_wait(sh, &sh.q_full, 0); issue_qk(0); }
      __syncwarp();
      put_v(vr, 0);
      load(vr, 1, ids1, 1);
      for (int j = 0; j < n_steps; ++j) {
        const int ids2 = page_of(j + 2);
        if (j + 1 < n_steps) {
          qp_wait(sh, &sh.s_full, j & 1);               // the step's product has read the keys' memory
          put_k(kr, j + 1, ids1);
          load(kr, j + 2, ids2, 0);
        }
        if (issuer) {
          issue_pv(j);
          if (j + 1 < n_steps) issue_qk(j + 1);
        }
        __syncwarp();
        if (j + 1 < n_steps) {
          qp_wait(sh, &sh.o_full, j & 1);
          put_v(vr, j + 1);
          load(vr, j + 2, ids2, 1);
        }
        ids1 = ids2;
      }
    }
  } else {                                              // ---- weights: a thread a column
    const int col = tid;
    const bool real = col < u.cols;
    const int row = u.row0 + min(col, u.cols - 1) / a.G, head = u.h * a.G + min(col, u.cols - 1) % a.G;
    const int see = real ? qt_visible(c, u, a.G, col) : 0x7fffffff;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    float qs;                                           // what S is multiplied with
    {
      const unsigned short* src = a.q + (size_t)row * a.q_stride + (size_t)head * D;
      float mx = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint4 w = *reinterpret_cast<const uint4*>(src + i * 8);
        for (uint32_t e : {w.x, w.y, w.z, w.w}) { const float2 x = qc_elems(e, a.f16); mx = fmaxf(mx, fmaxf(fabsf(x.x), fabsf(x.y))); }
      }
      const int ex = max((int)(__float_as_uint(mx) >> 23) - 127, -100), up = min(14 - ex, 114);      // largest magnitude to 2^14 .. 2^15, as in the other kernel
      const float mul = real ? __uint_as_float((uint32_t)(127 + up) << 23) : 0.f;
      qs = 1.4426950408889634f * rsqrtf((float)D) * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        uint4 w = *reinterpret_cast<const uint4*>(src + i * 8);
        for (uint32_t* e : {&w.x, &w.y, &w.z, &w.w}) {
          const float2 x = qc_elems(*e, a.f16);
          const __half2 h = __floats2half2_rn(real ? x.x * mul : 0.f, real ? x.y * mul : 0.f);
          *e = *reinterpret_cast<const uint32_t*>(&h);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_smem + (i >> 3) * QP_BLOCK + col * 128 + (((i & 7) ^ (col & 7)) << 4)), "r"(w.x), "r"(w.y), "r"(w.z),
                     "r"(w.w)
                     : "memory");
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) qp_arrive(&sh.q_full);
    }
    float M = -INFINITY, L = 0.f;                       // M: less the lift
    float E = 0.f;                                      // set at the first step
    for (int j = 0; j < n_steps; ++j) {
      qp_wait(sh, &sh.s_full, j & 1);
      qp_fence_after();
      const int t0 = u.t0 + j * QP_N;
      const bool part = t0 + QP_N > see;                // the row does not see all of the step
      float kf[8], ev[8];
      float top = -1000.f;
      bool gone = false;
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        kf[g] = sh.ks[j & 1][g]; ev[g] = sh.ev[j & 1][g];
        if (kf[g] < 0.f) { gone = true; ev[g] = 0.f; }
        else top = fmaxf(top, ev[g]);
      }
      const bool masked = __any_sync(0xffffffffu, part) || gone;
      // the largest s + ev of the step
      float mx = -INFINITY;
#pragma unroll
      for (int g2 = 0; g2 < 4; ++g2) {
        float s[32];
        qp_ld32(tmem + lanes + T_S + g2 * 32, s);
        qp_wait_ld();
        if (masked) {
#pragma unroll
          for (int e = 0; e < 32; ++e) s[e] = t0 + g2 * 32 + e < see && kf[g2 * 2 + (e >> 4)] >= 0.f ? s[e] : -INFINITY;
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          float m = s[hf * 16];
#pragma unroll
          for (int e = 1; e < 16; ++e) m = fmaxf(m, s[hf * 16 + e]);
          mx = fmaxf(mx, fmaf(m, fmaxf(kf[g2 * 2 + hf] * qs, 1.2e-38f), ev[g2 * 2 + hf]));
        }
      }
      // maximum and E
      float dE = 0.f;
      if (top > -1000.f) {
        if (j == 0) { E = top; }
        else if (top > E + 40.f) { dE = top - E; E = top; }
      }
      const bool over = mx > M + (QP_LIFT + QP_SLACK);
      if (__any_sync(0xffffffffu, over || dE != 0.f)) {
        float corr = 1.f;
        if (over) {
          const float n = mx - QP_LIFT;
          const float by = M - n;                       // (-infinity at first)
          corr = qt_exp2(by);
          L = L > 0.f ? L * qt_exp2(fminf(dE + by, 100.f)) : L * corr;
          M = n;
        } else if (dE != 0.f) {
          L *= qt_exp2(fminf(dE, 100.f));
        }
        if (j > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
          qp_wait(sh, &sh.o_full, (j - 1) & 1);         // all of O is there
          qp_fence_after();
#pragma unroll
          for (int g = 0; g < D / 32; ++g) {
            float o[32];
            qp_ld32(tmem + lanes + T_O + g * 32, o);
            qp_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= corr;
            qp_st32(tmem + lanes + T_O + g * 32, o);
          }
        }
      }
      const float zero = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int g2 = 0; g2 < 4; ++g2) {
        float s[32];
        qp_ld32(tmem + lanes + T_S + g2 * 32, s);
        qp_wait_ld();
        if (masked) {
#pragma unroll
          for (int e = 0; e < 32; ++e) s[e] = t0 + g2 * 32 + e < see && kf[g2 * 2 + (e >> 4)] >= 0.f ? s[e] : -INFINITY;
        }
        uint32_t hi[16], lo[16];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float f = fmaxf(kf[g2 * 2 + hf] * qs, 1.2e-38f), b = ev[g2 * 2 + hf] - zero;
          float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float p0 = qt_exp2(fmaf(s[hf * 16 + e], f, b)), p1 = qt_exp2(fmaf(s[hf * 16 + e + 1], f, b));
            sum0 += p0; sum1 += p1;
            const __half2 h = __floats2half2_rn(p0, p1);
            hi[hf * 8 + e / 2] = *reinterpret_cast<const uint32_t*>(&h);
            if (TERMS == 2) {
              const float2 b2 = __half22float2(h);
              const __half2 r = __floats2half2_rn(p0 - b2.x, p1 - b2.y);
              lo[hf * 8 + e / 2] = *reinterpret_cast<const uint32_t*>(&r);
            }
          }
          L = fmaf(sum0 + sum1, qt_exp2(fminf(E - ev[g2 * 2 + hf], 100.f)), L);
        }
        qp_st16(tmem + lanes + T_P + g2 * 16, hi);
        if (TERMS == 2) qp_st16(tmem + lanes + T_P + 64 + g2 * 16, lo);
      }
      qp_wait_st();
      qp_fence_before();
      __syncwarp();
      if (lane == 0) qp_arrive(&sh.p_full);
    }
    if (n_steps > 0) {
      qp_wait(sh, &sh.o_full, (n_steps - 1) & 1);
      qp_fence_after();
    }
    // out = 2^E O / L; a part of a result: 2^E O, M - E, L
    const float scale = exp2f(E), inv = L != 0.f ? scale / L : 0.f;      // (a NaN sum is not 0)
    float* part = n_split > 1 ? a.part + ((size_t)blockIdx.x * QP_M + col) * ST : nullptr;
    const size_t rh = ((size_t)row * a.Hq + head) * D;
#pragma unroll
    for (int g = 0; g < D / 32; ++g) {
      float o[32];
      __syncwarp();
      if (n_steps > 0) {
        qp_ld32(tmem + lanes + T_O + g * 32, o);
        qp_wait_ld();
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
      }
      if (!real) {
      } else if (part) {
#pragma unroll
        for (int e = 0; e < 32; ++e) part[g * 32 + e] = o[e] * scale;
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
    if (part && real) { part[D] = M == -INFINITY ? M : M - E; part[D + 1] = L; }
  }
  qp_fence_before();
  __syncthreads();
  if (warp == QP_ISSUER) {
    qp_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
  }
  if (tid == 0 && sh.dead && c.status) atomicOr(c.status, GP_E_SPIN);
  if (sh.nan && warp < QT_WARPS)                        // some row may have met another's NaN: all of the block in plain arithmetic
    qt_plain<D>(c, a, u, reinterpret_cast<float*>(smem_raw), n_split > 1 ? a.part + (size_t)blockIdx.x * QP_M * ST : nullptr);
}

template <int D, int TERMS>
int qp_run(const QcDev& c, const QtArgs& a, const QpPlan& p, cudaStream_t s) {
  auto kern = qp_kernel<D, TERMS>;
  size_t smem = 3 * (D / 64) * QP_BLOCK + 1024;
  if (TERMS == 2 && smem < 120 * 1024) smem = 120 * 1024;      // one block an SM: it holds all of its tensor memory
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return GP_ERR_CUDA;
  if (gp_launch(kern, (int)p.blocks, QP_THREADS, smem, s, false, c, a, p.tiles, p.n_split) != cudaSuccess) return GP_ERR_CUDA;
  if (p.n_split > 1 && gp_launch(qt_merge_kernel<D, QP_M, 1>, (int)p.blocks * QP_M, D, 0, s, true, a) != cudaSuccess) return GP_ERR_CUDA;
  return GP_OK;
}

}  // namespace

QpPlan qp_plan(const QcDev& c, int G) {
  QpPlan p;
  p.rows_tile = QP_M / G;
  p.tiles = (c.max_rows + p.rows_tile - 1) / p.rows_tile;
  const long long units = (long long)c.n_seq * p.tiles * c.Hkv;
  // two blocks an SM; where there are fewer units, their tokens are split, no shorter than four steps
  long long n = units > 0 && units < 296 ? 296 / units : 1;
  const long long most = ((long long)c.limit + 4 * QP_N - 1) / (4 * QP_N);
  if (n > most) n = most;
  p.n_split = (int)(n < 1 ? 1 : n);
  p.blocks = units * p.n_split;
  return p;
}
size_t qp_bytes(const QpPlan& p, int d) {
  return p.n_split > 1 ? (size_t)p.blocks * (2 * sizeof(int4) + (size_t)QP_M * (d + 2) * sizeof(float)) : 0;
}
int qp_launch(const QcDev& c, QtArgs a, const QpPlan& p, int d, void* work, cudaStream_t s) {
  if (p.blocks * QP_M > 0x7fffffff) return GP_ERR_INVALID;
  a.joins = static_cast<int4*>(work);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(work) + (size_t)p.blocks * 2 * sizeof(int4));
  a.rows_tile = p.rows_tile;
  if (d == 128) return a.out_type == GP_TYPE_F32 ? qp_run<128, 2>(c, a, p, s) : qp_run<128, 1>(c, a, p, s);
  return a.out_type == GP_TYPE_F32 ? qp_run<64, 2>(c, a, p, s) : qp_run<64, 1>(c, a, p, s);
}
