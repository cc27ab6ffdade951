// Attention over the 8-bit cache for many rows of a sequence at once (chunks of prompts): both products on the fifth-generation tensor cores.
#include "gp_qprompt.cuh"

#include <utility>

namespace {

constexpr int QP_M = 128;                      // columns (row, query head of the group) of a half of a block's tile: the rows of a product
constexpr int QP_COLS = 2 * QP_M;
constexpr int QP_N = 64;                       // tokens of a step
constexpr int QP_RING = 4;                     // steps whose keys and values there is room for
constexpr int QP_SOFT = 256;                   // threads that turn logits into weights, a column each (warps 0 .. 7)
constexpr int QP_TURN = 3;                     // warps that turn keys into fp16, a step each in turn (8 .. 10); as many turn values (11 .. 13)
constexpr int QP_ISSUER = 14;                  // the first of the two warps that issue the products, one for each half
constexpr int QP_THREADS = QP_SOFT + (2 * QP_TURN + 2) * 32;
constexpr int QP_UNIT = 640;                   // what a unit costs beside its tokens, in tokens (chunks with 256 / 512 / 640 / 768 / 1024: 204 / 198 / 196 / 195 / 196 us;
                                               // six sequences of 100 to 700 rows: 202 / 158 / 146 / 146 / 150)
constexpr float QP_SLACK = 7.f;                // a row's maximum is brought up to date when something passes it by 2^7
constexpr float QP_LIFT = 8.f;
constexpr float QP_LAG = 30.f;                 // the maximum that the sum of weights refers to is brought up to date when a logit passes it by 2^30, or with the other
constexpr float QP_FAR = 80.f;
constexpr int QP_QBLOCK = QP_M * 128;          // bytes of 64 fp16 channels of the queries of a half
constexpr int QP_BLOCK = QP_N * 128;           // ... of the tokens of a step

__device__ __forceinline__ uint64_t qp_desc(uint32_t addr, uint32_t lbo) {      // shared-memory matrix, 128-byte swizzle, groups of 8 rows 1024 bytes apart
  return (uint64_t)((addr >> 4) & 0x3fff) | (uint64_t)((lbo >> 4) & 0x3fff) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// These are executed by a whole warp, whose control flow and operands are the same in all lanes (they then live in uniform registers; in a
// branch of a single lane each product waits for four of them to be moved); one lane issues.
__device__ __forceinline__ void qp_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
               "l"(a), "l"(b), "r"(idesc), "r"(add)
               : "memory");
}
__device__ __forceinline__ void qp_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {      // A in tensor memory
  asm volatile("{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
               "r"(a), "l"(b), "r"(idesc), "r"(add)
               : "memory");
}
__device__ __forceinline__ void qp_commit(uint32_t bar) {
  asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
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
template <int AT>
__device__ __forceinline__ void qp_store16(uint32_t to, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0 + %5], {%1, %2, %3, %4};" ::"r"(to), "r"(x), "r"(y), "r"(z), "r"(w), "n"(AT) : "memory");
}
// f(0) .. f(N - 1), each number a constant
template <class F, int... I>
__device__ __forceinline__ void qp_each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void qp_each(F&& f) { qp_each_of(f, std::make_integer_sequence<int, N>{}); }
// The two warps of weights of a scheduler (one of each half) take turns at the exponentials, so that one's wait, logits and maximum fall into the other's
// turn; left to themselves they run in step or not by chance (chunks of 32 768 tokens 608 to 657 us; 579 so).  Both make a turn of each step of a piece
// whether the half is used or not, and whether a wait gave up or not, and all their other waits are bounded: every turn comes.
__device__ __forceinline__ void qp_turn(int id) { __syncwarp(); asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void qp_pass(int id) { __syncwarp(); asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory"); }
// 32, 16, 8 columns of the warp's 32 lanes
__device__ __forceinline__ void qp_ld32(uint32_t t, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(t));
}
__device__ __forceinline__ void qp_st8(uint32_t t, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(t), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
               "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void qp_ld16(uint32_t t, float* x) {
  uint32_t* r = reinterpret_cast<uint32_t*>(x);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                 "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(t));
}
__device__ __forceinline__ void qp_st16(uint32_t t, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(t), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}

struct QpShared {
  // [half], and by the place of the step in its ring
  uint64_t q_full[2], k_full[QP_RING], v_full[QP_RING], k_free[QP_RING], v_free[QP_RING], s_full[2][QP_RING], p_full[2][2], o_full[2][QP_RING], end[2];
  uint32_t tmem;
  int dead;                                    // a wait ran out: all others do at once
  int nan[8];                                  // by the number of the piece: that number, where a value that not all rows see is no number
  alignas(16) float ks[2 * QP_RING][QP_N / 16], ev[2 * QP_RING][QP_N / 16];      // per group of 16 tokens: scale of the keys (-1: no such page), exponent of that of the values
  long long x1, share, upto[QP_THREADS], warp[QP_THREADS / 32];
  uint32_t least[8][128];                      // beside nan, per channel: ~piece << 9 | the least row of the tile that sees such a value (an earlier piece's is larger)
  float qs[2][QP_M];
};
// (Without a time to suspend for, which brings a second look and a timer to each try: 627 -> 608 us.)
__device__ __forceinline__ bool qp_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void qp_wait(QpShared& sh, const QtArgs& a, uint64_t* bar, uint32_t parity) {
  const uint32_t at = smem_u32(bar);
  if (qp_try(at, parity)) return;
  const long long since = clock64();
  while (!qp_try(at, parity))
    if (clock64() - since > a.patience || *reinterpret_cast<volatile int*>(&sh.dead)) { *reinterpret_cast<volatile int*>(&sh.dead) = 1; break; }
}
// Whether no wait of the block has given up; the same in all lanes.  In a block with one that has, all waits end at once: its warps that issue products leave at the next step
// and wait for what they issued, the others go through the rest of their steps and turns with whatever lies there, and no result is written.  (Asked for behind each wait
// of the issuing warps: chunks 218 us for 214; in every step by the warps that convert 3 more, by those of weights 7.)
__device__ __forceinline__ bool qp_alive(const QpShared& sh) { return !__any_sync(0xffffffffu, *reinterpret_cast<const volatile int*>(&sh.dead)); }

// The line of work (as in the other kernel): sequence by sequence, KV head by KV head, tile of rows by tile of rows, measured in tokens.  Tile t of
// a sequence has s + R (t + 1) + QP_UNIT of it, with R the rows of a tile and s the slot of the sequence's first row, so T tiles have
__device__ __forceinline__ long long qp_line(const QcSeq& q, int R, long long T) {
  return T * (max(q.slot0, 0) + QP_UNIT) + R * (T * (T + 1) / 2);
}
__device__ __forceinline__ long long qp_head_line(const QcSeq& q, int R, const QtArgs& a) {
  return q.rows * a.G > a.few ? qp_line(q, R, (q.rows + R - 1) / R) : 0;        // (few rows: the other kernel's)
}

struct QpPiece {                               // a stretch of a unit (one without steps has no number: nobody waits for another in it)
  QtUnit u;                                    // of all of the tile
  int n_steps;
  bool whole, begins;                          // all of the unit; at the start of the block's stretch
};
// Walks along a block's stretch of the line; every thread does, and keeps no more than its place between two pieces.
struct QpWalk {
  long long x;
  __device__ __forceinline__ bool start(const QcDev& c, const QtArgs& a, int R, QpShared& sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int run = (c.n_seq + QP_THREADS - 1) / QP_THREADS;
    long long up = 0;
    for (int s = tid * run; s < min((tid + 1) * run, c.n_seq); ++s) up += c.Hkv * qp_head_line(qc_seq(c, s), R, a);
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
    const long long share = max((all + gridDim.x - 1) / gridDim.x, 512ll);
    x = blockIdx.x * share;
    if (tid == 0) { sh.share = share; sh.x1 = min(all, x + share); }
    __syncthreads();
    return x < all;
  }
  // (one copy for all warps: code that runs once a unit is fetched anew each time)  join[0], [1]: what is to be joined at its end
  __device__ __noinline__ bool next(const QcDev& c, const QtArgs& a, int R, const QpShared& sh, QpPiece& p, int4* join) {
    const int run = (c.n_seq + QP_THREADS - 1) / QP_THREADS;
    const long long x1 = sh.x1, x0 = blockIdx.x * sh.share;
    for (;;) {
      if (x >= x1) return false;
      int lo = 0, hi = QP_THREADS - 1;                  // the run that x lies in: first with upto > x
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (sh.upto[mid] > x) hi = mid;
        else lo = mid + 1;
      }
      int seq = lo * run;
      long long xs = lo ? sh.upto[lo - 1] : 0;          // where sequence `seq` begins
      QcSeq sq = qc_seq(c, seq);
      long long per_head = qp_head_line(sq, R, a);
      while (x >= xs + per_head * c.Hkv) {
        xs += per_head * c.Hkv;
        sq = qc_seq(c, ++seq);
        per_head = qp_head_line(sq, R, a);
      }
      QtUnit& u = p.u;
      u.seq = seq;
      // quotients and roots from fp32, put right by whole numbers
      u.h = (int)__fdividef((float)(x - xs), (float)per_head);
      while (u.h > 0 && u.h * per_head > x - xs) --u.h;
      while ((u.h + 1) * per_head <= x - xs) ++u.h;
      const long long xh = xs + u.h * per_head;
      // the tile: the root of R T^2 / 2 + (s + QP_UNIT + R / 2) T = x - xh
      const float b = (float)(max(sq.slot0, 0) + QP_UNIT) + 0.5f * R;
      long long T = (long long)__fdividef(sqrtf(b * b + 2.f * R * (float)(x - xh)) - b, (float)R);
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
        int from = (int)__fdividef((float)xu, (float)sh.share);
        while (from > 0 && from * sh.share > xu) --from;
        while ((from + 1) * sh.share <= xu) ++from;
        join[0] = make_int4(u.cols, from * 2 + (xu == from * sh.share ? 0 : 1), from + 1, blockIdx.x);
        join[1] = make_int4(u.row0, u.h, 0, 0);
      }
      return true;
    }
  }
};

// A block takes tiles of up to 256 columns (row, query head of the group) of one (sequence, KV head), in two halves, and a stretch of their tokens,
// 64 at a step.  Per half:
//   S [128 columns x 64 tokens] = Q K^T       (tcgen05, fp16 in shared memory, S in tensor memory)
//   P = weights of S                           (four warps, a thread a column; fp16, over S in tensor memory)
//   O [128 columns x d] += P V                 (tcgen05, P from tensor memory, V in shared memory)
// There are two S of each half, so that the logits of the next step are there when the weights of one are done.  Six more warps bring codes in and
// write them to shared memory as fp16, which holds them exactly and unscaled: K and V in the same image (a token's channels along a row, 64 a
// swizzled 128 bytes), which the first product reads with the channels, the second with the tokens as inner dimension; four steps of them are there.
// A warp more for each half issues its products.
// Values that are no numbers: in steps that not all rows see whole they are put down as 0, with the least row that sees one per channel, whose results (and those of the
// rows behind) are set at the end.
// Scales of pages cost nothing per element: 16 columns of S lie in one page, so the keys' scale joins the factor of the logits s and the exponent e of
// the values' scale the constant that is added before the exponential: p' = 2^(s + e - M), M the running maximum of s + e of the tokens that the row sees.  O is then a plain
// sum of p' times codes.  The sum of weights has a maximum of its own, m of s: L = sum of 2^(s - m), taken of p' group by group times 2^(M - m - e).  M - m is a whole
// number (`apart`), so that O and L refer to each other exactly; M itself is not, and the largest p' is 2^8 when M is its own.  For L's sake no e counts as less than
// M - m - 80: a token of such a group has at most 2^-50 of the largest p' then (its values count for nothing either way), and keeps a weight down to 2^-46 of the
// largest.  out = 2^(M - m) O / L.
// Measured: 301 to 1101 rows of three sequences of up to 9000 tokens, 8 KV heads, groups of 4, d = 128 (165 GFLOP): 196 us, 842 TFLOP/s.
// What would bound it: 2 x 128 x 64 exponentials a step and SM (16 a cycle) against 2 x 128 x 64 x 2 d multiply-adds (4096 a cycle): with
// d = 128 the same, 1024 cycles.  What does: the chain of a warp's step (logits, their largest, exponentials, handing on), 2100 cycles for two
// warps a scheduler; and 20 000 cycles between two units.
template <int D, int TERMS>
__global__ void __launch_bounds__(QP_THREADS, 1)
qp_kernel(const __grid_constant__ QcDev c, const __grid_constant__ QtArgs a) {
  constexpr int CH = D / 16, ST = qt_part(D);
  constexpr int QOPERAND = D / 64 * QP_QBLOCK, OPERAND = D / 64 * QP_BLOCK;      // bytes of a half's Q, of a step's K or V in shared memory
  // tensor memory: two S (and P over them) and O of each half; the second terms of the weights over the S columns that P leaves free
  constexpr uint32_t T_S = 0, T_O = 256;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) QpShared sh;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = base, k_smem = base + 2 * QOPERAND, v_smem = k_smem + QP_RING * OPERAND;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int RT = QP_M / a.G, R = 2 * RT;                // rows of a half, of a tile

  if (tid == 0) {
    for (int h = 0; h < 2; ++h) {
      mbar_init(&sh.q_full[h], 4); mbar_init(&sh.end[h], 1);
      for (int i = 0; i < 2; ++i) mbar_init(&sh.p_full[h][i], 4);
      for (int i = 0; i < QP_RING; ++i) { mbar_init(&sh.s_full[h][i], 2); mbar_init(&sh.o_full[h][i], 2); }
    }
    for (int i = 0; i < QP_RING; ++i) { mbar_init(&sh.k_full[i], 1); mbar_init(&sh.v_full[i], 1); mbar_init(&sh.k_free[i], 2); mbar_init(&sh.v_free[i], 2); }
    for (int i = 0; i < 8; ++i) sh.nan[i] = -1;
    sh.dead = 0;
    fence_mbar_init();
    a.joins[blockIdx.x * 2] = make_int4(0, 0, 0, 0);
  }
  for (int i = tid; i < 8 * 128; i += QP_THREADS) sh.least[0][i] = ~0u;
  if (warp == QP_ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  qp_fence_before();
  QpWalk walk;
  const bool any = walk.start(c, a, R, sh);                // (meets twice)
  qp_fence_after();
  gp_pdl_launch_dependents();
  const uint32_t tmem = sh.tmem;
  int n = 0;                                            // steps before the piece
  QpPiece p;

  if (!any) {
  } else if (warp >= QP_ISSUER) {                       // ---- products of a half
    const uint32_t idesc = 1u << 4 | (QP_M / 16u) << 24, qk = idesc | (QP_N / 8u) << 17, pv = idesc | 1u << 16 | (D / 8u) << 17;
    const uint32_t half = __shfl_sync(0xffffffffu, (uint32_t)(warp - QP_ISSUER), 0), tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t dq = qp_desc(q_smem + half * QOPERAND, 16), dk = qp_desc(k_smem, 16), dv = qp_desc(v_smem, QP_BLOCK);
    const uint32_t t_s = tm + T_S + half * 128, t_o = tm + T_O + half * 128, s_full = smem_u32(&sh.s_full[half][0]), o_full = smem_u32(&sh.o_full[half][0]),
                   k_free = smem_u32(sh.k_free), v_free = smem_u32(sh.v_free);
    int4 join[2];
    join[0].x = 0;
    bool ok = true;
    for (int piece = 0; ok && walk.next(c, a, R, sh, p, join); piece += p.n_steps > 0) {
      const int steps = __shfl_sync(0xffffffffu, p.n_steps, 0), n0 = __shfl_sync(0xffffffffu, n, 0);
      const bool used = __shfl_sync(0xffffffffu, (int)(half == 0 || p.u.cols > RT * a.G), 0);
      if (steps > 0) qp_wait(sh, a, &sh.q_full[half], piece & 1);
      for (int j = 0; j <= steps && (ok = qp_alive(sh)); ++j) {                // the next logits, then the product with the weights of the step before
        const uint32_t s = n0 + j;
        if (j < steps) {
          qp_wait(sh, a, &sh.k_full[s & (QP_RING - 1)], (s / QP_RING) & 1);
          qp_fence_after();
          if (used) {
            const uint64_t k0 = dk + (s & (QP_RING - 1)) * (OPERAND >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              qp_mma_ss(t_s + (s & 1) * 64, dq + (((k >> 2) * QP_QBLOCK + (k & 3) * 32) >> 4), k0 + (((k >> 2) * QP_BLOCK + (k & 3) * 32) >> 4), qk, k > 0);
          }
          qp_commit(s_full + (s & (QP_RING - 1)) * 8);
          if (lane == 0) qp_arrive(&sh.s_full[half][s & (QP_RING - 1)]);      // hands on what it saw of the step: its scales
          qp_commit(k_free + (s & (QP_RING - 1)) * 8);
        }
        if (j > 0) {
          const uint32_t b = s - 1;
          qp_wait(sh, a, &sh.v_full[b & (QP_RING - 1)], (b / QP_RING) & 1);
          qp_wait(sh, a, &sh.p_full[half][b & 1], (b >> 1) & 1);
          qp_fence_after();
          if (used) {
            const uint64_t v0 = dv + (b & (QP_RING - 1)) * (OPERAND >> 4);
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
#pragma unroll
              for (int k = 0; k < QP_N / 16; ++k)
                qp_mma_ts(t_o, t_s + (b & 1) * 64 + t * 32 + k * 8, v0 + k * (2048 >> 4), pv, t > 0 || k > 0 ? 1u : (uint32_t)(j > 1));
          }
          qp_commit(o_full + (b & (QP_RING - 1)) * 8);
          if (lane == 0) qp_arrive(&sh.o_full[half][b & (QP_RING - 1)]);      // hands on, too: which values are no numbers
          qp_commit(v_free + (b & (QP_RING - 1)) * 8);
        }
      }
      n += p.n_steps;
    }
    qp_commit(smem_u32(&sh.end[half]));                 // all that was issued: before the tensor memory is given back and the block's shared memory ends
    const long long since = clock64();
    while (!__all_sync(0xffffffffu, qp_try(smem_u32(&sh.end[half]), 0)))
      if (__any_sync(0xffffffffu, clock64() - since > QT_PATIENCE)) { *reinterpret_cast<volatile int*>(&sh.dead) = 1; break; }
    if (ok && warp == QP_ISSUER && lane == 0 && join[0].x > 0) { a.joins[blockIdx.x * 2] = join[0]; a.joins[blockIdx.x * 2 + 1] = join[1]; }
  } else if (warp >= 8) {                               // ---- codes to fp16: three warps the keys, three the values, a step each in turn
    const int kv = (warp - 8) / QP_TURN, turn = (warp - 8) % QP_TURN;
    constexpr int TPI = 32 / CH;                        // tokens of a round: 4 or 8
    constexpr int IT = QP_N / TPI;
    const int ch = lane % CH, tt = lane / CH;           // piece of 16 channels; token in the round
    // its place in a row of 128 bytes, swizzled; the two halves of 128 channels write their two pieces in opposite order: no bank twice
    const int flip = (ch >> 2) & 1;
    const uint32_t dst = (kv ? v_smem : k_smem) + (ch >> 2) * QP_BLOCK + tt * 128, at0 = ((((ch & 3) * 2 + flip) ^ (tt & 7)) << 4), at1 = at0 ^ 16;
    const size_t page_bytes = (size_t)c.Hkv * 2 * c.page * D;
    const uint32_t full = smem_u32(kv ? sh.v_full : sh.k_full);
    uint64_t* empty = kv ? sh.v_free : sh.k_free;       // both halves' products have read what was there
    const bool hold = a.withhold & 2 && blockIdx.x == 0 && !kv;
    int4 join[2];
    for (int piece = 0; walk.next(c, a, R, sh, p, join); piece += p.n_steps > 0) {
      const QtUnit& u = p.u;
      const int vis0 = qt_visible(c, a, u, 0);        // of the first row: the least
      const uint8_t* src = c.codes + (size_t)(u.h * 2 + kv) * c.page * D + ch * 16;
      const int* table = c.table + (size_t)u.seq * c.stride;
      // lanes 0 .. 3: page of a group of 16 tokens of a step, as the table has it (looked at a turn later: nothing waits for it here)
      auto page_of = [&](int j) {
        const int t = u.t0 + j * QP_N + lane * 16;
        return lane < QP_N / 16 && t < u.t1 ? table[t >> c.page_log] : -1;
      };
      uint4 r[IT];
      float2 sc;
      auto load = [&](int j, int ids) {
        const int first = u.t0 + j * QP_N;
        if ((unsigned)ids >= (unsigned)c.n_pages) {
          if (lane < QP_N / 16 && first + lane * 16 < u.t1 && c.status) atomicOr(c.status, GP_E_BOUNDS);
          ids = -1;
        }
        const bool all = first + QP_N <= u.t1 && __all_sync(0xffffffffu, ids >= 0 || lane >= QP_N / 16);
        const int slot0 = first & (c.page - 1);
#pragma unroll
        for (int g = 0; g < QP_N / 16; ++g) {           // (a step's groups of 16 tokens lie in one page each)
          const int id = __shfl_sync(0xffffffffu, ids, g);
          const uint8_t* from = src + (size_t)max(id, 0) * page_bytes + (((slot0 + g * 16) & (c.page - 1)) + tt) * D;
          const int left = all ? 16 : id >= 0 ? u.t1 - first - g * 16 - tt : 0;
#pragma unroll
          for (int i = 0; i < 16 / TPI; ++i)
            r[g * (16 / TPI) + i] = i * TPI < left ? __ldg(reinterpret_cast<const uint4*>(from + i * TPI * D)) : make_uint4(0, 0, 0, 0);
        }
        sc = make_float2(-1.f, 1.f);
        if (!kv && ids >= 0) sc = *reinterpret_cast<const float2*>(c.scales + ((size_t)ids * c.Hkv + u.h) * 2);
      };
      const int j0 = (turn + QP_TURN - n % QP_TURN) % QP_TURN;      // its first step of the piece
      int next = page_of(j0);
      for (int j = j0 - QP_TURN; j < p.n_steps; j += QP_TURN) {      // what the turn before asked for, then what the next will want
        if (j >= 0) {
        const int s = n + j;
        const int at = s & (QP_RING - 1);
        bool nan = false;
        if (s >= QP_RING) qp_wait(sh, a, empty + at, ((s - QP_RING) / QP_RING) & 1);
        if (!kv) {
          const int slot = s & (2 * QP_RING - 1);       // (twice the ring: the weights of a step may still be computed when its keys are replaced)
          if (lane < QP_N / 16) { sh.ks[slot][lane] = sc.x; sh.ev[slot][lane] = (float)((int)((__float_as_uint(sc.y) >> 23) & 255) - 127); }
        } else if (u.t0 + (j + 1) * QP_N > vis0) {      // rows see different tokens of the step
#pragma unroll
          for (int i = 0; i < IT; ++i)
            nan |= (__vcmpeq4(r[i].x & 0x7f7f7f7f, 0x7f7f7f7f) | __vcmpeq4(r[i].y & 0x7f7f7f7f, 0x7f7f7f7f) | __vcmpeq4(r[i].z & 0x7f7f7f7f, 0x7f7f7f7f) |
                    __vcmpeq4(r[i].w & 0x7f7f7f7f, 0x7f7f7f7f)) != 0;
        }
        const uint32_t to = dst + at * OPERAND, to0 = to + at0, to1 = to + at1, odd0 = to + (at0 ^ 64), odd1 = to + (at1 ^ 64);
        qp_each<IT>([&](auto no) {
          constexpr int i = decltype(no)::value;
          const uint32_t xa = flip ? r[i].z : r[i].x, ya = flip ? r[i].w : r[i].y, xb = flip ? r[i].x : r[i].z, yb = flip ? r[i].y : r[i].w;
          constexpr bool odd = TPI == 4 && (i & 1);     // (token & 7 goes by the round too)
          qp_store16<i * TPI * 128>(odd ? odd0 : to0, e4m3x2_to_f16x2(xa), e4m3x2_hi_to_f16x2(xa), e4m3x2_to_f16x2(ya), e4m3x2_hi_to_f16x2(ya));
          qp_store16<i * TPI * 128>(odd ? odd1 : to1, e4m3x2_to_f16x2(xb), e4m3x2_hi_to_f16x2(xb), e4m3x2_to_f16x2(yb), e4m3x2_hi_to_f16x2(yb));
        });
        if (__any_sync(0xffffffffu, nan)) {             // values that are no numbers: 0, and who sees them
          __syncwarp();
#pragma unroll 1
          for (int i = lane; i < QP_N * D / 2; i += 32) {      // two channels of a token: [64 channels][token][swizzled piece of 8][pair]
            const int t = i / 32 % QP_N, c0 = i / (32 * QP_N) * 64 + ((i / 4 % 8) ^ (t & 7)) * 8 + i % 4 * 2;
            const uint32_t where = v_smem + at * OPERAND + i * 4;
            uint32_t w;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(where));
            const uint32_t bad = __vcmpgtu2(w & 0x7fff7fffu, 0x7c007c00u);
            if (!bad) continue;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(where), "r"(w & ~bad) : "memory");
            const uint32_t key = ~(uint32_t)piece << 9 | (uint32_t)max(u.t0 + j * QP_N + t + 1 - vis0, 0);
            if (bad & 1) atomicMin(&sh.least[piece & 7][c0], key);
            if (bad >> 16) atomicMin(&sh.least[piece & 7][c0 + 1], key);
          }
          *reinterpret_cast<volatile int*>(&sh.nan[piece & 7]) = piece;
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0 && !(hold && s == 0)) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full + at * 8) : "memory");
        }
        if (j + QP_TURN < p.n_steps) {
          load(j + QP_TURN, next);
          next = page_of(j + 2 * QP_TURN);
        }
      }
      n += p.n_steps;
    }
  } else {                                              // ---- weights: a thread a column
    const int half = warp >> 2, t128 = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + T_S + half * 128, t_o = tmem + lanes + T_O + half * 128;
    const int turn = 3 + (warp & 3) * 2;              // barriers 3 .. 10
    if (half) qp_pass(turn);
    bool ok = true;
    int4 join[2];
    for (int piece = 0; walk.next(c, a, R, sh, p, join); piece += p.n_steps > 0) {
      QtUnit u = p.u;                                   // of this half
      u.row0 += half * RT; u.slot0 += half * RT;
      u.rows = max(min(RT, u.rows - half * RT), 0);
      u.cols = u.rows * a.G;
      const bool used = u.cols > 0, real = t128 < u.cols;
      const int see = real ? qt_visible(c, a, u, t128) : 0x7fffffff;
      const int least = __reduce_min_sync(0xffffffffu, see);
      float qs = 0.f;                                   // what S is multiplied with
      if (used && ok && p.n_steps > 0) {                // the warp's 32 columns, D / 8 lanes a column
        constexpr int LPC = D / 8, CPR = 32 / LPC, ROUNDS = 32 / CPR;
        const int piece8 = lane % LPC;
        int col = (warp & 3) * 32 + lane / LPC;
        auto place = [&](int cc) { return q_smem + half * QOPERAND + (piece8 >> 3) * QP_QBLOCK + cc * 128 + (((piece8 & 7) ^ (cc & 7)) << 4); };
        // as they are, to where they will lie; then each brought to its scale there.  (Short loops: see QpWalk::next)
#pragma unroll 1
        for (int i = 0; i < ROUNDS; ++i, col += CPR) {
          const int r = qt_row(a, min(col, u.cols - 1)), cc = min(col, u.cols - 1);
          const unsigned short* from = a.q + (size_t)(u.row0 + r) * a.q_stride + (size_t)(u.h * a.G + cc - r * a.G) * D + piece8 * 8;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(place(col)), "l"(from), "r"(col < u.cols ? 16 : 0) : "memory");
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncwarp();
        col -= ROUNDS * CPR;
        const float root = 1.4426950408889634f * rsqrtf((float)D);
#pragma unroll 1
        for (int i = 0; i < ROUNDS; i += 4, col += 4 * CPR) {      // four at once: a chain of 400 cycles
          uint4 w[4];
          float mx[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[k].x), "=r"(w[k].y), "=r"(w[k].z), "=r"(w[k].w) : "r"(place(col + k * CPR)));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            mx[k] = 0.f;
            for (uint32_t e : {w[k].x, w[k].y, w[k].z, w[k].w}) { const float2 x = qc_elems(e, a.f16); mx[k] = fmaxf(mx[k], fmaxf(fabsf(x.x), fabsf(x.y))); }
          }
#pragma unroll
          for (int o = 1; o < LPC; o <<= 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], __shfl_xor_sync(0xffffffffu, mx[k], o));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int ex = max((int)(__float_as_uint(mx[k]) >> 23) - 127, -100), up = min(14 - ex, 114);    // largest magnitude to 2^14 .. 2^15, as in the other kernel
            const float mul = __uint_as_float((uint32_t)(127 + up) << 23);
            if (piece8 == 0) sh.qs[half][col + k * CPR] = root * __uint_as_float((uint32_t)(127 - up) << 23);
            for (uint32_t* e : {&w[k].x, &w[k].y, &w[k].z, &w[k].w}) {
              const float2 x = qc_elems(*e, a.f16);
              const __half2 h = __floats2half2_rn(x.x * mul, x.y * mul);
              *e = *reinterpret_cast<const uint32_t*>(&h);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place(col + k * CPR)), "r"(w[k].x), "r"(w[k].y), "r"(w[k].z), "r"(w[k].w) : "memory");
          }
        }
        fence_proxy_async();
        __syncwarp();
        qs = sh.qs[half][t128];
      }
      __syncwarp();
      if (lane == 0 && p.n_steps > 0) qp_arrive(&sh.q_full[half]);
      float M = -INFINITY, apart = 0.f, L = 0.f;        // M: less the lift; M - m
      for (int j = 0; j < p.n_steps; ++j) {
        const int s = n + j;
        const int slot = s & (2 * QP_RING - 1);
        qp_wait(sh, a, &sh.s_full[half][s & (QP_RING - 1)], (s / QP_RING) & 1);
        qp_fence_after();
        if (used) {
          const uint32_t t_x = t_s + (s & 1) * 64;
          const float4 kq = *reinterpret_cast<const float4*>(sh.ks[slot]), eq = *reinterpret_cast<const float4*>(sh.ev[slot]);
          const int t0 = u.t0 + j * QP_N;
          int masked = t0 + QP_N > least || fminf(fminf(kq.x, kq.y), fminf(kq.z, kq.w)) < 0.f;      // some row does not see all of the step
          const float ks[4] = {kq.x, kq.y, kq.z, kq.w};
          float ev[4] = {eq.x, eq.y, eq.z, eq.w};
          float f[4];
#pragma unroll
          for (int g = 0; g < 4; ++g) f[g] = fmaxf(ks[g] * qs, 1.2e-38f);
          float x0[32], x1[32];
#pragma unroll 1
          for (;;) {
            qp_ld32(t_x, x0);
            qp_ld32(t_x + 32, x1);
            qp_wait_ld();
            if (!masked) break;
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {               // -infinity where a row does not see a token, in tensor memory: two forms of x would cost 64 moves a step
              float x[16];
              qp_ld16(t_x + g * 16, x);
              qp_wait_ld();
              const int left = sh.ks[slot][g] < 0.f ? 0 : see - t0 - g * 16;
#pragma unroll
              for (int e = 0; e < 16; ++e) x[e] = e < left ? x[e] : -INFINITY;
              qp_st16(t_x + g * 16, reinterpret_cast<const uint32_t*>(x));
            }
            qp_wait_st();
            masked = 0;
            asm volatile("" : "+r"(masked));            // (or the compiler makes two of it)
          }
          float mx = -INFINITY, ms = -INFINITY;         // the step's largest s + e and s
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const float* x = (g & 2 ? x1 : x0) + (g & 1) * 16;
            float m0 = qp_max3(x[0], x[1], x[2]), m1 = qp_max3(x[3], x[4], x[5]);
            m0 = qp_max3(m0, x[6], x[7]); m1 = qp_max3(m1, x[8], x[9]);
            m0 = qp_max3(m0, x[10], x[11]); m1 = qp_max3(m1, x[12], x[13]);
            m0 = qp_max3(m0, x[14], x[15]);
            const float t = fmaxf(m0, m1) * f[g];
            ms = fmaxf(ms, t); mx = fmaxf(mx, t + ev[g]);
          }
          const bool over = mx > M + (QP_LIFT + QP_SLACK) || ms > M - apart + QP_LAG;
          if (__any_sync(0xffffffffu, over)) {
            float corr = 1.f;
            if (over) {
              const float to = fmaxf(M, mx - QP_LIFT), by = M - to, now = ceilf(to - fmaxf(M - apart, ms));      // (minus infinity at first; m may fall by less than 1)
              corr = qt_exp2(by);
              L *= qt_exp2(by + (now - apart));
              M = to; apart = now;
            }
            if (j > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
              qp_wait(sh, a, &sh.o_full[half][(s - 1) & (QP_RING - 1)], ((s - 1) / QP_RING) & 1);      // all of O is there
              qp_fence_after();
#pragma unroll 1
              for (int g = 0; g < D / 16; ++g) {
                float o[16];
                qp_ld16(t_o + g * 16, o);
                qp_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] *= corr;
                qp_st16(t_o + g * 16, reinterpret_cast<const uint32_t*>(o));
              }
            }
          }
          const float zero = M == -INFINITY ? 0.f : M;
#pragma unroll
          for (int g = 0; g < 4; ++g) ev[g] = fmaxf(ev[g], apart - QP_FAR);
          qp_turn(turn + half);
#pragma unroll
          for (int g = 0; g < 4; ++g) {                 // weights of 16 columns to tensor memory
            const float* x = (g & 2 ? x1 : x0) + (g & 1) * 16;
            const uint64_t ff = qp_pack2(f[g], f[g]), b = qp_pack2(ev[g] - zero, ev[g] - zero);
            uint64_t acc = 0;
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float p0, p1;
              qp_unpack2(qp_fma2(qp_pack2(x[e], x[e + 1]), ff, b), p0, p1);
              p0 = qt_exp2(p0); p1 = qt_exp2(p1);
              acc = qp_add2(acc, qp_pack2(p0, p1));
              const __half2 h = __floats2half2_rn(p0, p1);
              hi[e / 2] = *reinterpret_cast<const uint32_t*>(&h);
              if (TERMS == 2) {
                const float2 b2 = __half22float2(h);
                const __half2 r = __floats2half2_rn(p0 - b2.x, p1 - b2.y);
                lo[e / 2] = *reinterpret_cast<const uint32_t*>(&r);
              }
            }
            float s0, s1;
            qp_unpack2(acc, s0, s1);
            L = fmaf(s0 + s1, qt_exp2(apart - ev[g]), L);
            qp_st8(t_x + g * 8, hi);
            if (TERMS == 2) qp_st8(t_x + 32 + g * 8, lo);
          }
          qp_pass(turn + 1 - half);
          qp_wait_st();
        } else {
          qp_turn(turn + half);
          qp_pass(turn + 1 - half);
        }
        qp_fence_before();
        __syncwarp();
        if (lane == 0) qp_arrive(&sh.p_full[half][s & 1]);
      }
      n += p.n_steps;
      if (ok && p.n_steps > 0) {
        qp_wait(sh, a, &sh.o_full[half][(n - 1) & (QP_RING - 1)], ((n - 1) / QP_RING) & 1);
        ok = qp_alive(sh);
        qp_fence_after();
      }
      if (!used || !ok) continue;
      const bool nan = p.n_steps > 0 && *reinterpret_cast<volatile int*>(&sh.nan[piece & 7]) == piece;
      const int row = half * RT + qt_row(a, t128);
      float* parts = p.whole ? nullptr : a.part + (size_t)(blockIdx.x * 2 + (p.begins ? 0 : 1)) * QP_COLS * ST + (size_t)half * RT * a.G * ST;
      // by way of the memory of the warp's own 32 queries (no product reads them any more), so that lanes store what lies together
      const uint32_t stage = q_smem + half * QOPERAND + (warp & 3) * (32 * 128);
      auto place = [&](int col, int pc) { return stage + (pc >> 3) * QP_QBLOCK + col * 128 + (((pc & 7) ^ (col & 7)) << 4); };
      constexpr int PIECES = D / 8;                     // of 16 bytes, of a column there
      const bool wide = parts || a.out_type == GP_TYPE_F32;      // two rounds of half of the channels in 32 bits, else one of all in 16
      const float inv = parts ? 1.f : L != 0.f ? 1.f / L : 0.f, scale = parts ? 1.f : exp2f(apart);      // (a NaN sum is not 0)
#pragma unroll 1
      for (int round = 0; round < (wide ? 2 : 1); ++round) {
        const int chans = wide ? D / 2 : D;
#pragma unroll 1
        for (int g = 0; g < chans / 16; ++g) {
          float o[16];
          __syncwarp();
          if (p.n_steps > 0) {
            qp_ld16(t_o + round * (D / 2) + g * 16, o);
            qp_wait_ld();
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = o[e] * inv * scale;
          if (nan)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint32_t key = sh.least[piece & 7][round * (D / 2) + g * 16 + e];
              if (key >> 9 == (~(uint32_t)piece & 0x7fffffu) && (int)(key & 511) <= row) o[e] = __int_as_float(0x7fffffff);
            }
          if (wide) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place(lane, g * 4 + e)), "f"(o[4 * e]), "f"(o[4 * e + 1]),
                           "f"(o[4 * e + 2]), "f"(o[4 * e + 3])
                           : "memory");
          } else {
            const bool f16 = a.out_type == GP_TYPE_F16;
#pragma unroll
            for (int e = 0; e < 2; ++e)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(place(lane, g * 2 + e)), "r"(qc_pack(o[8 * e], o[8 * e + 1], f16)),
                           "r"(qc_pack(o[8 * e + 2], o[8 * e + 3], f16)), "r"(qc_pack(o[8 * e + 4], o[8 * e + 5], f16)), "r"(qc_pack(o[8 * e + 6], o[8 * e + 7], f16))
                           : "memory");
          }
        }
        __syncwarp();
#pragma unroll 1
        for (int i = 0; i < PIECES; i += 4) {           // 32 pieces a time
          const int pc = lane % PIECES;
          uint4 w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[k].x), "=r"(w[k].y), "=r"(w[k].z), "=r"(w[k].w)
                         : "r"(place((i + k) * (32 / PIECES) + lane / PIECES, pc)));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int cc = (warp & 3) * 32 + (i + k) * (32 / PIECES) + lane / PIECES;
            if (cc >= u.cols) continue;
            if (parts) {
              float2* to = reinterpret_cast<float2*>(parts + (size_t)cc * ST + round * (D / 2) + pc * 4);
              to[0] = make_float2(__uint_as_float(w[k].x), __uint_as_float(w[k].y));
              to[1] = make_float2(__uint_as_float(w[k].z), __uint_as_float(w[k].w));
            } else {
              uint8_t* to = static_cast<uint8_t*>(a.out) + qt_query(a, u, cc) * D * (wide ? 4 : 2);
              *reinterpret_cast<uint4*>(to + round * (2 * D) + pc * 16) = w[k];
            }
          }
        }
        __syncwarp();
      }
      if (parts && real) *reinterpret_cast<float4*>(parts + (size_t)t128 * ST + D) = make_float4(fmaxf(M - apart, QT_NONE), L, apart, 0.f);
    }
    if (!half) qp_turn(turn);
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
  const size_t smem = (D / 64) * (2 * QP_QBLOCK + 2 * QP_RING * QP_BLOCK) + 1024;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return GP_ERR_CUDA;
  if (gp_launch(kern, p.blocks, QP_THREADS, smem, s, false, c, a) != cudaSuccess) return GP_ERR_CUDA;
  if (p.blocks > 1 && gp_launch(qt_merge_kernel<D, QP_COLS, 2>, p.blocks * (QP_COLS / 4), 128, 0, s, true, a) != cudaSuccess) return GP_ERR_CUDA;
  return GP_OK;
}

}  // namespace

QpPlan qp_plan(const QcDev& c, int G) {
  const int R = QP_COLS / G / 2 * 2;
  const long long units = (long long)c.n_seq * ((c.max_rows + R - 1) / R) * c.Hkv;
  const long long most = units * ((long long)c.limit + R + QP_UNIT);             // of the line, more than there can be
  const long long blocks = (most + 511) / 512;
  QpPlan p;
  p.blocks = (int)(blocks < 148 ? blocks : 148);                                 // a block has an SM's tensor memory
  return p;
}
size_t qp_bytes(const QpPlan& p, int d) { return (size_t)p.blocks * 2 * (sizeof(int4) + (size_t)QP_COLS * qt_part(d) * sizeof(float)); }
int qp_launch(const QcDev& c, QtArgs a, const QpPlan& p, int d, void* work, cudaStream_t s) {
  a.joins = static_cast<int4*>(work);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(work) + (size_t)p.blocks * 2 * sizeof(int4));
  if (d == 128) return a.out_type == GP_TYPE_F32 ? qp_run<128, 2>(c, a, p, s) : qp_run<128, 1>(c, a, p, s);
  return a.out_type == GP_TYPE_F32 ? qp_run<64, 2>(c, a, p, s) : qp_run<64, 1>(c, a, p, s);
}
