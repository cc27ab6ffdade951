// What the calls of the 8-bit cache (gp_qcache_append, gp_qcache_select, gp_qcache_attention) share: the device view of cache and
// batch, the checks of the arguments, the conversions between e4m3 and wider types.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/growpage.h"
#include "gp_dev.cuh"

#define QC_E_MIN (-117)        // the smallest code 2^-9 in the smallest scale is the smallest normal fp32 and bf16 number
#define QC_E_MAX 119           // 448 * 2^119 is the largest code times a power of two that fp32 holds

#define QC_MAX_LEN 0x7fff0000  // slots, and places of a list times the page size: what is added to them on the way stays below 2^31

struct QcDev {                 // a gp_qcache and a gp_qbatch as the kernels take them
  uint8_t* codes;
  float* scales;
  uint8_t* bounds;
  int* status;
  const int* row_start;
  const int* seq_len;
  const int* table;
  long long n_pages;
  int Hkv, page, page_log, n_seq, stride, n_rows, max_rows, limit;     // limit: tokens of a sequence that are looked at, at most
};

// Rows of a sequence, as every kernel reads them.
struct QcSeq {
  int r0, rows;                // first row in the batch's tensors; rows that are looked at
  int slot0;                   // slot of the first row (negative where the sequence claims fewer tokens than rows)
};
__device__ __forceinline__ QcSeq qc_seq(const QcDev& c, int s) {
  QcSeq q;
  const int a = c.row_start[s], b = c.row_start[s + 1], n = max(c.seq_len[s], 0);
  q.r0 = min(max(a, 0), c.n_rows);
  const int all = max(min(b, c.n_rows) - q.r0, 0);
  q.rows = min(all, c.max_rows);
  q.slot0 = n - all;
  return q;
}
// page id of place `lp` of a sequence's table, -1 (and a bit in the status word) where it is none of the cache's
__device__ __forceinline__ int qc_page(const QcDev& c, int s, int lp) {
  const int id = c.table[(size_t)s * c.stride + lp];
  if ((unsigned)id < (unsigned)c.n_pages) return id;
  if (c.status) atomicOr(c.status, GP_E_BOUNDS);
  return -1;
}
// The sequence a row belongs to (-1: none): every thread of the block looks at some of the sequences, s_out is shared memory.  One round
// trip, where a binary search would take one per level.
__device__ __forceinline__ int qc_seq_of_row(const QcDev& c, int row, int* s_out) {
  if (threadIdx.x == 0) *s_out = -1;
  __syncthreads();
  for (int s = threadIdx.x; s < c.n_seq; s += blockDim.x) {
    const QcSeq q = qc_seq(c, s);
    if (row >= q.r0 && row < q.r0 + q.rows) *s_out = s;
  }
  __syncthreads();
  return *s_out;
}

// two e4m3 codes (low and high byte) to two fp16 numbers: exact, NaN to NaN
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_hi_to_f16x2(uint32_t four) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(four));
  return r;
}
// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col)
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D = A B
__device__ __forceinline__ void mma_f16_first(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// four fp32 numbers to e4m3: to nearest, at most 448 in magnitude, NaN to NaN; an infinite one to NaN
__device__ __forceinline__ uint32_t qc_codes(float a, float b, float c, float d) {
  auto fin = [](float x) { return fabsf(x) < INFINITY ? x : __int_as_float(0x7fffffff); };
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "f"(fin(a)), "f"(fin(b)), "f"(fin(c)), "f"(fin(d)));
  return r;
}
__device__ __forceinline__ uint32_t f16x4_to_e4m3x4(uint32_t lo2, uint32_t hi2) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f16x2 lo, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 hi, %2;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "r"(lo2), "r"(hi2));
  return r;
}
__device__ __forceinline__ float2 qc_half2(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// two 16-bit elements of a batch's tensors
__device__ __forceinline__ float2 qc_elems(uint32_t w, bool f16) {
  return f16 ? qc_half2(w) : make_float2(bf16_lo_f(w), bf16_hi_f(w));
}
__device__ __forceinline__ float qc_elem(unsigned short w, bool f16) {
  return f16 ? __half2float(__ushort_as_half(w)) : __uint_as_float((uint32_t)w << 16);
}
__device__ __forceinline__ uint32_t qc_pack(float a, float b, bool f16) {
  if (f16) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
  return pack_bf16(a, b);
}

// ---- host -------------------------------------------------------------------------------------------------
inline bool qc_misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Arguments of cache and batch that all three calls check; fills the device view.
inline int qc_check(const gp_qcache* c, const gp_qbatch* b, QcDev* d) {
  if (!c || !b || !c->codes || !c->scales) return GP_ERR_INVALID;
  if (b->n_seq > 0 && b->n_rows > 0 && (!b->row_start || !b->seq_len || !b->page_table)) return GP_ERR_INVALID;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || (c->head_dim != 64 && c->head_dim != 128)) return GP_ERR_INVALID;
  if (c->page_size < 16 || c->page_size > GP_MAX_BLK || (c->page_size & (c->page_size - 1))) return GP_ERR_INVALID;
  if (c->n_pages < 1 || c->n_pages > 0x7fffffff || c->device < 0) return GP_ERR_INVALID;
  if (qc_misaligned(c->codes, 16) || qc_misaligned(c->scales, 8) || qc_misaligned(c->bounds, 16) || qc_misaligned(c->status, 4)) return GP_ERR_INVALID;
  if (b->n_seq < 0 || b->table_stride < 1 || b->n_rows < 0 || b->max_rows < 0 || b->max_len < 0 || b->reserved) return GP_ERR_INVALID;
  if (qc_misaligned(b->row_start, 4) || qc_misaligned(b->seq_len, 4) || qc_misaligned(b->page_table, 4)) return GP_ERR_INVALID;
  d->codes = static_cast<uint8_t*>(c->codes);
  d->scales = c->scales;
  d->bounds = static_cast<uint8_t*>(c->bounds);
  d->status = c->status;
  d->row_start = b->row_start; d->seq_len = b->seq_len; d->table = b->page_table;
  d->n_pages = c->n_pages;
  d->Hkv = c->n_kv_heads; d->page = c->page_size;
  d->page_log = 0;
  while ((1 << d->page_log) < c->page_size) ++d->page_log;
  d->n_seq = b->n_seq; d->stride = b->table_stride; d->n_rows = b->n_rows;
  d->max_rows = b->max_rows < b->n_rows ? b->max_rows : b->n_rows;
  const long long room = (long long)b->table_stride * c->page_size;
  if (room > QC_MAX_LEN && b->max_len > QC_MAX_LEN) return GP_ERR_TOO_LARGE;
  d->limit = room < b->max_len ? (int)room : b->max_len;
  return GP_OK;
}
inline bool qc_empty(const QcDev& d) { return d.n_seq == 0 || d.n_rows == 0 || d.max_rows == 0; }
inline bool qc_check_q(const gp_qcache* c, const void* q, int64_t q_stride, int32_t n_q_heads, int32_t type) {
  return !qc_misaligned(q, 16) && n_q_heads >= c->n_kv_heads && n_q_heads % c->n_kv_heads == 0 && n_q_heads / c->n_kv_heads <= 8 &&
         q_stride >= (int64_t)n_q_heads * c->head_dim && q_stride % 8 == 0 && (type == GP_TYPE_BF16 || type == GP_TYPE_F16);
}

// The cache's device is current while this lives.
struct QcDevice {
  int before = -1;
  bool ok = false;
  explicit QcDevice(int device) {
    if (cudaGetDevice(&before) != cudaSuccess) return;
    ok = before == device || cudaSetDevice(device) == cudaSuccess;
    if (before == device) before = -1;
  }
  ~QcDevice() { if (before >= 0) cudaSetDevice(before); }
};
