// The paged 4-bit key/value cache: where a vector lies, and the plan of a forward's rows.
//
// A vector x[DH] (the rotated key or the value of one token and kv head) is held as DH codes 0..15 and two bf16 numbers:
// zero, the largest not above min x, and scale, the smallest not below (max x - zero) / 15; it stands for
// zero + scale * code.  Rounding the two outwards keeps x inside [zero, zero + 15 scale] whatever its offset, so that the
// error is half a scale and not biased by the rounding of zero.
//
// Sixteen consecutive slots of a page are a granule, the unit that the attention kernels read: for each (page, kv head)
// [granule][K codes | V codes | parameters].  Codes come as 32-bit words of eight: word l of a vector holds dims
// 4l .. 4l+3 in nibbles 0..3 and dims DH/2 + 4l .. + 3 in nibbles 4..7 (both halves of a rotation pair, so that the
// thread that rotates has all eight).  Inside a granule words lie in the order in which the 32 lanes of a warp hold
// them as operand A of an m16n8k16 multiply, 16 bytes per lane and load, for K with slots as rows and dims as depth, for V with
// dims as rows and slots as depth: lane (g, t) = 4 g + t has
//   K: words [t * DH/32, (t + 1) * DH/32) of slots g and g + 8
//   V: words [g * DH/64, (g + 1) * DH/64) of slots 2t, 2t + 1, 2t + 8, 2t + 9
// and the parameters of slots g and g + 8 are 16 bytes: K of g, K of g + 8, V of g, V of g + 8 (scale low, zero high half).
#pragma once
#include "common.cuh"

namespace koala {

constexpr int KV4_G = 16;                       // slots per granule
constexpr int KV4_PARAMS = KV4_G * 8;           // bytes of a granule's parameters
__host__ __device__ constexpr int kv4_granule_bytes(int dh) { return KV4_G * dh + KV4_PARAMS; }

// Byte of word l of slot s (0..15) inside its granule.
template <int DH> __device__ __forceinline__ int kv4_k_at(int s, int l) {
  return DH == 128 ? s * 64 + l * 4 : (s & 7) * 64 + (l >> 1) * 16 + (s >> 3) * 8 + (l & 1) * 4;
}
template <int DH> __device__ __forceinline__ int kv4_v_at(int s, int l) {
  const int t = (s & 7) >> 1, odd = s & 1, hi = s >> 3;
  return KV4_G * DH / 2 + (DH == 128 ? hi * 512 + ((l >> 1) * 4 + t) * 16 + odd * 8 + (l & 1) * 4 : (l * 4 + t) * 16 + hi * 8 + odd * 4);
}
template <int DH> __device__ __forceinline__ int kv4_p_at(int s, int is_v) {
  return KV4_G * DH + (s & 7) * 16 + is_v * 8 + (s >> 3) * 4;
}

// The cache of one layer (of all layers: layer_bytes apart) and its page table.
struct Kv4Cache {
  unsigned char *pages;
  size_t layer_bytes;
  int n_layers, n_kv_heads, n_pages, gpp_shift;  // granules per page = 1 << gpp_shift
  const int32_t *table;                          // [B][table_stride] page of slots page_size * i ..; anything outside 0..n_pages-1: none
  int table_stride;
  // offset of granule g of sequence b and kv head h, or a negative number if the table gives no page
  template <int DH> __device__ __forceinline__ long long granule(int page, int h, int g) const {
    if ((unsigned)page >= (unsigned)n_pages) return -1;
    return (long long)((unsigned long long)number(page, h, g) * (unsigned)kv4_granule_bytes(DH));
  }
  // which of the layer's granules that is, for a page that exists (below 2^31: the host's check)
  __device__ __forceinline__ unsigned number(int page, int h, int g) const {
    return ((unsigned)(page * n_kv_heads + h) << gpp_shift) + (unsigned)(g & ((1 << gpp_shift) - 1));
  }
  __device__ __forceinline__ int page_of(int b, int g) const {
    const int i = g >> gpp_shift;
    return (g < 0 || i >= table_stride) ? -1 : table[(size_t)b * table_stride + i];
  }
};

// two floats at a time
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 both(float x, float y) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
  return d;
}
__device__ __forceinline__ float2 apart(f32x2 v) {
  float2 d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(v));
  return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Which rows a call works on, and of which sequences.
struct Kv4Rows {
  int B, total, max_rows;
  const int32_t *row_start;   // [B + 1]; null: max_rows rows each
  const int32_t *ctx_len;     // [B] slots that every row of the sequence sees; row i lies at slot ctx_len + i unless `slot` says otherwise
  const int32_t *kv_len;      // [B] slots in use; null: ctx_len + rows
  const int32_t *slot;        // [total], negative: row not in use; null
  const uint64_t *mask;       // [total][2] visibility of the slots ctx_len .. ctx_len + 127; null: slots up to the row's own
  const int32_t *seq;         // page-table row of each group of rows; null: its own index
  int *status;
  // rows of sequence b: [first, first + count)
  __device__ __forceinline__ void range(int b, int &first, int &count) const {
    if (row_start == nullptr) {
      first = b * max_rows;
      count = min(max_rows, total - first);
      return;
    }
    first = row_start[b];
    const int end = row_start[b + 1];
    const bool bad = first < 0 || end < first || end > total || end - first > max_rows;
    if (bad) report();
    count = bad ? 0 : end - first;
  }
  // sequence that row r belongs to, or -1
  __device__ __forceinline__ int sequence_of(int r) const {
    if (row_start == nullptr) return r / max_rows;
    int lo = 0, hi = B;                                    // row_start[lo] <= r < row_start[hi], if it is in order
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (row_start[mid] <= r) lo = mid;
      else hi = mid;
    }
    return row_start[lo] <= r && r < row_start[lo + 1] ? lo : -1;
  }
  // an impossible row_start need not give any row to anybody: one block looks at all of it
  __device__ __forceinline__ void check() const {
    if (status == nullptr || row_start == nullptr || blockIdx.x != 0 || blockIdx.y + 1 != gridDim.y || blockIdx.z != 0) return;
    for (int b = threadIdx.x; b < B; b += blockDim.x) {
      int first, count;
      range(b, first, count);
    }
  }
  __device__ __forceinline__ int cache_of(int b) const { return seq == nullptr ? b : seq[b]; }
  __device__ __forceinline__ void report() const {
    if (status != nullptr) atomicMax(status, 1);           // KOALA_E_INVALID
  }
};

// A strided [rows][heads][DH] tensor of one of the storage types; strides in elements.
struct Kv4Tensor {
  void *p;
  long long row, head;
};
// Where row r lies: its slot and page; page -1: it is to be left out.
struct Kv4Place {
  int slot, page, first, i, count;
};
__device__ __forceinline__ Kv4Place kv4_place(const Kv4Cache &c, const Kv4Rows &rows, int r) {
  Kv4Place p{-1, -1, 0, 0, 0};
  if (r >= rows.total) return p;
  const int b = rows.sequence_of(r);
  if (b < 0) return p;
  rows.range(b, p.first, p.count);
  p.i = r - p.first;
  if (p.i < 0 || p.i >= p.count) return p;
  p.slot = rows.slot != nullptr ? rows.slot[r] : rows.ctx_len[b] + p.i;
  if (p.slot < 0) {
    if (rows.slot == nullptr) rows.report();
    return p;
  }
  p.page = c.page_of(rows.cache_of(b), p.slot >> 4);
  if ((unsigned)p.page >= (unsigned)c.n_pages) {
    rows.report();
    p.page = -1;
  }
  return p;
}

enum { KV4_FP32 = 0, KV4_BF16 = 1, KV4_FP16 = 2, KV4_PAIR = 3 };   // PAIR: output as two bf16 tensors, value and rounding residual

}  // namespace koala
