// Writing, moving and reading rows of the paged 4-bit cache (kv4.cuh has the format).
#include <cuda_fp16.h>

#include "kv4.h"

namespace koala {
namespace {

template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };
__device__ __forceinline__ float up(float v) { return v; }
__device__ __forceinline__ float up(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float up(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T down(float v);
template <> __device__ __forceinline__ float down<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 down<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half down<__half>(float v) { return __float2half_rn(v); }

template <typename T> __device__ __forceinline__ void load4(const T *p, float *x) {
  const Four<T> f = *reinterpret_cast<const Four<T> *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = up(f.v[i]);
}
template <typename T> __device__ __forceinline__ void store4(T *p, const float *x) {
  Four<T> f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f.v[i] = down<T>(x[i]);
  *reinterpret_cast<Four<T> *>(p) = f;
}

// Where the new rows come from: the caller's tensors, or the partial sums of the Q/K/V multiply.
template <typename T> struct FromTensors {
  Kv4Tensor x[3];      // q, k, v
  __device__ __forceinline__ void load(int which, int r, int h, int c, float *a) const {
    load4(reinterpret_cast<const T *>(x[which].p) + (long long)r * x[which].row + (long long)h * x[which].head + c, a);
  }
  __device__ __forceinline__ float scale(int) const { return 1.f; }
};

// One vector of a row: DH / 8 lanes, lane l with dims 4l .. 4l+3 (a) and DH/2 + 4l .. (b).
// The products of the rotation are rounded one by one, so that codes do not depend on how a compiler contracts them.
__device__ __forceinline__ void rotate4(float *a, float *b, const float *cs) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = a[i], y = b[i], c = cs[2 * i], s = cs[2 * i + 1];
    a[i] = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
    b[i] = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
  }
}

// Codes of this lane's eight numbers as a word, and the vector's parameters (scale in the low half).
template <int DH> __device__ __forceinline__ uint32_t quantise(const float *a, const float *b, uint32_t &params) {
  constexpr int LPV = DH / 8;
  float lo = a[0], hi = a[0];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo = fminf(lo, fminf(a[i], b[i]));
    hi = fmaxf(hi, fmaxf(a[i], b[i]));
    bad = bad || !(fabsf(a[i]) < INFINITY) || !(fabsf(b[i]) < INFINITY);
  }
#pragma unroll
  for (int o = LPV / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const unsigned group = (LPV == 16 ? 0xffffu : 0xffu) << ((threadIdx.x & 31) / LPV * LPV);
  bad = (__ballot_sync(0xffffffffu, bad) & group) != 0u;
  const bf16 z = __float2bfloat16_rd(lo);
  const float zero = __bfloat162float(z);
  bf16 s = __float2bfloat16_ru(__fdiv_rn(__fsub_rn(hi, zero), 15.f));
  const float scale = __bfloat162float(s);
  bad = bad || !(scale < INFINITY);
  const bool flat = scale < 7.888609052210118e-31f;       // 2^-100
  if (flat) s = __float2bfloat16_rn(0.f);
  params = bad ? 0x7fff7fffu : (uint32_t)__bfloat16_as_ushort(s) | (uint32_t)__bfloat16_as_ushort(z) << 16;
  if (flat || bad) return 0u;
  uint32_t w = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float ca = fminf(fmaxf(__fdiv_rn(__fsub_rn(a[i], zero), scale), 0.f), 15.f);
    const float cb = fminf(fmaxf(__fdiv_rn(__fsub_rn(b[i], zero), scale), 0.f), 15.f);
    w |= (uint32_t)__float2int_rn(ca) << (4 * i) | (uint32_t)__float2int_rn(cb) << (16 + 4 * i);
  }
  return w;
}

// grid (rows, groups of vectors): a block takes 256 * 8 / DH of the row's n_q + 2 n_kv vectors.
template <int DH, typename Src, typename TQ>
__global__ void __launch_bounds__(256) kv4_append_kernel(Kv4Cache c, size_t layer_off, Kv4Rows rows, Src src, int n_q, Kv4Tensor q_out,
                                                         const float *rope, const int32_t *pos, int n_pos) {
  constexpr int LPV = DH / 8;
  pdl_launch_dependents();
  pdl_wait();
  const int r = blockIdx.x, lane = threadIdx.x & 31;
  const int vec = blockIdx.y * (256 / LPV) + threadIdx.x / LPV, l = threadIdx.x % LPV;
  const int n_vec = n_q + 2 * c.n_kv_heads;
  rows.check();
  const int b = rows.sequence_of(r, lane);
  if (b < 0) return;
  int first, count;
  rows.range(b, first, count);
  const int i = r - first;
  if (i >= count) return;
  const int slot = rows.slot != nullptr ? rows.slot[r] : rows.ctx_len[b] + i;
  if (slot < 0) {
    if (rows.slot == nullptr) rows.report();
    return;
  }
  const int p = pos != nullptr ? pos[r] : slot;
  if (rope != nullptr && (unsigned)p >= (unsigned)n_pos) { rows.report(); return; }
  const int page = c.page_of(rows.cache_of(b), slot >> 4);
  if ((unsigned)page >= (unsigned)c.n_pages) { rows.report(); return; }
  bool shadowed = false;        // a later row of the sequence has the same slot: that one is kept
  if (rows.slot != nullptr)
    for (int j = i + 1 + lane; j < count; j += 32) shadowed = shadowed || rows.slot[first + j] == slot;
  shadowed = __any_sync(0xffffffffu, shadowed);
  const int which = vec < n_q ? 0 : vec < n_q + c.n_kv_heads ? 1 : 2;
  const int h = which == 0 ? vec : which == 1 ? vec - n_q : vec - n_q - c.n_kv_heads;
  float a[4] = {0.f, 0.f, 0.f, 0.f}, e[4] = {0.f, 0.f, 0.f, 0.f};
  const bool live = vec < n_vec;
  if (live) {
    src.load(which, r, h, 4 * l, a);
    src.load(which, r, h, DH / 2 + 4 * l, e);
  }
  if (rope != nullptr && which < 2) {
    float cs[8];
    const float4 *t = reinterpret_cast<const float4 *>(rope + ((size_t)p * (DH / 2) + 4 * l) * 2);
    *reinterpret_cast<float4 *>(cs) = t[0];
    *reinterpret_cast<float4 *>(cs + 4) = t[1];
    rotate4(a, e, cs);
  }
  if (live && which == 0) {
    TQ *o = reinterpret_cast<TQ *>(q_out.p) + (long long)r * q_out.row + (long long)h * q_out.head + 4 * l;
    store4(o, a);
    store4(o + DH / 2, e);
  }
  uint32_t params;
  const uint32_t w = quantise<DH>(a, e, params);          // (whole warps: the vectors of a warp may be of both kinds)
  if (live && which != 0 && !shadowed) {
    unsigned char *g = c.pages + layer_off + c.granule<DH>(page, h, slot >> 4);
    const int s = slot & 15;
    *reinterpret_cast<uint32_t *>(g + (which == 1 ? kv4_k_at<DH>(s, l) : kv4_v_at<DH>(s, l))) = w;
    if (l == 0) *reinterpret_cast<uint32_t *>(g + kv4_p_at<DH>(s, which - 1)) = params;
  }
}

// grid (rows, groups of vectors, layers)
template <int DH, typename T>
__global__ void __launch_bounds__(256) kv4_read_kernel(Kv4Cache c, int layer0, Kv4Rows rows, Kv4Tensor k_out, Kv4Tensor v_out, long long k_layer,
                                                       long long v_layer) {
  constexpr int LPV = DH / 8;
  pdl_launch_dependents();
  pdl_wait();
  const int r = blockIdx.x, lane = threadIdx.x & 31;
  const int vec = blockIdx.y * (256 / LPV) + threadIdx.x / LPV, l = threadIdx.x % LPV;
  rows.check();
  const int b = rows.sequence_of(r, lane);
  if (b < 0) return;
  int first, count;
  rows.range(b, first, count);
  const int i = r - first;
  if (i >= count || vec >= 2 * c.n_kv_heads) return;
  const int slot = rows.slot != nullptr ? rows.slot[r] : rows.ctx_len[b] + i;
  const int page = slot < 0 ? -1 : c.page_of(rows.cache_of(b), slot >> 4);
  if ((unsigned)page >= (unsigned)c.n_pages) {
    if (slot >= 0 || rows.slot == nullptr) rows.report();
    return;
  }
  const int is_v = vec >= c.n_kv_heads, h = is_v ? vec - c.n_kv_heads : vec, s = slot & 15;
  const unsigned char *g = c.pages + (size_t)(layer0 + blockIdx.z) * c.layer_bytes + c.granule<DH>(page, h, slot >> 4);
  const uint32_t w = *reinterpret_cast<const uint32_t *>(g + (is_v ? kv4_v_at<DH>(s, l) : kv4_k_at<DH>(s, l)));
  const uint32_t params = *reinterpret_cast<const uint32_t *>(g + kv4_p_at<DH>(s, is_v));
  const float scale = __uint_as_float(params << 16), zero = __uint_as_float(params & 0xffff0000u);
  float a[4], e[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {          // scale * code is exact in fp32
    a[k] = zero + scale * (float)((w >> (4 * k)) & 15u);
    e[k] = zero + scale * (float)((w >> (16 + 4 * k)) & 15u);
  }
  const Kv4Tensor &t = is_v ? v_out : k_out;
  if (t.p == nullptr) return;
  T *o = reinterpret_cast<T *>(t.p) + (long long)blockIdx.z * (is_v ? v_layer : k_layer) + (long long)r * t.row + (long long)h * t.head + 4 * l;
  store4(o, a);
  store4(o + DH / 2, e);
}

// grid (kv heads, sequences, layers): slot dst[i] <- slot src[i], i < n, all reads before all writes.
template <int DH>
__global__ void __launch_bounds__(128) kv4_move_kernel(Kv4Cache c, Kv4Moves m) {
  constexpr int LPV = DH / 8, NW = 2 * LPV + 2;         // words of a slot: codes of K and of V, two words of parameters
  __shared__ long long from[KV4_MAX_MOVES], to[KV4_MAX_MOVES];
  __shared__ int in_granule[KV4_MAX_MOVES];             // slots inside their granules: source | destination << 8
  __shared__ int dst_slot[KV4_MAX_MOVES];
  extern __shared__ uint32_t words[];                   // [n][NW]
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.x, b = blockIdx.y;
  const int n = min(m.count != nullptr ? m.count[b] : m.n, m.n);
  unsigned char *base = c.pages + (size_t)blockIdx.z * c.layer_bytes;
  const int S = m.base != nullptr ? m.base[b] : 0;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    int src = m.src[(size_t)b * m.stride + i], dst = m.dst != nullptr ? m.dst[(size_t)b * m.stride + i] : i;
    const bool used = src >= 0 && dst >= 0;
    if (used) { src += S; dst += S; }
    long long f = -1, t = -1;
    if (used && src != dst) {
      f = c.granule<DH>(c.page_of(b, src >> 4), h, src >> 4);
      t = c.granule<DH>(c.page_of(b, dst >> 4), h, dst >> 4);
      if (f < 0 || t < 0) {
        if (m.status != nullptr) atomicMax(m.status, 1);
        f = t = -1;
      }
    }
    from[i] = f;
    to[i] = t;
    in_granule[i] = (src & 15) | (dst & 15) << 8;
    dst_slot[i] = used ? dst : -1;
  }
  __syncthreads();
  auto at = [&](int s, int w) { return w < LPV ? kv4_k_at<DH>(s, w) : w < 2 * LPV ? kv4_v_at<DH>(s, w - LPV) : kv4_p_at<DH>(s, w - 2 * LPV); };
  for (int e = threadIdx.x; e < n * NW; e += blockDim.x) {
    const int i = e / NW, w = e - i * NW;
    if (from[i] >= 0) words[e] = *reinterpret_cast<const uint32_t *>(base + from[i] + at(in_granule[i] & 15, w));
  }
  // of moves to the same slot the last one is kept
  for (int i = threadIdx.x; i < n; i += blockDim.x)
    for (int j = i + 1; j < n; ++j)
      if (dst_slot[i] >= 0 && dst_slot[j] == dst_slot[i]) to[i] = -1;
  __syncthreads();
  for (int e = threadIdx.x; e < n * NW; e += blockDim.x) {
    const int i = e / NW, w = e - i * NW;
    if (from[i] >= 0 && to[i] >= 0) *reinterpret_cast<uint32_t *>(base + to[i] + at(in_granule[i] >> 8, w)) = words[e];
  }
}

template <int DH, typename T>
cudaError_t append_t(Launch L, const Kv4Cache &c, size_t layer_off, const Kv4Rows &rows, const Kv4Tensor *x, int n_q, Kv4Tensor q_out, const float *rope,
                     const int32_t *pos, int n_pos) {
  const int per = 256 * 8 / DH, n_vec = n_q + 2 * c.n_kv_heads;
  const FromTensors<T> src{{x[0], x[1], x[2]}};
  return launch_k(kv4_append_kernel<DH, FromTensors<T>, T>, dim3(rows.total, (n_vec + per - 1) / per), dim3(256), 0, L.st, L.pdl, c, layer_off, rows,
                  src, n_q, q_out, rope, pos, n_pos);
}
template <int DH, typename T>
cudaError_t read_t(Launch L, const Kv4Cache &c, int layer0, int layers, const Kv4Rows &rows, Kv4Tensor k, Kv4Tensor v, long long k_layer, long long v_layer) {
  const int per = 256 * 8 / DH;
  return launch_k(kv4_read_kernel<DH, T>, dim3(rows.total, (2 * c.n_kv_heads + per - 1) / per, layers), dim3(256), 0, L.st, L.pdl, c, layer0, rows, k, v,
                  k_layer, v_layer);
}

}  // namespace

#define KV4_DISPATCH(dh, dtype, F, ...)                                                                                   \
  (dh == 128 ? (dtype == KV4_FP32 ? F<128, float>(__VA_ARGS__) : dtype == KV4_BF16 ? F<128, bf16>(__VA_ARGS__) : F<128, __half>(__VA_ARGS__)) \
             : (dtype == KV4_FP32 ? F<64, float>(__VA_ARGS__) : dtype == KV4_BF16 ? F<64, bf16>(__VA_ARGS__) : F<64, __half>(__VA_ARGS__)))

cudaError_t kv4_append(Launch L, int dh, int dtype, const Kv4Cache &c, size_t layer_off, const Kv4Rows &rows, const Kv4Tensor *qkv, int n_q, Kv4Tensor q_out,
                       const float *rope, const int32_t *pos, int n_pos) {
  return KV4_DISPATCH(dh, dtype, append_t, L, c, layer_off, rows, qkv, n_q, q_out, rope, pos, n_pos);
}
cudaError_t kv4_read(Launch L, int dh, int dtype, const Kv4Cache &c, int layer0, int layers, const Kv4Rows &rows, Kv4Tensor k, Kv4Tensor v, long long k_layer,
                     long long v_layer) {
  return KV4_DISPATCH(dh, dtype, read_t, L, c, layer0, layers, rows, k, v, k_layer, v_layer);
}
cudaError_t kv4_move(Launch L, int dh, const Kv4Cache &c, int B, const Kv4Moves &m) {
  const dim3 grid(c.n_kv_heads, B, c.n_layers);
  const size_t smem = (size_t)m.n * (2 * (dh / 8) + 2) * sizeof(uint32_t);
  return dh == 128 ? launch_k(kv4_move_kernel<128>, grid, dim3(128), smem, L.st, L.pdl, c, m) : launch_k(kv4_move_kernel<64>, grid, dim3(128), smem, L.st, L.pdl, c, m);
}

}  // namespace koala
