// Attention of a few query rows over the paged 4-bit cache (kv4.cuh has the format), on mma.sync.
//
// One CTA = (key chunk, tile of 8 NT query rows, kv head of a sequence); a query row is a (token, head) pair of the heads that
// share the kv head.  Its warps take the chunk's granules of 16 slots in turn.  With x = zero + scale * code
//   q . K_j        = scaleK_j (q . codeK_j) + zeroK_j sum(q)
//   sum_j p_j V_j  = sum_j (p_j scaleV_j) codeV_j + sum_j p_j zeroV_j
// so the multiplies take bare codes and nothing is expanded in memory: a warp loads a granule straight into the registers
// of operand A (16 bytes per lane and load, the cache's order), S^T = K Q^T with slots as rows, then O^T += V^T P^T with
// dims as rows; P^T changes from accumulator to operand layout by an 8x8 transposition of registers.
// A code 0..15 in the low bits of an fp16 IS that number times 2^-24 (subnormal), and in bits 4..7 16 times that: masking a
// word gives two operands without any conversion.  The factors 2^-24 and 16 are powers of two and go into q, the row's
// factor or the final scale, exactly.  For V the codes are centred first (one fp16 subtraction of 8 per two codes, exact): the
// tensor core adds by truncation, about 2e-8 of the sum per multiply, and without it the sum carries 7.5 times the sum of the
// weights, hundreds of times the result where many slots average out (131071 slots: 2e-3 off instead of 3e-4).  With fp32
// queries a granule's product starts from zero and is added to the sum in registers, rounded.
// Rounding: q enters as fp16, each row first scaled by a power of two to a maximum of 2^14 .. 2^15 (bf16 and fp16 queries
// lose nothing down to 2^-29 of the row's maximum); fp32 queries as two fp16 values (22 bits).  A weight p_j scaleV_j
// enters as one fp16 value scaled by a power of two (11 bits: relative error 2^-12, as much as the rounding of an fp16
// result, an eighth of a bf16 one); with fp32 queries as two.  Everything else is fp32.
// The softmax is online with a reference maximum that is raised only when a score exceeds it by more than 2^4: in the common
// case a granule needs no shuffles but one vote.
#include <cuda_fp16.h>

#include "kv4.h"

namespace koala {
namespace {

constexpr int WARPS = 4;
constexpr float RAISE = 4.f;            // log2: the reference maximum follows when a score exceeds it by more
constexpr float WEIGHT_TOP = 2048.f;    // scaleV * C stays at or below: times 2^RAISE well inside fp16

__device__ __forceinline__ void mma_f16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }

__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
  const __half2 h = __hadd2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&h);
}

// element c of a row of q
__device__ __forceinline__ float q_at(const void *p, int type, long long at) {
  if (type == KV4_FP32) return reinterpret_cast<const float *>(p)[at];
  if (type == KV4_BF16) return __bfloat162float(reinterpret_cast<const bf16 *>(p)[at]);
  return __half2float(reinterpret_cast<const __half *>(p)[at]);
}
__device__ __forceinline__ void out_at(void *p, void *lo, int type, long long at, float v) {
  if (type == KV4_FP32) reinterpret_cast<float *>(p)[at] = v;
  else if (type == KV4_FP16) reinterpret_cast<__half *>(p)[at] = __float2half_rn(v);
  else {
    const bf16 hi = __float2bfloat16_rn(v);
    reinterpret_cast<bf16 *>(p)[at] = hi;
    if (type == KV4_PAIR && lo != nullptr) reinterpret_cast<bf16 *>(lo)[at] = __float2bfloat16_rn(v - __bfloat162float(hi));
  }
}

// 2^k as a float, k within the range of normal numbers
__device__ __forceinline__ float pow2i(int k) { return __int_as_float((k + 127) << 23); }

__device__ __forceinline__ float ld_cluster(uint32_t local_addr, uint32_t rank) {
  uint32_t ra;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(local_addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(ra) : "memory");
  return v;
}

template <int DH> struct Granule { uint4 k[DH / 64], v[DH / 64], p; };

// grid (chunks, row tiles, sequences * kv heads), clusters of `chunks` CTAs
template <int DH, int NT, bool PAIR>
__global__ void __launch_bounds__(32 * WARPS) kv4_attn_kernel(const Kv4Attn A, int chunks) {
  constexpr int KS = DH / 16;              // depth steps of S
  constexpr int MT = DH / 16;              // tiles of 16 dims of O
  constexpr int ROWS = 8 * NT, OS = DH + 2;
  __shared__ float part[WARPS][ROWS][OS];
  __shared__ float mine[ROWS][OS];
  pdl_launch_dependents();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int chunk = blockIdx.x, hk = blockIdx.z % A.c.n_kv_heads, b = blockIdx.z / A.c.n_kv_heads;
  const int G = A.n_heads / A.c.n_kv_heads;
  int first, count;
  A.rows.range(b, first, count);
  const int row0 = blockIdx.y * ROWS;      // of the count * G rows of this kv head
  const int ctx = A.rows.ctx_len[b];
  int kv = A.rows.kv_len != nullptr ? A.rows.kv_len[b] : ctx + count;
  const bool bad = ctx < 0 || kv < 0;
  if (bad && threadIdx.x == 0) A.rows.report();
  kv = bad || row0 >= count * G ? 0 : min(kv, A.c.table_stride << (A.c.gpp_shift + 4));
  const int granules = (kv + KV4_G - 1) / KV4_G;
  const int lo = (int)((long long)granules * chunk / chunks), hi = (int)((long long)granules * (chunk + 1) / chunks);
  const int cache_row = A.rows.cache_of(b);

  // ---- this thread's two sets of rows: row g as a column of operand B (q), rows 2t and 2t + 1 as columns of the scores
  uint32_t qf[PAIR ? 2 : 1][NT][KS][2];
  float F[NT][2], Z[NT][2];
  uint64_t m0[NT][2], m1[NT][2];
  int last[NT][2];                         // slot up to which a row sees (no mask: its own); -2: not in use
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = row0 + 8 * n + g, i = r / G;
    const bool in = r < count * G;
    const long long at = in ? (long long)(first + i) * A.q.row + (long long)(hk * G + r % G) * A.q.head : 0;
    float x[KS][4];
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      // step s takes pairs 2 (s & 1) and 2 (s & 1) + 1 of the thread's word s / 2
      const int d = 4 * (t * (DH / 32) + (s >> 1)) + 2 * (s & 1);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        x[s][2 * e] = in ? q_at(A.q.p, A.q_type, at + d + e) : 0.f;
        x[s][2 * e + 1] = in ? q_at(A.q.p, A.q_type, at + DH / 2 + d + e) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) { top = fmaxf(top, fabsf(x[s][e])); sum += x[s][e]; }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    int ex = (int)(__float_as_uint(top) >> 23) - 127;       // 2^ex <= top < 2^(ex + 1)
    ex = max(-112, min(ex, 126));                            // (rows of zeros; infinities stay infinities)
    const float up = pow2i(14 - ex);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float f = e == 0 ? up : up * 0.0625f;          // the second pair's codes come 16 times as large
        const float y0 = x[s][2 * e] * f, y1 = x[s][2 * e + 1] * f;
        qf[0][n][s][e] = pack2(y0, y1);
        if constexpr (PAIR) {
          const float2 h = unpack2(qf[0][n][s][e]);
          qf[PAIR ? 1 : 0][n][s][e] = pack2(y0 - h.x, y1 - h.y);
        }
      }
    const float scale = A.scale * 1.4426950408889634f;
    const float f = fminf(scale * 16777216.f / up, 3e38f), z = sum * scale;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      F[n][j] = __shfl_sync(0xffffffffu, f, (2 * t + j) * 4);
      Z[n][j] = __shfl_sync(0xffffffffu, z, (2 * t + j) * 4);
      const int rr = row0 + 8 * n + 2 * t + j, ii = rr / G;
      const bool used = rr < count * G && !(A.rows.slot != nullptr && A.rows.slot[first + ii] < 0);
      m0[n][j] = used && A.rows.mask != nullptr ? A.rows.mask[(size_t)(first + ii) * 2] : 0ull;
      m1[n][j] = used && A.rows.mask != nullptr ? A.rows.mask[(size_t)(first + ii) * 2 + 1] : 0ull;
      last[n][j] = !used ? -2 : A.rows.mask != nullptr ? ctx - 1 : ctx + ii;
    }
  }
  const bool tree = A.rows.mask != nullptr;

  float o[NT][MT][4], mref[NT][2], mu[NT][2], l[NT][2], zs[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < MT; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
#pragma unroll
    for (int j = 0; j < 2; ++j) { mref[n][j] = -INFINITY; mu[n][j] = 0.f; l[n][j] = 0.f; zs[n][j] = 0.f; }
  }
  float C = pow2i(100);                    // power of two on the V scales, lowered as larger ones come

  const unsigned char *base = A.c.pages + A.layer_off;
  auto fetch = [&](int gi, Granule<DH> &f) -> bool {
    const long long off = gi < hi ? A.c.granule<DH>(A.c.page_of(cache_row, gi), hk, gi) : -1;
    if (off < 0) {
      if (gi < hi && lane == 0) A.rows.report();
      return false;
    }
    const unsigned char *p = base + off;
#pragma unroll
    for (int i = 0; i < DH / 64; ++i) {
      f.k[i] = *reinterpret_cast<const uint4 *>(p + i * 512 + lane * 16);
      f.v[i] = *reinterpret_cast<const uint4 *>(p + KV4_G * DH / 2 + i * 512 + lane * 16);
    }
    f.p = *reinterpret_cast<const uint4 *>(p + KV4_G * DH + g * 16);
    return true;
  };

  Granule<DH> cur, nxt;
  bool have = fetch(lo + warp, cur);
#pragma unroll 1
  for (int gi = lo + warp; gi < hi; gi += WARPS) {
    const bool have_n = fetch(gi + WARPS, nxt);
    if (have) {
      const int key0 = gi * KV4_G;
      // ---- S^T, two chains of accumulation
      float acc[NT][2][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) acc[n][e][0] = acc[n][e][1] = acc[n][e][2] = acc[n][e][3] = 0.f;
#pragma unroll
      for (int w = 0; w < KS / 2; ++w) {
        uint32_t x, y;                     // word w of slots g and g + 8
        if constexpr (DH == 128) {
          x = (&cur.k[0].x)[w];
          y = (&cur.k[DH / 64 - 1].x)[w];
        } else {
          x = (&cur.k[0].x)[w];
          y = (&cur.k[0].x)[2 + w];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t a[4] = {x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(acc[n][e], a, qf[0][n][2 * w + e][0], qf[0][n][2 * w + e][1]);
            if constexpr (PAIR) mma_f16(acc[n][e], a, qf[PAIR ? 1 : 0][n][2 * w + e][0], qf[PAIR ? 1 : 0][n][2 * w + e][1]);
          }
          x >>= 8;
          y >>= 8;
        }
      }
      // ---- scores: accumulator e is slot g + 8 (e >> 1), row 2t + (e & 1)
      const uint32_t pk[2] = {cur.p.x, cur.p.y}, pv[2] = {cur.p.z, cur.p.w};
      float ks[2], kz[2], sv[2], zv[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ks[e] = __uint_as_float(pk[e] << 16); kz[e] = __uint_as_float(pk[e] & 0xffff0000u);
        sv[e] = __uint_as_float(pv[e] << 16); zv[e] = fmaf(8.f, sv[e], __uint_as_float(pv[e] & 0xffff0000u));
      }
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s[n][e] = fmaf(ks[e >> 1], (acc[n][0][e] + acc[n][1][e]) * F[n][e & 1], kz[e >> 1] * Z[n][e & 1]);
      const bool open = key0 + KV4_G <= min(ctx, kv);
      unsigned seen = 0xffffffffu;         // bit 4 n + e
      if (!open) {
        seen = 0u;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = key0 + g + 8 * (e >> 1), rel = key - ctx, j = e & 1;
            bool v = last[n][j] != -2;
            if (rel >= 0) v = tree ? (rel < 64 ? (m0[n][j] >> rel) & 1ull : rel < 128 ? (m1[n][j] >> (rel - 64)) & 1ull : 0ull) != 0ull : key <= last[n][j];
            if (key >= kv) v = false;
            s[n][e] = v ? s[n][e] : -INFINITY;
            seen |= v ? 1u << (4 * n + e) : 0u;
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {      // what no row sees may hold anything, NaN included
          bool any = false;
#pragma unroll
          for (int n = 0; n < NT; ++n) any = any || (seen >> (4 * n + 2 * e) & 3u) != 0u;
          if (!any) { sv[e] = 0.f; zv[e] = 0.f; }
        }
      }
      float svc[2] = {sv[0] * C, sv[1] * C};
      bool raise = svc[0] > WEIGHT_TOP || svc[1] > WEIGHT_TOP;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) raise = raise || s[n][e] > mref[n][e & 1] + RAISE;
      if (__any_sync(0xffffffffu, raise)) {
        float most = fmaxf(sv[0], sv[1]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        float less = 1.f;                  // uniform over the warp
        if (most * C > WEIGHT_TOP) {
          const float to = pow2i(136 - (int)(__float_as_uint(most) >> 23));          // most * to in [2^9, 2^10)
          less = to / C;
          C = to;
          svc[0] = sv[0] * C;
          svc[1] = sv[1] * C;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float f[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float mx = fmaxf(s[n][j], s[n][2 + j]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            f[j] = 1.f;
            if (mx > mref[n][j]) {
              f[j] = mref[n][j] == -INFINITY ? 0.f : ex2(mref[n][j] - mx);
              mref[n][j] = mu[n][j] = mx;
            }
            l[n][j] *= f[j];
            zs[n][j] *= f[j];
            f[j] *= less;
          }
#pragma unroll
          for (int i = 0; i < MT; ++i) { o[n][i][0] *= f[0]; o[n][i][1] *= f[1]; o[n][i][2] *= f[0]; o[n][i][3] *= f[1]; }
        }
      }
      // ---- weights
      uint32_t pb[PAIR ? 2 : 1][NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = ex2(s[n][e] - mu[n][e & 1]);
          const bool v = open || (seen >> (4 * n + e) & 1u) != 0u;
          l[n][e & 1] += p;
          zs[n][e & 1] += v ? p * zv[e >> 1] : 0.f;
          w[e] = v ? p * svc[e >> 1] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t h = pack2(w[2 * e], w[2 * e + 1]);
          pb[0][n][e] = transpose8x8(h);
          if constexpr (PAIR) {
            const float2 back = unpack2(h);
            pb[PAIR ? 1 : 0][n][e] = transpose8x8(pack2(w[2 * e] - back.x, w[2 * e + 1] - back.y));
          }
        }
      }
      // ---- O^T: lane (g, t) has words g * DH/64 .. of slots 2t, 2t + 1 (first plane or half) and 2t + 8, 2t + 9
#pragma unroll
      for (int w = 0; w < DH / 64; ++w) {
        uint32_t a0, a1, b0, b1;           // slots 2t, 2t + 1, 2t + 8, 2t + 9
        if constexpr (DH == 128) {
          a0 = (&cur.v[0].x)[w]; a1 = (&cur.v[0].x)[2 + w];
          b0 = (&cur.v[DH / 64 - 1].x)[w]; b1 = (&cur.v[DH / 64 - 1].x)[2 + w];
        } else {
          a0 = cur.v[0].x; a1 = cur.v[0].y; b0 = cur.v[0].z; b1 = cur.v[0].w;
        }
        uint32_t x = __byte_perm(a0, a1, 0x5410), xh = __byte_perm(a0, a1, 0x7632);      // two slots side by side: dims 4l .., DH/2 + 4l ..
        uint32_t y = __byte_perm(b0, b1, 0x5410), yh = __byte_perm(b0, b1, 0x7632);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t mask = (i & 1) ? 0x00f000f0u : 0x000f000fu, eight = (i & 1) ? 0x80808080u : 0x80088008u;      // -8 * 16, -8
          const uint32_t a[4] = {add2(x & mask, eight), add2(xh & mask, eight), add2(y & mask, eight), add2(yh & mask, eight)};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (PAIR) {
              float d[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16(d, a, pb[0][n][0], pb[0][n][1]);
              mma_f16(d, a, pb[PAIR ? 1 : 0][n][0], pb[PAIR ? 1 : 0][n][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[n][4 * w + i][e] += d[e];
            } else {
              mma_f16(o[n][4 * w + i], a, pb[0][n][0], pb[0][n][1]);
            }
          }
          if (i == 1) { x >>= 8; xh >>= 8; y >>= 8; yh >>= 8; }
        }
      }
    }
    cur = nxt;
    have = have_n;
  }

  // ---- this warp's sums, in true units
  const float back = 1.f / C;              // a power of two
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], d);
        zs[n][j] += __shfl_xor_sync(0xffffffffu, zs[n][j], d);
      }
      float *to = part[warp][8 * n + 2 * t + j];
#pragma unroll
      for (int w = 0; w < DH / 64; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = 4 * (g * (DH / 64) + w) + i;
          const float f = (i & 1) ? 1048576.f : 16777216.f;          // 2^24, less the 16 of the upper nibbles
          to[d] = fmaf(o[n][4 * w + i][j] * f, back, zs[n][j]);
          to[DH / 2 + d] = fmaf(o[n][4 * w + i][2 + j] * f, back, zs[n][j]);
        }
      if (g == 0) { to[DH] = mref[n][j]; to[DH + 1] = l[n][j]; }
    }
  }
  __syncthreads();
  // ---- the warps together, then the chunks of the cluster
  auto weight = [](float m, float top) { return m == -INFINITY ? 0.f : exp2f(m - top); };
  auto finish = [&](int r, int d, float v, float sum) {
    const int rr = row0 + r;
    if (rr >= count * G) return;
    const long long at = (long long)(first + rr / G) * A.out.row + (long long)(hk * G + rr % G) * A.out.head + d;
    // a row that sees nothing or is not in use is 0; one whose sum is NaN stays NaN
    const bool none = sum == 0.f || (A.rows.slot != nullptr && A.rows.slot[first + rr / G] < 0);
    out_at(A.out.p, A.out_lo, A.out_type, at, none ? 0.f : v / sum);
  };
  for (int e = threadIdx.x; e < ROWS * DH; e += 32 * WARPS) {
    const int r = e / DH, d = e - r * DH;
    float top = -INFINITY, sum = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, part[w][r][DH]);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = weight(part[w][r][DH], top);
      if (f == 0.f && part[w][r][DH + 1] == 0.f) continue;
      sum += f * part[w][r][DH + 1];
      v += f * part[w][r][d];
    }
    if (chunks == 1) {
      finish(r, d, v, sum);
    } else {
      mine[r][d] = v;
      if (d == 0) { mine[r][DH] = top; mine[r][DH + 1] = sum; }
    }
  }
  if (chunks == 1) return;
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  const int share = DH / chunks;
  const uint32_t addr = (uint32_t)__cvta_generic_to_shared(&mine[0][0]);
  for (int e = threadIdx.x; e < ROWS * share; e += 32 * WARPS) {
    const int r = e / share, d = chunk * share + e % share;
    float m[8], sm[8], v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = -INFINITY; sm[k] = 0.f; v[k] = 0.f;
      if (k < chunks) {
        m[k] = ld_cluster(addr + (uint32_t)(r * OS + DH) * 4u, (uint32_t)k);
        sm[k] = ld_cluster(addr + (uint32_t)(r * OS + DH + 1) * 4u, (uint32_t)k);
        v[k] = ld_cluster(addr + (uint32_t)(r * OS + d) * 4u, (uint32_t)k);
      }
    }
    float top = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = fmaxf(top, m[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {          // in chunk order
      const float f = weight(m[k], top);
      if (f == 0.f && sm[k] == 0.f) continue;
      sum += f * sm[k];
      x += f * v[k];
    }
    finish(r, d, x, sum);
  }
  // no CTA leaves while another may still read its sums
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

template <int DH, int NT, bool PAIR> cudaError_t go(Launch L, const Kv4Attn &a, int chunks) {
  const int G = a.n_heads / a.c.n_kv_heads, tiles = (a.rows.max_rows * G + 8 * NT - 1) / (8 * NT);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(chunks, tiles, a.rows.B * a.c.n_kv_heads);
  cfg.blockDim = dim3(32 * WARPS);
  cfg.stream = L.st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = L.pdl ? 1 : 0;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = chunks;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = chunks > 1 ? 2 : 1;
  ++g_launches;
  return cudaLaunchKernelEx(&cfg, kv4_attn_kernel<DH, NT, PAIR>, a, chunks);
}

}  // namespace

cudaError_t kv4_attention(Launch L, int dh, const Kv4Attn &a, int num_sms) {
  const int G = a.n_heads / a.c.n_kv_heads, rows = a.rows.max_rows * G;
  const bool pair = a.q_type == KV4_FP32, wide = rows > 8;
  const int tiles = (rows + (wide ? 15 : 7)) / (wide ? 16 : 8);
  int chunks = 1;
  while (chunks < 8 && (long long)2 * chunks * tiles * a.rows.B * a.c.n_kv_heads <= 3 * num_sms) chunks *= 2;
#define KV4_GO(D, N) (pair ? go<D, N, true>(L, a, chunks) : go<D, N, false>(L, a, chunks))
  if (dh == 128) return wide ? KV4_GO(128, 2) : KV4_GO(128, 1);
  return wide ? KV4_GO(64, 2) : KV4_GO(64, 1);
#undef KV4_GO
}

}  // namespace koala
