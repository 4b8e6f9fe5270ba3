// Attention of many query rows over the paged 4-bit cache (kv4.cuh has the format), on tcgen05.
//
// One CTA per SM walks through its share of the work (kv4_work.cuh): tiles of 128 (token, head) rows of one kv head, keys in tiles
// of 64.  Per key tile
//   eight warps expand the codes of K (four) and V (four): shared memory, fp16, in the layouts that the MMAs read
//   S[128 x 64]   = Q K^T    tcgen05.mma, A = Q and B = K from tensor and shared memory
//   P             = 2^(...)  four warps, a thread per row; P goes where S was, in tensor memory
//   O[128 x DH]  += P V      tcgen05.mma, A = P from tensor memory, B = V as [key][dim] (MN-major)
// With x = zero + scale code = (zero + 8 scale) + scale (code - 8): scale (code - 8) times a power of two is EXACT in fp16 (8 bits by 3),
// so K and V are expanded without rounding, and the constants of the vectors come in as more columns of the products: four
// columns of depth for S (Z_r kz_j, both as two fp16 values), two columns of O (sum of p_j zv_j, likewise).  The power of two is
// chosen for each granule of 16 keys, so that neither large nor small vectors leave fp16's range; for K it is taken off with the
// scores (a factor per 16 columns), for V it goes into P, relative to the largest power so far.
// Dims are in the order in which words unpack: position 2 d of a row is dim d, position 2 d + 1 dim d + DH/2.
// Rounding: Q one fp16 value with the row's maximum at 2^7 .. 2^8 (exact for bf16 and fp16 queries down to 2^-22 of the row's maximum), P one
// fp16 value (2^-12); with fp32 queries two of each.  Products and sums are fp32.
// The form with 64 rows has every row twice, in lanes l and l + 16 of a warp, each with half of the keys to take 2^x of (half the work of the
// rows); with fp32 queries the two lanes hold the two parts of Q and P.
// O stays in tensor memory; a row's reference maximum is raised only when a score exceeds it by more than 2^4, then its O is rescaled in place.
// Every wait is bounded: on expiry the kernel records a timeout in *status and leaves.
#include "kv4_work.cuh"
#include "tc_ptx.cuh"

namespace koala {
namespace {

constexpr int TK = 64;                     // keys of a tile
constexpr int UG = TK / KV4_G;             // granules of a tile
constexpr int NB = 3;                      // buffers of K and of V
constexpr int RING = 4;                    // tiles of codes on their way per expanding warp
constexpr int INFO = 8;                    // tiles whose powers of two are kept (expanding runs at most NB + 2 tiles ahead of the rows)
constexpr int BLK = TK * 128;              // [64 keys][64 dims]
constexpr int ROW_WARPS = 4, EXPANDERS = 8, MMA_WARP = ROW_WARPS + EXPANDERS;
constexpr int THREADS = 32 * (MMA_WARP + 1);
constexpr int E_TIMEOUT = 6;
constexpr float RAISE = 4.f;
constexpr int P_TOP = 10;                  // P = 2^P_TOP at the reference maximum
constexpr int COL_S = 0, COL_O = 2 * TK, COL_Q = COL_O + 144;
constexpr int TMEM_COLS = 512;

enum { FULL = 0, HALF = 1, PAIR = 2 };     // 128 rows; 64 rows twice; 64 rows as two values
template <int MODE> constexpr int TILE_ROWS = MODE == FULL ? 128 : 64;
template <int DH> struct Lay {
  static constexpr int NBLK = DH / 64 + 1;                   // blocks of 64 dims, and the constants
  static constexpr int ONE = NBLK * BLK;
  static constexpr int K = 0, V = NB * ONE, CODES = 2 * NB * ONE;
  static constexpr int PART = KV4_G * DH / 2 + KV4_PARAMS;   // what an expanding warp fetches per tile: a granule's K or V and its parameters
  static constexpr int BYTES = CODES + EXPANDERS * RING * PART;
};
template <int DH> constexpr unsigned SMEM = Lay<DH>::BYTES + 1024;

struct TileInfo {
  float k_back[UG];                        // what a score of the granule is multiplied with
  int v_exp[UG];                           // V of the granule was divided by 2^v_exp
  unsigned poison[UG], poison_v[UG];       // slots whose K / V is NaN
};
struct alignas(16) Sync {
  uint64_t q_full, k_full[NB], k_empty[NB], v_full[NB], v_empty[NB], s_full[2], p_full[2], pv_done[2], info_full[INFO], drain;
  uint32_t tmem;
  int error;
  TileInfo info[INFO];
};

__device__ __forceinline__ void arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A from tensor memory
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<const __half2 *>(&v); }
__device__ __forceinline__ uint32_t as_u32(__half2 v) { return *reinterpret_cast<const uint32_t *>(&v); }

// Eight codes as (code - 8) * scale: pairs (nibble i, nibble i + 4).  1024 + code and 1024 + 16 code are fp16 numbers with the code in their bits.
__device__ __forceinline__ void expand(uint32_t w, __half2 scale, uint32_t *x) {
  const __half2 back = as_half2(0xe408e408u), sixteenth = as_half2(0x2c002c00u), back16 = as_half2(0xd480d480u);      // -1032, 1/16, -72
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t lo = (w & 0x000f000fu) | 0x64006400u, hi = (w & 0x00f000f0u) | 0x64006400u;
    x[2 * e] = as_u32(__hmul2(__hadd2(as_half2(lo), back), scale));
    x[2 * e + 1] = as_u32(__hmul2(__hfma2(as_half2(hi), sixteenth, back16), scale));
    w >>= 8;
  }
}

// rows of a tile of 64 keys that a row sees: bit j is key0 + j
__device__ __forceinline__ uint64_t ones_below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }
__device__ __forceinline__ uint64_t tree_bits(uint64_t m0, uint64_t m1, int shift) {      // shift = key0 - ctx
  if (shift <= -64) return ~0ull;
  if (shift < 0) return (m0 << -shift) | ((1ull << -shift) - 1ull);
  if (shift == 0) return m0;
  if (shift < 64) return (m0 >> shift) | (m1 << (64 - shift));
  return shift < 128 ? m1 >> (shift - 64) : 0ull;
}

template <int DH, int MODE>
__global__ void __launch_bounds__(THREADS, 1) kv4_attn_tc_kernel(const Kv4Attn A, float *__restrict__ scratch, int tiles) {
  constexpr int ROWS = TILE_ROWS<MODE>;
  constexpr int NC = MODE == FULL ? 64 : 32;          // keys of a tile per row thread
  constexpr int NG = NC / KV4_G;
  typedef Lay<DH> LY;
  extern __shared__ unsigned char smem_raw[];
  __shared__ Sync sync;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_raw), sb = raw + ((1024u - (raw & 1023u)) & 1023u);
  const int G = A.n_heads / A.c.n_kv_heads;
  const bool tree = A.rows.mask != nullptr;

  if (threadIdx.x == 0) {
    mbar_init(&sync.q_full, ROW_WARPS);
    for (int i = 0; i < NB; ++i) {
      mbar_init(&sync.k_full[i], EXPANDERS / 2); mbar_init(&sync.k_empty[i], 1);
      mbar_init(&sync.v_full[i], EXPANDERS / 2); mbar_init(&sync.v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) { mbar_init(&sync.s_full[i], 1); mbar_init(&sync.p_full[i], ROW_WARPS); mbar_init(&sync.pv_done[i], 1); }
    for (int i = 0; i < INFO; ++i) mbar_init(&sync.info_full[i], EXPANDERS);
    mbar_init(&sync.drain, 1);
    sync.error = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();                              // before the allocation: the launch before may not have made its own yet
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sync.tmem)), "r"((uint32_t)TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // the second 16 bytes of the constants' rows stay zero
  for (int e = threadIdx.x; e < 2 * NB * TK; e += THREADS) {
    const int key = e % TK;
    sts128(sb + (uint32_t)(e / TK * LY::ONE + (LY::NBLK - 1) * BLK + key * 128 + ((1 ^ (key & 7)) << 4)), 0u, 0u, 0u, 0u);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sync.tmem;
  pdl_launch_dependents();                 // after the allocation: what follows may want tensor memory too; and after the wait: the joining kernel reads the plan early

  Walk<ROWS, UG> walk;
  bool more = walk.begin(A, tiles, G, lane, blockIdx.x == 0 && warp == 0);
  Piece pc;
  int tt = 0;                              // tiles before this piece (of this CTA)
  bool ok = true;

  if (warp >= ROW_WARPS && warp < MMA_WARP) {
    // ------------------------------------------------------------------ expanding warps: granule gq of every tile, K or V
    const int w = warp - ROW_WARPS, gq = w & 3, g = lane >> 2, t = lane & 3;
    const bool is_v = w >= 4;
    const uint32_t codes = sb + LY::CODES + (uint32_t)(w * RING * LY::PART);
    uint64_t *full = is_v ? sync.v_full : sync.k_full, *empty = is_v ? sync.v_empty : sync.k_empty;
    const uint32_t out0 = sb + (is_v ? LY::V : LY::K);
    while (more && ok && walk.next(A, G, lane, pc)) {
      const int n = pc.hi - pc.lo, kv = min(pc.kv, pc.hi * TK), cache_row = A.rows.cache_of(pc.b);
      uint64_t or0 = ~0ull, or1 = ~0ull;   // slots behind ctx that some row sees
      if (tree && pc.hi * TK > pc.ctx) {
        or0 = or1 = 0ull;
        for (int i = lane; i < pc.count; i += 32) {
          if (A.rows.slot != nullptr && A.rows.slot[pc.first + i] < 0) continue;
          or0 |= A.rows.mask[(size_t)(pc.first + i) * 2];
          or1 |= A.rows.mask[(size_t)(pc.first + i) * 2 + 1];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          or0 |= __shfl_xor_sync(0xffffffffu, or0, o);
          or1 |= __shfl_xor_sync(0xffffffffu, or1, o);
        }
      }
      auto pages_from = [&](int i) {       // of tiles i .. i + 31 of the piece
        const int gi = (pc.lo + i + lane) * UG + gq;
        if (i + lane >= n || gi * KV4_G >= kv) return -1;
        const int page = A.c.page_of(cache_row, gi);
        if ((unsigned)page >= (unsigned)A.c.n_pages) A.rows.report();
        return page;
      };
      int page_now = pages_from(0), page_next = pages_from(32);
      unsigned have = 0u;
      auto request = [&](int i) {
        bool there = false;
        if (i < n) {
          const int page = __shfl_sync(0xffffffffu, page_now, i & 31);
          there = (unsigned)page < (unsigned)A.c.n_pages;
          if (there) {
            const unsigned char *src = A.c.pages + A.layer_off + A.c.granule<DH>(page, pc.hk, (pc.lo + i) * UG + gq);
            const uint32_t dst = codes + (uint32_t)(i % RING * LY::PART);
#pragma unroll
            for (int k = 0; k < DH / 64; ++k) copy16(dst + k * 512 + lane * 16, src + (is_v ? KV4_G * DH / 2 : 0) + k * 512 + lane * 16);
            if (lane < KV4_PARAMS / 16) copy16(dst + KV4_G * DH / 2 + lane * 16, src + KV4_G * DH + lane * 16);
          }
          if ((i & 31) == 31) {
            page_now = page_next;
            page_next = pages_from(i + 33);
          }
        }
        have = have << 1 | (there ? 1u : 0u);
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
#pragma unroll
      for (int i = 0; i < RING - 1; ++i) request(i);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        __syncwarp();
        request(i + RING - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
        __syncwarp();
        const bool there = (have >> (RING - 1) & 1u) != 0u;
        const uint32_t at = codes + (uint32_t)(i % RING * LY::PART);
        // ---- parameters of this lane's vectors: K of slots g, g + 8; V of slots 2t, 2t + 1, 2t + 8, 2t + 9
        constexpr int NV = 4;
        float sc[NV], zc[NV];
        int slot[NV];
        {
          const uint4 e0 = lds128(at + KV4_G * DH / 2 + (is_v ? 2 * t : g) * 16), e1 = lds128(at + KV4_G * DH / 2 + (is_v ? 2 * t + 1 : g) * 16);
          const uint32_t p[NV] = {is_v ? e0.z : e0.x, is_v ? e1.z : e0.y, is_v ? e0.w : e0.x, is_v ? e1.w : e0.y};
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            slot[k] = is_v ? 2 * t + (k & 1) + 8 * (k >> 1) : g + 8 * (k & 1);
            sc[k] = __uint_as_float(p[k] << 16);
            zc[k] = fmaf(8.f, sc[k], __uint_as_float(p[k] & 0xffff0000u));
          }
        }
        const int key0 = (pc.lo + i) * TK + gq * KV4_G;
        float most = 0.f;
        unsigned poison = 0u;              // this lane's slots
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int key = key0 + slot[k], rel = key - pc.ctx;
          bool v = there && key < kv;
          if (tree && rel >= 0) v = v && (rel < 64 ? (or0 >> rel) & 1ull : rel < 128 ? (or1 >> (rel - 64)) & 1ull : 0ull) != 0ull;
          const bool finite = fabsf(zc[k]) < INFINITY && sc[k] < INFINITY;
          if (v && !finite) poison |= 1u << slot[k];
          if (!v || !finite) { sc[k] = 0.f; zc[k] = 0.f; }
          most = fmaxf(most, fmaxf(8.f * sc[k], fabsf(zc[k])));
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (__any_sync(0xffffffffu, poison != 0u)) {
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) poison |= __shfl_xor_sync(0xffffffffu, poison, o);
        }
        const int ex = most > 0.f ? max(-112, (int)(__float_as_uint(most) >> 23) - 127) : 13;      // most in [2^ex, 2^(ex + 1))
        const float norm = pow2i(13 - ex);
        const int now = tt + i;
        if (lane == 0) {
          TileInfo &f = sync.info[now & (INFO - 1)];
          if (is_v) {
            f.v_exp[gq] = most > 0.f ? ex - 13 : -200;
            f.poison_v[gq] = poison;
          } else {
            f.k_back[gq] = 1.f / norm;
            f.poison[gq] = poison;
          }
          arrive(&sync.info_full[now & (INFO - 1)]);
        }
        if (now >= NB) ok = __all_sync(0xffffffffu, mbar_wait(&empty[now % NB], (uint32_t)(now / NB - 1) & 1u));
        if (!ok) break;
        const uint32_t out = out0 + (uint32_t)(now % NB * LY::ONE);
        auto put = [&](uint32_t word, int s, int l, float scale) {
          const int key = gq * KV4_G + s;
          const __half2 sc2 = __float2half2_rn(scale * norm);
          uint32_t x[4];
          expand(word, sc2, x);
          sts128(out + (uint32_t)((l >> 3) * BLK + key * 128 + (((l & 7) ^ (key & 7)) << 4)), x[0], x[1], x[2], x[3]);
        };
        const uint4 c0 = lds128(at + lane * 16), c1 = DH == 128 ? lds128(at + 512 + lane * 16) : c0;
        if constexpr (DH == 128) {
          // words in an order in which a quarter of the warp writes to eight places of 16 bytes that lie in different banks
          if (is_v) {
            const bool odd = (g & 1) != 0;
            const int l0 = 2 * g + (odd ? 1 : 0), l1 = 2 * g + (odd ? 0 : 1);
            put(odd ? c0.y : c0.x, slot[0], l0, sc[0]); put(odd ? c0.x : c0.y, slot[0], l1, sc[0]);
            put(odd ? c0.w : c0.z, slot[1], l0, sc[1]); put(odd ? c0.z : c0.w, slot[1], l1, sc[1]);
            put(odd ? c1.y : c1.x, slot[2], l0, sc[2]); put(odd ? c1.x : c1.y, slot[2], l1, sc[2]);
            put(odd ? c1.w : c1.z, slot[3], l0, sc[3]); put(odd ? c1.z : c1.w, slot[3], l1, sc[3]);
          } else {
            const bool far = t >= 2;
            const int f2 = far ? 2 : 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint4 c = k == 0 ? c0 : c1;
              put(far ? c.z : c.x, slot[k], 4 * t + (0 ^ f2), sc[k]);
              put(far ? c.w : c.y, slot[k], 4 * t + (1 ^ f2), sc[k]);
              put(far ? c.x : c.z, slot[k], 4 * t + (2 ^ f2), sc[k]);
              put(far ? c.y : c.w, slot[k], 4 * t + (3 ^ f2), sc[k]);
            }
          }
        } else if (is_v) {
          put(c0.x, slot[0], g, sc[0]); put(c0.y, slot[1], g, sc[1]); put(c0.z, slot[2], g, sc[2]); put(c0.w, slot[3], g, sc[3]);
        } else {
          put(c0.x, slot[0], 2 * t, sc[0]); put(c0.y, slot[0], 2 * t + 1, sc[0]);
          put(c0.z, slot[1], 2 * t, sc[1]); put(c0.w, slot[1], 2 * t + 1, sc[1]);
        }
        // ---- the constants: K has them twice side by side (for the two values of Z), V once
        if (is_v ? g == 0 : t == 0) {
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            if (!is_v && k >= 2) break;
            const int key = gq * KV4_G + slot[k];
            const float z = zc[k] * norm, zh = __half2float(__float2half_rn(z));
            const uint32_t both = pack2(zh, z - zh);
            sts128(out + (uint32_t)((LY::NBLK - 1) * BLK + key * 128 + ((key & 7) << 4)), both, is_v ? 0u : both, 0u, 0u);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) arrive(&full[now % NB]);
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      tt += n;
    }
    if (!ok) atomicExch(&sync.error, 1);
  } else if (warp == MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuer
    const uint32_t idesc_s = (1u << 4) | ((uint32_t)(TK >> 3) << 17) | ((128u >> 4) << 24);                                  // fp32, fp16 x fp16, N = 64
    const uint32_t idesc_o = (1u << 4) | (1u << 16) | ((uint32_t)((DH + 16) >> 3) << 17) | ((128u >> 4) << 24);               // N = DH + 16, B MN-major
    int pieces = 0;
    while (more && ok && walk.next(A, G, lane, pc)) {
      const int n = pc.hi - pc.lo;
      if (n > 0 && lane == 0) {
        auto issue_s = [&](int now) -> bool {
          if (!mbar_wait(&sync.k_full[now % NB], (uint32_t)(now / NB) & 1u)) return false;
          fence_after();
          const uint32_t kb = sb + LY::K + (uint32_t)(now % NB * LY::ONE), d = tmem + (uint32_t)(COL_S + (now & 1) * TK);
#pragma unroll
          for (int k = 0; k < DH / 16 + 1; ++k)             // the last step: the constants
            umma_ts(d, tmem + (uint32_t)(COL_Q + 8 * k), smem_desc_sw128(kb + (uint32_t)((k >> 2) * BLK)) + (uint64_t)(2 * (k & 3)), idesc_s, k ? 1u : 0u);
          umma_commit(&sync.s_full[now & 1]);
          umma_commit(&sync.k_empty[now % NB]);
          return true;
        };
        auto issue_pv = [&](int now, bool first) -> bool {
          if (!mbar_wait(&sync.p_full[now & 1], (uint32_t)(now >> 1) & 1u)) return false;
          if (!mbar_wait(&sync.v_full[now % NB], (uint32_t)(now / NB) & 1u)) return false;
          fence_after();
          const uint32_t vb = sb + LY::V + (uint32_t)(now % NB * LY::ONE), p = tmem + (uint32_t)(COL_S + (now & 1) * TK);
#pragma unroll
          for (int k = 0; k < TK / 16; ++k)
            umma_ts(tmem + (uint32_t)COL_O, p + (uint32_t)(8 * k), smem_desc_mn_sw128(vb + (uint32_t)(k * 2048), BLK, 1024), idesc_o, (first && k == 0) ? 0u : 1u);
          umma_commit(&sync.v_empty[now % NB]);
          umma_commit(&sync.pv_done[now & 1]);
          return true;
        };
        ok = mbar_wait(&sync.q_full, (uint32_t)pieces & 1u);
        for (int i = -1; i < n && ok; ++i) {
          if (i + 1 < n) ok = issue_s(tt + i + 1);
          if (i >= 0 && ok) ok = issue_pv(tt + i, i == 0);
        }
      }
      ok = __all_sync(0xffffffffu, ok);
      if (n > 0) ++pieces;
      tt += n;
    }
    if (!ok) atomicExch(&sync.error, 1);
  } else if (warp < ROW_WARPS) {
    // ------------------------------------------------------------------ rows
    const int half = MODE == FULL ? 0 : lane >> 4;
    const int row = MODE == FULL ? warp * 32 + lane : warp * 16 + (lane & 15);
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const float log2_scale = A.scale * 1.4426950408889634f;
    while (more && ok && walk.next(A, G, lane, pc)) {
      const int n = pc.hi - pc.lo, kv = min(pc.kv, pc.hi * TK);
      const int rr = pc.row0 + row, n_rows = pc.count * G, i_row = A.by_group(rr);
      const bool in = rr < n_rows;
      float m_run = -INFINITY, l_run = 0.f, factor_row = 0.f;
      int k_ref = -200;
      bool nan_row = false, have_o = false;
      if (n > 0) {
        // ---- Q into tensor memory: column d holds dims d and d + DH/2
        const long long at = in ? (long long)(pc.first + i_row) * A.q.row + (long long)(pc.hk * G + rr - i_row * G) * A.q.head : 0;
        auto four = [&](int d, float *x) {
          if (!in) { x[0] = x[1] = x[2] = x[3] = 0.f; return; }
          if constexpr (MODE == PAIR) {
            const float4 v = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(A.q.p) + at + d);
            x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(reinterpret_cast<const __half *>(A.q.p) + at + d);
            const bool is_bf16 = A.q_type == KV4_BF16;
            const float2 a = is_bf16 ? make_float2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u)) : unpack2(v.x);
            const float2 b = is_bf16 ? make_float2(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)) : unpack2(v.y);
            x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
          }
        };
        float top = 0.f, sum = 0.f;
#pragma unroll 8
        for (int d = 0; d < DH; d += 4) {
          float x[4];
          four(d, x);
#pragma unroll
          for (int e = 0; e < 4; ++e) { top = fmaxf(top, fabsf(x[e])); sum += x[e]; }
        }
        const int ex = max(-112, min((int)(__float_as_uint(top) >> 23) - 127, 126));
        const float up = pow2i(7 - ex);
        factor_row = fminf(log2_scale / up, 3e38f);
#pragma unroll 1
        for (int c = 0; c < DH / 2; c += 16) {
          uint32_t q[16];
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            float x[4], y[4];
            four(c + e, x);
            four(DH / 2 + c + e, y);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float a = x[k] * up, b = y[k] * up;
              q[e + k] = pack2(a, b);
              if constexpr (MODE == PAIR) {
                const float2 h = unpack2(q[e + k]);
                if (half) q[e + k] = pack2(a - h.x, b - h.y);
              }
            }
          }
          __syncwarp();
          tmem_st16(tmem + lanes + (uint32_t)(COL_Q + c), q);
        }
        {
          // the row's sum against the constants, as two values (three with two parts: the second lane adds the rest)
          const float z = sum * up, zh = __half2float(__float2half_rn(z)), zl = __half2float(__float2half_rn(z - zh)), zr = z - zh - zl;
          uint32_t q[8] = {pack2(zh, zh), pack2(zl, zl), 0u, 0u, 0u, 0u, 0u, 0u};
          if (MODE == PAIR && half) { q[0] = pack2(zr, zr); q[1] = 0u; }
          asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(tmem + lanes + (uint32_t)(COL_Q + DH / 2)),
                       "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]), "r"(q[4]), "r"(q[5]), "r"(q[6]), "r"(q[7]) : "memory");
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(&sync.q_full);
      }
      const bool used = in && !(A.rows.slot != nullptr && A.rows.slot[pc.first + i_row] < 0);
      const uint64_t mk0 = tree && used ? A.rows.mask[(size_t)(pc.first + i_row) * 2] : 0ull, mk1 = tree && used ? A.rows.mask[(size_t)(pc.first + i_row) * 2 + 1] : 0ull;
      const int sees_below = !used ? 0 : tree ? kv : min(kv, pc.ctx + i_row + 1);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const int now = tt + i;
        ok = __all_sync(0xffffffffu, mbar_wait(&sync.info_full[now & (INFO - 1)], (uint32_t)(now / INFO) & 1u) && mbar_wait(&sync.s_full[now & 1], (uint32_t)(now >> 1) & 1u));
        if (!ok) break;
        fence_after();
        const TileInfo &f = sync.info[now & (INFO - 1)];
        const uint32_t s_at = tmem + lanes + (uint32_t)(COL_S + (now & 1) * TK);
        float v[NC];
        {
          uint32_t all[TK];
#pragma unroll
          for (int c = 0; c < TK; c += 16) tmem_ld16(s_at + (uint32_t)c, all + c);
          wait_ld();
          if constexpr (MODE == FULL) {
#pragma unroll
            for (int j = 0; j < NC; ++j) v[j] = __uint_as_float(all[j]);
          } else {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
              v[j] = __uint_as_float(half ? all[32 + j] : all[j]);
              if constexpr (MODE == PAIR) v[j] += __shfl_xor_sync(0xffffffffu, __uint_as_float(half ? all[j] : all[32 + j]), 16);
            }
          }
        }
        const int key0 = (pc.lo + i) * TK;
        float fk[NG];
        int top_exp = -200;
        unsigned any_poison = 0u;
#pragma unroll
        for (int k = 0; k < UG; ++k) {
          top_exp = max(top_exp, f.v_exp[k]);
          any_poison |= f.poison[k] | f.poison_v[k];
        }
#pragma unroll
        for (int k = 0; k < NG; ++k) fk[k] = fminf(factor_row * f.k_back[NG * half + k], 3e38f);
        if (key0 + TK > min(pc.ctx, kv) || any_poison != 0u) {
          uint64_t see = ones_below(sees_below - key0);
          if (tree) see &= tree_bits(mk0, mk1, key0 - pc.ctx);
          if (any_poison != 0u) {
#pragma unroll
            for (int k = 0; k < UG; ++k) nan_row = nan_row || (see >> (KV4_G * k) & (f.poison[k] | f.poison_v[k])) != 0ull;
          }
          see >>= NC * half;
#pragma unroll
          for (int j = 0; j < NC; ++j) v[j] = (see >> j & 1ull) ? v[j] : -INFINITY;
        }
        float m_t = -INFINITY;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
          float a = v[16 * k], b = v[16 * k + 1];
#pragma unroll
          for (int j = 2; j < 16; j += 2) { a = fmaxf(a, v[16 * k + j]); b = fmaxf(b, v[16 * k + j + 1]); }
          m_t = fmaxf(m_t, fmaxf(a, b) * fk[k]);
        }
        if (MODE != FULL) m_t = fmaxf(m_t, __shfl_xor_sync(0xffffffffu, m_t, 16));
        float factor = 1.f;
        if (m_t > m_run + RAISE) {         // (the first visible key sets it)
          factor = m_run == -INFINITY ? 0.f : ex2(m_run - m_t);
          m_run = m_t;
        }
        const int k_was = k_ref;
        k_ref = max(k_ref, top_exp);
        const bool rescale = have_o && (k_ref != k_was || __any_sync(0xffffffffu, factor != 1.f));
        l_run *= factor;
        if (rescale) {
          // every P V issued so far has landed before O is touched; none is issued before this warp has handed over its P
          ok = __all_sync(0xffffffffu, mbar_wait(&sync.pv_done[(now - 1) & 1], (uint32_t)((now - 1) >> 1) & 1u));
          if (!ok) break;
          fence_after();
          const float both = factor * (k_was - k_ref < -126 ? 0.f : pow2i(k_was - k_ref));
#pragma unroll 1
          for (int c = 0; c < DH + 16; c += 16) {
            uint32_t o[16];
            tmem_ld16(tmem + lanes + (uint32_t)(COL_O + c), o);
            wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * both);
            tmem_st16(tmem + lanes + (uint32_t)(COL_O + c), o);
          }
          wait_st();
        }
        const float mu = m_run == -INFINITY ? 0.f : m_run;
        uint32_t p[NC / 2], p_lo[MODE == PAIR ? NC / 2 : 1];
        float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NG; ++k) {
          const float pg = pow2i(max(f.v_exp[NG * half + k] - k_ref, -110) + P_TOP);
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const float a = ex2(fmaf(v[16 * k + j], fk[k], -mu)), b = ex2(fmaf(v[16 * k + j + 1], fk[k], -mu));
            l4[j & 2] += a;
            l4[(j & 2) + 1] += b;
            const uint32_t h = pack2(a * pg, b * pg);
            p[8 * k + j / 2] = h;
            if constexpr (MODE == PAIR) {
              const float2 back = unpack2(h);
              p_lo[8 * k + j / 2] = pack2(a * pg - back.x, b * pg - back.y);
            }
          }
        }
        l_run += (l4[0] + l4[1]) + (l4[2] + l4[3]);
        __syncwarp();
        // ---- P where S was: every lane of this warp has read its S
        if constexpr (MODE == FULL) {
          tmem_st16(s_at, p);
          tmem_st16(s_at + 16u, p + 16);
        } else if constexpr (MODE == HALF) {
          uint32_t a[16], b[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) { a[j] = half ? 0u : p[j]; b[j] = half ? p[j] : 0u; }
          tmem_st16(s_at, a);
          tmem_st16(s_at + 16u, b);
        } else {
          // lane l: the values of all keys, lane l + 16: the residuals
          uint32_t a[16], b[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, half ? p[j] : p_lo[j], 16);
            a[j] = half ? other : p[j];          // keys 0 .. 31
            b[j] = half ? p_lo[j] : other;       // keys 32 .. 63
          }
          tmem_st16(s_at, a);
          tmem_st16(s_at + 16u, b);
        }
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(&sync.p_full[now & 1]);
        have_o = true;
      }
      if (!ok) break;
      // ---- the piece's result
      if (n > 0) {
        const int last = tt + n - 1;
        ok = __all_sync(0xffffffffu, mbar_wait(&sync.pv_done[last & 1], (uint32_t)(last >> 1) & 1u));
        if (!ok) break;
        fence_after();
      }
      if (MODE != FULL) {
        l_run += __shfl_xor_sync(0xffffffffu, l_run, 16);
        const int other = __shfl_xor_sync(0xffffffffu, nan_row ? 1 : 0, 16);      // (by every lane, whatever it has itself)
        nan_row = nan_row || other != 0;
      }
      if (nan_row) l_run = NAN;
      const float unit = exp2f((float)(k_ref - P_TOP));
      float zs = 0.f;
      if (n > 0) {
        uint32_t o[16];
        tmem_ld16(tmem + lanes + (uint32_t)(COL_O + DH), o);
        wait_ld();
        zs = __uint_as_float(o[0]) + __uint_as_float(o[1]);
        if (MODE != FULL) zs += __shfl_xor_sync(0xffffffffu, zs, 16);
      }
      float *part = part_of<DH, ROWS>(scratch, blockIdx.x, pc.begins) + row * PART_ROW<DH>;
#pragma unroll 1
      for (int c = 0; c < DH; c += 16) {   // two words: dims 4l .. 4l + 3 and DH/2 + 4l ..
        uint32_t o[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] = 0u;
        if (n > 0) {
          tmem_ld16(tmem + lanes + (uint32_t)(COL_O + c), o);
          wait_ld();
        }
        float x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          x[j] = __uint_as_float(o[j]);
          if (MODE != FULL) x[j] += __shfl_xor_sync(0xffffffffu, x[j], 16);
          x[j] = (x[j] + zs) * unit;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (!in || (MODE != FULL && k != half)) continue;
          const int d = 4 * (c / 8 + k);
          const float4 lo4 = make_float4(x[8 * k], x[8 * k + 2], x[8 * k + 4], x[8 * k + 6]), hi4 = make_float4(x[8 * k + 1], x[8 * k + 3], x[8 * k + 5], x[8 * k + 7]);
          if (pc.whole) {
            finish(A, pc.first, pc.hk, G, rr, d, lo4, l_run);
            finish(A, pc.first, pc.hk, G, rr, DH / 2 + d, hi4, l_run);
          } else {
            *reinterpret_cast<float4 *>(part + d) = lo4;
            *reinterpret_cast<float4 *>(part + DH / 2 + d) = hi4;
          }
        }
        __syncwarp();
      }
      if (!pc.whole && in && half == 0) *reinterpret_cast<float2 *>(part + DH) = make_float2(m_run, l_run);
      fence_before();
      tt += n;
    }
    if (!ok) atomicExch(&sync.error, 1);
  }

  fence_before();
  __syncthreads();
  const bool failed = sync.error != 0;
  if (warp == MMA_WARP) {
    // MMAs issued before a wait ran out may still be running: no free under them
    if (failed && lane == 0) {
      umma_commit(&sync.drain);
      (void)mbar_wait(&sync.drain, 0);
    }
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)TMEM_COLS) : "memory");
  }
  if (threadIdx.x == 0 && failed && A.rows.status != nullptr) atomicMax(A.rows.status, E_TIMEOUT);
}

template <int DH, int MODE> cudaError_t go(Launch L, const Kv4Attn &a, int num_sms) {
  static SmemOptIn optin;
  cudaError_t e = optin.ensure((const void *)kv4_attn_tc_kernel<DH, MODE>, SMEM<DH>);
  if (e != cudaSuccess) return e;
  constexpr int ROWS = TILE_ROWS<MODE>, RB = 8, JOINERS = 2;
  const int rows = a.rows.max_rows * (a.n_heads / a.c.n_kv_heads), tiles = (rows + ROWS - 1) / ROWS;
  e = launch_k(kv4_attn_tc_kernel<DH, MODE>, dim3(num_sms), dim3(THREADS), SMEM<DH>, L.st, L.pdl, a, a.scratch, tiles);
  if (e != cudaSuccess) return e;
  const int in_tile = rows < ROWS ? rows : ROWS;
  return launch_k(kv4_join_kernel<DH, ROWS, UG, RB, JOINERS>, dim3(a.rows.B * tiles, a.c.n_kv_heads, (in_tile + RB - 1) / RB), dim3(DH / 4 * RB * JOINERS), 0,
                  L.st, L.pdl, a, a.scratch, tiles, (unsigned)num_sms);
}

}  // namespace

size_t kv4_attention_tc_scratch(int dh, int num_sms) { return (size_t)num_sms * 2 * 128 * (dh + 4) * sizeof(float); }

// a.g_inv is set
cudaError_t kv4_attention_tc(Launch L, int dh, const Kv4Attn &a, int num_sms) {
  const int rows = a.rows.max_rows * (a.n_heads / a.c.n_kv_heads);
  const int mode = a.q_type == KV4_FP32 ? PAIR : rows <= 64 ? HALF : FULL;
  if (dh == 128) return mode == PAIR ? go<128, PAIR>(L, a, num_sms) : mode == HALF ? go<128, HALF>(L, a, num_sms) : go<128, FULL>(L, a, num_sms);
  return mode == PAIR ? go<64, PAIR>(L, a, num_sms) : mode == HALF ? go<64, HALF>(L, a, num_sms) : go<64, FULL>(L, a, num_sms);
}

}  // namespace koala
