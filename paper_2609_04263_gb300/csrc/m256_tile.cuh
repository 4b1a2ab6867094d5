// The tile machinery of the tcgen05 attention kernels over affine, symmetric and KIVI
// caches (attend_prefill_m256.cu, attend_shared.cu): shared-memory layout, the packed
// tile's copies, and the reconstruction of its key and value operand tiles.
#pragma once

#include "tc_common.cuh"

namespace kvq {
namespace m256 {
using namespace tc;

constexpr int kM = 128;              // rows per query tile (MMA M)
constexpr int kTok = 64;             // tokens per KV tile
constexpr int kRowsCta = 2 * kM;     // query rows per CTA
constexpr int kProdWarps = 4;
constexpr int kThreads = 14 * 32;    // 8 softmax, 4 producer, 1 issuer, 1 loader warp
constexpr float kRescale = 8.f;      // log2 growth of a row maximum that forces a rescale

// Shared memory (bytes from a 1024-aligned base).
template <int D, int BITS>
struct M256Layout {
  // Two CTAs share each K/V tile where building it bounds the kernel: D = 128 takes
  // 1745 us alone and 1335 paired, D = 64 179 alone and 192 paired (shapes above).
  static constexpr bool PAIR = D == 128;
  static constexpr int KT = PAIR ? kTok / 2 : kTok; // tokens of K per CTA
  static constexpr int VC = PAIR ? D / 2 : D;       // channels of V per CTA
  static constexpr int NP = 32 * kProdWarps;        // producer threads
  static constexpr int KC = KT * D / NP;            // channels of K per thread
  static constexpr int CV = VC * 8 / NP;            // channels of V per thread
  static_assert(KC == 32 && CV == 4, "build_tile: one group of K, one or two code bytes of V a token");
  // score tiles (TMEM) per query tile: what O (2 D columns) leaves of 512
  static constexpr int SB = 2;
  // Reconstructed K/V tile buffers.  A buffer is held from the start of its build to
  // the end of its P V, about three tile times.
  static constexpr int KVB = 4;
  static constexpr int QT = kM * D * 2;             // one query tile: D/64 atoms of 16 KB
  static constexpr int Q_OFF = 0;
  static constexpr int KV_OFF = 2 * QT;
  static constexpr int KH = 0;                      // K hi: D/64 atoms of KT rows x 128 B
  static constexpr int KL = KT * D * 2;             // K lo: the same
  static constexpr int VT = 2 * KT * D * 2;         // V^T: VC rows x 128 B (64 tokens)
  static constexpr int KV_B = VT + VC * 128;
  // packed tile as stored in the cache planes: 64 code rows of K and of V,
  // then four metadata pieces of 4 D bytes each (per-token group scales and
  // offsets of 64 tokens, or KIVI's per-channel scales and offsets of the
  // tile's two 32-token key blocks)
  static constexpr int CROW = D * BITS / 8;         // code bytes per token
  static constexpr int RKC = 0, RVC = kTok * CROW;
  static constexpr int RKS = 2 * kTok * CROW, RKZ = RKS + 4 * D, RVS = RKZ + 4 * D,
                       RVZ = RVS + 4 * D;
  static constexpr int RAW_B = RVZ + 4 * D;
  static constexpr int RAW_OFF = KV_OFF + KVB * KV_B;
  static constexpr int RAW = 3;                     // packed-tile stages (copied ahead)
  static constexpr int KS_OFF = RAW_OFF + RAW * RAW_B;   // KIVI: a key warp's fp32 scales and offsets
  static constexpr int TOTAL = KS_OFF + NP / 32 * 2 * KC * 4;
  static constexpr int ALLOC = TOTAL + 1024;        // alignment slack
  static_assert(ALLOC <= 226 * 1024, "one CTA's shared memory");
};

// The instructions of one CTA or of a pair.
template <bool PAIR>
__device__ __forceinline__ void mma_a_fill(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
  if (PAIR) umma_pair_a_fill(d, a, b, id, acc);
  else umma_a_fill(d, a, b, id, acc);
}
template <bool PAIR>
__device__ __forceinline__ void mma_a_lastuse(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
  if (PAIR) umma_pair_a_lastuse(d, a, b, id, acc);
  else umma_a_lastuse(d, a, b, id, acc);
}
template <bool PAIR>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
  if (PAIR) umma_pair_ts(d, a, b, id, acc);
  else umma_ts(d, a, b, id, acc);
}
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  if (PAIR) umma_commit_pair(bar);
  else umma_commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void arrive_first(uint64_t* bar) {   // on the first CTA's barrier
  if (PAIR) mbar_arrive_pair(mapa(bar, 0));
  else mbar_arrive(bar);
}
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc512(uint32_t* base) {
  if (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(base)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(base)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free512(uint32_t tmem) {
  if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

__device__ __forceinline__ void bulk_copy(void* dst, const void* src, uint32_t bytes,
                                          uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
      ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// Bytes of one packed tile the loader copies (codes of K and V, metadata).
template <int D, int BITS, int FMT>
__host__ __device__ constexpr int raw_bytes() {
  return 2 * kTok * (D * BITS / 8) + (FMT == KVQ_FMT_SYMMETRIC ? 2 : 4) * 4 * D;
}

// Loader: the packed rows of tile t0 .. t0 + 63 of every plane the tile
// reads, one bulk copy per plane.  Planes hold whole 64-row tiles (their
// row counts are padded to multiples of 64), so a tile reaching past the
// stored tokens copies rows that are never used.
template <int D, int BITS, int FMT>
__device__ __forceinline__ void load_raw(const Geom& g, int b, int h, int t0, unsigned char* raw,
                                         uint64_t* bar) {
  using S = M256Layout<D, BITS>;
  constexpr uint32_t CB = kTok * S::CROW;
  mbar_expect_tx(bar, raw_bytes<D, BITS, FMT>());
  // a tile lies in one page of a paged cache: tok_ptr finds its rows
  bulk_copy(raw + S::RKC, tok_ptr<uint8_t>(g, KVQ_PLANE_K_CODES, b, h, t0), CB, bar);
  bulk_copy(raw + S::RVC, tok_ptr<uint8_t>(g, KVQ_PLANE_V_CODES, b, h, t0), CB, bar);
  // KIVI: two key blocks of D channels
  const __half* ks = FMT == KVQ_FMT_KIVI ? blk_ptr<__half>(g, KVQ_PLANE_K_SCALE, b, h, t0 / 32)
                                         : tok_ptr<__half>(g, KVQ_PLANE_K_SCALE, b, h, t0);
  bulk_copy(raw + S::RKS, ks, 4 * D, bar);
  if (FMT != KVQ_FMT_SYMMETRIC) {
    const __half* kz = FMT == KVQ_FMT_KIVI
                           ? blk_ptr<__half>(g, KVQ_PLANE_K_ZERO, b, h, t0 / 32)
                           : tok_ptr<__half>(g, KVQ_PLANE_K_ZERO, b, h, t0);
    bulk_copy(raw + S::RKZ, kz, 4 * D, bar);
  }
  bulk_copy(raw + S::RVS, tok_ptr<__half>(g, KVQ_PLANE_V_SCALE, b, h, t0), 4 * D, bar);
  if (FMT != KVQ_FMT_SYMMETRIC)
    bulk_copy(raw + S::RVZ, tok_ptr<__half>(g, KVQ_PLANE_V_ZERO, b, h, t0), 4 * D, bar);
}

// K: 8 channels reconstructed in fp32 and split into a bf16 high part (the
// value truncated) and the bf16 of the remainder.
__device__ __forceinline__ void split_store(const uint64_t (&k2)[4], unsigned char* hi_dst,
                                            unsigned char* lo_dst) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, c;
    f2unpack(k2[i], a, c);
    const uint32_t ab = __float_as_uint(a) & 0xFFFF0000u, cb = __float_as_uint(c) & 0xFFFF0000u;
    h[i] = __byte_perm(ab, cb, 0x7632);
    float ra, rc;
    f2unpack(fadd2(k2[i], f2pack(-__uint_as_float(ab), -__uint_as_float(cb))), ra, rc);
    l[i] = pack_bf16(ra, rc);
  }
  *reinterpret_cast<uint4*>(hi_dst) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4*>(lo_dst) = make_uint4(l[0], l[1], l[2], l[3]);
}

// Producers: reconstruct this CTA's share of the K and V operand tiles of KV tile t0 from the
// packed tile in `raw` (tokens below tq), the KIVI residual ring (tq <= t < T) or zeros
// (t >= T).  tid 0..127:
//   K: thread (tk = tid % KT, hf = tid / KT): token KT rank + tk, channels
//      KC hf .. KC hf + KC - 1.
//   V: thread (tb = tid % 8, vq = tid % NP / 8): tokens 8 tb .. 8 tb + 7 and
//      channels CV vq .. CV vq + CV - 1 of this CTA's, in half2 arithmetic, stored
//      as rows of the transposed tile (half a 16-byte chunk per row and trip).
template <int D, int BITS, int FMT>
__device__ __forceinline__ void build_tile(const Geom& g, int b, int h, int t0, int T, int tq,
                                           int tid, int rank, const unsigned char* raw, float* ksz,
                                           unsigned char* kv) {
  using S = M256Layout<D, BITS>;
  constexpr bool KIVI = FMT == KVQ_FMT_KIVI;
  constexpr bool SYM = FMT == KVQ_FMT_SYMMETRIC;
  constexpr int NCH = S::KC / 8;                  // K chunks of 8 channels per thread
  constexpr int NKW = S::KC * BITS / 32;          // K code words per thread
  const int tk = tid % S::KT, hf = tid / S::KT, tt = rank * S::KT + tk;
  const int t = t0 + tt;
  // KIVI: the warp's tokens are one block; its scales and offsets of the warp's
  // channels are converted once (a lane one or two channels) and read back as fp32.
  // Converted by every lane for its own token, 128 conversions a tile kept the unit
  // that also serves the softmax warps' exponentials busy (2,282 us against
  // 1,796, shape above, in the version with 64 channels to a thread).
  float* kf = ksz + (tid >> 5) * (2 * S::KC);
  if constexpr (KIVI) {
    __syncwarp();                                  // the previous tile's are read
#pragma unroll
    for (int i = 0; i < S::KC / 32; ++i) {
      const int e = 32 * i + (tid & 31);
      const __half* sp = reinterpret_cast<const __half*>(raw + S::RKS) + (tt >> 5) * D + hf * S::KC + e;
      kf[e] = __half2float(sp[0]);
      kf[S::KC + e] = __half2float(sp[(S::RKZ - S::RKS) / 2]);
    }
    __syncwarp();
  }
  if (t < tq) {
    uint32_t kw[NKW];
    const unsigned char* cp = raw + S::RKC + tt * S::CROW + hf * (S::KC * BITS / 8);
    if constexpr (NKW >= 4) {
#pragma unroll
      for (int i = 0; i < NKW / 4; ++i) {
        const uint4 u = *reinterpret_cast<const uint4*>(cp + 16 * i);
        kw[4 * i] = u.x; kw[4 * i + 1] = u.y; kw[4 * i + 2] = u.z; kw[4 * i + 3] = u.w;
      }
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(cp);
      kw[0] = u.x; kw[1] = u.y;
    }
    uint32_t ks = 0, kz = 0;                      // affine/symmetric: the group's metadata
    if constexpr (!KIVI) {
      const unsigned char* sp = raw + S::RKS + tt * (D / 16) + hf * (S::KC / 16);
      ks = *reinterpret_cast<const unsigned short*>(sp);
      if (!SYM) kz = *reinterpret_cast<const unsigned short*>(sp + (S::RKZ - S::RKS));
    }
    const uint64_t bias2 = f2pack(-8388608.f, -8388608.f);
    constexpr int WT = BITS / 2;                  // code words per trip
#pragma unroll
    for (int c0 = 0; c0 < NCH; c0 += 2) {
      uint32_t cw[WT];
#pragma unroll
      for (int i = 0; i < WT; ++i) cw[i] = kw[i];
#pragma unroll
      for (int i = 0; i + WT < NKW; ++i) kw[i] = kw[i + WT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = c0 + u, cc = hf * NCH + c;    // chunk along D
      const uint32_t w = BITS == 4 ? cw[u * (WT - 1)] : cw[0] >> (16 * u);
      uint64_t k2[4];
      if constexpr (KIVI) {
        const float4* sp = reinterpret_cast<const float4*>(kf + 8 * c);
        const float4* zp = reinterpret_cast<const float4*>(kf + S::KC + 8 * c);
        const float4 sv[2] = {sp[0], sp[1]}, zv[2] = {zp[0], zp[1]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 sq = sv[i / 2], zq = zv[i / 2];
          const uint64_t c2 = fadd2(f2pack(code_biased<BITS>(w, 2 * i), code_biased<BITS>(w, 2 * i + 1)), bias2);
          k2[i] = i & 1 ? ffma2(c2, f2pack(sq.z, sq.w), f2pack(zq.z, zq.w))
                        : ffma2(c2, f2pack(sq.x, sq.y), f2pack(zq.x, zq.y));
        }
      } else {
        const float s = __half2float(__ushort_as_half((unsigned short)ks));
        const float m = SYM ? -(float)(1 << (BITS - 1)) * s : __half2float(__ushort_as_half((unsigned short)kz));
        const uint64_t ss = f2pack(s, s), mm = f2pack(m, m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t c2 = fadd2(f2pack(code_biased<BITS>(w, 2 * i), code_biased<BITS>(w, 2 * i + 1)), bias2);
          k2[i] = ffma2(c2, ss, mm);
        }
      }
      unsigned char* base = kv + (cc >> 3) * (S::KT * 128);
      split_store(k2, base + S::KH + sw128(tk, cc & 7), base + S::KL + sw128(tk, cc & 7));
    }
    }
  } else {
    // KIVI residual window (full precision) or beyond the cache (zeros)
#pragma unroll 1
    for (int c = 0; c < NCH; ++c) {
      const int cc = hf * NCH + c;
      uint4 u = make_uint4(0, 0, 0, 0);
      if (KIVI && t < T)
        u = *reinterpret_cast<const uint4*>(
            plane_ptr<__nv_bfloat16>(g, KVQ_PLANE_K_FULL, b, h, t % g.ring, 8 * cc));
      unsigned char* base = kv + (cc >> 3) * (S::KT * 128);
      *reinterpret_cast<uint4*>(base + S::KH + sw128(tk, cc & 7)) = u;
      *reinterpret_cast<uint4*>(base + S::KL + sw128(tk, cc & 7)) = make_uint4(0, 0, 0, 0);
    }
  }
  constexpr int CV = S::CV;
  // V^T tile: rows CV vq + e, 16-byte chunk tb (tokens 8 tb ..)
  const int tb = tid & 7, vq = tid % S::NP >> 3;
  const int ch = rank * S::VC + vq * CV, grp_v = ch / 32;
  const __half2 bias = __float2half2_rn(1024.f);
#pragma unroll
  for (int p0 = 0; p0 < 4; p0 += 2) {             // tokens 2 p0 .. 2 p0 + 3
  uint32_t out[CV][2];
#pragma unroll
  for (int pp = 0; pp < 2; ++pp) {                // token pair (2p, 2p + 1)
    const int p = p0 + pp;
    uint32_t w2[2], s2u, z2u;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int tv = 8 * tb + 2 * p + u;          // token within the tile
      const unsigned char* cp = raw + S::RVC + tv * S::CROW + ch * BITS / 8;
      if constexpr (BITS == 4) w2[u] = *reinterpret_cast<const unsigned short*>(cp);
      else w2[u] = *cp;
    }
    {
      const int tv = 8 * tb + 2 * p;
      const unsigned short* sp = reinterpret_cast<const unsigned short*>(raw + S::RVS) + tv * (D / 32) + grp_v;
      s2u = (uint32_t)sp[0] | ((uint32_t)sp[D / 32] << 16);
      if constexpr (SYM) {
        const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&s2u),
                                  __float2half2_rn(-(float)(1 << (BITS - 1))));
        z2u = *reinterpret_cast<const uint32_t*>(&z);
      } else {
        const unsigned short* zp = reinterpret_cast<const unsigned short*>(raw + S::RVZ) + tv * (D / 32) + grp_v;
        z2u = (uint32_t)zp[0] | ((uint32_t)zp[D / 32] << 16);
      }
    }
    const uint32_t pw = w2[0] | (w2[1] << 16);
    const __half2 s2 = *reinterpret_cast<const __half2*>(&s2u);
    const __half2 z2 = *reinterpret_cast<const __half2*>(&z2u);
#pragma unroll
    for (int e = 0; e < CV; ++e) {
      constexpr uint32_t m2 = ((1u << BITS) - 1) * 0x00010001u;
      const uint32_t x = ((pw >> (e * BITS)) & m2) | 0x64006400u;
      const __half2 c2 = __hsub2(*reinterpret_cast<const __half2*>(&x), bias);
      const __half2 v2 = __hfma2(s2, c2, z2);
      out[e][pp] = *reinterpret_cast<const uint32_t*>(&v2);
    }
  }
  // tokens of the KIVI residual window, or beyond the cache, replace theirs
  const int tv0 = t0 + 8 * tb + 2 * p0;
  if (tv0 + 3 >= tq) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int tv = tv0 + i;
      if (tv < tq) continue;
      __nv_bfloat16 vals[CV];
      if (KIVI && tv < T) {
        const __nv_bfloat16* src = plane_ptr<__nv_bfloat16>(g, KVQ_PLANE_V_FULL, b, h, tv % g.ring, ch);
        const uint2 u = *reinterpret_cast<const uint2*>(src);
        memcpy(vals, &u, sizeof(vals));
      } else {
#pragma unroll
        for (int e = 0; e < CV; ++e) vals[e] = __float2bfloat16_rn(0.f);
      }
#pragma unroll
      for (int e = 0; e < CV; ++e) {
        const uint32_t hv = __half_as_ushort(__float2half_rn(__bfloat162float(vals[e])));
        out[e][i >> 1] = (i & 1) ? ((out[e][i >> 1] & 0xFFFFu) | (hv << 16))
                                 : ((out[e][i >> 1] & 0xFFFF0000u) | hv);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < CV; ++e)
    *reinterpret_cast<uint2*>(kv + S::VT + sw128(CV * vq + e, tb) + 4 * p0) = make_uint2(out[e][0], out[e][1]);
  }
}

}  // namespace m256
}  // namespace kvq
