// Attention of a paged cache whose sequences share pages (Sections 3.1-3.3 over a
// serving batch): the packed tokens of a run of pages that several sequences hold are read
// and reconstructed once, for the query rows of all of them.
//
// The tree of shared runs (SharedNode, kvq_internal.cuh) cuts every sequence's tokens into
// the nodes on its path and its own leaf.  Softmax over the pieces merges exactly: with
// m_i the maximum, l_i the sum and O_i the weighted values of piece i,
//   M = max m_i,  out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i   (log2 units).
// Three kernels:
//   shared_tc_kernel   the nodes (prefill: the leaves too), tcgen05: the members' rows
//                      stacked to tiles of 128 a CTA, the (node, kv head, row tile) space's
//                      64-token tiles cut into equal ranges, one for each CTA or pair;
//   leaf_kernel        decode: each sequence's own tokens, mma.sync, at most 8 query
//                      heads at a time as the columns of the MMAs;
//   merge_kernel       a warp (or CTA) per query row merges its pieces' partials.
// Everything that depends on lengths or forks is read on the device, so a captured call
// follows the cache.  Long prompts that fill the tiles without other sequences' rows go
// sequence by sequence (alone_faster).
#include <math.h>

#include <algorithm>
#include <atomic>

#include "m256_tile.cuh"
#include "stream_common.cuh"

namespace kvq {
namespace {
using namespace m256;

constexpr int kEntries = kMaxShared + KVQ_MAX_SEQS;   // nodes, then (prefill) leaves
constexpr int kMinTiles = 4;              // places of the work split a CTA (or pair) takes at least
// Places that a unit takes in the work split beside its tiles: what a segment costs a CTA
// whatever its length, and what the tiles of a KIVI leaf's full-precision window cost
// more.  Measured at 2, 3, 5, 7 for all units: 32 sequences' 5 drafted tokens behind 4096
// (affine, short leaves) 56, 58, 66, 69 us, 16 questions behind 16384 (KIVI) 316, 286, 243,
// 219 us.
__host__ __device__ constexpr int unit_cost(int fmt, bool leaf) {
  return 2 + (fmt == KVQ_FMT_KIVI && leaf ? 5 : 0);
}

// N places in P ranges: the first N mod P of them one place longer.
struct Ranges {
  int32_t n, p, q, r;                     // q = N / P, r = N mod P
  __device__ __forceinline__ int start(int c) const { return c * q + min(c, r); }
  __device__ __forceinline__ int of(int x) const {   // the range that holds place x
    const int head = r * (q + 1);
    return x < head ? x / (q + 1) : r + (x - head) / q;
  }
};
__device__ __forceinline__ Ranges make_ranges(int n, int p) { return Ranges{n, p, n / p, n % p}; }

// The schedule, written into the workspace by the first CTA for merge_kernel.
struct Sched {
  Ranges w;                               // places, over CTAs (or pairs)
  int32_t ok, pad[3];
  int32_t tp[kEntries + 1];               // first tile of an entry, all entries' tiles last
  int32_t up[kEntries + 1];               // first unit (kv head, row tile) of an entry
  int32_t roff[KVQ_MAX_SEQS + 1];         // rows of the members before, in the plan's order
};
struct SchedOut : Sched {
  int32_t inv[KVQ_MAX_SEQS];              // place of a sequence in that order
};
constexpr size_t kSchedBytes = (sizeof(SchedOut) + 255) / 256 * 256;

// Query rows of a unit: 128 of each CTA that shares a tile (M256Layout::PAIR).
__host__ __device__ inline int unit_rows_of(int D) { return D == 128 ? 2 * kM : kM; }

// Floats of a slot: O [rows][D], then (m, l) [rows].
__host__ __device__ inline size_t slot_floats(int D) { return (size_t)unit_rows_of(D) * (D + 2); }

// Query rows of sequence b a head (a replayed call attends at most its L).
__device__ __forceinline__ int new_rows(const Geom& g, int b, int L, int decode) {
  return decode ? 1 : min(g.seq_new[b], L);
}

// Rows, tiles and first token of entry e (a node, or the leaf of sequence e - n_nodes).
__device__ __forceinline__ void entry_of(const Geom& g, const int32_t* plan, int n_nodes, int e,
                                         const int32_t* roff, int L, int* rows, int* tiles, int* t0) {
  if (e < n_nodes) {
    const SharedNode nd = plan_nodes(plan)[e];
    *rows = roff[nd.first + nd.count] - roff[nd.first];
    *tiles = (nd.p1 - nd.p0) * (kPageTok / kTok);
    *t0 = nd.p0 * kPageTok;
  } else {
    const int b = e - n_nodes;
    *t0 = plan_leaf_page(plan, g.B)[b] * kPageTok;
    *rows = new_rows(g, b, L, 0) * (g.Hq / g.H);
    *tiles = max(0, g.seq_len[b] - *t0 + kTok - 1) / kTok;
  }
}

// Exclusive sums in place of n values (a[n] receives the total): warp 0.
__device__ __forceinline__ void warp_scan(int32_t* a, int n) {
  const int lane = threadIdx.x & 31;
  int run = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += 32) {
    const int v = i0 + lane < n ? a[i0 + lane] : 0;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    __syncwarp();
    if (i0 + lane < n) a[i0 + lane] = run + incl - v;
    run += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (lane == 0) a[n] = run;
}

// Largest i in [lo, hi) with a[i] <= x (a ascending, a[lo] <= x).
__device__ __forceinline__ int find_le(const int32_t* a, int lo, int hi, int x) {
#pragma unroll 1
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A place in the flattened space: position `at` of row tile ut of head `head` of entry e.
// The roles walk on from the first one of the CTA (or pair) without a division: seven
// copies of the searches and divisions that find a place took 5,000 cycles to fetch.
struct Walk {
  int x, e, head, ut, at;
};
// A piece of a unit that one CTA (or pair) works through: rows of the unit, its first row in
// the entry, its first token and its tiles.
struct Segment {
  int e, head, slot, rows, row0, n, t0, b;
};
// The next segment with tiles before place x1 (n = 0: none).
template <int FMT>
__device__ __forceinline__ Segment next_segment(const Geom& g, const Sched& sc, Walk& w, int x1, int ne,
                                                int n_nodes, int L, int RU, int gr) {
  Segment s;
  s.n = 0;
#pragma unroll 1
  while (w.x < x1 && s.n <= 0) {
    int rows, tiles;
    entry_of(g, g.shared_plan, n_nodes, w.e, sc.roff, L, &rows, &tiles, &s.t0);
    const int per = (rows + RU - 1) / RU, cost = unit_cost(FMT, w.e >= n_nodes), len = tiles + cost;
    const int take = min(len - w.at, x1 - w.x);          // places, a unit's first without tiles
    const int tile0 = max(0, w.at - cost);
    s.n = w.at + take - cost - tile0;
    s.e = w.e;
    s.head = w.head;
    s.row0 = w.ut * RU;
    s.rows = min(RU, rows - s.row0);
    s.slot = sc.up[w.e] + w.head * per + w.ut + gr;
    s.b = w.e < n_nodes ? plan_order(g.shared_plan)[plan_nodes(g.shared_plan)[w.e].first] : w.e - n_nodes;
    s.t0 += tile0 * kTok;
    w.x += take;
    w.at = 0;
    if (++w.ut == per) {
      w.ut = 0;
      if (++w.head == g.H) {
        w.head = 0;
        do ++w.e; while (w.e < ne && sc.up[w.e + 1] == sc.up[w.e]);
      }
    }
  }
  s.n = max(s.n, 0);
  return s;
}

// =============================================================================
// nodes (and leaves of a prefill) on tcgen05.  128 query rows a CTA, two CTAs that share
// each K/V tile at head_dim 128 (the tiles and their producers' code are those of
// attend_prefill_m256.cu).  A CTA (or pair) goes through segments of several units, each
// of which leaves a partial.  Roles:
//   softmax (warps 0-3 and 4-7): two streams that take the tiles in turn, each with its own
//     running m and l and its own O in TMEM, thread r of a stream owning row r; joined
//     when the segment's partial is stored (a thread stores half of a row's channels);
//   producers (warps 8-19): three groups that take the tiles in turn, each warp a quarter of
//     the CTA's keys and values (a tile's waits, fences and arrivals take as long as half of
//     its build, and a tile built by all at once would pay them every time);
//   MMAs, a warp each: Q K^T (warp 20), ahead of P V (warp 22) by up to four score
//     buffers and across segments (two Q tiles, the next segment's loaded while this one
//     runs).  One warp for both spent 1,700 of 2,050 cycles a tile on the way between its
//     waits;
//   loaders: the keys' packed tiles (warp 21), the values' (warp 23).
// What bounds it, per 64-token tile at D = 128, about 1,500 cycles (16 questions behind 16384
// tokens, KIVI 4-bit: 184 us, 630 TFLOP/s counted once for Q K^T; MMAs busy 44 %, issue slots 57 %,
// shared memory 60 % of the time): no one unit, but the roles' latencies beside each other on
// six warps a scheduler.  The MMAs alone are 768 cycles (Q K_hi^T, Q K_lo^T and P V for 128 rows
// a CTA), building a tile 4,300 by each of three groups, a stream's softmax 1,250 to 2,300 for
// every second tile.  Tried: P apart from the scores in TMEM, so that a score buffer is free as
// soon as it is read, 184 -> 186 us; 256 rows a CTA that share a built tile, 14 % less a row tile
// but units twice as coarse (64 samples of one context 102 -> 127 us); keys as one fp16 operand
// (512 cycles of MMAs, half the building) 172 us, for 11 bits of a key in place of 16 and
// fp16's range: not taken.
// =============================================================================
constexpr int kTcWarps = 24;
constexpr int kBuildWarps = 12, kGroups = 3;           // producers: groups of 4 warps
// Registers a thread: the block starts with kRegs each (launch bounds; checked before the
// launch) and its warpgroups share them out anew.
constexpr int kRegs = 80, kRegsSoftmax = 112, kRegsBuild = 64, kRegsIssue = 64;
static_assert(2 * kRegsSoftmax + 3 * kRegsBuild + kRegsIssue <= 6 * kRegs, "no more than the block has");
template <int N>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr int kTcThreads = kTcWarps * 32;
constexpr int kSBuf = 4;                               // score buffers (TMEM)

template <int D, int BITS>
struct TcLayout {
  using M = M256Layout<D, BITS>;
  // Buffers of keys (high, low), of values, and packed tiles copied ahead.  Multiples of
  // kGroups: each group of producers takes every third tile, and a barrier's parity tells a
  // phase only from its neighbours, so a group has to meet every phase of its buffers.
  static constexpr int KB = 3, VB = 6, RAW = 6;
  static constexpr int K_B = 2 * M::KT * D * 2, V_B = M::VC * 128;
  static constexpr int KH = 0, KL = M::KT * D * 2;     // of a key buffer
  // a packed tile: this CTA's keys' codes, all values' codes, scales and offsets of both
  static constexpr int CROW = M::CROW, KMETA = 4 * D * M::KT / kTok, VMETA = 4 * D;
  static constexpr int RKC = 0, RVC = M::KT * CROW, RKS = RVC + kTok * CROW, RKZ = RKS + KMETA,
                       RVS = RKZ + KMETA, RVZ = RVS + VMETA, RAW_B = RVZ + VMETA;
  static constexpr int Q_OFF = 0;                      // two Q tiles
  static constexpr int K_OFF = 2 * M::QT;
  static constexpr int V_OFF = K_OFF + KB * K_B;
  static constexpr int RAW_OFF = V_OFF + VB * V_B;
  static constexpr int KS_OFF = RAW_OFF + RAW * RAW_B;
  static constexpr int TOTAL = KS_OFF + kBuildWarps * 256;   // the producers' tables
  static constexpr int ALLOC = TOTAL + 1024;           // alignment slack
  static_assert(KB % kGroups == 0 && VB % kGroups == 0 && RAW % kGroups == 0, "see above");
  static_assert(ALLOC + (int)sizeof(Sched) + 2700 <= 227 * 1024, "one CTA's shared memory");
};

// ---- operand tiles of 64 tokens.  Coded tokens end at a multiple of 32 where a KIVI window
// follows, so a warp's 32 keys are all coded or all at full precision; values may be of both.
// Keys behind the last token may be anything (their scores are replaced), values are 0. ----

// This CTA's keys, 128 threads: a token tk, 32 channels from 32 hf each.  A code c is
// read as the float x = 1 + c 2^(k - 23): its bits k.. of the mantissa, in place for 8 bits of
// codes at a time (k = 15 ..), so that one FMA gives s c + z = s' x + (z - s') with
// s' = s 2^(23 - k) <= 256 s (the constant's rounding, 2^-16 s at most, is that of the low
// part).  Then the bf16 high part (truncated) and the bf16 of the remainder.
// sz: the warp's table of s' and z - s' (KIVI).
template <int D, int BITS, int FMT>
__device__ __forceinline__ void keys_tile(int tid, const unsigned char* raw, float* sz,
                                          unsigned char* kv) {
  using S = M256Layout<D, BITS>;
  using Y = TcLayout<D, BITS>;
  constexpr bool KIVI = FMT == KVQ_FMT_KIVI, SYM = FMT == KVQ_FMT_SYMMETRIC;
  constexpr int NW = BITS;                               // words of 32 channels' codes
  constexpr int WIN = 8 / BITS;                          // codes of 8 bits
  const int lane = tid & 31;
  int tk, hf;
  if constexpr (KIVI) {                                  // (a warp's table holds its 32 channels)
    tk = tid % S::KT;
    hf = tid / S::KT;
  } else if constexpr (S::KT == 32) {
    // a warp takes 8 tokens: lanes that load or store together (8, bits 0 .. 2) differ in bank
    hf = (lane >> 1) & 3;
    tk = (tid >> 5) * 8 + (lane & 1) + ((hf & 2) ^ ((lane >> 2) & 2)) + ((lane >> 2) & 4);
  } else {
    hf = lane & 1;
    tk = tid >> 1;
  }
  // weight of the code at place i of its 8 bits
  const auto weight = [](int i) { return (float)(1 << (8 - BITS * i)); };
  uint32_t w[NW];
  {
    const unsigned char* cp = raw + Y::RKC + tk * S::CROW + hf * (4 * BITS);
    if constexpr (NW == 4) {
      const uint4 u = *reinterpret_cast<const uint4*>(cp);
      w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(cp);
      w[0] = u.x; w[1] = u.y;
    }
  }
  uint64_t s2[WIN / 2], z2[WIN / 2], st[4], zt[4];       // per-token groups: by place; KIVI: of 8 channels
  if constexpr (KIVI) {
    __syncwarp();                                        // the previous tile's table is read
    const __half* sp = reinterpret_cast<const __half*>(raw + Y::RKS) + (tk >> 5) * D + hf * 32 + lane;
    const float sc = __half2float(sp[0]) * weight(lane % WIN);
    sz[lane] = sc;
    sz[32 + lane] = __half2float(sp[(Y::RKZ - Y::RKS) / 2]) - sc;
    __syncwarp();
  } else {
    const unsigned char* sp = raw + Y::RKS + tk * (D / 16) + hf * 2;
    const float sc = __half2float(*reinterpret_cast<const __half*>(sp));
    const float z = SYM ? -(float)(1 << (BITS - 1)) * sc
                        : __half2float(*reinterpret_cast<const __half*>(sp + (Y::RKZ - Y::RKS)));
#pragma unroll
    for (int i = 0; i < WIN / 2; ++i) {
      const float a = sc * weight(2 * i), b = sc * weight(2 * i + 1);
      s2[i] = f2pack(a, b);
      z2[i] = f2pack(z - a, z - b);
    }
  }
  const uint64_t neg1 = f2pack(-1.f, -1.f);
  unsigned char* base = kv + (hf >> 1) * (S::KT * 128);
#pragma unroll
  for (int c = 0; c < 4; ++c) {                          // 8 channels
    uint32_t h[4], l[4];
    if constexpr (KIVI) {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(sz + 8 * c + 2 * i);
        const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(sz + 32 + 8 * c + 2 * i);
        st[i] = a.x; st[i + 1] = a.y;
        zt[i] = b.x; zt[i + 1] = b.y;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {                        // channels 8 c + 2 i, + 1
      const int ch = 8 * c + 2 * i, bit = ch * BITS, at = bit % 32 / 8;
      const uint32_t word = w[bit / 32];
      const uint32_t x = at == 0 ? word << 15 : at == 1 ? word << 7 : at == 2 ? word >> 1 : word >> 9;
      constexpr uint32_t mask = (1u << BITS) - 1;
      const int k = 15 + bit % 8;
      const uint64_t x2 = f2pack(__uint_as_float((x & (mask << k)) | 0x3F800000u),
                                 __uint_as_float((x & (mask << (k + BITS))) | 0x3F800000u));
      uint64_t sv, zv;
      if constexpr (KIVI) {
        sv = st[i];
        zv = zt[i];
      } else {
        sv = s2[ch % WIN / 2];
        zv = z2[ch % WIN / 2];
      }
      const uint64_t kk = ffma2(x2, sv, zv);
      float a, b;
      f2unpack(kk, a, b);
      const uint32_t ab = __float_as_uint(a) & 0xFFFF0000u, bb = __float_as_uint(b) & 0xFFFF0000u;
      h[i] = __byte_perm(ab, bb, 0x7632);
      f2unpack(ffma2(f2pack(__uint_as_float(ab), __uint_as_float(bb)), neg1, kk), a, b);
      l[i] = pack_bf16(a, b);
    }
    const int at = sw128(tk, (4 * hf + c) & 7);
    *reinterpret_cast<uint4*>(base + Y::KH + at) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(base + Y::KL + at) = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// The same from a KIVI window: token t (its slot of the ring), nothing in the low part.
template <int D, int BITS>
__device__ __forceinline__ void keys_window(const Geom& g, int b, int h, int t, int tid, unsigned char* kv) {
  using S = M256Layout<D, BITS>;
  using Y = TcLayout<D, BITS>;
  const int tk = tid % S::KT, hf = tid / S::KT;
  const uint4* src = reinterpret_cast<const uint4*>(
      plane_ptr<__nv_bfloat16>(g, KVQ_PLANE_K_FULL, b, h, t % g.ring, 32 * hf));
  uint4 v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = src[c];
  unsigned char* base = kv + (hf >> 1) * (S::KT * 128);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int at = sw128(tk, (4 * hf + c) & 7);
    *reinterpret_cast<uint4*>(base + Y::KH + at) = v[c];
    *reinterpret_cast<uint4*>(base + Y::KL + at) = make_uint4(0, 0, 0, 0);
  }
}

// This CTA's values, 128 threads: tokens 2 (tid / 4), + 1, and 16 channels from 16 (tid % 4), as
// words of the transposed tile's rows, from a channel on that differs by 2 between a warp's
// groups of channels, so that its 32 words differ in bank.  left: tokens of the tile.
// v = c s + z in fp16, one rounding (c exact: 1024 + c less 1024).
// (With 16 channels to a warp its lanes read codes 128 bytes apart, 32 wavefronts for 2: 42 % of
// all shared memory's were conflicts, and 16 questions behind 16384 took 189 us, now 184.)
template <int D, int BITS, int FMT>
__device__ __forceinline__ void values_tile(int tid, int rank, const unsigned char* raw, int left,
                                            unsigned char* vt) {
  using S = M256Layout<D, BITS>;
  using Y = TcLayout<D, BITS>;
  constexpr bool SYM = FMT == KVQ_FMT_SYMMETRIC;
  static_assert(S::VC == 64, "16 channels a warp");
  constexpr int NW = BITS / 2;                           // words of 16 channels' codes
  const int tp = tid >> 2, vq = tid & 3, ch = rank * S::VC + 16 * vq;
  uint32_t w[2][NW], s2, z2 = 0;
  {
    const unsigned char* cp = raw + Y::RVC + 2 * tp * S::CROW + ch * BITS / 8;
    const unsigned short* sp = reinterpret_cast<const unsigned short*>(raw + Y::RVS) + 2 * tp * (D / 32) + ch / 32;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (NW == 2) {
        const uint2 u = *reinterpret_cast<const uint2*>(cp + t * S::CROW);
        w[t][0] = __funnelshift_r(u.x, u.y, 8 * vq);
        w[t][1] = __funnelshift_r(u.y, u.x, 8 * vq);
      } else {
        const uint32_t u = *reinterpret_cast<const uint32_t*>(cp + t * S::CROW);
        w[t][0] = __funnelshift_r(u, u, 4 * vq);
      }
    }
    s2 = (uint32_t)sp[0] | ((uint32_t)sp[D / 32] << 16);
    if constexpr (!SYM) {
      const unsigned short* zp = sp + (Y::RVZ - Y::RVS) / 2;
      z2 = (uint32_t)zp[0] | ((uint32_t)zp[D / 32] << 16);
    }
    // rows behind the last token may hold anything: their scales and offsets count as 0
    const uint32_t live = 2 * tp >= left ? 0u : 2 * tp + 1 >= left ? 0xFFFFu : 0xFFFFFFFFu;
    s2 &= live;
    z2 &= live;
  }
  // 1024 (and a symmetric code's zero) off, exactly
  constexpr uint32_t off = (0x6400u + (SYM ? (1u << (BITS - 1)) : 0u)) * 0x00010001u;
  constexpr uint32_t m2 = ((1u << BITS) - 1) * 0x00010001u;
  const __half2 o2 = *reinterpret_cast<const __half2*>(&off);
  const __half2 sc = *reinterpret_cast<const __half2*>(&s2), zz = *reinterpret_cast<const __half2*>(&z2);
  // rows r = 16 vq + (e + 2 vq) % 16, the 16-byte chunk tp / 4 of each, word tp % 4
  const auto value = [&](int e) {
    const int bit = e * BITS;
    // both tokens' codes, 16 bits of each to a word
    const uint32_t pw = __byte_perm(w[0][bit / 32], w[1][bit / 32], bit % 32 < 16 ? 0x5410 : 0x7632);
    const uint32_t x = ((pw >> (bit % 16)) & m2) | 0x64006400u;
    const __half2 c2 = __hsub2(*reinterpret_cast<const __half2*>(&x), o2);
    const __half2 v = SYM ? __hmul2(c2, sc) : __hfma2(c2, sc, zz);
    return *reinterpret_cast<const uint32_t*>(&v);
  };
  unsigned char* dst = vt + 2 * vq * 1024 + 4 * (tp & 3);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int r = e + 2 * vq;                            // (of 16; below 14)
    const int at = r * 128 + (((tp >> 2) ^ (r & 7)) << 4);
    *reinterpret_cast<uint32_t*>(dst + at) = value(e);
    *reinterpret_cast<uint32_t*>(dst + (at ^ 1024)) = value(e + 8);
  }
}

// The same from a KIVI window (and zeros behind it), for a thread whose tokens t, t + 1 are there.
template <int D, int BITS>
__device__ __forceinline__ void values_window(const Geom& g, int b, int h, int t, int T, int tid, int rank,
                                              unsigned char* vt) {
  using S = M256Layout<D, BITS>;
  const int tp = tid >> 2, vq = tid & 3;
  const int slot = t % g.ring, slot1 = slot + 1 == g.ring ? 0 : slot + 1;
  const __nv_bfloat16* base = plane_ptr<__nv_bfloat16>(g, KVQ_PLANE_V_FULL, b, h, 0, rank * S::VC + 16 * vq);
  const uint4* a = reinterpret_cast<const uint4*>(base + (size_t)slot * D);
  const uint4* c = reinterpret_cast<const uint4*>(base + (size_t)slot1 * D);
  unsigned char* dst = vt + 2 * vq * 1024 + 4 * (tp & 3);
  const auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
  const auto hi = [](uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); };
  const uint4 z = make_uint4(0, 0, 0, 0);
  uint4 u[2], w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u[i] = t < T ? a[i] : z;
    w[i] = t + 1 < T ? c[i] : z;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t x = reinterpret_cast<const uint32_t*>(u)[i], y = reinterpret_cast<const uint32_t*>(w)[i];
    *reinterpret_cast<uint32_t*>(dst + sw128(2 * i, tp >> 2)) = pack_h2(lo(x), lo(y));
    *reinterpret_cast<uint32_t*>(dst + sw128(2 * i + 1, tp >> 2)) = pack_h2(hi(x), hi(y));
  }
}

// The bounded waits of tc_common.cuh with the SM's own clock: a wait that does not find its
// phase complete at once would otherwise read the global timer first.
constexpr long long kWaitCycles = 2000000000ll;        // about a second
__device__ __forceinline__ bool bar_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
#pragma unroll 1
  while (!mbar_try_wait(bar, parity)) {
    if (*abort) return false;
    if (clock64() - t0 > kWaitCycles) {
      *abort = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool warp_bar_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xffffffffu, bar_wait(bar, parity, abort));
}
// Two waits, both barriers asked before the first answer is there.
__device__ __forceinline__ bool warp_bar_wait2(uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1, volatile int* abort) {
  const bool d0 = mbar_try_wait(b0, p0), d1 = mbar_try_wait(b1, p1);
  return __all_sync(0xffffffffu, (d0 || bar_wait(b0, p0, abort)) && (d1 || bar_wait(b1, p1, abort)));
}
// Whether a phase is complete, without waiting.
__device__ __forceinline__ bool bar_done(uint64_t* bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
               "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return done;
}
__device__ __forceinline__ void softmax_sync() {       // the softmax warps
  asm volatile("bar.sync 1, 256;" ::: "memory");
}

template <int D, int BITS, int FMT>
__global__ void __launch_bounds__(kTcThreads, 1)
shared_tc_kernel(const __grid_constant__ Geom g, const __nv_bfloat16* __restrict__ q, int L, int decode, float scale,
                 SchedOut* sched, float* __restrict__ slots, int cap, int* err) {
  using S = M256Layout<D, BITS>;
  using Y = TcLayout<D, BITS>;
  constexpr int NC = S::PAIR ? 2 : 1;                  // CTAs that share a K/V tile
  constexpr int RU = NC * kM;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t raw_k[Y::RAW], raw_v[Y::RAW], raw_k_free[Y::RAW], raw_v_free[Y::RAW], k_full[Y::KB], k_free[Y::KB], v_full[Y::VB],
      v_free[Y::VB], s_full[kSBuf], p_full[kSBuf], s_free[kSBuf], q_full[2], o_free, done_bar;
  __shared__ uint32_t tmem_base;
  __shared__ int abort_flag;
  __shared__ float2 row_ml[2][kM];                     // a stream's (m, l) of each row
  __shared__ Sched sc;
  __shared__ Walk first_place;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = S::PAIR ? cluster_rank() : 0;
  const int grp = g.Hq / g.H;
  if (threadIdx.x == 0) {
    for (int i = 0; i < Y::RAW; ++i) {
      mbar_init(&raw_k[i], 1);
      mbar_init(&raw_v[i], 1);
      mbar_init(&raw_k_free[i], 4);
      mbar_init(&raw_v_free[i], 4);
    }
    for (int i = 0; i < Y::KB; ++i) {
      mbar_init(&k_full[i], NC * 4);
      mbar_init(&k_free[i], 1);
    }
    for (int i = 0; i < Y::VB; ++i) {
      mbar_init(&v_full[i], NC * 4);
      mbar_init(&v_free[i], 1);
    }
    for (int i = 0; i < kSBuf; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], NC * 4);
      mbar_init(&s_free[i], 1);
    }
    mbar_init(&q_full[0], NC * 8);
    mbar_init(&q_full[1], NC * 8);
    mbar_init(&o_free, NC * 8);
    mbar_init(&done_bar, 2);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 20) tmem_alloc512<S::PAIR>(&tmem_base);
  pdl_wait();
  const int32_t* plan = g.shared_plan;
  const int n_nodes = plan[0], ne = n_nodes + (decode ? 0 : g.B);
  volatile int* abort = &abort_flag;
  pdl_trigger();

  // ---- the schedule (every CTA forms the same) ----
  if (!decode) {
#pragma unroll 1
    for (int i = threadIdx.x; i < g.B; i += kTcThreads)
      sc.roff[i] = new_rows(g, n_nodes ? plan_order(plan)[i] : i, L, 0) * grp;
    __syncthreads();
    if (warp == 0) warp_scan(sc.roff, g.B);
  } else {
#pragma unroll 1
    for (int i = threadIdx.x; i <= g.B; i += kTcThreads) sc.roff[i] = i * grp;
  }
  __syncthreads();
#pragma unroll 1
  for (int e = threadIdx.x; e < ne; e += kTcThreads) {
    int rows, tiles, t0;
    entry_of(g, plan, n_nodes, e, sc.roff, L, &rows, &tiles, &t0);
    const int units = tiles > 0 ? g.H * ((rows + RU - 1) / RU) : 0;
    sc.up[e] = units;
    sc.tp[e] = units * (tiles + unit_cost(FMT, e >= n_nodes));
  }
  __syncthreads();
  if (warp == 0) warp_scan(sc.up, ne);
  if (warp == 1) warp_scan(sc.tp, ne);
  __syncthreads();
  const int N = sc.tp[ne], P = max(1, min((int)gridDim.x / NC, N / kMinTiles));
  const Ranges ranges = make_ranges(N, P);
  const bool ok_cap = sc.up[ne] + P <= cap;
  if (blockIdx.x == 0) {                                 // for merge_kernel
    if (threadIdx.x == 0) {
      sched->w = ranges;
      sched->ok = ok_cap;
      if (!ok_cap) atomicOr(&g.state->error, kErrWorkspace);
    }
#pragma unroll 1
    for (int i = threadIdx.x; i <= ne; i += kTcThreads) {
      sched->tp[i] = sc.tp[i];
      sched->up[i] = sc.up[i];
    }
#pragma unroll 1
    for (int i = threadIdx.x; i < g.B; i += kTcThreads) {
      sched->roff[i] = sc.roff[i];
      sched->inv[n_nodes ? plan_order(plan)[i] : i] = i;
    }
  }
  // ---- where this CTA (or pair) starts and ends ----
  const int gr = blockIdx.x / NC;
  const bool idle = !ok_cap || gr >= P || N == 0;
  const int x1 = idle ? 0 : ranges.start(gr + 1);
  if (threadIdx.x == 0) {
    Walk w{0, 0, 0, 0, 0};
    if (!idle) {
      w.x = ranges.start(gr);
      w.e = find_le(sc.tp, 0, ne, w.x);
      const int units = sc.up[w.e + 1] - sc.up[w.e], len = (sc.tp[w.e + 1] - sc.tp[w.e]) / units, per = units / g.H;
      const int r = w.x - sc.tp[w.e], u = r / len;
      w.at = r - u * len;
      w.head = u / per;
      w.ut = u - w.head * per;
    }
    first_place = w;
  }
  auto segment = [&](Walk& w) { return next_segment<FMT>(g, sc, w, x1, ne, n_nodes, L, RU, gr); };

  tc_fence_before();
  if (S::PAIR) cluster_sync();                         // both CTAs' barriers are set up
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base;
  Walk walk = first_place;

  if (warp >= 8 + kBuildWarps) {
  regs_dec<kRegsIssue>();
  if (warp == 21 || warp == 23) {
    // ---------------- loaders: packed tiles into the raw rings, of the keys and the values ----
    // One elected lane copies a tile's codes, scales and offsets (of the keys, this CTA's
    // tokens or block).  The page's number is read a page ahead: six look-ups a tile by one
    // thread, each in the way of the next, took 2,000 cycles a tile, and six lanes' copies
    // in one warp 1,700.
    constexpr bool SYM = FMT == KVQ_FMT_SYMMETRIC;
    const bool keys = warp == 21;
    const Plane &pc = g.pl[keys ? KVQ_PLANE_K_CODES : KVQ_PLANE_V_CODES],
                &ps = g.pl[keys ? KVQ_PLANE_K_SCALE : KVQ_PLANE_V_SCALE],
                &pz = g.pl[keys ? KVQ_PLANE_K_ZERO : KVQ_PLANE_V_ZERO];
    // bytes a tile (kTok tokens) takes in a plane of codes and of scales or offsets, and this CTA's
    constexpr uint32_t kCodes = kTok * S::CROW, kMeta = 4 * D;
    const uint32_t codes = keys ? kCodes * S::KT / kTok : kCodes, meta = keys ? Y::KMETA : kMeta;
    const uint32_t skip_c = keys ? rank * codes : 0, skip_m = keys ? rank * meta : 0;
    const uint32_t bytes = codes + (SYM ? 1 : 2) * meta;
    unsigned char* dst_c = smem + Y::RAW_OFF + (keys ? Y::RKC : Y::RVC);
    unsigned char* dst_s = smem + Y::RAW_OFF + (keys ? Y::RKS : Y::RVS);
    uint64_t *full = keys ? raw_k : raw_v, *free = keys ? raw_k_free : raw_v_free;
    const bool leader = elect_one();
    uint32_t st = 0, ph = 1;                             // (free at first)
    int issued = 0;
    bool ok = true;
    while (ok) {
      const Segment s = segment(walk);
      if (s.n == 0) break;
      // a page's rows of this head in each plane
      const char* c_head = static_cast<const char*>(pc.p) + (int64_t)s.head * pc.rows * S::CROW + skip_c;
      const int64_t m_head = (int64_t)s.head * ps.rows * ps.cols * 2 + skip_m;
      const char *s_head = static_cast<const char*>(ps.p) + m_head, *z_head = static_cast<const char*>(pz.p) + m_head;
      const int32_t* pages = g.page_table + (size_t)s.b * g.max_pages;
      const int last = (s.t0 + s.n * kTok - 1) >> kPageShift;
      int page = pages[s.t0 >> kPageShift], ahead = pages[min((s.t0 >> kPageShift) + 1, last)];
#pragma unroll 1
      for (int j = 0; j < s.n; ++j) {
        const int t0 = s.t0 + j * kTok, in_page = (t0 & (kPageTok - 1)) / kTok;
        if (j && in_page == 0) {
          page = ahead;
          ahead = pages[min((t0 >> kPageShift) + 1, last)];
        }
        ok = warp_bar_wait(&free[st], ph, abort);
        if (!ok) break;
        if (leader) {
          const int64_t tile = (int64_t)page * (kPageTok / kTok) + in_page;
          mbar_expect_tx(&full[st], bytes);
          bulk_copy(dst_c + st * Y::RAW_B, c_head + tile * kCodes, codes, &full[st]);
          bulk_copy(dst_s + st * Y::RAW_B, s_head + tile * kMeta, meta, &full[st]);
          if (!SYM) bulk_copy(dst_s + st * Y::RAW_B + meta, z_head + tile * kMeta, meta, &full[st]);
        }
        __syncwarp();
        ++issued;
        if (++st == Y::RAW) st = 0, ph ^= 1;
      }
    }
    // no copy may still be landing in shared memory when the CTA exits
    if (lane == 0)
      for (int i = max(0, issued - Y::RAW); i < issued; ++i)
        if (!mbar_wait(&full[i % Y::RAW], (i / Y::RAW) & 1)) *abort = 1;
  } else if (warp == 20 && rank == 0) {
    // ---------------- scores: S = Q K_hi^T + Q K_lo^T of each tile ----------------
    // The warp stays whole (its values are uniform) and one elected lane issues.
    // Descriptors are formed once: a K step of 16 elements advances the start address by 32
    // bytes (2 in the descriptor's 16-byte units).
    constexpr uint32_t id_qk = idesc_bf16(NC * kM, kTok);
    const uint64_t qdesc0 = sw128_desc(smem + Y::Q_OFF), kdesc0 = sw128_desc(smem + Y::K_OFF);
    uint32_t kb = 0, kph = 0, bf = 0, sph = 1, qb = 0, qph = 0;   // s_free: free at first
    bool ahead = false;                                  // the next tile is known to be ready
    const bool leader = elect_one();
    bool ok = true;
    while (ok) {
      const int n = segment(walk).n;
      if (n == 0 || !warp_bar_wait(&q_full[qb], qph, abort)) break;   // the segment's queries
      const uint64_t qd = qdesc0 + qb * (S::QT >> 4);
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        ok = ahead || warp_bar_wait2(&k_full[kb], kph, &s_free[bf], sph, abort);
        if (!ok) break;
        tc_fence_after();
        const uint32_t kb0 = kb, bf0 = bf;
        if (++kb == Y::KB) kb = 0, kph ^= 1;
        if (++bf == kSBuf) bf = 0, sph ^= 1;
        const bool k_next = bar_done(&k_full[kb], kph), s_next = bar_done(&s_free[bf], sph);
        if (leader) {
          const uint32_t ts = tmem + bf0 * kTok;
          const uint64_t kd = kdesc0 + kb0 * (Y::K_B >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            // Q atom: 128 rows x 128 B (1024 units); K atom: KT rows x 128 B (8 KT units)
            const uint64_t a = qd + ((kk >> 2) * 1024 + (kk & 3) * 2), k = kd + ((kk >> 2) * (8 * S::KT) + (kk & 3) * 2);
            mma_a_fill<S::PAIR>(ts, a, k + (S::KH >> 4), id_qk, kk > 0);   // Q read once
            mma_a_lastuse<S::PAIR>(ts, a, k + (S::KL >> 4), id_qk, 1);     // for K hi and lo
          }
          mma_commit<S::PAIR>(&s_full[bf0]);
          mma_commit<S::PAIR>(&k_free[kb0]);
        }
        __syncwarp();
        ahead = __all_sync(0xffffffffu, k_next && s_next);
      }
      qb ^= 1;
      qph ^= qb ^ 1;
    }
    if (leader) mma_commit<S::PAIR>(&done_bar);          // every MMA issued above has completed
    if (lane == 0 && !mbar_wait(&done_bar, 0)) *abort = 1;
    __syncwarp();
  } else if (warp == 22 && rank == 0) {
    // ---------------- values: O += P V of each tile, of its stream's O ----------------
    constexpr uint32_t id_pv = idesc_f16(NC * kM, D);
    const uint64_t vdesc0 = sw128_desc(smem + Y::V_OFF);
    uint32_t vb = 0, vph = 0, bf = 0, pph = 0, oph = 1;  // o_free: nothing in it at first
    const bool leader = elect_one();
    bool ok = true;
    while (ok) {
      const int n = segment(walk).n;
      if (n == 0 || !warp_bar_wait(&o_free, oph, abort)) break;   // the last segment's O has been read
      oph ^= 1;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        ok = warp_bar_wait2(&v_full[vb], vph, &p_full[bf], pph, abort);
        if (!ok) break;
        tc_fence_after();
        if (leader) {
          const uint32_t tp = tmem + bf * kTok, to = tmem + kSBuf * kTok + (bf & 1) * D;
          const uint64_t vd = vdesc0 + vb * (Y::V_B >> 4);
          const uint32_t acc = j > 1;                    // (a stream's first tile clears its O)
#pragma unroll
          for (int kk = 0; kk < kTok / 16; ++kk)         // P (fp16 pairs) over S's columns
            mma_ts<S::PAIR>(to, tp + kk * 8, vd + kk * 2, id_pv, kk > 0 ? 1u : acc);
          mma_commit<S::PAIR>(&s_free[bf]);              // S/P buffer free, and O holds the tile
          mma_commit<S::PAIR>(&v_free[vb]);
        }
        __syncwarp();
        if (++vb == Y::VB) vb = 0, vph ^= 1;
        if (++bf == kSBuf) bf = 0, pph ^= 1;
      }
    }
    if (leader) mma_commit<S::PAIR>(&done_bar);
    if (lane == 0 && !mbar_wait(&done_bar, 0)) *abort = 1;
    __syncwarp();
  }
  } else if (warp >= 8) {
    regs_dec<kRegsBuild>();
    // ---------------- producers: keys, then values, of every third tile ----------------
    const int u = (warp - 8) >> 2, tid = threadIdx.x & 127;
    float* sz = reinterpret_cast<float*>(smem + Y::KS_OFF) + (warp - 8) * 64;
    int todo = u, kb = u, vb = u, st = u;                // (tiles of the segment before the group's next)
    uint32_t kph = 1, vph = 1, rph = 0;                  // buffers are free at first
    bool ok = true;
    while (ok) {
      const Segment s = segment(walk);
      if (s.n == 0) break;
      const int T = g.seq_len[s.b], tq = FMT == KVQ_FMT_KIVI ? kivi_tq(T, g.R, g.G) : T;
#pragma unroll 1
      for (; todo < s.n; todo += kGroups) {
        const int t0 = s.t0 + todo * kTok;
        const unsigned char* raw = smem + Y::RAW_OFF + st * Y::RAW_B;
        // K
        ok = __all_sync(0xffffffffu, bar_wait(&raw_k[st], rph, abort) && bar_wait(&k_free[kb], kph, abort));
        if (!ok) break;
        const int tt = (int)rank * S::KT + tid % S::KT;
        unsigned char* buf = smem + Y::K_OFF + kb * Y::K_B;
        if (FMT != KVQ_FMT_KIVI || t0 + (tt & ~31) < tq) keys_tile<D, BITS, FMT>(tid, raw, sz, buf);
        else keys_window<D, BITS>(g, s.b, s.head, t0 + tt, tid, buf);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // for the MMAs' reads
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&raw_k_free[st]);
          arrive_first<S::PAIR>(&k_full[kb]);
        }
        // V
        ok = __all_sync(0xffffffffu, bar_wait(&raw_v[st], rph, abort) && bar_wait(&v_free[vb], vph, abort));
        if (!ok) break;
        const int t = t0 + 2 * (tid >> 2);
        buf = smem + Y::V_OFF + vb * Y::V_B;
        if (FMT != KVQ_FMT_KIVI || t < tq) values_tile<D, BITS, FMT>(tid, (int)rank, raw, tq - t0, buf);
        else values_window<D, BITS>(g, s.b, s.head, t, T, tid, (int)rank, buf);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&raw_v_free[st]);
          arrive_first<S::PAIR>(&v_full[vb]);
        }
        if ((kb += kGroups) >= Y::KB) kb -= Y::KB, kph ^= 1;
        if ((vb += kGroups) >= Y::VB) vb -= Y::VB, vph ^= 1;
        if ((st += kGroups) >= Y::RAW) st -= Y::RAW, rph ^= 1;
      }
      todo -= s.n;
    }
  } else {
    regs_inc<kRegsSoftmax>();
    // ---------------- softmax: one row per thread of a stream ----------------
    const int x = warp >> 2;                             // stream
    const int r = threadIdx.x & 127;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + lane_base;
    const uint32_t o_col = tmem + lane_base + kSBuf * kTok;
    const float c2 = scale * 1.4426950408889634f;        // scores in log2 units
    const uint64_t c22 = f2pack(c2, c2);
    const int rr = (int)rank * kM + r;                   // row within the unit
    // half of the row's query into Q tile `buf`; returns the row's position (-1: no row)
    auto load_q = [&](const Segment& s, int buf) -> int {
      int pos = -1;
      unsigned char* qt = smem + Y::Q_OFF + buf * S::QT;
      const __nv_bfloat16* src = nullptr;
      if (rr < s.rows) {
        const int R = s.row0 + rr;
        int b = s.b, idx = R;
        if (s.e < n_nodes) {
          const int first = plan_nodes(plan)[s.e].first, count = plan_nodes(plan)[s.e].count;
          const int i = find_le(sc.roff, first, first + count, sc.roff[first] + R);
          b = plan_order(plan)[i];
          idx = R - (sc.roff[i] - sc.roff[first]);
        }
        const int l = idx / grp, hl = idx - l * grp;
        pos = g.seq_len[b] - new_rows(g, b, L, decode) + l;
        src = q + (((int64_t)b * g.Hq + s.head * grp + hl) * L + l) * D;
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const int c = x * (D / 16) + i;
        *reinterpret_cast<uint4*>(qt + (c >> 3) * (kM * 128) + sw128(r, c & 7)) =
            src ? *reinterpret_cast<const uint4*>(src + 8 * c) : make_uint4(0, 0, 0, 0);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_first<S::PAIR>(&q_full[buf]);
      return pos;
    };
    int it = 0, pos = -1;
    bool ok = true;
    Segment s;
    for (int seg = -1;; ++seg) {
      // the next segment's queries take the Q tile of the one before this, whose scores
      // are all formed
      const Segment nx = segment(walk);
      const int pos_nx = nx.n ? load_q(nx, (seg + 1) & 1) : -1;
      if (seg < 0) {                                     // (nothing to work through yet)
        if (nx.n == 0) break;
        s = nx;
        pos = pos_nx;
        continue;
      }
      float m = -INFINITY, l = 0.f;
      bool fresh = true;
      const int end = it + s.n;
      int last = -1;
#pragma unroll 1
      for (int i = it + ((it ^ x) & 1); i < end && ok; i += 2) {
        const int bf = i % kSBuf, t0 = s.t0 + (i - it) * kTok;
        // The second CTA of a pair waits for every phase of s_free (a parity tells a phase
        // only from its neighbours); the first CTA's issuer saw the skipped one end.
        if ((rank == 1 && i >= kSBuf && !warp_bar_wait(&s_free[bf], ((i - kSBuf) / kSBuf) & 1, abort)) ||
            !warp_bar_wait(&s_full[bf], (i / kSBuf) & 1, abort)) {
          ok = false;
          break;
        }
        tc_fence_after();
        uint32_t sr[kTok];
#pragma unroll
        for (int c = 0; c < kTok; c += 16) tmem_ld16_nowait(s_col + bf * kTok + c, sr + c);
        tmem_wait_ld();
        if (t0 + kTok - 1 > pos) {                       // a key of the tile is masked
#pragma unroll
          for (int k = 0; k < kTok; ++k)
            if (t0 + k > pos) sr[k] = __float_as_uint(-INFINITY);
        }
        float mx4[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const uint32_t* v = sr + 16 * a;
          float mv = fmax3(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]));
#pragma unroll
          for (int k = 3; k < 15; k += 2)
            mv = fmax3(mv, __uint_as_float(v[k]), __uint_as_float(v[k + 1]));
          mx4[a] = fmaxf(mv, __uint_as_float(v[15]));
        }
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        const float m_new = fmaxf(m, mx * c2);           // (c2 > 0: the maximum commutes)
        if (fresh) {
          m = m_new;
          fresh = false;
        } else if (__any_sync(0xffffffffu, m_new > m + kRescale)) {
          // O is rewritten: the stream's P V before must have completed
          if (!warp_bar_wait(&s_free[(i - 2) % kSBuf], ((i - 2) / kSBuf) & 1, abort)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const float alpha = m_new > m ? ex2_approx(m - m_new) : 1.f;
          if (m_new > m) {
            l *= alpha;
            m = m_new;
          }
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tmem_ld16_nowait(o_col + x * D + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
            tmem_st16(o_col + x * D + c, o);
          }
        }
        // P = 2^(s c2 - m) as fp16 pairs over the first 32 columns of this S buffer
        // (masked keys hold -inf: 2^-inf = 0; a row without a visible key so far subtracts 0)
        const float nm = m == -INFINITY ? 0.f : -m;
        const uint64_t negm = f2pack(nm, nm);
        uint64_t sum2 = f2pack(0.f, 0.f);
        uint32_t pk[kTok / 2];
#pragma unroll
        for (int k = 0; k < kTok; k += 2) {
          float a0, a1;
          f2unpack(ffma2(f2pack(__uint_as_float(sr[k]), __uint_as_float(sr[k + 1])), c22, negm), a0, a1);
          const float p0 = ex2_approx(a0), p1 = ex2_approx(a1);
          sum2 = fadd2(sum2, f2pack(p0, p1));
          pk[k / 2] = pack_h2(p0, p1);
        }
        tmem_st16(s_col + bf * kTok, pk);
        tmem_st16(s_col + bf * kTok + 16, pk + 16);
        float s0, s1;
        f2unpack(sum2, s0, s1);
        l += s0 + s1;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_first<S::PAIR>(&p_full[bf]);
        last = i;
      }
      it = end;
      // ---------------- the segment's partial: the streams' O joined ----------------
      if (ok && last >= 0 && !warp_bar_wait(&s_free[last % kSBuf], (last / kSBuf) & 1, abort)) ok = false;
      row_ml[x][r] = make_float2(m, l);
      softmax_sync();                                    // both streams' P V are complete
      ok = __all_sync(0xffffffffu, ok && !*abort);
      if (ok) {
        tc_fence_after();
        const float2 a = row_ml[0][r], b = row_ml[1][r];
        const float M = fmaxf(a.x, b.x);
        const float f0 = a.x == -INFINITY ? 0.f : ex2_approx(a.x - M);
        const float f1 = b.x == -INFINITY ? 0.f : ex2_approx(b.x - M);
        float* slot = slots + (size_t)s.slot * slot_floats(D);
        const bool one = s.n == 1;                       // the other stream's O holds nothing
        const int x_one = (end - 1) & 1;
#pragma unroll 1
        for (int c = x * (D / 2); c < (x + 1) * (D / 2); c += 16) {
          uint32_t o0[16], o1[16];
          tmem_ld16_nowait(o_col + c, o0);
          tmem_ld16_nowait(o_col + D + c, o1);
          tmem_wait_ld();
          float o[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const float v0 = one && x_one == 1 ? 0.f : __uint_as_float(o0[k]);
            const float v1 = one && x_one == 0 ? 0.f : __uint_as_float(o1[k]);
            o[k] = f0 * v0 + f1 * v1;
          }
          if (rr < s.rows) {
#pragma unroll
            for (int k = 0; k < 16; k += 4)
              *reinterpret_cast<float4*>(slot + (size_t)rr * D + c + k) =
                  make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          }
        }
        if (x == 0 && rr < s.rows)
          *reinterpret_cast<float2*>(slot + (size_t)RU * D + 2 * rr) = make_float2(M, f0 * a.y + f1 * b.y);
        tc_fence_before();                               // O has been read
      }
      __syncwarp();
      if (lane == 0) arrive_first<S::PAIR>(&o_free);
      softmax_sync();                                    // (m, l) may be written again
      if (nx.n == 0) break;
      s = nx;
      pos = pos_nx;
    }
  }
  // the issuer's last arrival on the second CTA's barriers has landed
  if (warp == 20 && lane == 0 && rank == 1 && !mbar_wait(&done_bar, 0)) *abort = 1;
  tc_fence_before();
  if (S::PAIR) cluster_sync();                         // neither CTA's TMEM or shared memory is in use
  else __syncthreads();
  if (threadIdx.x == 0 && *abort) atomicOr(err, 8);
  if (warp == 20) {
    tc_fence_after();
    tmem_free512<S::PAIR>(tmem);
  }
}

// =============================================================================
// leaves of a decode call: mma.sync, tokens (scores) and channels (values) as the MMA
// rows, up to 8 query heads as its columns.  The (sequence, kv head, 32-token block)
// space is cut into equal ranges, one for each warp: a warp copies its blocks' packed rows
// ahead of it into a ring of its own (bulk copies, an mbarrier a stage), and leaves a
// partial for each head that its range touches.  A KIVI sequence's full-precision tokens are
// read from their window directly.
//   scores  KIVI keys: A = codes in place, c 2^e 2^-24 as fp16 bits (a subnormal, exact),
//           B = q 2^-e s as fp16 high + low parts (an FMA gives the product's rounding
//           error), the sum times 2^24; the offsets sum_d q z by an MMA of their own.
//           Per-token groups: A = 128 + c in bf16, one accumulator a group, then
//           s (acc - 128 sum q) + z sum q.
//   values  A = v_hat = c s + z in fp16 (one rounding): codes biased by 1024 and carried
//           to the accumulator so would cost ten bits of it.
// =============================================================================
constexpr int kLeafWarps = 4, kLeafCtas = 4;           // warps of a CTA, CTAs of a SM
constexpr int kLeafBlocks = 2;                         // blocks a warp takes at least

// The leaves' work split, written into the workspace for merge_kernel: blocks of the
// sequences before (one head of up to 8 query heads each), and of all.
struct LeafSched {
  Ranges w;                               // blocks, over warps
  int32_t pre[KVQ_MAX_SEQS + 1];
};
constexpr size_t kLeafSchedBytes = (sizeof(LeafSched) + 255) / 256 * 256;
// Floats of a leaf partial: O [8 heads][D], then (m, l) [8].
__host__ __device__ inline size_t leaf_floats(int D) { return 8 * (size_t)(D + 2); }

template <int D, int BITS>
struct Leaf {
  static constexpr int NG = D / 32, CH = D / 8, MT = D / 16, KSS = D / 16;
  static constexpr int CROW = D * BITS / 8;            // code bytes of a token
  static constexpr int HW = CH * BITS / 16;            // 16-bit pieces of a thread's value channels
  // KIVI keys: a word holds CPW channels; register i is position i % RPW of word i / RPW, the
  // pair (channel p, p + CPW / 2) at bit BITS p, read in place PER positions to a shift
  static constexpr int CPW = 32 / BITS, RPW = CPW / 2, NWT = D * BITS / 128, NR = D / 8;
  static constexpr int PER = BITS == 2 ? 3 : 2;
  static constexpr uint32_t MASK = BITS == 2 ? 0x00030003u : 0x000F000Fu;
  __host__ __device__ static constexpr int e(int p) { return BITS * (p % PER); }
  __host__ __device__ static constexpr int lo(int i) { return (i / RPW) * CPW + i % RPW; }
  __host__ __device__ static constexpr int hi(int i) { return lo(i) + CPW / 2; }
  // a ring stage: one block's rows of every plane (KIVI keys: a row of D scales and offsets)
  static constexpr int KC = 0, VC = 32 * CROW, KM = 2 * VC, VM = 64 * NG;   // VM: bytes of V's scales
  template <int FMT>
  static constexpr int kmeta() { return FMT == KVQ_FMT_KIVI ? 2 * D : VM; }
  template <int FMT>
  static constexpr int bytes() { return 2 * VC + (FMT == KVQ_FMT_SYMMETRIC ? 1 : 2) * (kmeta<FMT>() + VM); }
  static constexpr int STAGE = (2 * VC + 4 * D + 2 * VM + 127) / 128 * 128;
  static constexpr int NS = 13 * 1024 / STAGE < 4 ? 13 * 1024 / STAGE : 4;
};
__device__ __forceinline__ uint32_t hsub2u(uint32_t a, uint32_t b) {
  __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t hfma2u(uint32_t a, uint32_t b, uint32_t c) {
  __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b),
                      *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<uint32_t*>(&r);
}
__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}
template <int W>                                       // W consecutive 32-bit words
__device__ __forceinline__ void ldg_words(const void* p, uint32_t (&w)[W]) {
  if constexpr (W == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  } else if constexpr (W == 2) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x; w[1] = u.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

template <int D, int BITS, int FMT>
__global__ void __launch_bounds__(kLeafWarps * 32, kLeafCtas)
leaf_kernel(Geom g, const __nv_bfloat16* __restrict__ q, float scale, LeafSched* __restrict__ sched,
            float* __restrict__ slots, int* err) {
  using Z = Leaf<D, BITS>;
  using dattn::bulk_g2s;
  using dattn::magic2;
  using dattn::magic2h;
  using dattn::mma16816;
  using dattn::mma16816_f16;
  using dattn::pack_f16;
  using dattn::pack_raw;
  using stream::hfma2u_neg;
  using stream::hmul2u;
  using stream::movmatrix_t;
  constexpr int NG = Z::NG, MT = Z::MT, KSS = Z::KSS, CH = Z::CH, NS = Z::NS;
  constexpr bool KIVI = FMT == KVQ_FMT_KIVI, SYM = FMT == KVQ_FMT_SYMMETRIC;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t full[kLeafWarps][NS];
  __shared__ int32_t pre[KVQ_MAX_SEQS + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tid = lane & 3;
  const int grp = g.Hq / g.H, halves = (grp + 7) / 8, heads = g.H * halves;
  unsigned char* ring = smem + warp * NS * Z::STAGE;
  if (lane == 0) {
    for (int i = 0; i < NS; ++i) mbar_init(&full[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // No wait here: the node kernel before waited for what the cache and this call's workspace
  // need before it let this one start, so the leaves fill the SMs as its CTAs end; it has
  // ended when this kernel has (below).
  pdl_trigger();
  const int32_t* leaf_page = plan_leaf_page(g.shared_plan, g.B);
  for (int i = threadIdx.x; i < g.B; i += kLeafWarps * 32)
    pre[i] = max(0, g.seq_len[i] - leaf_page[i] * kPageTok + 31) / 32 * heads;
  __syncthreads();
  if (warp == 0) warp_scan(pre, g.B);
  __syncthreads();
  const int N = pre[g.B], P = max(1, min((int)gridDim.x * kLeafWarps, N / kLeafBlocks));
  const Ranges ranges = make_ranges(N, P);
  if (blockIdx.x == 0) {                                 // for merge_kernel
    if (threadIdx.x == 0) sched->w = ranges;
    for (int i = threadIdx.x; i <= g.B; i += kLeafWarps * 32) sched->pre[i] = pre[i];
  }
  // a SM's CTAs take ranges far apart, so that few warps leave some SMs fewer of them
  const int wr = warp * (int)gridDim.x + blockIdx.x;
  if (wr >= P || N == 0) {
    pdl_wait();
    return;
  }
  const int x0 = ranges.start(wr), x1 = ranges.start(wr + 1);
  const float c2 = scale * 1.4426950408889634f;

  // a place in the flattened space: block blk of nb of sequence b's head uh
  struct Place {
    int b, uh, blk, nb;
  };
  auto blocks_of = [&](int b) { return (pre[b + 1] - pre[b]) / heads; };
  auto next = [&](Place& p) {
    if (++p.blk < p.nb) return;
    p.blk = 0;
    if (++p.uh < heads) return;
    p.uh = 0;
    do ++p.b; while (p.b < g.B && pre[p.b + 1] == pre[p.b]);
    p.nb = p.b < g.B ? blocks_of(p.b) : 0;
  };
  Place at;
  at.b = find_le(pre, 0, g.B, x0);
  at.nb = blocks_of(at.b);
  at.uh = (x0 - pre[at.b]) / at.nb;
  at.blk = (x0 - pre[at.b]) - at.uh * at.nb;
  // copies of a block's packed rows into its stage, lane c those of one plane (none for
  // full-precision tokens)
  constexpr int planes[6] = {KVQ_PLANE_K_CODES, KVQ_PLANE_V_CODES, KVQ_PLANE_K_SCALE,
                             KVQ_PLANE_V_SCALE, KVQ_PLANE_K_ZERO, KVQ_PLANE_V_ZERO};
  constexpr int km = Z::template kmeta<FMT>();
  constexpr int places[6] = {Z::KC, Z::VC, Z::KM, Z::KM + 2 * km, Z::KM + km, Z::KM + 2 * km + Z::VM};
  const int lc = min(lane, 5);
  const Plane& lpl = g.pl[planes[lc]];
  const char* lplane = static_cast<const char*>(lpl.p);
  const int64_t lrow = lpl.cols * lpl.elem, lhead = lpl.rows * lrow;
  const int lplace = places[lc];
  const uint32_t lbytes = lc < 2 ? Z::VC : (lc & 1) ? Z::VM : km;
  const int lshift = KIVI && (lc == 2 || lc == 4) ? 5 : 0;   // a row a block, or a token
  auto issue = [&](const Place& p, int st) {
    const int T = g.seq_len[p.b], t0 = leaf_page[p.b] * kPageTok + 32 * p.blk, hkv = p.uh / halves;
    uint64_t* bar = &full[warp][st];
    if (KIVI && t0 >= kivi_tq(T, g.R, 32)) {
      // full-precision rows are read from the window itself: only drawn into the L2 here,
      // lanes 0 and 1 those to the window's end, 2 and 3 those that wrap to its start
      if (lane == 0) mbar_arrive(bar);
      const int at = t0 % g.ring, n = min(32, g.ring - at), rows = lane < 2 ? n : 32 - n;
      if (lane < 4 && rows > 0)
        prefetch_l2(plane_ptr<__nv_bfloat16>(g, (lane & 1) ? KVQ_PLANE_V_FULL : KVQ_PLANE_K_FULL, p.b, hkv,
                                             lane < 2 ? at : 0, 0), rows * D * 2);
      return;
    }
    const int64_t row = (int64_t)g.page_table[(size_t)p.b * g.max_pages + (t0 >> kPageShift)] * kPageTok +
                        (t0 & (kPageTok - 1));           // a block lies in one page
    if (lane == 0) mbar_expect_tx(bar, Z::template bytes<FMT>());
    __syncwarp();
    if (lane < (SYM ? 4 : 6))
      bulk_g2s(ring + st * Z::STAGE + lplace, lplane + hkv * lhead + (row >> lshift) * lrow, lbytes, bar);
  };
  Place ahead = at;
  int issued = 0;
  for (; issued < NS && x0 + issued < x1; ++issued) {
    issue(ahead, issued);
    next(ahead);
  }

  uint32_t qw[KIVI ? Z::NR : 1];                       // KIVI: q 2^-e, fp16 pairs
  uint32_t qb[KIVI ? 1 : KSS][2];                      // else bf16 B fragments, per-group sums
  float qs[KIVI ? 1 : NG][2];
  float m_run[2], l_run[2], o[MT][4];
  bool ok = true;
  int T = 0, ts = 0, tq = 0, b = 0, hkv = 0, nh = 0;
  const __nv_bfloat16* qh = nullptr;

  for (int x = x0; x < x1 && ok; ++x) {
    const int k = at.blk, slot = (at.b * heads + at.uh) + wr;
    if (x == x0 || k == 0) {
      // ---- a head starts: its tokens and queries ----
      b = at.b;
      hkv = at.uh / halves;
      const int h0 = 8 * (at.uh - hkv * halves);
      nh = min(8, grp - h0);
      T = g.seq_len[b];
      ts = leaf_page[b] * kPageTok;
      tq = KIVI ? kivi_tq(T, g.R, 32) : T;
      qh = q + ((int64_t)b * g.Hq + hkv * grp + h0) * D;
      if constexpr (KIVI) {
        const __nv_bfloat16* qr = qh + gid * D + tid * (D / 4);
        uint32_t u[Z::NR];                               // D / 4 bf16
#pragma unroll
        for (int i = 0; i < Z::NR; i += 4) {
          const uint4 v = gid < nh ? *reinterpret_cast<const uint4*>(qr + 2 * i) : make_uint4(0, 0, 0, 0);
          u[i] = v.x; u[i + 1] = v.y; u[i + 2] = v.z; u[i + 3] = v.w;
        }
        const auto el = [&](int c) { return __uint_as_float((c & 1) ? u[c >> 1] & 0xFFFF0000u : u[c >> 1] << 16); };
#pragma unroll
        for (int i = 0; i < Z::NR; ++i) {
          const float w = 1.f / (float)(1 << Z::e(i % Z::RPW));
          qw[i] = pack_f16(el(Z::lo(i)) * w, el(Z::hi(i)) * w);
        }
      } else {
#pragma unroll
        for (int gq = 0; gq < NG; ++gq) {
          uint4 u = make_uint4(0, 0, 0, 0);
          if (gid < nh) u = *reinterpret_cast<const uint4*>(qh + gid * D + 32 * gq + 8 * tid);
          const uint16_t* e = reinterpret_cast<const uint16_t*>(&u);
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) s += __uint_as_float((uint32_t)e[i] << 16);
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            qb[2 * gq + sub][0] = pack_raw(e[dattn::qk_chan<BITS>(sub, 0, 0)], e[dattn::qk_chan<BITS>(sub, 0, 1)]);
            qb[2 * gq + sub][1] = pack_raw(e[dattn::qk_chan<BITS>(sub, 1, 0)], e[dattn::qk_chan<BITS>(sub, 1, 1)]);
          }
          s += __shfl_xor_sync(0xffffffffu, s, 1);
          s += __shfl_xor_sync(0xffffffffu, s, 2);       // head gid, group gq
          qs[gq][0] = __shfl_sync(0xffffffffu, s, 4 * (2 * tid));
          qs[gq][1] = __shfl_sync(0xffffffffu, s, 4 * (2 * tid + 1));
        }
      }
      m_run[0] = m_run[1] = -INFINITY;
      l_run[0] = l_run[1] = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    }
    const int st = (x - x0) % NS;
    ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][st], ((x - x0) / NS) & 1));
    if (!ok) {
      if (lane == 0) atomicOr(err, 1);
      break;
    }
    const unsigned char* sp = ring + st * Z::STAGE;
    const unsigned char* kmp = sp + Z::KM;
    const int t0 = ts + 32 * k, nv = min(32, T - t0);
    const bool coded = !KIVI || t0 < tq;
    // the window's slot of the block's i-th token
    const int slot0 = KIVI && !coded ? t0 % g.ring : 0;
    const auto slot_of = [&](int i) { return slot0 + i < g.ring ? slot0 + i : slot0 + i - g.ring; };
    // ---- scores: S[mt][i], tokens 16 mt + gid (i < 2) and + 8, heads 2 tid + i % 2 ----
    float S[2][4];
    if (KIVI && coded) {
      if constexpr (KIVI) {
        const unsigned char* kc = sp + Z::KC + tid * (4 * Z::NWT);
        uint32_t cw[2][2][Z::NWT];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int r = 0; r < 2; ++r) ldg_words(kc + (16 * mt + gid + 8 * r) * Z::CROW, cw[mt][r]);
        uint32_t sw[D / 8], zw[D / 8];
#pragma unroll
        for (int i = 0; i < D / 8; i += 4) {
          const uint4 u = *reinterpret_cast<const uint4*>(kmp + tid * (D / 2) + 4 * i);
          const uint4 v = *reinterpret_cast<const uint4*>(kmp + km + tid * (D / 2) + 4 * i);
          sw[i] = u.x; sw[i + 1] = u.y; sw[i + 2] = u.z; sw[i + 3] = u.w;
          zw[i] = v.x; zw[i + 1] = v.y; zw[i + 2] = v.z; zw[i + 3] = v.w;
        }
        float sz[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) S[mt][0] = S[mt][1] = S[mt][2] = S[mt][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KSS; ++ks) {
          uint32_t bh[2], bl[2], az[2], bz[2];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int i = 2 * ks + hf;
            const int sel = (Z::lo(i) & 1) ? 0x7632 : 0x5410;
            const uint32_t as = __byte_perm(sw[Z::lo(i) >> 1], sw[Z::hi(i) >> 1], sel);
            const uint32_t w2 = ((uint32_t)(15 + Z::e(i % Z::RPW)) << 10) * 0x00010001u;   // (2^e, 2^e)
            // (q taken back up by 2^e, exactly, and not z, which would overflow from 2^12 on)
            az[hf] = __byte_perm(zw[Z::lo(i) >> 1], zw[Z::hi(i) >> 1], sel);
            bz[hf] = hmul2u(qw[i], w2);
            bh[hf] = hmul2u(qw[i], as);
            bl[hf] = hfma2u_neg(qw[i], as, bh[hf]);
          }
          const uint32_t aZ[4] = {az[0], az[0], az[1], az[1]};
          mma16816_f16(sz, aZ, bz[0], bz[1]);
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            uint32_t a[4];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const int i = 2 * ks + hf, p = i % Z::RPW;
                const uint32_t w = cw[mt][r][i / Z::RPW] >> (BITS * Z::PER * (p / Z::PER));
                a[2 * hf + r] = w & (Z::MASK << Z::e(p));
              }
            mma16816_f16(S[mt], a, bh[0], bh[1]);
            mma16816_f16(S[mt], a, bl[0], bl[1]);
          }
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int i = 0; i < 4; ++i) S[mt][i] = fmaf(S[mt][i], 16777216.f, sz[i & 1]);
      }
    } else if (coded) {
      if constexpr (!KIVI) {
        constexpr uint32_t kmask = BITS == 4 ? 0x000F000Fu : 0x00030003u;
        const unsigned char* kc = sp + Z::KC;
        const __half* ksp = reinterpret_cast<const __half*>(kmp);
        const __half* kzp = reinterpret_cast<const __half*>(kmp + km);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          const unsigned char* r0 = kc + (16 * mt + gid) * Z::CROW;
          const unsigned char* r1 = r0 + 8 * Z::CROW;
          float acc[NG][4];
#pragma unroll
          for (int gq = 0; gq < NG; ++gq) {
            acc[gq][0] = acc[gq][1] = acc[gq][2] = acc[gq][3] = 0.f;
            uint32_t w0, w1;
            if (BITS == 4) {
              w0 = *reinterpret_cast<const uint32_t*>(r0 + 16 * gq + 4 * tid);
              w1 = *reinterpret_cast<const uint32_t*>(r1 + 16 * gq + 4 * tid);
            } else {
              const uint32_t v0 = *reinterpret_cast<const uint16_t*>(r0 + 8 * gq + 2 * tid);
              const uint32_t v1 = *reinterpret_cast<const uint16_t*>(r1 + 8 * gq + 2 * tid);
              w0 = v0 | (v0 << 14);
              w1 = v1 | (v1 << 14);
            }
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
              const uint32_t a[4] = {magic2(w0 >> (8 * sub), kmask), magic2(w1 >> (8 * sub), kmask),
                                     magic2(w0 >> (8 * sub + 4), kmask), magic2(w1 >> (8 * sub + 4), kmask)};
              mma16816(acc[gq], a, qb[2 * gq + sub][0], qb[2 * gq + sub][1]);
            }
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int t = 16 * mt + gid + 8 * r;
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int gq = 0; gq < NG; gq += 2) {
              const float2 sg = __half22float2(*reinterpret_cast<const __half2*>(ksp + t * NG + gq));
              float2 zg;
              if (SYM) zg = make_float2(-(float)(1 << (BITS - 1)) * sg.x, -(float)(1 << (BITS - 1)) * sg.y);
              else zg = __half22float2(*reinterpret_cast<const __half2*>(kzp + t * NG + gq));
              s0 += sg.x * (acc[gq][2 * r] - 128.f * qs[gq][0]) + zg.x * qs[gq][0];
              s1 += sg.x * (acc[gq][2 * r + 1] - 128.f * qs[gq][1]) + zg.x * qs[gq][1];
              s0 += sg.y * (acc[gq + 1][2 * r] - 128.f * qs[gq + 1][0]) + zg.y * qs[gq + 1][0];
              s1 += sg.y * (acc[gq + 1][2 * r + 1] - 128.f * qs[gq + 1][1]) + zg.y * qs[gq + 1][1];
            }
            S[mt][2 * r] = s0;
            S[mt][2 * r + 1] = s1;
          }
        }
      }
    } else {
      // full-precision keys: k-step ks takes channels D/4 tid + 4 ks .. + 3 of a row
      const __nv_bfloat16* qr = qh + gid * D + tid * (D / 4);
      const __nv_bfloat16* kw = plane_ptr<__nv_bfloat16>(g, KVQ_PLANE_K_FULL, b, hkv, 0, tid * (D / 4));
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        S[mt][0] = S[mt][1] = S[mt][2] = S[mt][3] = 0.f;
        const int ta = t0 + 16 * mt + gid, tb = ta + 8;
        const __nv_bfloat16 *ka = kw + (int64_t)slot_of(16 * mt + gid) * D,
                            *kb = kw + (int64_t)slot_of(16 * mt + gid + 8) * D;
        const uint4 z = make_uint4(0, 0, 0, 0);
        uint4 va[D / 32], vb[D / 32];                  // all under way before the first is used
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          va[c] = ta < T ? reinterpret_cast<const uint4*>(ka)[c] : z;
          vb[c] = tb < T ? reinterpret_cast<const uint4*>(kb)[c] : z;
        }
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {             // 8 channels: two k-steps
          const uint4 ua = va[c], ub = vb[c];
          const uint4 uq = gid < nh ? reinterpret_cast<const uint4*>(qr)[c] : z;
          const uint32_t a0[4] = {ua.x, ub.x, ua.y, ub.y}, a1[4] = {ua.z, ub.z, ua.w, ub.w};
          mma16816(S[mt], a0, uq.x, uq.y);
          mma16816(S[mt], a1, uq.z, uq.w);
        }
      }
    }
    // ---- softmax over the block's tokens ----
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        S[mt][i] = 16 * mt + gid + 8 * (i >> 1) < nv ? S[mt][i] * c2 : -INFINITY;
        mx[i & 1] = fmaxf(mx[i & 1], S[mt][i]);
      }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 4));
      mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 8));
      mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 16));
      mx[j] = fmaxf(m_run[j], mx[j]);                  // (-inf: no score above it so far)
    }
    if (__any_sync(0xffffffffu, mx[0] != m_run[0] || mx[1] != m_run[1])) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float alpha = m_run[j] == -INFINITY ? 0.f : ex2_approx(m_run[j] - mx[j]);
        m_run[j] = mx[j];
        l_run[j] *= alpha;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          o[i][j] *= alpha;
          o[i][2 + j] *= alpha;
        }
      }
    }
    // (a head whose scores are all -inf so far, of infinite keys or overflowing products, subtracts 0)
    const float base[2] = {m_run[0] == -INFINITY ? 0.f : m_run[0], m_run[1] == -INFINITY ? 0.f : m_run[1]};
    uint32_t pb[2][2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = ex2_approx(S[mt][i] - base[i & 1]);
        l_run[i & 1] += p[i];
      }
      pb[mt][0] = movmatrix_t(pack_f16(p[0], p[1]));
      pb[mt][1] = movmatrix_t(pack_f16(p[2], p[3]));
    }
    // ---- values: m-tile u holds channels CH gid + 2 u (rows gid) and + 1 (rows gid + 8) ----
    if (coded) {
      uint32_t vx[2][2][Z::HW];                        // [mt][tokens 2 tid | +1, or + 8], pieces paired
      uint32_t vs[2][2], vz[2][2];
      const unsigned char* vc = sp + Z::VC + gid * (CH * BITS / 8);
      const uint16_t* vsp = reinterpret_cast<const uint16_t*>(kmp + 2 * km) + gid * CH / 32;
      const uint16_t* vzp = vsp + Z::VM / 2;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int ta = 16 * mt + 8 * hf + 2 * tid;
          // rows behind the last token may hold anything: their scales and offsets count as 0
          const uint32_t sa = ta < nv ? vsp[ta * NG] : 0u, sb = ta + 1 < nv ? vsp[(ta + 1) * NG] : 0u;
          vs[mt][hf] = sa | (sb << 16);
          if constexpr (!SYM) {
            const uint32_t za = ta < nv ? vzp[ta * NG] : 0u, zb = ta + 1 < nv ? vzp[(ta + 1) * NG] : 0u;
            vz[mt][hf] = za | (zb << 16);
          }
          const unsigned char* pa = vc + ta * Z::CROW;
          const unsigned char* pc = pa + Z::CROW;
          if constexpr (Z::HW == 1) {
            vx[mt][hf][0] = (uint32_t)*reinterpret_cast<const uint16_t*>(pa) |
                            ((uint32_t)*reinterpret_cast<const uint16_t*>(pc) << 16);
          } else {
            uint32_t wa[Z::HW / 2], wb[Z::HW / 2];
            ldg_words(pa, wa);
            ldg_words(pc, wb);
#pragma unroll
            for (int i = 0; i < Z::HW / 2; ++i) {
              vx[mt][hf][2 * i] = __byte_perm(wa[i], wb[i], 0x5410);
              vx[mt][hf][2 * i + 1] = __byte_perm(wa[i], wb[i], 0x7632);
            }
          }
        }
      constexpr int PP = 16 / BITS;                    // channels of a 16-bit piece
      constexpr uint32_t vmask = BITS == 4 ? 0x000F000Fu : 0x00030003u;
      // 1024 (and a symmetric code's zero) off, exactly
      constexpr uint32_t off = (0x6400u + (SYM ? (1u << (BITS - 1)) : 0u)) * 0x00010001u;
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int u = 0; u < MT; ++u) {
          uint32_t a[4];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int c = 2 * u + r;
              const uint32_t code = hsub2u(magic2h(vx[mt][hf][c / PP] >> (BITS * (c % PP)), vmask), off);
              a[2 * hf + r] = SYM ? hmul2u(code, vs[mt][hf]) : hfma2u(code, vs[mt][hf], vz[mt][hf]);
            }
          mma16816_f16(o[u], a, pb[mt][0], pb[mt][1]);
        }
    } else {
      const __nv_bfloat16* vw = plane_ptr<__nv_bfloat16>(g, KVQ_PLANE_V_FULL, b, hkv, 0, CH * gid);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        uint4 wv[CH / 8][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 16 * mt + 8 * (i >> 1) + 2 * tid + (i & 1);
          const __nv_bfloat16* vr = vw + (int64_t)slot_of(j) * D;
#pragma unroll
          for (int c = 0; c < CH / 8; ++c)
            wv[c][i] = j < nv ? reinterpret_cast<const uint4*>(vr)[c] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int c = 0; c < CH / 8; ++c) {             // 8 channels of the thread's: 4 m-tiles
          const uint4* w = wv[c];
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t* w0 = reinterpret_cast<const uint32_t*>(&w[0]);
            const uint32_t* w1 = reinterpret_cast<const uint32_t*>(&w[1]);
            const uint32_t* w2 = reinterpret_cast<const uint32_t*>(&w[2]);
            const uint32_t* w3 = reinterpret_cast<const uint32_t*>(&w[3]);
            auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
            auto hi = [](uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); };
            const uint32_t a[4] = {pack_f16(lo(w0[v]), lo(w1[v])), pack_f16(hi(w0[v]), hi(w1[v])),
                                   pack_f16(lo(w2[v]), lo(w3[v])), pack_f16(hi(w2[v]), hi(w3[v]))};
            mma16816_f16(o[4 * c + v], a, pb[mt][0], pb[mt][1]);
          }
        }
      }
    }
    // ---- the stage is read: the block NS ahead takes it ----
    __syncwarp();
    if (x0 + issued < x1) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      issue(ahead, st);
      next(ahead);
      ++issued;
    }
    next(at);
    if (at.blk == 0 || x + 1 == x1) {
      // ---- the head, or the warp's share of it, is through ----
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        l_run[j] += __shfl_xor_sync(0xffffffffu, l_run[j], 4);
        l_run[j] += __shfl_xor_sync(0xffffffffu, l_run[j], 8);
        l_run[j] += __shfl_xor_sync(0xffffffffu, l_run[j], 16);
      }
      float* part = slots + (size_t)slot * leaf_floats(D);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int h = 2 * tid + j;
        if (h < nh) {
#pragma unroll
          for (int u = 0; u < MT; ++u)
            *reinterpret_cast<float2*>(part + h * D + CH * gid + 2 * u) = make_float2(o[u][j], o[u][2 + j]);
          if (gid == 0) *reinterpret_cast<float2*>(part + 8 * D + 2 * h) = make_float2(m_run[j], l_run[j]);
        }
      }
    }
  }
  // no copy may still be landing when the CTA exits (after a timeout)
  if (!ok && lane == 0)
    for (int i = max(0, issued - NS); i < issued; ++i) mbar_wait(&full[warp][i % NS], (i / NS) & 1);
  pdl_wait();
}

// =============================================================================
// merge: a warp per query row, or a CTA where the rows are few: a long leaf of few sequences
// has hundreds of partials a row (2 sequences of 30,000 own tokens, 32 / 4 heads of 64: 72 us
// with a warp a row, 32 with a CTA).  A warp takes 4 us to find its row's partials whatever
// their number, so many rows want few warps: 512 rows 44.2 and 40.9 us, 592 rows 42.1 and
// 40.8, 1024 rows 30.2 and 32.3, 2048 rows 100.8 and 109.8 (whole calls).
// =============================================================================
constexpr int kMergeWarps = 8;
constexpr int kMergeRowsPerSm = 4;        // up to so many rows (608) a CTA takes one

template <int D, int W>                                // W warps to a row
__global__ void __launch_bounds__(kMergeWarps * 32)
merge_kernel(const __grid_constant__ Geom g, int L, int decode, const SchedOut* __restrict__ sc,
             const float* __restrict__ slots, const LeafSched* __restrict__ ls,
             const float* __restrict__ leaf, __nv_bfloat16* __restrict__ out) {
  pdl_trigger();
  constexpr int V = D / 32;                              // channels a lane
  const int RU = unit_rows_of(D), lane = threadIdx.x & 31;
  const int warp = threadIdx.x >> 5, sub = warp % W, row = blockIdx.x * (kMergeWarps / W) + warp / W;
  const int l = row % L, h = row / L % g.Hq, b = row / L / g.Hq;
  const bool mine = b < g.B && l < new_rows(g, min(b, g.B - 1), L, decode);
  const int grp = g.Hq / g.H, hkv = h / grp, hl = h - hkv * grp, idx = l * grp + hl;
  const int32_t* plan = g.shared_plan;
  const int n_nodes = plan[0], parent = mine ? plan_leaf_parent(plan, g.B)[b] : 0;
  pdl_wait();
  if (!mine || !sc->ok) return;

  float M = -INFINITY, sum = 0.f, acc[V];
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.f;
  const Ranges w = sc->w;
  const int roff = n_nodes ? sc->roff[sc->inv[b]] : 0;
  // the row's partials, one a lane at a time and the warps in turn: those of the nodes on
  // its path, then its leaf's
  for (int base = 0, total = W; base * W < total; base += 32) {
    total = 0;
    const float *o = nullptr, *mlp = nullptr;
    const auto parts = [&](int n, const float* first, size_t stride, int at_o, int at_ml) {
      const int i = (base + lane) * W + sub - total;
      if (i >= 0 && i < n) {
        o = first + i * stride + at_o;
        mlp = first + i * stride + at_ml;
      }
      total += n;
    };
    const auto entry = [&](int e, int R) {
      const int up = sc->up[e], tp = sc->tp[e], units = sc->up[e + 1] - up, tiles = sc->tp[e + 1] - tp;
      if (tiles == 0) return;
      const int len = tiles / units, u = hkv * (units / g.H) + R / RU, rr = R % RU;
      const int g0 = tp + u * len, c0 = w.of(g0 + unit_cost(g.fmt, e >= n_nodes)), c1 = w.of(g0 + len - 1);
      parts(c1 - c0 + 1, slots + (size_t)(up + u + c0) * slot_floats(D), slot_floats(D), rr * D, RU * D + 2 * rr);
    };
    for (int p = parent; p;) {
      const SharedNode nd = plan_nodes(plan)[p - 1];
      entry(p - 1, roff - sc->roff[nd.first] + idx);
      p = nd.parent;
    }
    if (!decode) {
      entry(n_nodes + b, idx);
    } else {
      const int halves = (grp + 7) / 8, heads = g.H * halves, uh = hkv * halves + hl / 8;
      const int pre = ls->pre[b], nb = (ls->pre[b + 1] - pre) / heads;
      if (nb > 0) {
        const Ranges lw = ls->w;
        const int g0 = pre + uh * nb, w0 = lw.of(g0), w1 = lw.of(g0 + nb - 1);
        parts(w1 - w0 + 1, leaf + (size_t)(b * heads + uh + w0) * leaf_floats(D), leaf_floats(D), (hl & 7) * D,
              8 * D + 2 * (hl & 7));
      }
    }
    float2 ml = mlp ? *reinterpret_cast<const float2*>(mlp) : make_float2(-INFINITY, 0.f);
    if (ml.y != ml.y) ml.x = INFINITY;                   // a NaN score (maxima skip it): the row is NaN
    float mb = ml.x;
#pragma unroll
    for (int k = 16; k; k >>= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, k));
    mb = fmaxf(mb, M);
    if (mb == -INFINITY) continue;                       // nothing visible so far
    const float r = M == -INFINITY ? 0.f : exp2f(M - mb);
    const float wt = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mb);
    float lsum = wt * ml.y;
#pragma unroll
    for (int k = 16; k; k >>= 1) lsum += __shfl_xor_sync(0xffffffffu, lsum, k);
    sum = sum * r + lsum;
    M = mb;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] *= r;
    const int n = min(32, (total - sub + W - 1) / W - base);
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const float wi = __shfl_sync(0xffffffffu, wt, i);
      const float* oi = reinterpret_cast<const float*>(
          __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(o), i));
      if (wi != 0.f) {                                   // (an empty piece's values are not read)
        float x[V];
        if constexpr (V == 4) *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(oi + V * lane);
        else *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(oi + V * lane);
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] = fmaf(wi, x[v], acc[v]);
      }
    }
  }
  if constexpr (W > 1) {                                 // the warps' shares joined by the first
    __shared__ float2 wml[kMergeWarps];
    __shared__ __align__(16) float wo[kMergeWarps][D];
    if (lane == 0) wml[warp] = make_float2(M, sum);
#pragma unroll
    for (int v = 0; v < V; ++v) wo[warp][V * lane + v] = acc[v];
    __syncthreads();
    if (sub) return;
    float m = M;
#pragma unroll
    for (int k = 1; k < W; ++k) m = fmaxf(m, wml[warp + k].x);
    const float f = M == -INFINITY ? 0.f : exp2f(M - m);
    sum *= f;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] *= f;
#pragma unroll
    for (int k = 1; k < W; ++k) {
      const float2 ml = wml[warp + k];
      const float fk = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m);
      sum = fmaf(fk, ml.y, sum);
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] = fmaf(fk, wo[warp + k][V * lane + v], acc[v]);
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;        // (no visible key: 0)
  uint32_t pk[V / 2];
#pragma unroll
  for (int v = 0; v < V; v += 2) pk[v / 2] = pack_bf16(acc[v] * inv, acc[v + 1] * inv);
  __nv_bfloat16* dst = out + (size_t)row * D + V * lane;
  if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pk[0], pk[1]);
  else *reinterpret_cast<uint32_t*>(dst) = pk[0];
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
struct Call {
  const __nv_bfloat16* q;
  int L, decode, cap;
  float scale;
  __nv_bfloat16* out;
  SchedOut* sched;
  LeafSched* leaf_sched;
  float *leaf, *slots;                    // partials: of a decode's leaves; of shared_tc_kernel
  int* err;
};

// A kernel's shared memory is asked for once a device, and the registers that its warpgroups
// share out are looked up (regs > 0).
template <typename K>
cudaError_t prepare_kernel(K kern, int smem, int regs, std::atomic<uint64_t>& done) {
  int dev;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load() >> dev & 1))) return e;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess && regs) {
    cudaFuncAttributes a;
    e = cudaFuncGetAttributes(&a, kern);
    if (e == cudaSuccess && a.numRegs < regs) e = cudaErrorLaunchOutOfResources;
  }
  if (e == cudaSuccess && dev < 64) done |= 1ull << dev;
  return e;
}

template <int D, int BITS, int FMT>
cudaError_t launch_shared_t(const Geom& g, const Call& c, cudaStream_t s) {
  auto kern = shared_tc_kernel<D, BITS, FMT>;
  constexpr int NC = M256Layout<D, BITS>::PAIR ? 2 : 1;
  const size_t sm = TcLayout<D, BITS>::ALLOC;
  static std::atomic<uint64_t> tc_done{0}, leaf_done{0};
  cudaError_t e = prepare_kernel(kern, (int)sm, kRegs, tc_done);
  if (e != cudaSuccess) return e;
  const dim3 grid(num_sms() / NC * NC);
  if (NC == 2)
    launch_pdl_pair(kern, grid, dim3(kTcThreads), sm, s, g, c.q, c.L, c.decode, c.scale, c.sched, c.slots, c.cap, c.err);
  else
    launch_pdl(kern, grid, dim3(kTcThreads), sm, s, g, c.q, c.L, c.decode, c.scale, c.sched, c.slots, c.cap, c.err);
  if (c.decode) {
    const size_t lm = (size_t)kLeafWarps * Leaf<D, BITS>::NS * Leaf<D, BITS>::STAGE;
    auto leaf = leaf_kernel<D, BITS, FMT>;
    e = prepare_kernel(leaf, (int)lm, 0, leaf_done);
    if (e != cudaSuccess) return e;
    launch_pdl(leaf, dim3(num_sms() * kLeafCtas), dim3(kLeafWarps * 32), lm, s, g, c.q, c.scale, c.leaf_sched, c.leaf, c.err);
  }
  const int64_t rows = (int64_t)g.B * g.Hq * c.L;
  const auto merge = [&](auto kern_, int W) {
    const int per = kMergeWarps / W;
    launch_pdl(kern_, dim3((unsigned)((rows + per - 1) / per)), dim3(kMergeWarps * 32), 0, s, g, c.L, c.decode, c.sched,
               c.slots, c.leaf_sched, c.leaf, c.out);
  };
  if (rows <= (int64_t)kMergeRowsPerSm * num_sms()) merge(merge_kernel<D, kMergeWarps>, kMergeWarps);
  else merge(merge_kernel<D, 1>, 1);
  return cudaGetLastError();
}

template <int D, int BITS>
cudaError_t launch_shared_f(const Geom& g, const Call& c, cudaStream_t s) {
  return g.fmt == KVQ_FMT_KIVI        ? launch_shared_t<D, BITS, KVQ_FMT_KIVI>(g, c, s)
         : g.fmt == KVQ_FMT_SYMMETRIC ? launch_shared_t<D, BITS, KVQ_FMT_SYMMETRIC>(g, c, s)
                                      : launch_shared_t<D, BITS, KVQ_FMT_AFFINE>(g, c, s);
}

cudaError_t launch_shared(const Geom& g, const Call& c, cudaStream_t s) {
  if (g.D == 64) return g.kb == 4 ? launch_shared_f<64, 4>(g, c, s) : launch_shared_f<64, 2>(g, c, s);
  return g.kb == 4 ? launch_shared_f<128, 4>(g, c, s) : launch_shared_f<128, 2>(g, c, s);
}

// Whether a prefill is faster sequence by sequence (attend_prefill_m256.cu: 512 rows a pair of
// CTAs, or 256 a CTA, share a tile, the keys behind them are skipped, and a unit's keys are not
// split) than here (half the rows, every tile of a leaf, any split of the keys): long prompts
// fill its tiles without other sequences' rows.  Both times are estimated from what a 64-token
// tile took, in ns, and here from 1 ns a query row to merge; on 60 shapes (1 to 16 sequences,
// 16 to 2048 rows behind 512 to 16384 tokens) the estimate is mostly within 20 % and took the
// slower side 4 times, by 3 % at most (of 2 and 4 bits, which it takes alike; since then the
// kernel there got 3 % faster).  2 x 256 rows behind 4096 tokens, 32 / 8 heads of 128, KIVI:
// 103 us there, 82 here; 2 x 1024: 222 and 313; 8 x 2048 behind 512, affine: 555 and 1850;
// 4 x 64 behind 17,384: 396 and 121.
bool alone_faster(const kvq_cache* c) {
  const Geom& g = c->g;
  if (!prefill_m256_supported(g)) return false;
  const bool kivi = g.fmt == KVQ_FMT_KIVI, pair = g.D == 128;
  const double tile_alone = pair ? (kivi ? 1570 : 1270) : (kivi ? 1450 : 1190);
  const double tile_here = pair && !kivi ? 1150 : 850;
  const int grp = g.Hq / g.H, P = num_sms() / (pair ? 2 : 1), RU = unit_rows_of(g.D);
  const int nq = 256 / grp * (pair ? 2 : 1);             // its queries a unit
  const auto units = [&](int64_t rows) { return (rows + RU - 1) / RU; };
  double total = 0, longest = 0, places = 0, merge = 0;
  int64_t n_units = 0;
  const int32_t* plan = c->plan.empty() ? nullptr : c->plan.data();
  for (int b = 0; b < g.B; ++b) {
    const int n = c->seq_n[b], T = c->seq_T[b];
    if (n <= 0) continue;
    const int64_t u = (n + nq - 1) / nq;
    total += (double)u * g.H * ((T - n + std::min<double>(n, 0.5 * (n + nq))) / kTok + 5);
    longest = std::max(longest, (double)T / kTok + 5);   // (5: a unit's start and end)
    n_units += u * g.H;
    const int leaf = plan ? T - plan_leaf_page(plan, g.B)[b] * kPageTok : T;
    if (leaf > 0) places += (double)units((int64_t)n * grp) * g.H * ((leaf + kTok - 1) / kTok + unit_cost(g.fmt, true));
    merge += (double)n * g.Hq;
  }
  if (plan)
    for (int i = 0; i < plan[0]; ++i) {
      const SharedNode& nd = plan_nodes(plan)[i];
      int64_t rows = 0;
      for (int k = 0; k < nd.count; ++k) rows += (int64_t)c->seq_n[plan_order(plan)[nd.first + k]] * grp;
      places += (double)units(rows) * g.H * ((nd.p1 - nd.p0) * (kPageTok / kTok) + unit_cost(g.fmt, false));
    }
  const double alone = tile_alone * (n_units <= P ? longest : total / P + longest / 2);
  return alone < tile_here * places / P + merge + 8000;
}

// Slots that a call with L rows a sequence needs at the cache's present plan.
int64_t shared_slots(const kvq_cache* c, int L) {
  const Geom& g = c->g;
  const int64_t RU = unit_rows_of(g.D), grp = g.Hq / g.H;
  int64_t units = 0;
  if (!c->plan.empty()) {
    const SharedNode* nd = plan_nodes(c->plan.data());
    for (int i = 0; i < c->plan[0]; ++i) units += (nd[i].count * grp * L + RU - 1) / RU;
  }
  units += g.B * ((grp * L + RU - 1) / RU);              // a prefill's leaves
  return units * g.H + num_sms();
}

}  // namespace
}  // namespace kvq

using namespace kvq;

extern "C" {

// [schedule][the leaves' schedule][leaf partials][slots]
static size_t leaf_at() { return kSchedBytes + kLeafSchedBytes; }
static size_t slots_at(const Geom& g) {
  const size_t units = (size_t)g.B * g.H * ((g.Hq / g.H + 7) / 8);
  const size_t n = units + (size_t)num_sms() * kLeafCtas * kLeafWarps;
  return leaf_at() + (n * leaf_floats(g.D) * 4 + 255) / 256 * 256;
}

// Whether rows, and places of the work split whatever the forks and lengths of a later replay,
// can be counted in 32 bits: an entry of r rows and t tiles has at most H (r / RU + 1)
// units of t + 7 places; a row's entries hold its tokens once, and are at most 65.
static bool countable(const Geom& g, int L) {
  const double rows = (double)g.B * (g.Hq / g.H) * L / unit_rows_of(g.D), tiles = (double)g.Tmax / kTok + 1;
  const double places = g.H * ((rows + g.B + kMaxShared) * tiles + 7 * ((kMaxShared + 1) * rows + g.B + kMaxShared));
  return (double)g.B * g.Hq * L < 2147483584.0 && places < 2147483584.0;
}

size_t kvq_attend_shared_workspace(const kvq_cache* cache, int L) {
  if (!cache || cache->g.layout != KVQ_LAYOUT_PAGED || L <= 0 || !countable(cache->g, L)) return 0;
  // (one size for both calls of L = 1)
  return slots_at(cache->g) + (size_t)shared_slots(cache, L) * slot_floats(cache->g.D) * 4;
}

static kvq_status attend_shared(kvq_cache* cache, const void* q, int L, int n_q_heads, float scale,
                                void* out, void* workspace, size_t workspace_bytes, void* stream,
                                bool decode) {
  if (!cache) return set_error(KVQ_ERR_ARG, "cache is NULL");
  const Geom& g = cache->g;
  if (g.layout != KVQ_LAYOUT_PAGED)
    return set_error(KVQ_ERR_UNSUPPORTED, "shared pages need a paged cache");
  if (L <= 0) return set_error(KVQ_ERR_ARG, "L = %d must be positive", L);
  if (!q || !out || !workspace) return set_error(KVQ_ERR_ARG, "q, out or workspace is NULL");
  if (reinterpret_cast<uintptr_t>(q) % 16 || reinterpret_cast<uintptr_t>(out) % 16)
    return set_error(KVQ_ERR_ARG, "q and out must be 16-byte aligned");
  if (!(scale > 0.f) || scale > 2.35e38f)                // (scores in log2 units: times 1.4427)
    return set_error(KVQ_ERR_ARG, "softmax_scale must be positive and below 2.35e38");
  if (n_q_heads != g.Hq)
    return set_error(KVQ_ERR_SHAPE, "n_q_heads %d != cache q_heads %d", n_q_heads, g.Hq);
  if (!decode)
    for (int b = 0; b < g.B; ++b)
      if (cache->seq_n[b] > L)
        return set_error(KVQ_ERR_SHAPE, "sequence %d appended %d tokens, more than L = %d query "
                         "rows", b, cache->seq_n[b], L);
  if (reinterpret_cast<uintptr_t>(workspace) % 256)
    return set_error(KVQ_ERR_ARG, "workspace must be 256-byte aligned");
  if (!countable(g, L))
    return set_error(KVQ_ERR_SHAPE, "%d query rows a sequence are too many for one call", L);
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e = cudaSuccess;
  if (!cache->plan_known) {
    // a launch failed since the plan was last sent: all of it goes first
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    e = cudaStreamIsCapturing(s, &st);
    if (e == cudaSuccess && st != cudaStreamCaptureStatusNone)
      return set_error(KVQ_ERR_UNSUPPORTED, "the shared pages are sent anew after a failed launch: this "
                       "call cannot be captured in a graph");
    if (e == cudaSuccess) e = update_shared_plan(cache, s);
    if (e != cudaSuccess) return set_error(KVQ_ERR_CUDA, "attend_shared: %s", cudaGetErrorString(e));
  }
  const size_t need = kvq_attend_shared_workspace(cache, L);
  if (workspace_bytes < need)
    return set_error(KVQ_ERR_CAPACITY, "workspace of %zu bytes < %zu", workspace_bytes, need);
  int* err = device_error_word();
  if (!err) return set_error(KVQ_ERR_CUDA, "cannot resolve the device error word");
  Call c;
  c.q = static_cast<const __nv_bfloat16*>(q);
  c.L = L;
  c.decode = decode;
  c.scale = scale;
  c.out = static_cast<__nv_bfloat16*>(out);
  c.err = err;
  c.sched = static_cast<SchedOut*>(workspace);
  c.leaf_sched = reinterpret_cast<LeafSched*>(static_cast<char*>(workspace) + kSchedBytes);
  c.leaf = reinterpret_cast<float*>(static_cast<char*>(workspace) + leaf_at());
  c.slots = reinterpret_cast<float*>(static_cast<char*>(workspace) + slots_at(g));
  c.cap = (int)std::min<size_t>((workspace_bytes - slots_at(g)) / (slot_floats(g.D) * 4), 1 << 30);
  // (captured calls always run the kernels here: a replay follows the forks and lengths of its
  // time)
  if (!decode && alone_faster(cache)) {
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    e = cudaStreamIsCapturing(s, &st);
    if (e == cudaSuccess && st == cudaStreamCaptureStatusNone)
      return kvq_attend_prefill(cache, q, L, n_q_heads, scale, out, stream);
  }
  if (e == cudaSuccess) e = ensure_cache_init(cache, s);
  if (e == cudaSuccess) e = launch_shared(g, c, s);
  if (e == cudaErrorStreamCaptureUnsupported)
    return set_error(KVQ_ERR_UNSUPPORTED, "attend_shared: the first call on a paged cache after it was created "
                     "or reset cannot be captured in a graph: its replays would empty the cache");
  if (e != cudaSuccess) return set_error(KVQ_ERR_CUDA, "attend_shared: %s", cudaGetErrorString(e));
  return KVQ_OK;
}

kvq_status kvq_attend_decode_shared(kvq_cache* cache, const void* q, int n_q_heads,
                                    float softmax_scale, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  return attend_shared(cache, q, 1, n_q_heads, softmax_scale, out, workspace, workspace_bytes,
                       stream, true);
}

kvq_status kvq_attend_prefill_shared(kvq_cache* cache, const void* q, int L, int n_q_heads,
                                     float softmax_scale, void* out, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  return attend_shared(cache, q, L, n_q_heads, softmax_scale, out, workspace, workspace_bytes,
                       stream, false);
}

}  // extern "C"
