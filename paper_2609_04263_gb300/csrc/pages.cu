// Pages and sequences of ragged and paged caches: forking, copying between caches,
// rolling back, freeing and compacting (a serving batch of the incremental cache of
// Section 3.1: several continuations of one prompt, drafted tokens that are rejected,
// sequences that come and go).
//
// A page is shared (page_refs > 1) only once all its tokens are final: coded, and below
// the count of every sequence that holds it.  What an append may still write (a
// part-filled page; the pages of a KIVI cache that its uncoded window reaches, and the
// window itself) belongs to one sequence alone and is copied by a fork, so appends need
// no copy-on-write and their kernels no check.
//
// The host keeps the lists of pages, their holders and the tree of shared runs; the
// device follows through kernels whose arguments carry the changed entries, so nothing
// is staged in host memory and a call returns without waiting.  Rows move in one
// kernel: a CTA takes the rows of one page (or a piece of a full-precision window) of
// one kv head in all planes.
#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "kvq_internal.cuh"

namespace kvq {

// ---------------------------------------------------------------------------
// the pool
// ---------------------------------------------------------------------------
int page_take(kvq_cache* c) {
  int& w = c->free_from;
  while (c->free_bits[w] == 0) ++w;
  const int p = 64 * w + __builtin_ctzll(c->free_bits[w]);
  c->free_bits[w] &= c->free_bits[w] - 1;
  --c->n_free;
  c->page_refs[p] = 1;
  return p;
}

void page_drop(kvq_cache* c, int page) {
  if (--c->page_refs[page] > 0) return;
  c->free_bits[page / 64] |= 1ull << (page % 64);
  c->free_from = std::min(c->free_from, page / 64);
  ++c->n_free;
}

// Pages lo and above are free, those below are not.
static void free_above(kvq_cache* c, int lo) {
  const int n = c->desc.num_pages;
  std::fill(c->free_bits.begin(), c->free_bits.end(), 0);
  for (int p = lo; p < n; ++p) c->free_bits[p / 64] |= 1ull << (p % 64);
  c->n_free = n - lo;
  c->free_from = lo / 64;
}

void pages_reset(kvq_cache* c) {
  const int n = c->desc.num_pages;
  c->free_bits.resize((n + 63) / 64);
  c->page_refs.assign(n, 0);
  free_above(c, 0);
  c->plan.clear();                                       // the device's is zeroed with its state
  c->plan_known = true;
}

void refresh_max_tokens(kvq_cache* c) {
  int t = 0;
  for (int x : c->seq_T) t = std::max(t, x);
  c->T = t;
}

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------
// kernels.  Lists travel as kernel arguments (at most 32,764 bytes); short ones in
// a smaller struct, which launches faster.
// ---------------------------------------------------------------------------

template <int N>
struct Words {
  int32_t n, at;
  int32_t w[N];
};
template <int N>
__global__ void plan_words_kernel(Geom g, const __grid_constant__ Words<N> a) {
  pdl_wait();
  pdl_trigger();
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) g.shared_plan[a.at + i] = a.w[i];
}

__device__ __forceinline__ void copy16(const char* s, char* d, int n16, int first, int step) {
  // four loads in flight a thread
  for (int i = first; i < n16; i += 4 * step) {
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < n16) v[k] = reinterpret_cast<const uint4*>(s)[i + k * step];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < n16) reinterpret_cast<uint4*>(d)[i + k * step] = v[k];
  }
}

// Rows 0 .. rows - 1 of a page, all planes of one kv head: page sp of batch index sb (RAGGED /
// UNIFORM: the sequence's page-sized range of rows; PAGED: sb = 0 and a pool page) to
// page dp of db.  A KIVI cache's key scales and offsets have a row per 32-token block
// (rows is a multiple of 32 then).
__device__ __forceinline__ void copy_page(const Geom& to, const Geom& from, int h, int sb, int sp, int db,
                                          int dp, int rows) {
  constexpr int planes[6] = {KVQ_PLANE_K_CODES, KVQ_PLANE_V_CODES, KVQ_PLANE_K_SCALE,
                             KVQ_PLANE_V_SCALE, KVQ_PLANE_K_ZERO, KVQ_PLANE_V_ZERO};
#pragma unroll
  for (int p = 0; p < 6; ++p) {
    const int which = planes[p];
    const Plane& pl = to.pl[which];
    if (pl.p == nullptr) continue;                       // symmetric caches have no offsets
    const bool blk = to.fmt == KVQ_FMT_KIVI && (which == KVQ_PLANE_K_SCALE || which == KVQ_PLANE_K_ZERO);
    const int per = blk ? kPageTok / 32 : kPageTok, n = blk ? rows / 32 : rows;
    const int64_t row_b = pl.cols * pl.elem;             // a multiple of 4 bytes
    const char* s = reinterpret_cast<const char*>(from.pl[which].p) +
                    (((int64_t)sb * from.H + h) * from.pl[which].rows + (int64_t)sp * per) * row_b;
    char* d = reinterpret_cast<char*>(pl.p) + (((int64_t)db * to.H + h) * pl.rows + (int64_t)dp * per) * row_b;
    const int bytes = (int)(n * row_b), n16 = bytes / 16;
    copy16(s, d, n16, threadIdx.x, kThreads);
    const int tail = (bytes - 16 * n16) / 4;
    if ((int)threadIdx.x < tail)
      reinterpret_cast<uint32_t*>(d + 16 * (int64_t)n16)[threadIdx.x] =
          reinterpret_cast<const uint32_t*>(s + 16 * (int64_t)n16)[threadIdx.x];
  }
}

// Roll-backs and compaction: new counts, changed table entries, and the first `rows` rows of
// pages that move within the pool (nothing reads the table for those).
struct SeqEdit {
  int32_t b, len;
};
struct TableEntry {
  int32_t index, page;
};
struct Job {
  int32_t src, dst, rows;
};
template <int N, int M, int J>
struct Changes {
  int32_t n, m;
  SeqEdit e[N];
  TableEntry t[M];
  Job j[J];
};
template <int N, int M, int J>
__global__ void __launch_bounds__(kThreads) change_kernel(Geom g, const __grid_constant__ Changes<N, M, J> a, int jobs) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    for (int i = threadIdx.x; i < a.n; i += kThreads) {
      g.seq_len[a.e[i].b] = a.e[i].len;
      g.seq_new[a.e[i].b] = 0;
    }
    for (int i = threadIdx.x; i < a.m; i += kThreads) g.page_table[a.t[i].index] = a.t[i].page;
  }
  if ((int)blockIdx.x < jobs) {
    const Job j = a.j[blockIdx.x];
    copy_page(g, g, blockIdx.y, 0, j.src, 0, j.dst, j.rows);
  }
}

// Fork or copy: sequence dst becomes the first `tokens` tokens of src, its first `keep` pages
// shared, the others' numbers at pages[first ..] (PAGED); pages lo .. upto - 1 are this
// entry's (a long sequence takes several, lo = keep in its first).  A CTA takes the rows of one
// page of one kv head, or 64 tokens of the full-precision window; the first of an entry
// its counts and table row.  Bound by HBM where the batch is large (rows are read and
// written once), by the launch where it is small: pages and places are worked out here, as the
// entries of every copy (24 bytes each) took 10 us to hand over.
struct Take {
  int32_t src, dst, keep, tokens, first, lo, upto;
};
template <int N, int M>
struct Takes {
  int32_t window;                                        // window pieces an entry (K and V)
  Take t[N];
  int32_t pages[M];
};
template <int N, int M>
__global__ void __launch_bounds__(kThreads)
take_kernel(const __grid_constant__ Geom to, const __grid_constant__ Geom from, const __grid_constant__ Takes<N, M> a) {
  pdl_wait();
  pdl_trigger();
  const Take t = a.t[blockIdx.z];
  const int h = blockIdx.y, x = blockIdx.x;
  const bool paged = to.layout == KVQ_LAYOUT_PAGED, from_pages = from.layout == KVQ_LAYOUT_PAGED;
  const int coded = to.fmt == KVQ_FMT_KIVI ? kivi_tq(t.tokens, to.R, to.G) : t.tokens;
  const bool begins = t.lo == t.keep;
  if (x == 0 && h == 0) {
    if (paged)
      for (int j = (begins ? 0 : t.lo) + threadIdx.x; j < t.upto; j += kThreads)
        to.page_table[(size_t)t.dst * to.max_pages + j] =
            j < t.keep ? to.page_table[(size_t)t.src * to.max_pages + j] : a.pages[t.first + j - t.lo];
    if (threadIdx.x == 0) {
      to.seq_len[t.dst] = t.tokens;
      to.seq_new[t.dst] = 0;
    }
  }
  if (x < a.window) {
    if (!begins) return;
    const int lo = coded + 64 * (x >> 1), n = min(64, t.tokens - lo);
    if (n <= 0) return;
    // (a window is no longer than its ring: the rows wrap at most once)
    const int which = x & 1 ? KVQ_PLANE_V_FULL : KVQ_PLANE_K_FULL, row = 2 * to.D;   // bytes
    const int slot0 = lo % to.ring, n0 = min(n, to.ring - slot0);
    char* d = reinterpret_cast<char*>(plane_ptr<__nv_bfloat16>(to, which, t.dst, h, 0, 0));
    const char* s = reinterpret_cast<const char*>(plane_ptr<__nv_bfloat16>(from, which, t.src, h, 0, 0));
    const int64_t at = (int64_t)slot0 * row;
    copy16(s + at, d + at, n0 * row / 16, threadIdx.x, kThreads);
    copy16(s, d, (n - n0) * row / 16, threadIdx.x, kThreads);
    return;
  }
  const int j = t.lo + x - a.window, rows = min(kPageTok, coded - j * kPageTok);
  if (j >= t.upto || rows <= 0) return;
  const int sp = from_pages ? from.page_table[(size_t)t.src * from.max_pages + j] : j;
  copy_page(to, from, h, from_pages ? 0 : t.src, sp, paged ? 0 : t.dst, paged ? a.pages[t.first + j - t.lo] : j, rows);
}

template <int N, int M, int J>
void launch_changes_n(const Geom& g, const SeqEdit* e, size_t ne, const TableEntry* t, size_t nt, const Job* j,
                      size_t nj, cudaStream_t s) {
  Changes<N, M, J> a;
  a.n = (int)ne;
  a.m = (int)nt;
  std::copy(e, e + ne, a.e);
  std::copy(t, t + nt, a.t);
  std::copy(j, j + nj, a.j);
  launch_pdl(change_kernel<N, M, J>, dim3(std::max<unsigned>(1, (unsigned)nj), nj ? g.H : 1), dim3(kThreads), 0, s, g, a, (int)nj);
}

cudaError_t launch_changes(const Geom& g, const std::vector<SeqEdit>& e, const std::vector<TableEntry>& t,
                           const std::vector<Job>& j, cudaStream_t s) {
  constexpr size_t N = KVQ_MAX_SEQS, M = 1200, J = 1200, n = 64, m = 64, k = 64;   // 28.1 and 1.8 KB
  for (size_t e0 = 0, t0 = 0, j0 = 0; e0 < e.size() || t0 < t.size() || j0 < j.size();) {
    const size_t le = e.size() - e0, lt = t.size() - t0, lj = j.size() - j0;
    const bool few = le <= n && lt <= m && lj <= k;
    const size_t ne = std::min(N, le), nt = std::min(M, lt), nj = std::min(J, lj);
    if (few) launch_changes_n<n, m, k>(g, e.data() + e0, ne, t.data() + t0, nt, j.data() + j0, nj, s);
    else launch_changes_n<N, M, J>(g, e.data() + e0, ne, t.data() + t0, nt, j.data() + j0, nj, s);
    e0 += ne;
    t0 += nt;
    j0 += nj;
  }
  return cudaGetLastError();
}

constexpr int kTakePages = 5400;                         // pages of an entry at most

template <int N, int M>
void launch_takes_n(const Geom& to, const Geom& from, const Take* t, int n, const int32_t* pages,
                    int first, int np, int window, cudaStream_t s) {
  Takes<N, M> a;
  a.window = window;
  int most = 0;
  for (int i = 0; i < n; ++i) {
    a.t[i] = t[i];
    a.t[i].first -= first;
    most = std::max(most, t[i].upto - t[i].lo);
  }
  std::copy(pages + first, pages + first + np, a.pages);
  launch_pdl(take_kernel<N, M>, dim3((unsigned)std::max(1, window + most), to.H, n), dim3(kThreads), 0, s, to, from, a);
}

// Entries in as many launches as their pages' numbers fit into.
cudaError_t launch_takes(const Geom& to, const Geom& from, const std::vector<Take>& t,
                         const std::vector<int32_t>& pages, int window, cudaStream_t s) {
  constexpr int N = 256, M = kTakePages, n = 64, m = 256;   // 28.8 and 2.8 KB of arguments
  for (size_t i = 0; i < t.size();) {
    size_t k = i;
    int np = 0;
    const int first = t[i].first;
    for (; k < t.size() && k - i < (size_t)N; ++k) {
      const int end = (k + 1 < t.size() ? t[k + 1].first : (int)pages.size()) - first;
      if (end > M) break;
      np = end;
    }
    if (k - i <= (size_t)n && np <= m) launch_takes_n<n, m>(to, from, &t[i], (int)(k - i), pages.data(), first, np, window, s);
    else launch_takes_n<N, M>(to, from, &t[i], (int)(k - i), pages.data(), first, np, window, s);
    i = k;
  }
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// the plan of shared pages
// ---------------------------------------------------------------------------
struct PlanBuilder {
  const kvq_cache* c;
  std::vector<SharedNode> nodes;
  std::vector<int32_t> order, leaf_page, leaf_parent;

  // `m` share their first `page` pages, the last node above them is `parent`
  void split(const std::vector<int>& m, int page, int parent) {
    std::vector<std::pair<int, int>> by;                 // (shared page at this place or -1, sequence)
    by.reserve(m.size());
    for (int b : m) {
      const std::vector<int>& pg = c->seq_pages[b];
      by.emplace_back(page < (int)pg.size() && c->page_refs[pg[page]] > 1 ? pg[page] : -1, b);
    }
    std::sort(by.begin(), by.end());
    for (size_t i = 0; i < by.size();) {
      size_t k = i + 1;
      while (k < by.size() && by[k].first == by[i].first) ++k;
      if (by[i].first < 0 || k - i == 1) {
        for (; i < k; ++i) {
          order.push_back(by[i].second);
          leaf_page[by[i].second] = page;
          leaf_parent[by[i].second] = parent;
        }
        continue;
      }
      // how far all of them agree
      const std::vector<int>& first = c->seq_pages[by[i].second];
      int p1 = (int)first.size();
      std::vector<int> sub;
      sub.reserve(k - i);
      for (size_t j = i; j < k; ++j) {
        const std::vector<int>& pg = c->seq_pages[by[j].second];
        sub.push_back(by[j].second);
        const int most = std::min(p1, (int)pg.size());
        p1 = (int)(std::mismatch(first.begin() + page, first.begin() + most, pg.begin() + page).first - first.begin());
      }
      const int id = (int)nodes.size();
      nodes.push_back(SharedNode{page, p1, (int32_t)order.size(), (int32_t)sub.size(), parent, {0, 0, 0}});
      split(sub, p1, id + 1);
      i = k;
    }
  }

  // The nodes worth a pass of their own, parents first, at most kMaxShared; the
  // members of the others start their leaves there.
  void prune() {
    const int n = (int)nodes.size();
    std::vector<char> keep(n, 1);
    int kept = n;
    const auto gain = [&](int i) { return (int64_t)(nodes[i].count - 1) * (nodes[i].p1 - nodes[i].p0); };
    while (kept > kMaxShared) {                          // rare: the least useful without a kept child
      std::vector<char> inner(n, 0);
      for (int i = 0; i < n; ++i)
        if (keep[i] && nodes[i].parent) inner[nodes[i].parent - 1] = 1;
      int worst = -1;
      for (int i = 0; i < n; ++i)
        if (keep[i] && !inner[i] && (worst < 0 || gain(i) < gain(worst))) worst = i;
      keep[worst] = 0;
      --kept;
    }
    std::vector<int> id(n, 0);
    std::vector<SharedNode> out;
    for (int i = 0; i < n; ++i) {                        // (parents stand before children)
      if (!keep[i]) continue;
      SharedNode x = nodes[i];
      if (x.parent) x.parent = id[x.parent - 1];
      out.push_back(x);
      id[i] = (int)out.size();
    }
    for (size_t b = 0; b < leaf_parent.size(); ++b) {
      int p = leaf_parent[b];
      while (p && !keep[p - 1]) {
        leaf_page[b] = nodes[p - 1].p0;
        p = nodes[p - 1].parent;
      }
      leaf_parent[b] = p ? id[p - 1] : 0;
    }
    nodes.swap(out);
  }
};

template <int N>
cudaError_t launch_words_n(const Geom& g, const int32_t* w, int at, int n, cudaStream_t s) {
  Words<N> a;
  a.n = n;
  a.at = at;
  std::copy(w + at, w + at + n, a.w);
  return launch_pdl(plan_words_kernel<N>, dim3(1), dim3(256), 0, s, g, a);
}

}  // namespace

// (throws where host memory runs out, before anything is sent)
static cudaError_t send_shared_plan(kvq_cache* c, cudaStream_t s) {
  const Geom& g = c->g;
  bool shared = false;
  for (int b = 0; b < g.B && !shared; ++b)
    shared = !c->seq_pages[b].empty() && c->page_refs[c->seq_pages[b][0]] > 1;
  if (!shared && c->plan.empty() && c->plan_known) return cudaSuccess;   // none before, none now
  PlanBuilder pb{c, {}, {}, std::vector<int32_t>(g.B, 0), std::vector<int32_t>(g.B, 0)};
  std::vector<int> all(g.B);
  for (int b = 0; b < g.B; ++b) all[b] = b;
  pb.split(all, 0, 0);
  pb.prune();
  std::vector<int32_t> w(plan_words(g.B), 0);
  w[0] = (int32_t)pb.nodes.size();
  for (size_t i = 0; i < pb.nodes.size(); ++i)
    std::copy_n(reinterpret_cast<const int32_t*>(&pb.nodes[i]), sizeof(SharedNode) / 4,
                w.begin() + kPlanHead + i * (sizeof(SharedNode) / 4));
  std::copy(pb.order.begin(), pb.order.end(), w.begin() + kPlanNodes);
  std::copy(pb.leaf_page.begin(), pb.leaf_page.end(), w.begin() + kPlanNodes + g.B);
  std::copy(pb.leaf_parent.begin(), pb.leaf_parent.end(), w.begin() + kPlanNodes + 2 * g.B);
  // the changed range alone, in argument-sized pieces
  int lo = 0, hi = (int)w.size();
  if (c->plan_known && c->plan.size() == w.size()) {
    while (lo < hi && w[lo] == c->plan[lo]) ++lo;
    while (hi > lo && w[hi - 1] == c->plan[hi - 1]) --hi;
  }
  c->plan.swap(w);
  c->plan_known = false;
  constexpr int N = 4000, n = 700;
  cudaError_t e = cudaSuccess;
  for (int at = lo; at < hi && e == cudaSuccess; at += N) {
    const int k = std::min(N, hi - at);
    e = k <= n ? launch_words_n<n>(g, c->plan.data(), at, k, s) : launch_words_n<N>(g, c->plan.data(), at, k, s);
  }
  c->plan_known = e == cudaSuccess;
  if (e != cudaSuccess) (void)cudaGetLastError();        // (reported here)
  return e;
}

cudaError_t update_shared_plan(kvq_cache* c, cudaStream_t s) {
  if (c->g.layout != KVQ_LAYOUT_PAGED) return cudaSuccess;
  try {
    return send_shared_plan(c, s);
  } catch (...) {
    // the plan without shared runs is right for any pages, and needs no memory
    c->plan.clear();
    const cudaError_t e = cudaMemsetAsync(c->g.shared_plan, 0, (size_t)plan_words(c->g.B) * 4, s);
    c->plan_known = e == cudaSuccess;
    return e;
  }
}

namespace {

int coded_tokens(const Geom& g, int t) {
  return g.fmt == KVQ_FMT_KIVI ? kivi_tq(t, g.R, g.G) : t;
}
int pages_of(int t) { return (t + kPageTok - 1) / kPageTok; }

// Calls that change the lists on the host take effect once, when they are made.
kvq_status no_capture(cudaStream_t s, const char* what) {
  cudaStreamCaptureStatus st;
  const cudaError_t e = cudaStreamIsCapturing(s, &st);
  if (e != cudaSuccess) return set_error(KVQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  if (st != cudaStreamCaptureStatusNone)
    return set_error(KVQ_ERR_UNSUPPORTED, "%s changes the cache's lists on the host: it cannot be "
                     "captured in a graph", what);
  return KVQ_OK;
}

kvq_status cuda_error(cudaError_t e, const char* what) {
  return set_error(KVQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

int seq_count(const kvq_cache* c, int b) {
  return c->g.layout == KVQ_LAYOUT_UNIFORM ? c->T : c->seq_T[b];
}

// A sequence of t tokens can be cut to n: KIVI keeps the window at full precision, and
// tokens once coded do not come back to it.
kvq_status check_cut(const Geom& g, const char* what, int b, int t, int n) {
  if (n < 0 || n > t)
    return set_error(KVQ_ERR_ARG, "%s: %d tokens of sequence %d, which holds %d", what, n, b, t);
  if (g.fmt == KVQ_FMT_KIVI && n > 0 && coded_tokens(g, n) != coded_tokens(g, t))
    return set_error(KVQ_ERR_UNSUPPORTED, "%s: the first %d of sequence %d's %d tokens would have "
                     "%d at full precision, which are coded already", what, n, b, t,
                     n - coded_tokens(g, n));
  return KVQ_OK;
}

// src[i], dst[i], tokens[i] of a fork or copy: dst distinct, and none of them a source
// where both are one cache's.
kvq_status check_lists(const char* what, const kvq_cache* to, const kvq_cache* from, int n,
                       const int* src, const int* dst, const int* tokens) {
  if (n < 0) return set_error(KVQ_ERR_ARG, "%s: n = %d < 0", what, n);
  if (n > to->g.B) return set_error(KVQ_ERR_ARG, "%s: %d sequences, the cache has %d", what, n, to->g.B);
  if (n > 0 && (!src || !dst)) return set_error(KVQ_ERR_ARG, "%s: src or dst is NULL", what);
  std::vector<char> used(to->g.B, 0);
  for (int i = 0; i < n; ++i) {
    if (src[i] < 0 || src[i] >= from->g.B)
      return set_error(KVQ_ERR_ARG, "%s: source %d outside [0, %d)", what, src[i], from->g.B);
    if (dst[i] < 0 || dst[i] >= to->g.B)
      return set_error(KVQ_ERR_ARG, "%s: destination %d outside [0, %d)", what, dst[i], to->g.B);
    if (used[dst[i]]) return set_error(KVQ_ERR_ARG, "%s: destination %d twice", what, dst[i]);
    used[dst[i]] = 1;
  }
  for (int i = 0; i < n; ++i) {
    if (to == from && used[src[i]])
      return set_error(KVQ_ERR_ARG, "%s: sequence %d is both a source and a destination", what, src[i]);
    const int t = seq_count(from, src[i]), k = tokens ? tokens[i] : t;
    if (kvq_status st = check_cut(from->g, what, src[i], t, k)) return st;
    if (k > to->g.Tmax)
      return set_error(KVQ_ERR_CAPACITY, "%s: %d tokens exceed max_tokens %d", what, k, to->g.Tmax);
  }
  return KVQ_OK;
}

// Fork (to == from) or copy: see kvq.h.
kvq_status take_sequences(const char* what, kvq_cache* to, kvq_cache* from, int n, const int* src,
                          const int* dst, const int* tokens, cudaStream_t s) {
  if (kvq_status st = check_lists(what, to, from, n, src, dst, tokens)) return st;
  if (kvq_status st = no_capture(s, what)) return st;
  if (n == 0) return KVQ_OK;
  const Geom& g = to->g;
  const bool paged = g.layout == KVQ_LAYOUT_PAGED, share = paged && to == from;
  std::vector<int> cnt(n), keep(n, 0), same(n, 0);
  int need = 0, freed = 0;
  for (int i = 0; i < n; ++i) {
    cnt[i] = tokens ? tokens[i] : seq_count(from, src[i]);
    if (share) {
      keep[i] = coded_tokens(g, cnt[i]) / kPageTok;      // whole final pages
      // those that the destination holds already stay (beams and samples of one prompt)
      const std::vector<int> &own = to->seq_pages[dst[i]], &pg = from->seq_pages[src[i]];
      const auto upto = own.begin() + std::min<int>(keep[i], (int)own.size());
      same[i] = (int)(std::mismatch(own.begin(), upto, pg.begin()).first - own.begin());
    }
    need += pages_of(cnt[i]) - keep[i];
  }
  std::vector<Take> takes;
  takes.reserve(n + need / kTakePages);
  std::vector<int32_t> fresh;
  if (paged) {
    fresh.reserve(need);
    for (int i = 0; i < n; ++i) to->seq_pages[dst[i]].reserve(pages_of(cnt[i]));
  }
  cudaError_t e = ensure_cache_init(from, s);
  if (e == cudaSuccess && to != from) e = ensure_cache_init(to, s);
  if (e != cudaSuccess) return cuda_error(e, what);
  if (paged) {
    // the destinations' other pages go back first; where they are needed, counted before
    if (need > to->n_free) {
      for (int i = 0; i < n; ++i)
        for (size_t j = same[i]; j < to->seq_pages[dst[i]].size(); ++j)
          freed += --to->page_refs[to->seq_pages[dst[i]][j]] == 0;
      for (int i = 0; i < n; ++i)
        for (size_t j = same[i]; j < to->seq_pages[dst[i]].size(); ++j) ++to->page_refs[to->seq_pages[dst[i]][j]];
    }
    if (need > to->n_free + freed)
      return set_error(KVQ_ERR_CAPACITY, "%s needs %d pages, %d are free", what, need, to->n_free + freed);
    for (int i = 0; i < n; ++i) {
      std::vector<int>& own = to->seq_pages[dst[i]];
      for (size_t j = same[i]; j < own.size(); ++j) page_drop(to, own[j]);
      own.resize(same[i]);
    }
  }
  int window = 0;
  for (int i = 0; i < n; ++i) {
    const int t = cnt[i], db = dst[i];
    if (g.fmt == KVQ_FMT_KIVI) window = std::max(window, 2 * ((t - coded_tokens(g, t) + 63) / 64));
    for (int lo = keep[i], all = pages_of(t); lo == keep[i] || lo < all; lo += kTakePages)
      takes.push_back(Take{src[i], db, keep[i], t, (int32_t)fresh.size() + (paged ? lo - keep[i] : 0), lo,
                           std::min(all, lo + kTakePages)});
    if (paged) {
      std::vector<int>& own = to->seq_pages[db];         // (with room for all)
      for (int j = same[i]; j < keep[i]; ++j) {
        own.push_back(from->seq_pages[src[i]][j]);
        ++to->page_refs[own.back()];
      }
      for (int j = keep[i]; j < pages_of(t); ++j) {
        const int p = page_take(to);
        own.push_back(p);
        fresh.push_back(p);
      }
    }
    to->seq_T[db] = t;
    to->seq_n[db] = 0;
  }
  refresh_max_tokens(to);
  e = launch_takes(g, from->g, takes, fresh, window, s);
  const cudaError_t sent = update_shared_plan(to, s);    // (of the lists as they are, whatever e is)
  if (e == cudaSuccess) e = sent;
  return e == cudaSuccess ? KVQ_OK : cuda_error(e, what);
}

kvq_status truncate(kvq_cache* c, int n, const int* seqs, const int* tokens, cudaStream_t s) {
  const char* what = "kvq_seq_truncate";
  const Geom& g = c->g;
  if (g.layout == KVQ_LAYOUT_UNIFORM)
    return set_error(KVQ_ERR_UNSUPPORTED, "%s needs a ragged or paged cache", what);
  if (n < 0 || n > g.B) return set_error(KVQ_ERR_ARG, "%s: n = %d outside [0, %d]", what, n, g.B);
  if (n > 0 && (!seqs || !tokens)) return set_error(KVQ_ERR_ARG, "%s: seqs or tokens is NULL", what);
  std::vector<char> used(g.B, 0);
  for (int i = 0; i < n; ++i) {
    const int b = seqs[i];
    if (b < 0 || b >= g.B) return set_error(KVQ_ERR_ARG, "%s: sequence %d outside [0, %d)", what, b, g.B);
    if (used[b]) return set_error(KVQ_ERR_ARG, "%s: sequence %d twice", what, b);
    used[b] = 1;
    if (kvq_status st = check_cut(g, what, b, c->seq_T[b], tokens[i])) return st;
  }
  if (kvq_status st = no_capture(s, what)) return st;
  if (n == 0) return KVQ_OK;
  const bool paged = g.layout == KVQ_LAYOUT_PAGED;
  // a part-filled last page that others hold too is replaced by a copy of its own (a
  // KIVI sequence's last pages are its own already)
  std::vector<SeqEdit> edits;
  std::vector<TableEntry> entries;
  std::vector<Job> jobs;
  edits.reserve(n);
  entries.reserve(n);
  jobs.reserve(n);
  cudaError_t e = ensure_cache_init(c, s);
  if (e != cudaSuccess) return cuda_error(e, what);
  if (paged) {
    // pages given up, then the copies that are needed: of a shared page, one for each
    // holder that cuts it but the last holder of all
    int need = 0, freed = 0;
    for (int i = 0; i < n; ++i) {
      const std::vector<int>& pg = c->seq_pages[seqs[i]];
      for (int j = pages_of(tokens[i]); j < (int)pg.size(); ++j) freed += --c->page_refs[pg[j]] == 0;
    }
    for (int i = 0; i < n; ++i) {
      const int j = tokens[i] / kPageTok;
      if (tokens[i] % kPageTok && c->page_refs[c->seq_pages[seqs[i]][j]] > 1) {
        --c->page_refs[c->seq_pages[seqs[i]][j]];
        entries.push_back(TableEntry{i, 0});             // (marks the copy)
        ++need;
      }
    }
    const int have = c->n_free + freed;
    for (const TableEntry& x : entries)
      ++c->page_refs[c->seq_pages[seqs[x.index]][tokens[x.index] / kPageTok]];
    for (int i = 0; i < n; ++i) {
      const std::vector<int>& pg = c->seq_pages[seqs[i]];
      for (int j = pages_of(tokens[i]); j < (int)pg.size(); ++j) ++c->page_refs[pg[j]];
    }
    entries.clear();
    if (need > have)
      return set_error(KVQ_ERR_CAPACITY, "%s needs %d pages, %d are free", what, need, have);
    for (int i = 0; i < n; ++i) {
      std::vector<int>& pg = c->seq_pages[seqs[i]];
      for (int j = pages_of(tokens[i]); j < (int)pg.size(); ++j) page_drop(c, pg[j]);
      pg.resize(pages_of(tokens[i]));
    }
  }
  for (int i = 0; i < n; ++i) {
    const int b = seqs[i], t = tokens[i], j = t / kPageTok;
    if (paged && t % kPageTok && c->page_refs[c->seq_pages[b][j]] > 1) {
      const int old = c->seq_pages[b][j], p = page_take(c);
      --c->page_refs[old];
      c->seq_pages[b][j] = p;
      entries.push_back(TableEntry{b * g.max_pages + j, p});
      jobs.push_back(Job{old, p, t % kPageTok});
    }
    edits.push_back(SeqEdit{b, t});
    c->seq_T[b] = t;
    c->seq_n[b] = 0;
  }
  refresh_max_tokens(c);
  e = launch_changes(g, edits, entries, jobs, s);
  const cudaError_t sent = update_shared_plan(c, s);
  if (e == cudaSuccess) e = sent;
  return e == cudaSuccess ? KVQ_OK : cuda_error(e, what);
}

kvq_status compact(kvq_cache* c, cudaStream_t s) {
  const char* what = "kvq_cache_compact";
  const Geom& g = c->g;
  if (g.layout != KVQ_LAYOUT_PAGED) return set_error(KVQ_ERR_UNSUPPORTED, "%s needs a paged cache", what);
  if (kvq_status st = no_capture(s, what)) return st;
  const int pool = c->desc.num_pages, held = pool - c->n_free;
  // held pages above the first `held` go to the free ones below, in ascending order
  std::vector<int> where(pool, -1);
  std::vector<Job> jobs;
  int low = 0;
  for (int p = held; p < pool; ++p) {
    if (c->page_refs[p] == 0) continue;
    while (c->page_refs[low] > 0) ++low;
    where[p] = low;
    jobs.push_back(Job{p, low++, kPageTok});
  }
  if (jobs.empty()) return KVQ_OK;
  std::vector<SeqEdit> edits;
  std::vector<TableEntry> entries;
  for (int b = 0; b < g.B; ++b)
    for (size_t j = 0; j < c->seq_pages[b].size(); ++j)
      if (const int p = where[c->seq_pages[b][j]]; p >= 0)
        entries.push_back(TableEntry{(int)(b * g.max_pages + j), p});
  for (const Job& j : jobs) {
    c->page_refs[j.dst] = c->page_refs[j.src];
    c->page_refs[j.src] = 0;
  }
  for (const TableEntry& x : entries)
    c->seq_pages[x.index / g.max_pages][x.index % g.max_pages] = x.page;
  free_above(c, held);
  cudaError_t e = launch_changes(g, edits, entries, jobs, s);
  return e == cudaSuccess ? KVQ_OK : cuda_error(e, what);
}

// No exception leaves a C entry point: lists that do not fit in host memory are the
// only ones here, and come before anything is changed.
template <typename F>
kvq_status guarded(const char* what, F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return set_error(KVQ_ERR_CAPACITY, "%s: out of host memory", what);
  } catch (...) {
    return set_error(KVQ_ERR_ARG, "%s: host error", what);
  }
}

}  // namespace
}  // namespace kvq

using namespace kvq;

extern "C" {

kvq_status kvq_seq_fork(kvq_cache* cache, int n, const int* src, const int* dst,
                        const int* tokens, void* stream) {
  if (!cache) return set_error(KVQ_ERR_ARG, "cache is NULL");
  if (cache->g.layout == KVQ_LAYOUT_UNIFORM)
    return set_error(KVQ_ERR_UNSUPPORTED, "kvq_seq_fork needs a ragged or paged cache");
  return guarded("kvq_seq_fork", [&] {
    return take_sequences("kvq_seq_fork", cache, cache, n, src, dst, tokens, (cudaStream_t)stream);
  });
}

kvq_status kvq_seq_copy(kvq_cache* to, kvq_cache* from, int n, const int* src, const int* dst,
                        const int* tokens, void* stream) {
  if (!to || !from) return set_error(KVQ_ERR_ARG, "cache is NULL");
  if (to == from) return set_error(KVQ_ERR_ARG, "kvq_seq_copy within one cache: use kvq_seq_fork");
  if (to->g.layout == KVQ_LAYOUT_UNIFORM)
    return set_error(KVQ_ERR_UNSUPPORTED, "kvq_seq_copy needs a ragged or paged destination");
  const Geom &a = to->g, &b = from->g;
  const bool kivi = a.fmt == KVQ_FMT_KIVI;
  if (a.fmt != b.fmt || a.kb != b.kb || a.vb != b.vb || a.G != b.G || a.H != b.H || a.D != b.D ||
      a.act != b.act || (kivi && a.R != b.R))
    return set_error(KVQ_ERR_SHAPE, "kvq_seq_copy: the caches' formats or head shapes differ");
  return guarded("kvq_seq_copy", [&] {
    return take_sequences("kvq_seq_copy", to, from, n, src, dst, tokens, (cudaStream_t)stream);
  });
}

kvq_status kvq_seq_truncate(kvq_cache* cache, int n, const int* seqs, const int* tokens,
                            void* stream) {
  if (!cache) return set_error(KVQ_ERR_ARG, "cache is NULL");
  return guarded("kvq_seq_truncate", [&] { return truncate(cache, n, seqs, tokens, (cudaStream_t)stream); });
}

kvq_status kvq_cache_compact(kvq_cache* cache, void* stream) {
  if (!cache) return set_error(KVQ_ERR_ARG, "cache is NULL");
  return guarded("kvq_cache_compact", [&] { return compact(cache, (cudaStream_t)stream); });
}

}  // extern "C"
