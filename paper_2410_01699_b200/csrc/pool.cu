// Pages of the 8-bit cache: giving (with a copy where a shared page is written), sharing, taking back, moving together.
//
// Every decision is taken on the device from refs (table entries per page) and the table.  Who gets which page follows from the order of
// the claims and of the free pages' indices alone, so results do not hang on the order in which threads run: a prefix count numbers the
// claims that need a page and another one the free pages, and number i gets number i.
// Bound: the copies (a page's bytes read and written once each) at the rate of a device copy; without copies the launches (one block that
// plans, which the copying launch overlaps as far as its own start).  Compaction that moves 320 pages of 4.2 MB (2.69 GB read and written):
// 475 us, 5.7 TB/s.  Sixteen children of a prompt, fork, reserve with 16 copies of 4.2 MB (134 MB) and free: 24.5 us.  Two
// children in a pool of one small layer, fork, reserve and free: 12.4 us, three launches.
#include "common.cuh"

namespace sjd {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kListMax = SJD_POOL_MAX_LIST;
// One block does what takes it less than a launch more would: copies of 128 KB (8 rounds of 16 KB), tables of 16384 entries (16 rounds).
// Fork, reserve and free of two children of a small prompt (32 KB to copy): 12.4 us so, 13.6 with the launches that larger ones take.
constexpr size_t kCopyHere = 128 << 10;
constexpr int kForkHere = 16384;

// device scratch of a call: counts, then int32 lists of n_pages each
constexpr int kLists = 6;
struct PlanScratch {
  int32_t *count;                      // [0] copies, [1] pages in use (compact)
  int32_t *src, *dst;                  // copies: from page, to page
  int32_t *free_list, *old, *claims, *to;
};
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline size_t scratch_bytes(int n_pages) { return 256 + kLists * up256((size_t)n_pages * 4); }
inline PlanScratch scratch_of(void *ws, int n_pages) {
  int32_t *w = (int32_t *)ws, *lists = w + 64;
  const size_t step = up256((size_t)n_pages * 4) / 4;
  return PlanScratch{w, lists, lists + step, lists + 2 * step, lists + 3 * step, lists + 4 * step, lists + 5 * step};
}

// numbers the true predicates of a block in thread order; *total: how many there are.  All threads call it.
__device__ __forceinline__ int block_number(bool pred, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const unsigned m = __ballot_sync(0xffffffffu, pred);
  __syncthreads();   // (the sums of the call before have been read)
  if (lane == 0) warp_sums[warp] = __popc(m);
  __syncthreads();
  int before = 0, all = 0;
  const int mine = lane < n_warps ? warp_sums[lane] : 0;
  before = __reduce_add_sync(0xffffffffu, lane < warp ? mine : 0);
  all = __reduce_add_sync(0xffffffffu, mine);
  *total = all;
  return before + __popc(m & ((1u << lane) - 1));
}

// number of set flags of four neighbouring pages a thread, and the first one's number among all of the block's (in index order)
__device__ __forceinline__ int block_number4(int mine, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  const int sum = warp_sums[lane];   // (32 warps)
  *total = __reduce_add_sync(0xffffffffu, sum);
  return __reduce_add_sync(0xffffffffu, lane < warp ? sum : 0) + x - mine;
}

// whether a list names a sequence twice or one that does not exist; seen: a bit for each sequence.  All threads of the block call it.
__device__ bool list_bad(const int32_t *seqs, int n, int n_seqs, uint32_t *seen) {
  bool bad = false;
  for (int i = threadIdx.x; i < (n_seqs + 31) / 32; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int s = seqs[i];
    if (s < 0 || s >= n_seqs) bad = true;
    else if (atomicOr(&seen[s >> 5], 1u << (s & 31)) >> (s & 31) & 1u) bad = true;
  }
  return __syncthreads_or(bad) != 0;
}

// A claim is (list entry, page of its range); claims are numbered entry by entry.
__global__ void __launch_bounds__(kPlanThreads) reserve_plan_kernel(sjd_pool p, int n, const int32_t *__restrict__ seqs,
                                                                    const int32_t *__restrict__ begin, const int32_t *__restrict__ end,
                                                                    PlanScratch ps, size_t page_bytes, size_t page_exps, int copy_here) {
  extern __shared__ uint32_t seen[];
  __shared__ int warp_sums[32];
  __shared__ int first[kListMax + 1];   // number of the first claim of every list entry
  __shared__ int seq_of[kListMax], page0[kListMax], begin_of[kListMax];
  __shared__ int copies;
  const int tid = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  if (tid == 0) {
    *ps.count = 0;
    copies = 0;
  }
  bool bad = *(volatile int32_t *)p.status != 0;
  if (__syncthreads_or(bad)) return;
  bad = list_bad(seqs, n, p.n_seqs, seen);
  const long most = (long)p.pages_per_seq * KV_PAGE;
  int cnt = 0;
  if (tid < n) {
    const int b = begin[tid], e = end[tid];
    if (b < 0 || e > most || (e > b && b >= most)) bad = true;
    cnt = e > b ? (e - 1) / KV_PAGE - b / KV_PAGE + 1 : 0;
    seq_of[tid] = seqs[tid];
    page0[tid] = b / KV_PAGE;
    begin_of[tid] = b;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) pool_fault(p.status, SJD_ERR_BAD_ARG);
    return;
  }
  {   // exclusive prefix of the counts (kListMax <= kPlanThreads)
    const int lane = tid & 31, warp = tid >> 5;
    int x = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sums[lane] : 0);
    if (tid < kListMax) first[tid + 1] = before + x;
    if (tid == 0) first[0] = 0;
    __syncthreads();
  }
  const int n_claims = first[n];   // (every page at most once: no more than n_seqs * pages_per_seq)
  struct Claim {
    int i, at, page, refs;
  };
  auto claim = [&](int c) {
    Claim k;
    int lo = 0, hi = n - 1;
    while (lo < hi) {   // last entry whose first claim is not behind c
      const int mid = (lo + hi + 1) >> 1;
      if (first[mid] <= c) lo = mid; else hi = mid - 1;
    }
    k.i = lo;
    k.at = page0[lo] + c - first[lo];
    k.page = p.table[(size_t)seq_of[lo] * p.pages_per_seq + k.at];
    k.refs = 0;
    if (k.page >= 0 && k.page < p.n_pages) k.refs = p.refs[k.page];
    return k;
  };
  // Of a page that several claims of this call share, the last one may keep it, and does if no other holder is left then: with r
  // holders and c claims on it that is c == r.  claims[page]: their count, to[page]: the last one's number.
  bool any_shared = false;
  for (int c = tid; c < n_claims; c += kPlanThreads) {
    const Claim k = claim(c);
    if (k.page >= p.n_pages || (k.page >= 0 && k.refs < 1)) bad = true;
    else if (k.refs > 1) {
      ps.claims[k.page] = 0;
      ps.to[k.page] = -1;
      any_shared = true;
    }
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) pool_fault(p.status, SJD_ERR_BAD_ARG);
    return;
  }
  any_shared = __syncthreads_or(any_shared) != 0;
  if (any_shared) {
    for (int c = tid; c < n_claims; c += kPlanThreads) {
      const Claim k = claim(c);
      if (k.refs > 1) {
        atomicAdd(&ps.claims[k.page], 1);
        atomicMax(&ps.to[k.page], c);
      }
    }
    __syncthreads();
  }
  auto needs = [&](const Claim &k, int c) {
    if (k.page < 0) return true;
    if (k.refs <= 1) return false;
    return !(__ldcg(&ps.claims[k.page]) == k.refs && __ldcg(&ps.to[k.page]) == c);
  };
  int needed = 0;
  for (int c0 = 0; c0 < n_claims; c0 += kPlanThreads) {
    const int c = c0 + tid;
    bool need = false;
    if (c < n_claims) need = needs(claim(c), c);
    needed += __syncthreads_count(need);
  }
  if (needed == 0) return;
  // the free pages, lowest index first, as many as are needed
  int found = 0;
  for (int q0 = 0; q0 < p.n_pages && found < needed; q0 += kPlanThreads * 4) {
    const int q = q0 + tid * 4;
    int r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = q + j < p.n_pages ? p.refs[q + j] : 1;
    int total;
    int at = found + block_number4((r[0] == 0) + (r[1] == 0) + (r[2] == 0) + (r[3] == 0), warp_sums, &total);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (r[j] == 0) {
        if (at < needed) ps.free_list[at] = q + j;
        ++at;
      }
    found += total;
  }
  if (found < needed) {
    if (tid == 0) pool_fault(p.status, SJD_ERR_CAPACITY);
    return;
  }
  __syncthreads();
  int base = 0;
  for (int c0 = 0; c0 < n_claims; c0 += kPlanThreads) {
    const int c = c0 + tid;
    Claim k;
    k.page = -1;
    bool need = false;
    if (c < n_claims) {
      k = claim(c);
      need = needs(k, c);
    }
    int total;
    const int no = base + block_number(need, warp_sums, &total);
    if (need) {
      const int got = ps.free_list[no];
      p.table[(size_t)seq_of[k.i] * p.pages_per_seq + k.at] = got;
      ps.old[no] = k.page;
      if (k.page >= 0 && (long)k.at * KV_PAGE < begin_of[k.i]) {
        const int j = atomicAdd(&copies, 1);
        ps.src[j] = k.page;
        ps.dst[j] = got;
      }
    }
    base += total;
  }
  __syncthreads();
  // holders: not before all claims have been read against the counts as they were
  for (int i = tid; i < needed; i += kPlanThreads) {
    p.refs[ps.free_list[i]] = 1;
    if (ps.old[i] >= 0) atomicSub(&p.refs[ps.old[i]], 1);
  }
  if (tid == 0) *ps.count = copies;
  if (copy_here) {   // few bytes: a launch less
    for (int i = 0; i < copies; ++i) {
      const uint4 *src = reinterpret_cast<const uint4 *>((const char *)p.pages + (size_t)ps.src[i] * page_bytes);
      uint4 *dst = reinterpret_cast<uint4 *>((char *)p.pages + (size_t)ps.dst[i] * page_bytes);
#pragma unroll 4
      for (size_t j = tid; j < page_bytes / 16; j += kPlanThreads) dst[j] = src[j];
      const int32_t *es = reinterpret_cast<const int32_t *>(p.exps + (size_t)ps.src[i] * page_exps);
      int32_t *ed = reinterpret_cast<int32_t *>(p.exps + (size_t)ps.dst[i] * page_exps);
      for (int j = tid; j < (int)(page_exps / 4); j += kPlanThreads) ed[j] = es[j];
    }
  }
}

// pages src[i] -> dst[i], i < *count, in pieces of 16 KB (all of a thread's loads in flight before its stores); REMAP: tables first
template <bool REMAP>
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(sjd_pool p, PlanScratch ps, size_t page_bytes, size_t page_exps) {
  pdl_trigger();
  pdl_wait();
  if (REMAP) {
    const int in_use = ps.count[1];
    const size_t n = (size_t)p.n_seqs * p.pages_per_seq;
    for (size_t i = (size_t)blockIdx.x * kCopyThreads + threadIdx.x; in_use >= 0 && i < n; i += (size_t)gridDim.x * kCopyThreads) {
      const int page = p.table[i];
      if (page >= in_use && page < p.n_pages) p.table[i] = ps.to[page];
    }
  }
  constexpr int PER = 4;
  constexpr size_t PIECE = (size_t)kCopyThreads * PER * 16;
  const int count = *ps.count;
  const int per_page = (int)((page_bytes + PIECE - 1) / PIECE);
  for (long w = blockIdx.x; w < (long)count * per_page; w += gridDim.x) {
    const int i = (int)(w / per_page), piece = (int)(w - (long)i * per_page);
    const size_t from = (size_t)ps.src[i], to = (size_t)ps.dst[i];
    const char *src = (const char *)p.pages + from * page_bytes;
    char *dst = (char *)p.pages + to * page_bytes;
    uint4 v[PER];
    const size_t at = piece * PIECE + threadIdx.x * 16;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (at + j * (kCopyThreads * 16) < page_bytes) v[j] = __ldcs(reinterpret_cast<const uint4 *>(src + at + j * (kCopyThreads * 16)));
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (at + j * (kCopyThreads * 16) < page_bytes) __stcs(reinterpret_cast<uint4 *>(dst + at + j * (kCopyThreads * 16)), v[j]);
    if (piece == 0) {
      const int32_t *es = reinterpret_cast<const int32_t *>(p.exps + from * page_exps);
      int32_t *ed = reinterpret_cast<int32_t *>(p.exps + to * page_exps);
      for (int j = threadIdx.x; j < (int)(page_exps / 4); j += kCopyThreads) ed[j] = es[j];
    }
  }
}

__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(sjd_pool p, PlanScratch ps) {
  __shared__ int warp_sums[32];
  const int tid = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  if (tid == 0) {
    ps.count[0] = 0;
    ps.count[1] = -1;
  }
  const bool off = *(volatile int32_t *)p.status != 0;
  if (__syncthreads_or(off)) return;
  int live = 0;
  for (int q = tid; q < p.n_pages; q += kPlanThreads) live += p.refs[q] > 0;
  live = __reduce_add_sync(0xffffffffu, live);
  if ((tid & 31) == 0) warp_sums[tid >> 5] = live;
  __syncthreads();
  const int in_use = __reduce_add_sync(0xffffffffu, warp_sums[tid & 31]);
  // holes below in_use, pages in use from there on: as many of one as of the other
  int holes = 0, movers = 0;
  for (int q0 = 0; q0 < p.n_pages; q0 += kPlanThreads * 4) {
    const int q = q0 + tid * 4;
    bool f[4];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool used = q + j < p.n_pages && p.refs[q + j] > 0;
      f[j] = q + j < in_use ? !used : used;
      mine += f[j];
      if (q + j >= in_use && q + j < p.n_pages) ps.to[q + j] = q + j;
    }
    const int below = max(0, min(4, in_use - q));   // of the thread's four, how many lie below in_use
    int hole = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) hole += j < below && f[j];
    int n_holes, n_movers;
    int at_h = holes + block_number4(hole, warp_sums, &n_holes), at_m = movers + block_number4(mine - hole, warp_sums, &n_movers);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (!f[j]) continue;
      if (j < below) ps.dst[at_h++] = q + j;
      else ps.src[at_m++] = q + j;
    }
    holes += n_holes;
    movers += n_movers;
  }
  __syncthreads();
  for (int i = tid; i < movers; i += kPlanThreads) {
    const int from = ps.src[i], to = ps.dst[i];
    ps.to[from] = to;
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (tid == 0) {
    ps.count[0] = movers;
    ps.count[1] = in_use;
  }
}

// a block for each (source, child)
__global__ void __launch_bounds__(kCopyThreads) fork_check_kernel(sjd_pool p, int n, const int32_t *__restrict__ src,
                                                                  const int32_t *__restrict__ dst, const int32_t *__restrict__ len) {
  extern __shared__ uint32_t seen[];
  pdl_trigger();
  pdl_wait();
  bool bad = list_bad(dst, n, p.n_seqs, seen);
  if (!bad) {
    const int i = blockIdx.x, s = src[i], l = len[i];
    if (s < 0 || s >= p.n_seqs || l < 0 || l > (long)p.pages_per_seq * KV_PAGE) bad = true;
    else if (seen[s >> 5] >> (s & 31) & 1u) bad = true;
    else {
      const int32_t *from = p.table + (size_t)s * p.pages_per_seq, *to = p.table + (size_t)dst[i] * p.pages_per_seq;
      const int pages = (int)(((long)l + KV_PAGE - 1) / KV_PAGE);
      for (int j = threadIdx.x; j < p.pages_per_seq; j += kCopyThreads) {
        if (to[j] != -1) bad = true;
        if (j < pages && (from[j] < 0 || from[j] >= p.n_pages)) bad = true;
      }
    }
  }
  if (__syncthreads_or(bad) && threadIdx.x == 0) pool_fault(p.status, SJD_ERR_BAD_ARG);
}
__global__ void __launch_bounds__(kCopyThreads) fork_kernel(sjd_pool p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                            const int32_t *__restrict__ len) {
  pdl_trigger();
  pdl_wait();
  if (*(volatile int32_t *)p.status != 0) return;   // (what the check found, or an older fault)
  const int i = blockIdx.x, pages = (int)(((long)len[i] + KV_PAGE - 1) / KV_PAGE);
  const int32_t *from = p.table + (size_t)src[i] * p.pages_per_seq;
  int32_t *to = p.table + (size_t)dst[i] * p.pages_per_seq;
  for (int j = threadIdx.x; j < pages; j += kCopyThreads) {
    const int page = from[j];
    to[j] = page;
    atomicAdd(&p.refs[page], 1);
  }
}

// the same in one block, for lists and tables of few entries
__global__ void __launch_bounds__(kPlanThreads) fork_one_kernel(sjd_pool p, int n, const int32_t *__restrict__ src,
                                                                const int32_t *__restrict__ dst, const int32_t *__restrict__ len) {
  extern __shared__ uint32_t seen[];
  pdl_trigger();
  pdl_wait();
  bool bad = *(volatile int32_t *)p.status != 0;
  if (__syncthreads_or(bad)) return;
  bad = list_bad(dst, n, p.n_seqs, seen);
  for (int i = threadIdx.x; !bad && i < n; i += kPlanThreads) {
    const int s = src[i], l = len[i];
    bad = s < 0 || s >= p.n_seqs || l < 0 || l > (long)p.pages_per_seq * KV_PAGE || (seen[s >> 5] >> (s & 31) & 1u);
  }
  bad = __syncthreads_or(bad) != 0;
  const int all = n * p.pages_per_seq;
  if (!bad) {
    for (int x = threadIdx.x; x < all; x += kPlanThreads) {
      const int i = x / p.pages_per_seq, j = x - i * p.pages_per_seq;
      const int from = j * KV_PAGE < len[i] ? p.table[(size_t)src[i] * p.pages_per_seq + j] : 0;
      bad |= p.table[(size_t)dst[i] * p.pages_per_seq + j] != -1 || from < 0 || from >= p.n_pages;
    }
    bad = __syncthreads_or(bad) != 0;
  }
  if (bad) {
    if (threadIdx.x == 0) pool_fault(p.status, SJD_ERR_BAD_ARG);
    return;
  }
  for (int x = threadIdx.x; x < all; x += kPlanThreads) {
    const int i = x / p.pages_per_seq, j = x - i * p.pages_per_seq;
    if (j * KV_PAGE >= len[i]) continue;
    const int page = p.table[(size_t)src[i] * p.pages_per_seq + j];
    p.table[(size_t)dst[i] * p.pages_per_seq + j] = page;
    atomicAdd(&p.refs[page], 1);
  }
}

// a block for each sequence; every block sees from the list alone whether the call is refused
__global__ void __launch_bounds__(kCopyThreads) free_kernel(sjd_pool p, int n, const int32_t *__restrict__ seqs, const int32_t *__restrict__ keep) {
  extern __shared__ uint32_t seen[];
  pdl_trigger();
  pdl_wait();
  const bool off = *(volatile int32_t *)p.status != 0;
  if (__syncthreads_or(off)) return;
  bool bad = list_bad(seqs, n, p.n_seqs, seen);
  for (int i = threadIdx.x; i < n; i += kCopyThreads) bad |= keep[i] < 0;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) pool_fault(p.status, SJD_ERR_BAD_ARG);
    return;
  }
  const int i = blockIdx.x;
  int32_t *row = p.table + (size_t)seqs[i] * p.pages_per_seq;
  for (long j = ((long)keep[i] + KV_PAGE - 1) / KV_PAGE + threadIdx.x; j < p.pages_per_seq; j += kCopyThreads) {
    const int page = row[j];
    if (page < 0) continue;
    row[j] = -1;
    if (page < p.n_pages) atomicSub(&p.refs[page], 1);
  }
}

struct PdlScope {   // launches of a call wait on one another themselves
  PdlScope() { g_pdl = true; }
  ~PdlScope() { g_pdl = false; }
};
int sm_count(int *sms) {
  int dev = 0;
  SJD_CUDA(cudaGetDevice(&dev));
  SJD_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  return SJD_OK;
}
size_t seen_bytes(const sjd_pool &p) { return (size_t)(p.n_seqs + 31) / 32 * 4; }

template <bool REMAP>
int launch_copies(const sjd_pool &p, const PlanScratch &ps, long most, cudaStream_t stream) {
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc != SJD_OK) return rc;
  const size_t bytes = pool_page_bytes(p);
  long blocks = most * (long)((bytes + kCopyThreads * 64 - 1) / (kCopyThreads * 64));
  blocks = blocks < 8L * sms ? blocks : 8L * sms;
  SJD_CUDA(launch_kernel(copy_pages_kernel<REMAP>, dim3((unsigned)(blocks > 0 ? blocks : 1)), dim3(kCopyThreads), 0, stream, p, ps, bytes,
                         pool_page_exps(p)));
  SJD_CHECK_LAUNCH();
  return SJD_OK;
}

}  // namespace

int check_pool(const sjd_pool *p, bool with_refs) {
  if (!p || !p->pages || !p->exps || !p->table || !p->status || (with_refs && !p->refs)) return SJD_ERR_BAD_ARG;
  if (p->n_pages < 1 || p->n_seqs < 1 || p->pages_per_seq < 1 || p->n_layers < 1 || p->n_kv_heads < 1) return SJD_ERR_BAD_ARG;
  if (((uintptr_t)p->pages & 15u) != 0 || ((uintptr_t)p->exps & 3u) != 0) return SJD_ERR_BAD_ARG;
  if ((((uintptr_t)p->table | (uintptr_t)p->refs | (uintptr_t)p->status) & 3u) != 0) return SJD_ERR_BAD_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return SJD_ERR_UNSUPPORTED;
  // (counts and positions stay in 32 bits)
  if (p->pages_per_seq > 1 << 20 || p->n_seqs > 1 << 17 || p->n_pages > 1 << 30 || (long)p->n_layers * p->n_kv_heads > 1 << 20)
    return SJD_ERR_CAPACITY;
  return SJD_OK;
}

}  // namespace sjd

using namespace sjd;

extern "C" size_t sjd_pool_workspace_bytes(const sjd_pool *pool) { return check_pool(pool, true) == SJD_OK ? scratch_bytes(pool->n_pages) : 0; }

extern "C" int sjd_pool_reserve(const sjd_pool *pool, int n, const int32_t *seqs, const int32_t *begin, const int32_t *end, void *ws,
                                size_t ws_bytes, void *cuda_stream) {
  const int rc = check_pool(pool, true);
  if (rc != SJD_OK) return rc;
  if (n < 0 || (n > 0 && (!seqs || !begin || !end)) || !ws || ((uintptr_t)ws & 255u) != 0) return SJD_ERR_BAD_ARG;
  if (n > kListMax || ws_bytes < scratch_bytes(pool->n_pages)) return SJD_ERR_CAPACITY;
  if (n == 0) return SJD_OK;
  const PlanScratch ps = scratch_of(ws, pool->n_pages);
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  PdlScope pdl;
  const int copy_here = (size_t)n * pool_page_bytes(*pool) <= kCopyHere;
  SJD_CUDA(launch_kernel(reserve_plan_kernel, dim3(1), dim3(kPlanThreads), seen_bytes(*pool), stream, *pool, n, seqs, begin, end, ps,
                         pool_page_bytes(*pool), pool_page_exps(*pool), copy_here));
  SJD_CHECK_LAUNCH();
  if (copy_here) return SJD_OK;
  return launch_copies<false>(*pool, ps, n, stream);   // (only the page in which an entry begins can have positions before it)
}

extern "C" int sjd_pool_fork(const sjd_pool *pool, int n, const int32_t *src, const int32_t *dst, const int32_t *len, void *cuda_stream) {
  const int rc = check_pool(pool, true);
  if (rc != SJD_OK) return rc;
  if (n < 0 || (n > 0 && (!src || !dst || !len))) return SJD_ERR_BAD_ARG;
  if (n > kListMax) return SJD_ERR_CAPACITY;
  if (n == 0) return SJD_OK;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  PdlScope pdl;
  if ((int64_t)n * pool->pages_per_seq <= kForkHere) {
    SJD_CUDA(launch_kernel(fork_one_kernel, dim3(1), dim3(kPlanThreads), seen_bytes(*pool), stream, *pool, n, src, dst, len));
    SJD_CHECK_LAUNCH();
    return SJD_OK;
  }
  SJD_CUDA(launch_kernel(fork_check_kernel, dim3(n), dim3(kCopyThreads), seen_bytes(*pool), stream, *pool, n, src, dst, len));
  SJD_CHECK_LAUNCH();
  SJD_CUDA(launch_kernel(fork_kernel, dim3(n), dim3(kCopyThreads), 0, stream, *pool, src, dst, len));
  SJD_CHECK_LAUNCH();
  return SJD_OK;
}

extern "C" int sjd_pool_free(const sjd_pool *pool, int n, const int32_t *seqs, const int32_t *keep, void *cuda_stream) {
  const int rc = check_pool(pool, true);
  if (rc != SJD_OK) return rc;
  if (n < 0 || (n > 0 && (!seqs || !keep))) return SJD_ERR_BAD_ARG;
  if (n > kListMax) return SJD_ERR_CAPACITY;
  if (n == 0) return SJD_OK;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  PdlScope pdl;
  SJD_CUDA(launch_kernel(free_kernel, dim3(n), dim3(kCopyThreads), seen_bytes(*pool), stream, *pool, n, seqs, keep));
  SJD_CHECK_LAUNCH();
  return SJD_OK;
}

extern "C" int sjd_pool_compact(const sjd_pool *pool, void *ws, size_t ws_bytes, void *cuda_stream) {
  const int rc = check_pool(pool, true);
  if (rc != SJD_OK) return rc;
  if (!ws || ((uintptr_t)ws & 255u) != 0) return SJD_ERR_BAD_ARG;
  if (ws_bytes < scratch_bytes(pool->n_pages)) return SJD_ERR_CAPACITY;
  const PlanScratch ps = scratch_of(ws, pool->n_pages);
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  PdlScope pdl;
  SJD_CUDA(launch_kernel(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, *pool, ps));
  SJD_CHECK_LAUNCH();
  const long most = pool->n_pages / 2 > 0 ? pool->n_pages / 2 : 1;
  return launch_copies<true>(*pool, ps, most, stream);
}
