// Page tables and slot maps from request lengths: what a scheduling step does to block_table, the free list and the
// rows' slots, without the lengths ever visiting the host.
//
// reserve: need[s] = max(0, ceil((L + n) / page) - held); with E the exclusive prefix sum of need over the sequences,
//   the page at place held + i of sequence s has rank E[s] + i and is free_list[n_free - 1 - rank].
// release: first[s] = min(held, ceil(keep / page)); with E the prefix sum of held - first and T its total, the page at
//   place first + i goes to free_list[n_free + T - 1 - (E[s] + i)]: the stack then hands the same pages out again in
//   the same order.
// A sequence whose numbers are out of range (a negative length, held beyond the table) is refused: nothing of it changes.
//
// A few words per page and row: bound by latency (dependent trips to L2), not by bytes (release and reserve of a round at
// batch 32: 8.9 us on the device; admission of 64 prompts with 60,000 row slots: 12.6 us). One launch: every block
// computes the prefix sums of the whole batch for itself from unchanged inputs (S words) and fills its share of the
// pages and rows; the block that finishes last, known by a ticket, writes held, n_free and the lengths, which all the
// others have read by then. Sizes the blocks cannot know (the total of the needs) only bound loops.
#include "cod_internal.cuh"

namespace {

constexpr int PT = 256;                 // threads
constexpr int S_MAX = 4096;             // sequences: three words each in shared memory

struct PagesArgs {
  const int* len_in;          // n_new (reserve) or keep (release; null: committed_len)
  int* block_table;
  int* committed_len;
  int* carry_len;
  int* carry_hist;            // may be null
  int *free_list, *n_free, *held;
  int S, page, max_pages, n_pages, hist_len, advance;
  int *row_off, *slot, *row_pos, *row_seq;
  int max_rows;
  unsigned int* ticket;       // [0] blocks that are done, [1] release: a table held something that is no page
  uint32_t* status;
};

// Exclusive prefix sum over the block of one value per thread; total in every thread.
__device__ __forceinline__ long long block_scan(long long v, long long* red, long long& total) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                      // red may still be read by the previous call
  if (lane == 31) red[wid] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < PT / 32; ++w) {
    const long long t = red[w];
    if (w < wid) before += t;
    all += t;
  }
  total = all;
  return before + x - v;
}

// number of entries of off[0..S) that are <= v, minus one: the sequence that owns element v (off[0] = 0, v below the total)
__device__ __forceinline__ int owner(const int* off, int S, int v) {
  int lo = 0, hi = S;                   // off[lo] <= v; every entry from hi on is > v
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= v) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ bool last_block(unsigned int* ticket) {
  __shared__ bool last;
  __threadfence();                      // this block's reads and writes are done before its ticket counts
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  return last;
}

__global__ void __launch_bounds__(PT) k_pages_reserve(const PagesArgs a) {
  cod_pdl_prologue();
  extern __shared__ int sm[];
  __shared__ long long red[PT / 32];
  int* pfx = sm;                        // [S] rank of the sequence's first new page
  int* hold = sm + a.S;                 // [S] pages held before the call; bit 30 set: refused
  int* roff = sm + 2 * a.S;             // [S] its first row
  constexpr int REFUSED = 1 << 30;
  uint32_t flags = 0;
  int nf = *a.n_free;
  const bool list_ok = nf >= 0 && nf <= a.n_pages;       // else nothing is handed out and n_free stays
  if (!list_ok) { flags |= COD_DEV_BAD_LEN; nf = 0; }
  long long pages_before = 0, rows_before = 0;
  int granted = 0;                      // pages handed out to the sequences so far
  for (int s0 = 0; s0 < a.S; s0 += PT) {
    const int s = s0 + threadIdx.x;
    long long need = 0, n = 0;
    int h = 0;
    bool refused = false;
    if (s < a.S) {
      const int L = a.committed_len[s];
      n = a.len_in[s];
      h = a.held[s];
      if (n < 0) { flags |= COD_DEV_BAD_LEN; n = 0; refused = true; }
      if (h < 0 || h > a.max_pages) { flags |= COD_DEV_BAD_LEN; h = max(0, min(h, a.max_pages)); refused = true; }
      const long long end = L + n, cap = min(static_cast<long long>(a.max_pages) * a.page, 0x7FFFFFFFll - a.page);
      if (L < 0) { flags |= COD_DEV_BAD_LEN; refused = true; }
      else if (end > cap) { flags |= COD_DEV_PAGE_OVERFLOW; refused = true; }
      if (!refused) need = max(0ll, (end + a.page - 1) / a.page - h);
    }
    long long tot_p, tot_r;
    const long long ep = pages_before + block_scan(need, red, tot_p);
    const long long er = rows_before + block_scan(n, red, tot_r);
    pages_before += tot_p;
    rows_before += tot_r;
    int got = 0;
    if (s < a.S) {
      if (need > 0 && ep + need > nf) { flags |= COD_DEV_NO_PAGES; refused = true; }
      else if (!refused) got = static_cast<int>(need);
      // the served sequences with a need come before the first one refused for want of pages, so ranks below the
      // total of what is handed out are exactly theirs
      pfx[s] = static_cast<int>(min(ep, static_cast<long long>(nf)));
      hold[s] = h | (refused ? REFUSED : 0);
      roff[s] = static_cast<int>(min(er, 0x7FFFFFFFll));
    }
    long long tot_g;
    block_scan(got, red, tot_g);
    granted += static_cast<int>(tot_g);
  }
  __syncthreads();
  const int rows = static_cast<int>(min(rows_before, 0x7FFFFFFFll));
  if (rows > a.max_rows && a.slot != nullptr) flags |= COD_DEV_BAD_LEN;
  const int tid = blockIdx.x * PT + threadIdx.x, nt = gridDim.x * PT;
  auto page_of = [&](int rank) -> int {
    const int pg = a.free_list[nf - 1 - rank];
    if (pg < 0 || pg >= a.n_pages) { flags |= COD_DEV_BAD_PAGE; return -1; }
    return pg;
  };
  for (long long at = tid; at < granted; at += nt) {
    const int r = static_cast<int>(at);
    // sequences without a need share their rank with the next one: the last of equals owns it, unless it was refused
    int s = owner(pfx, a.S, r);
    a.block_table[static_cast<size_t>(s) * a.max_pages + (hold[s] & ~REFUSED) + (r - pfx[s])] = page_of(r);
  }
  if (a.slot != nullptr) {
    for (long long at = tid; at < a.max_rows; at += nt) {
      const int r = static_cast<int>(at);
      int sl = -1, pos = -1, sq = -1;
      if (r < rows) {
        sq = owner(roff, a.S, r);
        const int L = a.committed_len[sq], h = hold[sq];
        pos = static_cast<int>(min(L + static_cast<long long>(r - roff[sq]), 0x7FFFFFFFll));   // (beyond it: a refused sequence's)
        if (!(h & REFUSED)) {
          const int place = pos / a.page;
          const int pg = place < h ? a.block_table[static_cast<size_t>(sq) * a.max_pages + place] : page_of(pfx[sq] + place - h);
          if (pg < 0 || pg >= a.n_pages) flags |= COD_DEV_BAD_PAGE;
          else sl = pg * a.page + pos % a.page;
        }
      }
      a.slot[r] = sl;
      if (a.row_pos) a.row_pos[r] = pos;
      if (a.row_seq) a.row_seq[r] = sq;
    }
    for (int s = tid; s <= a.S; s += nt) a.row_off[s] = s < a.S ? roff[s] : rows;
  }
  if (flags) atomicOr(a.status, flags);
  if (!last_block(a.ticket)) return;
  for (int s = threadIdx.x; s < a.S; s += PT) {
    const int h = hold[s];
    if (h & REFUSED) continue;
    const int L = a.committed_len[s], n = a.len_in[s];
    const int want = (L + n + a.page - 1) / a.page;
    if (want > h) a.held[s] = want;
    if (a.advance) a.committed_len[s] = L + n;
  }
  if (threadIdx.x == 0) {
    if (list_ok) *a.n_free = nf - granted;
    *a.ticket = 0;
  }
}

__global__ void __launch_bounds__(PT) k_pages_release(const PagesArgs a) {
  cod_pdl_prologue();
  extern __shared__ int sm[];
  __shared__ long long red[PT / 32];
  int* pfx = sm;                        // [S] rank of the first page that goes
  int* first = sm + a.S;                // [S] its place in the table; -1: refused
  uint32_t flags = 0;
  int nf = *a.n_free;
  const bool list_ok = nf >= 0 && nf <= a.n_pages;       // else every sequence is refused
  if (!list_ok) { flags |= COD_DEV_BAD_LEN; nf = 0; }
  long long before = 0;
  for (int s0 = 0; s0 < a.S; s0 += PT) {
    const int s = s0 + threadIdx.x;
    long long gone = 0;
    int f = -1;
    if (s < a.S) {
      const int L = a.committed_len[s], keep = a.len_in ? a.len_in[s] : L, h = a.held[s];
      if (L < 0 || keep < 0 || h < 0 || h > a.max_pages) flags |= COD_DEV_BAD_LEN;
      else if (list_ok) {
        f = min(h, keep / a.page + (keep % a.page ? 1 : 0));
        gone = h - f;
      }
    }
    long long tot;
    const long long e = before + block_scan(gone, red, tot);
    before += tot;
    if (s < a.S) { pfx[s] = static_cast<int>(e); first[s] = f; }      // S_MAX * max_pages is below 2^31 (the host checks)
  }
  __syncthreads();
  const int total = static_cast<int>(before);
  const int tid = blockIdx.x * PT + threadIdx.x, nt = gridDim.x * PT;
  bool hole = false;
  for (long long r = tid; r < total; r += nt) {          // (table and list may each hold 2^31 - 1 entries)
    const int s = owner(pfx, a.S, static_cast<int>(r));
    int* e = a.block_table + static_cast<size_t>(s) * a.max_pages + first[s] + (r - pfx[s]);
    const int pg = *e;
    const long long at = nf + static_cast<long long>(total) - 1 - r;
    if (pg < 0 || pg >= a.n_pages) { flags |= COD_DEV_BAD_PAGE; hole = true; }
    if (at < a.n_pages) a.free_list[at] = pg; else flags |= COD_DEV_BAD_PAGE;    // more pages than there are: some came twice
    *e = -1;
  }
  if (hole) atomicOr(a.ticket + 1, 1u);
  if (flags) atomicOr(a.status, flags);
  if (!last_block(a.ticket)) return;
  int top = static_cast<int>(min(nf + static_cast<long long>(total), static_cast<long long>(a.n_pages)));
  if (*static_cast<volatile unsigned int*>(a.ticket + 1)) {   // what is no page does not stay on the list: one warp closes the gaps
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      int to = nf;
      for (long long i = nf; i < top; i += 32) {
        const int pg = i + lane < top ? *static_cast<volatile int*>(a.free_list + i + lane) : -1;
        const bool is_page = pg >= 0 && pg < a.n_pages;
        const unsigned m = __ballot_sync(0xffffffffu, is_page);         // (every lane has read before one writes: the places it
        if (is_page) a.free_list[to + __popc(m & ((1u << lane) - 1u))] = pg;      // writes lie at or below those of this step)
        to += __popc(m);
        __syncwarp();
      }
      top = to;
    }
  }
  for (int s = threadIdx.x; s < a.S; s += PT) {
    if (first[s] < 0) continue;
    const int keep = a.len_in ? a.len_in[s] : 0x7FFFFFFF, L = a.committed_len[s];
    a.held[s] = first[s];
    if (keep < L || keep == 0) {        // (a request of no tokens that ends may have carried rows, too)
      a.committed_len[s] = keep;
      a.carry_len[s] = 0;
      if (a.carry_hist) for (int j = 0; j < a.hist_len; ++j) a.carry_hist[static_cast<size_t>(s) * a.hist_len + j] = 0;
    }
  }
  if (threadIdx.x == 0) {
    if (list_ok) *a.n_free = top;
    a.ticket[0] = 0;
    a.ticket[1] = 0;
  }
}

PagesArgs common_args(cod_ctx* c, const cod_pages* pages, const int32_t* len_in, int S, const cod_state* st) {
  const cod_config& f = c->cfg;
  PagesArgs a{};
  a.len_in = len_in;
  a.block_table = st->block_table; a.committed_len = st->committed_len; a.carry_len = st->carry_len;
  a.carry_hist = c->carry_cap > f.block ? st->carry_hist : nullptr;
  a.hist_len = c->carry_cap / f.block;
  a.free_list = pages->free_list; a.n_free = pages->n_free; a.held = pages->held;
  a.S = S; a.page = f.page_size; a.max_pages = f.max_pages_per_seq; a.n_pages = f.n_pages;
  a.ticket = c->pages_ticket; a.status = c->status;
  return a;
}

// blocks for `items` pages or rows at most: one a thread, two blocks per SM at most (a row's slot is a chain of dependent reads;
// admission of 64 prompts: 12.6 us; when it took 11.6, one block per SM took 13.9, four rows a thread 15.8)
int blocks_for(const cod_ctx* c, long long items) {
  const long long b = (items + PT - 1) / PT;
  return static_cast<int>(b < 1 ? 1 : b > 2 * c->n_sm ? 2 * c->n_sm : b);
}

}  // namespace

bool cod_pages_fit(const cod_ctx* c, int S) {
  return S <= S_MAX && c->cfg.max_pages_per_seq < (1 << 30) && static_cast<long long>(S) * c->cfg.max_pages_per_seq < (1ll << 31);
}

int cod_launch_pages_reserve(cod_ctx* c, const cod_pages* pages, const int32_t* n_new, int S, const cod_state* st,
                             const cod_row_plan* plan, int advance, cudaStream_t stream) {
  ProfScope prof(c, COD_K_VERIFY, stream);
  PagesArgs a = common_args(c, pages, n_new, S, st);
  a.advance = advance;
  if (plan) { a.row_off = plan->row_off; a.slot = plan->slot; a.row_pos = plan->row_pos; a.row_seq = plan->row_seq; a.max_rows = plan->max_rows; }
  // with a plan the rows bound the new pages; without one the free list and the tables do
  const long long table = static_cast<long long>(S) * c->cfg.max_pages_per_seq;
  const long long pages_most = table < c->cfg.n_pages ? table : c->cfg.n_pages;
  const long long items = plan ? a.max_rows : pages_most;
  const size_t smem = 3 * sizeof(int) * S;
  if (smem > 40 * 1024 && cudaFuncSetAttribute(k_pages_reserve, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * sizeof(int) * S_MAX) != cudaSuccess)
    return COD_ERR_CUDA;
  cod_launch_pdl(c, k_pages_reserve, blocks_for(c, items), PT, smem, stream, a);
  COD_CHECK_LAUNCH(c);
  return COD_OK;
}

int cod_launch_pages_release(cod_ctx* c, const cod_pages* pages, const int32_t* keep, int S, const cod_state* st, cudaStream_t stream) {
  ProfScope prof(c, COD_K_VERIFY, stream);
  const PagesArgs a = common_args(c, pages, keep, S, st);
  const long long table = static_cast<long long>(S) * c->cfg.max_pages_per_seq;
  const long long items = table < c->cfg.n_pages ? table : c->cfg.n_pages;
  cod_launch_pdl(c, k_pages_release, blocks_for(c, items), PT, 2 * sizeof(int) * S, stream, a);
  COD_CHECK_LAUNCH(c);
  return COD_OK;
}
