// Tables of a decoding step from the requests' lengths: pages change hands between the requests and the pool, then
// row offsets, page lists, positions and slots.
//
// Bound by latency: a served batch moves some kilobytes.  The page exchange is a prefix sum over the requests (who gives and
// takes how much decides where on the stack), so one work-group does it, 1024 requests at a time; the lists are
// independent of each other once the sums stand.
#include "fd_common.h"

namespace fd {

constexpr int TB_BLOCK = 1024;            // threads that exchange pages, a request each
constexpr int TB_WAVES = TB_BLOCK / FD_WAVE;
constexpr int TB_SMALL = 16384;           // lists, positions and slots up to which the same work-group writes them too

// What request i asks for, clamped so that nothing derived from it leaves the arrays.
struct Request { int kv, k, m, need, held; uint32_t bad; };
__device__ __forceinline__ Request load_request(const fd_table_args& a, int i) {
  Request r;
  int kv = a.kv_len[i], k = a.verify_len[i], m = a.mask_rows ? a.mask_rows[i] : 0, held = a.table_len[i];
  r.bad = 0;
  if (kv < 0 || kv > (1 << 30)) r.bad |= FD_DEV_KV_LEN_RANGE;
  if (k < 0 || m < 0 || k > a.total_rows || m > a.total_rows) r.bad |= FD_DEV_ROWS_RANGE;
  if (held < 0 || held > a.table_stride) r.bad |= FD_DEV_PAGE_RANGE;
  r.kv = clampi(kv, 0, 1 << 30);
  r.k = clampi(k, 0, a.total_rows);
  r.m = clampi(m, 0, a.total_rows);
  r.held = clampi(held, 0, a.table_stride);
  const int need = (int)(((unsigned)(r.kv + r.k) + (unsigned)a.page_size - 1u) / (unsigned)a.page_size);
  if (need > a.table_stride) r.bad |= FD_DEV_PAGE_RANGE;
  r.need = need > a.table_stride ? a.table_stride : need;
  return r;
}

// Exclusive prefixes over the work-group and totals of N numbers a thread, in one trip through LDS.  Each is at most 2^20, so 1024 of them sum to
// 2^30 at most, and with the entries of an array (fewer than 2^30) or the rows (2^20) on top to less than 2^31.
template <int N>
__device__ __forceinline__ void block_excl_scan(const int (&x)[N], int (&before)[N], int (&total)[N], int (*sums)[TB_WAVES]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl[N];
#pragma unroll
  for (int n = 0; n < N; ++n) incl[n] = wave_incl_scan(x[n]);
  __syncthreads();                                   // (the last round's sums have been read)
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (lane == 63) sums[n][wave] = incl[n];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int s = wave_incl_scan(lane < TB_WAVES ? sums[n][lane] : 0);
    total[n] = __builtin_amdgcn_readlane(s, TB_WAVES - 1);
    before[n] = incl[n] - x[n] + (wave > 0 ? __builtin_amdgcn_readlane(s, wave - 1) : 0);
  }
}

// Runs too long for one lane, with where they are in the table and on the stack: all waves share them out.
struct LongRuns { int n; int count[TB_BLOCK]; int at[TB_BLOCK]; long long table[TB_BLOCK]; };

// count entries for each thread; every thread calls this.  GIVE: table[from ..] goes to stack[at ..]; else stack[at], stack[at - 1], ... go to
// table[from ..].  A few entries go lane by lane, longer runs (a request that ends gives back some thousand pages) in parts of 1024 to the
// waves in turn, sixteen entries a lane in flight.
template <bool GIVE>
__device__ __forceinline__ void copy_runs(int* table, int* stack, LongRuns& runs, long long from, int at, int count) {
  constexpr int FEW = 4, DEEP = 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (threadIdx.x == 0) runs.n = 0;
  __syncthreads();
  if (count > FEW) {
    const int r = atomicAdd(&runs.n, 1);               // (the order of the list changes nothing: runs do not overlap)
    runs.count[r] = count; runs.at[r] = at; runs.table[r] = from;
  } else if (count > 0) {
    int v[FEW];
#pragma unroll
    for (int j = 0; j < FEW; ++j) { const int k = min(j, count - 1); v[j] = GIVE ? table[from + k] : stack[at - k]; }
#pragma unroll
    for (int j = 0; j < FEW; ++j)
      if (j < count) { if (GIVE) stack[at + j] = v[j]; else table[from + j] = v[j]; }
  }
  __syncthreads();
  const int n = __builtin_amdgcn_readfirstlane(runs.n);
  for (int r0 = 0; r0 < n; r0 += 64) {               // a run a lane, then their parts to the waves
    const bool on = r0 + lane < n;
    const int entries = on ? runs.count[r0 + lane] : 0, where = on ? runs.at[r0 + lane] : 0;
    const long long row = on ? runs.table[r0 + lane] : 0;
    const int parts = (entries + 64 * DEEP - 1) / (64 * DEEP), incl = wave_incl_scan(parts), total = __builtin_amdgcn_readlane(incl, 63);
    for (int p = wave; p < total; p += TB_WAVES) {
      const int l = __ffsll((long long)__ballot(incl > p)) - 1;
      const int e = __builtin_amdgcn_readlane(entries, l), part = (p - __builtin_amdgcn_readlane(incl - parts, l)) * 64 * DEEP;
      const unsigned lo = __builtin_amdgcn_readlane((int)row, l), hi = __builtin_amdgcn_readlane((int)(row >> 32), l);
      int* t = table + (long long)(((unsigned long long)hi << 32) | lo);
      int* s = stack + __builtin_amdgcn_readlane(where, l);
      int v[DEEP];
#pragma unroll
      for (int u = 0; u < DEEP; ++u) { const int k = min(part + 64 * u + lane, e - 1); v[u] = GIVE ? t[k] : s[-k]; }
#pragma unroll
      for (int u = 0; u < DEEP; ++u) {
        const int k = part + 64 * u + lane;
        if (k < e) { if (GIVE) s[k] = v[u]; else t[k] = v[u]; }
      }
    }
  }
  __syncthreads();                                   // (also: what was copied is there for the whole work-group)
}

// Lists, positions and slots of request i, by `threads` threads of which this is number t.
__device__ __forceinline__ void expand_request(const fd_table_args& a, int i, int kv, int k, int m, int row0, int row1, int page0, int page1, int t,
                                               int threads) {
  const int* table = a.block_table + (long long)i * a.table_stride;
  const int pages = page1 - page0;
  for (int j0 = t; j0 < pages; j0 += 8 * threads) {
    int v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = table[min(j0 + u * threads, pages - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (j0 + u * threads < pages) a.page_indices[page0 + j0 + u * threads] = v[u];
  }
  if (!a.positions && !a.slot_map) return;
  int nb = 1;
  if (a.mask_blocks) {
    nb = a.mask_blocks[i];
    if (nb < 1 || m % nb) nb = 1;
  }
  int v = k - nb + 1 < 0 ? 0 : k - nb + 1;
  if (a.mask_vis) v = clampi(a.mask_vis[i], 0, k);
  const int per = m / nb > 0 ? m / nb : 1;
  for (int r = t; r < row1 - row0; r += threads) {
    int pos = kv + r;
    long long slot = -1;
    if (r < k) {
      const int lp = (int)((unsigned)pos / (unsigned)a.page_size);
      if (lp < pages) slot = (long long)table[lp] * a.page_size + (pos - lp * a.page_size);
    } else {
      const int b = (r - k) / per;
      pos = kv + (v + b < k ? v + b : k) + (r - k - b * per);
    }
    if (a.positions) a.positions[row0 + r] = pos;
    if (a.slot_map) a.slot_map[row0 + r] = slot;
  }
}

template <bool EXPAND>
__global__ __launch_bounds__(TB_BLOCK) void step_tables_kernel(fd_table_args a) {
  __shared__ int sums[3][TB_WAVES];
  __shared__ LongRuns runs;
  __shared__ int mine[5][EXPAND ? TB_BLOCK + 1 : 1];   // of each request: kv, k, m, first row, first page
  const int tid = threadIdx.x;
  uint32_t bad = 0;
  int count = a.free_count[0];
  const int rounds = (a.batch + TB_BLOCK - 1) / TB_BLOCK;
  Request q = {};
  if (rounds == 1 && tid < a.batch) q = load_request(a, tid);
  if (count < 0 || count > a.free_pages_len) { bad |= FD_DEV_PAGE_RANGE; count = clampi(count, 0, a.free_pages_len); }
  // 1. pages given back go onto the stack; with one round the other sums come along
  int top = count, before1[3] = {}, total1[3] = {};
  for (int c = 0; c < rounds; ++c) {
    const int i = c * TB_BLOCK + tid;
    if (rounds > 1) { q = Request{}; if (i < a.batch) q = load_request(a, i); }
    bad |= q.bad;
    const int give = q.held > q.need ? q.held - q.need : 0;
    const int x[3] = {give, q.need > q.held ? q.need - q.held : 0, min(q.k + q.m, a.total_rows)};
    block_excl_scan(x, before1, total1, sums);
    const int at = top + before1[0];
    int n = give;
    if (at + n > a.free_pages_len) { n = at < a.free_pages_len ? a.free_pages_len - at : 0; bad |= FD_DEV_PAGE_RANGE; }
    if (total1[0] > 0) copy_runs<true>(a.block_table, a.free_pages, runs, (long long)i * a.table_stride + q.need, at, n);
    top = min(top + total1[0], a.free_pages_len);
  }
  // 2. pages are taken from its top (copy_runs ended with a barrier: the stack is whole); 3. the prefix sums
  int left = top, rows0 = 0, pages0 = 0;
  for (int c = 0; c < rounds; ++c) {
    const int i = c * TB_BLOCK + tid;
    if (rounds > 1) {
      q = Request{};
      if (i < a.batch) q = load_request(a, i);
      const int x[3] = {0, q.need > q.held ? q.need - q.held : 0, min(q.k + q.m, a.total_rows)};
      block_excl_scan(x, before1, total1, sums);
    }
    const int take = q.need > q.held ? q.need - q.held : 0, rows = min(q.k + q.m, a.total_rows);
    const int there = left - before1[1];             // entries of the stack that are there for this request
    const int got = there < take ? (there > 0 ? there : 0) : take;
    if (got < take) bad |= FD_DEV_PAGE_RANGE;
    if (total1[1] > 0) copy_runs<false>(a.block_table, a.free_pages, runs, (long long)i * a.table_stride + q.held, there - 1, got);
    left = left > total1[1] ? left - total1[1] : 0;
    const int have = min(q.held + got, q.need);
    const int y[1] = {have};
    int before2[1], total2[1];
    block_excl_scan(y, before2, total2, sums);
    const int r = min(rows0 + before1[2], a.total_rows), p = min(pages0 + before2[0], a.page_indices_len);
    if (i < a.batch) {
      if (rows0 + before1[2] + rows > a.total_rows) bad |= FD_DEV_ROWS_RANGE;
      if (pages0 + before2[0] + have > a.page_indices_len) bad |= FD_DEV_PAGE_RANGE;
      if (a.mask_blocks) { const int nb = a.mask_blocks[i]; if (nb < 1 || q.m % nb) bad |= FD_DEV_ROWS_RANGE; }
      if (a.mask_vis) { const int v = a.mask_vis[i]; if (v < 0 || v > q.k) bad |= FD_DEV_ROWS_RANGE; }
      a.row_indptr[i] = r;
      a.page_indptr[i] = p;
      a.table_len_out[i] = have;
      if (EXPAND) { mine[0][i] = q.kv; mine[1][i] = q.k; mine[2][i] = q.m; mine[3][i] = r; mine[4][i] = p; }
    }
    rows0 = min(rows0 + total1[2], a.total_rows);
    pages0 = min(pages0 + total2[0], a.page_indices_len);
  }
  if (tid == 0) {
    a.row_indptr[a.batch] = rows0;
    a.page_indptr[a.batch] = pages0;
    a.free_count_out[0] = left;
    if (EXPAND) { mine[3][a.batch] = rows0; mine[4][a.batch] = pages0; }
  }
  if (bad) flag_status(a.status, bad);
  if (EXPAND) {
    __syncthreads();
    const int lane = tid & 63, wave = tid >> 6;
    // a request a wave, or fewer requests than waves: several waves a request
    const int share = a.batch < TB_WAVES ? TB_WAVES / max(a.batch, 1) : 1;
    for (int i = wave / share; i < a.batch; i += TB_WAVES / share)
      expand_request(a, i, mine[0][i], mine[1][i], mine[2][i], mine[3][i], mine[3][i + 1], mine[4][i], mine[4][i + 1], wave % share * 64 + lane, share * 64);
  }
}

__global__ __launch_bounds__(256) void step_lists_kernel(fd_table_args a) {
  const int i = blockIdx.x;
  const int r0 = a.row_indptr[i], r1 = a.row_indptr[i + 1], p0 = a.page_indptr[i], p1 = a.page_indptr[i + 1];
  const Request q = load_request(a, i);
  expand_request(a, i, q.kv, q.k, q.m, r0, r1, p0, p1, threadIdx.x, 256);
}

hipError_t run_step_tables(const fd_table_args& a, hipStream_t st) {
  // Small steps in one launch (at most a request a thread): there is less to write than a second launch costs (16 requests of 144 pages and
  // 16 rows: 6.5 us a call, in two launches 7.5).
  if (a.batch <= TB_BLOCK && (long long)a.page_indices_len + a.total_rows <= TB_SMALL) {
    hipLaunchKernelGGL(step_tables_kernel<true>, dim3(1), dim3(TB_BLOCK), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(step_tables_kernel<false>, dim3(1), dim3(TB_BLOCK), 0, st, a);
  if (a.batch > 0) hipLaunchKernelGGL(step_lists_kernel, dim3(a.batch), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace fd
