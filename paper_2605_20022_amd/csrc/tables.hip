// Tables of a decoding step from the requests' lengths: pages change hands between the requests and the pool, then
// row offsets, page lists, positions and slots.
//
// Bound by latency: a served batch moves some kilobytes.  The page exchange is a prefix sum over the requests (who gives and
// takes how much decides where on the stack), so one work-group does it, 1024 requests at a time; the lists are
// independent of each other once the sums stand.
#include "fd_common.h"

namespace fd {

constexpr int TB_BLOCK = 1024;            // threads that exchange pages, a request each (256 where that is enough)
constexpr int TB_SMALL = 8192;            // lists, positions and slots up to which the same work-group writes them too

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

// Exclusive prefix over the work-group and its total.  x is at most 2^20, so 1024 of them fit.
template <int WAVES>
__device__ __forceinline__ int block_excl_scan(int x, int* sums, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_incl_scan(x);
  __syncthreads();                                   // (the last round's sums have been read)
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  return before + incl - x;
}

// count entries from src (src_step apart, 1 or -1) to dst for each lane: a few entries lane by lane, long runs by the whole wave, sixteen
// entries a lane in flight (a request that ends gives back some thousand pages: 1024 requests, 30 of them ended, 26.6 us a call with four).
__device__ __forceinline__ void copy_runs(const int* src, int* dst, int src_step, int count) {
  constexpr int FEW = 4, DEEP = 16;
  const int lane = threadIdx.x & 63;
  if (count <= FEW)
    for (int j = 0; j < count; ++j) dst[j] = src[(long long)j * src_step];
  unsigned long long many = __ballot(count > FEW);
  while (many) {
    const int l = __ffsll((long long)many) - 1;
    many &= many - 1;
    const int* s = reinterpret_cast<const int*>(__shfl((unsigned long long)(uintptr_t)src, l));
    int* d = reinterpret_cast<int*>(__shfl((unsigned long long)(uintptr_t)dst, l));
    const int n = __shfl(count, l);
    for (int j0 = lane; j0 < n; j0 += 64 * DEEP) {
      int v[DEEP];
#pragma unroll
      for (int u = 0; u < DEEP; ++u) v[u] = s[(long long)min(j0 + 64 * u, n - 1) * src_step];
#pragma unroll
      for (int u = 0; u < DEEP; ++u)
        if (j0 + 64 * u < n) d[j0 + 64 * u] = v[u];
    }
  }
}

// Lists, positions and slots of request i, by `threads` threads of which this is number t.
__device__ __forceinline__ void expand_request(const fd_table_args& a, int i, int row0, int row1, int page0, int page1, int t, int threads) {
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
  const Request q = load_request(a, i);
  int nb = 1;
  if (a.mask_blocks) {
    nb = a.mask_blocks[i];
    if (nb < 1 || q.m % nb) nb = 1;
  }
  int v = q.k - nb + 1 < 0 ? 0 : q.k - nb + 1;
  if (a.mask_vis) v = clampi(a.mask_vis[i], 0, q.k);
  const int per = q.m / nb > 0 ? q.m / nb : 1;
  for (int r = t; r < row1 - row0; r += threads) {
    int pos = q.kv + r;
    long long slot = -1;
    if (r < q.k) {
      const int lp = (int)((unsigned)pos / (unsigned)a.page_size);
      if (lp < pages) slot = (long long)table[lp] * a.page_size + (pos - lp * a.page_size);
    } else {
      const int b = (r - q.k) / per;
      pos = q.kv + (v + b < q.k ? v + b : q.k) + (r - q.k - b * per);
    }
    if (a.positions) a.positions[row0 + r] = pos;
    if (a.slot_map) a.slot_map[row0 + r] = slot;
  }
}

template <int BLOCK, bool EXPAND>
__global__ __launch_bounds__(BLOCK) void step_tables_kernel(fd_table_args a) {
  constexpr int WAVES = BLOCK / FD_WAVE;
  __shared__ int sums[WAVES];
  const int tid = threadIdx.x;
  uint32_t bad = 0;
  int count = a.free_count[0];
  if (count < 0 || count > a.free_pages_len) { bad |= FD_DEV_PAGE_RANGE; count = clampi(count, 0, a.free_pages_len); }
  const int rounds = (a.batch + BLOCK - 1) / BLOCK;
  // 1. pages given back go onto the stack
  int top = count;
  Request q = {};
  for (int c = 0; c < rounds; ++c) {
    const int i = c * BLOCK + tid;
    q = Request{};
    if (i < a.batch) q = load_request(a, i);
    bad |= q.bad;
    const int give = q.held > q.need ? q.held - q.need : 0;
    int total;
    const int at = top + block_excl_scan<WAVES>(give, sums, total);
    int n = give;
    if (at + n > a.free_pages_len) { n = at < a.free_pages_len ? a.free_pages_len - at : 0; bad |= FD_DEV_PAGE_RANGE; }
    copy_runs(a.block_table + (long long)(i < a.batch ? i : 0) * a.table_stride + q.need, a.free_pages + (n > 0 ? at : 0), 1, n);
    top += total;
    if (top > a.free_pages_len) top = a.free_pages_len;
  }
  __syncthreads();                                   // the stack is whole before anyone takes from it
  // 2. pages are taken from its top; 3. the prefix sums
  int left = top, rows0 = 0, pages0 = 0;
  for (int c = 0; c < rounds; ++c) {
    const int i = c * BLOCK + tid;
    if (rounds > 1) { q = Request{}; if (i < a.batch) q = load_request(a, i); }
    const int take = q.need > q.held ? q.need - q.held : 0;
    int total;
    const int before = block_excl_scan<WAVES>(take, sums, total);
    const int mine = left - before;                  // entries of the stack that are there for this request
    const int got = mine < take ? (mine > 0 ? mine : 0) : take;
    if (got < take) bad |= FD_DEV_PAGE_RANGE;
    copy_runs(a.free_pages + (got > 0 ? mine - 1 : 0), a.block_table + (long long)(i < a.batch ? i : 0) * a.table_stride + q.held, -1, got);
    left = left > total ? left - total : 0;
    const int have = q.held + got < q.need ? q.held + got : q.need;
    int rows = q.k + q.m;
    if (rows > a.total_rows) rows = a.total_rows;
    int rows_total, pages_total;
    const int r = rows0 + block_excl_scan<WAVES>(rows, sums, rows_total);
    const int p = pages0 + block_excl_scan<WAVES>(have, sums, pages_total);
    if (i < a.batch) {
      if (r + rows > a.total_rows) bad |= FD_DEV_ROWS_RANGE;
      if (p + have > a.page_indices_len) bad |= FD_DEV_PAGE_RANGE;
      if (a.mask_blocks) { const int nb = a.mask_blocks[i]; if (nb < 1 || q.m % nb) bad |= FD_DEV_ROWS_RANGE; }
      if (a.mask_vis) { const int v = a.mask_vis[i]; if (v < 0 || v > q.k) bad |= FD_DEV_ROWS_RANGE; }
      a.row_indptr[i] = r < a.total_rows ? r : a.total_rows;
      a.page_indptr[i] = p < a.page_indices_len ? p : a.page_indices_len;
      a.table_len_out[i] = have;
    }
    rows0 = rows0 + rows_total < a.total_rows ? rows0 + rows_total : a.total_rows;
    pages0 = pages0 + pages_total < a.page_indices_len ? pages0 + pages_total : a.page_indices_len;
  }
  if (tid == 0) {
    a.row_indptr[a.batch] = rows0;
    a.page_indptr[a.batch] = pages0;
    a.free_count_out[0] = left;
  }
  if (bad) flag_status(a.status, bad);
  if (EXPAND) {
    __syncthreads();
    const int lane = tid & 63, wave = tid >> 6;
    // a request a wave, or fewer requests than waves: several waves a request
    const int share = a.batch < WAVES ? WAVES / a.batch : 1;
    for (int i = wave / share; i < a.batch; i += WAVES / share)
      expand_request(a, i, a.row_indptr[i], a.row_indptr[i + 1], a.page_indptr[i], a.page_indptr[i + 1], wave % share * 64 + lane, share * 64);
  }
}

__global__ __launch_bounds__(256) void step_lists_kernel(fd_table_args a) {
  const int i = blockIdx.x;
  expand_request(a, i, a.row_indptr[i], a.row_indptr[i + 1], a.page_indptr[i], a.page_indptr[i + 1], threadIdx.x, 256);
}

hipError_t run_step_tables(const fd_table_args& a, hipStream_t st) {
  // Small steps in one launch: there is less to write than a second launch costs (MEASURED).
  const bool small = (long long)a.page_indices_len + a.total_rows <= TB_SMALL && a.batch > 0;
  if (small && a.batch <= 256) { hipLaunchKernelGGL((step_tables_kernel<256, true>), dim3(1), dim3(256), 0, st, a); return hipGetLastError(); }
  if (small) { hipLaunchKernelGGL((step_tables_kernel<TB_BLOCK, true>), dim3(1), dim3(TB_BLOCK), 0, st, a); return hipGetLastError(); }
  if (a.batch <= 256) hipLaunchKernelGGL((step_tables_kernel<256, false>), dim3(1), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((step_tables_kernel<TB_BLOCK, false>), dim3(1), dim3(TB_BLOCK), 0, st, a);
  if (a.batch > 0) hipLaunchKernelGGL(step_lists_kernel, dim3(a.batch), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace fd
