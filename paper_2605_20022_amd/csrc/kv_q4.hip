// The 4-bit KV cache: commit of verified rows and read-back.
//
// Both take 64 tokens of one sequence and head per work-group, from a multiple of eight (read-back) or sixteen (commit: two tokens share a byte
// of v_codes, and no two work-groups may write one byte) slots on.  Sixteen lanes (eight at head dim 64) have a token, eight channels each: the
// rows are read and written whole, and a key's power of two and a value's scale are maxima over four of them, and all.  Values
// change between rows and the eight tokens to a word of v_codes in LDS.  Bound by HBM where there is much to do (rows 2 or 4 bytes
// an element, codes a half), else by the latencies of lengths, page and row, one after the other.
#include "kv_q4.h"

namespace fd {

constexpr int AQ_TOKENS = 64;

// Largest of a value over 4 or N lanes in a row of sixteen, by lane shifts.
template <int N>
__device__ __forceinline__ unsigned max_over(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));            // quad_perm 1 0 3 2
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));            // quad_perm 2 3 0 1
  if (N >= 8) v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));      // mirror in eight
  if (N >= 16) v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));     // mirror in sixteen
  return v;
}
__device__ __forceinline__ unsigned top_of(u32x4 w) {      // largest magnitude of eight bf16, as the bits of an fp32: in order, and a NaN above every number
  unsigned t = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) t = max(t, max(w[e] & 0x7fff0000u, (w[e] << 16) & 0x7fff0000u));
  return t;
}

template <int DH>
__global__ __launch_bounds__(256) void append_kv_q4_kernel(AttnParams p, Q4Cache c, const int* __restrict__ accept_len, int* kv_len_out) {
  constexpr int LPT = DH / 8, GR = DH / 32;          // lanes of a token, channel groups
  constexpr int PITCH = DH + 8;                      // LDS row in bf16: rows stay 16-byte aligned
  __shared__ __align__(16) bf16_t vals[AQ_TOKENS][PITCH];
  __shared__ float2 inv[AQ_TOKENS];                  // a value is divided by its scale as (v x) y
  const int seq = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
  const int accepted = sload(accept_len, seq);       // (requested with the lengths)
  const SeqInfo s = load_seq(p, seq);
  int rows = 0;
  const bool first = head == 0 && blockIdx.z == 0 && tid == 0;
  if (s.k > 0) {
    int acc = accepted;
    if (acc < 0 || acc >= s.k) { if (first) flag_status(p.status, FD_DEV_ROWS_RANGE); acc = clampi(acc, 0, s.k - 1); }
    rows = acc + 1;
    const long long room = (long long)s.npages * p.page_size - s.L;
    if (rows > room) { if (first) flag_status(p.status, FD_DEV_PAGE_RANGE); rows = room < 0 ? 0 : (int)room; }
  }
  if (first && kv_len_out) kv_len_out[seq] = s.L + rows;
  const int t0 = s.L / 16 * 16 + blockIdx.z * AQ_TOKENS;            // first position of this work-group
  const int lo = max(t0, s.L), hi = min(t0 + AQ_TOKENS, s.L + rows);
  if (lo >= hi) return;
  // where a position lies; < 0: nowhere
  auto token_at = [&](int pos) -> long long {
    const int lp = (int)(__umulhi((unsigned)pos, p.page_magic) >> p.page_magic_shift);
    const int page = p.page_indices[s.page0 + lp];
    if (page < 0 || page >= p.num_pages) { if (head == 0) flag_status(p.status, FD_DEV_PAGE_RANGE); return -1; }
    return q4_token(c, page, head, p.page_size, pos - lp * p.page_size);
  };
  const int g = tid % LPT;                           // channels 8 g ..
  constexpr int PASSES = AQ_TOKENS * LPT / 256;
  u32x4 kw[PASSES], vw[PASSES];
  long long at[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {                 // all rows are requested, with their pages, before the first is looked at
    const int pos = t0 + u * (256 / LPT) + tid / LPT;
    const bool on = pos >= lo && pos < hi;
    const long long row = ((long long)(s.row0 + (on ? pos : lo) - s.L) * p.Hkv + head) * DH + g * 8;
    at[u] = on ? token_at(pos) : -1;
    kw[u] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(p.k_new) + row);
    vw[u] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(p.v_new) + row);
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int t = u * (256 / LPT) + tid / LPT;
    const unsigned ktop = max_over<4>(top_of(kw[u])), vtop = max_over<LPT>(top_of(vw[u]));
    const bool kfinite = ktop < 0x7f800000u, vfinite = vtop < 0x7f800000u;
    const int kb = q4_key_exponent(__uint_as_float(ktop));
    const bf16_t vs = vfinite ? f32_to_bf16(__uint_as_float(vtop) / 6.f) : (bf16_t)0x7fc0;
    if (at[u] >= 0) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = ldexpf(__uint_as_float(kw[u][e] << 16), 127 - kb);
        x[2 * e + 1] = ldexpf(__uint_as_float(kw[u][e] & 0xffff0000u), 127 - kb);
      }
      *reinterpret_cast<unsigned*>(c.k_codes + at[u] * (DH / 2) + g * 4) = kfinite ? f32_to_q4(x) : 0u;
      if (g % 4 == 0) c.k_scales[at[u] * GR + g / 4] = kfinite ? (unsigned char)kb : (unsigned char)255;
      if (g == 0) c.v_scales[at[u]] = vs;
    }
    *reinterpret_cast<u32x4*>(&vals[t][g * 8]) = vfinite ? vw[u] : u32x4{0, 0, 0, 0};
    if (g == 0) {
      const float sc = bf16_to_f32(vs), pre = sc < 0x1p-100f ? 0x1p60f : 1.f;       // (the reciprocal of the smallest scales is no number)
      inv[t] = make_float2(pre, vfinite && sc > 0.f ? 1.f / (sc * pre) : 0.f);
    }
  }
  __syncthreads();
  {
    // eight tokens, channels 32 cc + j
    const int u = tid / 32, j = tid % 32, base = t0 + 8 * u;
    if (base < hi && base + 8 > lo) {
      const long long tok = token_at(base);
      if (tok >= 0) {
        unsigned* dst = reinterpret_cast<unsigned*>(c.v_codes + (tok & ~15ll) * (DH / 2) + ((tok >> 3 & 1) * 32 + j) * GR * 4);
        unsigned keep = 0;                           // nibbles of tokens that are not written here
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (base + e < lo || base + e >= hi) keep |= 15u << (4 * e);
        unsigned old[GR];
#pragma unroll
        for (int cc = 0; cc < GR; ++cc) old[cc] = keep ? dst[cc] : 0u;
#pragma unroll
        for (int cc = 0; cc < GR; ++cc) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 d = inv[8 * u + e];         // (of tokens that are not written: any)
            // Value and scale have eight bits each, so that a quotient that is not a midpoint between two codes is 2^-14 of it away: rounded to
            // sixteen bits, the product with the reciprocal (2^-22) is the midpoint where the quotient is, and on its side of it where it is not.
            const float y = bf16_to_f32(vals[8 * u + e][32 * cc + j]) * d.x * d.y;
            x[e] = __uint_as_float((__float_as_uint(y) + 0x80u) & 0xffffff00u);
          }
          old[cc] = (old[cc] & keep) | (f32_to_q4(x) & ~keep);
        }
        if (GR == 4) *reinterpret_cast<u32x4*>(dst) = u32x4{old[0], old[1], old[GR - 2], old[GR - 1]};
        else *reinterpret_cast<u32x2*>(dst) = u32x2{old[0], old[1]};
      }
    }
  }
}

// The new lengths, where they may replace the old ones that every work-group of the commit reads.
__global__ __launch_bounds__(256) void append_kv_q4_lengths_kernel(AttnParams p, const int* __restrict__ accept_len, int* kv_len_out) {
  const int seq = blockIdx.x * 256 + threadIdx.x;
  if (seq >= p.B) return;
  const SeqInfo s = load_seq_t<false>(p, seq);
  int rows = 0;
  if (s.k > 0) {
    rows = clampi(accept_len[seq], 0, s.k - 1) + 1;
    const long long room = (long long)s.npages * p.page_size - s.L;
    if (rows > room) rows = room < 0 ? 0 : (int)room;
  }
  kv_len_out[seq] = s.L + rows;
}

hipError_t run_append_kv_q4(const AttnParams& p, const Q4Cache& c, const int* accept_len, int* kv_len_out, hipStream_t st) {
  const bool in_place = kv_len_out == p.kv_len;
  if (p.max_new_rows > 0 && p.total_rows > 0) {
    const dim3 grid(p.B, p.Hkv, (p.max_new_rows + 15 + AQ_TOKENS - 1) / AQ_TOKENS);
    if (p.D == 128) hipLaunchKernelGGL(append_kv_q4_kernel<128>, grid, dim3(256), 0, st, p, c, accept_len, in_place ? nullptr : kv_len_out);
    else hipLaunchKernelGGL(append_kv_q4_kernel<64>, grid, dim3(256), 0, st, p, c, accept_len, in_place ? nullptr : kv_len_out);
    if (!in_place) return hipGetLastError();
  }
  hipLaunchKernelGGL(append_kv_q4_lengths_kernel, dim3((p.B + 255) / 256), dim3(256), 0, st, p, accept_len, kv_len_out);
  return hipGetLastError();
}

// ---- read-back --------------------------------------------------------------------------------
struct ReadParams {
  int B, Hkv, page_size, num_pages, page_entries, total_rows, last_wg;
  const int* page_indptr; const int* page_indices; const int* start; const int* out_indptr;
  uint32_t* status;
};

// Eight values to a row.
__device__ __forceinline__ void store8(float* dst, const float (&x)[8]) {
  *reinterpret_cast<f32x4*>(dst) = f32x4{x[0], x[1], x[2], x[3]};
  *reinterpret_cast<f32x4*>(dst + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16_t* dst, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = (unsigned)f32_to_bf16(x[2 * e]) | ((unsigned)f32_to_bf16(x[2 * e + 1]) << 16);
  *reinterpret_cast<u32x4*>(dst) = w;
}

template <int DH, typename T>
__global__ __launch_bounds__(256) void read_kv_q4_kernel(ReadParams p, Q4Cache c, T* __restrict__ k_out, T* __restrict__ v_out) {
  constexpr int LPT = DH / 8, GR = DH / 32;
  __shared__ __align__(16) unsigned vcodes[AQ_TOKENS / 8][32 * GR];
  __shared__ long long where[AQ_TOKENS];               // of each token; < 0: nowhere
  __shared__ float vscale[AQ_TOKENS];
  const int head = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  // Which 64 tokens: those of a sequence are counted from a multiple of eight on.  Every wave finds it by itself, a sequence a lane.
  int seq = -1, o0 = 0, n = 0, s0 = 0, chunk = 0;
  for (int c0 = 0, base = 0; c0 < p.B; c0 += 64) {
    const int i = c0 + lane;
    int a = 0, rows = 0, st = 0, chunks = 0;
    if (i < p.B) {
      a = clampi(p.out_indptr[i], 0, p.total_rows);
      rows = clampi(p.out_indptr[i + 1], 0, p.total_rows) - a;
      st = p.start ? p.start[i] : 0;
      if (rows > 0) chunks = ((st & 7) + rows + AQ_TOKENS - 1) / AQ_TOKENS;
    }
    const int incl = base + wave_incl_scan(chunks);
    const unsigned long long here = __ballot((int)blockIdx.x >= incl - chunks && (int)blockIdx.x < incl);
    if (here) {
      const int l = __ffsll((long long)here) - 1;
      auto from = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      seq = c0 + l; o0 = from(a); n = from(rows); s0 = from(st); chunk = blockIdx.x - from(incl - chunks);
      break;
    }
    base = __builtin_amdgcn_readlane(incl, 63);
  }
  if ((int)blockIdx.x == p.last_wg && head == 0)       // (it has seldom tokens to read)
    for (int i = tid; i < p.B; i += 256) {
      const int r0 = p.out_indptr[i], r1 = p.out_indptr[i + 1];
      if (r0 < 0 || r1 < r0 || r1 > p.total_rows) flag_status(p.status, FD_DEV_ROWS_RANGE);
    }
  if (seq < 0) return;
  const int pg0 = clampi(sload(p.page_indptr, seq), 0, p.page_entries), pg1 = clampi(sload(p.page_indptr, seq + 1), pg0, p.page_entries);
  const long long room = (long long)(pg1 - pg0) * p.page_size;
  const long long first = (long long)s0 - (s0 & 7) + (long long)chunk * AQ_TOKENS;           // position of token 0 of this work-group
  const long long shift = first - s0;                  // token t is row o0 + shift + t, where that is one of the n
  if (tid < AQ_TOKENS) {
    const long long pos = first + tid;
    const bool asked = shift + tid >= 0 && shift + tid < n;
    long long at = -1;
    bool bad = false;
    if (pos >= 0 && pos < room) {
      const int lp = (int)((unsigned)pos / (unsigned)p.page_size);
      const int page = p.page_indices[pg0 + lp];
      if (page >= 0 && page < p.num_pages) at = q4_token(c, page, head, p.page_size, (int)((unsigned)pos - (unsigned)lp * (unsigned)p.page_size));
      else bad = true;
    } else bad = true;
    if (bad && asked) flag_status(p.status, FD_DEV_PAGE_RANGE);
    where[tid] = at;
    vscale[tid] = at >= 0 ? bf16_to_f32(c.v_scales[at]) : 0.f;
  }
  __syncthreads();
  {
    const int u = tid / 32, j = tid % 32;              // (eight tokens that share their words lie in one page)
    const long long at = where[8 * u];
    unsigned w[GR] = {};
    if (at >= 0) {
      const unsigned char* src = c.v_codes + (at & ~15ll) * (DH / 2) + ((at >> 3 & 1) * 32 + j) * GR * 4;
      if (GR == 4) { const u32x4 x = *reinterpret_cast<const u32x4*>(src); w[0] = x[0]; w[1] = x[1]; w[GR - 2] = x[2]; w[GR - 1] = x[3]; }
      else { const u32x2 x = *reinterpret_cast<const u32x2*>(src); w[0] = x[0]; w[1] = x[1]; }
    }
#pragma unroll
    for (int cc = 0; cc < GR; ++cc) vcodes[u][j * GR + cc] = w[cc];
  }
  const int g = tid % LPT;
  constexpr int PASSES = AQ_TOKENS * LPT / 256;
  unsigned kc[PASSES], ks[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const long long at = where[u * (256 / LPT) + tid / LPT];
    kc[u] = 0; ks[u] = 127;
    if (at >= 0) { kc[u] = *reinterpret_cast<const unsigned*>(c.k_codes + at * (DH / 2) + g * 4); ks[u] = c.k_scales[at * GR + g / 4]; }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int t = u * (256 / LPT) + tid / LPT;
    if (where[t] < 0 || shift + t < 0 || shift + t >= n) continue;
    const long long row = ((o0 + shift + t) * p.Hkv + head) * (long long)DH + g * 8;
    float x[8];
    q4_to_f32(kc[u], q4_key_scale(ks[u]), x);
    store8(k_out + row, x);
    // the token's nibble of eight channels' words: channels 8 g .. have c = g / 4, j from 8 (g % 4) on
    const unsigned* w = &vcodes[t / 8][8 * (g % 4) * GR + g / 4];
    unsigned v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) v |= ((w[e * GR] >> (4 * (t % 8))) & 15u) << (4 * e);
    q4_to_f32(v, 1.f, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= vscale[t];
    store8(v_out + row, x);
  }
}

// Work-groups of a head: 64 tokens each; a sequence begins with up to seven that are not asked for, and ends in part of 64.
long long read_kv_q4_wgs(int batch, int total_rows) { return total_rows / AQ_TOKENS + 2ll * (batch < total_rows ? batch : total_rows); }

template <typename T>
static void launch_read(const ReadParams& p, const Q4Cache& c, int head_dim, void* k_out, void* v_out, hipStream_t st) {
  const dim3 grid(p.last_wg + 1, p.Hkv);
  if (head_dim == 128) hipLaunchKernelGGL((read_kv_q4_kernel<128, T>), grid, dim3(256), 0, st, p, c, reinterpret_cast<T*>(k_out), reinterpret_cast<T*>(v_out));
  else hipLaunchKernelGGL((read_kv_q4_kernel<64, T>), grid, dim3(256), 0, st, p, c, reinterpret_cast<T*>(k_out), reinterpret_cast<T*>(v_out));
}

hipError_t run_read_kv_q4(const Q4Cache& c, int batch, int num_kv_heads, int head_dim, int page_size, int num_pages, const int* page_indptr,
                          const int* page_indices, int page_entries, const int* start, const int* out_indptr, int total_rows, void* k_out,
                          void* v_out, int dtype, uint32_t* status, hipStream_t st) {
  const ReadParams p = {batch, num_kv_heads, page_size, num_pages, page_entries, total_rows, (int)read_kv_q4_wgs(batch, total_rows) - 1, page_indptr,
                        page_indices, start, out_indptr, status};
  if (dtype == FD_BF16) launch_read<bf16_t>(p, c, head_dim, k_out, v_out, st);
  else launch_read<float>(p, c, head_dim, k_out, v_out, st);
  return hipGetLastError();
}

}  // namespace fd
