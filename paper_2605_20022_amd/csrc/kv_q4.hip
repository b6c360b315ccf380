// The 4-bit KV cache: commit of verified rows and read-back.
//
// Commit.  A work-group takes up to 64 tokens of one sequence and head, from a multiple of 16 slots on, so that no two
// work-groups share a byte of v_codes (two tokens a byte).  A thread has 32 channels of one token: of the key it finds the
// shared power of two and writes sixteen bytes of codes; of the value it finds the largest magnitude, which four
// lanes combine to the token's scale, and leaves the values in LDS, from where they are taken eight tokens at a time.
//
// Read-back.  A work-group writes 64 rows of one head: keys by (token, 32 channels), values by (eight tokens, four
// channels), the units in which the codes lie.
#include "kv_q4.h"

namespace fd {

constexpr int AQ_TOKENS = 64;

__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <int DH>
__global__ __launch_bounds__(256) void append_kv_q4_kernel(AttnParams p, Q4Cache c, const int* __restrict__ accept_len, int* kv_len_out) {
  constexpr int GR = DH / 32;                        // channel groups of a token
  constexpr int PITCH = DH + 2;                      // LDS row in bf16: an odd number of words
  __shared__ bf16_t vals[AQ_TOKENS][PITCH];
  __shared__ float scales[AQ_TOKENS];
  const int seq = blockIdx.x, head = blockIdx.y, tid = threadIdx.x;
  const SeqInfo s = load_seq(p, seq);
  int rows = 0;
  const bool first = head == 0 && blockIdx.z == 0 && tid == 0;
  if (s.k > 0) {
    int acc = accept_len[seq];
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
    const int lp = pos / p.page_size;
    const int page = p.page_indices[s.page0 + lp];
    if (page < 0 || page >= p.num_pages) { if (head == 0) flag_status(p.status, FD_DEV_PAGE_RANGE); return -1; }
    return q4_token(c, page, head, p.page_size, pos - lp * p.page_size);
  };
  {
    const int t = tid / GR, g = tid % GR, pos = t0 + t;
    if (t < AQ_TOKENS && pos >= lo && pos < hi) {
      const long long row = ((long long)(s.row0 + pos - s.L) * p.Hkv + head) * DH + g * 32;
      const long long at = token_at(pos);
      u32x4 kw[4], vw[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kw[j] = reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(p.k_new) + row)[j];
        vw[j] = reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(p.v_new) + row)[j];
      }
      // magnitudes as integers: in order, and a NaN above every number
      unsigned ktop = 0, vtop = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ktop = max(ktop, max(kw[j][e] & 0x7fff0000u, (kw[j][e] << 16) & 0x7fff0000u));
          vtop = max(vtop, max(vw[j][e] & 0x7fff0000u, (vw[j][e] << 16) & 0x7fff0000u));
        }
#pragma unroll
      for (int d = 1; d < GR; d <<= 1) vtop = max(vtop, (unsigned)__shfl_xor((int)vtop, d));
      const bool kfinite = ktop < 0x7f800000u, vfinite = vtop < 0x7f800000u;
      const int kb = q4_key_exponent(__uint_as_float(ktop));
      const bf16_t vs = vfinite ? f32_to_bf16(__uint_as_float(vtop) / 6.f) : (bf16_t)0x7fc0;
      if (at >= 0) {
        u32x4 codes;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[2 * e] = ldexpf(__uint_as_float(kw[j][e] << 16), 127 - kb);
            x[2 * e + 1] = ldexpf(__uint_as_float(kw[j][e] & 0xffff0000u), 127 - kb);
          }
          codes[j] = kfinite ? f32_to_q4(x) : 0u;
        }
        *reinterpret_cast<u32x4*>(c.k_codes + at * (DH / 2) + g * 16) = codes;
        c.k_scales[at * GR + g] = kfinite ? (unsigned char)kb : (unsigned char)255;
        if (g == 0) c.v_scales[at] = vs;
      }
      unsigned* dst = reinterpret_cast<unsigned*>(&vals[t][g * 32]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[4 * j + e] = vw[j][e];
      if (g == 0) scales[t] = bf16_to_f32(vs);
    }
  }
  __syncthreads();
  {
    // eight tokens, channels 32 cc + j
    const int u = tid / 32, j = tid % 32, base = t0 + 8 * u;
    if (base < hi && base + 8 > lo) {
      const long long at = token_at(base);
      if (at >= 0) {
        unsigned* dst = reinterpret_cast<unsigned*>(c.v_codes + (at / 16 * 16) * (DH / 2) + ((at / 8 & 1) * 32 + j) * GR * 4);
        unsigned keep = 0;                           // nibbles of tokens that are not written here
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (base + e < lo || base + e >= hi) keep |= 15u << (4 * e);
#pragma unroll
        for (int cc = 0; cc < GR; ++cc) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int t = 8 * u + e;
            x[e] = 0.f;
            if (base + e >= lo && base + e < hi) {
              const float v = bf16_to_f32(vals[t][32 * cc + j]), sc = scales[t];
              // (a correctly rounded quotient is a tie only where the exact one is: value and scale have 8 bits each)
              x[e] = sc > 0.f ? v / sc : sc == 0.f ? copysignf(0.f, v) : 0.f;
            }
          }
          const unsigned w = f32_to_q4(x);
          dst[cc] = keep ? (dst[cc] & keep) | (w & ~keep) : w;
        }
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
  int B, Hkv, page_size, num_pages, page_entries, total_rows;
  const int* page_indptr; const int* page_indices; const int* start; const int* out_indptr;
  uint32_t* status;
};

template <int DH, typename T>
__global__ __launch_bounds__(256) void read_kv_q4_kernel(ReadParams p, Q4Cache c, T* __restrict__ k_out, T* __restrict__ v_out) {
  constexpr int GR = DH / 32;
  const int head = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int a = blockIdx.x * AQ_TOKENS, b = min(a + AQ_TOKENS, p.total_rows);
  // the last sequence that starts at or before row a
  int seq = -1;
  for (int i0 = 0; i0 < p.B; i0 += 64) {
    const unsigned long long at = __ballot(i0 + lane < p.B && p.out_indptr[i0 + lane] <= a);
    if (at) seq = i0 + 63 - __clzll((long long)at);
    if (at != ~0ull) break;
  }
  bool bad = false;
  for (seq = seq < 0 ? 0 : seq; seq < p.B; ++seq) {
    const int o0 = clampi(p.out_indptr[seq], 0, p.total_rows), o1 = clampi(p.out_indptr[seq + 1], 0, p.total_rows);
    if (o0 >= b) break;
    const int r0 = max(a, o0), r1 = min(b, o1);                    // rows of this sequence in this work-group
    if (r0 >= r1) continue;
    const int s0 = p.start ? p.start[seq] : 0;
    const int pg0 = clampi(p.page_indptr[seq], 0, p.page_entries), pg1 = clampi(p.page_indptr[seq + 1], pg0, p.page_entries);
    const long long room = (long long)(pg1 - pg0) * p.page_size;
    const long long first = (long long)s0 + (r0 - o0);             // position of row r0
    auto token_at = [&](long long pos) -> long long {
      if (pos < 0 || pos >= room) { bad = true; return -1; }
      const int lp = (int)((unsigned)pos / (unsigned)p.page_size);
      const int page = p.page_indices[pg0 + lp];
      if (page < 0 || page >= p.num_pages) { bad = true; return -1; }
      return q4_token(c, page, head, p.page_size, (int)((unsigned)pos - (unsigned)lp * (unsigned)p.page_size));
    };
    for (int i = tid; i < (r1 - r0) * GR; i += 256) {
      const int t = i / GR, g = i % GR;
      const long long at = token_at(first + t);
      if (at < 0) continue;
      const u32x4 codes = *reinterpret_cast<const u32x4*>(c.k_codes + at * (DH / 2) + g * 16);
      const float sc = q4_key_scale(c.k_scales[at * GR + g]);
      T* dst = k_out + ((long long)(r0 + t) * p.Hkv + head) * DH + g * 32;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[8];
        q4_to_f32(codes[j], sc, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) Elem<T>::store(dst + 8 * j + e, x[e]);
      }
    }
    // eight slots at a time, from a multiple of eight on
    const long long u0 = first >= 0 ? first / 8 : (first - 7) / 8;
    const int units = (int)((first + (r1 - r0) + 7 - u0 * 8) / 8);
    for (int i = tid; i < units * 32; i += 256) {
      const int j = i & 31;
      const long long base = (u0 + i / 32) * 8;
      const long long inside = base < first ? first : base;        // a position of the unit that is asked for
      const long long at = token_at(inside);
      if (at < 0) continue;
      const long long eight = at - (inside - base);
      const unsigned* src = reinterpret_cast<const unsigned*>(c.v_codes + (eight / 16 * 16) * (DH / 2) + ((eight / 8 & 1) * 32 + j) * GR * 4);
#pragma unroll
      for (int cc = 0; cc < GR; ++cc) {
        float x[8];
        q4_to_f32(src[cc], 1.f, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const long long t = base + e - first;
          if (t < 0 || t >= r1 - r0) continue;
          Elem<T>::store(v_out + ((long long)(r0 + t) * p.Hkv + head) * DH + 32 * cc + j, x[e] * bf16_to_f32(c.v_scales[eight + e]));
        }
      }
    }
  }
  if (bad) flag_status(p.status, FD_DEV_PAGE_RANGE);
}

template <typename T>
static void launch_read(const ReadParams& p, const Q4Cache& c, int head_dim, void* k_out, void* v_out, hipStream_t st) {
  const dim3 grid((p.total_rows + AQ_TOKENS - 1) / AQ_TOKENS, p.Hkv);
  if (head_dim == 128) hipLaunchKernelGGL((read_kv_q4_kernel<128, T>), grid, dim3(256), 0, st, p, c, reinterpret_cast<T*>(k_out), reinterpret_cast<T*>(v_out));
  else hipLaunchKernelGGL((read_kv_q4_kernel<64, T>), grid, dim3(256), 0, st, p, c, reinterpret_cast<T*>(k_out), reinterpret_cast<T*>(v_out));
}

hipError_t run_read_kv_q4(const Q4Cache& c, int batch, int num_kv_heads, int head_dim, int page_size, int num_pages, const int* page_indptr,
                          const int* page_indices, int page_entries, const int* start, const int* out_indptr, int total_rows, void* k_out,
                          void* v_out, int dtype, uint32_t* status, hipStream_t st) {
  const ReadParams p = {batch, num_kv_heads, page_size, num_pages, page_entries, total_rows, page_indptr, page_indices, start, out_indptr, status};
  if (dtype == FD_BF16) launch_read<bf16_t>(p, c, head_dim, k_out, v_out, st);
  else launch_read<float>(p, c, head_dim, k_out, v_out, st);
  return hipGetLastError();
}

}  // namespace fd
