// Hybrid-mask verify+draft attention (Sec. 4.1) over a KV cache held in 4 bits, head dim 128 or 64.
//
// An item is one (sequence, KV head, up to 128 tile rows); a tile row is (new row, query head of the group).  Its keys,
// cached ones and then the sequence's own new rows, form blocks of 32.  Items are cut into pieces of equal length, one per
// work-group; an item of several pieces leaves (maximum, sum, un-normalised O) partials for the combine kernel.
//
// A wave takes 32 tile rows and a stream of blocks, by itself: with up to 32 tile rows the four waves of a work-group
// take every fourth block, with up to 64 two waves a row block take every second, else each wave has its own rows and all blocks.
// They meet once, when the piece ends and their (maximum, sum, O) are merged through LDS.  Nothing of the cache goes through LDS:
//   S^T = K Q^T    v_mfma_f32_32x32x16_bf16.  A lane's eight channels of a key are one word of codes, so a lane loads its
//                  half of a key's codes (sixteen bytes each 64 channels, one scale) and converts them in registers
//   O^T += V^T P^T the layout of v_codes holds eight keys of a channel in one word for the same reason; the scale of a
//                  value (one a token and head) is multiplied into P, which a lane holds for eight keys in a row
// Which key a row of S^T stands for is free: row i = (b4 b3 b2 b1 b0) is key (b4 b2 b3 b1 b0), so that the sixteen scores that a lane holds
// are two runs of eight keys, as the second product wants them.
#include "kv_q4.h"

namespace fd {

constexpr int Q4_BLOCK = 256;
constexpr int Q4_TK = 32;                 // keys of a block
constexpr int Q4_ROWS = 128;              // tile rows of an item
constexpr float Q4_LAZY = 6.f;            // the softmax reference follows the row maximum in steps of at least 2^6
constexpr int Q4_PIECES = 1024;           // pieces aimed at
constexpr int Q4_MIN_PIECE = 8;           // blocks of a piece, at least (but for the last of a short item)

struct Q4Sched {
  int fixed;                // > 0: blocks of a piece, asked for by the caller
  int rt_max;               // items of a (sequence, head), at most
  int max_partials;         // partial slots in the workspace
  float* part_acc;          // [max_partials][128][D] un-normalised O
  float* part_ml;           // [max_partials][128][2] maximum (base 2), sum
  int4* entries;            // [B * Hkv * rt_max]: pieces, first partial slot, first packed row, new rows
};

// Row blocks that the waves of a work-group share out, for an item of so many tile rows.
__device__ __forceinline__ int q4_row_blocks(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }
// How long a block takes a work-group, in halves: four waves take four blocks of one row block side by side, or one block of four.
__device__ __forceinline__ int q4_weight(int rows) { return rows <= 32 ? 2 : rows <= 64 ? 3 : 6; }

struct Q4Cut { int blocks, full, tail_rows; };          // of one sequence: blocks of its keys, items of 128 tile rows, rows of the last item
__device__ __forceinline__ Q4Cut q4_cut(const AttnParams& p, const SeqInfo& s) {
  Q4Cut c;
  c.blocks = s.n > 0 ? (s.L + Q4_TK - 1) / Q4_TK + (s.n + Q4_TK - 1) / Q4_TK : 0;
  const int rows = s.n * p.G;
  c.full = rows / Q4_ROWS;
  c.tail_rows = rows - c.full * Q4_ROWS;
  return c;
}
// Pieces of an item of so many rows.  target: units of weight x blocks a piece should have.
__device__ __forceinline__ int q4_pieces(const Q4Sched& sc, int blocks, int rows, long long target) {
  if (blocks <= 0 || rows <= 0) return 0;
  long long per = sc.fixed > 0 ? sc.fixed : (target + q4_weight(rows) - 1) / q4_weight(rows);
  if (sc.fixed <= 0 && per < Q4_MIN_PIECE) per = Q4_MIN_PIECE;
  return (int)((blocks + per - 1) / per);
}

// One value summed over the work-group (all threads), exact for integers.
__device__ __forceinline__ long long q4_block_sum(long long v, long long* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  return sh[0] + sh[1] + sh[2] + sh[3];
}

struct Q4Piece { int seq, head, rt, piece, pieces, slot; };

// Which piece work-group w takes: pieces are numbered by (sequence, head, item, piece).  Every thread calls this; false: none.
__device__ __forceinline__ bool q4_find(const AttnParams& p, const Q4Sched& sc, int w, Q4Piece& out) {
  __shared__ long long sh_sum[4];
  __shared__ int sh_w[4][2];
  __shared__ int sh_found[8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rounds = (p.B + Q4_BLOCK - 1) / Q4_BLOCK;
  Q4Cut cut = {};
  auto load = [&](int c) {
    cut = Q4Cut{};
    const int i = c * Q4_BLOCK + tid;
    if (i < p.B) cut = q4_cut(p, load_seq_t<false>(p, i));
  };
  long long units = 0;
  for (int c = 0; c < rounds; ++c) {
    load(c);
    units += (long long)cut.blocks * p.Hkv * (cut.full * q4_weight(Q4_ROWS) + (cut.tail_rows ? q4_weight(cut.tail_rows) : 0));
  }
  const long long total = q4_block_sum(units, sh_sum);
  const long long target = (total + Q4_PIECES - 1) / Q4_PIECES;
  int base = 0, sbase = 0;
  if (tid == 0) sh_found[0] = -1;
  for (int c = 0; c < rounds; ++c) {
    if (rounds > 1) load(c);
    const int pf = q4_pieces(sc, cut.blocks, cut.full ? Q4_ROWS : 0, target), pt = q4_pieces(sc, cut.blocks, cut.tail_rows, target);
    const int mine = p.Hkv * (cut.full * pf + pt);
    const int split = p.Hkv * (cut.full * (pf > 1 ? pf : 0) + (pt > 1 ? pt : 0));
    const int it = wave_incl_scan(mine), st = wave_incl_scan(split);
    __syncthreads();
    if (lane == 63) { sh_w[wave][0] = it; sh_w[wave][1] = st; }
    __syncthreads();
    int b0 = base, s0 = sbase;
    for (int q = 0; q < 4; ++q) {
      if (q < wave) { b0 += sh_w[q][0]; s0 += sh_w[q][1]; }
      base += sh_w[q][0]; sbase += sh_w[q][1];
    }
    const int begin = b0 + it - mine;
    if (w >= begin && w < begin + mine) {
      int x = w - begin, sl = s0 + st - split;
      const int per_head = cut.full * pf + pt, split_head = cut.full * (pf > 1 ? pf : 0) + (pt > 1 ? pt : 0);
      const int head = x / per_head;
      x -= head * per_head; sl += head * split_head;
      int rt, pieces;
      if (x < cut.full * pf) { rt = x / pf; x -= rt * pf; pieces = pf; sl += pf > 1 ? rt * pf : 0; }
      else { rt = cut.full; x -= cut.full * pf; pieces = pt; sl += pf > 1 ? cut.full * pf : 0; }
      sh_found[0] = c * Q4_BLOCK + tid; sh_found[1] = head; sh_found[2] = rt; sh_found[3] = x; sh_found[4] = pieces; sh_found[5] = sl;
    }
    if (w < base) break;                                   // (uniform)
  }
  __syncthreads();
  out.seq = __builtin_amdgcn_readfirstlane(sh_found[0]);
  out.head = __builtin_amdgcn_readfirstlane(sh_found[1]);
  out.rt = __builtin_amdgcn_readfirstlane(sh_found[2]);
  out.piece = __builtin_amdgcn_readfirstlane(sh_found[3]);
  out.pieces = __builtin_amdgcn_readfirstlane(sh_found[4]);
  out.slot = __builtin_amdgcn_readfirstlane(sh_found[5]);
  return out.seq >= 0;
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }
__device__ __forceinline__ unsigned pack_bf16x2(float lo, float hi) {
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));      // round to nearest even
}
// The larger of a lane's value and that of lane ^ 32.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Codes and scales of a block as a lane holds them.
template <int DH> struct Q4Regs {
  u32x4 k[DH / 64];          // its key's channels 64 a + 32 h ..: eight words of eight
  unsigned ks;               // the key's scales, a byte each 32 channels
  unsigned v[2][DH / 32];    // eight keys of channels 32 c + lane % 32, of either sixteen keys
  u32x4 vs[2];               // the scales of those eight keys
};

template <int DH>
__global__ __launch_bounds__(Q4_BLOCK, 2) void attn_q4_kernel(AttnParams p, Q4Cache c, Q4Sched sc) {
  constexpr int NA = DH / 64, NC = DH / 32, STEPS = DH / 16;
  constexpr int OP = DH + 4;                             // pitch of an O row in LDS, floats: an odd number of 16-byte slots
  __shared__ float lds_o[4][32][OP];
  __shared__ float lds_ml[4][32][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l31 = lane & 31, h = lane >> 5;
  Q4Piece pc;
  if (!q4_find(p, sc, blockIdx.x, pc)) return;
  const SeqInfo s = load_seq(p, pc.seq);
  const int rows = min(Q4_ROWS, s.n * p.G - pc.rt * Q4_ROWS);
  const int RB = q4_row_blocks(rows), KS = 4 / RB;
  const int rb = wave & (RB - 1), slot = wave / RB;
  const int cached = (s.L + Q4_TK - 1) / Q4_TK, blocks = cached + (s.n + Q4_TK - 1) / Q4_TK;
  const int first = (int)((long long)blocks * pc.piece / pc.pieces), last = (int)((long long)blocks * (pc.piece + 1) / pc.pieces);

  // ---- this lane's row and its query, as the second operand of S^T = K Q^T ----
  const int tr = rb * 32 + l31;
  const bool row_on = tr < rows;
  const int ti = pc.rt * Q4_ROWS + (row_on ? tr : 0);
  const int nr = ti / p.G, g = ti - nr * p.G;            // new row, query head of the group
  const bf16_t* qrow = reinterpret_cast<const bf16_t*>(p.q) + ((long long)(s.row0 + nr) * p.Hq + pc.head * p.G + g) * DH;
  u32x4 qf[STEPS];
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(qrow + 64 * (t / 4) + 32 * h + 8 * (t % 4));
    qf[t] = row_on ? x : u32x4{0, 0, 0, 0};
  }
  const float scale2 = p.sm_scale * 1.44269504088896340736f;

  f32x16 o[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[cc][e] = 0.f;
  float m = -3e38f, l = 0.f;

  // scores (scaled, base 2) -> probabilities; the running maximum and sum, and what O has to shrink by
  auto softmax = [&](f32x16& x) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
    top = max_halves(top);
    if (__any(top > m + Q4_LAZY)) {
      const float mn = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int cc = 0; cc < NC; ++cc)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[cc][e] *= f;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) { x[e] = __builtin_amdgcn_exp2f(x[e] - m); l += x[e]; }
  };

  // ---- cached keys ----
  const int lo = first + slot, hi = min(last, cached);
  // where sixteen keys lie: lane t knows it for the sixteens of this wave's blocks lo + KS (t / 2), t % 2
  long long where = 0;
  auto find_pages = [&](int b0) {
    const int pos = 32 * (b0 + KS * (lane >> 1)) + 16 * (lane & 1);
    where = 0;
    if (pos < s.L) {
      const int lp = pos / p.page_size;
      int page = p.page_indices[s.page0 + lp];
      if (page < 0 || page >= p.num_pages) { flag_status(p.status, FD_DEV_PAGE_RANGE); page = 0; }
      where = q4_token(c, page, pc.head, p.page_size, pos - lp * p.page_size);
    }
  };
  auto lane_where = [&](int t) -> long long {
    const unsigned a = __builtin_amdgcn_readlane((unsigned)where, t), b = __builtin_amdgcn_readlane((unsigned)((unsigned long long)where >> 32), t);
    return (long long)(((unsigned long long)b << 32) | a);
  };
  const int key_of_row = (l31 & 16) | ((l31 & 4) << 1) | ((l31 & 8) >> 1) | (l31 & 3);
  auto request = [&](Q4Regs<DH>& r, int t) {             // t: which of the wave's blocks since find_pages
    const long long w0 = lane_where(2 * t), w1 = lane_where(2 * t + 1);
    const long long mine = (key_of_row & 16 ? w1 : w0) + (key_of_row & 15);
    const u32x4* k = reinterpret_cast<const u32x4*>(c.k_codes + mine * (DH / 2)) + h;
#pragma unroll
    for (int a = 0; a < NA; ++a) r.k[a] = k[2 * a];
    if (DH == 128) r.ks = *reinterpret_cast<const unsigned*>(c.k_scales + mine * 4);
    else r.ks = *reinterpret_cast<const unsigned short*>(c.k_scales + mine * 2);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const long long w = q ? w1 : w0;
      const unsigned* v = reinterpret_cast<const unsigned*>(c.v_codes + w * (DH / 2)) + lane * NC;
      if (DH == 128) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(v);
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) r.v[q][cc] = x[cc];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(v);
        r.v[q][0] = x[0]; r.v[q][1] = x[1];
      }
      r.vs[q] = *reinterpret_cast<const u32x4*>(c.v_scales + w + 8 * h);
    }
  };
  auto multiply = [&](const Q4Regs<DH>& r, int b) {
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      const float ks = q4_key_scale((r.ks >> (8 * (2 * (t / 4) + h))) & 255u);
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(q4_to_bf16(r.k[t / 4][t % 4], ks)), as_bf16x8(qf[t]), x, 0, 0, 0);
    }
    const int left = s.L - 32 * b;                       // keys of this block, if below 32
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= scale2;
    if (left < 32) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (16 * (e / 8) + 8 * h + e % 8 >= left) x[e] = -INFINITY;
    }
    softmax(x);
    // P times the values' scales; a slot behind the prefix holds anything, NaN too
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      u32x4 pf;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float p0 = x[8 * q + 2 * e] * __uint_as_float(r.vs[q][e] << 16), p1 = x[8 * q + 2 * e + 1] * __uint_as_float(r.vs[q][e] & 0xffff0000u);
        if (left < 32) {
          if (16 * q + 8 * h + 2 * e >= left) p0 = 0.f;
          if (16 * q + 8 * h + 2 * e + 1 >= left) p1 = 0.f;
        }
        pf[e] = pack_bf16x2(p0, p1);
      }
#pragma unroll
      for (int cc = 0; cc < NC; ++cc)
        o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(q4_to_bf16(r.v[q][cc], 1.f)), as_bf16x8(pf), o[cc], 0, 0, 0);
    }
  };
  if (lo < hi) {
    const int count = (hi - lo + KS - 1) / KS;           // blocks of this wave
    for (int c0 = 0; c0 < count; c0 += 32) {
      find_pages(lo + KS * c0);
      const int n = min(32, count - c0);
      Q4Regs<DH> now, next;
      request(now, 0);
      for (int t = 0; t < n; ++t) {
        if (t + 1 < n) request(next, t + 1);
        multiply(now, lo + KS * (c0 + t));
        now = next;
      }
    }
  }

  // ---- the sequence's own rows, in bf16 ----
  {
    int b = first > cached ? first : cached;             // the wave's first block at or behind `cached`
    b += ((slot - (b - first)) % KS + KS) % KS;
    const RowWindow win = row_window(nr, s);
    for (; b < last; b += KS) {
      const int t0 = 32 * (b - cached);
      const int key = t0 + key_of_row;
      const long long stride = (long long)p.Hkv * DH;
      const bf16_t* krow = reinterpret_cast<const bf16_t*>(p.k_new) + (s.row0 + (key < s.n ? key : 0)) * stride + (long long)pc.head * DH;
      f32x16 x;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
      for (int t = 0; t < STEPS; ++t) {
        u32x4 kf = *reinterpret_cast<const u32x4*>(krow + 64 * (t / 4) + 32 * h + 8 * (t % 4));
        if (key >= s.n) kf = u32x4{0, 0, 0, 0};
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf), as_bf16x8(qf[t]), x, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int t = t0 + 16 * (e / 8) + 8 * h + e % 8;
        x[e] = t < s.n && new_key_visible(win, t) ? x[e] * scale2 : -INFINITY;
      }
      softmax(x);
      const bf16_t* v0 = reinterpret_cast<const bf16_t*>(p.v_new) + s.row0 * stride + (long long)pc.head * DH;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        u32x4 pf;
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[e] = pack_bf16x2(x[8 * q + 2 * e], x[8 * q + 2 * e + 1]);
        bool odd = false;                                // a value that is no number: it must not reach a row that does not see it
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) {
          u32x4 vf;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int ta = t0 + 16 * q + 8 * h + 2 * e;
            unsigned va = ta < s.n ? v0[ta * stride + 32 * cc + l31] : 0u, vb = ta + 1 < s.n ? v0[(ta + 1) * stride + 32 * cc + l31] : 0u;
            if ((va & 0x7f80u) == 0x7f80u) { odd = true; va = 0; }
            if ((vb & 0x7f80u) == 0x7f80u) { odd = true; vb = 0; }
            vf[e] = va | (vb << 16);
          }
          o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vf), as_bf16x8(pf), o[cc], 0, 0, 0);
        }
        if (__any(odd)) {                                // rare: infinities and NaN are added one by one where they are seen
#pragma unroll
          for (int w = 0; w < 4; ++w)                    // a word of P: two keys of either half
            for (int u = 0; u < 4; ++u) {
              const int t = t0 + 16 * q + 8 * (u >> 1) + 2 * w + (u & 1);
              if (t >= s.n) continue;
              const unsigned pw = __shfl((int)pf[w], (u >> 1) * 32 + l31);
              const float pr = __uint_as_float(u & 1 ? pw & 0xffff0000u : pw << 16);
              if (!new_key_visible(win, t)) continue;
#pragma unroll
              for (int cc = 0; cc < NC; ++cc)
#pragma unroll
                for (int a = 0; a < 16; ++a) {
                  const float v = bf16_to_f32(v0[t * stride + 32 * cc + 8 * (a / 4) + 4 * h + a % 4]);
                  if (!(fabsf(v) < INFINITY)) o[cc][a] += pr * v;
                }
            }
        }
      }
    }
  }
  l = add_halves(l);

  // ---- the waves' parts of a row meet: O^T columns become rows of LDS ----
  if (h == 0) { lds_ml[wave][l31][0] = m; lds_ml[wave][l31][1] = l; }
#pragma unroll
  for (int cc = 0; cc < NC; ++cc)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 x = {o[cc][4 * q], o[cc][4 * q + 1], o[cc][4 * q + 2], o[cc][4 * q + 3]};
      *reinterpret_cast<f32x4*>(&lds_o[wave][l31][32 * cc + 8 * q + 4 * h]) = x;
    }
  __syncthreads();
  const int item = (pc.seq * p.Hkv + pc.head) * sc.rt_max + pc.rt;
  if (threadIdx.x == 0 && pc.piece == 0) sc.entries[item] = make_int4(pc.pieces, pc.slot, s.row0, s.n);
  constexpr int TPR = 8, CPT = DH / TPR;                 // threads of a row, channels of a thread
  const int part = threadIdx.x % TPR;
  for (int r = threadIdx.x / TPR; r < rows; r += Q4_BLOCK / TPR) {
    const int b = r / 32, lr = r % 32;
    float M = -3e38f;
    for (int k = 0; k < KS; ++k) M = fmaxf(M, lds_ml[b + RB * k][lr][0]);
    float acc[CPT], sum = 0.f;
#pragma unroll
    for (int e = 0; e < CPT; ++e) acc[e] = 0.f;
    for (int k = 0; k < KS; ++k) {
      const int w = b + RB * k;
      const float f = __builtin_amdgcn_exp2f(lds_ml[w][lr][0] - M);
      sum += f * lds_ml[w][lr][1];
#pragma unroll
      for (int e = 0; e < CPT; e += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&lds_o[w][lr][part * CPT + e]);
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[e + u] += f * x[u];
      }
    }
    if (pc.pieces > 1) {
      if (pc.slot + pc.piece >= sc.max_partials) continue;           // (cannot be: the workspace holds every split piece)
      const long long at = (long long)(pc.slot + pc.piece) * Q4_ROWS + r;
      float* dst = sc.part_acc + at * DH + part * CPT;
#pragma unroll
      for (int e = 0; e < CPT; e += 4) *reinterpret_cast<f32x4*>(dst + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
      if (part == 0) { sc.part_ml[at * 2] = M; sc.part_ml[at * 2 + 1] = sum; }
    } else {
      const int t = pc.rt * Q4_ROWS + r, n = t / p.G;
      const long long orow = (long long)(s.row0 + n) * p.Hq + pc.head * p.G + (t - n * p.G);
      const float inv = 1.f / sum;
      unsigned* dst = reinterpret_cast<unsigned*>(reinterpret_cast<bf16_t*>(p.out) + orow * DH + part * CPT);
#pragma unroll
      for (int e = 0; e < CPT; e += 2) dst[e / 2] = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
      if (part == 0 && p.lse) p.lse[orow] = (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
    }
  }
}

// Merge of the partials of split items, by rows: a row is taken by DH / 8 lanes.
template <int DH>
__global__ __launch_bounds__(256) void attn_q4_combine_kernel(AttnParams p, Q4Sched sc) {
  constexpr int TPR = DH / 8, RPB = 256 / TPR;
  const int item = blockIdx.x, rt = item % sc.rt_max, head = item / sc.rt_max % p.Hkv, seq = item / sc.rt_max / p.Hkv;
  // (a sequence without new rows, or with fewer, has no such item and no entry)
  const SeqInfo s = load_seq(p, seq);
  const int rows = min(Q4_ROWS, s.n * p.G - rt * Q4_ROWS);
  const int r = blockIdx.y * RPB + threadIdx.x / TPR, part = threadIdx.x % TPR;
  if (rows <= 0 || blockIdx.y * RPB >= rows) return;
  const int4 e = sc.entries[item];
  const int pieces = e.x, slot = e.y;
  if (pieces <= 1 || r >= rows || slot < 0 || (long long)slot + pieces > sc.max_partials) return;
  float M = -3e38f;
  for (int q = 0; q < pieces; ++q) M = fmaxf(M, sc.part_ml[((long long)(slot + q) * Q4_ROWS + r) * 2]);
  float acc[8] = {}, sum = 0.f;
  for (int q = 0; q < pieces; ++q) {
    const long long at = (long long)(slot + q) * Q4_ROWS + r;
    const float f = __builtin_amdgcn_exp2f(sc.part_ml[at * 2] - M);
    sum += f * sc.part_ml[at * 2 + 1];
    const f32x4* src = reinterpret_cast<const f32x4*>(sc.part_acc + at * DH + part * 8);
    const f32x4 x = src[0], y = src[1];
#pragma unroll
    for (int u = 0; u < 4; ++u) { acc[u] += f * x[u]; acc[4 + u] += f * y[u]; }
  }
  const int t = rt * Q4_ROWS + r, n = t / p.G;
  const long long orow = (long long)(s.row0 + n) * p.Hq + head * p.G + (t - n * p.G);
  const float inv = 1.f / sum;
  u32x4 w;
#pragma unroll
  for (int u = 0; u < 4; ++u) w[u] = pack_bf16x2(acc[2 * u] * inv, acc[2 * u + 1] * inv);
  *reinterpret_cast<u32x4*>(reinterpret_cast<bf16_t*>(p.out) + orow * DH + part * 8) = w;
  if (part == 0 && p.lse) p.lse[orow] = (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

// Items of the largest sequence, partial slots and work-groups that there can be, and the workspace.
struct Q4Shape { long long items, partials, wgs; int rt_max, fixed; size_t off_ml, off_entries, total; };
static Q4Shape q4_shape(int batch, int num_kv_heads, int group, int total_rows, int max_kv_len, int max_new_rows, int kv_chunk, int head_dim) {
  Q4Shape z;
  const long long tile_rows = (long long)max_new_rows * group;
  z.rt_max = (int)((tile_rows + Q4_ROWS - 1) / Q4_ROWS);
  if (z.rt_max < 1) z.rt_max = 1;
  z.fixed = kv_chunk / Q4_TK;
  const long long seqs = batch < total_rows ? batch : total_rows;       // sequences that have rows
  z.items = seqs * num_kv_heads * z.rt_max;
  const long long blocks = ((long long)max_kv_len + Q4_TK - 1) / Q4_TK + (max_new_rows + Q4_TK - 1) / Q4_TK;
  if (z.fixed > 0) {
    z.wgs = z.items * ((blocks + z.fixed - 1) / z.fixed);
    z.partials = z.wgs;
  } else {
    // pieces - 1 of an item stay below its weight x blocks / target, which sum to Q4_PIECES over all items
    z.wgs = z.items + Q4_PIECES;
    z.partials = 2 * Q4_PIECES;                                         // an item in c >= 2 pieces: c <= 2 (c - 1)
    const long long most = z.items * ((blocks + Q4_MIN_PIECE - 1) / Q4_MIN_PIECE);
    if (most < z.wgs) z.wgs = most;
    if (most < z.partials) z.partials = most;
  }
  auto round = [](size_t x) { return (x + 255) / 256 * 256; };
  z.off_ml = round((size_t)z.partials * Q4_ROWS * head_dim * sizeof(float));
  z.off_entries = z.off_ml + round((size_t)z.partials * Q4_ROWS * 2 * sizeof(float));
  z.total = z.off_entries + round((size_t)(batch > 0 ? batch : 1) * num_kv_heads * z.rt_max * sizeof(int4));
  return z;
}

// 0 where the call is too large for one launch.
size_t attn_q4_workspace(int batch, int num_kv_heads, int group, int total_rows, int max_kv_len, int max_new_rows, int kv_chunk, int head_dim) {
  const Q4Shape z = q4_shape(batch, num_kv_heads, group, total_rows, max_kv_len, max_new_rows, kv_chunk, head_dim);
  if (z.wgs >= (1ll << 31) || (long long)batch * num_kv_heads * z.rt_max >= (1ll << 31)) return 0;
  return z.total > 0 ? z.total : 256;
}

hipError_t run_attn_q4(const AttnParams& p, const Q4Cache& c, void* workspace, int kv_chunk, hipStream_t st) {
  const Q4Shape z = q4_shape(p.B, p.Hkv, p.G, p.total_rows, p.max_kv_len, p.max_new_rows, kv_chunk, p.D);
  char* ws = reinterpret_cast<char*>(workspace);
  const Q4Sched sc = {z.fixed, z.rt_max, (int)z.partials, reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + z.off_ml), reinterpret_cast<int4*>(ws + z.off_entries)};
  if (z.wgs == 0) return hipSuccess;
  const int per_row = p.D / 8, most_rows = (int)((long long)p.max_new_rows * p.G < Q4_ROWS ? p.max_new_rows * p.G : Q4_ROWS);
  const dim3 grid((unsigned)((long long)p.B * p.Hkv * z.rt_max), (most_rows * per_row + 255) / 256);
  if (p.D == 128) {
    hipLaunchKernelGGL(attn_q4_kernel<128>, dim3((unsigned)z.wgs), dim3(Q4_BLOCK), 0, st, p, c, sc);
    hipLaunchKernelGGL(attn_q4_combine_kernel<128>, grid, dim3(256), 0, st, p, sc);
  } else {
    hipLaunchKernelGGL(attn_q4_kernel<64>, dim3((unsigned)z.wgs), dim3(Q4_BLOCK), 0, st, p, c, sc);
    hipLaunchKernelGGL(attn_q4_combine_kernel<64>, grid, dim3(256), 0, st, p, sc);
  }
  return hipGetLastError();
}

}  // namespace fd
