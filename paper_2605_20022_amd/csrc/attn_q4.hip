// Hybrid-mask verify+draft attention (Sec. 4.1) over a KV cache held in 4 bits, head dim 128 or 64.
//
// An item is one (sequence, KV head, up to 128 tile rows); a tile row is (new row, query head of the group).  Its keys,
// cached ones and then the sequence's own new rows, form blocks of 32.  Items are cut into pieces of about equal time, one per
// work-group; an item of several pieces leaves (maximum, sum, un-normalised O) partials for the combine kernel, in fp32.
//
// A wave takes 32 tile rows and a stream of blocks, by itself: with up to 32 tile rows the four waves of a work-group
// take every fourth block, with up to 64 two waves a row block take every second, else each wave has its own rows and all blocks.
// They meet once, when the piece ends and their (maximum, sum, O) are merged through LDS.  Nothing of the cache goes through LDS, and two blocks of a
// wave are on their way while a third is worked on:
//   S^T = K Q^T    v_mfma_f32_32x32x16_bf16, with the query as it is: a lane's eight channels of a key are one word of codes, which four instructions
//                  make bf16 times the key's power of two, exactly.  (The scaled instructions for 4 and 8 bits take the codes as they lie, with the
//                  query as two e4m3 numbers, and 3% less time; but they add eight products at a time with some 14 bits below the largest: an lse of few
//                  keys was 4e-5 off, and one large channel of a query drowned the others.)
//   O^T += V^T P^T the same instruction.  The layout of v_codes holds eight keys of a channel in one word for the same reason;
//                  the scale of a value (one a token and head) is multiplied into P, which a lane holds for eight keys in a row
// Which key a row of S^T stands for is free: row i = (b4 b3 b2 b1 b0) is key (b4 b2 b3 b1 b0), so that the sixteen scores that a lane holds
// are two runs of eight keys, as the second product wants them.
//
// What bounds it: a block of 32 rows and 32 keys takes a SIMD 0.24 us of matrix instructions and 0.30 us of others, of which little runs side by side
// (0.5 us measured, two waves): 2 sequences of 2048 to 8192 keys, 272 rows and 32 query heads 68 us a call, 668 TFLOP/s.  With few rows HBM, for which
// the same arithmetic leaves little time: 128 sequences of 1024 to 8192 keys, up to 16 rows 174 us, 3.8 TB/s.  One short sequence is latency
// (15.5 us): lengths, pages, codes, merge, second launch.
#include "kv_q4.h"
#include "q4_shape.h"

namespace fd {

#define FD_INLINE __attribute__((always_inline))      // on a lambda: what it captures stays in registers

constexpr int Q4_BLOCK = 256;
constexpr float Q4_LAZY = 256.f;          // sum of a row's sixteen probabilities from which on the softmax reference follows the row maximum

struct Q4Sched {
  int fixed;                // > 0: blocks of a piece, asked for by the caller
  float a_fixed;            // pieces a block, then
  int unit_shift;           // work is counted in 2^unit_shift units
  int rt_max;               // items of a (sequence, head), at most
  int max_partials;         // partial slots in the workspace
  float* part_acc;          // [max_partials][128][D] the un-normalised O row
  float* part_ml;           // [max_partials][128][2] maximum (base 2), sum
  int2* entries;            // [B * Hkv * rt_max]: pieces, first partial slot
};

// Row blocks that the waves of a work-group share out, for an item of so many tile rows.
__device__ __forceinline__ int q4_row_blocks(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }
// How long a block takes a work-group, in halves: four waves take four blocks of one row block side by side, or one block of four.
__device__ __forceinline__ int q4_weight(int rows) { return rows <= 32 ? 2 : rows <= 64 ? 3 : 6; }

// How long a sequence's keys take, in cached blocks: the own rows' blocks that one of its rows sees (its own mask block's keys lie in two of them or
// so) count Q4_OWN each, the first Q4_OWN_START more.
__device__ __forceinline__ int q4_own(const SeqInfo& s) {
  const int all = (s.n + Q4_TK - 1) / Q4_TK;
  return Q4_OWN * (s.nb > 1 ? min((s.k + Q4_TK - 1) / Q4_TK + 2, all) : all);
}
__device__ __forceinline__ int q4_blocks(const SeqInfo& s) { return s.n > 0 ? (s.L + Q4_TK - 1) / Q4_TK + Q4_OWN_START + q4_own(s) : 0; }
// An item's tile rows: rows / 128 whole items and one of what is left.
__device__ __forceinline__ long long q4_units(int blocks, int rows) {           // of one head: weight x blocks
  const int tail = rows % Q4_ROWS;
  return (long long)blocks * (rows / Q4_ROWS * q4_weight(Q4_ROWS) + (tail ? q4_weight(tail) : 0));
}
// Pieces of an item: density (pieces a unit) x its units, rounded up, and no piece below Q4_MIN_PIECE blocks.  The products stay a little below the
// exact ones, so that pieces - 1 never exceeds density x units, which the host counts on.
__device__ __forceinline__ int q4_pieces(const Q4Sched& sc, int blocks, int rows, float density) {
  if (blocks <= 0 || rows <= 0) return 0;
  const float a_block = sc.fixed > 0 ? sc.a_fixed : fminf(density * (float)q4_weight(rows), 1.f / Q4_MIN_PIECE);
  return (int)((float)blocks * (a_block * 0.999999f)) + 1;
}
struct Q4Count { int full, tail; };       // pieces of a whole item and of the last
__device__ __forceinline__ Q4Count q4_count(const Q4Sched& sc, int blocks, int rows, float density) {
  return Q4Count{rows >= Q4_ROWS ? q4_pieces(sc, blocks, Q4_ROWS, density) : 0, q4_pieces(sc, blocks, rows % Q4_ROWS, density)};
}

// How long a sequence's longest piece takes a work-group, in units.
__device__ __forceinline__ int q4_longest(const Q4Sched& sc, int blocks, int rows, float density) {
  const int r = min(rows, Q4_ROWS);
  return rows > 0 ? (int)((float)blocks * (float)q4_weight(r) * __builtin_amdgcn_rcpf((float)q4_pieces(sc, blocks, r, density))) : 0;
}

struct Q4Piece { int head, rt, piece, pieces, slot, item; SeqInfo s; };

__device__ __forceinline__ int wave_max(int v) {         // of values >= 0
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(v, 63);
}

// Which piece work-group w takes: pieces are numbered by (class, sequence, head, item, piece).  Every wave finds it by itself, a sequence a lane, 64 at
// a time: the lengths are one latency of memory, the rest LDS of its own and lane shifts, and no wave waits for another.  false: none.
//
// How many pieces: with fewer than Q4_SLOTS items as many as run at once, found by bisection, so that one round does it (16 sequences of 512 to
// 4096 keys 27.3 us a call, in rounds 35.4; 2 of 272 rows 67.7, 84.2): a piece's start and
// end cost about as much as twelve blocks (find, pages, first codes, merge), and a second round would wait for the first.  Else Q4_PIECES and
// the items themselves, dealt out as work-groups become free, the sequences with the longest pieces first: one that began last would be waited for
// (128 sequences of 1024 to 8192 keys: 173 us, in the order of the batch 201; 768 pieces and items 182).
//
// FEW (up to 64 sequences): lengths stay in registers (16 sequences 27.3 us, by the general variant 30.2, whose code is longer and cold).
template <bool FEW>
__device__ __forceinline__ bool q4_find(const AttnParams& p, const Q4Sched& sc, int w, int4* kept, Q4Piece& out) {
  const int lane = threadIdx.x & 63;
  const int rounds = FEW ? 1 : (p.B + 63) / 64;
  SeqInfo only = {};
  auto load = [&](int c) FD_INLINE {
    uint32_t bad = 0;
    const int i = c * 64 + lane;
    SeqInfo s = load_seq_t<false>(p, min(i, p.B - 1), &bad);       // (no branch: the loads of two rounds go together)
    if (i >= p.B) s.n = 0;
    if (bad && w == 0 && threadIdx.x < 64) flag_status(p.status, bad);        // (work-group 0 comes by every sequence)
    return s;
  };
  auto get = [&](int c, int l) FD_INLINE {               // the round's l-th sequence
    if (FEW) return only;
    if (c >= Q4_KEPT) return load(c);
    const int4 a = kept[(c * 2) * 64 + l], b = kept[(c * 2 + 1) * 64 + l];
    return SeqInfo{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  };
  int total = 0, items = 0;                              // units of one head, in 2^unit_shift (the host's bounds say that they fit), and items
  auto count = [&](int c, const SeqInfo& s) FD_INLINE {
    if (FEW) only = s;
    else if (c < Q4_KEPT) {
      kept[(c * 2) * 64 + lane] = make_int4(s.L, s.row0, s.n, s.k);
      kept[(c * 2 + 1) * 64 + lane] = make_int4(s.v, s.nb, s.page0, s.npages);
    }
    const int rows = s.n * p.G;
    // (rounded up, so that there are never more pieces than the host counts on)
    total += wave_total((int)((q4_units(q4_blocks(s), rows) + (1ll << sc.unit_shift) - 1) >> sc.unit_shift));
    items += wave_total((rows + Q4_ROWS - 1) / Q4_ROWS);
  };
  if (FEW) count(0, load(0));
  else
#pragma unroll 1
    for (int c = 0; c < rounds; c += 2) {
      const SeqInfo s0 = load(c), s1 = load(c + 1);      // (behind the last sequence: without rows)
      count(c, s0);
      count(c + 1, s1);
    }
  const float all = ldexpf((float)total, sc.unit_shift) * (float)p.Hkv * 1.000001f;
  float density = (float)Q4_PIECES / fmaxf(all, 1.f);
  int classes = 1;
  float part = 0.f;                                      // classes a unit of time
  if (sc.fixed <= 0 && rounds <= Q4_KEPT) {
    if (items * (long long)p.Hkv < Q4_SLOTS) {
      // One a compute unit where that is not much work: two at a time start and end slower.  Then, first whether pieces of Q4_MIN_PIECE blocks fit,
      // after that between what fits and what is too many.
      const int slots = items * (long long)p.Hkv <= Q4_SLOTS / 4 && all <= (float)(Q4_SLOTS / 2 * Q4_ALONE) ? Q4_SLOTS / 2 : Q4_SLOTS;
      float lo = (float)(slots - items * p.Hkv) / fmaxf(all, 1.f), hi = (float)slots / fmaxf(all, 1.f);
      density = 1.f;
#pragma unroll 1
      for (int i = 0; i < 5; ++i) {
        int n = 0;
#pragma unroll 1
        for (int c = 0; c < rounds; ++c) {
          const SeqInfo s = get(c, lane);
          const int rows = s.n * p.G;
          const Q4Count k = q4_count(sc, q4_blocks(s), rows, density);
          n += rows / Q4_ROWS * k.full + k.tail;
        }
        const bool fits = wave_total(n) * p.Hkv <= slots;
        if (i == 0) { if (fits) { lo = density; break; } }
        else if (fits) lo = density;
        else hi = density;
        density = 0.5f * (lo + hi);
      }
      density = lo;
    } else {
      int top = 1;
#pragma unroll 1
      for (int c = 0; c < rounds; ++c) {
        const SeqInfo s = get(c, lane);
        top = max(top, q4_longest(sc, q4_blocks(s), s.n * p.G, density));
      }
      classes = Q4_CLASSES;
      part = (float)Q4_CLASSES / (float)wave_max(top);
    }
  }
  int base = 0, sbase = 0;
#pragma unroll 1
  for (int turn = 0; turn < classes; ++turn)
#pragma unroll 1
    for (int c = 0; c < rounds; ++c) {
      const SeqInfo s = get(c, lane);
      const int blocks = q4_blocks(s);
      int rows = s.n * p.G;
      if (classes > 1) {
        if (Q4_CLASSES - 1 - min((int)((float)q4_longest(sc, blocks, rows, density) * part), Q4_CLASSES - 1) != turn) rows = 0;
        if (__ballot(rows > 0) == 0) continue;
      }
      const Q4Count k = q4_count(sc, blocks, rows, density);
      const int full = rows / Q4_ROWS, per_head = full * k.full + k.tail, split_head = full * (k.full > 1 ? k.full : 0) + (k.tail > 1 ? k.tail : 0);
      const int it = wave_incl_scan(p.Hkv * per_head), st = wave_incl_scan(p.Hkv * split_head);
      const int end = base + it, begin = end - p.Hkv * per_head;
      const unsigned long long here = __ballot(w >= begin && w < end);
      if (here) {
        const int l = __ffsll((long long)here) - 1;
        auto from = [&](int v) FD_INLINE { return __builtin_amdgcn_readlane(v, l); };
        int x = w - from(begin), sl = sbase + from(st - p.Hkv * split_head);
        const int fl = from(full), f = from(k.full), t = from(k.tail), ph = from(per_head);
        out.head = x / ph;
        x -= out.head * ph; sl += out.head * from(split_head);
        if (x < fl * f) { out.rt = x / f; x -= out.rt * f; out.pieces = f; sl += f > 1 ? out.rt * f : 0; }
        else { out.rt = fl; x -= fl * f; out.pieces = t; sl += f > 1 ? fl * f : 0; }
        out.piece = x; out.slot = sl;
        out.item = ((c * 64 + l) * p.Hkv + out.head) * sc.rt_max + out.rt;
        out.s = SeqInfo{from(s.L), from(s.row0), from(s.n), from(s.k), from(s.v), from(s.nb), from(s.page0), from(s.npages)};
        return true;
      }
      base += __builtin_amdgcn_readlane(it, 63);
      sbase += __builtin_amdgcn_readlane(st, 63);
    }
  return false;
}

typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

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
template <int DH> struct Q4Keys {
  u32x4 code[DH / 64];       // its key's channels 64 a + 32 h ..: 32 each
  unsigned scale;            // the key's scales, a byte each 32 channels
};
template <int DH> struct Q4Values {
  unsigned code[2][DH / 32]; // eight keys of channels 32 c + lane % 32, of either sixteen keys
  u32x4 scale[2];            // the scales of those eight keys
};

template <int DH, bool FEW>
__global__ __launch_bounds__(Q4_BLOCK, 2) void attn_q4_kernel(AttnParams p, Q4Cache c, Q4Sched sc) {
  constexpr int NA = DH / 64, NC = DH / 32, STEPS = DH / 16;
  constexpr int OP = DH + 4;                             // pitch of an O row in LDS, floats: an odd number of 16-byte slots
  __shared__ __align__(16) float lds_o[4][32][OP];
  __shared__ float lds_ml[4][32][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l31 = lane & 31, h = lane >> 5;
  Q4Piece pc;
  static_assert(Q4_KEPT * 2 * 64 * sizeof(int4) <= sizeof(lds_o[0]), "the lengths fit a wave's part of LDS");
  if (!q4_find<FEW>(p, sc, blockIdx.x, reinterpret_cast<int4*>(&lds_o[wave][0][0]), pc)) return;
  const SeqInfo& s = pc.s;
  const int rows = min(Q4_ROWS, s.n * p.G - pc.rt * Q4_ROWS);
  const int RB = q4_row_blocks(rows), ks_shift = RB == 1 ? 2 : RB == 2 ? 1 : 0, KS = 1 << ks_shift;
  const int rb = wave & (RB - 1), slot = wave >> (2 - ks_shift);
  const int cached = (s.L + Q4_TK - 1) / Q4_TK, own = (s.n + Q4_TK - 1) / Q4_TK, length = q4_blocks(s);
  const float own_at = (float)own / (float)q4_own(s);
  auto cut = [&](int piece) FD_INLINE {                  // blocks before a piece
    const int at = (int)((long long)length * piece / pc.pieces), in_own = max(at - cached - Q4_OWN_START, 0);
    return at <= cached ? at : at == length ? cached + own : cached + min((int)((float)in_own * own_at), own);
  };
  const int first = cut(pc.piece), last = cut(pc.piece + 1);

  // ---- cached keys: which blocks, where they lie ----
  const int lo = first + slot, hi = min(last, cached);
  const int count = lo < hi ? (hi - lo + KS - 1) >> ks_shift : 0;        // blocks of this wave: lo, lo + KS, ...
  // Where the two sixteens of the wave's block t lie, as token numbers (q4_token; the host has seen to it that they fit 32 bits): lane t % 64 knows
  // it.  For what lies past the last block or the prefix: keys that are there.
  const unsigned page_tokens = (unsigned)c.sp * (unsigned)p.page_size, head_tokens = (unsigned)c.sh * (unsigned)p.page_size * (unsigned)pc.head;
  auto page_of = [&](int pos, unsigned& slot) FD_INLINE -> int {
    const int lp = (int)(__umulhi((unsigned)pos, p.page_magic) >> p.page_magic_shift);
    slot = (unsigned)(pos - lp * p.page_size);
    return p.page_indices[s.page0 + lp];
  };
  auto token_of = [&](int page, unsigned slot) FD_INLINE -> unsigned {
    const bool bad = (unsigned)page >= (unsigned)p.num_pages;
    if (bad) flag_status(p.status, FD_DEV_PAGE_RANGE);
    return (bad ? 0u : (unsigned)page) * page_tokens + head_tokens + slot;
  };
  unsigned where0 = 0, where1 = 0;
  auto find_pages = [&](int t) FD_INLINE {                         // t: a multiple of 64
    const int pos = 32 * (lo + (min(t + lane, count - 1) << ks_shift));
    unsigned slot0, slot1;
    const int page0 = page_of(pos, slot0), page1 = page_of(min(pos + 16, (s.L - 1) & ~15), slot1);
    where0 = token_of(page0, slot0);
    where1 = token_of(page1, slot1);
  };
  auto look_up = [&](int t, unsigned& at0, unsigned& at1) FD_INLINE {
    if ((t & 63) == 0 && t > 0) find_pages(t);
    at0 = __builtin_amdgcn_readlane(where0, t & 63);
    at1 = __builtin_amdgcn_readlane(where1, t & 63);
  };
  const int key_of_row = (l31 & 16) | ((l31 & 4) << 1) | ((l31 & 8) >> 1) | (l31 & 3);
  auto request_keys = [&](Q4Keys<DH>& r, unsigned at0, unsigned at1) FD_INLINE {
    const unsigned mine = (key_of_row & 16 ? at1 : at0) + (unsigned)(key_of_row & 15);
    const unsigned char* k = c.k_codes + (unsigned long long)mine * (DH / 2) + h * 16;
#pragma unroll
    for (int a = 0; a < NA; ++a) r.code[a] = *reinterpret_cast<const u32x4*>(k + 32 * a);
    const unsigned char* ks = c.k_scales + (unsigned long long)mine * (DH / 32);
    if (DH == 128) r.scale = *reinterpret_cast<const unsigned*>(ks);
    else r.scale = *reinterpret_cast<const unsigned short*>(ks);
  };
  auto request_values = [&](Q4Values<DH>& r, unsigned at0, unsigned at1) FD_INLINE {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const unsigned tok = q ? at1 : at0;
      const unsigned char* v = c.v_codes + (unsigned long long)tok * (DH / 2);
      if (DH == 128) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(v + (unsigned)lane * 16u);
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) r.code[q][cc] = x[cc];
      } else {
        const u32x2 x = *reinterpret_cast<const u32x2*>(v + (unsigned)lane * 8u);
        r.code[q][0] = x[0]; r.code[q][1] = x[1];
      }
      r.scale[q] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const unsigned char*>(c.v_scales) + (unsigned long long)tok * 2 + (unsigned)h * 16u);
    }
  };
  Q4Keys<DH> ka, kb;
  Q4Values<DH> va, vb;
  if (count > 0) find_pages(0);

  // ---- this lane's row and its query, as the second operand of S^T = K Q^T ----
  const int tr = rb * 32 + l31;
  const bool row_on = tr < rows;
  const int ti = pc.rt * Q4_ROWS + (row_on ? tr : 0);
  const int nr = ti / p.G, g = ti - nr * p.G;            // new row, query head of the group
  const bf16_t* qrow = reinterpret_cast<const bf16_t*>(p.q) + ((long long)(s.row0 + nr) * p.Hq + pc.head * p.G + g) * DH;
  u32x4 qw[4 * NA];                                      // channels 64 a + 32 h + 8 w ..: eight each, as the codes of a key lie
#pragma unroll
  for (int t = 0; t < 4 * NA; ++t) qw[t] = *reinterpret_cast<const u32x4*>(qrow + 64 * (t / 4) + 32 * h + 8 * (t % 4));
  if (count > 0) {
    unsigned at0, at1;
    look_up(0, at0, at1);
    request_keys(ka, at0, at1);
    request_values(va, at0, at1);
  }
  const float scale2 = p.sm_scale * 1.44269504088896340736f;

  f32x16 o[NC];
#pragma unroll
  for (int cc = 0; cc < NC; ++cc)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[cc][e] = 0.f;
  float m = -3e38f, l = 0.f;                             // running maximum (scaled, base 2) and sum

  // Scores -> probabilities.  They are taken against the running maximum as it stands; only where a row's sixteen sum to more than
  // Q4_LAZY (the first block does) is the maximum found, and what was summed so far shrunk to it.  Sums and bf16 probabilities have the same
  // relative precision whatever the reference, and a maximum costs as much as half the exponentials.
  auto exponentials = [&](const f32x16& x, f32x16& y) FD_INLINE {
    float t[4];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], scale2, -m));
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (y[4 * e] + y[4 * e + 1]) + (y[4 * e + 2] + y[4 * e + 3]);
    return (t[0] + t[1]) + (t[2] + t[3]);
  };
  auto settle = [&](const f32x16& x, f32x16& y, float sum) FD_INLINE {
    if (__any(sum > Q4_LAZY)) {
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
      const float mn = fmaxf(m, max_halves(top) * scale2), f = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int cc = 0; cc < NC; ++cc)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[cc][e] *= f;
      sum = exponentials(x, y);
    }
    l += sum;
  };
  // ---- the sequence's own rows, in bf16: keys as the first operand straight from memory, values through this wave's part of LDS and its transposing read ----
  int b = first > cached ? first : cached;               // the wave's first block at or behind `cached`
  b += (slot - (b - first)) & (KS - 1);
  RowWindow win = row_window(nr, s);
  if (!row_on) win = RowWindow{0, 0, 0};
  // a block that none of the wave's rows sees is passed over (2 sequences of 16 verify rows and 16 mask blocks of 16, where a row sees one: 67.7 us, else 76.8)
  auto seen_from = [&](int b) FD_INLINE {
    while (b < last) {
      const int t0 = 32 * (b - cached);
      if (__any((t0 < win.vr) | ((t0 < win.hi) & (t0 + 32 > win.lo)))) break;
      b += KS;
    }
    return b;
  };
  b = seen_from(b);
  if (b < last) {
    constexpr int VP = DH + 32;                          // pitch of a row of values, bf16: the four rows of a transposing read use every bank once
    static_assert(32 * VP * sizeof(bf16_t) <= sizeof(lds_o[0]), "a block of values fits a wave's part of LDS");
    constexpr int LPR = DH / 8, RPL = 64 / LPR;          // lanes of a row, rows of a load
    bf16_t* lv = reinterpret_cast<bf16_t*>(&lds_o[wave][0][0]);
    const long long stride = (long long)p.Hkv * DH;
    const bf16_t* k0 = reinterpret_cast<const bf16_t*>(p.k_new) + s.row0 * stride + (long long)pc.head * DH;
    const bf16_t* v0 = reinterpret_cast<const bf16_t*>(p.v_new) + s.row0 * stride + (long long)pc.head * DH;
    u32x4 kf[STEPS], vr[STEPS];
    // (behind the last row: that row, which the mask leaves out)
    auto load_k = [&](int t0) FD_INLINE {
      const bf16_t* krow = k0 + min(t0 + key_of_row, s.n - 1) * stride;
#pragma unroll
      for (int t = 0; t < STEPS; ++t) kf[t] = *reinterpret_cast<const u32x4*>(krow + 64 * (t / 4) + 32 * h + 8 * (t % 4));
    };
    auto load_v = [&](int t0) FD_INLINE {
#pragma unroll
      for (int t = 0; t < STEPS; ++t) vr[t] = *reinterpret_cast<const u32x4*>(v0 + min(t0 + RPL * t + lane / LPR, s.n - 1) * stride + lane % LPR * 8);
    };
    load_k(32 * (b - cached));
    load_v(32 * (b - cached));
    for (int next; b < last; b = next) {
      next = seen_from(b + KS);
      const int t0 = 32 * (b - cached);
      // A value that is no number must not reach a row that does not see it, and zero times it is NaN: it enters the product as zero.
      unsigned odd = 0;                                  // (an exponent of all ones, plus one in its last place, reaches the sign)
#pragma unroll
      for (int t = 0; t < STEPS; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= (vr[t][e] & 0x7f807f80u) + 0x00800080u;
      const bool any_odd = __any((odd & 0x80008000u) != 0);
      if (any_odd) {
#pragma unroll
        for (int t = 0; t < STEPS; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((vr[t][e] & 0x7f80u) == 0x7f80u) vr[t][e] &= 0xffff0000u;
            if ((vr[t][e] & 0x7f800000u) == 0x7f800000u) vr[t][e] &= 0xffffu;
          }
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
      for (int t = 0; t < STEPS; ++t) *reinterpret_cast<u32x4*>(lv + (RPL * t + lane / LPR) * VP + lane % LPR * 8) = vr[t];
      f32x16 x;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
      for (int t = 0; t < STEPS; ++t) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[t]), as_bf16x8(qw[t]), x, 0, 0, 0);
      if (next < last) { load_k(32 * (next - cached)); load_v(32 * (next - cached)); }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int t = t0 + 16 * (e / 8) + 8 * h + e % 8;
        x[e] = ((t < s.n) & new_key_visible(win, t)) ? x[e] : -INFINITY;
      }
      f32x16 y;
      const float sum = exponentials(x, y);
      settle(x, y, sum);
      x = y;
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      // (sixteen lanes read four keys of sixteen channels, and each gets its channel's four)
      const bf16_t* vt = lv + (8 * h + ((lane & 15) >> 2)) * VP + (l31 & 16) + 4 * (lane & 3);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        u32x4 pf;
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[e] = pack_bf16x2(x[8 * q + 2 * e], x[8 * q + 2 * e + 1]);
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) {
          const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + 16 * q * VP + 32 * cc));
          const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + (16 * q + 4) * VP + 32 * cc));
          const s16x8 v = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
          o[cc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), as_bf16x8(pf), o[cc], 0, 0, 0);
        }
      }
      if (any_odd) {                                     // rare: infinities and NaN are added one by one where they are seen
        float* mine = &lds_o[wave][l31][0];              // (a row's 32 probabilities, in place of the values)
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
#pragma unroll
        for (int e = 0; e < 16; ++e) mine[16 * (e / 8) + 8 * h + e % 8] = x[e];
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        const int n = min(32, s.n - t0);
#pragma unroll 1
        for (int t = 0; t < n; ++t) {
          if (!new_key_visible(win, t0 + t)) continue;
          const float pr = mine[t];
          const bf16_t* vrow = v0 + (t0 + t) * stride + 4 * h;
#pragma unroll
          for (int cc = 0; cc < NC; ++cc)
#pragma unroll
            for (int a = 0; a < 16; ++a) {
              const float v = bf16_to_f32(vrow[32 * cc + 8 * (a / 4) + a % 4]);
              if (!(fabsf(v) < INFINITY)) o[cc][a] += pr * v;
            }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  }
  if (count > 0) {
    unsigned at0, at1;
    look_up(1, at0, at1);
    request_keys(kb, at0, at1);
    request_values(vb, at0, at1);
  }
  // Eight codes of this lane's key with their power of two, as an operand: exact.
  auto key_part = [&](const Q4Keys<DH>& r, int i) FD_INLINE {
    const unsigned byte = (r.scale >> (8 * h) >> (16 * (i / 4))) & 255u;
    return q4_to_bf16(r.code[i / 4][i % 4], q4_key_scale(byte));
  };
  auto key_scores = [&](const Q4Keys<DH>& r) FD_INLINE {
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(key_part(r, i)), as_bf16x8(qw[i]), x, 0, 0, 0);
    return x;
  };
  // One block: its scores x become probabilities and weigh its values, while the matrix pipe works on the scores of the next.  left: keys of the
  // block, if below 32.
  auto block = [&](f32x16 x, Q4Values<DH>& r, const Q4Keys<DH>& next, int left) FD_INLINE {
    if (left < 32) {                                     // a slot behind the prefix holds anything, a NaN as its scale too
      asm volatile("");                                  // (a branch: as selects this would run for every block)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (16 * (e / 8) + 8 * h + e % 8 >= left) x[e] = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = 16 * (e / 4) + 8 * h + 2 * (e % 4);
        const unsigned w = r.scale[e / 4][e % 4];
        r.scale[e / 4][e % 4] = key >= left ? 0u : key + 1 >= left ? w & 0xffffu : w;
      }
    }
    // products for the next scores, with a share of the exponentials in between; the compiler's order (held to this one by barriers for the
    // scheduler, codes one product ahead: 4% slower)
    f32x16 y, xn;
    float part[STEPS];
#pragma unroll
    for (int e = 0; e < 16; ++e) xn[e] = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      constexpr int SHARE = 16 / STEPS;
      xn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(key_part(next, i)), as_bf16x8(qw[i]), xn, 0, 0, 0);
      part[i] = 0.f;
#pragma unroll
      for (int e = i * SHARE; e < (i + 1) * SHARE; ++e) y[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], scale2, -m));
#pragma unroll
      for (int e = i * SHARE; e < (i + 1) * SHARE; e += 2) part[i] = e == i * SHARE ? y[e] + y[e + 1] : part[i] + (y[e] + y[e + 1]);
    }
    float sum = (part[0] + part[1]) + (part[2] + part[3]);
    if (STEPS == 8) sum += (part[STEPS - 4] + part[STEPS - 3]) + (part[STEPS - 2] + part[STEPS - 1]);
    asm volatile("" : "+v"(xn));                         // (not to be moved past the branch)
    settle(x, y, sum);
    u32x4 pf[2];                                         // P times the values' scales
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        pf[q][e] = pack_bf16x2(y[8 * q + 2 * e] * __uint_as_float(r.scale[q][e] << 16), y[8 * q + 2 * e + 1] * __uint_as_float(r.scale[q][e] & 0xffff0000u));
#pragma unroll
    for (int i = 0; i < 2 * NC; ++i)
      o[i % NC] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(q4_to_bf16(r.code[i / NC][i % NC], 1.f)), as_bf16x8(pf[i / NC]), o[i % NC], 0, 0, 0);
    return xn;
  };
  // Keys and values of two blocks are held or on their way.  Past the end the last block is requested again (its lines are at hand), so that
  // nothing in the loop depends on the count; with an odd count the last step's second half weighs nothing.
  if (count > 0) {
    const int left0 = s.L - 32 * lo, step = 32 << ks_shift;
    f32x16 x = key_scores(ka);
    unsigned at0, at1, bt0, bt1;
    look_up(2, at0, at1);
    request_keys(ka, at0, at1);
    for (int t = 0; t < count; t += 2) {
      x = block(x, va, kb, left0 - t * step);
      request_values(va, at0, at1);
      look_up(t + 3, bt0, bt1);
      request_keys(kb, bt0, bt1);
      x = block(x, vb, ka, t + 1 < count ? left0 - (t + 1) * step : 0);
      request_values(vb, bt0, bt1);
      look_up(t + 4, at0, at1);
      request_keys(ka, at0, at1);
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
  if (threadIdx.x == 0 && pc.piece == 0) sc.entries[pc.item] = make_int2(pc.pieces, pc.slot);
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
      if (pc.slot + pc.piece >= sc.max_partials) continue;           // (only where the device's rows contradict the host's bounds)
      const long long at = (long long)(pc.slot + pc.piece) * Q4_ROWS + r;
      // In fp32: a row is a sum, whose channels may be of any size beside each other.  (As fp16 over the row's largest entry it would be half the bytes, 2
      // sequences of 272 rows 64.3 us a call instead of 68.2, 1 of 16 rows 15.1 instead of 15.5; but what is 2^-16 of that entry loses its digits, and beside
      // an infinity there is no largest entry.)
      f32x4* dst = reinterpret_cast<f32x4*>(sc.part_acc + at * DH + part * CPT);
#pragma unroll
      for (int e = 0; e < CPT; e += 4) dst[e / 4] = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
      if (part == 0) *reinterpret_cast<f32x2*>(sc.part_ml + at * 2) = f32x2{M, sum};
    } else {
      const int t = pc.rt * Q4_ROWS + r, n = t / p.G;
      const long long orow = (long long)(s.row0 + n) * p.Hq + pc.head * p.G + (t - n * p.G);
      const float inv = 1.f / sum;
      u32x4* dst = reinterpret_cast<u32x4*>(reinterpret_cast<bf16_t*>(p.out) + orow * DH + part * CPT);
#pragma unroll
      for (int e = 0; e < CPT; e += 8)
        dst[e / 8] = u32x4{pack_bf16x2(acc[e] * inv, acc[e + 1] * inv), pack_bf16x2(acc[e + 2] * inv, acc[e + 3] * inv),
                           pack_bf16x2(acc[e + 4] * inv, acc[e + 5] * inv), pack_bf16x2(acc[e + 6] * inv, acc[e + 7] * inv)};
      if (part == 0 && p.lse) p.lse[orow] = (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
    }
  }
}

// Merge of the partials of split items, by rows: a row is taken by TPR = DH / 8 lanes, eight channels each.  AT_ONCE pieces at a time, lane j of them
// knows the maximum and sum of piece j; their values are requested with those, so that a batch is one latency.  Where an item may have many pieces,
// 2^group_shift such groups of lanes share a row's and meet in LDS (1 sequence of 32 768 keys: 25.6 us a call, with one group 33.2).
template <int DH>
__global__ __launch_bounds__(256) void attn_q4_combine_kernel(AttnParams p, Q4Sched sc, int group_shift) {
  constexpr int TPR = DH / 8, SETS = 256 / TPR, AT_ONCE = 8;
  __shared__ float lds_acc[SETS][DH + 4], lds_ml[SETS][2];
  const int item = blockIdx.x, rt = item % sc.rt_max, head = item / sc.rt_max % p.Hkv, seq = item / sc.rt_max / p.Hkv;
  const int2 e = sc.entries[item];
  // (a sequence without new rows, or with fewer, has no such item: what stands in its entry is old)
  const int r0 = sload(p.row_indptr, seq), r1 = sload(p.row_indptr, seq + 1);
  const int row0 = clampi(r0, 0, p.total_rows), new_rows = min(clampi(r1 - r0, 0, p.max_new_rows), p.total_rows - row0);
  const int rows = min(Q4_ROWS, new_rows * p.G - rt * Q4_ROWS);
  const int pieces = __builtin_amdgcn_readfirstlane(e.x), slot = __builtin_amdgcn_readfirstlane(e.y);
  const int rows_here = SETS >> group_shift, first_row = (int)blockIdx.y * rows_here;
  if (first_row >= rows || pieces <= 1 || slot < 0 || (long long)slot + pieces > sc.max_partials) return;
  const int set = threadIdx.x / TPR, group = set >> (31 - __clz(SETS) - group_shift);         // (sets of one row are rows_here apart)
  const int r = first_row + (set & (rows_here - 1)), part = threadIdx.x % TPR;
  const int rr = r < rows ? r : 0;                       // (every lane takes part in the exchanges)
  const int j = part % AT_ONCE, lane0 = (threadIdx.x & 63) / TPR * TPR;
  float M = -3e38f, sum = 0.f, acc[8] = {};
  for (int q0 = 0; q0 < pieces; q0 += AT_ONCE << group_shift) {
    const int q = q0 + group * AT_ONCE, n = min(AT_ONCE, pieces - q);
    if (n <= 0) break;                                   // (the same for all lanes of a set)
    const long long at = (long long)(slot + q) * Q4_ROWS + rr;
    f32x2 ml = {-3e38f, 0.f};
    if (j < n) ml = *reinterpret_cast<const f32x2*>(sc.part_ml + (at + (long long)j * Q4_ROWS) * 2);
    f32x4 w[AT_ONCE][2];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const f32x4* src = reinterpret_cast<const f32x4*>(sc.part_acc + (at + (long long)min(u, n - 1) * Q4_ROWS) * DH + part * 8);
      w[u][0] = src[0]; w[u][1] = src[1];
    }
    float top = ml[0];
#pragma unroll
    for (int d = 1; d < AT_ONCE; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float mn = fmaxf(M, top), shrink = __builtin_amdgcn_exp2f(M - mn);
    const float f = __builtin_amdgcn_exp2f(ml[0] - mn);  // this lane's piece
    float add = f * ml[1];
#pragma unroll
    for (int d = 1; d < AT_ONCE; d <<= 1) add += __shfl_xor(add, d);
    M = mn;
    sum = sum * shrink + add;
#pragma unroll
    for (int u = 0; u < 8; ++u) acc[u] *= shrink;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (u >= n) break;                                 // (no zero times an infinity)
      const float g = __shfl(f, lane0 + u);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] += g * w[u][k / 4][k % 4];
    }
  }
  if (group_shift > 0) {
    if (part == 0) { lds_ml[set][0] = M; lds_ml[set][1] = sum; }
#pragma unroll
    for (int k = 0; k < 8; k += 4) *reinterpret_cast<f32x4*>(&lds_acc[set][part * 8 + k]) = f32x4{acc[k], acc[k + 1], acc[k + 2], acc[k + 3]};
    __syncthreads();
    if (group > 0) return;
    const int groups = min(1 << group_shift, (pieces + AT_ONCE - 1) / AT_ONCE);      // those that had a piece
    float top = M;
    for (int k = 1; k < groups; ++k) top = fmaxf(top, lds_ml[set + k * rows_here][0]);
    const float f0 = __builtin_amdgcn_exp2f(M - top);
    sum *= f0;
#pragma unroll
    for (int u = 0; u < 8; ++u) acc[u] *= f0;
    for (int k = 1; k < groups; ++k) {
      const int o = set + k * rows_here;
      const float f = __builtin_amdgcn_exp2f(lds_ml[o][0] - top);
      sum += f * lds_ml[o][1];
#pragma unroll
      for (int u = 0; u < 8; ++u) acc[u] += f * lds_acc[o][part * 8 + u];
    }
    M = top;
  }
  if (r >= rows) return;
  const int t = rt * Q4_ROWS + r, n = t / p.G;
  const long long orow = (long long)(row0 + n) * p.Hq + head * p.G + (t - n * p.G);
  const float inv = 1.f / sum;
  u32x4 w;
#pragma unroll
  for (int u = 0; u < 4; ++u) w[u] = pack_bf16x2(acc[2 * u] * inv, acc[2 * u + 1] * inv);
  *reinterpret_cast<u32x4*>(reinterpret_cast<bf16_t*>(p.out) + orow * DH + part * 8) = w;
  if (part == 0 && p.lse) p.lse[orow] = (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

// 0 where the call is too large for one launch (2^24 work-groups of 256 threads).
size_t attn_q4_workspace(int batch, int num_kv_heads, int group, int total_rows, int max_kv_len, int max_new_rows, int kv_chunk, int head_dim) {
  const Q4Shape z = q4_shape(batch, num_kv_heads, group, total_rows, max_kv_len, max_new_rows, kv_chunk, head_dim);
  if (z.wgs >= (1ll << 24) || (long long)batch * num_kv_heads * z.rt_max >= (1ll << 24)) return 0;
  return z.total > 0 ? z.total : 256;
}

hipError_t run_attn_q4(const AttnParams& p, const Q4Cache& c, void* workspace, int kv_chunk, hipStream_t st) {
  const Q4Shape z = q4_shape(p.B, p.Hkv, p.G, p.total_rows, p.max_kv_len, p.max_new_rows, kv_chunk, p.D);
  char* ws = reinterpret_cast<char*>(workspace);
  const Q4Sched sc = {z.fixed, z.fixed > 0 ? 1.f / (float)z.fixed : 0.f, z.unit_shift, z.rt_max, (int)z.partials, reinterpret_cast<float*>(ws), reinterpret_cast<float*>(ws + z.off_ml), reinterpret_cast<int2*>(ws + z.off_entries)};
  if (z.wgs == 0) return hipSuccess;
  // Pieces of an item, if the call's items are about equal: four of them to a group of lanes, so that twice as many are one batch (eight: 2 sequences of 272
  // rows 67.7 -> 67.2 us, 1 of 32 768 keys 25.6 -> 25.8; two: 2 of 272 rows 70.3).
  const int sets = 256 / (p.D / 8), most_rows = (int)((long long)p.max_new_rows * p.G < Q4_ROWS ? p.max_new_rows * p.G : Q4_ROWS);
  const long long pieces = z.fixed > 0 ? z.max_pieces : z.max_pieces < Q4_SLOTS / z.items ? z.max_pieces : Q4_SLOTS / z.items;
  int group_shift = 0;
  while ((4ll << group_shift) < pieces && (2 << group_shift) <= sets) ++group_shift;
  const dim3 grid((unsigned)((long long)p.B * p.Hkv * z.rt_max), (most_rows + (sets >> group_shift) - 1) / (sets >> group_shift));
  if (p.D == 128) {
    if (p.B <= 64) hipLaunchKernelGGL((attn_q4_kernel<128, true>), dim3((unsigned)z.wgs), dim3(Q4_BLOCK), 0, st, p, c, sc);
    else hipLaunchKernelGGL((attn_q4_kernel<128, false>), dim3((unsigned)z.wgs), dim3(Q4_BLOCK), 0, st, p, c, sc);
    hipLaunchKernelGGL(attn_q4_combine_kernel<128>, grid, dim3(256), 0, st, p, sc, group_shift);
  } else {
    if (p.B <= 64) hipLaunchKernelGGL((attn_q4_kernel<64, true>), dim3((unsigned)z.wgs), dim3(Q4_BLOCK), 0, st, p, c, sc);
    else hipLaunchKernelGGL((attn_q4_kernel<64, false>), dim3((unsigned)z.wgs), dim3(Q4_BLOCK), 0, st, p, c, sc);
    hipLaunchKernelGGL(attn_q4_combine_kernel<64>, grid, dim3(256), 0, st, p, sc, group_shift);
  }
  return hipGetLastError();
}

}  // namespace fd
