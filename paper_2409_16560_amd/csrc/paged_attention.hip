// Attention of a chunk of new tokens over a paged cache (dsbd_paged_attention).
//
// The rows of a KV head of one sequence are its new tokens times the query heads of the group, token-major: row r is token
// r / group, head r % group, so whatever shares keys shares a workgroup.  Up to 32 rows: the wave-private kernel, which streams the
// caches; above, the tile kernel, which is bound by its matrix products and exponentials.  Either cuts the keys into parts where
// there are fewer rows than the device takes at once; the parts' results (unnormalised output, reference exponent, sum) are joined
// by a second kernel.
//
// Wave-private kernel: each of the 4 waves takes 32-token steps of its own from memory through registers, a step ahead, into its
// LDS tiles;
//   S^T = K Q^T    MFMA 16x16x32, Q^T held in registers: a lane owns one query row, so the softmax stays inside the lane;
//   O^T += V^T P^T MFMA 16x16x32, P^T from the registers of S^T, V^T by the transposing LDS read.
// 8 heads of 128, bf16: one token for each of 64 sequences of 8192 tokens 342 us (6.3 TB/s of K and V; a plain streaming read makes
// 7.0); of 32 sequences of 1024 to 8192 tokens 111 us (5.8 TB/s); two of 32 tokens, 4 heads of 64, 6 us.
#include "common.h"
#include "paged.h"
#include "wave_f64.h"
#include <algorithm>

namespace {

#define PA_BLOCK 256
#define PA_STEP 32                 // tokens per wave step
#define PA_SLOTS 512               // workgroups of the wave-private kernel that the device holds (70 KB of LDS each)
#define PA_MIN_STEPS 4             // steps that a part has at least (one token behind each of 2 x 511, 32 heads: 11.9 us; with 8 14.0)
#define PA_TILE 64                 // tokens per tile
#define PA_TILE_SLOTS 512          // workgroups of 4 waves of the tile kernel that the device holds; half as many of 8

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) u32x4 gvec;

// The two element types.  Softmax numerators are rounded to the type for the product with V (half a step of each term: what the
// matrix units take); they are taken against a reference exponent that trails the row's maximum: SHIFT below it when it is set,
// raised when a score exceeds it by more than SLACK.  bf16 has the exponent range for any slack; 2^16 is rarely passed and leaves the
// sums of fp32, which end at 2^128, room for values of 2^100.  f16 ends at 2^16, and starts to lose bits at 2^-14: the shift keeps
// what is 2^-22 of the largest at full precision.  MOST: a sum of 32 numerators that is within the slack (f16: that does not hold one
// beyond the type's range).
template <typename T> struct Elem;
template <> struct Elem<__bf16> {
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  static constexpr float SLACK = 16.f, SHIFT = 0.f, MOST = 0x1p21f;
  static __device__ __forceinline__ floatx4 mfma(x8 a, x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ floatx16 mfma(x8 a, x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static constexpr unsigned INF = 0x7f80u;
};
template <> struct Elem<_Float16> {
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  static constexpr float SLACK = 15.f, SHIFT = 8.f, MOST = 0x1p15f;
  static __device__ __forceinline__ floatx4 mfma(x8 a, x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ floatx16 mfma(x8 a, x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static constexpr unsigned INF = 0x7c00u;
};

struct PagedAttnArgs {
  PagedArgs c;
  const void *k_pages, *v_pages, *q;
  long long q_tok, q_head, o_tok, o_head;      // elements
  void* out;
  float* lse;
  const uint64_t* anc;
  int n_rows, Hq, Hkv;
  FastDiv group, heads;                        // query heads per KV head; KV heads
  float scale_log2;                            // scale * log2(e): scores are kept in the log2 domain
  int page_run;                                // pages are whole multiples of this many tokens (8, or 1)
  int splits;                                  // whether units may be split
  float* part_o;                               // [grid][rows per block][D]
  float* part_ml;                              // [grid][rows per block][2]
  int2* row_parts;                             // [n_rows*Hq] first partial row, how many parts
  long long part_rows;                         // rows of part_o
  int block_rows;
  long long apart, shift;                      // row of part k > 0 of a row: the first one's + k * apart - shift
  int join;                                    // (row, head) per wave of the join kernel
  int per_head;                                // ranges of the wave-private kernel
  int32_t* fault;
};

struct Seq { int first, n, ctx; bool good, torn; };     // torn: no rows of the call
__device__ __forceinline__ Seq sequence(const PagedAttnArgs& a, int s) {
  Seq q;
  q.first = a.c.q_off[s]; q.ctx = a.c.ctx_len[s];
  const int next = a.c.q_off[s + 1];
  q.torn = q.first < 0 || next > a.n_rows || next < q.first;
  const bool rows = !q.torn && next > q.first;
  q.n = rows ? next - q.first : 0;
  q.good = rows && q.n <= a.c.max_new && q.ctx >= 0 && q.ctx <= a.c.max_len - q.n && !(a.anc && q.n > 64);
  if (!q.good) q.ctx = 0;
  return q;
}

struct Unit { int s, g, rb, part, nparts; };

// Which unit (sequence, block of rows, KV head) a workgroup of the tile kernel has, and which part of it: lengths lie in device
// memory, so every wave works it out for itself, a lane per sequence, 64 at a time.
//   Units that the device does not hold at once: longest first, so that they end together; what is a quarter longer than an even
//   share is cut.
//   (Three chunks of 600 to 2100 tokens behind up to 4100, 432 units for 256 workgroups: sequence by sequence, cut at the even share,
//   228 us, longest first 211, cut a quarter later 195.)
//   (One sequence, whose blocks are in order as they are, or more than 64: one by one, cut at the even share.)
//   Fewer: even parts of at most `len` tiles, where len is the shortest, to within a sixteenth, that makes no more parts than the
//   device holds workgroups (or, of more than 64 sequences, one that certainly does); so units that are more than half of that many
//   and alike are not cut.
//   (Behind 8192 tokens, 32 heads on 8, cut at the even share, in two rounds, and as it is: 56 trees of 31 nodes 434 us, 384; a chunk
//   of 1536 tokens 301, 256; three of 400 to 600 277, 234.)
// False: nothing to do.
__device__ __forceinline__ bool find_unit(const PagedAttnArgs& a, int slots, Unit& u, int& part_tiles) {
  const int lane = threadIdx.x & 63, rows = a.block_rows;
  // The head changes fastest: workgroups go to the 8 dies in turn, so that with 8 heads or a multiple what a die has in hand shares
  // the keys in its L2.
  const int at = quotient(a.heads, blockIdx.x);
  u.g = blockIdx.x - at * a.Hkv;
  Seq q;
  int nrb, longest, have = -1;                 // this lane's sequence: blocks of rows, tiles that its last block sees
  auto measure = [&](int s0) {
    if (s0 == have) return;
    have = s0; nrb = 0; longest = 0;
    if (s0 + lane < a.c.n_seqs) {
      q = sequence(a, s0 + lane);
      if (q.torn) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
      nrb = (int)(((long long)q.n * a.group.d + rows - 1) / rows);
      longest = q.good ? (q.ctx + q.n + PA_TILE - 1) / PA_TILE : 1;
    }
  };
  const bool several = a.c.n_seqs > 1 && a.c.n_seqs <= 64;      // (the blocks of one sequence are in order as they are)
  double seen = 0.0, full = 0.0, units = 0.0;  // tiles that the blocks see, about; as if all saw the last one's
  if (a.splits || several) {
    for (int s0 = 0; s0 < a.c.n_seqs; s0 += 64) {
      measure(s0);
      const int first = !q.good || a.anc ? longest : (q.ctx + min(quotient(a.group, rows), q.n) + PA_TILE - 1) / PA_TILE;
      seen += 0.5 * (double)nrb * ((double)first + (double)longest);
      full += (double)nrb * (double)longest;
      units += (double)nrb;
    }
    units = wave_sum(units) * a.Hkv;
  }
  if (several && units > slots) {
    int cut = a.splits ? max((int)fmin(ceil(1.25 * wave_sum(seen) * a.Hkv / slots), 1e9), PA_MIN_STEPS) : 0x7fffffff;
    // blocks of this lane's sequence that see at least t tiles (the last ones), and the parts that they make
    auto blocks = [&](int t) {
      if (nrb == 0 || t > longest) return 0;
      const long long x = !q.good || a.anc ? 0ll : 64ll * (t - 1) - q.ctx;      // a block sees t tiles if its last token is x or a later one
      return x <= 0 ? nrb : nrb - ((int)(x * a.group.d) >> (__ffs(rows) - 1));      // (rows: a power of two; no more of them than int holds)
    };
    auto parts = [&](int t) {
      int n = blocks(t);
      for (long long more = (long long)cut + 1; more <= longest; more += cut) n += blocks((int)max((long long)t, more));
      return n;
    };
    while (cut < (1 << 29) && wave_sum((double)parts(1)) * a.Hkv > (double)gridDim.x) cut *= 2;
    auto upto = [&](int n) {                   // inclusive sum over the lanes
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(n, d); if (lane >= d) n += o; }
      return n;
    };
    // the number of tiles t that the unit sees: more than `at` parts have t or more, at most `at` more than t
    int lo = 0, hi = longest + 1;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) hi = max(hi, __shfl_xor(hi, d));
    hi = __builtin_amdgcn_readfirstlane(hi);     // (the same in all lanes: what depends on it stays in scalar registers)
    cut = __builtin_amdgcn_readfirstlane(cut);
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (wave_sum((double)parts(mid)) > (double)at) lo = mid; else hi = mid;
    }
    if (lo == 0) return false;
    const int behind = parts(lo + 1), mine = parts(lo) - behind;
    const int incl = upto(mine), rank = at - (int)wave_sum((double)behind);
    const unsigned long long m = __ballot(rank >= incl - mine && rank < incl);
    if (!m) return false;
    const int l = (int)__ffsll((long long)m) - 1;
    u.s = l;
    u.nparts = (int)((unsigned)(lo - 1) / (unsigned)cut) + 1;
    part_tiles = (int)((unsigned)(lo + u.nparts - 1) / (unsigned)u.nparts);
    const int rel = rank - __builtin_amdgcn_readlane(incl - mine, l), block = rel / u.nparts;
    u.part = rel - block * u.nparts;
    u.rb = __builtin_amdgcn_readlane(nrb - blocks(lo + 1), l) - 1 - block;
    return u.rb >= 0;
  }
  auto count = [&](int len) { return longest > len ? (int)((unsigned)(longest + len - 1) / (unsigned)len) : 1; };
  int len = 0x7fffffff;
  if (a.splits) {
    len = max((int)fmin(ceil(wave_sum(full) * a.Hkv / slots), 1e9), PA_MIN_STEPS);
    if (2.0 * units <= slots || (units <= slots && a.c.n_seqs <= 64)) {
      auto fits = [&](int l) {
        double n = 0.0;
        for (int s0 = 0; s0 < a.c.n_seqs; s0 += 64) { measure(s0); n += (double)nrb * count(l); }
        return wave_sum(n) * a.Hkv <= slots;
      };
      int hi = 2 * len;                        // enough for slots / 2 units: as many parts of that length, and one more for each
      if (2.0 * units > slots) while (!fits(hi)) { len = hi; hi *= 2; }      // (ends where nothing is cut any more)
      while (hi - len > max(len / 16, 1)) {    // (at least 2 apart: mid lies between them)
        const int mid = (len + hi) / 2;
        if (fits(mid)) hi = mid; else len = mid;
      }
      len = hi;
    } else if (units <= slots) {
      // (no search, which would look at all of them again and again: as many parts of that length as there is room for, and one more
      // for each unit; 301 sequences, one of them long, 36 us, with a search 51)
      len = max(len, (int)fmin(ceil(wave_sum(full) * a.Hkv / (slots - units)), 1e9));
    }
  }
  long long base = 0;
  for (int s0 = 0; s0 < a.c.n_seqs; s0 += 64) {
    measure(s0);
    const int np = count(len);
    int upto = nrb * np;                       // inclusive sum over the lanes
    const int mine = upto;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(upto, d); if (lane >= d) upto += o; }
    const long long begin = base + upto - mine;
    const unsigned long long m = __ballot(at >= begin && at < begin + mine);
    if (m) {
      const int l = (int)__ffsll((long long)m) - 1;
      u.s = s0 + l;
      u.nparts = __builtin_amdgcn_readlane(np, l);
      part_tiles = (int)((unsigned)(__builtin_amdgcn_readlane(longest, l) + u.nparts - 1) / (unsigned)u.nparts);
      const int rel = at - (int)__builtin_amdgcn_readlane((int)begin, l);
      const int n = __builtin_amdgcn_readlane(nrb, l), block = rel / u.nparts;
      u.part = rel - block * u.nparts;
      u.rb = n - 1 - block;                    // blocks that see most first
      return block >= 0 && block < n;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// Bits of the tokens tok0 .. tok0+31 that a row sees: those in front of `limit`, or the context and its mask's bits.
__device__ __forceinline__ uint32_t seen_bits(const PagedAttnArgs& a, int tok0, int limit, int ctx, uint64_t anc) {
  if (!a.anc) {
    const int n = limit - tok0;
    return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
  }
  const int j = tok0 - ctx;
  if (j >= 64) return 0u;
  if (j >= 0) return (uint32_t)(anc >> j);
  if (j <= -32) return 0xffffffffu;
  return (uint32_t)(anc << -j) | ((1u << -j) - 1);
}

template <typename T>
__device__ __forceinline__ bool any_nonfinite(uint4 w) {
  const unsigned e = Elem<T>::INF, m = e | (e << 16);
  auto one = [&](unsigned x) { x &= m; return (x & 0xffffu) == e || (x >> 16) == e; };
  return one(w.x) | one(w.y) | one(w.z) | one(w.w);
}
__device__ __forceinline__ uint4 load16(const void* p) {
  const u32x4 v = __builtin_nontemporal_load((const gvec*)p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
// The wave's own LDS traffic so far is done.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four channels of a finished row, and once per row the log-sum-exp.  `lost`: two bits per channel whose sum is +Inf, -Inf, NaN.
template <typename T, int D>
__device__ __forceinline__ void write_row(const PagedAttnArgs& a, long long row, int head, int part, float M, float L, floatx4 acc, unsigned lost = 0) {
  const float inv = L != 0.f ? 1.f / L : 0.f;
  union { T h[4]; unsigned short b[4]; uint2 u; } pk;
#pragma unroll
  for (int i = 0; i < 4; ++i) pk.h[i] = (T)(L != 0.f ? acc[i] * inv : 0.f);
  if (lost) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned k = (lost >> (2 * i)) & 3;
      if (k) pk.b[i] = (unsigned short)(Elem<T>::INF | (k == 2 ? 0x8000u : k == 3 ? 0x40u | (Elem<T>::INF >> 1) : 0u));
    }
  }
  *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + row * a.o_tok + head * a.o_head + 4 * part) = pk.u;
  if (a.lse && part == 0) a.lse[row * a.Hq + head] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

// The same of a part's row, unnormalised.
template <int D>
__device__ __forceinline__ void write_part(const PagedAttnArgs& a, long long slot, int part, float M, float L, floatx4 acc, unsigned lost) {
  union { floatx4 f; unsigned b[4]; } c;
  c.f = acc;
  if (lost) {
#pragma unroll
    for (int k = 0; k < 4; ++k) if (const unsigned x = (lost >> (2 * k)) & 3) c.b[k] = x == 1 ? 0x7f800000u : x == 2 ? 0xff800000u : 0x7fc00000u;
  }
  *reinterpret_cast<floatx4*>(&a.part_o[slot * D + 4 * part]) = c.f;
  if (part == 0) { a.part_ml[2 * slot] = M; a.part_ml[2 * slot + 1] = L; }
}
// Workgroup barrier that orders LDS traffic only (loads in flight stay in flight).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One lane's value.
__device__ __forceinline__ long long lane_value(long long v, int l) {
  const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)v, l), hi = __builtin_amdgcn_readlane((int)(v >> 32), l);
  return (long long)((unsigned long long)hi << 32 | lo);
}

// Whatever a workgroup has to do: where there are too few (sequence, KV head) to fill the device, the steps of all sequences, one
// behind the other, are cut into `per_head` even ranges, a workgroup each and KV head.  So all workgroups end together whatever the
// lengths are; a range may end one sequence, take others whole and begin another, and has room for two partial results.  (One token for
// each of 32 sequences of 1024 to 8192 tokens: even parts of each sequence 122 us, ranges 111.)  The sequences' lengths lie in
// device memory, so every wave looks for its place itself, a lane per sequence, 64 at a time.
template <typename T, int D, int NRT>
__global__ __launch_bounds__(PA_BLOCK, 2) void paged_wave_kernel(PagedAttnArgs a) {
  typedef typename Elem<T>::x8 x8;
  constexpr int TW = PA_BLOCK / 64;
  constexpr int DS = D / 32, DT = D / 16, ROWS = 16 * NRT;
  constexpr int LPR = D / 8, TG = 64 / LPR, ROUNDS = PA_STEP / TG;
  constexpr int KP = D + 8, OP = D + 4;
  static_assert(ROWS * OP * 4 <= 2 * PA_STEP * KP * 2, "a wave's partial output takes the place of its tiles");
  __shared__ __attribute__((aligned(16))) T tiles[TW][2 * PA_STEP * KP];
  __shared__ float wave_ml[TW][ROWS][2];
  // two bits per row and channel whose sum is +Inf, -Inf or NaN (both)
  __shared__ unsigned lost[ROWS][D / 16];
  __shared__ int any_lost;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, qd = lane >> 4;
  const int b = quotient(a.heads, blockIdx.x), g = blockIdx.x - b * a.Hkv;      // (workgroups go to the 8 dies in turn)
  // ---- this workgroup's range, and the sequence that it begins in
  int s0 = 0, steps = 0;                       // the first of the 64 sequences at hand; steps of this lane's
  long long begin = 0, base = 0, next = 0;     // where they begin; where the first does, and the one behind the last
  auto scan = [&](int from, long long at) {
    s0 = from; steps = 0; base = at;
    if (s0 + lane < a.c.n_seqs) {
      const Seq q = sequence(a, s0 + lane);
      if (q.torn) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
      steps = q.n == 0 ? 0 : q.good ? (q.ctx + q.n + PA_STEP - 1) / PA_STEP : 1;
    }
    long long upto = steps;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const long long o = __shfl_up(upto, d); if (lane >= d) upto += o; }
    begin = base + upto - steps;
    next = base + lane_value(upto, 63);
  };
  long long x = 0, x_end = 0, per = 0;
  if (a.splits) {
    scan(0, 0);
    while (s0 + 64 < a.c.n_seqs) scan(s0 + 64, next);
    per = lane_value(max((long long)ceil((double)next / a.per_head), (long long)PA_MIN_STEPS), 0);
    x = b * per;
    x_end = min(x + per, next);
    if (x >= x_end) return;
    if (s0 > 0) scan(0, 0);
  }
  do {
    int s = b, st_begin = 0, st_end = 0x7fffffff, nparts = 1;
    if (a.splits) {
      unsigned long long m = __ballot(x >= begin && x < begin + steps);
      while (!m) {
        if (s0 + 64 >= a.c.n_seqs) return;
        scan(s0 + 64, next);
        m = __ballot(x >= begin && x < begin + steps);
      }
      const int l = (int)__ffsll((long long)m) - 1;
      s = s0 + l;
      const long long first = lane_value(begin, l);
      const int n = __builtin_amdgcn_readlane(steps, l);
      st_begin = (int)(x - first);
      st_end = (int)min(x_end - first, (long long)n);
      if (st_begin == 0) nparts = 1 + (int)((unsigned)(first - b * per + n - 1) / (unsigned)per);
      else nparts = 2;                         // (or more)
      x = first + st_end;
    }
    const Seq sq = sequence(a, s);
    const int R = sq.n * a.group.d, len = sq.ctx + sq.n;
    if (g == 0 && st_begin == 0 && threadIdx.x == 0 && (sq.torn || (sq.n > 0 && !sq.good))) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
    if (R == 0) return;                        // (no range has it)
    if (!sq.good) {                            // (any number of rows)
      for (long long i = threadIdx.x; i < (long long)R * (D / 4); i += PA_BLOCK) {
        const int r = (int)(i / (D / 4)), part = (int)(i % (D / 4)), tok = quotient(a.group, r), head = g * a.group.d + r - tok * a.group.d;
        write_row<T, D>(a, sq.first + tok, head, part, -INFINITY, 0.f, floatx4{0.f, 0.f, 0.f, 0.f});
        if (a.splits && part == 0) a.row_parts[(long long)(sq.first + tok) * a.Hq + head] = make_int2(0, 1);
      }
      continue;
    }
    st_end = min(st_end, (len + PA_STEP - 1) / PA_STEP);
    for (int i = threadIdx.x; i < ROWS * (D / 16); i += PA_BLOCK) lost[i / (D / 16)][i % (D / 16)] = 0;
    if (threadIdx.x == 0) any_lost = 0;
    lds_barrier();

    // ---- query rows
    x8 qf[NRT][DS];
    int limit[NRT];
    uint64_t anc[NRT];
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
      const int r = 16 * rt + col;
      const bool live = r < R;
      const int tok = quotient(a.group, live ? r : 0), head = g * a.group.d + (live ? r - tok * a.group.d : 0);
      limit[rt] = live ? sq.ctx + tok + 1 : 0;
      anc[rt] = live && a.anc ? a.anc[sq.first + tok] : 0ull;
      const T* qp = static_cast<const T*>(a.q) + (long long)(sq.first + tok) * a.q_tok + head * a.q_head + 8 * qd;
#pragma unroll
      for (int j = 0; j < DS; ++j) {
        union { u32x4 u; x8 v; } c;
        c.u = u32x4{0, 0, 0, 0};
        if (live) c.u = *(const gvec*)(qp + 32 * j);
        qf[rt][j] = c.v;
      }
    }
    floatx4 o[NRT][DT];
    float m_ref[NRT], l_run[NRT];
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
      m_ref[rt] = -INFINITY; l_run[rt] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[rt][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    T* const kt = tiles[wave];
    T* const vt = kt + PA_STEP * KP;
    const int piece = lane % LPR, ld_tok = ROUNDS * (lane / LPR);    // this lane loads tokens ld_tok .. ld_tok+ROUNDS-1 of a step
    const long long hoff = (long long)g * a.c.head_stride + 8 * piece;
    const T* const kp = static_cast<const T*>(a.k_pages) + hoff;
    const T* const vp = static_cast<const T*>(a.v_pages) + hoff;
    const int32_t* const table = a.c.page_table + (long long)s * a.c.table_stride;
    uint4 kr[ROUNDS], vr[ROUNDS];
    unsigned ok;                      // bit k: the lane's token k is there
    auto load_step = [&](int st) {
      const int t0 = st * PA_STEP + ld_tok;
      ok = 0;
      long long off = 0;
      bool there = false;
#pragma unroll
      for (int k = 0; k < ROUNDS; ++k) {
        const int t = t0 + k;
        if (k == 0 || a.page_run < ROUNDS) {
          const int p = quotient(a.c.page, min(t, len - 1));
          const int page = p < a.c.table_stride ? table[p] : -1;
          there = page >= 0 && page < a.c.n_pages;
          off = there ? (long long)page * a.c.page_stride + (long long)(min(t, len - 1) - p * a.c.page.d) * a.c.token_stride : 0;
          if (!there && t < len) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
        } else off += t < len ? a.c.token_stride : 0;
        kr[k] = vr[k] = make_uint4(0, 0, 0, 0);
        if (there && t < len) { kr[k] = load16(kp + off); vr[k] = load16(vp + off); ok |= 1u << k; }
      }
    };
    int st = st_begin + wave;
    if (st < st_end) load_step(st);
    const int open = sq.ctx + (a.anc ? 0 : 1);   // tokens in front of this are seen by all rows
    for (; st < st_end; st += TW) {
      const int tok0 = st * PA_STEP;
      uint32_t valid = 0xffffffffu;
      const bool whole = __all(ok == (1u << ROUNDS) - 1);
      if (!whole) {
        valid = 0;
#pragma unroll
        for (int k = 0; k < TG; ++k) valid |= (uint32_t)__builtin_amdgcn_readlane((int)ok, k * LPR) << (ROUNDS * k);
      }
      const bool masked = !whole || tok0 + PA_STEP > open;
      bool odd = false;                // values that no product with 0 makes 0
      if (masked) {
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) odd |= any_nonfinite<T>(vr[k]);
      }
      wave_lds_fence();
#pragma unroll
      for (int k = 0; k < ROUNDS; ++k) {
        *reinterpret_cast<uint4*>(&kt[(ld_tok + k) * KP + 8 * piece]) = kr[k];
        *reinterpret_cast<uint4*>(&vt[(ld_tok + k) * KP + 8 * piece]) = vr[k];
      }
      if (odd) {
        // NaN or Inf among values that not all rows see: a product with a numerator of 0 would be NaN, so they leave the tile, and the
        // rows that see them are marked.
        unsigned short* const e = reinterpret_cast<unsigned short*>(vt + ld_tok * KP + 8 * piece);
#pragma unroll 1
        for (int i = 0; i < 8 * ROUNDS; ++i) {
          const unsigned short v = e[i / 8 * KP + i % 8];
          if ((v & Elem<T>::INF) != Elem<T>::INF) continue;
          e[i / 8 * KP + i % 8] = 0;
          const int c = 8 * piece + i % 8, tok = tok0 + ld_tok + i / 8;
          const unsigned kind = (v & 0x7fffu) != Elem<T>::INF ? 3u : v & 0x8000u ? 2u : 1u;
#pragma unroll 1
          for (int r = 0; r < R; ++r) {
            const int rt = quotient(a.group, r);
            const bool sees = a.anc ? tok < sq.ctx || ((a.anc[sq.first + rt] >> (tok - sq.ctx)) & 1) : tok <= sq.ctx + rt;
            if (sees) atomicOr(&lost[r][c / 16], kind << (2 * (c % 16)));
          }
          any_lost = 1;
        }
      }
      wave_lds_fence();
      if (st + TW < st_end) load_step(st + TW);
      floatx4 x[NRT][2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        x8 kf[DS];
#pragma unroll
        for (int j = 0; j < DS; ++j) kf[j] = *reinterpret_cast<const x8*>(&kt[(16 * tt + col) * KP + 32 * j + 8 * qd]);
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) {
          floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < DS; ++j) acc = Elem<T>::mfma(kf[j], qf[rt][j], acc);
          x[rt][tt] = acc * a.scale_log2;
        }
      }
      if (masked) {
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) {
          const uint32_t b = valid & (limit[rt] ? seen_bits(a, tok0, limit[rt], sq.ctx, anc[rt]) : 0u);
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) if (!((b >> (16 * tt + 4 * qd + i)) & 1)) x[rt][tt][i] = -INFINITY;
        }
      }
      x8 pf[NRT];
#pragma unroll
      for (int rt = 0; rt < NRT; ++rt) {
        float mx = x[rt][0][0];
#pragma unroll
        for (int k = 1; k < 8; ++k) mx = fmaxf(mx, x[rt][k >> 2][k & 3]);
        if (__any(mx > m_ref[rt] + Elem<T>::SLACK)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          if (mx > m_ref[rt] + Elem<T>::SLACK) {
            const float to = mx - Elem<T>::SHIFT;
            const float f = m_ref[rt] == -INFINITY ? 0.f : exp2f(m_ref[rt] - to);
            m_ref[rt] = to;
            l_run[rt] *= f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[rt][dt] *= f;
          }
        }
        const float ref = m_ref[rt] == -INFINITY ? 0.f : m_ref[rt];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float p = __builtin_amdgcn_exp2f(x[rt][k >> 2][k & 3] - ref);
          x[rt][k >> 2][k & 3] = p;
          l_run[rt] += p;
          pf[rt][k] = (T)p;
        }
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        union { v4i16 h[2]; x8 v; } vf;
        const T* rowp = &vt[(4 * qd + (col >> 2)) * KP + 16 * dt + 4 * (col & 3)];
        vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(rowp));
        vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(rowp + 16 * KP));
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) o[rt][dt] = Elem<T>::mfma(vf.v, pf[rt], o[rt][dt]);
      }
    }
    // ---- the waves' results: sums over the lanes of a row, then everything through the LDS
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
      l_run[rt] += __shfl_xor(l_run[rt], 16);
      l_run[rt] += __shfl_xor(l_run[rt], 32);
    }
    float* const po = reinterpret_cast<float*>(tiles[wave]);
    wave_lds_fence();
#pragma unroll
    for (int rt = 0; rt < NRT; ++rt) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<floatx4*>(&po[(16 * rt + col) * OP + 16 * dt + 4 * qd]) = o[rt][dt];
      if (qd == 0) { wave_ml[wave][16 * rt + col][0] = m_ref[rt]; wave_ml[wave][16 * rt + col][1] = l_run[rt]; }
    }
    __syncthreads();
    const long long slot = ((long long)(2 * b + (st_begin == 0)) * a.Hkv + g) * ROWS;
    for (int i = threadIdx.x; i < R * (D / 4); i += PA_BLOCK) {
      const int r = i / (D / 4), part = i % (D / 4);
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < TW; ++w) M = fmaxf(M, wave_ml[w][r][0]);
      floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float m = wave_ml[w][r][0], l = wave_ml[w][r][1];
        if (l == 0.f) continue;                    // the wave's steps had nothing for this row
        const float f = m == M ? 1.f : exp2f(m - M);
        L += l * f;
        acc += *reinterpret_cast<const floatx4*>(&reinterpret_cast<const float*>(tiles[w])[r * OP + 4 * part]) * f;
      }
      const int tok = quotient(a.group, r), head = g * a.group.d + r - tok * a.group.d;
      const long long row = sq.first + tok;
      const unsigned gone = any_lost ? (lost[r][part / 4] >> (8 * (part % 4))) & 255u : 0u;
      if (nparts == 1) write_row<T, D>(a, row, head, part, M, L, acc, gone);
      else write_part<D>(a, slot + r, part, M, L, acc, gone);
      if (a.splits && part == 0 && st_begin == 0) a.row_parts[row * a.Hq + head] = make_int2((int)slot + r, nparts);
    }
    __syncthreads();                             // (the LDS, for the next)
    if (a.splits && x < x_end) scan(s0, base);     // (again: the registers have had other use)
  } while (a.splits && x < x_end);
}

// ---- tile kernel: many rows on the same keys
//
// Four or eight waves of 32 rows share tiles of 64 tokens of K and V in the LDS, two of each, filled by direct loads (no registers
// in between) a tile ahead; the pieces of a row are swizzled by the token, so that the operand reads, which go down the rows,
// spread over the banks.  MFMA 32x32x16: S^T = K Q^T and O^T += V^T P^T as in the wave-private kernel, a lane owns a query row
// together with the lane 32 further on, which has the other half of its tokens.

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void glb_cvoid;

// NW: waves, 4 where 128 rows hold all of a sequence's (two workgroups per CU), 8 above (one, which fills a tile for twice the rows):
// 8 trees of 31 nodes with 4 heads per KV head on 8192 tokens 78 us against 93; a prompt of 8192 tokens, 32 heads of 128, 599 us
// against 556; three chunks of 600 to 2100 tokens, 4 heads per KV head, 199 us against 200.  RUNS: pages are whole multiples of 8
// tokens, so what a load instruction takes begins at one address and needs no place of its own in every lane (the prompt 616 us
// against 655, in an earlier form of 4 waves).
template <typename T, int D, int NW, bool RUNS>
__global__ __launch_bounds__(64 * NW, 2) void paged_tile_kernel(PagedAttnArgs a) {
  typedef typename Elem<T>::x8 x8;
  constexpr int DS = D / 16, DT = D / 32;               // k-steps of S^T, channel tiles of O^T
  constexpr int BLOCK = 64 * NW, ROWS = 32 * NW;
  constexpr int PPR = D / 8, ROWB = 2 * D;              // 16-byte pieces and bytes of a row
  constexpr int TPI = 64 / PPR, ROUNDS = PA_TILE / (NW * TPI);    // tokens per load instruction, instructions per wave and tile
  __shared__ uint4 kA[PA_TILE * PPR], kB[PA_TILE * PPR], vA[PA_TILE * PPR], vB[PA_TILE * PPR];
  // two bits per row and channel whose sum is +Inf, -Inf or NaN (both)
  __shared__ unsigned lost[ROWS][D / 16];
  __shared__ int any_lost;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, h = lane >> 5;
  Unit u;
  int part_tiles;
  if (!find_unit(a, PA_TILE_SLOTS * 4 / NW, u, part_tiles)) return;
  const Seq sq = sequence(a, u.s);
  const int R = sq.n * a.group.d, row0 = u.rb * ROWS, len = sq.ctx + sq.n;
  if (u.g == 0 && u.rb == 0 && u.part == 0 && threadIdx.x == 0 && !sq.good) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
  const int last_tok = quotient(a.group, min(row0 + ROWS, R) - 1), first_tok = quotient(a.group, row0);
  const int upto = !sq.good ? 0 : a.anc ? len : sq.ctx + last_tok + 1;
  const int tiles = (upto + PA_TILE - 1) / PA_TILE;
  const int t_begin = u.nparts == 1 ? 0 : (int)min((long long)u.part * part_tiles, (long long)tiles);
  const int t_end = a.c.n_pages == 0 ? t_begin : u.nparts == 1 ? tiles : min(tiles, t_begin + part_tiles);
  if (a.c.n_pages == 0 && threadIdx.x == 0) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
  const int open = sq.ctx + (a.anc ? 0 : first_tok + 1);      // tokens in front of this are seen by all rows

  // ---- where tokens lie.  Tokens without a page read page 0, tokens behind the last whatever is in the last one's page; both are
  // masked.
  const int32_t* const table = a.c.page_table + (long long)u.s * a.c.table_stride;
  // swizzles: K is read down 16 tokens at one piece, V down 8 tokens at 4 pieces in a row
  auto swz_k = [](int t) { return D == 128 ? t & 15 : (t >> 1) & 7; };
  auto swz_v = [](int t) { return D == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1); };
  constexpr int RUN = NW * TPI;                // tokens per round of the waves
  const int ld_tok = TPI * wave + lane / PPR, ld_k = (lane % PPR) ^ swz_k(ld_tok), ld_v = (lane % PPR) ^ swz_v(ld_tok);
  static_assert(RUN % 16 == 0, "a round is a whole number of swizzle periods");
  const char* const kp = static_cast<const char*>(a.k_pages) + 2 * (long long)u.g * a.c.head_stride;
  const char* const vp = static_cast<const char*>(a.v_pages) + 2 * (long long)u.g * a.c.head_stride;
  const unsigned k_lane = (unsigned)(lane / PPR * 2 * (int)a.c.token_stride + 16 * ld_k), v_lane = (unsigned)(lane / PPR * 2 * (int)a.c.token_stride + 16 * ld_v);
  // lane l: the page of token l of a tile
  auto look_up = [&](int ti) __attribute__((always_inline)) {
    const int p = quotient(a.c.page, min(ti * PA_TILE + lane, len - 1));
    return p < a.c.table_stride ? table[p] : -1;
  };
  // which tokens of a tile are there, a bit each
  auto present = [&](int ti, int page) __attribute__((always_inline)) {
    const int n = len - ti * PA_TILE;
    const unsigned long long inside = n >= 64 ? ~0ull : (1ull << n) - 1, valid = __ballot(page >= 0 && page < a.c.n_pages);
    if (inside & ~valid) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
    return valid & inside;
  };
  // where token l of a tile lies, in bytes (RUNS: where the run of tokens that a load instruction takes begins, which lies in one page)
  auto offset = [&](int ti, int page) __attribute__((always_inline)) {
    const int t = min(ti * PA_TILE + lane, RUNS ? (len - 1) & ~(TPI - 1) : len - 1);
    page = page >= 0 && page < a.c.n_pages ? page : 0;
    return 2 * ((long long)page * a.c.page_stride + (long long)(t - quotient(a.c.page, t) * a.c.page.d) * a.c.token_stride);
  };
  // this wave's part of a tile of K and V
  auto issue = [&](int ti, int page, auto& Kb, auto& Vb) __attribute__((always_inline)) {
    const long long off = offset(ti, page);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if constexpr (RUNS) {
        const int from = RUN * r + TPI * wave;
        const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)off, from), hi = __builtin_amdgcn_readlane((int)(off >> 32), from);
        const long long o = (long long)((unsigned long long)hi << 32 | lo);
        __builtin_amdgcn_global_load_lds((glb_cvoid*)(kp + o + k_lane), (lds_void*)&Kb[(NW * r + wave) * 64], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((glb_cvoid*)(vp + o + v_lane), (lds_void*)&Vb[(NW * r + wave) * 64], 16, 0, 0);
      } else {
        const unsigned lo = __shfl((int)(unsigned)off, RUN * r + ld_tok), hi = __shfl((int)(off >> 32), RUN * r + ld_tok);
        const long long o = (long long)((unsigned long long)hi << 32 | lo);
        __builtin_amdgcn_global_load_lds((glb_cvoid*)(kp + o + 16 * ld_k), (lds_void*)&Kb[(NW * r + wave) * 64], 16, 0, 0);
        __builtin_amdgcn_global_load_lds((glb_cvoid*)(vp + o + 16 * ld_v), (lds_void*)&Vb[(NW * r + wave) * 64], 16, 0, 0);
      }
    }
  };

  // ---- query rows
  x8 qf[DS];
  const int my_row = row0 + 32 * wave + col;
  const bool live = my_row < R;
  const int my_tok = quotient(a.group, live ? my_row : row0);
  const int limit = live ? sq.ctx + my_tok + 1 : 0;
  const uint64_t anc = live && a.anc ? a.anc[sq.first + my_tok] : 0ull;
  {
    const int head = u.g * a.group.d + (live ? my_row - my_tok * a.group.d : 0);
    const T* qp = static_cast<const T*>(a.q) + (long long)(sq.first + my_tok) * a.q_tok + head * a.q_head + 8 * h;
#pragma unroll
    for (int j = 0; j < DS; ++j) {
      union { u32x4 u; x8 v; } c;
      c.u = u32x4{0, 0, 0, 0};
      if (live) c.u = *(const gvec*)(qp + 16 * j);
      qf[j] = c.v;
    }
  }
  floatx16 o[DT];
  float m_ref = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  // byte offsets of the operand reads inside a tile: K token col, piece 2j + h; V token 4h + (lane % 16) / 4, channels
  // 16 * (lane / 16 % 2) + 4 * (lane % 4) of a tile of 32
  int k_off[DS], v_off[DT];
#pragma unroll
  for (int j = 0; j < DS; ++j) k_off[j] = col * ROWB + (((2 * j + h) ^ swz_k(col)) << 4);
  {
    const int t = 4 * h + ((lane & 15) >> 2), c = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v_off[dt] = t * ROWB + (((4 * dt + (c >> 3)) ^ swz_v(t)) << 4) + ((c & 4) << 1);
  }

  // Operands are read from the LDS four at a time, a group ahead of the matrix instructions that take them: a group is 128 cycles
  // of the matrix unit, about what the LDS takes to answer.  (Vector instructions may move between.)
#define PA_GROUP() __builtin_amdgcn_sched_barrier(0x406)
  struct Four { x8 v[4]; };
  auto read_k = [&](int g, const char* kl) __attribute__((always_inline)) {      // group g of the tile's 2 DS operands of K
    Four f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = *reinterpret_cast<const x8*>(kl + 32 * (4 * g / DS) * ROWB + k_off[(4 * g + i) % DS]);
    return f;
  };
  auto read_v = [&](int g, const char* vl) __attribute__((always_inline)) {      // of its 4 DT operands of V
    Four f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = 4 * g + i;
      union { v4i16 q[2]; x8 v; } c;
      const char* const rowp = vl + 16 * (n / DT) * ROWB + v_off[n % DT];
      c.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(rowp));
      c.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(rowp + 8 * ROWB));
      f.v[i] = c.v;
    }
    return f;
  };
  auto mask = [&](uint32_t valid, int tok0, floatx16& s) __attribute__((always_inline)) {
    const uint32_t b = (valid & (limit ? seen_bits(a, tok0, limit, sq.ctx, anc) : 0u)) >> (4 * h);
#pragma unroll
    for (int i = 0; i < 16; ++i) if (!((b >> (8 * (i >> 2) + (i & 3))) & 1)) s[i] = -INFINITY;
  };
  // the row's reference, raised where a score of the tile is too far above
  auto refer = [&](const floatx16& s0, const floatx16& s1) __attribute__((always_inline)) {
    // (NaN is never the larger.  The start is hidden from the compiler, which otherwise takes the maximum of every tile, in front of
    // the branch that few tiles take: a prompt of 8192 tokens, 32 heads, 624 us against 577.)
    float m = -INFINITY;
    asm volatile("" : "+v"(m));
#pragma unroll
    for (int i = 0; i < 16; ++i) { m = s0[i] > m ? s0[i] : m; m = s1[i] > m ? s1[i] : m; }
    m *= a.scale_log2;
    m = fmaxf(m, __shfl_xor(m, 32));
    const float to = m > m_ref + Elem<T>::SLACK ? m - Elem<T>::SHIFT : m_ref;
    const float f = to == m_ref ? 1.f : exp2f(m_ref - to);
    m_ref = to;
    l_run *= f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
  };
  // numerators of half a tile, and their sum
  auto soften = [&](const floatx16& s, x8 (&pf)[2]) __attribute__((always_inline)) {
    const float ref = m_ref == -INFINITY ? 0.f : -m_ref;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale_log2, ref));
      sum += p;
      pf[i >> 3][i & 7] = (T)p;
    }
    return sum;
  };
  // NaN or Inf among values that not all rows see: a product with a numerator of 0 would be NaN, so they leave the tile, and the
  // rows that see them are marked.
  auto sanitize = [&](int tok0, unsigned long long valid, auto& Vb) __attribute__((always_inline)) {
    for (int i = threadIdx.x; i < PA_TILE * PPR; i += BLOCK) {
      if (!any_nonfinite<T>(Vb[i])) continue;
      const int t = i / PPR, piece = (i % PPR) ^ swz_v(t);
      unsigned short* const e = reinterpret_cast<unsigned short*>(&Vb[i]);
      for (int k = 0; k < 8; ++k) {
        const unsigned short x = e[k];
        if ((x & Elem<T>::INF) != Elem<T>::INF) continue;
        e[k] = 0;
        if (!((valid >> t) & 1)) continue;
        const int c = 8 * piece + k;
        const unsigned kind = (x & 0x7fffu) != Elem<T>::INF ? 3u : x & 0x8000u ? 2u : 1u;
        for (int rl = 0; rl < ROWS && row0 + rl < R; ++rl) {
          const int tok = quotient(a.group, row0 + rl);
          const bool sees = a.anc ? tok0 + t < sq.ctx || ((a.anc[sq.first + tok] >> (tok0 + t - sq.ctx)) & 1) : tok0 + t <= sq.ctx + tok;
          if (sees) atomicOr(&lost[rl][c / 16], kind << (2 * (c % 16)));
        }
        any_lost = 1;
      }
    }
    lds_barrier();
  };
  auto compute = [&](int ti, unsigned long long valid, auto& Kb, auto& Vb) __attribute__((always_inline)) {
    const char* const kl = reinterpret_cast<const char*>(&Kb[0]);
    const char* const vl = reinterpret_cast<const char*>(&Vb[0]);
    const int tok0 = ti * PA_TILE;
    const bool masked = valid != ~0ull || tok0 + PA_TILE > open;
    if (masked) sanitize(tok0, valid, Vb);
    floatx16 s[2];
    x8 p[2][2];
    float sum = 0.f;
    constexpr int KG = 2 * DS / 4, VG = 4 * DT / 4;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[hf][i] = 0.f;
    Four now = read_k(0, kl);
#pragma unroll
    for (int g = 0; g < KG; ++g) {
      const Four next = g + 1 < KG ? read_k(g + 1, kl) : read_v(0, vl);
      PA_GROUP();
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * g / DS] = Elem<T>::mfma(now.v[i], qf[(4 * g + i) % DS], s[4 * g / DS]);
      PA_GROUP();
      now = next;
    }
    if (masked) { mask((uint32_t)valid, tok0, s[0]); mask((uint32_t)(valid >> 32), tok0 + 32, s[1]); }
    // Rows that have seen nothing so far need a reference first.  Scores far above one show in the sums (no maximum of all scores
    // is needed for that): then once more with a new one.
    bool raise = __any(m_ref == -INFINITY);
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
      if (raise) refer(s[0], s[1]);
      sum = soften(s[0], p[0]) + soften(s[1], p[1]);
      raise = __any(!(sum <= Elem<T>::MOST));
      if (!raise) break;
    }
    l_run += sum;
#pragma unroll
    for (int g = 0; g < VG; ++g) {
      Four next = now;
      if (g + 1 < VG) next = read_v(g + 1, vl);
      PA_GROUP();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = 4 * g + i, ks = n / DT;
        o[n % DT] = Elem<T>::mfma(now.v[i], p[ks >> 1][ks & 1], o[n % DT]);
      }
      PA_GROUP();
      now = next;
    }
  };
  for (int i = threadIdx.x; i < ROWS * (D / 16); i += BLOCK) lost[i / (D / 16)][i % (D / 16)] = 0;
  if (threadIdx.x == 0) any_lost = 0;
  // One barrier per tile: every wave's part of it has landed, and everybody is done with the buffers that are filled next.
  if (t_begin < t_end) {
    int ti = t_begin;
    int page = look_up(ti);
    unsigned long long valid = present(ti, page), valid_next = 0;
    issue(ti, page, kA, vA);
    page = look_up(ti + 1);
    auto tile = [&](auto& K, auto& K_next, auto& V, auto& V_next) __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0)
      lds_barrier();
      if (ti + 1 < t_end) {
        valid_next = present(ti + 1, page);
        issue(ti + 1, page, K_next, V_next);
        page = look_up(ti + 2);
      }
      compute(ti, valid, K, V);
      valid = valid_next;
      ++ti;
    };
    while (true) {
      tile(kA, kB, vA, vB);
      if (ti >= t_end) break;
      tile(kB, kA, vB, vA);
      if (ti >= t_end) break;
    }
  }
  __syncthreads();                             // the buffers become the output staging: a part per wave
  l_run += __shfl_xor(l_run, 32);
  constexpr int QPR = D / 4, HALF = QPR / 2;   // 4-channel pieces of a row; they go through the LDS half a row at a time
  constexpr int PER = NW / 4;                  // waves per buffer
  static_assert(PER * 32 * HALF <= PA_TILE * PPR, "the output staging fits the buffers");
  uint4* const stage = (wave < PER ? kA : wave < 2 * PER ? kB : wave < 3 * PER ? vA : vB) + wave % PER * 32 * HALF;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    wave_lds_fence();
#pragma unroll
    for (int dt = 0; dt < DT / 2; ++dt)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        union { floatx4 f; uint4 u; } c;
#pragma unroll
        for (int i = 0; i < 4; ++i) c.f[i] = o[half * (DT / 2) + dt][4 * k + i];
        stage[col * HALF + ((8 * dt + 2 * k + h) ^ (col & 7))] = c.u;
      }
    wave_lds_fence();
#pragma unroll 4
    for (int i = lane; i < 32 * HALF; i += 64) {
      const int rl = i / HALF, q = i % HALF, part = half * HALF + q, r = row0 + 32 * wave + rl;
      const float M = __shfl(m_ref, rl), L = __shfl(l_run, rl);
      if (r >= R) continue;
      union { uint4 u; floatx4 f; } c;
      c.u = stage[rl * HALF + (q ^ (rl & 7))];
      const int tok = quotient(a.group, r), head = u.g * a.group.d + r - tok * a.group.d;
      const long long row = sq.first + tok, slot = (long long)blockIdx.x * ROWS + 32 * wave + rl;
      const unsigned gone = any_lost ? (lost[32 * wave + rl][part / 4] >> (8 * (part % 4))) & 255u : 0u;
      if (u.nparts == 1) {
        write_row<T, D>(a, row, head, part, M, L, c.f, gone);
      } else {
        write_part<D>(a, slot, part, M, L, c.f, gone);
      }
      if (a.splits && part == 0 && u.part == 0) a.row_parts[row * a.Hq + head] = make_int2((int)slot, u.nparts);
    }
  }
}

// A wave takes `join` (row, head) and joins those that were split: one, or, where there are so many that most were not, up to 4, which
// are looked up together (107808 of them, none split: one each 10.6 us, four 4.5; 7936, all of 8 parts: one each 8.3 us).  Groups of
// lanes take every GROUPS-th part, four at a time, and carry a maximum and a sum of their own, so that nothing but the list of parts
// is waited for before they are loaded.
template <typename T, int D>
__global__ __launch_bounds__(PA_BLOCK) void paged_join_kernel(PagedAttnArgs a) {
  const unsigned n = (unsigned)a.n_rows * (unsigned)a.Hq, base = (blockIdx.x * (PA_BLOCK / 64) + (threadIdx.x >> 6)) * (unsigned)a.join;
  const int lane = threadIdx.x & 63;
  if (base >= n) return;
  int2 mine = make_int2(0, 0);                 // this lane's (row, head): its first part and their number
  bool split = false;
  if (lane < a.join && base + lane < n) {
    mine = a.row_parts[base + lane];
    const int row = (int)((base + lane) / (unsigned)a.Hq);
    split = row >= a.c.q_off[0] && row < a.c.q_off[a.c.n_seqs] &&       // (not padding)
            mine.y > 1 && mine.x >= 0 && mine.x + (mine.y - 1) * a.apart - a.shift < a.part_rows;
  }
  constexpr int PIECES = D / 4, GROUPS = 64 / PIECES, AHEAD = 4;
  const int part = lane % PIECES, grp = lane / PIECES;
  const floatx4 none = {0.f, 0.f, 0.f, 0.f};
  for (unsigned long long m = __ballot(split); m; m &= m - 1) {
    const int who = (int)__ffsll((long long)m) - 1;
    const int2 rp = make_int2(__builtin_amdgcn_readlane(mine.x, who), __builtin_amdgcn_readlane(mine.y, who));
    const int row = (int)((base + who) / (unsigned)a.Hq), head = (int)((base + who) % (unsigned)a.Hq);
    floatx4 acc = none;
    float M = -INFINITY, L = 0.f;
    for (int k0 = grp; k0 < rp.y; k0 += AHEAD * GROUPS) {
      float x[AHEAD], l[AHEAD];
      floatx4 v[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int k = k0 + i * GROUPS;
        const int in = k < rp.y ? k : k0;
        const long long at = rp.x + (in > 0 ? in * a.apart - a.shift : 0);
        x[i] = a.part_ml[2 * at];
        l[i] = k < rp.y ? a.part_ml[2 * at + 1] : 0.f;
        v[i] = *reinterpret_cast<const floatx4*>(&a.part_o[at * D + 4 * part]);
      }
      float to = M;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) to = l[i] != 0.f ? fmaxf(to, x[i]) : to;      // (sums of 0: the part had nothing for this row)
      const float f = to == M ? 1.f : exp2f(M - to);
      L *= f;
      acc *= f;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const float g = x[i] == to ? 1.f : exp2f(x[i] - to);
        L += l[i] != 0.f ? l[i] * g : 0.f;
        acc += l[i] != 0.f ? v[i] * g : none;
      }
      M = to;
    }
    float to = M;
#pragma unroll
    for (int d = PIECES; d < 64; d <<= 1) to = fmaxf(to, __shfl_xor(to, d));
    const float f = M == to ? 1.f : exp2f(M - to);
    L *= f;
    acc *= f;
#pragma unroll
    for (int d = PIECES; d < 64; d <<= 1) {
      L += __shfl_xor(L, d);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], d);
    }
    if (grp == 0) write_row<T, D>(a, row, head, part, to, L, acc);
  }
}

// How a call is cut up.
struct Plan {
  int rows;                  // per block: 16 and 32 wave-private kernel, 128 and 256 tile kernel
  long long grid;
  bool splits;
  size_t bytes;
};
Plan plan(const dsbd_paged_kv* c, int n_rows, int Hq, int Hkv, int D, PagedAttnArgs* a, void* workspace) {
  Plan p;
  const long long group = Hq / Hkv, most = (long long)std::min(c->max_new, n_rows) * group;     // rows of a sequence and KV head
  // (17 to 32 rows, in the wave-private kernel and in the tile kernel: 7 nodes for each of 32 sequences of 1024 to 8192 tokens, 4 heads per
  // KV head, 127 us against 142; for each of 8 sequences of 8000 tokens, where the rule takes the slower one, 71 us against 64)
  p.rows = most <= 16 ? 16 : most <= 32 ? 32 : most <= 128 ? 128 : 256;
  const bool wave = p.rows <= 32;
  const long long slots = wave ? PA_SLOTS : p.rows == 128 ? PA_TILE_SLOTS : PA_TILE_SLOTS / 2;
  // Few units: what is split may be joined, in a workspace that depends on the shapes alone.  Sequences of up to 256 tokens
  // stay whole all the same: one token for each of 2 sequences of 255 tokens, 32 heads, 10.2 us against 11.9; of 511, 14.0 against 11.9.
  const long long units = wave ? (long long)c->n_seqs * Hkv : ((long long)n_rows * group / p.rows + c->n_seqs) * Hkv;      // at most
  const bool few = units < 2 * slots;
  const int per_head = (int)std::max<long long>(slots / Hkv, 1);
  p.splits = few && c->max_len > 256;
  const long long parts = wave ? 2ll * per_head * Hkv : units + (slots + Hkv - 1) / Hkv * Hkv;
  p.grid = wave ? p.splits ? (long long)per_head * Hkv : units : p.splits ? parts : units;
  WorkspaceCarver w(workspace);
  float *po = nullptr, *ml = nullptr;
  int2* rp = nullptr;
  if (few) {
    rp = w.take<int2>((size_t)n_rows * Hq);
    ml = w.take<float>((size_t)parts * p.rows * 2);
    po = w.take<float>((size_t)parts * p.rows * D);
  }
  p.bytes = std::max<size_t>(w.total(), 256);
  if (a) {
    a->splits = p.splits; a->part_o = po; a->part_ml = ml; a->row_parts = rp;
    a->part_rows = parts * p.rows; a->block_rows = p.rows; a->per_head = per_head;
    a->apart = (wave ? 2 : 1) * (long long)Hkv * p.rows; a->shift = wave ? (long long)Hkv * p.rows : 0;
  }
  return p;
}

int32_t check(const dsbd_paged_kv* cache, int32_t n_rows, int32_t Hq, int32_t Hkv, int32_t D) {
  if (!cache) return DSBD_ERR_INVALID;
  if (Hq < 1 || Hkv < 1 || Hq % Hkv) return DSBD_ERR_INVALID;
  if (D != 64 && D != 128) return DSBD_ERR_UNSUPPORTED;
  if (Hq > 65535 || (long long)n_rows * Hq > (1ll << 30)) return DSBD_ERR_UNSUPPORTED;
  return DSBD_OK;
}

}  // namespace

extern "C" size_t dsbd_paged_attention_workspace_bytes(const dsbd_paged_kv* cache, int32_t n_rows, int32_t Hq, int32_t Hkv, int32_t D) {
  if (check(cache, n_rows, Hq, Hkv, D) != DSBD_OK || n_rows < 0 || cache->n_seqs < 0 || cache->max_new < 0) return 0;
  return plan(cache, n_rows, Hq, Hkv, D, nullptr, nullptr).bytes;
}

extern "C" int32_t dsbd_paged_attention(const dsbd_paged_kv* cache, int32_t n_rows, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype,
                                        const dsbd_rows* q, float scale, const uint64_t* anc_mask, const dsbd_rows* out, float* lse,
                                        void* workspace, size_t workspace_bytes, int32_t* fault, void* stream_) {
  int32_t rc = check(cache, n_rows, Hq, Hkv, D);
  if (rc != DSBD_OK) return rc;
  if (dtype != DSBD_BF16 && dtype != DSBD_F16) return DSBD_ERR_UNSUPPORTED;
  rc = paged_check(cache, n_rows, Hkv);
  if (rc != DSBD_OK) return rc;
  if (anc_mask && cache->max_new > 64) return DSBD_ERR_UNSUPPORTED;
  if (n_rows == 0 || cache->n_seqs == 0) return DSBD_OK;
  if (!q || !out || !q->ptr || !out->ptr || !fault || !workspace) return DSBD_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(q->ptr) | reinterpret_cast<uintptr_t>(out->ptr)) & 15) return DSBD_ERR_INVALID;
  if (q->token_stride < 0 || q->head_stride < 0 || out->token_stride < 0 || out->head_stride < 0) return DSBD_ERR_INVALID;
  if ((q->token_stride | q->head_stride | out->token_stride | out->head_stride) & 7) return DSBD_ERR_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return DSBD_ERR_INVALID;
  PagedAttnArgs a;
  const Plan p = plan(cache, n_rows, Hq, Hkv, D, &a, workspace);
  if (workspace_bytes < p.bytes) return DSBD_ERR_WORKSPACE;
  if (a.part_rows > 0x7fffffffLL || p.grid > 0x7fffffffLL) return DSBD_ERR_UNSUPPORTED;
  a.c = paged_args(cache);
  a.k_pages = cache->k_pages; a.v_pages = cache->v_pages; a.q = q->ptr; a.out = out->ptr; a.lse = lse; a.anc = anc_mask;
  a.q_tok = q->token_stride; a.q_head = q->head_stride; a.o_tok = out->token_stride; a.o_head = out->head_stride;
  a.n_rows = n_rows; a.Hq = Hq; a.Hkv = Hkv; a.group = fast_div(Hq / Hkv); a.heads = fast_div(Hkv);
  a.scale_log2 = (float)((scale > 0.f ? (double)scale : 1.0 / sqrt((double)D)) * 1.4426950408889634);
  // (the tile kernel's short way adds a lane's place in a run of tokens as a 32-bit number of bytes)
  a.page_run = cache->page_size % 8 == 0 && cache->token_stride < (1 << 25) ? 8 : 1;
  a.fault = fault;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  const dim3 grid((unsigned)p.grid), block(PA_BLOCK);
  a.join = (int)std::min(4ll, 1 + (long long)n_rows * Hq / 16384);
  const dim3 join((unsigned)(((long long)n_rows * Hq + a.join * (PA_BLOCK / 64) - 1) / (a.join * (PA_BLOCK / 64))));
#define PA_TILES(T, DD, NW)                                                                                \
  do {                                                                                                     \
    if (a.page_run == 8) hipLaunchKernelGGL((paged_tile_kernel<T, DD, NW, true>), grid, dim3(64 * NW), 0, stream, a); \
    else hipLaunchKernelGGL((paged_tile_kernel<T, DD, NW, false>), grid, dim3(64 * NW), 0, stream, a);     \
  } while (0)
#define PA_ROWS(T, DD)                                                                                     \
  do {                                                                                                     \
    if (p.rows == 16) hipLaunchKernelGGL((paged_wave_kernel<T, DD, 1>), grid, block, 0, stream, a);        \
    else if (p.rows == 32) hipLaunchKernelGGL((paged_wave_kernel<T, DD, 2>), grid, block, 0, stream, a);   \
    else if (p.rows == 128) PA_TILES(T, DD, 4);                                                            \
    else PA_TILES(T, DD, 8);                                                                               \
    DSBD_HIP_LAUNCH_CHECK();                                                                               \
    if (p.splits) hipLaunchKernelGGL((paged_join_kernel<T, DD>), join, block, 0, stream, a);               \
  } while (0)
#define PA_TYPES(DD) do { if (dtype == DSBD_BF16) PA_ROWS(__bf16, DD); else PA_ROWS(_Float16, DD); } while (0)
  if (D == 128) PA_TYPES(128);
  else PA_TYPES(64);
#undef PA_TYPES
#undef PA_ROWS
#undef PA_TILES
  DSBD_HIP_LAUNCH_CHECK();
  return DSBD_OK;
}
