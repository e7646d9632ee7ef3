// Rules on logits (dsbd_process_logits): repetition, frequency and presence penalties, biases, temperature and grammar masks on
// the rows of a draft forest, in one pass over the logits.
//
// A workgroup takes a chunk of the vocabulary for a few rows.  How often a token occurs is counted in the LDS, a word per
// token of the chunk: the text in front of a tree's root, scanned once for all the rows of that tree that the workgroup has
// (integer atomics, so the order does not matter).  The tokens of the tree's nodes are marked there with the node that has them
// first; what a row's path adds is then the population count of (its ancestors & the nodes with that token).  Every thread keeps
// the places of its 16 tokens that have a word or a bias as a bit per piece and streams row after row, without a barrier between rows of a tree, the
// next row's loads on their way during a row's arithmetic.
// Bound by HBM: logits are read once and written once, a piece that a mask excludes as a whole is not read at all: 191 rows of 128256
// f32 with every rule 47.8 us, 198 MB at 4.1 TB/s (a large copy makes 5.2).  By latency where there are few rows: 7 us.
#include "common.h"
#include "paged.h"
#include "topology_device.h"
#include "wave_f64.h"
#include <algorithm>

namespace {

#define LG_BLOCK 256
#define LG_CHUNK 4096              // tokens of the vocabulary per workgroup
#define LG_SLOTS 1024              // workgroups that the device holds at once (4 per compute unit, by their LDS)
// a token's word:
#define LG_SEEN 0x80000000u        // it occurs in the prompt
#define LG_NODE 0x40000000u        // a node of the tree has it: its number behind LG_NODE_AT
#define LG_NODE_AT 24
#define LG_TIMES 0x00ffffffu       // how often it was generated in front of the root

struct LogitArgs {
  int n_rows, V, n_chunks;
  int groups;                      // workgroups per chunk
  // forest
  int n_prompts, n_trees, n_nodes, max_tree_nodes, max_depth;
  const int32_t *tree_prompt, *tree_off, *parent, *token, *row_node;
  const void* z;
  long long z_stride, out_stride;
  float* out;
  const int32_t *hist, *hist_off, *prompt_len;
  const float *repetition, *frequency, *presence, *temperature;
  const int32_t *bias_off, *bias_token;
  const float* bias_value;
  const uint32_t* mask;
  const int32_t* mask_row;
  long long mask_stride;
  int n_masks, n_hist, n_bias;
  int vec;                         // rows of logits, of out and of masks allow 4 values at a time
  int32_t* fault;
};

// Four logits as they lie in memory.
template <typename T> struct Piece {
  typedef unsigned int raw __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ void one(raw& v, int e, T x) {
    union { T t; unsigned short u; } c;
    c.t = x;
    v[e >> 1] = e & 1 ? (v[e >> 1] & 0xffffu) | (unsigned)c.u << 16 : (v[e >> 1] & 0xffff0000u) | c.u;
  }
  static __device__ __forceinline__ float value(raw v, int e) {
    union { unsigned short u; T t; } c;
    c.u = (unsigned short)(v[e >> 1] >> (16 * (e & 1)));
    return (float)c.t;
  }
};
template <> struct Piece<float> {
  typedef unsigned int raw __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ void one(raw& v, int e, float x) { v[e] = __float_as_uint(x); }
  static __device__ __forceinline__ float value(raw v, int e) { return __uint_as_float(v[e]); }
};

// Quotients by one number: the product with its reciprocal, corrected by what it leaves of the dividend, which a fused multiply-add
// knows exactly.  Off by half a step, or by 2^-130 where that is more (of numbers between 1 and 2, 5e9 quotients by 600 divisors are
// the divided ones to the last bit); divisors far from 1, and dividends that the correction makes NaN (Inf), are divided.
// (191 rows of 128256, f32, every rule: 47.8 us; everything divided 54, products with a rounded reciprocal alone 46.5.)
struct Divisor {
  float d, inv;
  bool near_1;
  __device__ __forceinline__ explicit Divisor(float v) : d(v), inv(1.f / v), near_1(v >= 0x1p-20f && v <= 0x1p20f) {}
  __device__ __forceinline__ void over(float (&x)[4]) const {      // (one branch for the four)
    float q[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      q[e] = x[e] * inv;
      q[e] = fmaf(fmaf(-q[e], d, x[e]), inv, q[e]);
    }
    const bool odd = !near_1 || __builtin_isunordered(q[0], q[1]) || __builtin_isunordered(q[2], q[3]);
    if (odd) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] = x[e] / d;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = q[e];
  }
};

// Pieces of 4 tokens that a thread has of a row.
constexpr int LG_PIECES = LG_CHUNK / (4 * LG_BLOCK);
constexpr int LG_TEXT = 16;                  // tokens of a text in flight per thread

template <typename T>
__global__ __launch_bounds__(LG_BLOCK) void logits_kernel(LogitArgs a) {
  typedef typename Piece<T>::raw raw;
  __shared__ __attribute__((aligned(16))) uint32_t words[LG_CHUNK];
  __shared__ __attribute__((aligned(16))) float bias[LG_CHUNK];
  __shared__ uint64_t anc[64];               // ancestors of the tree's nodes
  __shared__ uint64_t same[64];              // nodes with the token of a node
  const int tid = threadIdx.x, lane = tid & 63;
  const int chunk = blockIdx.x % a.n_chunks, group = blockIdx.x / a.n_chunks;
  const int v0 = chunk * LG_CHUNK, nv = min(LG_CHUNK, a.V - v0);
  const bool counts = a.repetition || a.frequency || a.presence;
  int bad = 0;
  bool known = true;               // the rows belong to nodes (one of row_node may belong to nothing: it is copied)

  // ---- rows on their way, one in front of the one in hand: the bits of a row's mask first, then the pieces that it does not
  // exclude as a whole
  struct Row { uint32_t bits[LG_PIECES]; raw x[LG_PIECES]; };
  Row now, next;
  auto load_bits = [&](int r, Row& to) {
    const uint32_t* mrow = nullptr;
    if (a.mask && known) {
      const int mi = a.mask_row ? a.mask_row[r] : r;
      if (mi >= a.n_masks) bad |= DSBD_FAULT_BOUNDS;
      else if (mi >= 0) mrow = a.mask + mi * a.mask_stride;
    }
#pragma unroll
    for (int k = 0; k < LG_PIECES; ++k) {
      const unsigned i = 4 * (threadIdx.x + k * LG_BLOCK);
      const int n = nv - (int)i;
      to.bits[k] = n >= 4 ? 15u : n > 0 ? (1u << n) - 1 : 0u;
      if (mrow && n > 0) to.bits[k] &= mrow[(v0 + i) >> 5] >> ((v0 + i) & 31);
    }
  };
  auto load_row = [&](int r, Row& to) {
    const T* const zr = static_cast<const T*>(a.z) + r * a.z_stride + v0;
#pragma unroll
    for (int k = 0; k < LG_PIECES; ++k) {
      const unsigned i = 4 * (threadIdx.x + k * LG_BLOCK);
      if (!to.bits[k]) continue;
      if (a.vec && (int)i + 4 <= nv) to.x[k] = __builtin_nontemporal_load((const __attribute__((address_space(1))) raw*)(zr + i));
      else
        for (int e = 0; e < 4; ++e) if ((int)i + e < nv) Piece<T>::one(to.x[k], e, zr[i + e]);
    }
  };

  // What there is to know of all trees and prompts, a lane each (if they are that few), in one trip to memory; otherwise it
  // takes two, and a search for the row's tree.
  const bool few = a.n_trees < 64 && a.n_prompts < 64 && a.n_trees > 0 && a.n_prompts > 0;
  int l_off = 0, l_prompt = 0, l_plen = 0, l_held = 0, l_bias = 0;
  float l_rep = 1.f, l_freq = 0.f, l_pres = 0.f, l_temp = 1.f;
  if (few) {
    const int t = min(lane, a.n_trees - 1), t1 = min(lane, a.n_trees), p = min(lane, a.n_prompts - 1), p1 = min(lane, a.n_prompts);
    l_off = a.tree_off[t1];
    l_prompt = a.tree_prompt[t];
    if (a.prompt_len) l_plen = a.prompt_len[t];
    if (a.hist_off) l_held = a.hist_off[t1];
    if (a.bias_off) l_bias = a.bias_off[p1];
    if (a.repetition) l_rep = a.repetition[p];
    if (a.frequency) l_freq = a.frequency[p];
    if (a.presence) l_pres = a.presence[p];
    if (a.temperature) l_temp = a.temperature[p];
  }
  const auto lane_f = [](float v, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };

  // ---- the workgroup's tree and rows: a number of the nodes of a tree, or the one row of row_node
  int t = -1, r0 = 0, r1 = 0, node0 = 0, base = 0, end = 0, lo = 0, hi = 0, plen = 0, prompt = -1, blo = 0, bhi = 0;
  int segments = 1, segment = 0;                // of a tree's nodes
  if (a.row_node) {
    r0 = group; r1 = r0 + 1;
    node0 = __builtin_amdgcn_readfirstlane(a.row_node[r0]);
    if (node0 >= 0 && node0 < a.n_nodes) {
      if (few) {
        const unsigned long long m = __ballot(lane <= a.n_trees && l_off <= node0);
        t = m ? 63 - __builtin_clzll(m) : -1;
      } else t = __builtin_amdgcn_readfirstlane(last_at_most(a.tree_off, a.n_trees + 1, node0, [](int v, int) { return v; }));
      if (t >= a.n_trees) t = -1;
    }
  } else if (few) {
    // as few nodes per workgroup as there are workgroups for (all of a tree's, at most: groups >= n_trees)
    const int from = l_off, to = __shfl_down(l_off, 1);
    const bool valid = lane < a.n_trees && from >= 0 && to <= a.n_nodes && to > from;
    const int n = valid ? min(to - from, DSBD_MAX_TREE_NODES) : 0;
    int per = max(1, ((int)wave_sum_f32((float)n) + a.groups - 1) / a.groups), mine = 0;
    for (; per <= DSBD_MAX_TREE_NODES; ++per) {
      mine = (n + per - 1) / per;
      if ((int)wave_sum_f32((float)mine) <= a.groups) break;
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const int o = __shfl_up(upto, d); if (lane >= d) upto += o; }
    if (group == 0 && lane < a.n_trees && !valid) bad |= DSBD_FAULT_TOPOLOGY;
    const unsigned long long m = __ballot(group >= upto - mine && group < upto);
    if (m) {
      t = (int)__ffsll((long long)m) - 1;
      segments = __builtin_amdgcn_readlane(mine, t);
      segment = group - (__builtin_amdgcn_readlane(upto, t) - segments);
    }
  } else {
    segments = a.groups / a.n_trees;
    t = group / segments;
    segment = group - t * segments;
    if (t >= a.n_trees) t = -1;
  }
  if (t >= 0) {
    if (few) {
      base = __builtin_amdgcn_readlane(l_off, t); end = __builtin_amdgcn_readlane(l_off, t + 1);
      prompt = __builtin_amdgcn_readlane(l_prompt, t); plen = __builtin_amdgcn_readlane(l_plen, t);
      lo = __builtin_amdgcn_readlane(l_held, t); hi = __builtin_amdgcn_readlane(l_held, t + 1);
    } else {
      base = a.tree_off[t]; end = a.tree_off[t + 1]; prompt = a.tree_prompt[t];
      if (a.prompt_len) plen = a.prompt_len[t];
      if (a.hist_off) { lo = a.hist_off[t]; hi = a.hist_off[t + 1]; }
    }
  }
  dsbd_tree_range tr = {0, 0, 0, a.row_node ? DSBD_FAULT_TOPOLOGY : 0, false};
  if (t >= 0) tr = dsbd_tree_range_between(base, end, a.n_nodes, a.max_tree_nodes);
  const int n_b = tr.valid ? tr.n : 0;
  bad |= tr.bad;
  if (!a.row_node) {
    if (n_b > 0) { r0 = base + n_b * segment / segments; r1 = base + n_b * (segment + 1) / segments; }
    node0 = r0;
    if (r0 >= r1) {
      if (chunk == 0 && bad) atomicOr(a.fault, bad);
      return;
    }
  }
  known = node0 >= base && node0 < base + n_b;
  if (!known) bad |= DSBD_FAULT_TOPOLOGY;
  if (t >= 0 && (prompt < 0 || prompt >= a.n_prompts)) { prompt = -1; bad |= DSBD_FAULT_TOPOLOGY; }
  if (lo < 0 || hi < lo || hi > a.n_hist || hi - lo > (int)LG_TIMES) { lo = hi = 0; bad |= DSBD_FAULT_BOUNDS; }
  float rep = 1.f, freq = 0.f, pres = 0.f, temp = 1.f;
  if (prompt >= 0) {
    if (few) {
      rep = lane_f(l_rep, prompt); freq = lane_f(l_freq, prompt); pres = lane_f(l_pres, prompt); temp = lane_f(l_temp, prompt);
      blo = __builtin_amdgcn_readlane(l_bias, prompt); bhi = __builtin_amdgcn_readlane(l_bias, prompt + 1);
    } else {
      if (a.repetition) rep = a.repetition[prompt];
      if (a.frequency) freq = a.frequency[prompt];
      if (a.presence) pres = a.presence[prompt];
      if (a.temperature) temp = a.temperature[prompt];
      if (a.bias_off) { blo = a.bias_off[prompt]; bhi = a.bias_off[prompt + 1]; }
    }
    if (!(rep > 0.f)) { rep = 1.f; bad |= DSBD_FAULT_BOUNDS; }
    if (!(temp > 0.f)) { temp = 1.f; bad |= DSBD_FAULT_BOUNDS; }
    if (blo < 0 || bhi < blo || bhi > a.n_bias) { blo = bhi = 0; bad |= DSBD_FAULT_BOUNDS; }
  }
  // the nodes of the tree, a lane each, in every wave; the first tokens of the text and of the bias list and the first row
  // travel meanwhile
  const int p_mine = dsbd_tree_parent_of(tr, lane, a.parent);
  int tok = lane < n_b ? a.token[base + lane] : -1;
  int text[LG_TEXT];
  const bool scan = counts && hi > lo;
  if (scan) {
#pragma unroll
    for (int k = 0; k < LG_TEXT; ++k) text[k] = a.hist[(unsigned)min(lo + tid + k * LG_BLOCK, hi - 1)];
  }
  const int b_tok = bhi > blo ? a.bias_token[min(blo + tid, bhi - 1)] : 0;
  const float b_val = bhi > blo ? a.bias_value[min(blo + tid, bhi - 1)] : 0.f;
  load_bits(r0, now);
  for (int i = 4 * tid; i < LG_CHUNK; i += 4 * LG_BLOCK) {
    *reinterpret_cast<uint4*>(&words[i]) = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(&bias[i]) = make_uint4(0, 0, 0, 0);
  }
  if (r0 + 1 < r1) load_bits(r0 + 1, next);
  uint64_t mine = 0;
  bad |= dsbd_tree_walk(tr, lane, p_mine, a.max_depth, nullptr, nullptr, &mine);
  if (lane < n_b && (tok < 0 || tok >= a.V)) { bad |= DSBD_FAULT_TOKEN; tok = -1; }
  // a node's place in the text of its path is held + depth: generated from prompt_len on
  const uint64_t made_nodes = __ballot(lane < n_b && (long long)(hi - lo) + __popcll(mine) - 1 >= plen);
  uint64_t twins = 0;
  if (counts && tid < 64) {
    for (int j = 0; j < n_b; ++j) twins |= (uint64_t)(tok == __builtin_amdgcn_readlane(tok, j)) << j;
    anc[lane] = mine;
    same[lane] = twins;
  }
  __syncthreads();
  if (bhi > blo) {
    // the last of a token's entries: 1 + its number, in the place of the word; then its value
    for (int i = blo + tid; i < bhi; i += LG_BLOCK) {
      const int v = i == blo + tid ? b_tok : a.bias_token[i];
      if ((unsigned)v >= (unsigned)a.V) bad |= DSBD_FAULT_TOKEN;
      else if ((unsigned)(v - v0) < (unsigned)nv) atomicMax(&words[v - v0], (uint32_t)(i - blo) + 1u);
    }
    __syncthreads();
    for (int i = blo + tid; i < bhi; i += LG_BLOCK) {
      const bool first = i == blo + tid;
      const int v = first ? b_tok : a.bias_token[i];
      if ((unsigned)(v - v0) < (unsigned)nv && words[v - v0] == (uint32_t)(i - blo) + 1u) bias[v - v0] = first ? b_val : a.bias_value[i];
    }
    __syncthreads();
    for (int i = 4 * tid; i < LG_CHUNK; i += 4 * LG_BLOCK) *reinterpret_cast<uint4*>(&words[i]) = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  // the text: what has arrived is counted with the next tokens and the first two rows on their way
  int more[LG_TEXT];
  auto load_text = [&](int i0) {
#pragma unroll
    for (int k = 0; k < LG_TEXT; ++k) more[k] = a.hist[(unsigned)min(i0 + k * LG_BLOCK, hi - 1)];
  };
  if (scan && lo + LG_TEXT * LG_BLOCK < hi) load_text(lo + LG_TEXT * LG_BLOCK + tid);
  load_row(r0, now);
  if (r0 + 1 < r1) load_row(r0 + 1, next);
  if (scan) {
    for (int i0 = lo;;) {
#pragma unroll
      for (int k = 0; k < LG_TEXT; ++k) {
        const int i = i0 + tid + k * LG_BLOCK, v = text[k];
        if (i < hi) {
          if ((unsigned)v >= (unsigned)a.V) bad |= DSBD_FAULT_TOKEN;
          else if ((unsigned)(v - v0) < (unsigned)nv) {      // (one that was generated has a count: no mark needed)
            if (i - lo >= plen) atomicAdd(&words[v - v0], 1u);
            else atomicOr(&words[v - v0], LG_SEEN);
          }
        }
      }
      i0 += LG_TEXT * LG_BLOCK;
      if (i0 >= hi) break;
#pragma unroll
      for (int k = 0; k < LG_TEXT; ++k) text[k] = more[k];
      if (i0 + LG_TEXT * LG_BLOCK < hi) load_text(i0 + LG_TEXT * LG_BLOCK + tid);
    }
  }
  // the tokens of the tree's nodes: the number of the first node that has it
  if (counts && tid < 64 && (unsigned)(tok - v0) < (unsigned)nv && (int)__ffsll((long long)twins) - 1 == lane)
    atomicOr(&words[tok - v0], LG_NODE | (uint32_t)lane << LG_NODE_AT);
  __syncthreads();
  uint32_t rare = 0;                         // bit k: a token of piece k has a word or a bias
#pragma unroll
  for (int k = 0; k < LG_PIECES; ++k) {
    const int at = 4 * (tid + k * LG_BLOCK);
    const uint4 q = *reinterpret_cast<const uint4*>(&words[at]), b = *reinterpret_cast<const uint4*>(&bias[at]);
    if (q.x | q.y | q.z | q.w | b.x | b.y | b.z | b.w) rare |= 1u << k;
  }
  // ---- the rows
  if (!known) rare = 0;
  const Divisor by_temp(known ? temp : 1.f), by_rep(rep);
  for (int r = r0; r < r1; ++r) {
    if (r > r0 && r + 1 < r1) { load_bits(r + 1, next); load_row(r + 1, next); }
    const uint64_t path = known && counts ? anc[node0 + (r - r0) - base] : 0ull;
    float* const outr = a.out + r * a.out_stride + v0;
#pragma unroll
    for (int k = 0; k < LG_PIECES; ++k) {
      const unsigned i = 4 * (threadIdx.x + k * LG_BLOCK);
      if ((int)i >= nv) continue;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = Piece<T>::value(now.x[k], e);
      if ((rare >> k) & 1) {
        const uint4 q4 = *reinterpret_cast<const uint4*>(&words[i]), b4 = *reinterpret_cast<const uint4*>(&bias[i]);
        const uint32_t qs[4] = {q4.x, q4.y, q4.z, q4.w}, bs[4] = {b4.x, b4.y, b4.z, b4.w};
        float less[4] = {x[0], x[1], x[2], x[3]};
        if (rep != 1.f) by_rep.over(less);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t q = qs[e];
          float y = x[e];
          if (q) {
            uint32_t times = q & LG_TIMES;
            bool seen = (q & (LG_SEEN | LG_TIMES)) != 0;
            if (q & LG_NODE) {
              const uint64_t here = path & same[(q >> LG_NODE_AT) & 63];
              seen |= here != 0;
              times += (uint32_t)__popcll(here & made_nodes);
            }
            if (seen) y = y > 0.f ? less[e] : y * rep;
            if (times) y = y - freq * (float)times - pres;
          }
          x[e] = y + __uint_as_float(bs[e]);
        }
      }
      by_temp.over(x);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (now.bits[k] >> e) & 1 ? x[e] : -INFINITY;
      if (a.vec && (int)i + 4 <= nv) {
        typedef float f4 __attribute__((ext_vector_type(4)));
        *(__attribute__((address_space(1))) f4*)(outr + i) = f4{x[0], x[1], x[2], x[3]};
      } else {
        for (int e = 0; e < 4; ++e) if ((int)i + e < nv) outr[i + e] = x[e];
      }
    }
    now = next;
  }
  if (chunk == 0 && bad) atomicOr(a.fault, bad);
}

}  // namespace

extern "C" int32_t dsbd_process_logits(const dsbd_forest* f, const int32_t* row_node, int32_t n_rows, int32_t V, int32_t dtype,
                                       const void* logits, int64_t logits_stride, const dsbd_logit_rules* rules, float* out,
                                       int64_t out_stride, int32_t* fault, void* stream_) {
  if (!f || !rules || !fault || n_rows < 0) return DSBD_ERR_INVALID;
  if (V < 1 || V > (1 << 30) || (dtype != DSBD_F32 && dtype != DSBD_BF16 && dtype != DSBD_F16)) return DSBD_ERR_UNSUPPORTED;
  if (f->n_prompts < 0 || f->n_trees < 0 || f->n_nodes < 0 || logits_stride < V || out_stride < V) return DSBD_ERR_INVALID;
  if (f->max_tree_nodes > DSBD_MAX_TREE_NODES) return DSBD_ERR_UNSUPPORTED;
  // (the kernel's indices run past the ends by a few thousand before they are compared)
  if (f->n_trees > (1 << 30) || rules->n_hist > (1 << 30) || rules->n_bias > (1 << 30)) return DSBD_ERR_UNSUPPORTED;
  if (!row_node && n_rows != f->n_nodes) return DSBD_ERR_INVALID;
  if (n_rows == 0) return DSBD_OK;
  if (!logits || !out || !f->tree_prompt || !f->tree_off || !f->parent || !f->token) return DSBD_ERR_INVALID;
  if (rules->n_hist < 0 || rules->n_bias < 0 || rules->n_masks < 0) return DSBD_ERR_INVALID;
  if (rules->hist_off && rules->n_hist > 0 && !rules->hist) return DSBD_ERR_INVALID;
  if (rules->bias_off && rules->n_bias > 0 && (!rules->bias_token || !rules->bias_value)) return DSBD_ERR_INVALID;
  if (rules->mask && rules->mask_stride < ((int64_t)V + 31) / 32) return DSBD_ERR_INVALID;
  const size_t size = dtype == DSBD_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(out) % 4) return DSBD_ERR_INVALID;
  if (static_cast<const void*>(out) == logits && (dtype != DSBD_F32 || logits_stride != out_stride)) return DSBD_ERR_INVALID;
  LogitArgs a;
  a.n_rows = n_rows; a.V = V;
  a.n_prompts = f->n_prompts; a.n_trees = f->n_trees; a.n_nodes = f->n_nodes;
  a.max_tree_nodes = f->max_tree_nodes; a.max_depth = f->max_depth;
  a.tree_prompt = f->tree_prompt; a.tree_off = f->tree_off; a.parent = f->parent; a.token = f->token; a.row_node = row_node;
  a.z = logits; a.z_stride = logits_stride; a.out = out; a.out_stride = out_stride;
  a.hist = rules->hist; a.hist_off = rules->hist_off; a.prompt_len = rules->prompt_len;
  a.repetition = rules->repetition; a.frequency = rules->frequency; a.presence = rules->presence; a.temperature = rules->temperature;
  a.bias_off = rules->bias_off; a.bias_token = rules->bias_token; a.bias_value = rules->bias_value;
  a.mask = rules->mask; a.mask_row = rules->mask_row; a.mask_stride = rules->mask_stride;
  a.n_masks = rules->n_masks; a.n_hist = rules->n_hist; a.n_bias = rules->n_bias;
  a.fault = fault;
  a.vec = logits_stride % 4 == 0 && out_stride % 4 == 0 && reinterpret_cast<uintptr_t>(logits) % (4 * size) == 0 &&
          reinterpret_cast<uintptr_t>(out) % 16 == 0;
  a.n_chunks = (V + LG_CHUNK - 1) / LG_CHUNK;
  // A workgroup takes as many of a tree's nodes as leaves no more workgroups than the device holds at once: the text is scanned once
  // for all of them (191 nodes of 8 trees behind texts of 8192 tokens, vocabulary 128256: 47 us; a node each 94, whole trees 111, with quotients as products).  Rows of row_node may each have another tree: one row per workgroup.
  a.groups = n_rows;
  if (!row_node) {
    const long long fit = LG_SLOTS / a.n_chunks, most = (long long)f->n_trees * std::max(1, f->max_tree_nodes);
    a.groups = (int)std::max<long long>(f->n_trees, std::min(fit, most));
  }
  const long long wgs = (long long)a.groups * a.n_chunks;
  if (wgs == 0) return DSBD_OK;
  if (wgs > 0x7fffffffLL) return DSBD_ERR_UNSUPPORTED;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  const dim3 grid((unsigned)wgs), block(LG_BLOCK);
  if (dtype == DSBD_F32) hipLaunchKernelGGL((logits_kernel<float>), grid, block, 0, stream, a);
  else if (dtype == DSBD_BF16) hipLaunchKernelGGL((logits_kernel<__bf16>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((logits_kernel<_Float16>), grid, block, 0, stream, a);
  DSBD_HIP_LAUNCH_CHECK();
  return DSBD_OK;
}
