// Rules on logits (dsbd_process_logits): repetition, frequency and presence penalties, biases, temperature and grammar masks on
// the rows of a draft forest, in one pass over the logits.
//
// A workgroup takes a chunk of the vocabulary for a few rows.  How often a token occurs is counted in the LDS, a word per
// token of the chunk: the text in front of a tree's root once for all the rows of that tree that the workgroup has (one scan of
// the list, integer atomics, so the order does not matter), the few nodes of a row's path added in front of the row and taken off
// again behind it.  Then every thread streams its pieces of the row: a token whose word is 0, whose piece has no bias and all
// of whose mask bits are set is only converted.
// Bound by HBM: logits are read once and written once, a piece that a mask excludes as a whole is not read at all.
#include "common.h"
#include "paged.h"
#include "topology_device.h"
#include <algorithm>

namespace {

#define LG_BLOCK 256
#define LG_CHUNK 4096              // tokens of the vocabulary per workgroup
#define LG_SEEN 0x80000000u        // the token occurs in the text; below: times it was generated

struct LogitArgs {
  int n_rows, V, rows_wg, n_chunks;
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

template <typename T>
__device__ __forceinline__ void load4(const T* p, float* x);
template <>
__device__ __forceinline__ void load4<float>(const float* p, float* x) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  const f4 v = *(const __attribute__((address_space(1))) f4*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = v[i];
}
template <>
__device__ __forceinline__ void load4<__bf16>(const __bf16* p, float* x) {
  typedef unsigned int u2 __attribute__((ext_vector_type(2)));
  const u2 v = *(const __attribute__((address_space(1))) u2*)p;
  x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
  x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
template <>
__device__ __forceinline__ void load4<_Float16>(const _Float16* p, float* x) {
  typedef unsigned int u2 __attribute__((ext_vector_type(2)));
  union { u2 u; _Float16 h[4]; } c;
  c.u = *(const __attribute__((address_space(1))) u2*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (float)c.h[i];
}

template <typename T>
__global__ __launch_bounds__(LG_BLOCK) void logits_kernel(LogitArgs a) {
  __shared__ uint32_t words[LG_CHUNK];       // LG_SEEN | times generated
  __shared__ uint32_t bias_at[LG_CHUNK];     // 1 + the number of the token's bias in the prompt's list
  __shared__ uint64_t anc[64];
  __shared__ int node_token[64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int chunk = blockIdx.x % a.n_chunks, group = blockIdx.x / a.n_chunks;
  const int v0 = chunk * LG_CHUNK, nv = min(LG_CHUNK, a.V - v0);
  const int r0 = group * a.rows_wg, r1 = min(a.n_rows, r0 + a.rows_wg);
  const bool reporter = chunk == 0;
  const bool counts = a.repetition || a.frequency || a.presence;
  int tree = -1, base = 0, n_b = 0, held = 0, plen = 0, prompt = -1, bias_lo = 0;
  float rep = 1.f, freq = 0.f, pres = 0.f, temp = 1.f;
  int bad = 0;

  for (int r = r0; r < r1; ++r) {
    const int node = a.row_node ? a.row_node[r] : r;
    int t = -1;
    if (node >= 0 && node < a.n_nodes) t = last_at_most(a.tree_off, a.n_trees + 1, node, [](int v, int) { return v; });
    if (t >= a.n_trees) t = -1;
    t = __builtin_amdgcn_readfirstlane(t);
    if (t != tree || r == r0) {
      // ---- another tree: its topology, its text and its prompt's rules
      tree = t;
      __syncthreads();
      for (int i = tid; i < LG_CHUNK; i += LG_BLOCK) { words[i] = 0; bias_at[i] = 0; }
      n_b = 0; held = 0; plen = 0; prompt = -1;
      rep = 1.f; freq = 0.f; pres = 0.f; temp = 1.f;
      if (t >= 0) {
        const dsbd_tree_range tr = dsbd_tree_range_of(t, a.n_nodes, a.tree_off, a.max_tree_nodes);
        if (tr.valid) { base = tr.base; n_b = tr.n; }
        uint64_t mine = 0;
        const int tb = dsbd_tree_walk(tr, lane, dsbd_tree_parent_of(tr, lane, a.parent), a.max_depth, nullptr, nullptr, &mine);
        if (tid < 64) {
          bad |= tb;
          anc[lane] = mine;
          const int tok = lane < n_b ? a.token[base + lane] : -1;
          if (lane < n_b && (tok < 0 || tok >= a.V)) bad |= DSBD_FAULT_TOKEN;
          node_token[lane] = tok;
        }
        prompt = a.tree_prompt[t];
        if (prompt < 0 || prompt >= a.n_prompts) { prompt = -1; bad |= DSBD_FAULT_TOPOLOGY; }
        plen = a.prompt_len ? a.prompt_len[t] : 0;
        if (prompt >= 0) {
          if (a.repetition) { rep = a.repetition[prompt]; if (!(rep > 0.f)) { rep = 1.f; bad |= DSBD_FAULT_BOUNDS; } }
          if (a.frequency) freq = a.frequency[prompt];
          if (a.presence) pres = a.presence[prompt];
          if (a.temperature) { temp = a.temperature[prompt]; if (!(temp > 0.f)) { temp = 1.f; bad |= DSBD_FAULT_BOUNDS; } }
        }
      }
      __syncthreads();
      if (t >= 0 && a.hist_off) {
        const int lo = a.hist_off[t], hi = a.hist_off[t + 1];
        if (lo >= 0 && hi >= lo && hi <= a.n_hist) {
          held = hi - lo;
          if (counts)
            for (int i = tid; i < held; i += LG_BLOCK) {
              const int tok = a.hist[lo + i];
              if (tok < 0 || tok >= a.V) bad |= DSBD_FAULT_TOKEN;
              else if ((unsigned)(tok - v0) < (unsigned)nv) {
                if (i >= plen) atomicAdd(&words[tok - v0], 1u);
                atomicOr(&words[tok - v0], LG_SEEN);
              }
            }
        } else bad |= DSBD_FAULT_BOUNDS;
      }
      if (prompt >= 0 && a.bias_off) {
        const int lo = a.bias_off[prompt], hi = a.bias_off[prompt + 1];
        if (lo >= 0 && hi >= lo && hi <= a.n_bias) {
          bias_lo = lo;
          for (int i = lo + tid; i < hi; i += LG_BLOCK) {
            const int tok = a.bias_token[i];
            if (tok < 0 || tok >= a.V) bad |= DSBD_FAULT_TOKEN;
            else if ((unsigned)(tok - v0) < (unsigned)nv) atomicMax(&bias_at[tok - v0], (unsigned)(i - lo) + 1u);
          }
        } else bad |= DSBD_FAULT_BOUNDS;
      }
      __syncthreads();
    }
    // ---- the row's path: the lanes of the first wave whose nodes are on it
    const bool known = t >= 0 && node >= base && node - base < n_b;
    if (!known) bad |= DSBD_FAULT_TOPOLOGY;
    int tok = -1;
    bool made = false, was = false;
    if (known && counts && tid < 64) {
      const uint64_t m = anc[node - base];
      if ((m >> lane) & 1) {
        tok = node_token[lane] - v0;
        if ((unsigned)tok >= (unsigned)nv) tok = -1;
        made = held + __popcll(m & ((1ull << lane) - 1)) >= plen;
      }
      if (tok >= 0) {
        if (made) atomicAdd(&words[tok], 1u);
        was = (atomicOr(&words[tok], LG_SEEN) & LG_SEEN) != 0;
      }
    }
    __syncthreads();
    const uint32_t* mrow = nullptr;
    if (a.mask) {
      const int mi = a.mask_row ? a.mask_row[r] : r;
      if (mi >= a.n_masks) bad |= DSBD_FAULT_BOUNDS;
      else if (mi >= 0) mrow = a.mask + mi * a.mask_stride;
    }
    const T* const zr = static_cast<const T*>(a.z) + r * a.z_stride;
    float* const outr = a.out + r * a.out_stride;
    const float f_rep = known ? rep : 1.f, f_temp = known ? temp : 1.f;
    for (int i = 4 * tid; i < nv; i += 4 * LG_BLOCK) {
      const int n = min(4, nv - i);
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t bits = 15u;
      if (mrow) bits = (mrow[(v0 + i) >> 5] >> ((v0 + i) & 31)) & 15u;
      if (a.vec && n == 4) load4<T>(zr + v0 + i, x);
      else for (int e = 0; e < n; ++e) x[e] = (float)zr[v0 + i + e];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = known ? words[i + e] : 0u, b = known ? bias_at[i + e] : 0u;
        float y = x[e];
        if (w & LG_SEEN) y = y > 0.f ? y / f_rep : y * f_rep;
        const uint32_t times = w & ~LG_SEEN;
        if (times) y = y - freq * (float)times - pres;
        if (b) y += a.bias_value[bias_lo + b - 1];
        y = y / f_temp;
        x[e] = (bits >> e) & 1 ? y : -INFINITY;
      }
      if (a.vec && n == 4) {
        typedef float f4 __attribute__((ext_vector_type(4)));
        *(__attribute__((address_space(1))) f4*)(outr + v0 + i) = f4{x[0], x[1], x[2], x[3]};
      } else for (int e = 0; e < n; ++e) outr[v0 + i + e] = x[e];
    }
    __syncthreads();
    if (tok >= 0) {
      // of several nodes with one token, whichever set the mark takes it off
      if (made) atomicAdd(&words[tok], 0xffffffffu);
      if (!was) atomicAnd(&words[tok], ~LG_SEEN);
    }
    __syncthreads();
  }
  if (reporter && bad) atomicOr(a.fault, bad);
}

}  // namespace

extern "C" int32_t dsbd_process_logits(const dsbd_forest* f, const int32_t* row_node, int32_t n_rows, int32_t V, int32_t dtype,
                                       const void* logits, int64_t logits_stride, const dsbd_logit_rules* rules, float* out,
                                       int64_t out_stride, int32_t* fault, void* stream_) {
  if (!f || !rules || !fault || n_rows < 0) return DSBD_ERR_INVALID;
  if (V < 1 || V > (1 << 30) || (dtype != DSBD_F32 && dtype != DSBD_BF16 && dtype != DSBD_F16)) return DSBD_ERR_UNSUPPORTED;
  if (f->n_prompts < 0 || f->n_trees < 0 || f->n_nodes < 0 || logits_stride < V || out_stride < V) return DSBD_ERR_INVALID;
  if (f->max_tree_nodes > DSBD_MAX_TREE_NODES) return DSBD_ERR_UNSUPPORTED;
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
  // rows per workgroup: several, so that a text is scanned once for them, as long as 2048 workgroups (8 per compute unit) are left
  a.rows_wg = (int)std::max(1LL, std::min(16LL, (long long)n_rows * a.n_chunks / 2048));
  const long long wgs = (long long)((n_rows + a.rows_wg - 1) / a.rows_wg) * a.n_chunks;
  if (wgs > 0x7fffffffLL) return DSBD_ERR_UNSUPPORTED;
  hipStream_t stream = static_cast<hipStream_t>(stream_);
  const dim3 grid((unsigned)wgs), block(LG_BLOCK);
  if (dtype == DSBD_F32) hipLaunchKernelGGL((logits_kernel<float>), grid, block, 0, stream, a);
  else if (dtype == DSBD_BF16) hipLaunchKernelGGL((logits_kernel<__bf16>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((logits_kernel<_Float16>), grid, block, 0, stream, a);
  DSBD_HIP_LAUNCH_CHECK();
  return DSBD_OK;
}
