// The rows of a projection on their way to the attention: norm of every head, rotation by the position, and where they go:
// dense rows (dsbd_qk_norm_rope) or the pages of a cache (dsbd_paged_append).
//
// One pass over the data: a row (token, head) lies in the registers of a group of 4, 8 or 16 lanes, two 16-byte pieces per
// lane.  The pieces of a lane are chosen so that both channels of every pair it turns are its own (halves: channels 8j.. and
// rot/2 + 8j..; interleaved: 16 channels in a row), so the rotation needs no exchange, and the norm's sum of squares is the only
// thing that crosses lanes.  A wave takes one token (or a part of its heads): its lanes work out the 8 angles of their pairs
// once, in 64 bits, and use them for all the heads they come by.
// Bound by HBM where there are many rows: 8191 tokens, 32 + 32 heads of 128, f16, half of each head turned: 53.5 us, 268 MB at
// 5.0 TB/s (a large copy makes 5.2); prompts of 300 to 2500 tokens, 40 + 40 + 40 heads, into pages: 77 us, 360 MB at 4.7.  By latency
// where there are few: q and k of 248 nodes, 32 + 8 heads, 6 us.  The loads of the next head while one is worked on cost more (append
// 86 us) than they hide, with 4 waves a SIMD; so do non-temporal stores (63 us instead of 53.5).
#include "common.h"
#include "paged.h"
#include <algorithm>

namespace {

#define QR_BLOCK 256

typedef unsigned int qr_u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) qr_u32x4 qr_gvec;

struct QkRowsArgs {
  int n_rows, Hq, Hk, Hv, D;       // Hk, Hv: 0 where there are no such rows
  int parts;                       // waves per token
  const char *q, *k, *v;
  long long q_tok, q_head, k_tok, k_head, v_tok, v_head;          // bytes
  char *q_out, *k_out, *v_out;                                    // (k_out, v_out: the pages, where `paged`)
  long long qo_tok, qo_head, ko_tok, ko_head, vo_tok, vo_head;    // bytes
  const int32_t* positions;
  const char *q_weight, *k_weight;
  const double* inv_freq;
  float eps, rot_scale;
  int rot, norm, per_head, interleaved;
  PagedArgs cache;
  int32_t* fault;
};

template <typename T> struct Half;      // 8 values of 16 bits
template <> struct Half<__bf16> {
  static __device__ __forceinline__ float up(unsigned int w, int hi) { return __uint_as_float(hi ? w & 0xffff0000u : w << 16); }
};
template <> struct Half<_Float16> {
  static __device__ __forceinline__ float up(unsigned int w, int hi) {
    union { unsigned short u; _Float16 h; } c;
    c.u = (unsigned short)(hi ? w >> 16 : w);
    return (float)c.h;
  }
};
template <typename T>
__device__ __forceinline__ void unpack(qr_u32x4 v, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = Half<T>::up(v[i], 0); x[2 * i + 1] = Half<T>::up(v[i], 1); }
}
template <typename T>
__device__ __forceinline__ qr_u32x4 pack(const float* x) {
  union { T h[8]; qr_u32x4 v; } c;
#pragma unroll
  for (int i = 0; i < 8; ++i) c.h[i] = (T)x[i];
  return c.v;
}

// LPR: lanes per row, at least D / 16 of them.
template <typename T, int LPR, bool PAGED>
__global__ __launch_bounds__(QR_BLOCK) void qk_rows_kernel(QkRowsArgs a) {
  constexpr int ROWS = 64 / LPR;             // rows that a wave has in hand
  const int lane = threadIdx.x & 63, sub = lane % LPR, slot = lane / LPR;
  const long long unit = (long long)blockIdx.x * (QR_BLOCK / 64) + (threadIdx.x >> 6);
  const int row = __builtin_amdgcn_readfirstlane((int)(unit / a.parts)), part = __builtin_amdgcn_readfirstlane((int)(unit % a.parts));
  if (row >= a.n_rows) return;
  const bool live = sub < a.D / 16;
  // this lane's pieces: channels p0 .. p0+7 and p1 .. p1+7; those below `rot` are turned with each other
  int p0 = 16 * sub, p1 = p0 + 8;
  if (!a.interleaved && p0 < a.rot) { p0 = 8 * sub; p1 = a.rot / 2 + 8 * sub; }
  if (!live) p0 = p1 = 0;
  const bool turns = live && 16 * sub < a.rot;

  // ---- where the row's keys and values go, and its position
  int pos = 0;
  long long kv_to = -1;                       // element offset of the token in the pages; -1: not stored
  if (PAGED) {
    const int s = last_at_most(a.cache.q_off, a.cache.n_seqs + 1, row, [](int v, int) { return v; });
    if (s < 0 || s >= a.cache.n_seqs) return;                                        // padding
    const int first = a.cache.q_off[s], next = a.cache.q_off[s + 1], ctx = a.cache.ctx_len[s];
    // (in this order no difference overflows: first <= row is known)
    const bool good = first >= 0 && next > row && next - first <= a.cache.max_new && ctx >= 0 && ctx <= a.cache.max_len - (next - first);
    pos = good ? ctx + (row - first) : 0;
    int page = -1;
    const int at = quotient(a.cache.page, pos);
    if (good && at < a.cache.table_stride) page = a.cache.page_table[(long long)s * a.cache.table_stride + at];
    if (page >= 0 && page < a.cache.n_pages)
      kv_to = (long long)page * a.cache.page_stride + (long long)(pos - at * a.cache.page.d) * a.cache.token_stride;
    else if (lane == 0 && part == 0) atomicOr(a.fault, DSBD_FAULT_BOUNDS);
    if (a.positions) pos = a.positions[row];
  } else {
    pos = a.positions ? a.positions[row] : 0;
  }

  // ---- the lane's angles: whole turns are taken off in 64 bits, what is left fits a float to 2^-25 of a turn
  float cs[8], sn[8];
  if (a.rot > 0) {
    const int i0 = a.interleaved ? 8 * sub : p0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      cs[i] = 1.f; sn[i] = 0.f;
      if (turns) {
        const double t = (double)pos * (a.inv_freq[i0 + i] * 0.15915494309189535);
        const float half = (float)(2.0 * (t - rint(t)));
        cs[i] = cospif(half) * a.rot_scale;
        sn[i] = sinpif(half) * a.rot_scale;
      }
    }
  }

  const int H = a.Hq + a.Hk + a.Hv;
  for (int h = part * ROWS + slot; h < H; h += a.parts * ROWS) {
    const int which = h < a.Hq ? 0 : h < a.Hq + a.Hk ? 1 : 2;
    const int g = h - (which == 0 ? 0 : which == 1 ? a.Hq : a.Hq + a.Hk);
    const char* const src = which == 0 ? a.q + row * a.q_tok + g * a.q_head
                          : which == 1 ? a.k + row * a.k_tok + g * a.k_head : a.v + row * a.v_tok + g * a.v_head;
    qr_u32x4 r0 = *(const qr_gvec*)(src + 2 * p0), r1 = *(const qr_gvec*)(src + 2 * p1);
    if (which < 2 && (a.norm || a.rot > 0)) {
      float x[16];
      unpack<T>(r0, x);
      unpack<T>(r1, x + 8);
      if (a.norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
        if (!live) ss = 0.f;
#pragma unroll
        for (int m = 1; m < LPR; m <<= 1) ss += __shfl_xor(ss, m);
        float inv = 1.0f / sqrtf(ss / (float)a.D + a.eps);
        if constexpr (__is_same(T, __bf16)) {
          // bf16 has fp32's exponents, its squares have not: such rows are brought near 1 (all lanes of the row agree)
          if (!(ss <= 0x1p120f) || (ss < 0x1p-80f && a.eps < 0x1p-80f)) {
            const float by = ss < 1.f ? 0x1p72f : 0x1p-72f;
            ss = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) { x[i] *= by; ss += x[i] * x[i]; }
            if (!live) ss = 0.f;
#pragma unroll
            for (int m = 1; m < LPR; m <<= 1) ss += __shfl_xor(ss, m);
            inv = 1.0f / sqrtf(ss / (float)a.D + a.eps * by * by);
          }
        }
        const char* const w = which == 0 ? a.q_weight : a.k_weight;
        float wt[16];
        if (w) {
          const char* const wp = w + (a.per_head ? 2ll * g * a.D : 0);
          unpack<T>(*(const qr_gvec*)(wp + 2 * p0), wt);
          unpack<T>(*(const qr_gvec*)(wp + 2 * p1), wt + 8);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= w ? inv * wt[i] : inv;
      }
      if (turns) {
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float u = x[2 * i], v = x[2 * i + 1];
            x[2 * i] = u * cs[i] - v * sn[i];
            x[2 * i + 1] = u * sn[i] + v * cs[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float u = x[i], v = x[8 + i];
            x[i] = u * cs[i] - v * sn[i];
            x[8 + i] = u * sn[i] + v * cs[i];
          }
        }
      }
      r0 = pack<T>(x);
      r1 = pack<T>(x + 8);
    }
    char* dst;
    if (which == 0) dst = a.q_out + row * a.qo_tok + g * a.qo_head;
    else if (PAGED) dst = (which == 1 ? a.k_out : a.v_out) + 2 * (kv_to + g * a.cache.head_stride);
    else dst = which == 1 ? a.k_out + row * a.ko_tok + g * a.ko_head : a.v_out + row * a.vo_tok + g * a.vo_head;
    if (live && !(PAGED && which > 0 && kv_to < 0)) {
      *(qr_gvec*)(dst + 2 * p0) = r0;
      *(qr_gvec*)(dst + 2 * p1) = r1;
    }
  }
}

bool rows_ok(const dsbd_rows* r) {
  return r->ptr && !(reinterpret_cast<uintptr_t>(r->ptr) & 15) && r->token_stride >= 0 && r->head_stride >= 0;
}
bool rows_aligned(const dsbd_rows* r) { return !((r->token_stride | r->head_stride) & 7); }

// Shared checks and launch; what is absent has no heads.
int32_t launch(QkRowsArgs& a, int32_t dtype, const dsbd_rows* q, const dsbd_rows* k, const dsbd_rows* v, const dsbd_rows* q_out,
               const dsbd_rows* k_out, const dsbd_rows* v_out, const dsbd_qk_prep* prep, bool paged, hipStream_t stream) {
  if (a.D < 16 || a.D > 256 || a.D % 16 || (dtype != DSBD_BF16 && dtype != DSBD_F16)) return DSBD_ERR_UNSUPPORTED;
  a.rot = a.norm = a.per_head = a.interleaved = 0;
  a.q_weight = a.k_weight = nullptr; a.inv_freq = nullptr; a.eps = 0.f; a.rot_scale = 1.f;
  if (prep) {
    if (prep->rot_dim < 0 || prep->rot_dim > a.D || !(prep->eps >= 0.f)) return DSBD_ERR_INVALID;
    if (prep->rot_dim % 16) return DSBD_ERR_UNSUPPORTED;
    if (prep->rot_dim > 0 && !prep->inv_freq) return DSBD_ERR_INVALID;
    if (prep->norm && ((reinterpret_cast<uintptr_t>(prep->q_weight) | reinterpret_cast<uintptr_t>(prep->k_weight)) & 15)) return DSBD_ERR_INVALID;
    a.rot = prep->rot_dim; a.norm = prep->norm != 0; a.per_head = prep->per_head != 0; a.interleaved = prep->interleaved != 0;
    a.q_weight = static_cast<const char*>(prep->q_weight); a.k_weight = static_cast<const char*>(prep->k_weight);
    a.inv_freq = prep->inv_freq; a.eps = prep->eps; a.rot_scale = prep->rot_scale;
  }
  const dsbd_rows* const all[6] = {q, k, v, q_out, k_out, v_out};
  for (const dsbd_rows* r : all) if (r && !rows_ok(r)) return DSBD_ERR_INVALID;
  for (const dsbd_rows* r : all) if (r && !rows_aligned(r)) return DSBD_ERR_UNSUPPORTED;
  a.q = a.k = a.v = nullptr; a.q_out = nullptr;
  a.q_tok = a.q_head = a.k_tok = a.k_head = a.v_tok = a.v_head = a.qo_tok = a.qo_head = a.ko_tok = a.ko_head = a.vo_tok = a.vo_head = 0;
  const auto in = [](const dsbd_rows* r, const char*& p, long long& t, long long& h) {
    if (r) { p = static_cast<const char*>(r->ptr); t = 2 * r->token_stride; h = 2 * r->head_stride; }
  };
  const auto out = [](const dsbd_rows* r, char*& p, long long& t, long long& h) {
    if (r) { p = static_cast<char*>(r->ptr); t = 2 * r->token_stride; h = 2 * r->head_stride; }
  };
  in(q, a.q, a.q_tok, a.q_head); in(k, a.k, a.k_tok, a.k_head); in(v, a.v, a.v_tok, a.v_head);
  out(q_out, a.q_out, a.qo_tok, a.qo_head); out(k_out, a.k_out, a.ko_tok, a.ko_head); out(v_out, a.v_out, a.vo_tok, a.vo_head);
  const int H = a.Hq + a.Hk + a.Hv;
  if (a.n_rows == 0 || H == 0) return DSBD_OK;
  const int lpr = a.D <= 64 ? 4 : a.D <= 128 ? 8 : 16, rows = 64 / lpr, most = (H + rows - 1) / rows;
  // waves per token: all of its heads in one wave, so that the angles are worked out once, but for few tokens, which would
  // leave the device empty (8 waves on each of 256 compute units): 248 nodes with 40 heads 6.8 us a call, 9.7 with one wave each;
  // 64 tokens with 48 heads on their way into pages 7.5 and 10.7
  a.parts = (int)std::max(1LL, std::min((long long)most, 2048LL / a.n_rows));
  const long long waves = (long long)a.n_rows * a.parts, wgs = (waves + QR_BLOCK / 64 - 1) / (QR_BLOCK / 64);
  if (wgs > 0x7fffffffLL) return DSBD_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)wgs), block(QR_BLOCK);
#define QR_LAUNCH(T, L)                                                                    \
  do {                                                                                     \
    if (paged) hipLaunchKernelGGL((qk_rows_kernel<T, L, true>), grid, block, 0, stream, a); \
    else hipLaunchKernelGGL((qk_rows_kernel<T, L, false>), grid, block, 0, stream, a);      \
  } while (0)
#define QR_TYPES(L) do { if (dtype == DSBD_BF16) QR_LAUNCH(__bf16, L); else QR_LAUNCH(_Float16, L); } while (0)
  if (lpr == 4) QR_TYPES(4);
  else if (lpr == 8) QR_TYPES(8);
  else QR_TYPES(16);
#undef QR_TYPES
#undef QR_LAUNCH
  DSBD_HIP_LAUNCH_CHECK();
  return DSBD_OK;
}

}  // namespace

extern "C" int32_t dsbd_qk_norm_rope(int32_t n_rows, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype,
                                     const dsbd_rows* q, const dsbd_rows* k, const dsbd_rows* v, const int32_t* positions,
                                     const dsbd_qk_prep* prep, const dsbd_rows* q_out, const dsbd_rows* k_out,
                                     const dsbd_rows* v_out, void* stream) {
  if (n_rows < 0 || (q && Hq < 1) || ((k || v) && Hkv < 1) || !q != !q_out || !k != !k_out || !v != !v_out) return DSBD_ERR_INVALID;
  if (n_rows > 0 && (q || k) && prep && prep->rot_dim > 0 && !positions) return DSBD_ERR_INVALID;
  QkRowsArgs a;
  a.n_rows = n_rows; a.Hq = q ? Hq : 0; a.Hk = k ? Hkv : 0; a.Hv = v ? Hkv : 0; a.D = D;
  if ((long long)a.Hq + a.Hk + a.Hv > 65535) return DSBD_ERR_UNSUPPORTED;
  a.positions = positions; a.k_out = a.v_out = nullptr; a.fault = nullptr; a.cache = PagedArgs();
  return launch(a, dtype, q, k, v, q_out, k_out, v_out, prep, false, static_cast<hipStream_t>(stream));
}

extern "C" int32_t dsbd_paged_append(const dsbd_paged_kv* cache, int32_t n_rows, int32_t Hq, int32_t Hkv, int32_t D, int32_t dtype,
                                     const dsbd_rows* q, const dsbd_rows* k, const dsbd_rows* v, const int32_t* positions,
                                     const dsbd_qk_prep* prep, const dsbd_rows* q_out, int32_t* fault, void* stream) {
  if (!cache || !k || !v || !fault || !q != !q_out || (q && Hq < 1)) return DSBD_ERR_INVALID;
  const int32_t rc = paged_check(cache, n_rows, Hkv);
  if (rc != DSBD_OK) return rc;
  QkRowsArgs a;
  a.n_rows = cache->n_seqs == 0 ? 0 : n_rows; a.Hq = q ? Hq : 0; a.Hk = Hkv; a.Hv = Hkv; a.D = D;
  if ((long long)a.Hq + a.Hk + a.Hv > 65535) return DSBD_ERR_UNSUPPORTED;
  a.positions = positions; a.fault = fault; a.cache = paged_args(cache);
  a.k_out = static_cast<char*>(cache->k_pages); a.v_out = static_cast<char*>(cache->v_pages);
  return launch(a, dtype, q, k, v, q_out, nullptr, nullptr, prep, true, static_cast<hipStream_t>(stream));
}
