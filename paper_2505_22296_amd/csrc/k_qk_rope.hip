// Norms and rotation of a rank's query and key heads, laid out for the Ulysses
// all-to-all, and the backward from what the reverse all-to-all returns (gfx950).
//
// Forward, for token t and slot h of rank j, whose head is g = map[j, h]:
//   n = x[t, g] (sum_d x^2 / D + eps)^(-1/2) (w + w_off)       (where w is given)
//   pairs (a, b) of n's first `rot` dims -> s (a cos - b sin, a sin + b cos)
//   dst[j, t, h] = bf16 of that; +0 where the map has -1; value heads are copied.
// Backward, for head g of token t:
//   c' = sum over g's slots, ascending, of the gradients there (float32)
//   c = the pairs of c' turned back, times s;  dw += c n';  c *= w + w_off
//   dx = r (c - n' mean(c n')),  n' = x r,  r = (sum x^2 / D + eps)^(-1/2).
// Both are bound by HBM: a head is read once (a replicated KV head once more from
// the caches a slot) and a slot written once, where the norm, the rotation and the
// pack as passes of their own read and write three times.
//
// An angle is a position times a frequency, of which only the fraction of a turn
// matters: frequencies are 64-bit fixed-point turns a position, the product with
// the position wraps by itself, and its upper 32 bits are the fraction, exact to
// 2^-32 turns at any position below 2^31.
//
// D / 16 neighbouring lanes hold a row (a head of a token), 16 dims each, so that
// both halves of a pair are in one lane.  A wavefront holds one head of 64 / (D / 16)
// tokens at a time and goes through a range of heads: what depends on the head --
// its kind, weights and slots -- is uniform and comes through the scalar cache, what
// depends on the token -- the angles -- is formed once for the whole range, and the
// next head's loads are in flight while one is worked on.  (Heads on the lanes and
// one token a wavefront instead: forward of 4096 tokens of 28 / 4 heads to 8 ranks,
// D = 128, 20.1 us, now 17.7, 5.9 TB/s; their backward, with the sum of the weight
// gradients, 53 us, now 31, 3.9 TB/s; of 8191 tokens of 40 / 8 heads from 16 ranks 104
// us, now 76 to 81, 4.9 TB/s.)
#include <algorithm>
#include <type_traits>

#include "dev_common.h"
#include "launch.h"

namespace spk {

namespace {

constexpr int kQB = 256;  // threads a workgroup (four wavefronts)

// The kernels' first argument where it lies, in constant memory: its tables are read
// at run-time indexes, for which the compiler copies the argument itself to scratch
// memory when its passes do not see through (25 times the time).
template <typename A>
using Arg = __attribute__((address_space(4))) A;

// The two 16-byte chunks of a row that lane l of the row holds: with `halves`
// pairing (i, i + rot/2) chunks l and l + rot/16 of the rotated dims; neighbour
// pairs (2i, 2i + 1) and the dims that are not rotated: chunks 2l, 2l + 1.
template <bool NEIGH>
SP_DEV void lane_chunks(int l, int rot, int& ca, int& cb) {
  const bool turned = !NEIGH && l < rot / 16;
  ca = turned ? l : 2 * l;
  cb = turned ? l + rot / 16 : 2 * l + 1;
}

// cos and sin (times the scale) of the lane's eight pairs at one position.  Pairs
// that are not turned have frequency 0 in the table: cos 1, sin 0, with no branch
// around a load (the compiler waits for each of eight in turn otherwise: +2 us a
// kernel).  The instructions take turns and are off by at most 1.3e-7 (measured over
// 2^22 values).
template <bool NEIGH, typename A>
SP_DEV void lane_angles(A a, int l, int64_t pos, float (&cs)[8], float (&sn)[8]) {
  uint64_t freq[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) freq[k] = a->freq[8 * l + k];  // (either pairing)
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float x = (float)(int32_t)(((uint64_t)pos * freq[k]) >> 32) * 0x1p-32f;  // in [-1/2, 1/2]
    const float scale = 8 * l + k < a->rot / 2 ? a->rope_scale : 1.f;
    cs[k] = __builtin_amdgcn_cosf(x) * scale;
    sn[k] = __builtin_amdgcn_sinf(x) * scale;
  }
}

// Pair k of the lane's 16 values turned by (cs, sn).
template <bool NEIGH>
SP_DEV void turn(float (&x)[16], const float (&cs)[8], const float (&sn)[8], float sign) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int i = NEIGH ? 2 * k : k, j = NEIGH ? 2 * k + 1 : k + 8;
    const float p = x[i], q = x[j];
    x[i] = p * cs[k] - sign * q * sn[k];
    x[j] = sign * p * sn[k] + q * cs[k];
  }
}

// Sum over the L = 4 or 8 lanes of a row, on each of them: exchanges inside quads,
// then the mirror image of half a row of 16 lanes (its quads hold equal sums).
template <int CTRL>
SP_DEV float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int L>
SP_DEV float row_sum(float x) {
  static_assert(L == 4 || L == 8, "lanes a row");
  x += dpp<0xb1>(x);                       // quad_perm [1, 0, 3, 2]
  x += dpp<0x4e>(x);                       // quad_perm [2, 3, 0, 1]
  if constexpr (L == 8) x += dpp<0x141>(x);  // row_half_mirror
  return x;
}

SP_DEV void unpack16(const u32x4& a, const u32x4& b, float (&x)[16]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(a[k] << 16);
    x[2 * k + 1] = __uint_as_float(a[k] & 0xffff0000u);
    x[8 + 2 * k] = __uint_as_float(b[k] << 16);
    x[8 + 2 * k + 1] = __uint_as_float(b[k] & 0xffff0000u);
  }
}
SP_DEV u32x4 pack_lo(const float (&x)[16]) {
  return pack_bf16x8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]);
}
SP_DEV u32x4 pack_hi(const float (&x)[16]) {
  return pack_bf16x8(x[8], x[9], x[10], x[11], x[12], x[13], x[14], x[15]);
}

// The lane's 16 weights (plus the offset) of its two chunks.
SP_DEV void lane_weights(const u32x4* w, int ca, int cb, float off, float (&x)[16]) {
  unpack16(w[ca], w[cb], x);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] += off;
}

// Heads of the backward's wavefronts: units [0, q_units) have q_span query heads each,
// the others kv_span key and value heads.
struct QkSpans {
  int q_units, q_span, kv_span;
};

// Chunk `chunk` of the lane's token in a row of tokens `stride` chunks apart: a
// uniform base and a 32-bit offset a lane (16 tokens of less than 2^26 elements).
template <typename P>
SP_DEV P* lane_chunk(P* base, int tok, int64_t stride, int chunk) {
  typedef std::conditional_t<std::is_const_v<P>, const char, char> Byte;
  return (P*)((Byte*)base + ((uint32_t)tok * (uint32_t)stride + (uint32_t)chunk) * 16u);
}

// Row i of a token's heads: its kind (0 query, 1 key, 2 value), the head, and its
// entries [s0, s1) in the kind's slot table.
struct HeadRow {
  int kind, head, s0, s1;
};
template <typename A>
SP_DEV HeadRow head_row(A a, int i) {
  const int kind = i < a->Hq ? 0 : i < a->Hq + a->Hkv ? 1 : 2;
  const int g = kind == 0 ? i : kind == 1 ? i - a->Hq : i - a->Hq - a->Hkv;
  return HeadRow{kind, g, kind == 0 ? a->q_start[g] : a->kv_start[g], kind == 0 ? a->q_start[g + 1] : a->kv_start[g + 1]};
}
// First chunk of token t0's row in a [sp, T, H, D] buffer at slot entry e, and the
// chunks from a token to the next.
template <typename A>
SP_DEV int64_t slot_chunk(A a, uint32_t e, int kind, int t0, int nch) {
  const int H = kind == 0 ? a->Hq_loc : a->Hkv_loc;
  return (((int64_t)(e >> 10) * a->T + t0) * H + (e & 1023)) * nch;
}
template <typename A>
SP_DEV int slot_stride(A a, int kind, int nch) {
  return (kind == 0 ? a->Hq_loc : a->Hkv_loc) * nch;
}
template <typename A>
SP_DEV uint32_t slot_entry(A a, int kind, int s) { return kind == 0 ? a->q_slot[s] : a->kv_slot[s]; }

// Head i's row.
template <typename A>
SP_DEV void load_row(A a, int i, int t0, int tok, int ca, int cb, int nch, const u32x4* q, const u32x4* k,
                     const u32x4* v, u32x4& lo, u32x4& hi) {
  const HeadRow h = head_row(a, i);
  const int64_t stride = h.kind == 0 ? a->sq : h.kind == 1 ? a->sk : a->sv;
  const u32x4* src = (h.kind == 0 ? q : h.kind == 1 ? k : v) + t0 * stride + h.head * nch;
  lo = *lane_chunk(src, tok, stride, ca);
  hi = *lane_chunk(src, tok, stride, cb);
}

// A workgroup's wavefronts take `span` heads each of the tokens of blockIdx.x;
// behind a token's heads come three rows for the dummy slots of each kind.
template <int D, bool NEIGH, typename A>
__global__ __launch_bounds__(kQB) void qk_rope_kernel(A args, int span, const u32x4* __restrict__ q,
                                                      const u32x4* __restrict__ k, const u32x4* __restrict__ v,
                                                      const int32_t* __restrict__ positions,
                                                      const u32x4* __restrict__ w_q, const u32x4* __restrict__ w_k,
                                                      u32x4* __restrict__ q_dst, u32x4* __restrict__ k_dst,
                                                      u32x4* __restrict__ v_dst) {
  constexpr int L = D / 16, R = 64 / L, NCH = D / 8;
  const Arg<A>* a = (const Arg<A>*)__builtin_amdgcn_kernarg_segment_ptr();
  const int lane = threadIdx.x & 63, l = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = blockIdx.x * R, tok = min(lane / L, a->T - 1 - t0);  // the lane's token is t0 + tok
  const bool live = lane / L == tok;
  const int heads = a->Hq + 2 * a->Hkv;
  const int r0 = (blockIdx.y * (kQB / 64) + wave) * span, r1 = min(r0 + span, heads + 3);
  if (r0 >= r1) return;
  int ca, cb;
  lane_chunks<NEIGH>(l, a->rot, ca, cb);
  u32x4 lo = {0u, 0u, 0u, 0u}, hi = lo;
  if (r0 < heads) load_row(a, r0, t0, tok, ca, cb, NCH, q, k, v, lo, hi);
  float cs[8], sn[8];
  lane_angles<NEIGH>(a, l, positions ? (int64_t)positions[t0 + tok] : (int64_t)a->pos_base + t0 + tok, cs, sn);
  for (int i = r0; i < r1; ++i) {
    u32x4 out_lo = lo, out_hi = hi;
    HeadRow h;
    if (i < heads) {
      h = head_row(a, i);
      if (i + 1 < min(r1, heads)) load_row(a, i + 1, t0, tok, ca, cb, NCH, q, k, v, lo, hi);
      if (h.kind < 2) {
        float x[16];
        unpack16(out_lo, out_hi, x);
        const u32x4* w = h.kind == 0 ? w_q : w_k;
        if (w) {
          float wt[16], ss = 0.f;
          lane_weights(w, ca, cb, a->w_off, wt);
#pragma unroll
          for (int d = 0; d < 16; ++d) ss = __builtin_fmaf(x[d], x[d], ss);
          const float r = rsqrtf(row_sum<L>(ss) * (1.f / D) + a->eps);
#pragma unroll
          for (int d = 0; d < 16; ++d) x[d] = x[d] * r * wt[d];
        }
        turn<NEIGH>(x, cs, sn, 1.f);
        out_lo = pack_lo(x);
        out_hi = pack_hi(x);
      }
    } else {  // the slots without a head
      const int kind = i - heads;
      h = HeadRow{kind, 0, kind == 0 ? a->q_start[a->Hq] : a->kv_start[a->Hkv], a->sp * (kind == 0 ? a->Hq_loc : a->Hkv_loc)};
      out_lo = out_hi = u32x4{0u, 0u, 0u, 0u};
    }
    u32x4* dst = h.kind == 0 ? q_dst : h.kind == 1 ? k_dst : v_dst;
    for (int s = h.s0; s < h.s1; ++s) {
      u32x4* p = dst + slot_chunk(a, slot_entry(a, h.kind, s), h.kind, t0, NCH);
      if (live) {
        st_stream(out_lo, lane_chunk(p, tok, slot_stride(a, h.kind, NCH), ca));
        st_stream(out_hi, lane_chunk(p, tok, slot_stride(a, h.kind, NCH), cb));
      }
    }
  }
}

// Head i's gradient at its first slot, and its row where there is a norm.
template <typename A>
SP_DEV void load_grad(A a, int i, int t0, int tok, int ca, int cb, int nch, const u32x4* q, const u32x4* k,
                      const u32x4* dq_src, const u32x4* dk_src, const u32x4* dv_src, const u32x4* w_q,
                      const u32x4* w_k, u32x4& glo, u32x4& ghi, u32x4& xlo, u32x4& xhi) {
  const HeadRow h = head_row(a, i);
  glo = ghi = u32x4{0u, 0u, 0u, 0u};
  if (h.s0 < h.s1) {
    const u32x4* p = (h.kind == 0 ? dq_src : h.kind == 1 ? dk_src : dv_src) +
                     slot_chunk(a, slot_entry(a, h.kind, h.s0), h.kind, t0, nch);
    glo = ld_stream(lane_chunk(p, tok, slot_stride(a, h.kind, nch), ca));
    ghi = ld_stream(lane_chunk(p, tok, slot_stride(a, h.kind, nch), cb));
  }
  if (h.kind == 0 ? w_q != nullptr : h.kind == 1 && w_k != nullptr) {
    const int64_t stride = h.kind == 0 ? a->sq : a->sk;
    const u32x4* xs = (h.kind == 0 ? q : k) + t0 * stride + h.head * nch;
    xlo = *lane_chunk(xs, tok, stride, ca);
    xhi = *lane_chunk(xs, tok, stride, cb);
  }
}

// The same division of heads and tokens, but a wavefront has query heads or key and
// value heads (weights and weight gradients of one kind in registers); a workgroup
// goes through every gridDim.x-th group of tokens and keeps a partial weight gradient.
template <int D, bool NEIGH, typename A>
__global__ __launch_bounds__(kQB, 4) void qk_rope_bwd_kernel(A args, QkStrides o, QkSpans n, const u32x4* q, const u32x4* k,
                                                          const u32x4* __restrict__ dq_src,
                                                          const u32x4* __restrict__ dk_src,
                                                          const u32x4* __restrict__ dv_src,
                                                          const int32_t* __restrict__ positions,
                                                          const u32x4* __restrict__ w_q, const u32x4* __restrict__ w_k,
                                                          u32x4* dq, u32x4* dk, u32x4* dv, float* __restrict__ part) {
  constexpr int L = D / 16, R = 64 / L, NCH = D / 8, NW = kQB / 64;
  const Arg<A>* a = (const Arg<A>*)__builtin_amdgcn_kernarg_segment_ptr();
  const int lane = threadIdx.x & 63, l = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int heads = a->Hq + 2 * a->Hkv;
  const int unit = blockIdx.y * NW + wave;
  const bool query = unit < n.q_units;
  const int r0 = query ? min(unit * n.q_span, a->Hq) : min(a->Hq + (unit - n.q_units) * n.kv_span, heads);
  const int r1 = query ? min(r0 + n.q_span, a->Hq) : min(r0 + n.kv_span, heads);
  const u32x4* w = query ? w_q : w_k;
  int ca, cb;
  lane_chunks<NEIGH>(l, a->rot, ca, cb);
  float acc[16];
#pragma unroll
  for (int d = 0; d < 16; ++d) acc[d] = 0.f;
  u32x4 wlo = {0u, 0u, 0u, 0u}, whi = wlo;
  if (w) {
    wlo = w[ca];
    whi = w[cb];
  }
  for (int t0 = blockIdx.x * R; t0 < a->T && r0 < r1; t0 += gridDim.x * R) {
    const int tok = min(lane / L, a->T - 1 - t0);  // the lane's token is t0 + tok
    const bool live = lane / L == tok;
    u32x4 glo, ghi, xlo, xhi;  // head i's gradient at its first slot, and its row
    load_grad(a, r0, t0, tok, ca, cb, NCH, q, k, dq_src, dk_src, dv_src, w_q, w_k, glo, ghi, xlo, xhi);
    float cs[8], sn[8];
    lane_angles<NEIGH>(a, l, positions ? (int64_t)positions[t0 + tok] : (int64_t)a->pos_base + t0 + tok, cs, sn);
    for (int i = r0; i < r1; ++i) {
      const HeadRow h = head_row(a, i);
      const u32x4 x0 = xlo, x1 = xhi;
      float c[16];
      unpack16(glo, ghi, c);
      if (i + 1 < r1) load_grad(a, i + 1, t0, tok, ca, cb, NCH, q, k, dq_src, dk_src, dv_src, w_q, w_k, glo, ghi, xlo, xhi);
      for (int s = h.s0 + 1; s < h.s1; ++s) {
        const u32x4* p = (h.kind == 0 ? dq_src : h.kind == 1 ? dk_src : dv_src) +
                         slot_chunk(a, slot_entry(a, h.kind, s), h.kind, t0, NCH);
        const int stride = slot_stride(a, h.kind, NCH);
        float y[16];
        unpack16(ld_stream(lane_chunk(p, tok, stride, ca)), ld_stream(lane_chunk(p, tok, stride, cb)), y);
#pragma unroll
        for (int d = 0; d < 16; ++d) c[d] += y[d];
      }
      const int64_t ostride = h.kind == 0 ? o.q : h.kind == 1 ? o.k : o.v;
      u32x4* out = (h.kind == 0 ? dq : h.kind == 1 ? dk : dv) + t0 * ostride + h.head * NCH;
      if (h.kind < 2) {
        turn<NEIGH>(c, cs, sn, -1.f);
        if (w) {
          float x[16];
          unpack16(x0, x1, x);
          float ss = 0.f, cx = 0.f;
#pragma unroll
          for (int d = 0; d < 16; ++d) ss = __builtin_fmaf(x[d], x[d], ss);
          const float r = rsqrtf(row_sum<L>(ss) * (1.f / D) + a->eps), rl = live ? r : 0.f;
          // the weights stay packed (8 registers less; four wavefronts a SIMD)
          u32x4 w0 = wlo, w1 = whi;
          asm volatile("" : "+v"(w0), "+v"(w1));
          float wt[16];
          unpack16(w0, w1, wt);
#pragma unroll
          for (int d = 0; d < 16; ++d) {
            acc[d] = __builtin_fmaf(c[d], x[d] * rl, acc[d]);
            c[d] *= wt[d] + a->w_off;  // the gradient of the normed row
            cx = __builtin_fmaf(c[d], x[d], cx);
          }
          const float m = row_sum<L>(cx) * r * r * (1.f / D);
#pragma unroll
          for (int d = 0; d < 16; ++d) c[d] = r * (c[d] - x[d] * m);
        }
      }
      if (live) {
        st_stream(pack_lo(c), lane_chunk(out, tok, ostride, ca));
        st_stream(pack_hi(c), lane_chunk(out, tok, ostride, cb));
      }
    }
  }
  if (!part) return;
  // the wavefront's tokens, then the four wavefronts, in a fixed order
  __shared__ float red[NW][2][D];
#pragma unroll
  for (int d = 0; d < 16; ++d) {
#pragma unroll
    for (int off = L; off < 64; off <<= 1) acc[d] += __shfl_xor(acc[d], off);
    if (lane < L) {
      const int dim = (d < 8 ? ca : cb) * 8 + (d & 7);
      red[wave][0][dim] = query ? acc[d] : 0.f;
      red[wave][1][dim] = query ? 0.f : acc[d];
    }
  }
  __syncthreads();
  const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  for (int e = threadIdx.x; e < 2 * D; e += kQB) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) x += red[w][e / D][e % D];
    part[wg * 2 * D + e] = x;
  }
}

// dw[e] = sum of the n workgroups' partials: a workgroup takes 16 entries as four
// vectors, 64 threads a vector, eight loads in flight each; then their sums in a
// fixed order.  (One entry a thread and one load in flight: 20 us for 1024 partials.)
__global__ __launch_bounds__(kQB) void qk_dw_kernel(const f32x4* __restrict__ part, int n, int D,
                                                    float* __restrict__ dw_q, float* __restrict__ dw_k) {
  const int c = threadIdx.x & 3, r = threadIdx.x >> 2, v = blockIdx.x * 4 + c, nv = D / 2;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = r; i0 < n; i0 += 64 * 8) {
    f32x4 y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) y[u] = i0 + u * 64 < n ? part[(int64_t)(i0 + u * 64) * nv + v] : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += y[u][k];
  }
  __shared__ f32x4 red[64][5];
  red[r][c] = x;
  __syncthreads();
  if (threadIdx.x < 16) {
    float y = 0.f;
    for (int i = 0; i < 64; ++i) y += red[i][threadIdx.x >> 2][threadIdx.x & 3];
    const int e = blockIdx.x * 16 + threadIdx.x;
    float* out = e < D ? dw_q : dw_k;
    if (out) out[e < D ? e : e - D] = y;
  }
}

// Grid for `rows` rows a token: about `waves` wavefronts in all, each with at least
// one row, and four (a workgroup) for all rows of its tokens at least.
struct QkGrid {
  int groups, parts;
};
QkGrid qk_grid(int T, int D, int rows, int waves) {
  const int R = 64 / (D / 16), groups = std::max(1, (T + R - 1) / R);
  return QkGrid{groups, std::max(1, std::min((rows + 3) / 4, waves / 4 / groups))};
}
constexpr int kQkFwdWaves = 4096, kQkBwdWaves = 4096;
// Workgroups of the backward, which keep a partial weight gradient each.
QkGrid qk_bwd_grid(const QkArgs& a, int D) {
  QkGrid g = qk_grid(a.T, D, a.Hq + 2 * a.Hkv, kQkBwdWaves);
  g.groups = std::min(g.groups, std::max(1, kQkBwdWaves / 4 / g.parts));
  return g;
}
// Its wavefronts' heads: the units of `parts` workgroups shared between query and
// other heads by their numbers, one at least for each.
QkSpans qk_spans(const QkArgs& a, int parts) {
  const int units = 4 * parts, rows = a.Hq + 2 * a.Hkv;
  const int q = std::max(1, std::min(units - 1, (units * a.Hq + rows / 2) / rows));
  return QkSpans{q, (a.Hq + q - 1) / q, (2 * a.Hkv + units - q - 1) / (units - q)};
}

}  // namespace

int qk_bwd_groups(const QkArgs& a, int D) {
  const QkGrid g = qk_bwd_grid(a, D);
  return g.groups * g.parts;
}

// Up to 64 slots and heads of either kind travel in arguments of their own size (the
// 6.7 KB of the largest cost a launch 1.5 us of host time).
template <typename F>
static hipError_t with_qk_args(const QkArgs& a, const F& f) {
  constexpr int N = QkArgsSmall::kSlots, M = QkArgsSmall::kHeads;
  const int nq = a.sp * a.Hq_loc, nk = a.sp * a.Hkv_loc;
  if (nq > N || nk > N || a.Hq > M || a.Hkv > M) return f(a);
  QkArgsSmall b;
  static_cast<QkBase&>(b) = a;
  std::copy(a.q_slot, a.q_slot + nq, b.q_slot);
  std::copy(a.kv_slot, a.kv_slot + nk, b.kv_slot);
  std::copy(a.q_start, a.q_start + a.Hq + 1, b.q_start);
  std::copy(a.kv_start, a.kv_start + a.Hkv + 1, b.kv_start);
  return f(b);
}

hipError_t launch_qk_rope(const QkArgs& args, int D, const void* q, const void* k, const void* v, const int32_t* positions,
                          const void* w_q, const void* w_k, void* q_dst, void* k_dst, void* v_dst, hipStream_t st) {
  return with_qk_args(args, [&](const auto& a) {
    using A = std::decay_t<decltype(a)>;
    auto* kernel = D == 128 ? (a.neigh ? qk_rope_kernel<128, true, A> : qk_rope_kernel<128, false, A>)
                            : (a.neigh ? qk_rope_kernel<64, true, A> : qk_rope_kernel<64, false, A>);
    const int rows = a.Hq + 2 * a.Hkv + 3;
    const QkGrid g = qk_grid(a.T, D, rows, kQkFwdWaves);
    const int span = (rows + 4 * g.parts - 1) / (4 * g.parts);
    return sp_launch(kKQkRope, kernel, dim3(g.groups, g.parts), dim3(kQB), st, a, span, (const u32x4*)q,
                     (const u32x4*)k, (const u32x4*)v, positions, (const u32x4*)w_q, (const u32x4*)w_k, (u32x4*)q_dst,
                     (u32x4*)k_dst, (u32x4*)v_dst);
  });
}

hipError_t launch_qk_rope_bwd(const QkArgs& args, const QkStrides& o, int D, const void* q, const void* k,
                              const void* dq_src, const void* dk_src, const void* dv_src, const int32_t* positions,
                              const void* w_q, const void* w_k, void* dq, void* dk, void* dv, float* dw_q, float* dw_k,
                              float* part, hipStream_t st) {
  const QkGrid g = qk_bwd_grid(args, D);
  const int n = args.T > 0 ? g.groups * g.parts : 0;
  if (n > 0) {
    hipError_t e = with_qk_args(args, [&](const auto& a) {
      using A = std::decay_t<decltype(a)>;
      auto* kernel = D == 128 ? (a.neigh ? qk_rope_bwd_kernel<128, true, A> : qk_rope_bwd_kernel<128, false, A>)
                              : (a.neigh ? qk_rope_bwd_kernel<64, true, A> : qk_rope_bwd_kernel<64, false, A>);
      return sp_launch(kKQkRopeBwd, kernel, dim3(g.groups, g.parts), dim3(kQB), st, a, o, qk_spans(args, g.parts),
                       (const u32x4*)q, (const u32x4*)k, (const u32x4*)dq_src, (const u32x4*)dk_src,
                       (const u32x4*)dv_src, positions, (const u32x4*)w_q, (const u32x4*)w_k, (u32x4*)dq, (u32x4*)dk,
                       (u32x4*)dv, part);
    });
    if (e != hipSuccess) return e;
  }
  if (!dw_q && !dw_k) return hipSuccess;
  return sp_launch(0, qk_dw_kernel, dim3(2 * D / 16), dim3(kQB), st, (const f32x4*)part, n, D, dw_q, dw_k);
}

}  // namespace spk
