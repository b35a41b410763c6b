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
// both halves of a pair are in one lane; a wavefront has 64 / (D / 16) rows of one
// token, whose angles are formed once for all its heads.
#include <algorithm>

#include "dev_common.h"
#include "launch.h"

namespace spk {

namespace {

constexpr int kQB = 256;  // threads a workgroup (four wavefronts)

// The two 16-byte chunks of a row that lane l of the row holds: with `halves`
// pairing (i, i + rot/2) chunks l and l + rot/16 of the rotated dims; neighbour
// pairs (2i, 2i + 1) and the dims that are not rotated: chunks 2l, 2l + 1.
template <bool NEIGH>
SP_DEV void lane_chunks(int l, int rot, int& ca, int& cb) {
  const bool turned = !NEIGH && l < rot / 16;
  ca = turned ? l : 2 * l;
  cb = turned ? l + rot / 16 : 2 * l + 1;
}

// cos and sin (times the scale) of the lane's eight pairs at one position.
template <bool NEIGH>
SP_DEV void lane_angles(const QkArgs& a, int l, int64_t pos, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int f = 8 * l + k;  // the pair's frequency (either pairing)
    cs[k] = 1.f;
    sn[k] = 0.f;
    if (f < a.rot / 2) {
      const uint64_t turns = (uint64_t)pos * a.freq[f];
      const float x = (float)(int32_t)(turns >> 32) * 0x1p-32f;  // in [-1/2, 1/2]
      float c, s;
      sincospif(2.f * x, &s, &c);
      cs[k] = c * a.rope_scale;
      sn[k] = s * a.rope_scale;
    }
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

template <int D, bool NEIGH>
__global__ __launch_bounds__(kQB) void qk_rope_kernel(QkArgs a, const u32x4* __restrict__ q, const u32x4* __restrict__ k,
                                                      const u32x4* __restrict__ v,
                                                      const int32_t* __restrict__ positions,
                                                      const u32x4* __restrict__ w_q, const u32x4* __restrict__ w_k,
                                                      u32x4* __restrict__ q_dst, u32x4* __restrict__ k_dst,
                                                      u32x4* __restrict__ v_dst) {
  constexpr int L = D / 16, R = 64 / L, NCH = D / 8;
  const int lane = threadIdx.x & 63, l = lane % L;
  const int t = blockIdx.x * (kQB / 64) + (threadIdx.x >> 6);
  if (t >= a.T) return;
  int ca, cb;
  lane_chunks<NEIGH>(l, a.rot, ca, cb);
  float cs[8], sn[8];
  lane_angles<NEIGH>(a, l, positions ? (int64_t)positions[t] : (int64_t)a.pos_base + t, cs, sn);
  const int nq = a.sp * a.Hq_loc, nk = a.sp * a.Hkv_loc;
  for (int i0 = 0; i0 < nq + 2 * nk; i0 += R) {
    const int i = i0 + lane / L;
    if (i >= nq + 2 * nk) break;
    const int kind = i < nq ? 0 : i < nq + nk ? 1 : 2;
    const uint32_t e = kind == 0 ? a.q_slot[i] : a.kv_slot[kind == 1 ? i - nq : i - nq - nk];
    const int h = e & 1023, j = (e >> 10) & 1023, g = (int)(e >> 20) - 1;  // slot, rank, head
    const int H = kind == 0 ? a.Hq_loc : a.Hkv_loc;
    u32x4* dst = (kind == 0 ? q_dst : kind == 1 ? k_dst : v_dst) + (((int64_t)j * a.T + t) * H + h) * NCH;
    u32x4 lo = {0u, 0u, 0u, 0u}, hi = lo;
    if (g >= 0) {
      const u32x4* src = kind == 0 ? q + t * a.sq : kind == 1 ? k + t * a.sk : v + t * a.sv;
      lo = src[g * NCH + ca];
      hi = src[g * NCH + cb];
    }
    if (kind < 2) {
      float x[16];
      unpack16(lo, hi, x);
      const u32x4* w = kind == 0 ? w_q : w_k;
      float ss = 0.f;
#pragma unroll
      for (int d = 0; d < 16; ++d) ss = __builtin_fmaf(x[d], x[d], ss);
      ss = row_sum<L>(ss);
      if (w) {
        float wt[16];
        lane_weights(w, ca, cb, a.w_off, wt);
        const float r = rsqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
        for (int d = 0; d < 16; ++d) x[d] = x[d] * r * wt[d];
      }
      turn<NEIGH>(x, cs, sn, 1.f);
      if (g >= 0) {
        lo = pack_lo(x);
        hi = pack_hi(x);
      }
    }
    st_stream(lo, &dst[ca]);
    st_stream(hi, &dst[cb]);
  }
}

template <int D, bool NEIGH>
__global__ __launch_bounds__(kQB) void qk_rope_bwd_kernel(QkBwdArgs b, const u32x4* q, const u32x4* k,
                                                          const u32x4* __restrict__ dq_src,
                                                          const u32x4* __restrict__ dk_src,
                                                          const u32x4* __restrict__ dv_src,
                                                          const int32_t* __restrict__ positions,
                                                          const u32x4* __restrict__ w_q, const u32x4* __restrict__ w_k,
                                                          u32x4* dq, u32x4* dk, u32x4* dv, float* __restrict__ part) {
  constexpr int L = D / 16, R = 64 / L, NCH = D / 8, NW = kQB / 64;
  const QkArgs& a = b.a;
  const int lane = threadIdx.x & 63, l = lane % L, wave = threadIdx.x >> 6;
  int ca, cb;
  lane_chunks<NEIGH>(l, a.rot, ca, cb);
  float aq[16], ak[16];
#pragma unroll
  for (int d = 0; d < 16; ++d) aq[d] = ak[d] = 0.f;
  const int rows = a.Hq + 2 * a.Hkv;
  for (int t = blockIdx.x * NW + wave; t < a.T; t += gridDim.x * NW) {
    float cs[8], sn[8];
    lane_angles<NEIGH>(a, l, positions ? (int64_t)positions[t] : (int64_t)a.pos_base + t, cs, sn);
    for (int i0 = 0; i0 < rows; i0 += R) {
      const int i = i0 + lane / L;
      if (i >= rows) break;
      const int kind = i < a.Hq ? 0 : i < a.Hq + a.Hkv ? 1 : 2;
      const int g = kind == 0 ? i : kind == 1 ? i - a.Hq : i - a.Hq - a.Hkv;
      const u32x4* src = kind == 0 ? dq_src : kind == 1 ? dk_src : dv_src;
      const int H = kind == 0 ? a.Hq_loc : a.Hkv_loc;
      const int s0 = kind == 0 ? b.q_start[g] : b.kv_start[g], s1 = kind == 0 ? b.q_start[g + 1] : b.kv_start[g + 1];
      float c[16];
#pragma unroll
      for (int d = 0; d < 16; ++d) c[d] = 0.f;
      for (int s = s0; s < s1; ++s) {
        const uint32_t e = kind == 0 ? a.q_slot[s] : a.kv_slot[s];
        const int h = e & 1023, j = (e >> 10) & 1023;
        const u32x4* p = src + (((int64_t)j * a.T + t) * H + h) * NCH;
        float y[16];
        unpack16(ld_stream(&p[ca]), ld_stream(&p[cb]), y);
#pragma unroll
        for (int d = 0; d < 16; ++d) c[d] += y[d];
      }
      u32x4* out = kind == 0 ? dq + t * b.dsq : kind == 1 ? dk + t * b.dsk : dv + t * b.dsv;
      if (kind < 2) {
        turn<NEIGH>(c, cs, sn, -1.f);
        const u32x4* w = kind == 0 ? w_q : w_k;
        if (w) {
          const u32x4* xs = (kind == 0 ? q + t * a.sq : k + t * a.sk) + g * NCH;
          float x[16], wt[16];
          unpack16(xs[ca], xs[cb], x);
          lane_weights(w, ca, cb, a.w_off, wt);
          float ss = 0.f, cx = 0.f;
#pragma unroll
          for (int d = 0; d < 16; ++d) {
            ss = __builtin_fmaf(x[d], x[d], ss);
            cx = __builtin_fmaf(c[d] * wt[d], x[d], cx);
          }
          ss = row_sum<L>(ss);
          cx = row_sum<L>(cx);
          const float r = rsqrtf(ss * (1.f / D) + a.eps);
          const float m = cx * r * r * (1.f / D);
#pragma unroll
          for (int d = 0; d < 16; ++d) {
            const float dw = c[d] * (x[d] * r);
            if (kind == 0) aq[d] += dw; else ak[d] += dw;
            c[d] = r * (c[d] * wt[d] - x[d] * m);
          }
        }
      }
      st_stream(pack_lo(c), &out[g * NCH + ca]);
      st_stream(pack_hi(c), &out[g * NCH + cb]);
    }
  }
  if (!part) return;
  // the wavefront's rows, then the four wavefronts, in a fixed order
  __shared__ float red[NW][2][D];
#pragma unroll
  for (int d = 0; d < 16; ++d) {
#pragma unroll
    for (int off = L; off < 64; off <<= 1) {
      aq[d] += __shfl_xor(aq[d], off);
      ak[d] += __shfl_xor(ak[d], off);
    }
    if (lane < L) {
      const int dim = (d < 8 ? ca : cb) * 8 + (d & 7);
      red[wave][0][dim] = aq[d];
      red[wave][1][dim] = ak[d];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * D; e += kQB) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) x += red[w][e / D][e % D];
    part[(int64_t)blockIdx.x * 2 * D + e] = x;
  }
}

// dw[e] = sum of the workgroups' partials, for 16 entries a workgroup: 16 threads
// an entry, then their sums in a fixed order.
__global__ __launch_bounds__(kQB) void qk_dw_kernel(const float* __restrict__ part, int n, int D,
                                                    float* __restrict__ dw_q, float* __restrict__ dw_k) {
  const int e = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
  float x = 0.f;
  for (int i = r; i < n; i += 16) x += part[(int64_t)i * 2 * D + e];
  __shared__ float red[16][17];
  red[r][threadIdx.x & 15] = x;
  __syncthreads();
  if (r == 0) {
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) y += red[i][threadIdx.x];
    float* out = e < D ? dw_q : dw_k;
    if (out) out[e < D ? e : e - D] = y;
  }
}

}  // namespace

// Workgroups of the backward, which keep a partial weight gradient each.
int qk_bwd_groups(int T) { return std::max(1, std::min((T + kQB / 64 - 1) / (kQB / 64), 1024)); }

hipError_t launch_qk_rope(const QkArgs& a, int D, const void* q, const void* k, const void* v, const int32_t* positions,
                          const void* w_q, const void* w_k, void* q_dst, void* k_dst, void* v_dst, hipStream_t st) {
  auto* kernel = D == 128 ? (a.neigh ? qk_rope_kernel<128, true> : qk_rope_kernel<128, false>)
                          : (a.neigh ? qk_rope_kernel<64, true> : qk_rope_kernel<64, false>);
  return sp_launch(kKQkRope, kernel, dim3((a.T + kQB / 64 - 1) / (kQB / 64)), dim3(kQB), st, a, (const u32x4*)q,
                   (const u32x4*)k, (const u32x4*)v, positions, (const u32x4*)w_q, (const u32x4*)w_k, (u32x4*)q_dst,
                   (u32x4*)k_dst, (u32x4*)v_dst);
}

hipError_t launch_qk_rope_bwd(const QkBwdArgs& b, int D, const void* q, const void* k, const void* dq_src,
                              const void* dk_src, const void* dv_src, const int32_t* positions, const void* w_q,
                              const void* w_k, void* dq, void* dk, void* dv, float* dw_q, float* dw_k, float* part,
                              hipStream_t st) {
  const int n = b.a.T > 0 ? qk_bwd_groups(b.a.T) : 0;
  if (n > 0) {
    auto* kernel = D == 128 ? (b.a.neigh ? qk_rope_bwd_kernel<128, true> : qk_rope_bwd_kernel<128, false>)
                            : (b.a.neigh ? qk_rope_bwd_kernel<64, true> : qk_rope_bwd_kernel<64, false>);
    hipError_t e = sp_launch(kKQkRopeBwd, kernel, dim3(n), dim3(kQB), st, b, (const u32x4*)q, (const u32x4*)k,
                             (const u32x4*)dq_src, (const u32x4*)dk_src, (const u32x4*)dv_src, positions,
                             (const u32x4*)w_q, (const u32x4*)w_k, (u32x4*)dq, (u32x4*)dk, (u32x4*)dv, part);
    if (e != hipSuccess) return e;
  }
  if (!dw_q && !dw_k) return hipSuccess;
  return sp_launch(0, qk_dw_kernel, dim3(2 * D / 16), dim3(kQB), st, (const float*)part, n, D, dw_q, dw_k);
}

}  // namespace spk
