// Clipped policy loss with a KL and an entropy term on gfx950, from the logits
// of one rank's token slice, and its gradient to them.
//
// For a counted token t (its label in [0, V) and not ignored, inside a
// sequence) with logits x, label y, advantage A:
//   lse  = log sum_v e^(x_v),  logp = x_y - lse,  H = lse - sum_v p_v x_v
//   r    = e^(logp - old),     pg = -min(r A, clamp(r, 1 - cl, 1 + ch) A)
//   d    = ref - logp,         kl = e^d - d - 1
//   term = pg + c_kl kl - c_ent H
// and for the gradient G of the token's sequence sum
//   g = G (dpg/dlogp + c_kl (1 - e^d)),  dpg/dlogp = -A r where r A <= clamp(r) A, else 0
//   dx_v = g (1[v == y] - p_v) + G c_ent p_v (log p_v + H).
// Both directions are bound by HBM: the forward reads a counted row once and
// nothing of the others, the backward reads and writes it once (rows that do
// not count are written as zeros and not read).
#include <math.h>

#include <algorithm>

#include "dev_common.h"
#include "launch.h"

namespace spk {

namespace {

constexpr int kPB = 256;  // threads a workgroup (four wavefronts)
constexpr int kPU = 4;    // 16-byte loads a thread has in flight

// Running sums of a part of a row in the log2 domain: b, the largest
// x log2(e) so far (finite: kLowest, below which a logit weighs nothing);
// s = sum 2^y and u = sum 2^y y with y = x log2(e) - b.
constexpr float kLowest = -1e30f;
struct RowSum {
  float b, s, u;
};

SP_DEV RowSum join(const RowSum& p, const RowSum& q) {
  const float b = fmaxf(p.b, q.b);
  const float dp = p.b - b, dq = q.b - b;
  const float wp = __builtin_amdgcn_exp2f(dp), wq = __builtin_amdgcn_exp2f(dq);
  // (a part without weight has s = 0 and a finite b)
  return RowSum{b, wp * p.s + wq * q.s,
                wp * __builtin_fmaf(p.s, dp, p.u) + wq * __builtin_fmaf(q.s, dq, q.u)};
}

// N chunks of eight logits into the running sums.
template <int N, bool ENT>
SP_DEV void add_chunks(RowSum& r, const u32x4 (&v)[N]) {
  float x[8 * N];
  float top = neg_inf();
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[8 * c + 2 * k] = __uint_as_float(v[c][k] << 16);
      x[8 * c + 2 * k + 1] = __uint_as_float(v[c][k] & 0xffff0000u);
      top = fmaxf(fmaxf(top, x[8 * c + 2 * k]), x[8 * c + 2 * k + 1]);
    }
  const float b = fmaxf(r.b, top * kLog2e);
  const float d = r.b - b, w = __builtin_amdgcn_exp2f(d);
  float s = w * r.s, u = w * __builtin_fmaf(r.s, d, r.u);
#pragma unroll
  for (int i = 0; i < 8 * N; ++i) {
    float y = __builtin_fmaf(x[i], kLog2e, -b);
    if constexpr (ENT) y = fmaxf(y, kLowest);  // a logit of -inf: 2^y = 0, and 2^y y too
    const float e = __builtin_amdgcn_exp2f(y);
    s += e;
    if constexpr (ENT) u = __builtin_fmaf(e, y, u);
  }
  r = RowSum{b, s, u};
}

SP_DEV int seq_of(const LossArgs& a, int t) {
  // sequence s with cu[s] <= t < cu[s+1], or -1
  if (t < a.cu[0] || t >= a.cu[a.n_seqs]) return -1;
  int lo = 0, hi = a.n_seqs;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}
SP_DEV bool label_counts(const LossArgs& a, int label) {
  return label != a.ignore_index && label >= 0 && label < a.V;
}

// What a token contributes, in 64 bits from the sums of its row: a thread does
// it once a row, and e^d - d - 1 of a small d keeps its digits.
struct TokenTerms {
  double term, kl;
  float ent, clipped;
};
SP_DEV TokenTerms token_terms(const PolicyArgs& p, const RowSum& r, uint16_t label_bits, const PolicyTokens& tok,
                              int t, int seq) {
  const float adv = tok.adv[p.adv_per_token ? t : seq];
  TokenTerms o;
  double lse, lp, ent = 0.0;
  if (r.s > 0.f) {
    // (back from the log2 domain by the float constant that led there)
    const double l2 = log2((double)r.s);
    lse = ((double)r.b + l2) / (double)kLog2e;
    lp = (double)bf16_to_f32(label_bits) - lse;
    if (p.entropy) ent = (l2 - (double)r.u / (double)r.s) / (double)kLog2e;
  } else if (r.s == 0.f) {  // every logit is the lowest there is: no distribution
    lse = lp = -__builtin_inf();
  } else {
    lse = lp = ent = __builtin_nan("");
  }
  const double ratio = exp(lp - (double)tok.old_logp[t]);
  const double held = fmin(fmax(ratio, 1.0 - (double)p.clip_low), 1.0 + (double)p.clip_high);
  // (an advantage of zero beside an infinite ratio is zero)
  const double free_obj = adv == 0.f ? 0.0 : ratio * (double)adv, held_obj = held * (double)adv;
  o.clipped = free_obj > held_obj ? 1.f : 0.f;
  o.term = -(free_obj > held_obj ? held_obj : free_obj);
  o.kl = 0.0;
  if (p.has_ref) {
    const double d = (double)tok.ref_logp[t] - lp;
    o.kl = expm1(d) - d;
    if (p.kl_coef != 0.f) o.term += (double)p.kl_coef * o.kl;
  }
  if (p.entropy) o.term -= (double)p.entropy_coef * ent;
  o.ent = (float)ent;
  tok.logp[t] = (float)lp;
  tok.lse[t] = (float)lse;
  if (p.entropy) tok.ent[t] = o.ent;
  return o;
}

// A workgroup sums one part of one row's vocabulary; WHOLE: the row, and its
// first thread writes what the token contributes (beside other workgroups' loads;
// the sums' few workgroups would take longer over it).  `part`: the parts' sums, or
// {term, kl, entropy, clipped} of every token.
template <bool ENT, bool WHOLE>
__global__ __launch_bounds__(kPB) void policy_rows_kernel(LossArgs a, PolicyArgs p, const u32x4* __restrict__ logits,
                                                          PolicyTokens tok, f32x4* __restrict__ part) {
  const int t = WHOLE ? blockIdx.x : blockIdx.x / p.parts, j = WHOLE ? 0 : blockIdx.x - t * p.parts;
  const int label = tok.labels[t], seq = seq_of(a, t);
  if (!label_counts(a, label) || seq < 0) {
    if (WHOLE && threadIdx.x == 0) {
      tok.logp[t] = 0.f;
      tok.lse[t] = 0.f;
      if (ENT) tok.ent[t] = 0.f;
    }
    return;
  }
  const int nch = a.V / 8;
  const int c0 = WHOLE ? 0 : (int)((int64_t)nch * j / p.parts);
  const int c1 = WHOLE ? nch : (int)((int64_t)nch * (j + 1) / p.parts);
  const u32x4* row = logits + (int64_t)t * nch;
  RowSum r{kLowest, 0.f, 0.f};
  int c = c0 + threadIdx.x;
  for (; c + (kPU - 1) * kPB < c1; c += kPU * kPB) {
    u32x4 v[kPU];
#pragma unroll
    for (int i = 0; i < kPU; ++i) v[i] = ld_stream(&row[c + i * kPB]);
    add_chunks<kPU, ENT>(r, v);
  }
  for (; c < c1; c += kPB) {
    const u32x4 v[1] = {ld_stream(&row[c])};
    add_chunks<1, ENT>(r, v);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    r = join(r, RowSum{__shfl_xor(r.b, off), __shfl_xor(r.s, off), __shfl_xor(r.u, off)});
  __shared__ RowSum sw[kPB / 64];
  if ((threadIdx.x & 63) == 0) sw[threadIdx.x >> 6] = r;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 1; i < kPB / 64; ++i) r = join(r, sw[i]);
    if constexpr (WHOLE) {
      const TokenTerms o = token_terms(p, r, ((const uint16_t*)row)[label], tok, t, seq);
      part[t] = f32x4{(float)o.term, (float)o.kl, o.ent, o.clipped};
    } else {
      part[(int64_t)t * p.parts + j] = f32x4{r.b, r.s, r.u, 0.f};
    }
  }
}

// One workgroup of B threads a sequence: sums what its tokens contribute, in a
// fixed order and 64 bits.  JOIN: it joins the parts of the tokens' rows first
// (few tokens); the first and the last workgroup then also write the tokens
// outside every sequence.
template <int B, bool JOIN>
__global__ __launch_bounds__(B) void policy_sums_kernel(LossArgs a, PolicyArgs p, const uint16_t* __restrict__ logits,
                                                        PolicyTokens tok, const f32x4* __restrict__ part,
                                                        float* __restrict__ seq_sum, float* __restrict__ stats) {
  const int s = blockIdx.x;
  const int b = a.n_seqs ? a.cu[s] : 0, e = a.n_seqs ? a.cu[s + 1] : 0;
  const int t0 = JOIN && s == 0 ? 0 : b, t1 = JOIN && s + 1 >= a.n_seqs ? a.T : e;
  double acc[5] = {0, 0, 0, 0, 0};  // term, kl, entropy, clipped, tokens
  for (int t = t0 + threadIdx.x; t < t1; t += B) {
    const int label = tok.labels[t];
    if (t < b || t >= e || !label_counts(a, label)) {
      if constexpr (JOIN) {
        tok.logp[t] = 0.f;
        tok.lse[t] = 0.f;
        if (p.entropy) tok.ent[t] = 0.f;
      }
      continue;
    }
    if constexpr (JOIN) {
      const f32x4* q = part + (int64_t)t * p.parts;
      RowSum r{q[0][0], q[0][1], q[0][2]};
      for (int i = 1; i < p.parts; ++i) r = join(r, RowSum{q[i][0], q[i][1], q[i][2]});
      const TokenTerms o = token_terms(p, r, logits[(int64_t)t * a.V + label], tok, t, s);
      acc[0] += o.term;
      acc[1] += o.kl;
      acc[2] += (double)o.ent;
      acc[3] += (double)o.clipped;
    } else {
      const f32x4 o = part[t];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += (double)o[i];
    }
    acc[4] += 1.0;
  }
  if (a.n_seqs == 0) return;
  __shared__ double red[B / 64][5];
#pragma unroll
  for (int i = 0; i < 5; ++i) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) acc[i] += __shfl_xor(acc[i], off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][i] = acc[i];
  }
  __syncthreads();
  if (threadIdx.x < 5) {
    double x = red[0][threadIdx.x];
    for (int w = 1; w < B / 64; ++w) x += red[w][threadIdx.x];
    if (threadIdx.x == 0)
      seq_sum[s] = (float)x;
    else
      stats[s * 4 + threadIdx.x - 1] = (float)x;
  }
}

// A workgroup takes kPU loads a thread of one row (few rows fill the chip too,
// and the chip reads and writes a few neighbouring rows at a time).  dlogits may
// be the logits: a thread stores only where it has loaded.
template <bool ENT>
__global__ __launch_bounds__(kPB) void policy_bwd_kernel(LossArgs a, PolicyArgs p, const u32x4* logits,
                                                         PolicyTokens tok, const float* __restrict__ grad_seq,
                                                         u32x4* dlogits, unsigned parts, unsigned nx) {
  const unsigned block = blockIdx.y * nx + blockIdx.x;
  const unsigned row = block / parts;
  if (row >= (unsigned)a.T) return;
  const int t = (int)row, part = (int)(block - row * parts);
  const int nch = a.V / 8;
  const int64_t base = (int64_t)t * nch;
  const int c0 = part * (kPB * kPU) + threadIdx.x;
  const int label = tok.labels[t], s = seq_of(a, t);
  const float l = tok.lse[t];
  if (s < 0 || !label_counts(a, label) || l == neg_inf()) {
#pragma unroll
    for (int i = 0; i < kPU; ++i)
      if (c0 + i * kPB < nch) st_stream(u32x4{0u, 0u, 0u, 0u}, &dlogits[base + c0 + i * kPB]);
    return;
  }
  u32x4 v[kPU];
#pragma unroll
  for (int i = 0; i < kPU; ++i)
    if (c0 + i * kPB < nch) v[i] = ld_stream(&logits[base + c0 + i * kPB]);
  const float G = grad_seq[s], A = tok.adv[p.adv_per_token ? t : s], lp = tok.logp[t];
  const float ratio = expf(lp - tok.old_logp[t]);
  const bool free_side = A >= 0.f ? ratio <= 1.f + p.clip_high : ratio >= 1.f - p.clip_low;
  float g = free_side && A != 0.f ? -A * ratio : 0.f;
  if (p.has_ref && p.kl_coef != 0.f) g -= p.kl_coef * expm1f(tok.ref_logp[t] - lp);
  g *= G;
  const float lb = l * kLog2e;
  // dx = 2^y (k1 y + k0) with y = log2 p: the entropy's part is G c_ent p (y ln 2 + H)
  const float k1 = ENT ? G * p.entropy_coef * kLn2 : 0.f;
  const float k0 = (ENT ? G * p.entropy_coef * tok.ent[t] : 0.f) - g;
#pragma unroll
  for (int i = 0; i < kPU; ++i) {
    const int c = c0 + i * kPB;
    if (c >= nch) break;
    float d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = __uint_as_float(k & 1 ? v[i][k >> 1] & 0xffff0000u : v[i][k >> 1] << 16);
      float y = __builtin_fmaf(x, kLog2e, -lb);
      const float e = __builtin_amdgcn_exp2f(y);
      if constexpr (ENT) {
        y = fmaxf(y, kLowest);  // (a logit of -inf: its gradient is 0)
        d[k] = e * __builtin_fmaf(k1, y, k0);
      } else {
        d[k] = e * k0;
      }
      if (c * 8 + k == label) d[k] += g;
    }
    st_stream(pack_bf16x8(d[0], d[1], d[2], d[3], d[4], d[5], d[6], d[7]), &dlogits[base + c]);
  }
}

}  // namespace

// Parts of a row in the forward: one where the rows fill the chip, else as many
// as give each workgroup one round of loads.
int policy_parts(int T, int V) {
  const int nch = V / 8;
  const int most = std::max(1, nch / (kPB * kPU));
  return std::min(most, std::max(1, 2048 / std::max(T, 1)));
}

hipError_t launch_policy_loss(const LossArgs& a, const PolicyArgs& p, const void* logits, const PolicyTokens& tok,
                              void* part, float* seq_sum, float* stats, hipStream_t st) {
  if (a.T > 0 && (a.n_seqs > 0 || p.parts == 1)) {
    auto* kernel = p.parts == 1 ? (p.entropy ? policy_rows_kernel<true, true> : policy_rows_kernel<false, true>)
                                : (p.entropy ? policy_rows_kernel<true, false> : policy_rows_kernel<false, false>);
    hipError_t e = sp_launch(kKPolicy, kernel, dim3((unsigned)a.T * p.parts), dim3(kPB), st, a, p, (const u32x4*)logits,
                             tok, (f32x4*)part);
    if (e != hipSuccess) return e;
  }
  if (p.parts == 1) {
    if (a.n_seqs == 0) return hipSuccess;
    return sp_launch(0, policy_sums_kernel<1024, false>, dim3(a.n_seqs), dim3(1024), st, a, p, (const uint16_t*)logits,
                     tok, (const f32x4*)part, seq_sum, stats);
  }
  return sp_launch(0, policy_sums_kernel<kPB, true>, dim3(std::max(a.n_seqs, 1)), dim3(kPB), st, a, p,
                   (const uint16_t*)logits, tok, (const f32x4*)part, seq_sum, stats);
}

hipError_t launch_policy_loss_bwd(const LossArgs& a, const PolicyArgs& p, const void* logits, const PolicyTokens& tok,
                                  const float* grad_seq, void* dlogits, hipStream_t st) {
  if (a.T <= 0) return hipSuccess;
  const unsigned parts = (unsigned)((a.V / 8 + kPB * kPU - 1) / (kPB * kPU));
  // (a grid dimension of 2^32 threads is refused: past 2^23 workgroups it gets a second one)
  const uint64_t n = (uint64_t)a.T * parts;
  const unsigned x = (unsigned)std::min<uint64_t>(n, 1u << 23);
  return sp_launch(kKPolicyBwd, p.entropy_coef != 0.f ? policy_bwd_kernel<true> : policy_bwd_kernel<false>,
                   dim3(x, (unsigned)((n + x - 1) / x)), dim3(kPB), st, a, p, (const u32x4*)logits, tok, grad_seq,
                   (u32x4*)dlogits, parts, x);
}

}  // namespace spk
