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

// N chunks of eight logits into the running sums.  MASKED: logits of -inf and of
// the type's lowest value, whose y is -inf, add 0 to u (else NaN: see row_sums).
// The maximum is the one that passes NaN on (one instruction for three operands;
// fmaxf first quiets each).
template <int N, bool ENT, bool MASKED>
SP_DEV void add_chunks(RowSum& r, const u32x4 (&v)[N]) {
  float x[8 * N];
  float top = neg_inf();
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[8 * c + 2 * k] = __uint_as_float(v[c][k] << 16);
      x[8 * c + 2 * k + 1] = __uint_as_float(v[c][k] & 0xffff0000u);
      top = max3_nonan(top, x[8 * c + 2 * k], x[8 * c + 2 * k + 1]);
    }
  const float b = __builtin_elementwise_maximum(r.b, top * kLog2e);
  const float d = r.b - b, w = __builtin_amdgcn_exp2f(d);
  float s = w * r.s, u = w * __builtin_fmaf(r.s, d, r.u);
#pragma unroll
  for (int i = 0; i < 8 * N; ++i) {
    float y = __builtin_fmaf(x[i], kLog2e, -b);
    if constexpr (ENT && MASKED) y = fmaxf(y, kLowest);
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

// a - b of log-probabilities; 0 where both are -inf (a banned token is banned in both).
template <typename T>
SP_DEV T log_ratio(T a, T b) {
  return a == b ? (T)0 : a - b;
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
  const double ratio = exp(log_ratio(lp, (double)tok.old_logp[t]));
  const double held = fmin(fmax(ratio, 1.0 - (double)p.clip_low), 1.0 + (double)p.clip_high);
  // (an advantage of zero beside an infinite ratio is zero)
  const double free_obj = adv == 0.f ? 0.0 : ratio * (double)adv, held_obj = held * (double)adv;
  o.clipped = free_obj > held_obj ? 1.f : 0.f;
  o.term = -(free_obj > held_obj ? held_obj : free_obj);
  o.kl = 0.0;
  if (p.has_ref) {
    // (a row without a distribution diverges from none; a label banned here alone, infinitely)
    const double d = r.s == 0.f ? 0.0 : log_ratio((double)tok.ref_logp[t], lp);
    o.kl = d < __builtin_inf() ? expm1(d) - d : d;
    if (p.kl_coef != 0.f) o.term += (double)p.kl_coef * o.kl;
  }
  if (p.entropy) o.term -= (double)p.entropy_coef * ent;
  o.ent = (float)ent;
  tok.logp[t] = (float)lp;
  tok.lse[t] = (float)lse;
  if (p.entropy) tok.ent[t] = o.ent;
  return o;
}

// The sums of chunks [c0, c1) of a row by a workgroup, on all its threads.
template <bool ENT, bool MASKED>
SP_DEV RowSum row_sums(const u32x4* row, int c0, int c1, RowSum* sw) {
  RowSum r{kLowest, 0.f, 0.f};
  for (int c = c0 + threadIdx.x; c < c1; c += kPU * kPB) {
    u32x4 v[kPU];
#pragma unroll
    for (int i = 0; i < kPU; ++i)  // (past the end: -1e38, which weighs nothing and keeps y finite)
      v[i] = c + i * kPB < c1 ? ld_stream(&row[c + i * kPB]) : u32x4{0xfe96fe96u, 0xfe96fe96u, 0xfe96fe96u, 0xfe96fe96u};
    add_chunks<kPU, ENT, MASKED>(r, v);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    r = join(r, RowSum{__shfl_xor(r.b, off), __shfl_xor(r.s, off), __shfl_xor(r.u, off)});
  if ((threadIdx.x & 63) == 0) sw[threadIdx.x >> 6] = r;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPB / 64; ++i) r = i ? join(r, sw[i]) : sw[0];
  return r;
}

// A workgroup sums one part of one row's vocabulary.  (The token's values formed
// here by the first thread, a workgroup a row: 145 instead of 137 us for 2800 counted
// rows of 152064 logits.)
template <bool ENT>
__global__ __launch_bounds__(kPB) void policy_rows_kernel(LossArgs a, PolicyArgs p, const u32x4* __restrict__ logits,
                                                          const int32_t* __restrict__ labels,
                                                          f32x4* __restrict__ part) {
  const int t = blockIdx.x / p.parts, j = blockIdx.x - t * p.parts;
  if (!label_counts(a, labels[t]) || seq_of(a, t) < 0) return;
  __shared__ RowSum sw[kPB / 64];
  const int nch = a.V / 8;
  const int c0 = (int)((int64_t)nch * j / p.parts), c1 = (int)((int64_t)nch * (j + 1) / p.parts);
  const u32x4* row = logits + (int64_t)t * nch;
  RowSum r = row_sums<ENT, false>(row, c0, c1, sw);
  // 2^y y of a masked logit is NaN in u alone: such a row is gone through once more
  // with y bounded (a row without masked logits saves that operation a logit)
  if (ENT && r.u != r.u && r.s == r.s) {
    __syncthreads();
    r = row_sums<ENT, true>(row, c0, c1, sw);
  }
  if (threadIdx.x == 0) part[(int64_t)t * p.parts + j] = f32x4{r.b, r.s, r.u, 0.f};
}

// Sum of five values over a workgroup in a fixed order; x[i] on thread i.
SP_DEV double sum5(double (&acc)[5]) {
  __shared__ double red[kPB / 64][5];
#pragma unroll
  for (int i = 0; i < 5; ++i) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) acc[i] += __shfl_xor(acc[i], off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6][i] = acc[i];
  }
  __syncthreads();
  double x = 0.0;
  if (threadIdx.x < 5)
    for (int w = 0; w < kPB / 64; ++w) x += red[w][threadIdx.x];
  return x;
}
SP_DEV void write_sums(int s, double x, float* seq_sum, float* stats) {
  if (threadIdx.x == 0)
    seq_sum[s] = (float)x;
  else if (threadIdx.x < 5)
    stats[s * 4 + threadIdx.x - 1] = (float)x;
}

// One workgroup for kSumTokens tokens of a sequence (blockIdx.y of blockIdx.x): joins
// the parts of their rows, writes what the tokens contribute and sums it in a fixed
// order and 64 bits, for a sequence of one workgroup to the outputs, else to
// `partial` [n_seqs, gridDim.y, 5].  The first workgroup of the first and of the last
// sequence also write the tokens outside every sequence.
constexpr int kSumTokens = 4 * kPB;
__global__ __launch_bounds__(kPB) void policy_sums_kernel(LossArgs a, PolicyArgs p, const uint16_t* __restrict__ logits,
                                                          PolicyTokens tok, const f32x4* __restrict__ part,
                                                          double* __restrict__ partial, float* __restrict__ seq_sum,
                                                          float* __restrict__ stats) {
  const int s = blockIdx.x;
  const int b = a.n_seqs ? a.cu[s] : 0, e = a.n_seqs ? a.cu[s + 1] : 0;
  auto zero = [&](int t) {
    tok.logp[t] = 0.f;
    tok.lse[t] = 0.f;
    if (p.entropy) tok.ent[t] = 0.f;
  };
  if (blockIdx.y == 0) {
    if (s == 0)
      for (int t = threadIdx.x; t < b; t += kPB) zero(t);
    if (s + 1 >= a.n_seqs)
      for (int t = e + threadIdx.x; t < a.T; t += kPB) zero(t);
  }
  double acc[5] = {0, 0, 0, 0, 0};  // term, kl, entropy, clipped, tokens
  const int t0 = b + blockIdx.y * kSumTokens, t1 = min(e, t0 + kSumTokens);
  for (int t = t0 + threadIdx.x; t < t1; t += kPB) {
    const int label = tok.labels[t];
    if (!label_counts(a, label)) {
      zero(t);
      continue;
    }
    const f32x4* q = part + (int64_t)t * p.parts;
    const uint16_t label_bits = logits[(int64_t)t * a.V + label];
    RowSum r{kLowest, 0.f, 0.f};
    for (int i0 = 0; i0 < p.parts; i0 += 8) {  // (eight loads in flight: 48 rows in 18 parts 7.3 -> 5.7 us)
      f32x4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i0 + i < p.parts ? q[i0 + i] : f32x4{kLowest, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 8; ++i) r = join(r, RowSum{x[i][0], x[i][1], x[i][2]});
    }
    const TokenTerms o = token_terms(p, r, label_bits, tok, t, s);
    acc[0] += o.term;
    acc[1] += o.kl;
    acc[2] += (double)o.ent;
    acc[3] += (double)o.clipped;
    acc[4] += 1.0;
  }
  if (a.n_seqs == 0) return;
  const double x = sum5(acc);
  if (gridDim.y == 1)
    write_sums(s, x, seq_sum, stats);
  else if (threadIdx.x < 5)
    partial[((int64_t)s * gridDim.y + blockIdx.y) * 5 + threadIdx.x] = x;
}
__global__ __launch_bounds__(kPB) void policy_join_kernel(const double* __restrict__ partial, int n,
                                                          float* __restrict__ seq_sum, float* __restrict__ stats) {
  double acc[5] = {0, 0, 0, 0, 0};
  for (int i = threadIdx.x; i < n; i += kPB)
#pragma unroll
    for (int k = 0; k < 5; ++k) acc[k] += partial[((int64_t)blockIdx.x * n + i) * 5 + k];
  write_sums(blockIdx.x, sum5(acc), seq_sum, stats);
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
  const float ratio = expf(log_ratio(lp, tok.old_logp[t]));
  const bool free_side = A >= 0.f ? ratio <= 1.f + p.clip_high : ratio >= 1.f - p.clip_low;
  float g = free_side && A != 0.f ? -A * ratio : 0.f;
  if (p.has_ref && p.kl_coef != 0.f) g -= p.kl_coef * expm1f(log_ratio(tok.ref_logp[t], lp));
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
    }
    if (c == label >> 3) {  // (one lane of one workgroup a row)
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] += (label & 7) == k ? g : 0.f;
    }
    st_stream(pack_bf16x8(d[0], d[1], d[2], d[3], d[4], d[5], d[6], d[7]), &dlogits[base + c]);
  }
}

}  // namespace

// Parts of a row in the forward.  Few rows: as many as give 2048 workgroups, down to
// one round of loads each.  Else four rounds each: rows end on a CU one after the
// other, and the last ones sooner (2800 rows of 152064 logits in 1 / 2 / 4 / 8 / 18
// parts: 145 / 137 / 137 / 139 / 166 us).
int policy_parts(int T, int V) {
  const int most = std::max(1, V / 8 / (kPB * kPU));
  return std::min(most, std::max({1, most / 4, 2048 / std::max(T, 1)}));
}
// Workspace: the parts' sums, then the sums of long sequences' pieces (at most one
// for every kSumTokens tokens and one a sequence).
size_t policy_partial_at(int T, int V) { return ((size_t)T * policy_parts(T, V) * 16 + 255) & ~size_t(255); }
size_t policy_workspace(int T, int V) {
  return policy_partial_at(T, V) + ((size_t)(T / kSumTokens + 1) * kMaxLossSeqs * 5 * sizeof(double) + 255 & ~size_t(255));
}

hipError_t launch_policy_loss(const LossArgs& a, const PolicyArgs& p, const void* logits, const PolicyTokens& tok,
                              void* ws, float* seq_sum, float* stats, hipStream_t st) {
  if (a.T > 0 && a.n_seqs > 0) {
    hipError_t e = sp_launch(kKPolicy, p.entropy ? policy_rows_kernel<true> : policy_rows_kernel<false>,
                             dim3((unsigned)a.T * p.parts), dim3(kPB), st, a, p, (const u32x4*)logits, tok.labels,
                             (f32x4*)ws);
    if (e != hipSuccess) return e;
  }
  if (a.T == 0 && a.n_seqs == 0) return hipSuccess;
  int longest = 0;
  for (int s = 0; s < a.n_seqs; ++s) longest = std::max(longest, a.cu[s + 1] - a.cu[s]);
  const int pieces = std::max(1, (longest + kSumTokens - 1) / kSumTokens);
  double* partial = (double*)((char*)ws + policy_partial_at(a.T, a.V));
  hipError_t e = sp_launch(0, policy_sums_kernel, dim3(std::max(a.n_seqs, 1), pieces), dim3(kPB), st, a, p,
                           (const uint16_t*)logits, tok, (const f32x4*)ws, partial, seq_sum, stats);
  if (e != hipSuccess || pieces == 1) return e;
  return sp_launch(0, policy_join_kernel, dim3(a.n_seqs), dim3(kPB), st, (const double*)partial, pieces, seq_sum, stats);
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
