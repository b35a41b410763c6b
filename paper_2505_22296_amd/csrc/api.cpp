// Host side of the SP attention library: argument validation, the block-skip
// scheduler, workspace layout and the C ABI declared in include/sp_attn.h.
//
// The scheduler replaces full masks (the paper notes the varlen path's
// overhead, Section 6.3): from cu_seqlens and the segments' position bases it
// lists one work item per (real head, segment, row tile) -- or per (real
// head, segment, key tile) for dK/dV -- carrying the tile's visible key (row)
// range and the causal offset delta (key j visible from row i iff
// j <= i + delta).  Dummy head slots (Section 4.1) never enter the list.
// Items are ordered longest first on every XCD, laid out for the order in
// which the hardware hands workgroups to XCDs and shader engines (see
// sort_items), so that its dispatch fills the 256 CUs the way
// longest-processing-time scheduling would.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <iterator>
#include <mutex>
#include <vector>

#include "../../include/sp_attn.h"
#include "launch.h"

namespace {

using spk::kItemInts;

constexpr int64_t kMaxTokens = int64_t(1) << 30;

struct Seg {
  int qa, qb, ka, kb, delta;
};

struct Problem {
  int D = 0;
  int n_real = 0;  // real local query heads: slots [0, n_real)
  // Row-side and key-side runs: rows [qa, qb) x keys [ka, kb) with key j
  // visible from row i iff j <= i + delta (causal).  For separate sequences
  // both lists are the segments; for one sequence in pieces they are the
  // maximal row (key) ranges over which the visible key (row) range grows
  // by 0 or 1 per row (key).
  std::vector<Seg> segs, segs_k;
  int q_pad = 0, k_pad = 0;  // first padding row / key
  std::vector<int> kv_of;    // per real local head
  std::vector<int> kv_lo, kv_hi;  // per local KV head: real heads [lo, hi) reading it
  bool direct = true;        // every KV head read by at most one real local head
  // SP_DESC_SHARED_PREFIX: per segment, the segment whose keys it sees too (-1:
  // none); empty without the flag.
  std::vector<int> prefix;
};


// One sequence in pieces (SP_DESC_SINGLE_SEQUENCE): rows [0, Qn) and keys
// [0, Kn) have strictly increasing positions, so the keys visible from row i
// are a prefix [0, n(i)) and the rows that see key j a suffix [m(j), Qn).
// n and m are split into maximal runs of constant step 0 or 1; each run is a
// Seg whose linear rule j <= i + delta reproduces the prefix / suffix.
sp_status single_sequence_runs(const sp_attn_desc* d, Problem& p) {
  const int n = d->num_seqs;
  if (n < 1 || !d->position_ids_q || !d->position_ids_k) return SP_ERR_INVALID_ARG;
  const int Qn = d->cu_seqlens_q[n], Kn = d->cu_seqlens_k[n];
  const int32_t* pq = d->position_ids_q;
  const int32_t* pk = d->position_ids_k;
  for (int i = 1; i < Qn; ++i)
    if (pq[i] <= pq[i - 1]) return SP_ERR_INVALID_ARG;
  for (int j = 1; j < Kn; ++j)
    if (pk[j] <= pk[j - 1]) return SP_ERR_INVALID_ARG;
  std::vector<int> cnt(Qn), first(Kn);
  for (int i = 0, j = 0; i < Qn; ++i) {  // n(i) = #keys with pos_k <= pos_q[i]
    if (d->causal)
      while (j < Kn && pk[j] <= pq[i]) ++j;
    cnt[i] = d->causal ? j : Kn;
  }
  for (int j = 0, i = 0; j < Kn; ++j) {  // m(j) = first row with pos_q >= pos_k[j]
    if (d->causal)
      while (i < Qn && pq[i] < pk[j]) ++i;
    first[j] = d->causal ? i : 0;
  }
  p.segs.clear();
  for (int i0 = 0; i0 < Qn;) {
    const int step = (i0 + 1 < Qn) ? cnt[i0 + 1] - cnt[i0] : 0;
    int i1 = i0 + 1;
    if (step == 0 || step == 1)
      while (i1 < Qn && cnt[i1] - cnt[i1 - 1] == step) ++i1;
    // step 1: keys [0, cnt[i]) = j <= i + cnt[i0] - 1 - i0; step 0 (or a
    // single row): keys [0, cnt[i0]), every one of them visible
    const int delta = (i1 - i0 > 1 && step == 1) ? cnt[i0] - 1 - i0 : cnt[i0];
    p.segs.push_back(Seg{i0, i1, 0, cnt[i1 - 1], delta});
    i0 = i1;
  }
  p.segs_k.clear();
  for (int j0 = 0; j0 < Kn;) {
    const int step = (j0 + 1 < Kn) ? first[j0 + 1] - first[j0] : 0;
    int j1 = j0 + 1;
    if (step == 0 || step == 1)
      while (j1 < Kn && first[j1] - first[j1 - 1] == step) ++j1;
    // step 1: rows [first[j], Qn) = j <= i + j0 - first[j0]; step 0 (or a
    // single key): rows [first[j0], Qn), visible from every key of the run
    const int delta = (j1 - j0 > 1 && step == 1) ? j0 - first[j0] : (j1 - 1) - first[j0];
    p.segs_k.push_back(Seg{first[j0], Qn, j0, j1, delta});
    j0 = j1;
  }
  return SP_OK;
}

// Shared prefixes (SP_DESC_SHARED_PREFIX).  The segments that share a prefix
// follow it, so the rows that see a prefix's keys are its own and then, to the
// group's end, every row: one range, for which the prefix's causal rule also holds
// behind its rows, as its last row sees all its keys.  Row tiles are another
// matter (RowTiles).
sp_status shared_prefixes(const sp_attn_desc* d, Problem& p) {
  const int n = d->num_seqs;
  if (n > 0 && !d->prefix_of) return SP_ERR_INVALID_ARG;
  p.prefix.assign(d->prefix_of, d->prefix_of + n);
  for (int s = 0; s < n; ++s) {
    const int f = p.prefix[s];
    if (f < -1 || f >= s) return SP_ERR_INVALID_ARG;
    if (f < 0) continue;
    if (p.prefix[f] != -1 || (f != s - 1 && p.prefix[s - 1] != f)) return SP_ERR_INVALID_ARG;
    Seg& k = p.segs_k[f];
    const Seg& own = p.segs[f];
    if (own.qb == own.qa)
      k.delta = own.kb - own.qa;  // no rows of its own: every row of the group sees every key
    else if (d->causal && (int64_t)own.delta < (int64_t)own.kb - own.qb)
      return SP_ERR_INVALID_ARG;
    k.qb = p.segs[s].qb;
  }
  // nothing shared: separate segments as ever
  if (std::all_of(p.prefix.begin(), p.prefix.end(), [](int f) { return f < 0; })) p.prefix.clear();
  return SP_OK;
}

// The O(T) checks that every segment's positions form a +1 ramp run unless
// the environment sets SPATTN_VALIDATE=0 (read once per process); without
// them only each segment's first position is read, and a malformed ramp
// gives a wrong mask, never an out-of-bounds access.
bool ramp_checks() {
  static const bool on = [] {
    const char* e = std::getenv("SPATTN_VALIDATE");
    return !(e && e[0] == '0' && e[1] == '\0');
  }();
  return on;
}

sp_status validate(const sp_attn_desc* d, Problem& p) {
  if (!d) return SP_ERR_INVALID_ARG;
  if (d->flags & ~(SP_DESC_SINGLE_SEQUENCE | SP_DESC_ROWSTATS_READY | SP_DESC_DQ_ACC_INIT | SP_DESC_SHARED_PREFIX))
    return SP_ERR_INVALID_ARG;
  const bool single = (d->flags & SP_DESC_SINGLE_SEQUENCE) != 0;
  const bool shared = (d->flags & SP_DESC_SHARED_PREFIX) != 0;
  if (single && shared) return SP_ERR_INVALID_ARG;
  if (d->T_q < 0 || d->T_k < 0 || d->T_q >= kMaxTokens || d->T_k >= kMaxTokens)
    return SP_ERR_INVALID_ARG;
  if (d->head_dim != 64 && d->head_dim != 128) return SP_ERR_UNSUPPORTED;
  if (d->H_loc < 1 || d->Hkv_loc < 1 || d->num_padded_heads < 1 || d->num_real_heads < 1 ||
      d->gqa_group < 1 || d->head_offset < 0 || d->kv_head_offset < 0 || d->num_seqs < 0)
    return SP_ERR_INVALID_ARG;
  if (d->Hkv_loc > spk::kMaxKv || d->H_loc > 4096) return SP_ERR_UNSUPPORTED;
  if (d->num_real_heads > d->num_padded_heads) return SP_ERR_INVALID_ARG;
  if (d->num_padded_heads % d->H_loc != 0 || d->head_offset % d->H_loc != 0 ||
      d->head_offset + d->H_loc > d->num_padded_heads)
    return SP_ERR_INVALID_ARG;
  const int sp = d->num_padded_heads / d->H_loc;
  if (d->num_padded_heads - d->num_real_heads >= sp) return SP_ERR_INVALID_ARG;
  if (d->num_real_heads % d->gqa_group != 0) return SP_ERR_INVALID_ARG;
  if (!(d->softmax_scale > 0.f) || !std::isfinite(d->softmax_scale)) return SP_ERR_INVALID_ARG;
  if (d->causal != 0 && d->causal != 1) return SP_ERR_INVALID_ARG;

  p.D = d->head_dim;
  p.n_real = std::max(0, std::min(d->H_loc, d->num_real_heads - d->head_offset));
  p.kv_of.resize(p.n_real);
  p.kv_lo.assign(d->Hkv_loc, 0);
  p.kv_hi.assign(d->Hkv_loc, 0);
  std::vector<int> cnt(d->Hkv_loc, 0);
  for (int y = 0; y < p.n_real; ++y) {
    int kv = (d->head_offset + y) / d->gqa_group - d->kv_head_offset;
    if (kv < 0 || kv >= d->Hkv_loc) return SP_ERR_INVALID_ARG;
    if (y > 0 && kv < p.kv_of[y - 1]) return SP_ERR_INVALID_ARG;  // monotone by construction
    p.kv_of[y] = kv;
    if (cnt[kv] == 0) p.kv_lo[kv] = y;
    p.kv_hi[kv] = y + 1;
    ++cnt[kv];
  }
  p.direct = true;
  for (int c : cnt)
    if (c > 1) p.direct = false;

  // segments
  const int n = d->num_seqs;
  p.segs.clear();
  p.q_pad = 0;
  p.k_pad = 0;
  if (n > 0) {
    if (!d->cu_seqlens_q || !d->cu_seqlens_k) return SP_ERR_INVALID_ARG;
    const int32_t* cq = d->cu_seqlens_q;
    const int32_t* ck = d->cu_seqlens_k;
    if (cq[0] != 0 || ck[0] != 0) return SP_ERR_INVALID_ARG;
    for (int s = 0; s < n; ++s)
      if (cq[s + 1] < cq[s] || ck[s + 1] < ck[s]) return SP_ERR_INVALID_ARG;
    if (cq[n] > d->T_q || ck[n] > d->T_k) return SP_ERR_INVALID_ARG;
    p.q_pad = cq[n];
    p.k_pad = ck[n];
    for (int s = 0; s < n; ++s) {
      Seg g{cq[s], cq[s + 1], ck[s], ck[s + 1], 0};
      int64_t pq = g.qa, pk = g.ka;  // default: positions restart at 0 per segment
      if (d->position_ids_q && g.qb > g.qa) {
        const int32_t* pos = d->position_ids_q;
        if (ramp_checks())
          for (int i = g.qa + 1; i < g.qb; ++i)
            if ((int64_t)pos[i] != (int64_t)pos[i - 1] + 1) return SP_ERR_INVALID_ARG;
        pq = (int64_t)g.qa - pos[g.qa];
      }
      if (d->position_ids_k && g.kb > g.ka) {
        const int32_t* pos = d->position_ids_k;
        if (ramp_checks())
          for (int i = g.ka + 1; i < g.kb; ++i)
            if ((int64_t)pos[i] != (int64_t)pos[i - 1] + 1) return SP_ERR_INVALID_ARG;
        pk = (int64_t)g.ka - pos[g.ka];
      }
      // key j visible from row i iff pos_k[j] <= pos_q[i]
      //   <=> j - pk <= i - pq  <=>  j <= i + (pk - pq)
      int64_t delta = pk - pq;
      if (delta > (int64_t(1) << 30) || delta < -(int64_t(1) << 30)) return SP_ERR_INVALID_ARG;
      g.delta = (int)delta;
      p.segs.push_back(g);
    }
  }
  p.segs_k = p.segs;
  if (single) return single_sequence_runs(d, p);
  if (shared) return shared_prefixes(d, p);
  return SP_OK;
}

struct Item {
  int v[kItemInts];
  int64_t cost;
};

// Launch order.  MI355X hands workgroup i of a launch to XCD i % 8, and an
// XCD hands its own workgroups, in order, to its four shader engines in
// turn, each to a free CU there; a workgroup whose shader engine has no free
// CU holds up the XCD's later ones even when other engines have free CUs.
// So the list is built per XCD:
//  (1) items sorted longest first (enumerated head by head; the sort keeps
//      that order among equal costs);
//  (2) with `grouped` (row items: forward, dQ), dealt to the XCDs in groups
//      of four consecutive items -- equal or near-equal costs, which the
//      XCD then runs one per shader engine, so its engines free CUs in
//      step -- eight groups a round, the rounds alternately forwards and
//      backwards over the XCDs so that no XCD always takes the round's
//      longest group; what is left after the last full round, and every
//      dK/dV item list (measured better that way), goes item by item in
//      list order;
//  (3) within each cost, the items an XCD was dealt are replaced by a
//      contiguous share of that cost's items, taken head by head, so each
//      XCD's L2 serves a few neighbouring heads (the costs per XCD stay);
//  (4) XCD x's items, longest first, fill the list positions that land on
//      XCD x.
// `n_front` items (zero fills) precede these in the launch and shift the
// position -> XCD map.
constexpr int kXcds = 8, kEngines = 4;

void sort_items(std::vector<Item>& items, std::vector<int32_t>& out, size_t n_front,
                bool grouped) {
  std::stable_sort(items.begin(), items.end(),
                   [](const Item& a, const Item& b) { return a.cost > b.cost; });
  const size_t N = items.size();
  auto xcd_of = [&](size_t p) { return (int)((n_front + p) % kXcds); };
  // (2) owner[i] = XCD of sorted item i
  std::vector<int> owner(N);
  constexpr size_t kRound = (size_t)kXcds * kEngines;
  const size_t full = grouped ? N / kRound * kRound : 0;
  for (size_t i = 0; i < full; ++i) {
    const size_t k = i % kRound / kEngines;      // group within the round
    const bool back = (i / kRound) & 1;
    owner[i] = xcd_of(back ? kXcds - 1 - k : k);
  }
  for (size_t i = full; i < N; ++i) owner[i] = xcd_of(i);
  // (3) contiguous per-XCD shares within each cost
  for (size_t s = 0; s < N;) {
    size_t e = s + 1;
    while (e < N && items[e].cost == items[s].cost) ++e;
    size_t n_x[kXcds] = {};
    for (size_t i = s; i < e; ++i) ++n_x[owner[i]];
    size_t i = s;
    for (int x = 0; x < kXcds; ++x)
      for (size_t j = 0; j < n_x[x]; ++j) owner[i++] = x;
    s = e;
  }
  // (4) per-XCD queues (longest first, as sorted) into their positions
  std::vector<std::vector<const Item*>> q(kXcds);
  for (size_t i = 0; i < N; ++i) q[owner[i]].push_back(&items[i]);
  size_t next[kXcds] = {};
  out.resize(N * kItemInts);
  for (size_t p = 0; p < N; ++p) {
    const int x = xcd_of(p);
    std::memcpy(&out[p * kItemInts], q[x][next[x]++]->v, sizeof(int) * kItemInts);
  }
}

// Workgroups an item is split over, for launches whose items would leave CUs
// idle.  With S workgroups an item, each owns 1 / S of its rows (keys) and its
// wavefronts form S groups that walk the keys (rows) side by side: 1 / S of
// the steps, but every staged tile serves 1 / S of the rows.  The model, in
// microseconds: `step`, an unsplit workgroup's step where half the CUs idle;
// `rel[i]`, a step's cost at S = 2^i against one at S = 1 (28 heads of 4096
// rows at D = 128, every CU busy: forward 122, 150, 193 us; dQ 163, 190, 234;
// dK/dV 229, 280); kStartUs, a workgroup's start and end.  A launch takes at
// least the average load of the 256 CUs and, for each k, k + 1 times its
// (256 k)-th longest workgroup (of the first 256 k + 1, k + 1 share a CU); the
// S with the lowest such bound is taken.  The largest items of small launches
// decide: 4 heads of 4096 rows take S = 4 in the forward (92 -> 43 us), 28
// heads of 4096 rows stay whole.
struct SplitModel {
  int n;  // S = 1, 2, .. 2^(n-1)
  double step, rel[3];
  double two;  // full CUs with two workgroups each against one (D = 64)
};
constexpr double kStartUs = 8;
constexpr int kMaxKeyParts = 64, kKeyPartChunks = 8;  // key_cuts
constexpr double kCutJoinUs = 10, kCutBytesUs = 4e6;
constexpr size_t kCus = 256;
constexpr SplitModel kSplitFwd{3, 2.0, {1.0, 1.22, 1.6}, 0.93};    // steps of 64 keys
constexpr SplitModel kSplitDq{3, 1.03, {1.0, 1.15, 1.45}, 0.94};   // steps of 32 keys
constexpr SplitModel kSplitDkdv{2, 0.72, {1.0, 1.22, 0}, 0.86};    // steps of 32 rows

// A work list's items: their steps, longest first, and the steps' sum.
struct Costs {
  std::vector<int> c;
  double sum = 0;
};

// The workgroups of one work list split S = 2^i ways.
struct WgList {
  const Costs& cost;
  const SplitModel& m;
  int i;
  size_t size() const { return cost.c.size() << i; }
  double us(size_t w) const {  // of the w-th longest
    return (double)cost.c[w >> i] / (1 << i) * m.rel[i] * m.step + kStartUs;
  }
  double total() const { return cost.sum * m.rel[i] * m.step + (double)size() * kStartUs; }
};

// Lower bounds of a launch of one list, and of two.
double launch_bound(const WgList& l) {
  double t = l.total() / kCus;
  for (size_t k = 0; k * kCus < l.size(); ++k) t = std::max(t, (double)(k + 1) * l.us(k * kCus));
  return t;
}
double launch_bound(const WgList& p, const WgList& q) {
  double t = (p.total() + q.total()) / kCus;
  // the two lists merged, an item's workgroups at a time
  const size_t sp = size_t(1) << p.i, sq = size_t(1) << q.i;
  for (size_t a = 0, b = 0, w = 0, k = 0; a < p.size() || b < q.size();) {
    const bool first = b >= q.size() || (a < p.size() && p.us(a) >= q.us(b));
    const double us = first ? p.us(a) : q.us(b);
    (first ? a : b) += first ? sp : sq;
    w += first ? sp : sq;
    for (; k * kCus < w; ++k) t = std::max(t, (double)(k + 1) * us);
  }
  return t;
}

// Items past which nothing is put into one launch: eight rounds of 256
// workgroups, whose end costs a few percent at most.
constexpr size_t kOneItems = 2048;

// Whether an unsplit list at head dimension 64 takes the kernels that run two
// workgroups a CU.  The tiles hold half the MFMA work of D = 128 beside the same
// exponentials, and four wavefronts a SIMD overlap the two better: full CUs get
// through a list in `two` of the time (16 heads of 32768 rows, one / two:
// forward 2428 / 2271 us, dQ 2900 / 2726, dK/dV 4599 / 3929).  But the longest
// workgroup, alone on its CU for the whole launch otherwise, shares it: with the
// 257th longest first, then with those that are left when the first 512 have
// been followed by 255 others (the longest's first partner ends last), and so
// on.  One workgroup a CU takes as long as longest-first scheduling on 256 CUs,
// run here on every 16th item and 16 CUs.  (Forward, one / two: 8 heads of 16384
// rows 309 / 359 us, with 32 segments of 256 rows beside it 330 / 375; 12 heads
// of 16384 rows 500 / 470; 40 full segments of 512 rows, 8 heads, 57 / 52.  The
// choice was the faster one in all but one of 78 lists of 26 shapes.)
bool two_a_cu(const WgList& l) {
  const size_t n = l.size();
  if (n <= kCus) return false;
  const double first = l.us(0), load = l.total() / kCus;
  double partners = l.us(kCus);
  for (size_t k = 3; k * kCus - 1 < n && partners < first; ++k) partners += l.us(k * kCus - 1);
  const double shared = first + (2 * l.m.two - 1) * std::min(first, partners);
  const double two = std::max(l.m.two * load, shared);
  if (two < std::max(load, first)) return true;  // (no schedule is shorter)
  if (n > kOneItems) return false;               // (past eight rounds the load decides)
  constexpr size_t kSample = 16;
  double cu[kCus / kSample] = {};  // the least loaded first (a heap)
  for (size_t w = kSample / 2; w < n; w += kSample) {
    std::pop_heap(std::begin(cu), std::end(cu), std::greater<double>());
    std::end(cu)[-1] += l.us(w);
    std::push_heap(std::begin(cu), std::end(cu), std::greater<double>());
  }
  return two < *std::max_element(std::begin(cu), std::end(cu));
}
constexpr double kTwoGain = 0.92;  // of a list, or a backward, that takes them
// The same for the two-way split forward (7 heads, 12289 rows in segments of
// about 700, 364 items: 40 -> 32.5 us; 16 heads of 5000 rows, 320: 83 -> 75; 14
// heads of 4096 rows, 224: 50 -> 52) and for the unsplit lists of a backward in
// one launch (the former 102 -> 94 us with 1078 items, 14 heads of 4096 rows, 672:
// 156 -> 174).  The bounds above misjudge these two (the former by 18%), so they
// go by their number of items; where one long sequence lies beside many short
// ones that loses (4 heads of 8192 rows and 60 segments of 200, forward 78 -> 83;
// of 16384 rows and 100 of 100, backward 531 -> 590; whole items, one workgroup a
// CU, two launches: 130, 637).
constexpr size_t kTwoSplitItems = 300, kTwoBwdItems = 900;
constexpr double kTwoSplitGain = 0.86;

// The shape of a launch of one list, and its bound.
spk::LaunchShape choose_shape(const Costs& cost, const SplitModel& m, int D,
                              double& best) {
  // by log2 of the split; the forward alone has the second
  const bool two[3] = {D == 64 && two_a_cu(WgList{cost, m, 0}),
                       D == 64 && cost.c.size() >= kTwoSplitItems && &m == &kSplitFwd, false};
  constexpr double kGain[3] = {kTwoGain, kTwoSplitGain, 1.0};
  spk::LaunchShape s{1, two[0]};
  best = 0;
  for (int i = 0; i < m.n; ++i) {
    const double t = launch_bound(WgList{cost, m, i}) * (two[i] ? kGain[i] : 1.0);
    if (i == 0 || t < best) {
      s = spk::LaunchShape{1 << i, two[i]};
      best = t;
    }
  }
  return s;
}

// How a backward call runs its two work lists: one after the other, each with
// the split it would take alone, or in one launch (the list with the longer
// workgroups first), where the second list fills the CUs that the first leaves
// idle at its end.  One launch is taken where the model sees at least 4% in it:
// 4 heads of 1024 rows 41 -> 24 us a call, 14 heads of 2734 rows without a mask
// 245 -> 193, 7 heads of 12289 rows in segments of about 700 213 -> 171; a ring
// chunk of 16384 rows, whose lists fill every round, is 1% slower that way.
struct BwdPlan {
  spk::LaunchShape q, k;
  bool one, dq_first;
};
BwdPlan plan_bwd(const Costs& cq, const Costs& ck, int D) {
  double tq = 0, tk = 0;
  BwdPlan p{choose_shape(cq, kSplitDq, D, tq), choose_shape(ck, kSplitDkdv, D, tk), false, false};
  const size_t n = cq.c.size() + ck.c.size();
  if (cq.c.empty() || ck.c.empty() || n > kOneItems) return p;
  constexpr double kLaunchUs = 4;
  double best = (tq + tk + kLaunchUs) / 1.04;
  constexpr int kPairs[3][2] = {{0, 0}, {1, 0}, {2, 1}};
  for (const auto& s : kPairs) {
    const WgList q{cq, kSplitDq, s[0]}, k{ck, kSplitDkdv, s[1]};
    const bool two = D == 64 && s[0] == 0 && n >= kTwoBwdItems;
    const double gain = two ? kTwoGain : 1.0;
    if ((q.total() + k.total()) / kCus * gain >= best) continue;
    const double t = launch_bound(q, k) * gain;
    if (t < best) {
      best = t;
      p = BwdPlan{{1 << s[0], two}, {1 << s[1], two}, true, q.us(0) > k.us(0)};
    }
  }
  return p;
}

Costs costs_of(const std::vector<Item>& sorted) {
  Costs r;
  r.c.resize(sorted.size());
  for (size_t i = 0; i < r.c.size(); ++i) r.sum += r.c[i] = (int)sorted[i].cost;
  return r;
}

// Row-tile items (forward, ring step, dQ).  Returns their steps, longest first.
Costs schedule_rows(const sp_attn_desc* d, const Problem& p, int BM, int BN, bool include_empty,
                    std::vector<int32_t>& out, size_t n_front) {
  std::vector<Item> items;
  for (int y = 0; y < p.n_real; ++y) {
    for (const Seg& g : p.segs) {
      // Causal row tiles end at the segment's end, so a partial tile is the
      // segment's first: its rows see the fewest keys.  (Aligned to the
      // start, the partial tile would be the last -- the segment's longest
      // item -- with most of its wavefronts idle.)
      const int len = g.qb - g.qa;
      const int first = d->causal && len % BM ? len % BM : BM;
      for (int a = g.qa, b = g.qa + std::min(first, len); a < g.qb;
           a = b, b = std::min(b + BM, g.qb)) {
        int k1 = g.kb;
        if (d->causal) k1 = (int)std::min<int64_t>(g.kb, (int64_t)b + g.delta);
        const int k0 = g.ka;
        const bool empty = k1 <= k0;
        if (empty && !include_empty) continue;
        Item it{{a, b, k0, empty ? k0 : k1, g.delta, y, p.kv_of[y], 0}, 0};
        it.cost = empty ? 0 : (int64_t)((k1 - (k0 & ~7)) + BN - 1) / BN;
        items.push_back(it);
      }
    }
    if (include_empty)
      for (int a = p.q_pad; a < d->T_q; a += BM)
        items.push_back(Item{{a, std::min(a + BM, d->T_q), 0, 0, 0, y, p.kv_of[y], 0}, 0});
  }
  sort_items(items, out, n_front, true);  // (leaves `items` longest first)
  return costs_of(items);
}

// Row tiles of a batch with shared prefixes: eight slots of up to 32 rows.  A slot
// holds rows of one segment; the slots of a tile share a prefix, whose keys the
// tile walks once for all of them, and then what they see of their own segments.
// A segment's full tiles are 256 rows at its end (causal: the rest are its first
// rows, which see the fewest keys); the rests of all segments of one prefix are
// put into tiles together (16 answers of 600 rows to a prompt of 8192: 42 tiles a
// head instead of 53).  Segments without a prefix are tiled one by one as ever.
struct RowTile {
  std::vector<spk::RowSlot> slots;  // at most 8
  int prefix = -1;                  // a segment
};
constexpr int kSlotRows = 32, kSlots = 8;
static_assert(spk::kFwdBM == kSlotRows * kSlots && spk::kDqBM == kSlotRows * kSlots, "slots of a row tile");

std::vector<RowTile> row_tiles(const sp_attn_desc* d, const Problem& p) {
  std::vector<RowTile> tiles;
  auto cut = [&](RowTile& t, const Seg& g, int a, int b) {  // rows [a, b), at most one tile's
    for (; a < b; a += kSlotRows)
      t.slots.push_back({a, std::min(a + kSlotRows, b), g.ka, g.kb, g.delta});
  };
  std::vector<spk::RowSlot> open;  // rests of segments of prefix `of`
  int of = -1;
  auto flush = [&] {
    for (size_t i = 0; i < open.size(); i += kSlots)
      tiles.push_back({{open.begin() + i, open.begin() + std::min(open.size(), i + kSlots)}, of});
    open.clear();
  };
  for (size_t s = 0; s < p.segs.size(); ++s) {
    const Seg& g = p.segs[s];
    const int BM = kSlotRows * kSlots, part = (g.qb - g.qa) % BM;
    const int f0 = d->causal ? g.qa + part : g.qa, f1 = d->causal ? g.qb : g.qb - part;  // full tiles
    const int r0 = d->causal ? g.qa : f1, r1 = d->causal ? f0 : g.qb;                    // the rest
    if (p.prefix[s] != of) {
      flush();
      of = p.prefix[s];
    }
    RowTile t;
    cut(t, g, r0, r1);
    if (of >= 0) {
      open.insert(open.end(), t.slots.begin(), t.slots.end());
    } else if (r1 > r0) {
      tiles.push_back(t);
    }
    for (int a = f0; a < f1; a += BM) {
      tiles.push_back({{}, of});
      cut(tiles.back(), g, a, a + BM);
    }
  }
  flush();
  const Seg pad{p.q_pad, d->T_q, 0, 0, 0};
  for (int a = pad.qa; a < pad.qb; a += kSlotRows * kSlots) {
    tiles.push_back({{}, -1});
    cut(tiles.back(), pad, a, std::min(a + kSlotRows * kSlots, pad.qb));
  }
  return tiles;
}

// Own keys [first, second) that a slot sees some of.
std::pair<int, int> own_keys(const sp_attn_desc* d, const spk::RowSlot& s) {
  const int k1 = d->causal ? (int)std::min<int64_t>(s.k1, (int64_t)s.row1 + s.delta) : s.k1;
  return {s.k0, std::max(s.k0, k1)};
}

// Key tiles of BN keys of the slots [a, b) of a tile; with `record`, their record
// (layout: RowSlot in dev_common.h) for a workgroup of n slots.
int slot_record(const sp_attn_desc* d, const Problem& p, const RowTile& t, size_t a, size_t b, int BN, int n,
                int32_t* record) {
  std::vector<std::pair<int, int>> own;
  for (size_t i = a; i < b; ++i) {
    const auto k = own_keys(d, t.slots[i]);
    if (k.second <= k.first) continue;
    // (slots ascend: ranges that meet or overlap are one)
    if (!own.empty() && k.first <= own.back().second)
      own.back().second = std::max(own.back().second, k.second);
    else
      own.push_back(k);
  }
  int tiles = 0, r = 0;
  auto range = [&](int k0, int k1) {
    const int first = k0 & ~7;
    tiles += (k1 - first + BN - 1) / BN;
    if (record) {
      int32_t* o = record + spk::kRecordRanges + 3 * r++;
      o[0] = tiles;
      o[1] = first;
      o[2] = k1;
    }
  };
  // (rows that do not exist see no prefix either)
  const bool prefix = t.prefix >= 0 && b > a && p.segs[t.prefix].kb > p.segs[t.prefix].ka;
  if (prefix) range(p.segs[t.prefix].ka, p.segs[t.prefix].kb);
  for (const auto& k : own) range(k.first, k.second);
  if (record) {
    record[0] = tiles;
    record[1] = prefix ? p.segs[t.prefix].ka : 0;
    record[2] = prefix;
    int32_t* o = record + spk::kRecordRanges + 3 * (1 + n);
    for (size_t i = a; i < b; ++i, o += 5) {
      const spk::RowSlot& s = t.slots[i];
      o[0] = s.row0; o[1] = s.row1; o[2] = s.k0; o[3] = s.k1; o[4] = s.delta;
    }
  }
  return tiles;
}

// Row items over such tiles; an item's first field is its tile's number until
// place_records puts the records' place there.  Leaves `items` longest first and
// returns their steps.
Costs schedule_tiles(const sp_attn_desc* d, const Problem& p, const std::vector<RowTile>& tiles, int BN,
                     std::vector<int32_t>& out, size_t n_front, std::vector<Item>& items) {
  std::vector<int> steps;
  for (const RowTile& t : tiles) steps.push_back(slot_record(d, p, t, 0, t.slots.size(), BN, kSlots, nullptr));
  for (int y = 0; y < p.n_real; ++y)
    for (size_t i = 0; i < tiles.size(); ++i)
      items.push_back(Item{{(int)i, 0, 0, 0, 0, y, p.kv_of[y], 0}, steps[i]});
  sort_items(items, out, n_front, true);
  return costs_of(items);
}

// The records of every tile for launches that split its rows over `split`
// workgroups; the row items' first fields become the records' places in a list where
// they start at int `base`.
std::vector<int32_t> place_records(const sp_attn_desc* d, const Problem& p, const std::vector<RowTile>& tiles, int split,
                                   int BN, std::vector<int32_t>& items, int base) {
  const int n = kSlots / split, ints = spk::record_ints(n);
  std::vector<int32_t> out((size_t)ints * split * tiles.size(), 0);
  for (size_t i = 0; i < tiles.size(); ++i)
    for (int w = 0; w < split; ++w) {
      const size_t a = std::min<size_t>(tiles[i].slots.size(), (size_t)w * n);
      const size_t b = std::min<size_t>(tiles[i].slots.size(), a + n);
      slot_record(d, p, tiles[i], a, b, BN, n, &out[(i * split + w) * ints]);
    }
  for (size_t i = 0; i < items.size(); i += kItemInts)
    if (items[i + 7] == 0) items[i] = base + items[i] * split * ints;
  return out;
}
// Either kind of row items.
Costs schedule_row_items(const sp_attn_desc* d, const Problem& p, const std::vector<RowTile>& tiles, int BM, int BN,
                         bool include_empty, std::vector<int32_t>& out, size_t n_front, std::vector<Item>& items) {
  return p.prefix.empty() ? schedule_rows(d, p, BM, BN, include_empty, out, n_front)
                          : schedule_tiles(d, p, tiles, BN, out, n_front, items);
}
// Ints of the records under any split.
size_t record_room(size_t n_tiles) { return n_tiles * 4 * (size_t)spk::record_ints(kSlots / 4); }

// Shared prefixes whose key items are cut into parts of their rows, in the order of
// the segments.  A short prompt's few key tiles see the rows of every answer: their
// items would go on long after the others.  Parts are summed in float32 by one more
// launch, in a fixed order.  The model: a backward takes the mean load of the CUs or its
// longest item, under the best of plan_bwd's splits; a part adds a workgroup's start,
// and its sums' way out and back; taken where that is 15% less or better.  Whole / in
// parts, D = 128: 16 answers of 1000 rows to 512 keys, one head, 260 / 80 us; 32 of 1500
// to 256, 4 heads, 876 / 446; 16 of 2000 to 512, 4 heads on one KV head, 569 / 468; 6 of
// 361 to 144, one head, 47 / 29.  (Of 57 drawn batches it is taken in four, 0.96 to 1.57
// times as fast.)
std::vector<spk::KeyCut> key_cuts(const sp_attn_desc* d, const Problem& p) {
  std::vector<spk::KeyCut> cuts;
  if (p.prefix.empty() || p.n_real == 0) return cuts;
  auto tiles = [](int n, int size) { return (double)((n + size - 1) / size); };
  auto own = [&](const Seg& g) { return (g.qb - g.qa) * (d->causal ? 0.5 : 1.0); };  // of its rows, at the mean
  double load_q = 0, load_k = 0, longest_q = 0, n_q = 0, n_k = 0;
  for (size_t s = 0; s < p.segs.size(); ++s) {
    const Seg& g = p.segs[s];
    const double nq = tiles(g.qb - g.qa, spk::kDqBM), nk = tiles(g.kb - g.ka, spk::kDkdvBN);
    const int prefix = p.prefix[s] < 0 ? 0 : p.segs[p.prefix[s]].kb - p.segs[p.prefix[s]].ka;
    const double seen = prefix + (g.kb - g.ka) * (d->causal ? 0.5 : 1.0);
    load_q += nq * seen / spk::kDqBN * kSplitDq.step;
    if (nq > 0) longest_q = std::max(longest_q, (prefix + g.kb - g.ka) / (double)spk::kDqBN * kSplitDq.step);
    const double rows = own(g) + p.segs_k[s].qb - g.qb;
    load_k += nk * rows / spk::kDkdvBQ * kSplitDkdv.step;
    n_q += nq * p.n_real;
    n_k += nk * p.n_real;
  }
  const double step = p.D == 64 ? 0.7 : 1.0;  // (8 answers of 1000 rows, one head: 0.53 us a chunk, 0.76)
  load_q *= step * p.n_real / kCus;
  load_k *= step * p.n_real / kCus;
  longest_q *= step;
  // of a backward whose longest key item takes `us`, with `more` key items, under the
  // splits that plan_bwd chooses from
  const bool one = n_q + n_k <= kOneItems;
  auto time = [&](double us, double more) {
    constexpr int kPairs[3][2] = {{0, 0}, {1, 0}, {2, 1}};
    double best = HUGE_VAL;
    for (const auto& s : kPairs) {
      const double rq = kSplitDq.rel[s[0]], rk = kSplitDkdv.rel[s[1]];
      const double lq = load_q * rq + (n_q * (1 << s[0])) * kStartUs / kCus;
      const double lk = load_k * rk + ((n_k + more) * (1 << s[1])) * kStartUs / kCus;
      const double tq = longest_q * rq / (1 << s[0]) + kStartUs, tk = us * rk / (1 << s[1]) + kStartUs;
      best = std::min(best, one ? std::max({lq + lk, tq, tk}) : std::max(lq, tq) + std::max(lk, tk));
    }
    return best;
  };
  int64_t row = 0;
  for (size_t s = 0; s < p.segs.size() && cuts.size() < (size_t)spk::kMaxCuts; ++s) {
    const Seg& g = p.segs_k[s];
    if (g.qb == p.segs[s].qb || g.kb <= g.ka) continue;  // shared by none, or empty
    const int len = g.kb - g.ka;
    const int chunks = (g.qb - g.qa) / spk::kDkdvBQ;
    const double longest = chunks * kSplitDkdv.step * step;
    int best = 1;
    double us = 0.85 * time(longest, 0);
    for (int n = 2; n <= std::min(kMaxKeyParts, chunks / kKeyPartChunks); ++n) {
      const double t = time(longest / n, tiles(len, spk::kDkdvBN) * p.n_real * (n - 1)) + kCutJoinUs +
                       (double)len * n * p.n_real * p.D * 16 / kCutBytesUs;
      if (t < us) {
        us = t;
        best = n;
      }
    }
    const int64_t rows = (int64_t)len * best * p.n_real;
    if (best == 1 || row + rows >= int64_t(1) << 28) continue;
    cuts.push_back(spk::KeyCut{g.ka, len, best, (int)row});
    row += rows;
  }
  return cuts;
}
int64_t cut_rows(const Problem& p, const std::vector<spk::KeyCut>& cuts) {
  return cuts.empty() ? 0 : cuts.back().row + (int64_t)cuts.back().len * cuts.back().parts * p.n_real;
}

// Key-tile items (dK / dV).  Every key of every real head gets exactly one
// item, or the parts of a cut.  Leaves `items` longest first and returns their steps.
Costs schedule_keys(const sp_attn_desc* d, const Problem& p, int BNK, int BQ, const std::vector<spk::KeyCut>& cuts,
                    std::vector<int32_t>& out, size_t n_front, std::vector<Item>& items) {
  for (int y = 0; y < p.n_real; ++y) {
    size_t next = 0;  // (cuts are in the order of the segments)
    for (const Seg& g : p.segs_k) {
      const bool is_cut = next < cuts.size() && cuts[next].ka == g.ka && g.kb > g.ka;
      const spk::KeyCut* cut = is_cut ? &cuts[next++] : nullptr;
      for (int a = g.ka; a < g.kb; a += BNK) {
        const int b = std::min(a + BNK, g.kb);
        int q0 = g.qa;
        if (d->causal) q0 = (int)std::max<int64_t>(g.qa, (int64_t)a - g.delta);
        const bool empty = q0 >= g.qb;
        if (cut) {  // (parts without rows write zeros)
          const int64_t n = std::max(0, g.qb - q0), rows = ((n + cut->parts - 1) / cut->parts + BQ - 1) / BQ * BQ;
          for (int i = 0; i < cut->parts; ++i) {
            const int r0 = (int)(g.qb - std::min(n, i * rows)), r1 = (int)(g.qb - std::min(n, (i + 1) * rows));
            const int at = cut->row + (i * p.n_real + y) * cut->len + (a - g.ka);
            items.push_back(Item{{a, b, r1, r0, g.delta, y, p.kv_of[y], 1 | (1 + at) << 2},
                                 r1 < r0 ? ((r0 - (r1 & ~7)) + BQ - 1) / BQ : 0});
          }
          continue;
        }
        Item it{{a, b, empty ? g.qb : q0, g.qb, g.delta, y, p.kv_of[y], 1}, 0};
        it.cost = empty ? 0 : (int64_t)((g.qb - (q0 & ~7)) + BQ - 1) / BQ;
        items.push_back(it);
      }
    }
    for (int a = p.k_pad; a < d->T_k; a += BNK)
      items.push_back(Item{{a, std::min(a + BNK, d->T_k), 0, 0, 0, y, p.kv_of[y], 1}, 0});
  }
  sort_items(items, out, n_front, false);
  return costs_of(items);
}

// Row and key items of a backward in one launch as one list, longest first by the
// model's time a step.  (Whole lists one after the other end with the second list's
// longest items: 4 groups of a prompt and 8 answers, 20730 rows, 4 heads, dQ's behind
// dK/dV's, 273 -> 255 us.)
std::vector<int32_t> merged_items(const std::vector<Item>& rows, const std::vector<Item>& keys, size_t n_front) {
  std::vector<Item> all;
  for (const Item& x : rows) {
    all.push_back(x);
    all.back().cost = std::llrint((double)x.cost * kSplitDq.step * 1e3);
  }
  for (const Item& x : keys) {
    all.push_back(x);
    all.back().cost = std::llrint((double)x.cost * kSplitDkdv.step * 1e3);
  }
  std::vector<int32_t> out;
  sort_items(all, out, n_front, false);
  return out;
}

// A shared-prefix forward of few rows: tiles of two slots, whose keys are cut into
// `parts`.  Taken where the model sees a fifth less time in it than in whole walks -- a
// workgroup takes kStartUs and its stages of four key tiles, kFewStageUs each, and the
// merge kFewJoinUs and the partial results' way out and back -- and where tiles and
// windows fit the launch's own list: a copy of them would take longer than it gains
// (a prompt of 1689 rows and 13 answers of 39, copied, 37 us, in whole walks 23).  16
// answers of one row to 32768 keys, 7 heads: 308 -> 21 us; 64 answers to 8192 keys, 4
// heads, 78 -> 17.  (Over 40 drawn sizes with parts 0.85 to 8.9 times as fast, 2.1 at the
// median; the losses are single calls of 12 to 16 us.)
constexpr double kFewStageUs = 1.6, kFewJoinUs = 8, kFewBytesUs = 2e6;
constexpr int kFewSlots = 2, kFewSplit = kSlots / kFewSlots;
struct FewPlan {
  int parts = 0;  // 0: not possible
  double us = 0;  // the model's time
  std::vector<spk::FewTile> tiles;
};
FewPlan few_plan(const sp_attn_desc* d, const Problem& p) {
  constexpr size_t kInts = std::size(decltype(spk::ItemList::v){});
  FewPlan f;
  if (p.prefix.empty() || p.n_real == 0 || d->T_q == 0 || (size_t)2 * d->T_q > kInts) return f;
  if ((int64_t)d->T_q * p.n_real > (int64_t)kCus / 2 * kFewSlots * kSlotRows) return f;
  int longest = 0;
  const int BN = spk::fwd_tile_keys(p.D, kFewSplit);
  for (int kv = 0; kv < d->Hkv_loc; ++kv) {
    const int n = p.kv_hi[kv] - p.kv_lo[kv], blocks = (n + kSlotRows - 1) / kSlotRows;
    for (int b = 0; b < blocks; ++b) {
      const int h0 = p.kv_lo[kv] + n * b / blocks, heads = p.kv_lo[kv] + n * (b + 1) / blocks - h0;
      const int rows = kFewSlots * (kSlotRows / heads);
      // rows of one prefix after the other, segment by segment (then those behind
      // the last segment, which see nothing)
      spk::FewTile t{0, 0, 0, 0, 0, 0, h0 | heads << 16, kv};
      int of = -1;
      auto flush = [&] {
        if (t.row1 > t.row0) {
          longest = std::max(longest, spk::few_steps(t.p0, t.p1, BN) + spk::few_steps(t.k0, t.k1, BN));
          f.tiles.push_back(t);
        }
        t.row0 = t.row1;
        t.k0 = t.k1 = 0;
      };
      auto add = [&](const Seg& g, int prefix) {
        if (g.qb <= g.qa) return;
        if (prefix != of) flush();
        of = prefix;
        t.p0 = prefix >= 0 ? p.segs[prefix].ka : 0;
        t.p1 = prefix >= 0 ? p.segs[prefix].kb : 0;
        for (int a = g.qa; a < g.qb; a = t.row1) {
          if (t.row1 - t.row0 == rows) flush();
          t.row1 = std::min(g.qb, t.row0 + rows);
          const int k1 = d->causal ? (int)std::min<int64_t>(g.kb, (int64_t)t.row1 + g.delta) : g.kb;
          if (k1 <= g.ka) continue;
          t.k0 = t.k1 > t.k0 ? std::min(t.k0, g.ka) : g.ka;
          t.k1 = std::max(t.k1, k1);
        }
      };
      for (size_t s = 0; s < p.segs.size(); ++s) add(p.segs[s], p.prefix[s]);
      add(Seg{p.q_pad, d->T_q, 0, 0, 0}, -1);
      flush();
      if (f.tiles.size() * 2 > kCus || f.tiles.size() * kItemInts + 2 * d->T_q > kInts) return f;
    }
  }
  const int stages = (longest + kFewSplit - 1) / kFewSplit;  // of four tiles
  const int parts = (int)std::min<size_t>({kCus / f.tiles.size(), (size_t)stages / 2, (size_t)spk::kMaxParts});
  if (parts < 2) return f;
  f.parts = parts;
  f.us = kStartUs + (double)((stages + parts - 1) / parts) * kFewStageUs + kFewJoinUs +
         2.0 * parts * d->T_q * d->H_loc * p.D * 4 / kFewBytesUs;
  return f;
}
// Whether it is taken; `whole_us`: the model's time of the launch without parts.
bool few_taken(const FewPlan& f, double whole_us) { return f.parts > 0 && f.us < 0.8 * whole_us; }
// Own keys [begin, end) of every row.
void few_windows(const sp_attn_desc* d, const Problem& p, int32_t* out) {
  std::fill(out, out + (size_t)2 * d->T_q, 0);
  for (const Seg& g : p.segs)
    for (int i = g.qa; i < g.qb; ++i) {
      const int k1 = d->causal ? (int)std::min<int64_t>(g.kb, (int64_t)i + g.delta + 1) : g.kb;
      out[2 * i] = g.ka;
      out[2 * i + 1] = std::max(g.ka, k1);
    }
}

// Zero fills as work items of the same launch (no extra kernels): dummy
// query slots (O = +0 and LSE = -inf, in the ring variant the accumulators'
// identity; dQ = +0) and, in the direct dK/dV mode, KV heads no real query
// head reads (dK = dV = +0).  One item covers kFillRows rows of one head;
// the items go to the FRONT of the list, so they finish in microseconds on
// a few CUs while the longest items start.
std::vector<int32_t> row_fills(const sp_attn_desc* d, const Problem& p) {
  std::vector<int32_t> out;
  for (int y = p.n_real; y < d->H_loc; ++y)
    for (int a = 0; a < d->T_q; a += spk::kFillRows) {
      const int32_t it[kItemInts] = {a, std::min(a + spk::kFillRows, d->T_q), 0, 0, 0, y, 0,
                                     spk::kItemFillQ};
      out.insert(out.end(), it, it + kItemInts);
    }
  return out;
}
bool kv_unread(const Problem& p, int kv) { return p.n_real == 0 || p.kv_hi[kv] == p.kv_lo[kv]; }
std::vector<int32_t> key_fills(const sp_attn_desc* d, const Problem& p) {
  std::vector<int32_t> out;
  if (!p.direct && p.n_real > 0) return out;  // the GQA reduction writes every KV head
  for (int kv = 0; kv < d->Hkv_loc; ++kv) {
    if (!kv_unread(p, kv)) continue;
    for (int a = 0; a < d->T_k; a += spk::kFillRows) {
      const int32_t it[kItemInts] = {a, std::min(a + spk::kFillRows, d->T_k), 0, 0, 0, 0, kv,
                                     spk::kItemFillKV};
      out.insert(out.end(), it, it + kItemInts);
    }
  }
  return out;
}
void prepend(std::vector<int32_t> fills, std::vector<int32_t>& items) {
  if (!fills.empty()) items.insert(items.begin(), fills.begin(), fills.end());
}
int n_unread_kv(const sp_attn_desc* d, const Problem& p) {
  if (!p.direct && p.n_real > 0) return 0;
  int n = 0;
  for (int kv = 0; kv < d->Hkv_loc; ++kv) n += kv_unread(p, kv);
  return n;
}

// Workspace layout.
struct Layout {
  size_t items_dq = 0, items_kv = 0, neg_d = 0, lse2 = 0, part_k = 0, part_v = 0, total = 0;
  size_t few_o = 0, few_lse = 0;  // a forward of few rows
  size_t cut_k = 0, cut_v = 0;    // parts of a backward's cut items
};

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

Layout layout_for(const sp_attn_desc* d, const Problem& p, int op, size_t n_items_a,
                  size_t n_items_b, int64_t n_cut_rows = 0) {
  Layout L;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    size_t o = off;
    off = align256(off + bytes);
    return o;
  };
  const size_t D = p.D;
  if (op == SP_OP_FWD || op == SP_OP_RING_STEP) {
    L.items_dq = take(n_items_a * kItemInts * 4);
  } else {
    // the row statistics first: their offsets depend on T_q and the real
    // heads only, so calls over other KV chunks can reuse them
    // (SP_DESC_ROWSTATS_READY)
    L.neg_d = take((size_t)std::max(p.n_real, 1) * d->T_q * 4);
    L.lse2 = take((size_t)std::max(p.n_real, 1) * d->T_q * 4);
    L.items_dq = take(n_items_a * kItemInts * 4);
    L.items_kv = take(n_items_b * kItemInts * 4);
    if (!p.direct) {
      L.part_k = take((size_t)p.n_real * d->T_k * D * 4);
      L.part_v = take((size_t)p.n_real * d->T_k * D * 4);
    }
    L.cut_k = take((size_t)n_cut_rows * D * 4);
    L.cut_v = take((size_t)n_cut_rows * D * 4);
  }
  L.total = std::max<size_t>(off, 256);
  return L;
}

// Workspace of a shared-prefix forward of few rows: the partial results.
Layout layout_few(const sp_attn_desc* d, const Problem& p, const FewPlan& f) {
  Layout L;
  const size_t rows = (size_t)f.parts * d->T_q * d->H_loc;
  L.few_lse = align256(rows * p.D * 4);
  L.total = L.few_lse + align256(rows * 4);
  return L;
}

// Item counts of schedule_rows with empty items included (the worst case
// the workspace is sized for) and of schedule_keys, without building them.
// (With the zero-fill items appended at launch.)
size_t row_item_count(const sp_attn_desc* d, const Problem& p, int BM) {
  const size_t fills =
      (size_t)(d->H_loc - p.n_real) * (size_t)((d->T_q + spk::kFillRows - 1) / spk::kFillRows);
  if (!p.prefix.empty()) {  // the records lie behind the items
    const size_t tiles = row_tiles(d, p).size();
    return tiles * (size_t)p.n_real + fills + record_room(tiles) / kItemInts;
  }
  size_t per_head = 0;
  for (const Seg& g : p.segs) per_head += (size_t)((g.qb - g.qa) + BM - 1) / BM;
  per_head += (size_t)((d->T_q - p.q_pad) + BM - 1) / BM;
  return per_head * (size_t)p.n_real + fills;
}
size_t key_item_count(const sp_attn_desc* d, const Problem& p, const std::vector<spk::KeyCut>& cuts, int BNK) {
  size_t per_head = 0;
  for (const spk::KeyCut& c : cuts) per_head += (size_t)(c.parts - 1) * ((c.len + BNK - 1) / BNK);
  for (const Seg& g : p.segs_k) per_head += (size_t)((g.kb - g.ka) + BNK - 1) / BNK;
  per_head += (size_t)((d->T_k - p.k_pad) + BNK - 1) / BNK;
  const size_t fills =
      (size_t)n_unread_kv(d, p) * (size_t)((d->T_k + spk::kFillRows - 1) / spk::kFillRows);
  return per_head * (size_t)p.n_real + fills;
}

// Worst-case item counts (with empty items) for sizing.
void item_counts(const sp_attn_desc* d, const Problem& p, int op, const std::vector<spk::KeyCut>& cuts, size_t& a,
                 size_t& b) {
  if (op == SP_OP_BWD) {
    a = row_item_count(d, p, spk::kDqBM);
    b = key_item_count(d, p, cuts, spk::kDkdvBN);
  } else {
    a = row_item_count(d, p, spk::kFwdBM);
    b = 0;
  }
}

inline bool aligned16(const void* ptr) { return ((uintptr_t)ptr & 15u) == 0; }

#define SP_HIP(call)                          \
  do {                                        \
    if ((call) != hipSuccess) return SP_ERR_HIP; \
  } while (0)

sp_status upload(void* dst, const std::vector<int32_t>& v, hipStream_t st) {
  if (v.empty()) return SP_OK;
  SP_HIP(hipMemcpyAsync(dst, v.data(), v.size() * sizeof(int32_t), hipMemcpyHostToDevice, st));
  return SP_OK;
}

// The attention entry points copy host-built work lists that do not fit the
// kernel arguments, which a captured graph would replay from freed host
// memory: they refuse a stream that is being captured, whatever the list.
sp_status refuse_capture(hipStream_t st) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &cs) != hipSuccess) return SP_ERR_HIP;
  return cs == hipStreamCaptureStatusNone ? SP_OK : SP_ERR_UNSUPPORTED;
}

sp_status check_ws(const Layout& L, void* ws, size_t ws_bytes) {
  if (!ws || ws_bytes < L.total || ((uintptr_t)ws & 255u) != 0) return SP_ERR_WORKSPACE;
  return SP_OK;
}

char* at(void* ws, size_t off) { return (char*)ws + off; }

}  // namespace

namespace spk {
KernelTimer& timer_for(int kernel_id) {
  static thread_local KernelTimer slots[kKCount];
  return slots[(kernel_id > 0 && kernel_id < kKCount) ? kernel_id : 0];
}
}  // namespace spk

extern "C" {

sp_status sp_profile_events(int32_t kernel_id, void* start_event, void* stop_event) {
  if (kernel_id < 1 || kernel_id >= spk::kKCount) return SP_ERR_INVALID_ARG;
  spk::KernelTimer& t = spk::timer_for(kernel_id);
  t.start = (hipEvent_t)start_event;
  t.stop = (hipEvent_t)stop_event;
  return SP_OK;
}

const char* sp_status_string(sp_status s) {
  switch (s) {
    case SP_OK: return "ok";
    case SP_ERR_INVALID_ARG: return "invalid argument";
    case SP_ERR_UNSUPPORTED: return "unsupported configuration";
    case SP_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case SP_ERR_HIP: return "HIP launch or copy failed";
  }
  return "unknown status";
}

int32_t sp_version(void) { return 100; }

sp_status sp_ulysses_pack(const void* src, int32_t T_loc, int32_t H_src, int32_t head_dim,
                          int32_t sp, int32_t H_dst_loc, const int32_t* head_map, void* dst,
                          void* stream) {
  if (T_loc < 0 || H_src < 1 || head_dim < 8 || head_dim % 8 != 0 || sp < 1 || H_dst_loc < 1 ||
      !head_map)
    return SP_ERR_INVALID_ARG;
  if ((int64_t)sp * H_dst_loc > spk::kMaxMap) return SP_ERR_UNSUPPORTED;
  spk::PackArgs a;
  a.sp = sp; a.T = T_loc; a.Hs = H_src; a.Hd = H_dst_loc; a.nch = head_dim / 8;
  for (int i = 0; i < sp * H_dst_loc; ++i) {
    if (head_map[i] < -1 || head_map[i] >= H_src) return SP_ERR_INVALID_ARG;
    a.map[i] = head_map[i];
  }
  if (T_loc == 0) return SP_OK;
  if (!src || !dst || !aligned16(src) || !aligned16(dst)) return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_pack(src, dst, a, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_ulysses_unpack(const void* src, int32_t T_loc, int32_t H_src_loc, int32_t head_dim,
                            int32_t sp, const int32_t* head_map, int32_t H_dst, void* dst,
                            void* stream) {
  if (T_loc < 0 || H_src_loc < 1 || head_dim < 8 || head_dim % 8 != 0 || sp < 1 || H_dst < 1 ||
      !head_map)
    return SP_ERR_INVALID_ARG;
  if ((int64_t)sp * H_src_loc > spk::kMaxMap || H_dst > spk::kMaxMap) return SP_ERR_UNSUPPORTED;
  spk::PackArgs a;
  a.sp = sp; a.T = T_loc; a.Hs = H_src_loc; a.Hd = H_dst; a.nch = head_dim / 8;
  std::vector<int> seen(H_dst, 0);
  for (int i = 0; i < sp * H_src_loc; ++i) {
    int g = head_map[i];
    if (g < -1 || g >= H_dst) return SP_ERR_INVALID_ARG;
    if (g >= 0) {
      if (seen[g]++) return SP_ERR_INVALID_ARG;
      a.map[g] = i;  // inverse map: dest head -> j*H_src_loc + h
    }
  }
  for (int g = 0; g < H_dst; ++g)
    if (seen[g] != 1) return SP_ERR_INVALID_ARG;
  if (T_loc == 0) return SP_OK;
  if (!src || !dst || !aligned16(src) || !aligned16(dst)) return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_unpack(src, dst, a, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_ulysses_unpack_add(const void* src, int32_t T_loc, int32_t H_src_loc,
                                int32_t head_dim, int32_t sp, const int32_t* head_map,
                                int32_t H_dst, void* dst, void* stream) {
  if (T_loc < 0 || H_src_loc < 1 || head_dim < 8 || head_dim % 8 != 0 || sp < 1 || H_dst < 1 ||
      !head_map)
    return SP_ERR_INVALID_ARG;
  if ((int64_t)sp * H_src_loc > spk::kMaxMap || H_dst > spk::kMaxAddDst) return SP_ERR_UNSUPPORTED;
  spk::PackAddArgs a;
  a.sp = sp; a.T = T_loc; a.Hs = H_src_loc; a.Hd = H_dst; a.nch = head_dim / 8;
  // counting sort of the slots by destination head keeps each head's slots
  // in ascending order
  std::vector<int> cnt(H_dst + 1, 0);
  const int n_slots = sp * H_src_loc;
  for (int i = 0; i < n_slots; ++i) {
    const int g = head_map[i];
    if (g < -1 || g >= H_dst) return SP_ERR_INVALID_ARG;
    if (g >= 0) ++cnt[g + 1];
  }
  for (int g = 0; g < H_dst; ++g) cnt[g + 1] += cnt[g];
  for (int g = 0; g <= H_dst; ++g) a.start[g] = (int16_t)cnt[g];
  std::vector<int> fill(cnt.begin(), cnt.end() - 1);
  for (int i = 0; i < n_slots; ++i)
    if (head_map[i] >= 0) a.slot[fill[head_map[i]]++] = (int16_t)i;
  if (T_loc == 0) return SP_OK;
  if (!src || !dst || !aligned16(src) || !aligned16(dst)) return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_unpack_add(src, dst, a, (hipStream_t)stream));
  return SP_OK;
}

namespace {
// Shared validation of the loss calls: vocabulary, sequences (host copy),
// alignment.  Fills the kernel arguments.
sp_status loss_args(int32_t T, int32_t V, int32_t ignore_index, const int32_t* cu,
                    int32_t num_seqs, spk::LossArgs& a) {
  if (T < 0 || V < 8 || V % 8 != 0 || num_seqs < 0) return SP_ERR_INVALID_ARG;
  if (num_seqs > spk::kMaxLossSeqs) return SP_ERR_UNSUPPORTED;
  if (num_seqs > 0 && !cu) return SP_ERR_INVALID_ARG;
  a.T = T; a.V = V; a.ignore_index = ignore_index; a.n_seqs = num_seqs;
  a.cu[0] = num_seqs > 0 ? cu[0] : 0;
  if (a.cu[0] < 0) return SP_ERR_INVALID_ARG;
  for (int s = 0; s < num_seqs; ++s) {
    if (cu[s + 1] < cu[s]) return SP_ERR_INVALID_ARG;
    a.cu[s + 1] = cu[s + 1];
  }
  if (a.cu[num_seqs] > T) return SP_ERR_INVALID_ARG;
  return SP_OK;
}
}  // namespace

sp_status sp_token_logprob(const void* logits, const int32_t* labels, int32_t T, int32_t V,
                           int32_t ignore_index, const int32_t* cu_seqlens, int32_t num_seqs,
                           float* logp, float* lse, float* seq_sum, void* stream) {
  spk::LossArgs a;
  sp_status st = loss_args(T, V, ignore_index, cu_seqlens, num_seqs, a);
  if (st != SP_OK) return st;
  if (T > 0 && (!logits || !labels || !logp || !lse || !aligned16(logits)))
    return SP_ERR_INVALID_ARG;
  if (num_seqs > 0 && !seq_sum) return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_token_logprob(a, logits, labels, logp, lse, seq_sum, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_token_logprob_bwd(const void* logits, const int32_t* labels, const float* lse,
                               int32_t T, int32_t V, int32_t ignore_index,
                               const int32_t* cu_seqlens, int32_t num_seqs,
                               const float* grad_seq, void* dlogits, void* stream) {
  spk::LossArgs a;
  sp_status st = loss_args(T, V, ignore_index, cu_seqlens, num_seqs, a);
  if (st != SP_OK) return st;
  if (T == 0) return SP_OK;
  if (!logits || !labels || !lse || !dlogits || !aligned16(logits) || !aligned16(dlogits) ||
      (num_seqs > 0 && !grad_seq))
    return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_token_logprob_bwd(a, logits, labels, lse, grad_seq, dlogits,
                                       (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_loss_reduce(const float* partial_sums, const float* ref_partial_sums, int32_t sp,
                         int32_t num_seqs, int32_t kind, float coef, float* loss, float* grad,
                         void* stream) {
  if (sp < 1 || num_seqs < 1 || (kind != SP_LOSS_SFT && kind != SP_LOSS_DPO) || !partial_sums ||
      !loss || !grad || !std::isfinite(coef))
    return SP_ERR_INVALID_ARG;
  if (kind == SP_LOSS_DPO && (num_seqs % 2 != 0 || !ref_partial_sums)) return SP_ERR_INVALID_ARG;
  if (num_seqs > 256 || sp > 4096) return SP_ERR_UNSUPPORTED;
  spk::LossReduceArgs a;
  a.sp = sp; a.n = num_seqs; a.kind = kind; a.coef = coef;
  SP_HIP(spk::launch_loss_reduce(a, partial_sums, ref_partial_sums, loss, grad,
                                 (hipStream_t)stream));
  return SP_OK;
}

namespace {
// Validation shared by the policy calls; fills the kernel arguments.
sp_status policy_args(const sp_policy_params* p, int32_t T, int32_t V, const int32_t* cu, int32_t num_seqs,
                      const float* ref_logp, const float* entropy, spk::LossArgs& a, spk::PolicyArgs& k) {
  if (!p) return SP_ERR_INVALID_ARG;
  sp_status st = loss_args(T, V, p->ignore_index, cu, num_seqs, a);
  if (st != SP_OK) return st;
  if (T >= 1 << 24) return SP_ERR_UNSUPPORTED;
  if (!(p->clip_low >= 0.f && p->clip_low <= 1.f) || !(p->clip_high >= 0.f) || !std::isfinite(p->clip_high) ||
      !std::isfinite(p->kl_coef) || !std::isfinite(p->entropy_coef) || (p->adv_per_token != 0 && p->adv_per_token != 1))
    return SP_ERR_INVALID_ARG;
  if ((!ref_logp && p->kl_coef != 0.f) || (!entropy && p->entropy_coef != 0.f)) return SP_ERR_INVALID_ARG;
  k = spk::PolicyArgs{p->clip_low, p->clip_high, p->kl_coef, p->entropy_coef, p->adv_per_token, ref_logp != nullptr,
                      entropy != nullptr, spk::policy_parts(T, V)};
  return SP_OK;
}
}  // namespace

sp_status sp_policy_workspace_size(int32_t T, int32_t V, size_t* bytes) {
  if (!bytes || T < 0 || V < 8 || V % 8 != 0) return SP_ERR_INVALID_ARG;
  if (T >= 1 << 24) return SP_ERR_UNSUPPORTED;
  *bytes = spk::policy_workspace(T, V);
  return SP_OK;
}

sp_status sp_policy_loss(const sp_policy_params* params, const void* logits, const int32_t* labels,
                         const float* old_logp, const float* ref_logp, const float* advantages,
                         int32_t T, int32_t V, const int32_t* cu_seqlens, int32_t num_seqs,
                         float* logp, float* lse, float* entropy, float* seq_sum,
                         float* seq_stats, void* workspace, size_t workspace_bytes, void* stream) {
  spk::LossArgs a;
  spk::PolicyArgs k;
  sp_status st = policy_args(params, T, V, cu_seqlens, num_seqs, ref_logp, entropy, a, k);
  if (st != SP_OK) return st;
  if (T > 0 && (!logits || !labels || !old_logp || !logp || !lse || !aligned16(logits))) return SP_ERR_INVALID_ARG;
  if (num_seqs > 0 && (!seq_sum || !seq_stats)) return SP_ERR_INVALID_ARG;
  if (T > 0 && num_seqs > 0 && !advantages) return SP_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < spk::policy_workspace(T, V) || ((uintptr_t)workspace & 255u) != 0)
    return SP_ERR_WORKSPACE;
  const spk::PolicyTokens tok{labels, old_logp, ref_logp, advantages, logp, lse, entropy};
  SP_HIP(spk::launch_policy_loss(a, k, logits, tok, workspace, seq_sum, seq_stats, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_policy_loss_bwd(const sp_policy_params* params, const void* logits,
                             const int32_t* labels, const float* logp, const float* lse,
                             const float* entropy, const float* old_logp, const float* ref_logp,
                             const float* advantages, int32_t T, int32_t V,
                             const int32_t* cu_seqlens, int32_t num_seqs, const float* grad_seq,
                             void* dlogits, void* stream) {
  spk::LossArgs a;
  spk::PolicyArgs k;
  sp_status st = policy_args(params, T, V, cu_seqlens, num_seqs, ref_logp, entropy, a, k);
  if (st != SP_OK) return st;
  if (T == 0) return SP_OK;
  if (!logits || !labels || !logp || !lse || !old_logp || !dlogits || !aligned16(logits) || !aligned16(dlogits) ||
      (num_seqs > 0 && (!grad_seq || !advantages)))
    return SP_ERR_INVALID_ARG;
  const spk::PolicyTokens tok{labels, old_logp, ref_logp, advantages, const_cast<float*>(logp), const_cast<float*>(lse),
                              const_cast<float*>(entropy)};
  SP_HIP(spk::launch_policy_loss_bwd(a, k, logits, tok, grad_seq, dlogits, (hipStream_t)stream));
  return SP_OK;
}

namespace {
// radians / 2 pi in 2^-64 turns, whole turns dropped: the product as a sum of two
// doubles, whose error is below 2^-104 of it.
uint64_t turns64(double radians) {
  constexpr double kInv = 0x1.45f306dc9c883p-3, kInvLow = -0x1.6b01ec5417056p-57;  // 1 / 2 pi
  const double hi = radians * kInv, lo = std::fma(radians, kInv, -hi) + radians * kInvLow;
  const double frac = hi - std::floor(hi);  // (exact, in [0, 1]: 1 for a tiny negative hi)
  const uint64_t part = frac < 1.0 ? (uint64_t)(frac * 0x1p64) : 0;
  const double low = std::fabs(lo) < 0.25 ? lo : std::fmod(lo, 0.25);
  return part + (uint64_t)(int64_t)std::llrint(low * 0x1p64);
}

// The slots of a map in the order of their heads (ascending within a head, those
// without one last), and where each head's begin; false for a bad entry.
bool by_head(const int32_t* map, int sp, int H_loc, int H, uint32_t* slot, int* start) {
  const int n = sp * H_loc;
  int next[spk::kMaxQkHeads + 1] = {};
  for (int i = 0; i < n; ++i) {
    if (map[i] < -1 || map[i] >= H) return false;
    if (map[i] >= 0) ++next[map[i]];
  }
  int at = 0;
  for (int g = 0; g < H; ++g) {
    start[g] = at;
    at += next[g];
    next[g] = start[g];
  }
  start[H] = next[H] = at;
  for (int j = 0, i = 0; j < sp; ++j)
    for (int h = 0; h < H_loc; ++h, ++i) slot[next[map[i] < 0 ? H : map[i]]++] = (uint32_t)h | (uint32_t)j << 10;
  return true;
}

// Validation of a sp_qk_desc; fills the forward's kernel arguments.
sp_status qk_args(const sp_qk_desc* d, spk::QkArgs& a) {
  if (!d) return SP_ERR_INVALID_ARG;
  if (d->T < 0 || d->H_q < 1 || d->H_kv < 1 || d->sp < 1 || d->Hq_loc < 1 || d->Hkv_loc < 1 || d->rotary_dim < 0 ||
      (d->interleaved != 0 && d->interleaved != 1) || !d->q_map || !d->kv_map || (d->rotary_dim > 0 && !d->inv_freq))
    return SP_ERR_INVALID_ARG;
  if (d->head_dim != 64 && d->head_dim != 128) return SP_ERR_UNSUPPORTED;
  if (d->rotary_dim % 16 != 0 || d->rotary_dim > d->head_dim) return SP_ERR_INVALID_ARG;
  if (!std::isfinite(d->rope_scale) || !std::isfinite(d->weight_offset) || !(d->eps >= 0.f) || !std::isfinite(d->eps))
    return SP_ERR_INVALID_ARG;
  if ((int64_t)d->sp * d->Hq_loc > spk::kMaxMap || (int64_t)d->sp * d->Hkv_loc > spk::kMaxMap ||
      d->H_q > spk::kMaxQkHeads || d->H_kv > spk::kMaxQkHeads || d->T >= 1 << 24)
    return SP_ERR_UNSUPPORTED;
  a.T = d->T; a.Hq = d->H_q; a.Hkv = d->H_kv; a.sp = d->sp; a.Hq_loc = d->Hq_loc; a.Hkv_loc = d->Hkv_loc;
  a.rot = d->rotary_dim; a.neigh = d->interleaved; a.pos_base = d->position_base;
  a.rope_scale = d->rope_scale; a.eps = d->eps; a.w_off = d->weight_offset;
  for (int i = 0; i < d->rotary_dim / 2; ++i) {
    if (!std::isfinite(d->inv_freq[i])) return SP_ERR_INVALID_ARG;
    a.freq[i] = turns64(d->inv_freq[i]);
  }
  if (!by_head(d->q_map, d->sp, d->Hq_loc, d->H_q, a.q_slot, a.q_start) ||
      !by_head(d->kv_map, d->sp, d->Hkv_loc, d->H_kv, a.kv_slot, a.kv_start))
    return SP_ERR_INVALID_ARG;
  return SP_OK;
}
bool qk_stride_ok(const sp_qk_desc* d, int64_t stride, int H) {
  return stride % 8 == 0 && stride >= (int64_t)H * d->head_dim && stride < (int64_t(1) << 26);
}
size_t qk_workspace(const spk::QkArgs& a, int D) {
  return align256((size_t)spk::qk_bwd_groups(a, D) * 2 * D * sizeof(float));
}
}  // namespace

sp_status sp_qk_norm_rope(const sp_qk_desc* d, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                          const void* v, int64_t v_stride, const int32_t* positions, const void* w_q, const void* w_k,
                          void* q_dst, void* k_dst, void* v_dst, void* stream) {
  spk::QkArgs a{};
  sp_status s = qk_args(d, a);
  if (s != SP_OK) return s;
  if (!qk_stride_ok(d, q_stride, d->H_q) || !qk_stride_ok(d, k_stride, d->H_kv) || !qk_stride_ok(d, v_stride, d->H_kv))
    return SP_ERR_INVALID_ARG;
  if (d->T == 0) return SP_OK;
  for (const void* ptr : {q, k, v, (const void*)q_dst, (const void*)k_dst, (const void*)v_dst})
    if (!ptr || !aligned16(ptr)) return SP_ERR_INVALID_ARG;
  if (!aligned16(w_q) || !aligned16(w_k)) return SP_ERR_INVALID_ARG;
  a.sq = q_stride / 8; a.sk = k_stride / 8; a.sv = v_stride / 8;
  SP_HIP(spk::launch_qk_rope(a, d->head_dim, q, k, v, positions, w_q, w_k, q_dst, k_dst, v_dst, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_qk_workspace_size(const sp_qk_desc* d, size_t* bytes) {
  if (!bytes) return SP_ERR_INVALID_ARG;
  spk::QkArgs a;
  sp_status s = qk_args(d, a);
  if (s != SP_OK) return s;
  *bytes = qk_workspace(a, d->head_dim);
  return SP_OK;
}

sp_status sp_qk_norm_rope_bwd(const sp_qk_desc* d, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                              const void* dq_src, const void* dk_src, const void* dv_src, const int32_t* positions,
                              const void* w_q, const void* w_k, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride,
                              void* dv, int64_t dv_stride, float* dw_q, float* dw_k, void* ws, size_t ws_bytes,
                              void* stream) {
  spk::QkArgs a{};
  sp_status s = qk_args(d, a);
  if (s != SP_OK) return s;
  if (!qk_stride_ok(d, dq_stride, d->H_q) || !qk_stride_ok(d, dk_stride, d->H_kv) || !qk_stride_ok(d, dv_stride, d->H_kv) ||
      (w_q && !qk_stride_ok(d, q_stride, d->H_q)) || (w_k && !qk_stride_ok(d, k_stride, d->H_kv)))
    return SP_ERR_INVALID_ARG;
  if (!w_q != !dw_q || !w_k != !dw_k) return SP_ERR_INVALID_ARG;
  if (d->T > 0) {
    for (const void* ptr : {dq_src, dk_src, dv_src, (const void*)dq, (const void*)dk, (const void*)dv})
      if (!ptr || !aligned16(ptr)) return SP_ERR_INVALID_ARG;
    if ((w_q && !q) || (w_k && !k)) return SP_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(w_q) || !aligned16(w_k)) return SP_ERR_INVALID_ARG;
  }
  if (!ws || ws_bytes < qk_workspace(a, d->head_dim) || ((uintptr_t)ws & 255u) != 0) return SP_ERR_WORKSPACE;
  a.sq = q_stride / 8; a.sk = k_stride / 8;
  const spk::QkStrides o{dq_stride / 8, dk_stride / 8, dv_stride / 8};
  SP_HIP(spk::launch_qk_rope_bwd(a, o, d->head_dim, q, k, dq_src, dk_src, dv_src, positions, w_q, w_k, dq, dk, dv, dw_q, dw_k,
                                 w_q || w_k ? (float*)ws : nullptr, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_attn_workspace_size(const sp_attn_desc* desc, int32_t op, size_t* bytes) {
  if (!bytes) return SP_ERR_INVALID_ARG;
  if (op != SP_OP_FWD && op != SP_OP_BWD && op != SP_OP_RING_STEP) return SP_ERR_INVALID_ARG;
  Problem p;
  sp_status s = validate(desc, p);
  if (s != SP_OK) return s;
  if (op == SP_OP_RING_STEP && !p.prefix.empty()) return SP_ERR_UNSUPPORTED;
  size_t a = 0, b = 0;
  const std::vector<spk::KeyCut> cuts = op == SP_OP_BWD ? key_cuts(desc, p) : std::vector<spk::KeyCut>();
  item_counts(desc, p, op, cuts, a, b);
  *bytes = layout_for(desc, p, op, a, b, cut_rows(p, cuts)).total;
  if (op == SP_OP_FWD) {  // (either way of a shared-prefix forward fits)
    const FewPlan f = few_plan(desc, p);
    if (f.parts) *bytes = std::max(*bytes, layout_few(desc, p, f).total);
  }
  return SP_OK;
}

sp_status sp_attn_schedule(const sp_attn_desc* desc, int32_t op, int32_t* items, int32_t capacity,
                           int32_t* n_items) {
  if (!n_items || capacity < 0) return SP_ERR_INVALID_ARG;
  Problem p;
  sp_status s = validate(desc, p);
  if (s != SP_OK) return s;
  std::vector<int32_t> v;
  std::vector<Item> items_;
  // in launch order: the fill items that precede the listed ones there
  // shift the workgroup -> XCD map
  if ((op == SP_OP_FWD || op == SP_OP_RING_STEP) && !p.prefix.empty()) {
    if (op == SP_OP_RING_STEP) return SP_ERR_UNSUPPORTED;
    const std::vector<RowTile> tiles = row_tiles(desc, p);
    std::vector<int32_t> it;
    schedule_tiles(desc, p, tiles, spk::kFwdBN, it, row_fills(desc, p).size() / kItemInts, items_);
    for (size_t i = 0; i < it.size(); i += kItemInts) {  // slot by slot
      const RowTile& t = tiles[it[i]];
      for (const spk::RowSlot& s : t.slots) {
        const auto own = own_keys(desc, s);
        v.insert(v.end(), {s.row0, s.row1, own.first, own.second, s.delta, it[i + 5], it[i + 6], 0});
        if (t.prefix >= 0)
          v.insert(v.end(), {s.row0, s.row1, p.segs[t.prefix].ka, p.segs[t.prefix].kb, 1 << 30, it[i + 5], it[i + 6], 0});
      }
    }
  } else if (op == SP_OP_FWD || op == SP_OP_RING_STEP)
    schedule_rows(desc, p, spk::kFwdBM, spk::kFwdBN, true, v,
                  row_fills(desc, p).size() / kItemInts);
  else if (op == SP_OP_BWD)
    schedule_keys(desc, p, spk::kDkdvBN, spk::kDkdvBQ, {}, v, key_fills(desc, p).size() / kItemInts, items_);
  else
    return SP_ERR_INVALID_ARG;
  const int32_t n = (int32_t)(v.size() / kItemInts);
  *n_items = n;
  if (items) std::memcpy(items, v.data(), sizeof(int32_t) * kItemInts * std::min(n, capacity));
  return SP_OK;
}

sp_status sp_attn_plan(const sp_attn_desc* desc, int32_t op, int32_t* plan) {
  if (!plan) return SP_ERR_INVALID_ARG;
  if (op != SP_OP_FWD && op != SP_OP_BWD && op != SP_OP_RING_STEP) return SP_ERR_INVALID_ARG;
  Problem p;
  sp_status s = validate(desc, p);
  if (s != SP_OK) return s;
  if (op == SP_OP_RING_STEP && !p.prefix.empty()) return SP_ERR_UNSUPPORTED;
  const std::vector<RowTile> tiles = p.prefix.empty() ? std::vector<RowTile>() : row_tiles(desc, p);
  std::vector<int32_t> v;
  std::vector<Item> rows;
  BwdPlan b{};
  if (op == SP_OP_BWD) {
    std::vector<Item> keys;
    const Costs q = schedule_row_items(desc, p, tiles, spk::kDqBM, spk::kDqBN, true, v, 0, rows);
    const Costs k = schedule_keys(desc, p, spk::kDkdvBN, spk::kDkdvBQ, key_cuts(desc, p), v, 0, keys);
    b = plan_bwd(q, k, p.D);
  } else {
    double us;
    b.q = choose_shape(schedule_row_items(desc, p, tiles, spk::kFwdBM, spk::kFwdBN, true, v, 0, rows), kSplitFwd,
                       p.D, us);
    const FewPlan few = few_plan(desc, p);
    if (few_taken(few, us)) b.k.split = few.parts;
  }
  const int32_t r[SP_PLAN_INTS] = {b.q.split, b.q.two, b.k.split, b.k.two, b.one, b.dq_first};
  std::copy(r, r + SP_PLAN_INTS, plan);
  return SP_OK;
}

}  // extern "C"

namespace {

// ---- Scratch of the allocation-free forward (sp_attn_fwd_static).  A
// file-scope device array: every GPU the library runs on holds its own copy
// at its own address until the process ends.  In host code `scratch` is a
// host-side stand-in, never a device address: the device copy's address is
// looked up once per device with hipGetSymbolAddress (that device current)
// and only that pointer is handed to kernels and copies.
__device__ __align__(256) unsigned char scratch[SP_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
std::atomic<void*> g_scratch_ptr[kMaxDevices];

// Device address of the current device's scratch (looked up on first use).
sp_status static_scratch(void** out) {
  int dev = -1;
  SP_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return SP_ERR_UNSUPPORTED;
  void* p = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (!p) {
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    p = g_scratch_ptr[dev].load(std::memory_order_relaxed);
    if (!p) {
      if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return SP_ERR_HIP;
      g_scratch_ptr[dev].store(p, std::memory_order_release);
    }
  }
  *out = p;
  return SP_OK;
}

// The stream must belong to the current device (the scratch looked up is
// that device's).
sp_status stream_on_current_device(hipStream_t st) {
  if (!st) return SP_OK;
  int cur = -1, sdev = -1;
  SP_HIP(hipGetDevice(&cur));
  SP_HIP(hipStreamGetDevice(st, &sdev));
  return sdev == cur ? SP_OK : SP_ERR_INVALID_ARG;
}

}  // namespace

extern "C" {

// A shared-prefix forward of few rows (arguments are checked).
static sp_status fwd_few(const sp_attn_desc* d, const Problem& p, const FewPlan& few, const void* q, const void* k,
                         const void* v, void* o, float* lse, void* ws, size_t ws_bytes, hipStream_t st) {
  const Layout L = layout_few(d, p, few);
  sp_status s = check_ws(L, ws, ws_bytes);
  if (s != SP_OK) return s;
  if ((s = refuse_capture(st)) != SP_OK) return s;
  spk::FwdArgs a{};
  spk::ItemList list{};
  std::memcpy(list.v, few.tiles.data(), few.tiles.size() * sizeof(spk::FewTile));
  few_windows(d, p, list.v + few.tiles.size() * kItemInts);
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.o = (uint16_t*)o; a.lse = lse;
  a.o_acc = (float*)at(ws, L.few_o); a.lse_acc = (float*)at(ws, L.few_lse);
  a.T_q = d->T_q; a.T_k = d->T_k; a.H = d->H_loc; a.Hkv = d->Hkv_loc;
  a.scale_log2 = d->softmax_scale * 1.4426950408889634f;
  a.n_items = (int)few.tiles.size();
  a.parts = few.parts;
  SP_HIP(spk::launch_attn_few(a, list, p.D, p.n_real, st));
  return SP_OK;
}

// Forward / ring step.  `static_ws`: the work list goes to the current
// device's static scratch instead of the caller's workspace (sp_attn_fwd_static).
static sp_status fwd_common(const sp_attn_desc* d, const void* q, const void* k, const void* v,
                            void* o, float* lse, float* o_acc, float* lse_acc, int init,
                            void* o_out, void* ws, size_t ws_bytes, void* stream, bool ring,
                            bool static_ws = false) {
  Problem p;
  sp_status s = validate(d, p);
  if (s != SP_OK) return s;
  // pointers are required for tensors that have elements: no query rows is a
  // no-op; no keys leaves every row with O = 0 and LSE = -inf
  if (d->T_q > 0 && !q) return SP_ERR_INVALID_ARG;
  if (d->T_k > 0 && (!k || !v)) return SP_ERR_INVALID_ARG;
  if (d->T_q > 0 && (ring ? (!o_acc || !lse_acc) : (!o || !lse))) return SP_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || (o && !aligned16(o)) ||
      (o_acc && !aligned16(o_acc)) || (o_out && !aligned16(o_out)))
    return SP_ERR_INVALID_ARG;
  if (init != 0 && init != 1) return SP_ERR_INVALID_ARG;
  const bool prefix = !p.prefix.empty();
  if (ring && prefix) return SP_ERR_UNSUPPORTED;
  if (d->T_q == 0) return SP_OK;
  const bool include_empty = !ring || init || o_out;
  std::vector<int32_t> items;
  const std::vector<int32_t> fills = include_empty ? row_fills(d, p) : std::vector<int32_t>();
  const std::vector<RowTile> tiles = prefix ? row_tiles(d, p) : std::vector<RowTile>();
  std::vector<Item> rows;
  const Costs cost = schedule_row_items(d, p, tiles, spk::kFwdBM, spk::kFwdBN, include_empty, items,
                                        fills.size() / kItemInts, rows);
  prepend(fills, items);
  const int n_items = (int)(items.size() / kItemInts);
  double us;
  const spk::LaunchShape shape = choose_shape(cost, kSplitFwd, p.D, us);
  if (prefix && !static_ws) {
    const FewPlan few = few_plan(d, p);
    if (few_taken(few, us)) return fwd_few(d, p, few, q, k, v, o, lse, ws, ws_bytes, (hipStream_t)stream);
  }
  if (prefix) {
    const std::vector<int32_t> records =
        place_records(d, p, tiles, shape.split, spk::fwd_tile_keys(p.D, shape.split), items, (int)items.size());
    items.insert(items.end(), records.begin(), records.end());
  }
  hipStream_t st = (hipStream_t)stream;
  void* items_dev = nullptr;
  if (static_ws) {
    if (items.size() * sizeof(int32_t) > SP_STATIC_SCRATCH_BYTES) return SP_ERR_UNSUPPORTED;
    if ((s = refuse_capture(st)) != SP_OK) return s;
    if ((s = stream_on_current_device(st)) != SP_OK) return s;
    if ((s = static_scratch(&items_dev)) != SP_OK) return s;
  } else {
    Layout L = layout_for(d, p, ring ? SP_OP_RING_STEP : SP_OP_FWD,
                          row_item_count(d, p, spk::kFwdBM), 0);
    if ((s = check_ws(L, ws, ws_bytes)) != SP_OK) return s;
    if ((s = refuse_capture(st)) != SP_OK) return s;
    items_dev = at(ws, L.items_dq);
  }
  if (n_items > 0) {
    spk::FwdArgs a{};
    spk::ItemList list{};
    if (items.size() <= std::size(list.v)) {
      std::copy(items.begin(), items.end(), list.v);
    } else {
      if ((s = upload(items_dev, items, st)) != SP_OK) return s;
      a.items = (const int32_t*)items_dev;
    }
    a.q = (const uint16_t*)q;
    a.k = (const uint16_t*)k;
    a.v = (const uint16_t*)v;
    a.o = (uint16_t*)o;
    a.lse = lse;
    a.o_acc = o_acc;
    a.lse_acc = lse_acc;
    a.o_out = (uint16_t*)o_out;
    a.T_q = d->T_q; a.T_k = d->T_k; a.H = d->H_loc; a.Hkv = d->Hkv_loc;
    a.scale_log2 = d->softmax_scale * 1.4426950408889634f;
    a.causal = d->causal;
    a.init = init;
    a.n_items = n_items;
    SP_HIP(spk::launch_attn_fwd(a, list, shape, p.D, ring, prefix, st));
  }
  return SP_OK;
}

sp_status sp_attn_fwd(const sp_attn_desc* desc, const void* q, const void* k, const void* v,
                      void* o, float* lse, void* workspace, size_t workspace_bytes,
                      void* stream) {
  return fwd_common(desc, q, k, v, o, lse, nullptr, nullptr, 1, nullptr, workspace,
                    workspace_bytes, stream, false);
}

sp_status sp_attn_fwd_static(const sp_attn_desc* desc, const void* q, const void* k,
                             const void* v, void* o, float* lse, void* stream) {
  return fwd_common(desc, q, k, v, o, lse, nullptr, nullptr, 1, nullptr, nullptr, 0, stream,
                    false, true);
}

sp_status sp_ring_step(const sp_attn_desc* desc, const void* q, const void* k_chunk,
                       const void* v_chunk, float* o_acc, float* lse_acc, int32_t init,
                       void* o_out, void* workspace, size_t workspace_bytes, void* stream) {
  return fwd_common(desc, q, k_chunk, v_chunk, nullptr, nullptr, o_acc, lse_acc, init, o_out,
                    workspace, workspace_bytes, stream, true);
}

sp_status sp_attn_bwd(const sp_attn_desc* d, const void* q, const void* k, const void* v,
                      const void* o, const float* lse, const void* dout, void* dq,
                      float* dq_acc, void* dk, void* dv, void* ws, size_t ws_bytes,
                      void* stream) {
  Problem p;
  sp_status s = validate(d, p);
  if (s != SP_OK) return s;
  // pointers are required for tensors that have elements
  if (d->T_q > 0 && (!q || !o || !lse || !dout || (!dq && !dq_acc))) return SP_ERR_INVALID_ARG;
  if (d->T_k > 0 && (!k || !v || !dk || !dv)) return SP_ERR_INVALID_ARG;
  for (const void* ptr : {q, k, v, o, dout, (const void*)dk, (const void*)dv})
    if (!aligned16(ptr)) return SP_ERR_INVALID_ARG;
  if ((dq && !aligned16(dq)) || (dq_acc && !aligned16(dq_acc))) return SP_ERR_INVALID_ARG;
  if (d->T_q == 0) {  // no rows: the keys receive no gradient
    SP_HIP(spk::launch_zero_heads_bf16(dk, d->T_k, d->Hkv_loc, p.D, 0, d->Hkv_loc,
                                       (hipStream_t)stream));
    SP_HIP(spk::launch_zero_heads_bf16(dv, d->T_k, d->Hkv_loc, p.D, 0, d->Hkv_loc,
                                       (hipStream_t)stream));
    return SP_OK;
  }
  std::vector<int32_t> it_dq, it_kv;
  // a dq_acc's dummy slots stay untouched
  const std::vector<int32_t> fq = dq ? row_fills(d, p) : std::vector<int32_t>();
  const std::vector<int32_t> fkv = key_fills(d, p);
  const bool prefix = !p.prefix.empty();
  const std::vector<RowTile> tiles = prefix ? row_tiles(d, p) : std::vector<RowTile>();
  std::vector<Item> rows, keys;
  const Costs cost_q =
      schedule_row_items(d, p, tiles, spk::kDqBM, spk::kDqBN, true, it_dq, fq.size() / kItemInts, rows);
  prepend(fq, it_dq);
  const std::vector<spk::KeyCut> cuts = key_cuts(d, p);
  const Costs cost_k =
      schedule_keys(d, p, spk::kDkdvBN, spk::kDkdvBQ, cuts, it_kv, fkv.size() / kItemInts, keys);
  prepend(fkv, it_kv);
  const size_t na = it_dq.size() / kItemInts, nb = it_kv.size() / kItemInts;
  // (the records of row tiles lie behind the dQ items, or in a launch's own list
  // behind all items)
  Layout L = layout_for(d, p, SP_OP_BWD, na + record_room(tiles.size()) / kItemInts, nb, cut_rows(p, cuts));
  if ((s = check_ws(L, ws, ws_bytes)) != SP_OK) return s;
  hipStream_t st = (hipStream_t)stream;
  if ((s = refuse_capture(st)) != SP_OK) return s;
  const int D = p.D;
  const BwdPlan plan = plan_bwd(cost_q, cost_k, D);
  // dK, dV written over K, V: a key's rows are read and written by one dK/dV
  // workgroup, but dQ reads all of them, so it ends first (same splits, same
  // bits)
  const bool over_kv = dk == k || dk == v || dv == k || dv == v;
  // one list where its items are whole (it takes the place of dQ's)
  const bool merged = prefix && plan.one && !over_kv && plan.q.split == 1 && plan.k.split == 1;
  if (merged) {
    it_dq = merged_items(rows, keys, (fq.size() + fkv.size()) / kItemInts);
    prepend(fkv, it_dq);
    prepend(fq, it_dq);
    it_kv.clear();
  }
  const size_t n_rec = tiles.size() * plan.q.split * spk::record_ints(kSlots / plan.q.split);
  const bool by_value = it_dq.size() + it_kv.size() + n_rec <= std::size(spk::ItemList().v);
  const size_t rec_at = by_value ? it_dq.size() + it_kv.size() : it_dq.size();
  std::vector<int32_t> records;
  if (prefix)
    records = place_records(d, p, tiles, plan.q.split, spk::kDqBN, it_dq, (int)rec_at);
  {
    // Work lists that fit a launch's arguments go there (a launch of its own
    // for dK/dV has its list first).  Else both in one copy (they are adjacent
    // in the workspace): every host-to-device copy sits between two kernels on
    // the stream.
    spk::ItemList list{};
    if (by_value) {
      std::copy(records.begin(), records.end(), list.v + rec_at);
    } else {
      const size_t gap = merged ? rec_at + n_rec : (L.items_kv - L.items_dq) / sizeof(int32_t);
      std::vector<int32_t> both(gap + it_kv.size(), 0);
      std::copy(it_dq.begin(), it_dq.end(), both.begin());
      std::copy(records.begin(), records.end(), both.begin() + rec_at);
      std::copy(it_kv.begin(), it_kv.end(), both.begin() + gap);
      if ((s = upload(at(ws, L.items_dq), both, st)) != SP_OK) return s;
    }
    float* neg_d = (float*)at(ws, L.neg_d);
    float* lse2 = (float*)at(ws, L.lse2);
    if (p.n_real > 0 && !(d->flags & SP_DESC_ROWSTATS_READY))
      SP_HIP(spk::launch_rowdot(o, dout, lse, neg_d, lse2, d->T_q, d->H_loc, p.n_real, D, st));
    const float sl2 = d->softmax_scale * 1.4426950408889634f;
    spk::DqArgs a{};
    a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
    a.dout = (const uint16_t*)dout;
    a.lse = lse; a.neg_d = neg_d; a.dq = (uint16_t*)dq; a.dq_acc = dq_acc;
    a.dq_init = dq_acc && (d->flags & SP_DESC_DQ_ACC_INIT) ? 1 : 0;
    a.items = by_value ? nullptr : (const int32_t*)at(ws, L.items_dq);
    a.T_q = d->T_q; a.T_k = d->T_k; a.H = d->H_loc; a.Hkv = d->Hkv_loc;
    a.scale_log2 = sl2; a.scale = d->softmax_scale; a.causal = d->causal;
    a.n_items = (int)(it_dq.size() / kItemInts);

    spk::DkdvArgs b{};
    b.q = (const uint16_t*)q;
    b.dout = (const uint16_t*)dout;
    b.lse2 = lse2; b.neg_d = neg_d; b.k = (const uint16_t*)k; b.v = (const uint16_t*)v;
    b.dk = (uint16_t*)dk; b.dv = (uint16_t*)dv;
    b.part_k = p.direct ? nullptr : (float*)at(ws, L.part_k);
    b.part_v = p.direct ? nullptr : (float*)at(ws, L.part_v);
    b.cut_k = cuts.empty() ? nullptr : (float*)at(ws, L.cut_k);
    b.cut_v = cuts.empty() ? nullptr : (float*)at(ws, L.cut_v);
    b.items = by_value ? nullptr : (const int32_t*)at(ws, L.items_kv);
    b.T_q = d->T_q; b.T_k = d->T_k; b.H = d->H_loc; b.Hkv = d->Hkv_loc;
    b.scale_log2 = sl2; b.scale = d->softmax_scale; b.causal = d->causal; b.direct = p.direct;
    b.n_items = merged ? a.n_items : (int)nb;
    if (merged) b.items = a.items;
    if (by_value) std::copy(it_dq.begin(), it_dq.end(), list.v);
    if (plan.one && !over_kv) {
      if (by_value) std::copy(it_kv.begin(), it_kv.end(), list.v + it_dq.size());
      SP_HIP(spk::launch_attn_bwd(a, b, list, plan.q, plan.k, plan.dq_first, D, prefix, merged, st));
    } else {
      SP_HIP(spk::launch_attn_dq(a, list, plan.q, D, prefix, st));
      if (by_value) std::copy(it_kv.begin(), it_kv.end(), list.v);
      SP_HIP(spk::launch_attn_dkdv(b, list, plan.k, D, st));
    }
    spk::CutArgs c{};
    spk::ReduceArgs& r = c.r;
    r.T = d->T_k; r.Hkv = d->Hkv_loc; r.D = D;
    for (int kv = 0; kv < d->Hkv_loc; ++kv) {
      r.head_lo[kv] = p.kv_lo[kv];
      r.head_hi[kv] = p.kv_hi[kv];
    }
    if (!p.direct && p.n_real > 0) SP_HIP(spk::launch_reduce_kv(b.part_k, b.part_v, dk, dv, r, st));
    if (!cuts.empty()) {
      c.n_real = p.n_real;
      c.n = (int)cuts.size();
      std::copy(cuts.begin(), cuts.end(), c.c);
      SP_HIP(spk::launch_cut_join(b.cut_k, b.cut_v, dk, dv, c, st));
    }
  }
  return SP_OK;
}

sp_status sp_lse_merge(float* o_acc, float* lse_acc, const void* o_part, int32_t o_part_is_bf16,
                       const float* lse_part, int32_t T, int32_t H, int32_t head_dim,
                       void* o_out_bf16, void* stream) {
  if (T < 0 || H < 1 || head_dim < 8 || head_dim > 512 || (head_dim & (head_dim - 1)) != 0)
    return SP_ERR_INVALID_ARG;
  if (o_part_is_bf16 != 0 && o_part_is_bf16 != 1) return SP_ERR_INVALID_ARG;
  if (T == 0) return SP_OK;
  if (!o_acc || !lse_acc || !o_part || !lse_part) return SP_ERR_INVALID_ARG;
  if (!aligned16(o_acc) || !aligned16(o_part) || (o_out_bf16 && !aligned16(o_out_bf16)))
    return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_merge(o_acc, lse_acc, o_part, o_part_is_bf16 != 0, lse_part, T, H, head_dim,
                           o_out_bf16, (hipStream_t)stream));
  return SP_OK;
}

sp_status sp_f32_to_bf16(const float* src, void* dst, int64_t n, void* stream) {
  if (n < 0) return SP_ERR_INVALID_ARG;
  if (n == 0) return SP_OK;
  if (!src || !dst || !aligned16(src) || !aligned16(dst)) return SP_ERR_INVALID_ARG;
  SP_HIP(spk::launch_f32_to_bf16(src, dst, n, (hipStream_t)stream));
  return SP_OK;
}

}  // extern "C"
