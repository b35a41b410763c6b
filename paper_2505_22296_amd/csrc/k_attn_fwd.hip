// Attention forward for one SP rank's real heads on gfx950.
//
// One workgroup = 8 wavefronts = 256 query rows of one head (a work item from
// the host block-skip scheduler; KW = 1, see below for KW > 1); wavefront w
// owns rows q_begin + 32w .. +32.  The key loop walks 64-key tiles of the segment.  K and V tiles are
// copied global -> LDS by DMA into the blocked layout of dev_common.h (no
// padding, no transposed copy: V^T fragments come from transposing LDS
// reads), four tiles resident: while a pair of tiles is consumed the next
// pair lands, and the eight wavefronts meet at a barrier once per pair.  Each
// tile is shared by all eight wavefronts.
//
// Per 64-key tile and wavefront:
//   S^T = K Q^T      (32x32x16 bf16 MFMA; Q^T kept in registers as B operand)
//   online softmax   (fp32; the 32x32 C layout gives each lane one query row,
//                     16 keys per tile half; the row max needs one exchange
//                     with lane l^32)
//   O^T += V^T P^T   (V^T by ds_read_b64_tr_b16 from the V tile; P^T from the
//                     C registers directly: K rows are loaded in perm32 order
//                     so each lane half's C registers are 8 consecutive keys,
//                     i.e. a B operand k-slice)
// The running max is only raised when it grows by more than 2^8 (exact:
// the final normalisation uses the same max).  Masking is evaluated only on
// tiles that straddle a segment edge or the causal diagonal; a wavefront
// skips the arithmetic of tiles that lie wholly past its causal diagonal.
//
// Launches of few items (short sequences, few heads) leave CUs idle and last
// as long as their longest item's serial walk over the keys.  There the host
// splits every item over KW = 2 or 4 workgroups of 256 / KW rows whose
// wavefronts form KW key groups, each walking every KW-th tile; the groups'
// (m, l, O) meet in LDS at the end.  The walk is KW times shorter and KW times
// as many CUs work; each staged tile serves KW times fewer rows, which is why
// a full chip keeps KW = 1.  Measured, 4 heads on one causal sequence, D = 128,
// KW = 1 / 2 / 4: 1024 rows 29.7 / 23.2 / 18.1 us, 4096 rows 92.2 / 59.3 /
// 43.0 us, 16384 rows 381 / 293 / 362 us; 28 heads of 4096 rows 122 / 150 /
// 193 us.
//
// The ring variant (MERGE) folds the chunk's normalised (O_c, LSE_c) into
// float32 accumulators with the log-sum-exp rule in the epilogue.
#include "dev_common.h"
#include "launch.h"

namespace spk {

namespace {

constexpr int NW = kFwdWaves;         // wavefronts per workgroup
constexpr int NT = 64 * NW;
constexpr int kJoinThreads = 256;  // of a row's merge
static_assert(kMaxParts <= kJoinThreads, "a part's weight a thread");
static_assert(kFwdBM == 32 * NW, "fwd tiling");

// LDS stage of the forward: for each of the KW key groups a K and a V tile
// [BN][D] in the blocked layout (D/32 sub-tiles [BN][32]), filled by DMA in
// 1 KB blocks by the RW wavefronts of the group.
template <int D, int KW>
struct FwdStage {
  static constexpr int RW = NW / KW;           // row groups of 32 rows
  static constexpr int BN = fwd_tile_keys(D, KW);  // keys per tile
  static constexpr int NST = KW == 1 ? kFwdStages : 2;         // resident stages
  static constexpr int TPB = KW == 1 ? kFwdTilesPerSync : 1;   // stages per barrier
  static_assert(NST % TPB == 0 && NST >= 2 * TPB, "fwd pipeline");
  static constexpr int SUB = BN * 4;           // chunks per sub-tile
  static constexpr int KB = BN * (D / 8) / 64; // 1 KB blocks per tile
  static constexpr int NBK = KB / RW;          // blocks per wavefront and tile
  static_assert(KB % RW == 0, "DMA blocks per wavefront");
  static constexpr int OFF_V = KB * 64, TILE = 2 * KB * 64;  // 16-byte chunks
  static constexpr int STAGE = KW * TILE;
  // partial results of the key groups, exchanged through the same LDS: O^T of
  // every wavefront (quad i of 4 dims: 64 lanes x 16 bytes), then (m, l)
  static constexpr int NQ = D / 8, OFF_ML = NW * NQ * 64;
  static constexpr int XCH = KW > 1 ? OFF_ML + NW * 32 : 0;
  static constexpr int SMEM = NST * STAGE > XCH ? NST * STAGE : XCH;
};

// KW key groups of RW = 8 / KW wavefronts: row group w % RW owns 32 query
// rows, key group w / RW the tiles n * KW + w / RW.  An item's rows are split
// over KW workgroups (of 256 / KW rows each), all on the item's XCD, one
// after the other, the last rows (the longest under a causal mask) first.
// TWO: at most 128 VGPRs, so that two workgroups share a CU.
// PFX: segments share prefixes; the items name records of slots and key ranges
// (dev_common.h), the workgroup's rows come from several segments.
// FEW (with PFX, KW = 4): a call of few rows, whose items would leave most CUs idle
// behind long walks.  The list holds tiles of two slots (FewTile) and the rows'
// windows; workgroup b takes one part of one tile's key tiles, eight parts at a time
// so that a part's tiles, which share keys, are on one XCD (b % 8).  A slot holds 32 /
// g rows for each of the g query heads that share a KV head (lane i: row i / g, head
// i % g; a token an answer then still fills a slot), of any segments of one prefix, so
// that the own keys are a window per lane; the part's normalised result goes to
// float32 buffers that attn_join_kernel merges.
typedef const __attribute__((address_space(4))) int32_t* TablePtr;
template <int D, bool MERGE, int KW, bool TWO, bool PFX, bool FEW = false>
__global__ __launch_bounds__(NT, TWO ? 4 : 1) void attn_fwd_kernel(FwdArgs a, ItemList list) {
  using S = FwdStage<D, KW>;
  constexpr int RW = S::RW, BN = S::BN, NST = S::NST, TPB = S::TPB;
  constexpr int KS = D / 16;   // MFMA k-steps over D
  constexpr int DB = D / 32;   // 32-dim blocks of O^T
  constexpr int G = BN / 32;   // 32-key halves of a tile
  constexpr int NBK = S::NBK, NBW = 2 * NBK, STAGE = S::STAGE, SUB = S::SUB;

  __shared__ u32x4 smem[S::SMEM];

  static_assert(sizeof(FwdArgs) % alignof(ItemList) == 0, "the list follows the arguments");
  const TablePtr table = (TablePtr)__builtin_amdgcn_kernarg_segment_ptr() + sizeof(FwdArgs) / 4;  // FEW
  int pos, sub = 0, part = 0;
  if constexpr (FEW) {
    // (divisions happen in vector registers: back to scalar ones)
    const int first = __builtin_amdgcn_readfirstlane(blockIdx.x / (8 * a.n_items) * 8);
    const int width = min(8, a.parts - first), in = blockIdx.x - first * a.n_items;
    pos = __builtin_amdgcn_readfirstlane(in / width);
    part = first + in - pos * width;
  } else {
    if (!split_pos<KW>(blockIdx.x, a.n_items, pos, sub)) return;
  }
  int32_t it[kItemInts];
  if constexpr (FEW) {
#pragma unroll
    for (int j = 0; j < kItemInts; ++j) it[j] = __builtin_amdgcn_readfirstlane(table[pos * kItemInts + j]);
  } else {
    load_item(a.items, list, 0, pos, it);
  }
  static_assert(!PFX || !MERGE, "a ring step has no shared prefixes");
  static_assert(!FEW || (PFX && KW == 4), "few rows");
  int q0 = it[0], q1 = it[1], k1 = it[3];
  int k0 = it[2], delta = it[4];
  const int head = FEW ? it[6] & 0xffff : it[5], kvh = FEW ? it[7] : it[6];
  const int tid = threadIdx.x;
  if constexpr (KW > 1 && !FEW) {
    if (!PFX || it[7] == kItemFillQ)
      if (!split_rows<KW>(it[7] == kItemFillQ, 32 * RW, sub, q0, q1)) return;
    if (!PFX && a.causal) k1 = max(k0, min(k1, q1 + delta));
  }
  if (!FEW && it[7] == kItemFillQ) {
    // dummy slot: O = +0, LSE = -inf (ring: the accumulators' identity on the
    // first chunk, and +0 in the bf16 copy)
    if constexpr (!MERGE) {
      fill_rows_bf16(a.o, q0, q1, a.H, head, D, tid, NT);
      fill_span_f32(a.lse + (int64_t)head * a.T_q + q0, q1 - q0, neg_inf(), tid, NT);
    } else {
      if (a.init) {
        fill_rows_f32(a.o_acc, q0, q1, a.H, head, D, tid, NT);
        fill_span_f32(a.lse_acc + (int64_t)head * a.T_q + q0, q1 - q0, neg_inf(), tid, NT);
      }
      if (a.o_out) fill_rows_bf16(a.o_out, q0, q1, a.H, head, D, tid, NT);
    }
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, hh = lane >> 5, l32 = lane & 31;
  const int rg = KW > 1 ? w % RW : w, kg = KW > 1 ? w / RW : 0;
  const int record = it[0] + sub * record_ints(RW);  // PFX, not FEW
  int pk0 = 0;
  bool has_prefix = false;
  const int g = FEW ? it[6] >> 16 : 1;  // query heads in a slot
  // FEW: key tiles of the prefix and of all, the first of the part
  int pk1 = 0, n_pre = 0, v0 = 0, n_keytiles = 0;
  if constexpr (FEW) {
    pk0 = it[2];
    pk1 = it[3];
    k0 = it[4];
    k1 = it[5];
    n_pre = few_steps(pk0, pk1, BN);
    const int all = n_pre + few_steps(k0, k1, BN);
    const int each = __builtin_amdgcn_readfirstlane(all / a.parts), more = all - each * a.parts;
    v0 = part * each + min(part, more);
    n_keytiles = each + (part < more);
    const int rows = __builtin_amdgcn_readfirstlane(32 / g);
    q0 = it[0] + rg * rows;
    q1 = min(it[1], q0 + rows);
    if (q0 >= q1) q0 = q1 = it[0];  // (a row that exists, for addresses)
  } else if constexpr (PFX) {
    const RowSlot slot = load_slot(a.items, list, record, RW, rg);
    q0 = slot.row0;
    q1 = slot.row1;
    k0 = slot.k0;
    k1 = slot.k1;
    delta = slot.delta;
    pk0 = table_at(a.items, list, record + 1);
    has_prefix = table_at(a.items, list, record + 2) != 0;
  }
  const int wr0 = PFX ? q0 : q0 + rg * 32;  // the wavefront's first row
  const int row = wr0 + (FEW ? l32 / g : l32);
  const bool row_ok = row < q1;
  const int qhead = FEW ? head + l32 % g : head;
  int own0 = 0, own1 = 0;  // FEW: the row's window of its own segment's keys
  if constexpr (FEW) {
    const TablePtr win = table + a.n_items * kItemInts + 2 * (row_ok ? row : q0);
    own0 = win[0];
    own1 = win[1];
  }
  // last key any row of this wavefront may see (tiles past it are skipped; PFX:
  // of its own segment)
  const int wave_rows = min(32, q1 - wr0);
  const int wave_kmax = wave_rows <= 0 ? -1 : a.causal && !FEW ? min(k1, wr0 + wave_rows + delta) : k1;

  // Q^T as B operand: lane holds query row `row`, dims ks*16 + hh*8 + [0..7].
  u32x4 qf[KS];
  {
    const uint16_t* qp = a.q + ((int64_t)(row_ok ? row : q0) * a.H + (row_ok ? qhead : head)) * D + hh * 8;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qf[s] = *(const u32x4*)(qp + s * 16);
      if (!row_ok) qf[s] = u32x4{0u, 0u, 0u, 0u};
    }
  }

  f32x16 oacc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[d][r] = 0.f;
  float m_run = neg_inf(), l_part = 0.f;
  const float c2 = a.scale_log2;
  // Carried with the running max (they change only when it is raised):
  // msc = m_run * c2 (0 while m_run is -inf), and the score above which the
  // max is raised, m_run + 8 / c2 (-inf while m_run is -inf)
  const float raise_by = 8.f / c2;
  float msc = 0.f, m_thr = neg_inf();

  const int kt_first = k0 & ~7;
  // stages of KW tiles (PFX: of the record's key tiles)
  if constexpr (PFX && !FEW) n_keytiles = table_at(a.items, list, record);
  const int n_tiles = PFX ? (n_keytiles + KW - 1) / KW : (k1 > k0) ? (k1 - kt_first + BN * KW - 1) / (BN * KW) : 0;
  KeyWalk walk_in, walk;  // of the copies and of the tiles in use

  // Per-lane, tile-independent element offsets of this wavefront's DMA
  // blocks rg + RW*j: the first NBK of them in the K tile, the rest in V;
  // both tiles have the same shape and source row stride.
  const int kstride = a.Hkv * D;
  int off[NBK], key_of[NBK];
#pragma unroll
  for (int j = 0; j < NBK; ++j) {
    const int t = (rg + RW * j) * 64 + lane;   // chunk slot within the tile
    const int ts = t % S::SUB, r = ts / 4;
    key_of[j] = r;
    off[j] = 2 * (r * kstride + (t / S::SUB) * 32 + blk_chunk(r, ts % 4) * 8);  // bytes
  }
  const uint16_t* kbase = a.k + (int64_t)kvh * D;
  const uint16_t* vbase = a.v + (int64_t)kvh * D;
  const int kend = k1;
  // FEW: the part's first key tile, and what changes behind the prefix
  const int few_kt = (pk0 & ~7) + v0 * BN, few_skip = (k0 & ~7) - (pk0 & ~7) - n_pre * BN, few_end = kend - pk1;
  auto issue = [&](int n) {
    int kt = kt_first + (n * KW + kg) * BN, k1 = kend;
    if constexpr (PFX) {
      const int v = n * KW + kg;
      if (KW > 1 && v >= n_keytiles) return;
      if constexpr (FEW) {
        // (selected by arithmetic: as ?: the compiler selects between captured
        // addresses and keeps the values in scratch memory)
        const int behind = v0 + v < n_pre ? 0 : -1;
        kt = few_kt + v * BN + (behind & few_skip);
        k1 = pk1 + (behind & few_end);
      } else {
        walk_in.seek(a.items, list, record, v);
        kt = walk_in.kt0 + (v - walk_in.v0) * BN;
        k1 = walk_in.k1;
      }
    }
    if (KW > 1 && kt >= k1) return;  // the key group has no tile in the last stage
    u32x4* stg = smem + (n % NST) * STAGE + kg * S::TILE + rg * 64;
    const int64_t rowoff = (int64_t)kt * kstride;
    if (kt + BN <= k1) {
#pragma unroll
      for (int j = 0; j < NBK; ++j) {
        dma16s(kbase + rowoff, off[j], stg + RW * j * 64);
        dma16s(vbase + rowoff, off[j], stg + S::OFF_V + RW * j * 64);
      }
    } else {  // keys past k1 (masked) are clamped to k1-1
#pragma unroll
      for (int j = 0; j < NBK; ++j) {
        const int o = off[j] + 2 * (min(kt + key_of[j], k1 - 1) - kt - key_of[j]) * kstride;
        dma16s(kbase + rowoff, o, stg + RW * j * 64);
        dma16s(vbase + rowoff, o, stg + S::OFF_V + RW * j * 64);
      }
    }
  };
  // Lane-constant LDS offsets of the fragments.  K fragment (g, ks): tile row
  // g*32 + perm32(l32), logical chunk 2ks + hh -> sub-tile ks/2 (immediate)
  // and one of two lane bases (ks even / odd).  V^T fragments: transposing
  // reads at two lane offsets; dim block, k-step and stage are immediates.
  const int kr = perm32(l32);
  const int kf0 = kr * 4 + blk_chunk(kr, hh), kf1 = kr * 4 + blk_chunk(kr, 2 + hh);
  const int vt0 = S::OFF_V * 8 + blk_tr_off(lane), vt1 = S::OFF_V * 8 + blk_tr_off2(lane);

  for (int n = 0; n < NST - TPB && n < n_tiles; ++n) issue(n);

  for (int n0 = 0; n0 < n_tiles; n0 += NST) {
#pragma unroll
    for (int u = 0; u < NST; ++u) {
      const int n = n0 + u;
      if (n >= n_tiles) break;
      if (u % TPB == 0) {
        // stages n .. n+TPB-1 landed; every wavefront is done with the
        // memory of stages n-TPB .. n-1, which receives n+NST-TPB ..
        const int issued = min(n_tiles, n + NST - TPB);
        wait_batches<NBW, NST - 2 * TPB>(issued - min(n_tiles, n + TPB));
        __syncthreads();
        // KW = 4: a stage is consumed in one step, about as long as a copy
        // takes to land, so the next stage's copies go first
        if constexpr (KW == 4)
          if (n + 1 < n_tiles) issue(n + 1);
      }
      // stage n + NST - TPB was freed at the last barrier; its copy is issued
      // after this tile's first MFMAs (spreads the DMA burst)
      const bool pf = KW < 4 && n + NST - TPB < n_tiles;
      int kt = kt_first + (n * KW + kg) * BN;
      // what the wavefront sees of the tile: keys [m0, m1), under the causal rule if
      // `causal`, none of them where kt >= kmax
      int m0 = k0, m1 = k1, causal = FEW ? 0 : a.causal, kmax = wave_kmax;
      int own = FEW;
      if constexpr (PFX) {
        const int v = n * KW + kg;
        bool live = KW == 1 || v < n_keytiles;
        bool in_prefix;  // visible to every row
        if constexpr (FEW) {
          in_prefix = v0 + v < n_pre;
          kt = few_kt + v * BN + (in_prefix ? 0 : few_skip);
        } else {
          if (live) walk.seek(a.items, list, record, v);
          kt = walk.kt0 + (v - walk.v0) * BN;
          in_prefix = has_prefix & (walk.range == 0);
        }
        if (in_prefix) {
          m0 = pk0;
          m1 = FEW ? pk1 : walk.k1;
          causal = own = 0;
          kmax = wave_rows > 0 ? m1 : -1;
        }
        live &= kt + BN > m0;
        // The values are made opaque: the compiler otherwise keeps a path for tiles
        // of the prefix beside the one for own keys, moves the accumulators from one
        // to the other and spills (D = 128: 34 registers; 64 answers of 256 rows to
        // 16384 keys, 4 heads, 702 instead of 502 us)
        m0 = __builtin_amdgcn_readfirstlane(m0);
        m1 = __builtin_amdgcn_readfirstlane(m1);
        causal = __builtin_amdgcn_readfirstlane(causal);
        own = __builtin_amdgcn_readfirstlane(own);
        kmax = __builtin_amdgcn_readfirstlane(live ? kmax : 0);
        kt = __builtin_amdgcn_readfirstlane(kt);
      }
      if (kt >= kmax) {  // nothing of it for this wavefront's rows
        if (pf) issue(n + NST - TPB);
        continue;
      }
      const u32x4* stg = smem + u * STAGE + kg * S::TILE;

      // ---- S^T = K Q^T for the 32-key halves of the tile.  The K
      // fragment reads are issued together ahead of the MFMAs; the compiler
      // places the MFMAs among them (measured faster than holding every
      // MFMA behind the last read).
      u32x4 kfr[G * KS];
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          kfr[g * KS + ks] = stg[(ks >> 1) * SUB + g * 128 + ((ks & 1) ? kf1 : kf0)];
      f32x16 s[G];
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[g][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int g = 0; g < G; ++g) s[g] = mfma32(kfr[g * KS + ks], qf[ks], s[g]);
      // V^T fragments of this tile, read while the softmax runs (TWO: after it,
      // for the 128 registers)
      const uint16_t* stg16 = (const uint16_t*)stg;
      u32x4 vfr[DB * 2 * G];
      auto read_v = [&](int ks0, int ks1) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int ks = ks0; ks < ks1; ++ks) {
            const int o = d * SUB * 8 + ks * 16 * 32;
            const u32x2 lo = lds_tr16(stg16 + vt0 + o), hi = lds_tr16(stg16 + vt1 + o);
            vfr[d * 2 * G + ks] = u32x4{lo[0], lo[1], hi[0], hi[1]};
          }
      };
      if constexpr (!TWO) {
        read_v(0, 2 * G);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (pf) issue(n + NST - TPB);

      // ---- mask (only on edge / diagonal tiles)
      const bool need_mask = (kt < m0) | (kt + BN > m1) | (causal & (kt + BN - 1 > wr0 + delta)) | (FEW && own);
      if (need_mask) {
        // keys [lo, hi) of the lane half's, counted from kt + 8 hh
        const int lo = (FEW && own ? own0 : m0) - kt - hh * 8;
        const int hi = (FEW && own ? own1 : causal ? min(m1, row + delta + 1) : m1) - kt - hh * 8;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = g * 32 + c_row_of(r, 0);
            if (key < lo || key >= hi) s[g][r] = neg_inf();
          }
      }

      // ---- online softmax (lazy rescale).  Row max of the lane's 32
      // scores (finite or -inf): four chains of three-input maxima, 18 VALU
      // operations (a wavefront's dependent VALU operations issue back to
      // back, so short chains buy nothing)
      float mx4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mx4[i] = max3_nonan(s[0][i], s[0][i + 4], s[0][i + 8]);
        if constexpr (G == 2) {
          mx4[i] = max3_nonan(mx4[i], s[0][i + 12], s[1][i]);
          mx4[i] = max3_nonan(mx4[i], s[1][i + 4], s[1][i + 8]);
        }
        mx4[i] = max3_nonan(mx4[i], s[G - 1][i + 12], s[G - 1][i + 12]);
      }
      const float mx = wave_max_xor32(max3_nonan(max3_nonan(mx4[0], mx4[1], mx4[2]), mx4[3], mx4[3]));
      const bool need = mx > m_thr;  // false while every score is -inf
      if (__ballot(need)) {
        float alpha = need ? exp2f((m_run - mx) * c2) : 1.f;
        if (need) {
          m_run = mx;
          msc = mx * c2;
          m_thr = mx + raise_by;
        }
        l_part *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[d][r] *= alpha;
      }
      u32x4 pb[2 * G];
      float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][r], c2, -msc));
          ps[r & 3] += p[r];
        }
        pb[2 * g] = pack_bf16x8(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]);
        pb[2 * g + 1] = pack_bf16x8(p[8], p[9], p[10], p[11], p[12], p[13], p[14], p[15]);
      }
      l_part += (ps[0] + ps[1]) + (ps[2] + ps[3]);

      // ---- O^T += V^T P^T
      if constexpr (TWO) {
        __builtin_amdgcn_sched_barrier(0);
        read_v(0, 2 * G);
      }
#pragma unroll
      for (int ks = 0; ks < 2 * G; ++ks)
#pragma unroll
        for (int d = 0; d < DB; ++d) oacc[d] = mfma32(vfr[d * 2 * G + ks], pb[ks], oacc[d]);
    }
  }

  // ---- epilogue: quad i of the row (4 dims at (i >> 2) * 32 + (i & 3) * 8
  // + hh * 4); the key groups share out the quads of a row
  constexpr int NQW = S::NQ / KW;
  float l_tot = wave_sum_xor32(l_part);
  float la = neg_inf();  // ring: the row's accumulated LSE
  float acc[NQW][4];
  if constexpr (KW == 1) {
#pragma unroll
    for (int i = 0; i < NQW; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[i][x] = oacc[i >> 2][(i & 3) * 4 + x];
  } else {
    // the groups' partial results meet in LDS (every copy has landed: the
    // last stage's barrier waited for it) and are summed in group order
    __syncthreads();
    f32x4* xo = (f32x4*)smem;
    f32x2* xml = (f32x2*)(smem + S::OFF_ML);
#pragma unroll
    for (int i = 0; i < S::NQ; ++i)
      xo[(w * S::NQ + i) * 64 + lane] = f32x4{oacc[i >> 2][(i & 3) * 4], oacc[i >> 2][(i & 3) * 4 + 1],
                                              oacc[i >> 2][(i & 3) * 4 + 2], oacc[i >> 2][(i & 3) * 4 + 3]};
    xml[w * 64 + lane] = f32x2{m_run, l_tot};
    if constexpr (MERGE) {
      // every group reads it before one of them writes it below: the value
      // has arrived (the empty asm consumes it) when the barrier is reached
      if (!a.init) la = a.lse_acc[(int64_t)head * a.T_q + (row_ok ? row : q0)];
      asm volatile("" : "+v"(la) : : "memory");
    }
    __syncthreads();
    f32x2 ml[KW];
#pragma unroll
    for (int p = 0; p < KW; ++p) ml[p] = xml[(rg + RW * p) * 64 + lane];
    m_run = ml[0][0];
#pragma unroll
    for (int p = 1; p < KW; ++p) m_run = fmaxf(m_run, ml[p][0]);
    l_tot = 0.f;
#pragma unroll
    for (int i = 0; i < NQW; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[i][x] = 0.f;
#pragma unroll
    for (int p = 0; p < KW; ++p) {
      // a group that saw no key of the row weighs nothing
      const float wt = ml[p][0] == neg_inf() ? 0.f : exp2f((ml[p][0] - m_run) * c2);
      l_tot += wt * ml[p][1];
#pragma unroll
      for (int i = 0; i < NQW; ++i) {
        const f32x4 o = xo[((rg + RW * p) * S::NQ + kg * NQW + i) * 64 + lane];
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[i][x] += wt * o[x];
      }
    }
  }
  const bool has = l_tot > 0.f;
  const float inv = has ? 1.f / l_tot : 0.f;
  const float lse_v = has ? (m_run * c2 + __log2f(l_tot)) * kLn2 : neg_inf();
  if (!row_ok) return;
  const int64_t obase = ((int64_t)row * a.H + qhead) * D + hh * 4;
  // element offset of the wavefront's quad i
  auto dim = [&](int i) { return ((kg * NQW + i) >> 2) * 32 + ((kg * NQW + i) & 3) * 8; };
  if constexpr (FEW) {
    float* o = a.o_acc + (int64_t)part * a.T_q * a.H * D + obase;
#pragma unroll
    for (int i = 0; i < NQW; ++i)
      *(float4*)(o + dim(i)) = make_float4(acc[i][0] * inv, acc[i][1] * inv, acc[i][2] * inv, acc[i][3] * inv);
    if (hh == 0 && kg == 0) a.lse_acc[((int64_t)part * a.H + qhead) * a.T_q + row] = lse_v;
  } else if constexpr (!MERGE) {
#pragma unroll
    for (int i = 0; i < NQW; ++i)
      *(u32x2*)(a.o + obase + dim(i)) =
          pack_bf16x4(acc[i][0] * inv, acc[i][1] * inv, acc[i][2] * inv, acc[i][3] * inv);
    if (hh == 0 && kg == 0) a.lse[(int64_t)head * a.T_q + row] = lse_v;
  } else {
    // every accumulator value is loaded before the first store (the stores
    // could alias later loads for all the compiler knows, which would
    // serialize one memory round trip per 16 bytes), together with the
    // accumulated LSE
    float4 old[NQW];
#pragma unroll
    for (int i = 0; i < NQW; ++i)
      old[i] = a.init ? make_float4(0.f, 0.f, 0.f, 0.f) : *(const float4*)(a.o_acc + obase + dim(i));
    const int64_t li = (int64_t)head * a.T_q + row;
    if constexpr (KW == 1)
      if (!a.init) la = a.lse_acc[li];
    float wa = 0.f, wb = 0.f, L = neg_inf();
    const float m = fmaxf(la, lse_v);
    if (m != neg_inf()) {
      float ea = __expf(la - m), eb = __expf(lse_v - m);
      float ssum = ea + eb;
      L = m + __logf(ssum);
      wa = ea / ssum;
      wb = eb / ssum * inv;  // folds the chunk's 1/l normalisation
    }
#pragma unroll
    for (int i = 0; i < NQW; ++i) {
      const float4 o = old[i];
      float4 nv = make_float4(wa * o.x + wb * acc[i][0], wa * o.y + wb * acc[i][1],
                              wa * o.z + wb * acc[i][2], wa * o.w + wb * acc[i][3]);
      *(float4*)(a.o_acc + obase + dim(i)) = nv;
      if (a.o_out) *(u32x2*)(a.o_out + obase + dim(i)) = pack_bf16x4(nv.x, nv.y, nv.z, nv.w);
    }
    if (hh == 0 && kg == 0) a.lse_acc[li] = L;
  }
}

// Merge of the parts of a call of few rows, one workgroup for each row and head:
// O = sum_p w_p O_p with w_p = e^(L_p - L), L = log sum_p e^(L_p).  Dummy slots, and
// rows that no part sees a key of, get O = +0, LSE = -inf.  The parts are read D / 4
// lanes wide, as many at a time as the threads hold, and summed in a fixed order.
template <int D>
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(FwdArgs a, int n_real) {
  const int parts = a.parts;
  constexpr int L = D / 4, G = kJoinThreads / L;
  __shared__ float wt[kMaxParts];
  __shared__ float4 red[G][L];
  const int row = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, l = tid % L, g = tid / L;
  const bool real = head < n_real;
  float m = neg_inf();
  float mine = neg_inf();
  if (real && tid < parts) mine = a.lse_acc[((int64_t)tid * a.H + head) * a.T_q + row];
  __shared__ float wm[kJoinThreads / 64], ws[kJoinThreads / 64];
  m = mine;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  if ((tid & 63) == 0) wm[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kJoinThreads / 64; ++i) m = fmaxf(m, wm[i]);
  const float e = mine == neg_inf() ? 0.f : __expf(mine - m);
  float s = e;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
  if ((tid & 63) == 0) ws[tid >> 6] = s;
  if (tid < kMaxParts) wt[tid] = e;
  __syncthreads();
  s = 0.f;
#pragma unroll
  for (int i = 0; i < kJoinThreads / 64; ++i) s += ws[i];
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (s > 0.f) {
    const float* o = a.o_acc + ((int64_t)row * a.H + head) * D + l * 4;
    const int64_t stride = (int64_t)a.T_q * a.H * D;
#pragma unroll 8
    for (int p = g; p < parts; p += G) {
      const float4 v = *(const float4*)(o + p * stride);
      const float w = wt[p];
      x.x += w * v.x; x.y += w * v.y; x.z += w * v.z; x.w += w * v.w;
    }
  }
  red[g][l] = x;
  __syncthreads();
  if (g == 0) {
#pragma unroll
    for (int i = 1; i < G; ++i) {
      const float4 v = red[i][l];
      x.x += v.x; x.y += v.y; x.z += v.z; x.w += v.w;
    }
    const float inv = s > 0.f ? 1.f / s : 0.f;
    *(u32x2*)(a.o + ((int64_t)row * a.H + head) * D + l * 4) = pack_bf16x4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    if (l == 0) a.lse[(int64_t)head * a.T_q + row] = s > 0.f ? m + __logf(s) : neg_inf();
  }
}

}  // namespace

hipError_t launch_attn_few(const FwdArgs& a, const ItemList& list, int D, int n_real, hipStream_t st) {
  const dim3 parts(a.n_items * a.parts), rows(a.T_q, a.H);
  const hipError_t e =
      D == 128 ? sp_launch(kKFwd, attn_fwd_kernel<128, false, 4, false, true, true>, parts, dim3(NT), st, a, list)
               : sp_launch(kKFwd, attn_fwd_kernel<64, false, 4, false, true, true>, parts, dim3(NT), st, a, list);
  if (e != hipSuccess) return e;
  return D == 128 ? sp_launch(0, attn_join_kernel<128>, rows, dim3(kJoinThreads), st, a, n_real)
                  : sp_launch(0, attn_join_kernel<64>, rows, dim3(kJoinThreads), st, a, n_real);
}

template <int D, int KW, bool TWO>
static hipError_t launch_fwd(const FwdArgs& a, const ItemList& list, bool merge, bool prefix, hipStream_t st) {
  const dim3 grid(split_grid(a.n_items, KW)), block(NT);
  return merge    ? sp_launch(kKFwd, attn_fwd_kernel<D, true, KW, TWO, false>, grid, block, st, a, list)
         : prefix ? sp_launch(kKFwd, attn_fwd_kernel<D, false, KW, TWO, true>, grid, block, st, a, list)
                  : sp_launch(kKFwd, attn_fwd_kernel<D, false, KW, TWO, false>, grid, block, st, a, list);
}

hipError_t launch_attn_fwd(const FwdArgs& a, const ItemList& list, LaunchShape s, int D, bool merge, bool prefix,
                           hipStream_t st) {
  if (a.n_items <= 0) return hipSuccess;
  if (merge && prefix) return hipErrorInvalidValue;
  if (D == 128) {
    if (s.split == 4) return launch_fwd<128, 4, false>(a, list, merge, prefix, st);
    if (s.split == 2) return launch_fwd<128, 2, false>(a, list, merge, prefix, st);
    return launch_fwd<128, 1, false>(a, list, merge, prefix, st);
  }
  if (s.split == 4) return launch_fwd<64, 4, false>(a, list, merge, prefix, st);
  if (s.split == 2)
    return s.two ? launch_fwd<64, 2, true>(a, list, merge, prefix, st)
                 : launch_fwd<64, 2, false>(a, list, merge, prefix, st);
  if (s.two) return launch_fwd<64, 1, true>(a, list, merge, prefix, st);
  return launch_fwd<64, 1, false>(a, list, merge, prefix, st);
}

}  // namespace spk
