// Linear attention with a decay for each key/value head over a shared prefix:
//   o_t = c sum_{s <= t} l^(t-s) (q_t . k_s) v_s   over the keys that a row sees in the grouped layout,
// as a recurrence S_t = l S_{t-1} + k_t v_t^T, o_t = c S_t^T q_t with a D x D state for each kv head. A member's
// state starts from the one its group's prefix ends with, so the prefix is walked once for all members.
//
// Chunked form. Rows are taken kC at a time; with S the state before a chunk, row i of it is
//   o_i = c (l^(i+1) S^T q_i + sum_{j <= i} l^(i-j) (q_i . k_j) v_j),     S' = l^n S + sum_j l^(n-1-j) k_j v_j^T,
// three matrix products and a masked one on the matrix cores. A workgroup carries S in fp32 registers through an
// *item*, at most L rows of one segment (a prefix or a member), and keeps a copy of it in the tensors' type in LDS as
// an operand. Items run side by side, so the states between them come first: state kernel (each item's own share),
// scan kernels (prefixes, then members, in item order), then the kernel that writes the outputs. A member of one item
// needs no share: it starts from the prefix's state. All of it is bound by memory (a row of a query head is 4 D
// elements read and written for 4 D^2 multiply-adds and its share of a state update), small calls by launches.
//
// Gradients: dq is the same walk with do in the place of q, v of k and k of v. dk and dv walk each segment backwards
// with R_s = l R_{s+1} + sum_heads q_s do_s^T, members first; a prefix starts from the sum of its members' states, in
// member order (the sum over the G copies of the prefix that Lemma 1 of the shared-prefix attention has too).
//
// Every power of the decay that is formed has an exponent >= 0, so none overflows however strong the decay is.
//
// Rounding (bf16 calls): the decayed scores and the state are rounded to bf16 as operands (relative 2^-8 at most, of
// the same size as the output's own rounding); the decayed rows of a state update are split into two bf16 parts
// (2^-16), three where the states themselves are returned (2^-24), because a state sums over all earlier rows.
#pragma once
#include "pg_common.hpp"
#include "pg_plan.hpp"

namespace pg {

// rows [row0, row0 + nrows) of a prefix (part 0) or of a member's response (part 1); seg: the group or member.
// prev: slot of the state before it, kNoState, or kInitState (the group's initial state); self: its own slot.
struct LinItem {
  int row0, nrows, part, seg, prev, last, group, self;
};
constexpr int kNoState = -1, kInitState = -2;

struct LinArgs {
  const void *q[2], *k[2], *v[2], *d_o[2];  // prefix, responses
  void *out[2];                             // o, or dq
  void *dk[2], *dv[2];
  const float* log_decay;
  const float* state_in;  // [n_groups, h_kv, D, D] or NULL
  float* state_out[2];    // [n_groups or n_suffixes, h_kv, D, D] or NULL
  float* slots;           // [max_items + n_groups, h_kv, D, D]
  const int* seg_off;     // first item of each prefix, then of each member
  const LinItem* items;
  const int* n_items;     // 0 when the grouping arrays are inconsistent
  const int *cu_p, *cu_s;
  const PlanHeader* hdr;
  const GroupInfoEx* ginfo;
  int ng, ns, h_q, h_kv, max_items;
  int l_pre, l_suf;   // rows of a prefix's and of a member's items
  int alone;          // no states between items: a workgroup walks what its own starts from
  int members_first;  // backward: the members' gradients are done before the prefixes' walk starts
  float scale;
};

// Powers of a head's decay: l^n = 2^(g n), g clamped so that no product with n = 0 is a NaN and a decay of zero
// (a log of -inf) gives l^0 = 1, l^n = 0.
__device__ __forceinline__ float log2_decay(const float* log_decay, int h) {
  return fmaxf(log_decay[h] * kLog2e, -1e5f);
}

// ---------------------------------------------------------------- items
// One walk's items: where they go and how many rows they hold.
struct LinList {
  int* seg_off;     // [n_groups + n_suffixes + 1]
  LinItem* items;   // [max_items]
  int* n_items;
  int l_pre, l_suf, max_items, reverse;
  int round;  // workgroups' places: see item_place; 0: items in order
};

// Place in the launch of the item of rank r by length (0 the longest) among n. Items that are whole members differ in
// length, and two workgroups share a CU: the `round` longest go first, one to a CU, the next `round` in the opposite
// order, the shortest beside the longest, what is left longest first (64 members of 128..2048 rows: the output kernel
// 584 -> 521 us, dk and dv 679 -> 585).
__device__ __forceinline__ int item_place(int r, int n, int round) {
  return r < round || r >= 2 * round ? r : min(2 * round, n) - 1 - (r - round);
}

// One block: item offsets of all segments (prefixes, then members), then the items themselves. `off`: seg_off, or a
// copy of it in LDS (then both are written).
__device__ __forceinline__ void lin_items(const LinList& L, const int* cu_p, const int* cu_s, const GroupInfoEx* ginfo,
                                          int ng, int ns, int* off, int* tmp, int& carry, int* work) {
  const int t = threadIdx.x, segs = ng + ns;
  auto count = [&](int s) {
    if (s >= segs) return 0;
    return s < ng ? ceil_div(cu_p[s + 1] - cu_p[s], L.l_pre) : ceil_div(cu_s[s - ng + 1] - cu_s[s - ng], L.l_suf);
  };
  __syncthreads();
  if (t == 0) carry = 0;
  __syncthreads();
  if (segs < kPlanThreads) {  // one segment a thread: wave scans, two barriers
    int n[1] = {count(t)};
    block_exclusive_sums(n, segs, (int(*)[kPlanThreads / 64])tmp);
    if (t <= segs) off[t] = n[0];
    if (t < segs && off != L.seg_off) L.seg_off[t] = n[0];
    if (t == segs) carry = n[0];
    __syncthreads();
  }
  for (int base = segs < kPlanThreads ? segs : 0; base < segs; base += kPlanThreads) {
    const int s = base + t;
    const int n = count(s);
    const int inc = block_inclusive_scan<kPlanThreads>(n, tmp);
    if (s < segs) {
      off[s] = carry + inc - n;
      if (off != L.seg_off) L.seg_off[s] = off[s];
    }
    __syncthreads();
    if (t == kPlanThreads - 1) carry += inc;
    __syncthreads();
  }
  const int total = min(carry, L.max_items);
  if (t == 0) {
    off[segs] = L.seg_off[segs] = total;
    *L.n_items = total;
  }
  __syncthreads();
  const bool ranked = work && L.round > 0 && total <= kPlanThreads;
  for (int i = t; i < total || ranked; i += kPlanThreads) {
    LinItem it = {};
    if (i < total) {
      const int s = upper_index(off, 0, segs, i), c = i - off[s];
      it.part = s >= ng;
      const int rows = it.part ? L.l_suf : L.l_pre;
      it.seg = it.part ? s - ng : s;
      const int lo = it.part ? cu_s[it.seg] : cu_p[s], hi = it.part ? cu_s[it.seg + 1] : cu_p[s + 1];
      it.nrows = min(rows, hi - lo - c * rows);
      it.row0 = L.reverse ? hi - c * rows - it.nrows : lo + c * rows;
      it.last = c == ceil_div(hi - lo, rows) - 1;
      it.group = s;
      if (it.part) {
        int a = 0, b = ng;  // the group of the member: the last one whose members start at or before it
        while (b - a > 1) {
          const int mid = (a + b) >> 1;
          if (ginfo[mid].m0 <= it.seg) a = mid; else b = mid;
        }
        it.group = a;
      }
      if (c > 0) it.prev = i - 1;
      else if (!it.part) it.prev = kInitState;
      else if (L.reverse) it.prev = kNoState;
      else it.prev = cu_p[it.group + 1] > cu_p[it.group] ? off[it.group + 1] - 1 : kInitState;
      it.self = i;
    }
    if (!ranked) {
      L.items[i] = it;
      continue;
    }
    work[t] = i < total ? it.nrows : -1;  // one item a thread
    __syncthreads();
    if (i < total) L.items[item_place(rank_among(work, 0, (total + 3) & ~3, 0, it.nrows, i), total, L.round)] = it;
    break;
  }
}

// The items alone, behind plan_groups_kernel: for grouping arrays of any size.
__global__ void __launch_bounds__(kPlanThreads) lin_items_kernel(const int* __restrict__ cu_p,
                                                                 const int* __restrict__ cu_s, int ng, int ns,
                                                                 const LinList L, const PlanHeader* hdr,
                                                                 const GroupInfoEx* __restrict__ ginfo) {
  alignas(16) __shared__ int tmp[kPlanThreads];
  __shared__ int carry;
  if (hdr->error) {
    if (threadIdx.x == 0) *L.n_items = 0;
    return;
  }
  lin_items(L, cu_p, cu_s, ginfo, ng, ns, L.seg_off, tmp, carry, nullptr);
}

// Groups and the items of one walk or two in one launch, for grouping arrays that fit LDS (the usual case): three
// launches of dependent one-block kernels cost 5 us each.
__global__ void __launch_bounds__(kPlanThreads) lin_plan_kernel(const int* __restrict__ cu_p,
                                                                const int* __restrict__ cu_s,
                                                                const int* __restrict__ gsz, int ng, int ns, int tp,
                                                                int ts, PlanHeader* hdr, GroupInfoEx* ginfo, int* qoff,
                                                                int* kvoff, const LinList a, const LinList b,
                                                                int lists) {
  __shared__ PlanLds lds;
  __shared__ int off[kLdsGroups + kLdsMembers + 1];
  alignas(16) __shared__ int tmp[kPlanThreads];
  __shared__ int carry;
  const bool ok = plan_groups_lds(cu_p, cu_s, gsz, ng, ns, tp, ts, kFwdBM, kKvBN, 1, 0, 0x7fffffffL, 0x7fffffffL, hdr,
                                  ginfo, qoff, kvoff, lds);
  __syncthreads();
  if (!ok) {
    if (threadIdx.x == 0) {
      *a.n_items = 0;
      if (lists > 1) *b.n_items = 0;
    }
    return;
  }
  lin_items(a, lds.cu_p, lds.cu_s, lds.gi, ng, ns, off, tmp, carry, lds.work[0]);
  if (lists > 1) lin_items(b, lds.cu_p, lds.cu_s, lds.gi, ng, ns, off, tmp, carry, lds.work[1]);
}

// ---------------------------------------------------------------- pieces of the walks
// Tile shapes of a walk: C rows a chunk, NW waves. 32 rows of 128-wide bf16 heads leave room for two workgroups on a CU
// (80 KB each), which hide one another's loads and barriers; 128-row chunks with one workgroup of eight waves have half
// the vector work a row and ran no faster (932 us against 899).
template <typename T, int D, int C, int NW>
struct LinTiles {
  static constexpr int kC = C, kNW = NW, kNT = 64 * NW;
  static constexpr int kNB = D / 32;            // 32-wide blocks of a head
  static constexpr int kNQ = C / 32;            // 32-row tiles of a chunk
  static constexpr int kAcc = kNB * kNB / NW;   // 32 x 32 state tiles of a wave
  static constexpr int kTileBytes = LdsTile<T, D>::bytes(C);
  static constexpr int kStateBytes = LdsTile<T, D>::bytes(D);
};

// B operand whose k values are the permuted ones of a transposed fragment (row 4h + (s & 3) + 8 (s >> 2)), here
// elements of a row: for products of a row with a transposed tile.
template <int D>
__device__ __forceinline__ bf16x8 row_perm(const char* tile, int row, int kk, int h, bf16) {
  using L = LdsTile<bf16, D>;
  const i16x4 a = *(const i16x4*)(tile + L::elem_off(row, 16 * kk + 4 * h));
  const i16x4 b = *(const i16x4*)(tile + L::elem_off(row, 16 * kk + 8 + 4 * h));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <int D>
__device__ __forceinline__ Elt<float>::Frag row_perm(const char* tile, int row, int kk, int h, float) {
  using L = LdsTile<float, D>;
  const f32x4 a = *(const f32x4*)(tile + L::elem_off(row, 16 * kk + 4 * h));
  const f32x4 b = *(const f32x4*)(tile + L::elem_off(row, 16 * kk + 8 + 4 * h));
  Elt<float>::Frag f;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    f.v[s] = a[s];
    f.v[4 + s] = b[s];
  }
  return f;
}

// The decays of a chunk's rows in a state update, l^e with e = n-1-row (forward) or row (backward), as products of a
// power for the 16-row step and one for the lane's rows in it, both of exponents >= 0.
template <bool REV>
struct RowDecay {
  float in_step[8];  // of row 4h + (s & 3) + 8 (s >> 2) of a 16-row step
  float g;
  int h;
  __device__ __forceinline__ void init(float g_, int h_) {
    g = g_;
    h = h_;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int row = 4 * h + (s & 3) + 8 * (s >> 2);
      in_step[s] = fast_exp2(g * (float)(REV ? row : 15 - row));
    }
  }
  // before (backward): rows of the segment in front of the chunk, whose decay is not in the state yet
  __device__ __forceinline__ void step(int t, int n, float (&w)[8], int before) const {
    if (REV || 16 * t + 16 <= n) {
      const float f = fast_exp2(g * (float)(REV ? before + 16 * t : n - 16 - 16 * t));
#pragma unroll
      for (int s = 0; s < 8; ++s) w[s] = f * in_step[s];
    } else {  // the step that the chunk ends in: its rows past the end are zero
#pragma unroll
      for (int s = 0; s < 8; ++s) w[s] = fast_exp2(g * (float)max(n - 1 - 16 * t - (4 * h + (s & 3) + 8 * (s >> 2)), 0));
    }
  }
};

// acc[kb] += sum over the chunk's n rows of a_row^T (l^e(row) b_row) (backward: e + before): a's columns 32 (kb0 + kb).., b's columns 32 nb.. .
template <typename T, int D, int C, bool REV, int SPLIT, int N>
__device__ __forceinline__ void state_update(f32x16 (&acc)[N], const char* ta, const char* tb,
                                             const FragOffsets<T, D>& fo, const RowDecay<REV>& rd, int kb0, int nb,
                                             int n, int before = 0) {
  using E = Elt<T>;
#pragma unroll
  for (int t = 0; t < C / 16; ++t) {
    if (t > 0 && 16 * t >= n) break;
    float w[8], x[8];
    rd.step(t, n, w, before);
    const typename E::Frag b = fo.tr(tb, t, nb);
#pragma unroll
    for (int s = 0; s < 8; ++s) x[s] = E::frag_elem(b, s) * w[s];
    typename E::Frag part[SPLIT];
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      part[p] = E::to_frag(x);
      if (p + 1 < SPLIT) {
#pragma unroll
        for (int s = 0; s < 8; ++s) x[s] -= E::frag_elem(part[p], s);
      }
    }
#pragma unroll
    for (int kb = 0; kb < N; ++kb) {
      const typename E::Frag a = fo.tr(ta, t, kb0 + kb);
#pragma unroll
      for (int p = 0; p < SPLIT; ++p) acc[kb] = E::mma(a, part[p], acc[kb]);
    }
  }
}

// The decays of a 32 x 32 score tile (transposed: register r holds row 8 (r / 4) + 4h + r % 4 of the tile's rows, the
// lane its column), from registers filled once: on the diagonal l^(dist) where dist >= 0, else 0; off it l^(31 - a)
// l^(1 + b) l^(32 (tiles - 1)), a and b the earlier and the later row's place in its tile. REV: the registers run
// over the later rows.
template <bool REV>
struct TileDecay {
  float diag[16], reg[16], lane_f;
  float g;
  __device__ __forceinline__ void init(float g_, int lane) {
    g = g_;
    const int l = lane & 31, h = lane >> 5;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 8 * (r / 4) + 4 * h + r % 4, dist = REV ? row - l : l - row;
      diag[r] = dist >= 0 ? fast_exp2(g * (float)dist) : 0.f;
      reg[r] = fast_exp2(g * (float)(REV ? 1 + row : 31 - row));
    }
    lane_f = fast_exp2(g * (float)(REV ? 31 - l : 1 + l));
  }
  // sc *= decays, `tiles` tiles off the diagonal
  __device__ __forceinline__ void apply(f32x16& sc, int tiles) const {
    if (tiles == 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] *= diag[r];
    } else {
      const float f = lane_f * fast_exp2(g * (float)(32 * (tiles - 1)));
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] *= f * reg[r];
    }
  }
};

// A wave's state tiles: rows (of k) 32 (kb0 + kb) + 8 (r / 4) + 4h + r % 4, column (of v) 32 nb + lane % 32.
template <int N>
__device__ __forceinline__ void state_scale(f32x16 (&acc)[N], float f) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] *= f;
}
template <int D, int N>
__device__ __forceinline__ void state_load(f32x16 (&acc)[N], const float* src, int kb0, int nb, int lane) {
  if (src) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        acc[i][r] = src[(32 * (kb0 + i) + 8 * (r / 4) + 4 * (lane >> 5) + r % 4) * D + 32 * nb + (lane & 31)];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;
  }
}
template <int D, int N>
__device__ __forceinline__ void state_store(const f32x16 (&acc)[N], float* dst, int kb0, int nb, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      dst[(32 * (kb0 + i) + 8 * (r / 4) + 4 * (lane >> 5) + r % 4) * D + 32 * nb + (lane & 31)] = acc[i][r];
}
// the state as an LDS operand: row = column of v, four consecutive rows of k a store
template <typename T, int D, int N>
__device__ __forceinline__ void state_to_lds(const f32x16 (&acc)[N], char* st, int kb0, int nb, int lane) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      Elt<T>::store4((T*)(st + LdsTile<T, D>::elem_off(32 * nb + (lane & 31), 32 * (kb0 + i) + 8 * j + 4 * (lane >> 5))),
                     acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]);
}

// An item in scalar registers (it is the same for the whole workgroup; buffer descriptors are formed from it).
__device__ __forceinline__ LinItem uniform_item(const LinItem* items, int i) {
  LinItem it = items[i];
  it.row0 = uniform(it.row0);
  it.nrows = uniform(it.nrows);
  it.part = uniform(it.part);
  it.seg = uniform(it.seg);
  it.prev = uniform(it.prev);
  it.last = uniform(it.last);
  it.group = uniform(it.group);
  it.self = uniform(it.self);
  return it;
}

// Output tiles acc (transposed: register r of tile d holds column 32 (c0 + d) + 8 (r / 4) + 4h + r % 4 of the lane's
// row) times `scale`, to row `row` of an LDS tile.
template <typename T, int D, int N>
__device__ __forceinline__ void rows_to_lds(const f32x16 (&acc)[N], char* tile, int row, int c0, int h, float scale) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      Elt<T>::store4((T*)(tile + LdsTile<T, D>::elem_off(row, 32 * (c0 + d) + 8 * j + 4 * h)), scale * acc[d][4 * j],
                     scale * acc[d][4 * j + 1], scale * acc[d][4 * j + 2], scale * acc[d][4 * j + 3]);
}

// The first `valid` rows of an LDS tile to memory, by the mapping of the loader that brings in such tiles: 16 bytes a
// lane, whole rows by consecutive lanes. Stores straight from the accumulators are 16-byte pieces of 32 rows, loads
// straight into operands 32-byte ones, and the cache takes as long for each as for a line: the output kernel of 78k rows
// x 40 heads ran 1270 us with both, 580 through LDS. Rows past the range are dropped, without a branch: a wait for a
// later load would otherwise wait for the stores too.
template <typename T, int ROWS, int D, int NT>
__device__ __forceinline__ void tile_to_memory(const TileLoader<T, ROWS, D, NT>& m, const char* tile, T* base,
                                               int gstride, int valid) {
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  const int bytes = range_bytes(valid, ROWS, gstride * (int)sizeof(T));
  __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, bytes, 0x00020000);
#pragma unroll
  for (int i = 0; i < m.kPer; ++i) {
    const u32x4 u = *(const u32x4*)(tile + m.loff + i * m.kRowStep * LdsTile<T, D>::kPitch);
    __builtin_amdgcn_raw_buffer_store_b128(u, rs, m.goff + i * m.gstep, 0, 0);
  }
}

// state before an item, NULL for zero
template <int D>
__device__ __forceinline__ const float* state_before(const LinArgs& a, const LinItem& it, int kv, bool reverse) {
  const size_t per = (size_t)D * D;
  if (it.prev >= 0 && !a.alone) return a.slots + ((size_t)it.prev * a.h_kv + kv) * per;
  if (it.prev == kNoState || (a.alone && reverse)) return nullptr;
  if (reverse) return a.slots + ((size_t)(a.max_items + it.group) * a.h_kv + kv) * per;
  return a.state_in ? a.state_in + ((size_t)it.group * a.h_kv + kv) * per : nullptr;
}

// ---------------------------------------------------------------- state kernel
// An item's own share of the state after it. Forward: sum l^.. k v^T of one kv head; backward: sum l^.. q do^T over
// the query heads that share it. Items whose state nobody reads are skipped: a member's last (forward), a prefix's
// last (backward). The next tiles are loaded to registers while the present ones are used.
template <typename T, int D>
using LinStateTiles = LinTiles<T, D, D == 128 && sizeof(T) == 4 ? 32 : 64, 4>;
constexpr int kLinStateThreads = 256;
template <typename T, int D, bool REV, int SPLIT>
__device__ __forceinline__ void lin_state_walk(const LinArgs& a, unsigned block,
                                               char (&lds)[2][2 * LinStateTiles<T, D>::kTileBytes]) {
  using S = LinStateTiles<T, D>;
  static_assert(S::kNT == kLinStateThreads, "threads");
  const BlockSlot slot = xcd_slot(block, a.h_kv, 1);
  if (slot.unit >= a.max_items) return;
  const LinItem it = uniform_item(a.items, slot.unit);  // loaded beside the number of items, not behind it
  if (slot.unit >= *a.n_items) return;
  if (it.last && (it.part == (REV ? 0 : 1) || (REV && a.members_first))) return;
  const int kv = slot.head, ratio = a.h_q / a.h_kv;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int nb = wave % S::kNB, kb0 = (wave / S::kNB) * S::kAcc;
  const float g = log2_decay(a.log_decay, kv);
  const int heads = REV ? a.h_q : a.h_kv, reps = REV ? ratio : 1;
  const T* pa = (const T*)(REV ? a.q[it.part] : a.k[it.part]);
  const T* pb = (const T*)(REV ? a.d_o[it.part] : a.v[it.part]);
  const int gs = heads * D;
  TileLoader<T, S::kC, D, S::kNT> la, lb;
  la.init(gs, wave, lane);
  lb.init(gs, wave, lane);
  FragOffsets<T, D> fo;
  fo.init(lane);
  RowDecay<REV> rd;
  rd.init(g, lane >> 5);
  f32x16 acc[S::kAcc];
  state_load<D>(acc, nullptr, kb0, nb, lane);
  // step i: chunk i / reps, head i % reps
  const int steps = ceil_div(it.nrows, S::kC) * reps;
  auto load = [&](int i) {
    const int done = i / reps * S::kC, n = min(S::kC, it.nrows - done);
    const int row = it.row0 + (REV ? it.nrows - done - n : done);
    const size_t off = ((size_t)row * heads + (REV ? kv * ratio + i % reps : kv)) * D;
    la.load(nullptr, pa + off, gs, n);
    lb.load(nullptr, pb + off, gs, n);
  };
  load(0);
  for (int i = 0; i < steps; ++i) {
    char *ta = lds[i & 1], *tb = ta + S::kTileBytes;
    la.store(ta);
    lb.store(tb);
    __syncthreads();
    if (i + 1 < steps) load(i + 1);
    const int n = min(S::kC, it.nrows - i / reps * S::kC);
    if (i % reps == 0) state_scale(acc, fast_exp2(g * (float)n));
    state_update<T, D, S::kC, REV, SPLIT>(acc, ta, tb, fo, rd, kb0, nb, n);
  }
  state_store<D>(acc, a.slots + ((size_t)it.self * a.h_kv + kv) * (size_t)(D * D), kb0, nb, lane);
}

// One walk's items, or (`first` > 0) those of both walks of a backward call: `first` workgroups of the reverse one, r's,
// which reads more, then the forward one's.
template <typename T, int D, int SPLIT>
__global__ void __launch_bounds__(kLinStateThreads, 2) lin_state_kernel(const LinArgs a, const LinArgs r, unsigned first) {
  __shared__ __align__(16) char lds[2][2 * LinStateTiles<T, D>::kTileBytes];
  if (blockIdx.x < first) lin_state_walk<T, D, true, SPLIT>(r, blockIdx.x, lds);
  else lin_state_walk<T, D, false, SPLIT>(a, blockIdx.x - first, lds);
}

// ---------------------------------------------------------------- scans
// In place over a segment's items: slot := l^rows (state before) + own share. Prefixes (PART 0) and members (PART 1)
// follow one another, members first in a backward walk; D * D / (256 V::kN) workgroups a kv head and segment. Chains of
// dependent sums, all latency, so a thread has kBatch loads in flight. A prefix has many items and there are few
// prefixes: one entry a thread, 32 loads; members have few items or none to do: four entries a thread, 8 loads, fewer
// workgroups (P 16384 in 32 items, 16 members summed: 53 -> 16 us; 64 members with nothing to do 17 -> 6 us).
constexpr int kScanThreads = 256;
template <int PART>
struct ScanVec {
  using type = float;
  static constexpr int kN = 1, kBatch = 32;
};
template <>
struct ScanVec<1> {
  using type = f32x4;
  static constexpr int kN = 4, kBatch = 8;
};

// segments and workgroups that a scan has side by side
template <int D, int PART>
__host__ __device__ inline int scan_segs(const LinArgs& a) {
  const int most = (1 << 20) / (D * D / (kScanThreads * ScanVec<PART>::kN) * a.h_kv), segs = PART ? a.ns : a.ng;
  return segs < most ? segs : most;
}
template <int D, int PART>
__host__ __device__ inline unsigned scan_blocks(const LinArgs& a) {
  return D * D / (kScanThreads * ScanVec<PART>::kN) * a.h_kv * scan_segs<D, PART>(a);
}

template <int D, bool REV, int PART>
__device__ __forceinline__ void lin_scan(const LinArgs& a, unsigned block) {
  using S = ScanVec<PART>;
  using V = typename S::type;
  constexpr int kBatch = S::kBatch, kParts = D * D / (kScanThreads * S::kN);
  const int kv = block / kParts % a.h_kv, seg0 = block / kParts / a.h_kv, step = scan_segs<D, PART>(a);
  const size_t e = S::kN * ((size_t)(block % kParts) * kScanThreads + threadIdx.x), per = (size_t)D * D;
  const float g = log2_decay(a.log_decay, kv);
  auto at = [&](int slot) { return (V*)(a.slots + ((size_t)slot * a.h_kv + kv) * per + e); };
  auto user = [&](const float* p, int seg) { return (V*)(p + ((size_t)seg * a.h_kv + kv) * per + e); };
  const float full = fast_exp2(g * (float)(PART ? a.l_suf : a.l_pre));  // the rows of all items but a segment's last
  for (int seg = seg0; seg < (PART ? a.ns : a.ng); seg += step) {
    const int s = PART ? a.ng + seg : seg;
    const int i0 = a.seg_off[s], i1 = a.seg_off[s + 1];
    // the last item holds what the others leave
    const int len = PART ? a.cu_s[seg + 1] - a.cu_s[seg] : a.cu_p[seg + 1] - a.cu_p[seg];
    const float tail = fast_exp2(g * (float)(len - max(i1 - i0 - 1, 0) * (PART ? a.l_suf : a.l_pre)));
    if (a.hdr->error) return;  // loaded beside the offsets, which mean nothing then
    V st = {};
    if (!PART) {
      if (REV) {  // the members' states, in member order
        const int m0 = a.ginfo[seg].m0, m1 = a.ginfo[seg].m1;
        for (int m = m0; m < m1; m += kBatch) {
          V u[kBatch];
#pragma unroll
          for (int j = 0; j < kBatch; ++j) {
            u[j] = V{};
            if (m + j < m1) {
              const int e0 = a.seg_off[a.ng + m + j], e1 = a.seg_off[a.ng + m + j + 1];
              if (e1 > e0) u[j] = *at(e1 - 1);
            }
          }
#pragma unroll
          for (int j = 0; j < kBatch; ++j) st += u[j];
        }
        *at(a.max_items + seg) = st;
      } else if (a.state_in) {
        st = *user(a.state_in, seg);
      }
    } else if (!REV) {
      const bool handed = a.state_out[1] && i1 == i0;  // an empty member's state is its prefix's
      if (i1 - i0 < 2 && !handed) continue;
      int lo = 0, hi = a.ng;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.ginfo[mid].m0 <= seg) lo = mid; else hi = mid;
      }
      const int p0 = a.seg_off[lo], p1 = a.seg_off[lo + 1];
      if (p1 > p0) st = *at(p1 - 1);
      else if (a.state_in) st = *user(a.state_in, lo);
      if (handed) *user(a.state_out[1], seg) = st;
    }
    // the last item's state has no reader in a prefix walked backwards and in a member walked forwards; members_first:
    // it is the gradient kernel that stores a member's
    const int end = PART ? (REV && !a.members_first ? i1 : i1 - 1) : (REV ? i1 - 1 : i1);
    for (int i = i0; i < end; i += kBatch) {
      V u[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (i + j < end) u[j] = *at(i + j);
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (i + j < end) {
          const float f = i + j < i1 - 1 ? full : tail;
          st = st * f + u[j];
          *at(i + j) = st;
        }
    }
    if (!PART && !REV && a.state_out[0]) *user(a.state_out[0], seg) = st;
  }
}

// Scans of the first kind (a forward walk's prefixes, a reverse one's members) or the second, of the walks that come:
// `first` workgroups for a, the forward walk, the others for r.
template <int D, bool SECOND>
__global__ void __launch_bounds__(kScanThreads) lin_scan_kernel(const LinArgs a, const LinArgs r, unsigned first) {
  if (blockIdx.x < first) lin_scan<D, false, SECOND ? 1 : 0>(a, blockIdx.x);
  else lin_scan<D, true, SECOND ? 0 : 1>(r, blockIdx.x - first);
}

// ---------------------------------------------------------------- outputs (and dq, with the roles swapped)
// One workgroup: one item and `hpw` of the query heads of one kv head, which share the keys, the values and the state
// in LDS. Wave w: query rows 32 (w % kNQ).. of each chunk, columns 32 kDT (w / kNQ).. of the output. Queries come and
// outputs go through LDS in whole rows; what the next head or chunk needs is loaded to registers meanwhile.
template <typename T, int D>
using LinOutTiles = LinTiles<T, D, D == 128 ? 32 : 64, 4>;
constexpr int kLinThreads = 256;

template <typename T, int D>
constexpr int kLinLds = 4 * LinOutTiles<T, D>::kTileBytes + LinOutTiles<T, D>::kStateBytes;

template <typename T, int D, int SPLIT>
__device__ __forceinline__ void lin_out(const LinArgs& a, int hpw, unsigned block, char (&lds)[kLinLds<T, D>]) {
  using S = LinOutTiles<T, D>;
  using E = Elt<T>;
  static_assert(S::kNT == kLinThreads, "threads");
  constexpr int kDT = S::kNB / (S::kNW / S::kNQ), kKK = D / 16;
  const int ratio = a.h_q / a.h_kv, parts = ratio / hpw;
  const BlockSlot slot = xcd_slot(block, a.h_kv * parts, parts);
  if (slot.unit >= a.max_items) return;
  const LinItem it = uniform_item(a.items, slot.unit);  // loaded beside the number of items, not behind it
  if (slot.unit >= *a.n_items) return;
  const int kv = slot.head / parts, h0 = slot.head * hpw;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, l = lane & 31;
  const int nb = wave % S::kNB, kb0 = (wave / S::kNB) * S::kAcc;
  const int qi = S::kNQ == 1 ? 0 : wave % S::kNQ, dt0 = (wave / S::kNQ) * kDT;
  const float g = log2_decay(a.log_decay, kv);
  char *tk = lds, *tv = lds + S::kTileBytes, *tq = lds + 2 * S::kTileBytes, *to = lds + 3 * S::kTileBytes,
       *ts = lds + 4 * S::kTileBytes;
  const int gs = a.h_kv * D, gq = a.h_q * D;
  TileLoader<T, S::kC, D, S::kNT> lk, lv, lq;
  lk.init(gs, wave, lane);
  lv.init(gs, wave, lane);
  lq.init(gq, wave, lane);
  FragOffsets<T, D> fo;
  fo.init(lane);
  RowDecay<false> rd;
  rd.init(g, h);
  TileDecay<false> td;
  td.init(g, lane);
  const float from_state = fast_exp2(g * (float)(32 * qi + l + 1));
  const T *q = (const T*)a.q[it.part], *k = (const T*)a.k[it.part], *v = (const T*)a.v[it.part];
  T* o = (T*)a.out[it.part];
  // the states are returned: the first query head of a kv head stores its member's
  const bool keep = a.state_out[1] && it.part == 1 && it.last && slot.head % parts == 0;

  f32x16 acc[S::kAcc];
  state_load<D>(acc, state_before<D>(a, it, kv, false), kb0, nb, lane);
  // past the item's end: an empty range, nothing is read
  auto load_kv = [&](int done) {
    const int n = min(S::kC, it.nrows - done);
    const size_t at = ((size_t)(it.row0 + done) * a.h_kv + kv) * D;
    lk.load(nullptr, k + at, gs, n);
    lv.load(nullptr, v + at, gs, n);
  };
  auto load_q = [&](int done, int r) {
    lq.load(nullptr, q + ((size_t)(it.row0 + done) * a.h_q + h0 + r) * D, gq, min(S::kC, it.nrows - done));
  };
  if (a.alone && it.part) {  // a member: its group's prefix first
    const T *pk = (const T*)a.k[0], *pv = (const T*)a.v[0];
    const int p0 = uniform(a.cu_p[it.group]), p1 = uniform(a.cu_p[it.group + 1]);
    for (int r = p0; r < p1; r += S::kC) {
      const int n = min(S::kC, p1 - r);
      lk.load(nullptr, pk + ((size_t)r * a.h_kv + kv) * D, gs, n);
      lv.load(nullptr, pv + ((size_t)r * a.h_kv + kv) * D, gs, n);
      __syncthreads();
      lk.store(tk);
      lv.store(tv);
      __syncthreads();
      state_scale(acc, fast_exp2(g * (float)n));
      state_update<T, D, S::kC, false, SPLIT>(acc, tk, tv, fo, rd, kb0, nb, n);
    }
  }
  load_kv(0);
  load_q(0, 0);
  for (int done = 0; done < it.nrows; done += S::kC) {
    const int n = min(S::kC, it.nrows - done);
    __syncthreads();  // the last chunk's keys, values and state have been read
    lk.store(tk);
    lv.store(tv);
    state_to_lds<T, D>(acc, ts, kb0, nb, lane);
    for (int r = 0; r < hpw; ++r) {
      lq.store(tq);  // the last head's were read before the barrier in front of its outputs' way out
      __syncthreads();
      if (r == 0) load_kv(done + S::kC);
      const bool last = r + 1 == hpw;
      load_q(last ? done + S::kC : done, last ? 0 : r + 1);
      // two workgroups share a CU: the one that computes goes before the one that moves tiles (519 -> 497 us at 78k rows
      // x 40 heads, 108 -> 101 at 21k x 32)
      __builtin_amdgcn_s_setprio(1);
      // the state's share, transposed (rows: columns of v; column: the query), scaled for the row's distance from it
      f32x16 acc_o[kDT];
#pragma unroll
      for (int d = 0; d < kDT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc_o[d][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk)
#pragma unroll
        for (int d = 0; d < kDT; ++d)
          acc_o[d] = E::mma(fo.row(ts, 32 * (dt0 + d), kk), fo.row(tq, 32 * qi, kk), acc_o[d]);
      state_scale(acc_o, from_state);
      // the chunk's own keys
      for (int kt = 0; kt <= qi; ++kt) {
        f32x16 sc;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < kKK; ++kk) sc = E::mma(fo.row(tk, 32 * kt, kk), fo.row(tq, 32 * qi, kk), sc);
        td.apply(sc, S::kNQ == 1 ? 0 : qi - kt);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const typename E::Frag p = E::acc_to_frag(sc, half);
#pragma unroll
          for (int d = 0; d < kDT; ++d) acc_o[d] = E::mma(fo.tr(tv, 2 * kt + half, dt0 + d), p, acc_o[d]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      rows_to_lds<T, D>(acc_o, to, 32 * qi + l, dt0, h, a.scale);
      __syncthreads();
      tile_to_memory(lq, to, o + ((size_t)(it.row0 + done) * a.h_q + h0 + r) * D, gq, n);
    }
    if (done + n < it.nrows || keep) {
      state_scale(acc, fast_exp2(g * (float)n));
      state_update<T, D, S::kC, false, SPLIT>(acc, tk, tv, fo, rd, kb0, nb, n);
    }
  }
  if (keep) state_store<D>(acc, a.state_out[1] + ((size_t)it.seg * a.h_kv + kv) * (size_t)(D * D), kb0, nb, lane);
}

template <typename T, int D, int SPLIT>
__global__ void __launch_bounds__(kLinThreads, sizeof(T) == 2 ? 2 : 1) lin_out_kernel(const LinArgs a, int hpw) {
  __shared__ __align__(16) char lds[kLinLds<T, D>];
  lin_out<T, D, SPLIT>(a, hpw, blockIdx.x, lds);
}

// ---------------------------------------------------------------- dk, dv
// One workgroup: one item, one kv head, walked backwards; the query heads that share it follow one another in each
// chunk. Wave w: key rows 32 (w % kNQ).., and of the kNW / kNQ others the first half dv, the second dk, kWT tiles of
// columns each. Everything passes LDS in whole rows; what the next head or chunk needs is loaded to registers meanwhile.
template <typename T, int D, int SPLIT>
__device__ __forceinline__ void lin_grad(const LinArgs& a, int only, unsigned block, char (&lds)[kLinLds<T, D>]) {
  using S = LinOutTiles<T, D>;
  using E = Elt<T>;
  constexpr int kParts = S::kNW / S::kNQ, kWT = S::kNB / (kParts / 2), kKK = D / 16;
  const BlockSlot slot = xcd_slot(block, a.h_kv, 1);
  if (slot.unit >= a.max_items) return;
  const LinItem it = uniform_item(a.items, slot.unit);  // loaded beside the number of items, not behind it
  if (slot.unit >= *a.n_items) return;
  if (only >= 0 && it.part != only) return;
  const int kv = slot.head, ratio = a.h_q / a.h_kv;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, l = lane & 31;
  const int nb = wave % S::kNB, kb0 = (wave / S::kNB) * S::kAcc;
  const int si = S::kNQ == 1 ? 0 : wave % S::kNQ, part = wave / S::kNQ;
  const bool is_dk = part >= kParts / 2;
  const int ct0 = (part % (kParts / 2)) * kWT;
  const float g = log2_decay(a.log_decay, kv);
  char *tk = lds, *tv = lds + S::kTileBytes, *tq = lds + 2 * S::kTileBytes, *tdo = lds + 3 * S::kTileBytes,
       *ts = lds + 4 * S::kTileBytes;
  const int gs = a.h_kv * D, gq = a.h_q * D;
  TileLoader<T, S::kC, D, S::kNT> lk, lv, lq, ld;
  lk.init(gs, wave, lane);
  lv.init(gs, wave, lane);
  lq.init(gq, wave, lane);
  ld.init(gq, wave, lane);
  FragOffsets<T, D> fo;
  fo.init(lane);
  RowDecay<true> rd;
  rd.init(g, h);
  TileDecay<true> td;
  td.init(g, lane);
  const T *q = (const T*)a.q[it.part], *k = (const T*)a.k[it.part], *v = (const T*)a.v[it.part],
          *d_o = (const T*)a.d_o[it.part];
  T *dk = (T*)a.dk[it.part], *dv = (T*)a.dv[it.part];
  // members first: the prefix starts from what the members' last items store
  const bool keep = a.members_first && it.part == 1 && it.last;
  // this wave's key-side rows, query-side rows and what the scores weight
  const char *key = is_dk ? tv : tk, *qry = is_dk ? tdo : tq, *val = is_dk ? tq : tdo;

  f32x16 acc[S::kAcc];
  state_load<D>(acc, state_before<D>(a, it, kv, true), kb0, nb, lane);
  // the chunk that is `done` rows from the item's end: its number of rows (none past the item's start) and first row
  auto rows = [&](int done) { return min(S::kC, it.nrows - done); };
  auto first = [&](int done) { return (size_t)(it.row0 + max(it.nrows - done - S::kC, 0)); };
  auto load_kv = [&](int done) {
    const size_t at = (first(done) * a.h_kv + kv) * D;
    lk.load(nullptr, k + at, gs, rows(done));
    lv.load(nullptr, v + at, gs, rows(done));
  };
  auto load_q = [&](int done, int r) {
    const size_t at = (first(done) * a.h_q + kv * ratio + r) * D;
    lq.load(nullptr, q + at, gq, rows(done));
    ld.load(nullptr, d_o + at, gq, rows(done));
  };
  if (a.alone && !it.part) {  // a prefix: its members' rows first, each by its distance from the prefix's end
    const T *sq = (const T*)a.q[1], *sd = (const T*)a.d_o[1];
    const int m0 = uniform(a.ginfo[it.group].m0), m1 = uniform(a.ginfo[it.group].m1);
    for (int m = m0; m < m1; ++m) {
      const int r0 = uniform(a.cu_s[m]), r1 = uniform(a.cu_s[m + 1]);
      for (int r = r0; r < r1; r += S::kC)
        for (int j = 0; j < ratio; ++j) {
          const int n = min(S::kC, r1 - r);
          const size_t at = ((size_t)r * a.h_q + kv * ratio + j) * D;
          lq.load(nullptr, sq + at, gq, n);
          ld.load(nullptr, sd + at, gq, n);
          __syncthreads();
          lq.store(tq);
          ld.store(tdo);
          __syncthreads();
          state_update<T, D, S::kC, true, SPLIT>(acc, tq, tdo, fo, rd, kb0, nb, n, r - r0);
        }
    }
    __syncthreads();
  }
  load_kv(0);
  load_q(0, 0);
  for (int done = 0; done < it.nrows; done += S::kC) {
    const int n = rows(done);
    lk.store(tk);
    lv.store(tv);
    state_to_lds<T, D>(acc, ts, kb0, nb, lane);
    state_scale(acc, fast_exp2(g * (float)n));
    f32x16 acc_o[kWT];
    for (int r = 0; r < ratio; ++r) {
      lq.store(tq);
      ld.store(tdo);
      __syncthreads();
      if (r == 0) load_kv(done + S::kC);
      const bool last = r + 1 == ratio;
      load_q(last ? done + S::kC : done, last ? 0 : r + 1);
      if (r == 0) {
#pragma unroll
        for (int w = 0; w < kWT; ++w) {
#pragma unroll
          for (int e = 0; e < 16; ++e) acc_o[w][e] = 0.f;
#pragma unroll
          for (int kk = 0; kk < kKK; ++kk) {
            if (is_dk)  // the state's rows of k: a transposed read
              acc_o[w] = E::mma(fo.tr(ts, kk, ct0 + w), row_perm<D>(tv, 32 * si + l, kk, h, T{}), acc_o[w]);
            else
              acc_o[w] = E::mma(fo.row(ts, 32 * (ct0 + w), kk), fo.row(tk, 32 * si, kk), acc_o[w]);
          }
        }
        state_scale(acc_o, fast_exp2(g * (float)max(n - 32 * si - l, 0)));
      }
      for (int tt = si; tt < S::kNQ; ++tt) {
        f32x16 sc;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < kKK; ++kk) sc = E::mma(fo.row(qry, 32 * tt, kk), fo.row(key, 32 * si, kk), sc);
        td.apply(sc, S::kNQ == 1 ? 0 : tt - si);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const typename E::Frag p = E::acc_to_frag(sc, half);
#pragma unroll
          for (int w = 0; w < kWT; ++w) acc_o[w] = E::mma(fo.tr(val, 2 * tt + half, ct0 + w), p, acc_o[w]);
        }
      }
      if (done + n < it.nrows || keep) state_update<T, D, S::kC, true, SPLIT>(acc, tq, tdo, fo, rd, kb0, nb, n);
      __syncthreads();  // q, do (and after the last head k, v and the state) have been read
    }
    // dv and dk go out through the tiles of q and do
    rows_to_lds<T, D>(acc_o, is_dk ? tdo : tq, 32 * si + l, ct0, h, a.scale);
    __syncthreads();
    const size_t at = (first(done) * a.h_kv + kv) * D;
    tile_to_memory(lk, tq, dv + at, gs, n);
    tile_to_memory(lk, tdo, dk + at, gs, n);
    __syncthreads();
  }
  if (keep) state_store<D>(acc, a.slots + ((size_t)it.self * a.h_kv + kv) * (size_t)(D * D), kb0, nb, lane);
}

template <typename T, int D, int SPLIT>
__global__ void __launch_bounds__(kLinThreads, sizeof(T) == 2 ? 2 : 1) lin_grad_kernel(const LinArgs a, int only) {
  __shared__ __align__(16) char lds[kLinLds<T, D>];
  lin_grad<T, D, SPLIT>(a, only, blockIdx.x, lds);
}

// dk and dv (`first` workgroups, of g) and dq in one launch, the longer workgroups first: one does not wait for the
// other's last ones.
template <typename T, int D, int SPLIT>
__global__ void __launch_bounds__(kLinThreads, sizeof(T) == 2 ? 2 : 1) lin_grads_kernel(const LinArgs dq, int hpw,
                                                                                       const LinArgs g, unsigned first,
                                                                                       int only) {
  __shared__ __align__(16) char lds[kLinLds<T, D>];
  if (blockIdx.x < first) lin_grad<T, D, SPLIT>(g, only, blockIdx.x, lds);
  else lin_out<T, D, SPLIT>(dq, hpw, blockIdx.x - first, lds);
}

// ---------------------------------------------------------------- single tokens
// state' = l state + k v^T, o = c state'^T q for the query heads of a kv head. Reads and writes D * D fp32 values a
// (sequence, kv head) for 2 (h_q / h_kv + 1) D * D operations: bound by the state's traffic. A workgroup takes
// kCols columns of one state: kCols / 4 lanes cover a row (16 bytes each), the rest of the threads the rows.
struct LinStepArgs {
  const void *q, *k, *v;
  const float *log_decay, *state;
  void* o;
  float* state_out;
  int n, h_q, h_kv;
  float scale;
};
constexpr int kStepThreads = 256, kStepHeads = 8;  // query heads a pass over the state serves

template <typename T, int D, int COLS>
__global__ void __launch_bounds__(kStepThreads) lin_step_kernel(const LinStepArgs a) {
  constexpr int kLanes = COLS / 4, kRowGroups = kStepThreads / kLanes, kRows = D / kRowGroups;
  static_assert(D % kRowGroups == 0, "rows");
  __shared__ float sq[kStepHeads][D], sk[D];
  __shared__ __align__(16) float red[kRowGroups][kStepHeads][COLS];
  const int ratio = a.h_q / a.h_kv, slices = D / COLS;
  const int t = threadIdx.x, lane = t % kLanes, rg = t / kLanes;
  const long units = (long)a.n * a.h_kv * slices;
  for (long u = blockIdx.x; u < units; u += gridDim.x) {
    const int sl = (int)(u % slices);
    const long nk = u / slices;  // sequence * h_kv + kv head
    const long seq = nk / a.h_kv;
    const int kv = (int)(nk % a.h_kv), c0 = sl * COLS + 4 * lane;
    const float decay = fast_exp2(log2_decay(a.log_decay, kv));
    const float* src = a.state + (size_t)nk * D * D;
    float* dst = a.state_out + (size_t)nk * D * D;
    const T* q = (const T*)a.q + ((size_t)seq * a.h_q + (size_t)kv * ratio) * D;
    f32x4 s[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) s[i] = *(const f32x4*)(src + (size_t)(rg + kRowGroups * i) * D + c0);
    const T* pv = (const T*)a.v + (size_t)nk * D + c0;
    const f32x4 v4 = {(float)pv[0], (float)pv[1], (float)pv[2], (float)pv[3]};
    if (t < D) sk[t] = (float)((const T*)a.k)[(size_t)nk * D + t];
    for (int h0 = 0; h0 < ratio; h0 += kStepHeads) {
      const int nh = min(kStepHeads, ratio - h0);
      for (int i = t; i < nh * D; i += kStepThreads) sq[i / D][i % D] = (float)q[(size_t)h0 * D + i];
      __syncthreads();
      if (h0 == 0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const int r = rg + kRowGroups * i;
          s[i] = s[i] * decay + sk[r] * v4;
          *(f32x4*)(dst + (size_t)r * D + c0) = s[i];
        }
      }
      for (int j = 0; j < nh; ++j) {
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kRows; ++i) o += sq[j][rg + kRowGroups * i] * s[i];
        *(f32x4*)&red[rg][j][4 * lane] = o;
      }
      __syncthreads();
      for (int i = t; i < nh * COLS; i += kStepThreads) {
        const int j = i / COLS, c = i % COLS;
        float sum = 0.f;
#pragma unroll 8
        for (int r = 0; r < kRowGroups; ++r) sum += red[r][j][c];
        ((T*)a.o)[((size_t)seq * a.h_q + (size_t)kv * ratio + h0 + j) * D + sl * COLS + c] = (T)(a.scale * sum);
      }
      __syncthreads();
    }
  }
}

}  // namespace pg
