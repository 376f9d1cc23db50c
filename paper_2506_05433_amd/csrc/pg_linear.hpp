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
// needs no share: it starts from the prefix's state.
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
// prev: slot of the state before it, kNoState, or kInitState (the group's initial state).
struct LinItem {
  int row0, nrows, part, seg, prev, last, group, pad;
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
  const PlanHeader* hdr;
  const GroupInfoEx* ginfo;
  int ng, ns, h_q, h_kv, max_items;
  float scale;
};

// Powers of a head's decay: l^n = 2^(g n), g clamped so that no product with n = 0 is a NaN and a decay of zero
// (a log of -inf) gives l^0 = 1, l^n = 0.
__device__ __forceinline__ float log2_decay(const float* log_decay, int h) {
  return fmaxf(log_decay[h] * kLog2e, -1e5f);
}

// ---------------------------------------------------------------- items
// One block: item offsets of all segments (prefixes, then members), then the items themselves.
__global__ void __launch_bounds__(kPlanThreads) lin_items_kernel(const int* __restrict__ cu_p,
                                                                 const int* __restrict__ cu_s, int ng, int ns, int L,
                                                                 int max_items, int reverse, PlanHeader* hdr,
                                                                 const GroupInfoEx* __restrict__ ginfo, int* seg_off,
                                                                 LinItem* items) {
  __shared__ int tmp[kPlanThreads];
  __shared__ int carry;
  const int t = threadIdx.x, segs = ng + ns;
  if (hdr->error) {
    if (t == 0) hdr->n_qtiles = 0;
    return;
  }
  if (t == 0) carry = 0;
  __syncthreads();
  for (int base = 0; base < segs; base += kPlanThreads) {
    const int s = base + t;
    int n = 0;
    if (s < segs) n = ceil_div(s < ng ? cu_p[s + 1] - cu_p[s] : cu_s[s - ng + 1] - cu_s[s - ng], L);
    const int inc = block_inclusive_scan<kPlanThreads>(n, tmp);
    if (s < segs) seg_off[s] = carry + inc - n;
    __syncthreads();
    if (t == kPlanThreads - 1) carry += inc;
    __syncthreads();
  }
  const int total = min(carry, max_items);
  if (t == 0) {
    seg_off[segs] = total;
    hdr->n_qtiles = total;
  }
  __syncthreads();
  for (int i = t; i < total; i += kPlanThreads) {
    const int s = upper_index(seg_off, 0, segs, i), c = i - seg_off[s];
    LinItem it;
    it.part = s >= ng;
    it.seg = it.part ? s - ng : s;
    const int lo = it.part ? cu_s[it.seg] : cu_p[s], hi = it.part ? cu_s[it.seg + 1] : cu_p[s + 1];
    it.nrows = min(L, hi - lo - c * L);
    it.row0 = reverse ? hi - c * L - it.nrows : lo + c * L;
    it.last = c == ceil_div(hi - lo, L) - 1;
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
    else if (reverse) it.prev = kNoState;
    else it.prev = cu_p[it.group + 1] > cu_p[it.group] ? seg_off[it.group + 1] - 1 : kInitState;
    it.pad = 0;
    items[i] = it;
  }
}

// ---------------------------------------------------------------- pieces of the walks
// Tile shapes: kC rows a chunk, kNW waves. 32-row chunks keep two workgroups of 128-wide bf16 heads on a CU.
constexpr int kLinThreads = 256;
template <typename T, int D>
struct LinShape {
  static constexpr int kNT = kLinThreads, kNW = kNT / 64;
  static constexpr int kC = D == 128 ? 32 : 64;
  static constexpr int kNB = D / 32;                // 32-wide blocks of a head
  static constexpr int kNQ = kC / 32;               // 32-row tiles of a chunk
  static constexpr int kAcc = kNB * kNB / kNW;      // 32 x 32 state tiles of a wave
  static constexpr int kTileBytes = LdsTile<T, D>::bytes(kC);
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

// acc[kb] (+)= sum over the chunk's rows of a_row^T (l^e(row) b_row), e = n-1-row (forward) or row (backward): a's
// columns 32 (kb0 + kb).., b's columns 32 nb.. . Rows past the chunk's end are zero in both tiles.
template <typename T, int D, bool REV, int SPLIT, int N>
__device__ __forceinline__ void state_update(f32x16 (&acc)[N], const char* ta, const char* tb,
                                             const FragOffsets<T, D>& fo, int kb0, int nb, int n, float g, int h) {
  using S = LinShape<T, D>;
  using E = Elt<T>;
#pragma unroll
  for (int t = 0; t < S::kC / 16; ++t) {
    const typename E::Frag b = fo.tr(tb, t, nb);
    float x[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int row = 16 * t + 4 * h + (s & 3) + 8 * (s >> 2);
      const int e = REV ? row : max(n - 1 - row, 0);
      x[s] = E::frag_elem(b, s) * fast_exp2(g * (float)e);
    }
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
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      acc[i][r] = src ? src[(32 * (kb0 + i) + 8 * (r / 4) + 4 * (lane >> 5) + r % 4) * D + 32 * nb + (lane & 31)] : 0.f;
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

// state before an item, NULL for zero
template <int D>
__device__ __forceinline__ const float* state_before(const LinArgs& a, const LinItem& it, int kv, bool reverse) {
  const size_t per = (size_t)D * D;
  if (it.prev >= 0) return a.slots + ((size_t)it.prev * a.h_kv + kv) * per;
  if (it.prev == kNoState) return nullptr;
  if (reverse) return a.slots + ((size_t)(a.max_items + it.group) * a.h_kv + kv) * per;
  return a.state_in ? a.state_in + ((size_t)it.group * a.h_kv + kv) * per : nullptr;
}

// ---------------------------------------------------------------- state kernel
// An item's own share of the state after it. Forward: sum l^.. k v^T of one kv head; backward: sum l^.. q do^T over
// the query heads that share it. Items whose state nobody reads are skipped: a member's last (forward), a prefix's
// last (backward).
template <typename T, int D, bool REV, int SPLIT>
__global__ void __launch_bounds__(kLinThreads, 2) lin_state_kernel(const LinArgs a) {
  using S = LinShape<T, D>;
  __shared__ __align__(16) char lds[2 * S::kTileBytes];
  const BlockSlot slot = xcd_slot(blockIdx.x, a.h_kv, 1);
  if (slot.unit >= a.hdr->n_qtiles) return;  // 0 when the grouping arrays are inconsistent
  const LinItem it = a.items[slot.unit];
  if (it.last && it.part == (REV ? 0 : 1)) return;
  const int kv = slot.head, ratio = a.h_q / a.h_kv;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int nb = wave % S::kNB, kb0 = (wave / S::kNB) * S::kAcc;
  const float g = log2_decay(a.log_decay, kv);
  const int heads = REV ? a.h_q : a.h_kv;
  const T* pa = (const T*)(REV ? a.q[it.part] : a.k[it.part]);
  const T* pb = (const T*)(REV ? a.d_o[it.part] : a.v[it.part]);
  const int gs = heads * D;
  Stager<T, S::kC, D, S::kNT> ld;
  ld.init(gs, wave, lane);
  Stager<T, S::kC, D, S::kNT> ld2;
  ld2.init(gs, wave, lane);
  FragOffsets<T, D> fo;
  fo.init(lane);
  f32x16 acc[S::kAcc];
  state_load<D>(acc, nullptr, kb0, nb, lane);
  char *ta = lds, *tb = lds + S::kTileBytes;
  const int reps = REV ? ratio : 1;
  for (int done = 0; done < it.nrows; done += S::kC) {
    const int n = min(S::kC, it.nrows - done);
    const int row = it.row0 + (REV ? it.nrows - done - n : done);
    state_scale(acc, fast_exp2(g * (float)n));
    for (int r = 0; r < reps; ++r) {
      const size_t off = ((size_t)row * heads + (REV ? kv * ratio + r : kv)) * D;
      ld.load(ta, pa + off, gs, n);
      ld2.load(tb, pb + off, gs, n);
      ld.store(ta);
      ld2.store(tb);
      ld.wait();
      __syncthreads();
      state_update<T, D, REV, SPLIT>(acc, ta, tb, fo, kb0, nb, n, g, lane >> 5);
      __syncthreads();
    }
  }
  state_store<D>(acc, a.slots + ((size_t)slot.unit * a.h_kv + kv) * (size_t)(D * D), kb0, nb, lane);
}

// ---------------------------------------------------------------- scans
// In place over a segment's items: slot := l^rows (state before) + own share. One thread for four entries of a
// state; grid (D * D / 1024, h_kv, segments). Prefixes (part 0) and members (part 1) are separate launches, members
// first in a backward walk.
constexpr int kScanThreads = 256;
template <int D, bool REV>
__global__ void __launch_bounds__(kScanThreads) lin_scan_kernel(const LinArgs a, int part) {
  if (a.hdr->error) return;
  const int kv = blockIdx.y;
  const size_t e = 4 * ((size_t)blockIdx.x * kScanThreads + threadIdx.x), per = (size_t)D * D;
  const float g = log2_decay(a.log_decay, kv);
  auto at = [&](int slot) { return a.slots + ((size_t)slot * a.h_kv + kv) * per + e; };
  for (int seg = blockIdx.z; seg < (part ? a.ns : a.ng); seg += gridDim.z) {
    const int s = part ? a.ng + seg : seg;
    const int i0 = a.seg_off[s], i1 = a.seg_off[s + 1];
    f32x4 st = {0.f, 0.f, 0.f, 0.f};
    if (!part) {
      if (REV) {  // the members' states, in member order
        for (int m = a.ginfo[seg].m0; m < a.ginfo[seg].m1; ++m)
          if (a.seg_off[a.ng + m + 1] > a.seg_off[a.ng + m]) st += *(const f32x4*)at(a.seg_off[a.ng + m + 1] - 1);
        *(f32x4*)at(a.max_items + seg) = st;
      } else if (a.state_in) {
        st = *(const f32x4*)(a.state_in + ((size_t)seg * a.h_kv + kv) * per + e);
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
      if (p1 > p0) st = *(const f32x4*)at(p1 - 1);
      else if (a.state_in) st = *(const f32x4*)(a.state_in + ((size_t)lo * a.h_kv + kv) * per + e);
      if (handed) *(f32x4*)(a.state_out[1] + ((size_t)seg * a.h_kv + kv) * per + e) = st;
    }
    // the last item's state has no reader in a prefix walked backwards and in a member walked forwards
    const int end = (part != 0) == REV ? i1 : i1 - 1;
    for (int i = i0; i < end; ++i) {
      const f32x4 u = *(const f32x4*)at(i);
      const float f = fast_exp2(g * (float)a.items[i].nrows);
      st = st * f + u;
      *(f32x4*)at(i) = st;
    }
    if (!part && !REV && a.state_out[0])
      *(f32x4*)(a.state_out[0] + ((size_t)seg * a.h_kv + kv) * per + e) = st;
  }
}

// ---------------------------------------------------------------- outputs (and dq, with the roles swapped)
// One workgroup: one item, one query head. Wave w: query tile w % kNQ of each chunk, columns 32 kDT (w / kNQ).. .
template <typename T, int D, int SPLIT>
__global__ void __launch_bounds__(kLinThreads, 2) lin_out_kernel(const LinArgs a) {
  using S = LinShape<T, D>;
  using E = Elt<T>;
  constexpr int kDT = S::kNB / (S::kNW / S::kNQ);
  __shared__ __align__(16) char lds[3 * S::kTileBytes + S::kStateBytes];
  const BlockSlot slot = xcd_slot(blockIdx.x, a.h_q, a.h_q / a.h_kv);
  if (slot.unit >= a.hdr->n_qtiles) return;
  const LinItem it = a.items[slot.unit];
  const int hq = slot.head, ratio = a.h_q / a.h_kv, kv = hq / ratio;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, l = lane & 31;
  const int nb = wave % S::kNB, kb0 = (wave / S::kNB) * S::kAcc;
  const int qi = wave % S::kNQ, dt0 = (wave / S::kNQ) * kDT;
  const float g = log2_decay(a.log_decay, kv);
  char *tq = lds, *tk = lds + S::kTileBytes, *tv = lds + 2 * S::kTileBytes, *ts = lds + 3 * S::kTileBytes;
  Stager<T, S::kC, D, S::kNT> lq, lk, lv;
  lq.init(a.h_q * D, wave, lane);
  lk.init(a.h_kv * D, wave, lane);
  lv.init(a.h_kv * D, wave, lane);
  FragOffsets<T, D> fo;
  fo.init(lane);
  const T *q = (const T*)a.q[it.part], *k = (const T*)a.k[it.part], *v = (const T*)a.v[it.part];
  T* o = (T*)a.out[it.part];
  // the states are returned: the first query head of a kv head stores its member's
  const bool keep = a.state_out[1] && it.part == 1 && it.last && hq == kv * ratio;

  f32x16 acc[S::kAcc];
  state_load<D>(acc, state_before<D>(a, it, kv, false), kb0, nb, lane);
  for (int done = 0; done < it.nrows; done += S::kC) {
    const int n = min(S::kC, it.nrows - done);
    const size_t row = it.row0 + done;
    lq.load(tq, q + (row * a.h_q + hq) * D, a.h_q * D, n);
    lk.load(tk, k + (row * a.h_kv + kv) * D, a.h_kv * D, n);
    lv.load(tv, v + (row * a.h_kv + kv) * D, a.h_kv * D, n);
    state_to_lds<T, D>(acc, ts, kb0, nb, lane);
    lq.store(tq);
    lk.store(tk);
    lv.store(tv);
    lq.wait();
    __syncthreads();
    // the state's share, transposed (rows: columns of v; column: the query), scaled for the row's distance from it
    f32x16 acc_o[kDT];
#pragma unroll
    for (int d = 0; d < kDT; ++d) {
#pragma unroll
      for (int r = 0; r < 16; ++r) acc_o[d][r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        acc_o[d] = E::mma(fo.row(ts, 32 * (dt0 + d), kk), fo.row(tq, 32 * qi, kk), acc_o[d]);
    }
    state_scale(acc_o, fast_exp2(g * (float)(32 * qi + l + 1)));
    // the chunk's own keys
    for (int kt = 0; kt <= qi; ++kt) {
      f32x16 sc;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) sc = E::mma(fo.row(tk, 32 * kt, kk), fo.row(tq, 32 * qi, kk), sc);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int dist = 32 * (qi - kt) + l - (8 * (r / 4) + 4 * h + r % 4);
        sc[r] = dist >= 0 ? sc[r] * fast_exp2(g * (float)dist) : 0.f;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const typename E::Frag p = E::acc_to_frag(sc, half);
#pragma unroll
        for (int d = 0; d < kDT; ++d) acc_o[d] = E::mma(fo.tr(tv, 2 * kt + half, dt0 + d), p, acc_o[d]);
      }
    }
    if (32 * qi + l < n) {
      T* dst = o + ((row + 32 * qi + l) * a.h_q + hq) * D;
#pragma unroll
      for (int d = 0; d < kDT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          E::store4(dst + 32 * (dt0 + d) + 8 * j + 4 * h, a.scale * acc_o[d][4 * j], a.scale * acc_o[d][4 * j + 1],
                    a.scale * acc_o[d][4 * j + 2], a.scale * acc_o[d][4 * j + 3]);
    }
    if (done + n < it.nrows || keep) {
      state_scale(acc, fast_exp2(g * (float)n));
      state_update<T, D, false, SPLIT>(acc, tk, tv, fo, kb0, nb, n, g, h);
    }
    __syncthreads();
  }
  if (keep) state_store<D>(acc, a.state_out[1] + ((size_t)it.seg * a.h_kv + kv) * (size_t)(D * D), kb0, nb, lane);
}

// ---------------------------------------------------------------- dk, dv
// One workgroup: one item, one kv head, walked backwards; the query heads that share it follow one another in each
// chunk. Wave w: key rows 32 (w % kNQ).., and of the kNW / kNQ others the first half dv, the second dk, kWT tiles of
// columns each.
template <typename T, int D, int SPLIT>
__global__ void __launch_bounds__(kLinThreads, 2) lin_grad_kernel(const LinArgs a) {
  using S = LinShape<T, D>;
  using E = Elt<T>;
  constexpr int kParts = S::kNW / S::kNQ, kWT = S::kNB / (kParts / 2);
  __shared__ __align__(16) char lds[4 * S::kTileBytes + S::kStateBytes];
  const BlockSlot slot = xcd_slot(blockIdx.x, a.h_kv, 1);
  if (slot.unit >= a.hdr->n_qtiles) return;
  const LinItem it = a.items[slot.unit];
  const int kv = slot.head, ratio = a.h_q / a.h_kv;
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5, l = lane & 31;
  const int nb = wave % S::kNB, kb0 = (wave / S::kNB) * S::kAcc;
  const int si = wave % S::kNQ, part = wave / S::kNQ;
  const bool is_dk = part >= kParts / 2;
  const int ct0 = (part % (kParts / 2)) * kWT;
  const float g = log2_decay(a.log_decay, kv);
  char *tk = lds, *tv = lds + S::kTileBytes, *tq = lds + 2 * S::kTileBytes, *td = lds + 3 * S::kTileBytes,
       *ts = lds + 4 * S::kTileBytes;
  Stager<T, S::kC, D, S::kNT> lkv, lk2, lqd, lq2;
  lkv.init(a.h_kv * D, wave, lane);
  lk2.init(a.h_kv * D, wave, lane);
  lqd.init(a.h_q * D, wave, lane);
  lq2.init(a.h_q * D, wave, lane);
  FragOffsets<T, D> fo;
  fo.init(lane);
  const T *q = (const T*)a.q[it.part], *k = (const T*)a.k[it.part], *v = (const T*)a.v[it.part],
          *d_o = (const T*)a.d_o[it.part];
  T* out = (T*)(is_dk ? a.dk[it.part] : a.dv[it.part]);
  const char* key = is_dk ? tv : tk;  // the key-side rows and the query-side rows of this wave's scores
  const char* qry = is_dk ? td : tq;
  const char* val = is_dk ? tq : td;  // what the scores weight

  f32x16 acc[S::kAcc];
  state_load<D>(acc, state_before<D>(a, it, kv, true), kb0, nb, lane);
  for (int done = 0; done < it.nrows; done += S::kC) {
    const int n = min(S::kC, it.nrows - done);
    const size_t row = it.row0 + (it.nrows - done - n);
    lkv.load(tk, k + (row * a.h_kv + kv) * D, a.h_kv * D, n);
    lk2.load(tv, v + (row * a.h_kv + kv) * D, a.h_kv * D, n);
    state_to_lds<T, D>(acc, ts, kb0, nb, lane);
    lkv.store(tk);
    lk2.store(tv);
    state_scale(acc, fast_exp2(g * (float)n));
    f32x16 acc_o[kWT];
    for (int r = 0; r < ratio; ++r) {
      const size_t off = (row * a.h_q + kv * ratio + r) * D;
      lqd.load(tq, q + off, a.h_q * D, n);
      lq2.load(td, d_o + off, a.h_q * D, n);
      lqd.store(tq);
      lq2.store(td);
      lqd.wait();
      __syncthreads();
      if (r == 0) {
#pragma unroll
        for (int c = 0; c < kWT; ++c) {
#pragma unroll
          for (int e = 0; e < 16; ++e) acc_o[c][e] = 0.f;
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            if (is_dk)  // the state's rows of k: a transposed read
              acc_o[c] = E::mma(fo.tr(ts, kk, ct0 + c), row_perm<D>(tv, 32 * si + l, kk, h, T{}), acc_o[c]);
            else
              acc_o[c] = E::mma(fo.row(ts, 32 * (ct0 + c), kk), fo.row(tk, 32 * si, kk), acc_o[c]);
          }
        }
        state_scale(acc_o, fast_exp2(g * (float)max(n - 32 * si - l, 0)));
      }
      for (int tt = si; tt < S::kNQ; ++tt) {
        f32x16 sc;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) sc = E::mma(fo.row(qry, 32 * tt, kk), fo.row(key, 32 * si, kk), sc);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int dist = 32 * (tt - si) + (8 * (e / 4) + 4 * h + e % 4) - l;
          sc[e] = dist >= 0 ? sc[e] * fast_exp2(g * (float)dist) : 0.f;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const typename E::Frag p = E::acc_to_frag(sc, half);
#pragma unroll
          for (int c = 0; c < kWT; ++c) acc_o[c] = E::mma(fo.tr(val, 2 * tt + half, ct0 + c), p, acc_o[c]);
        }
      }
      if (done + n < it.nrows) state_update<T, D, true, SPLIT>(acc, tq, td, fo, kb0, nb, n, g, h);
      __syncthreads();
    }
    if (32 * si + l < n) {
      T* dst = out + ((row + 32 * si + l) * a.h_kv + kv) * D;
#pragma unroll
      for (int c = 0; c < kWT; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          E::store4(dst + 32 * (ct0 + c) + 8 * j + 4 * h, a.scale * acc_o[c][4 * j], a.scale * acc_o[c][4 * j + 1],
                    a.scale * acc_o[c][4 * j + 2], a.scale * acc_o[c][4 * j + 3]);
    }
  }
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
