// Log-probabilities of the responses' tokens from the logits, their gradient, and the clipped policy loss.
//
// In the grouped layout response row j of a member predicts token j + 1 of it, and the last prefix row of a group
// predicts the first token of every one of its members: one softmax with as many targets as the group has members,
// whose gradient sums over them (Lemma 1's sum over the copies of the prefix, for its last row).
//
// Both logits kernels read a row once, one workgroup a row, 16 bytes a lane and load, and are bound by that traffic:
// forward with a running maximum and sum (softmax statistics and the entropy's sum in fp32), backward from the saved
// log-sum-exp. Rows start at any alignment the element type has; a row's first elements up to a 16-byte boundary and
// its last ones are taken one by one.
#pragma once
#include <cfloat>
#include "pg_common.hpp"
#include "pg_plan.hpp"

namespace pg {

struct LogprobArgs {
  const void *last, *suf;  // logits [n_groups, vocab], [total_suffix, vocab]
  void *d_last, *d_suf;
  long ld_last, ld_suf, ldd_last, ldd_suf;  // elements between rows
  const void* tokens;                       // [total_suffix], int32 or int64
  int tok64;
  float *logp, *lse, *entropy;
  const float* dlogp;
  float* target;  // [n_suffixes]: gradient at the first token of each member, summed over those that share it
  const int *cu_p, *cu_s;
  const PlanHeader* hdr;
  const GroupInfoEx* ginfo;
  int ng, ns, ts, vocab;
  float inv_temp;
};

// Largest index i in [0, n) with a[i] <= x (a nondecreasing, a[0] <= x), by a whole wave: 64 entries a step.
__device__ __forceinline__ int wave_upper_index(const int* __restrict__ a, int n, int x) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 63) / 64;
    const int i = lo + lane * step;
    const bool le = lane * step < len && a[i] <= x;  // true for a prefix of the lanes, lane 0 among them
    const int cnt = __popcll(__ballot(le));
    const int first = (cnt - 1) * step;
    lo += first;
    len = min(step, len - first);
  }
  return uniform(lo);
}

// The token at response row r, or -1 where it is outside [0, vocab).
__device__ __forceinline__ int token_at(const LogprobArgs& a, int r) {
  const long t = a.tok64 ? ((const long long*)a.tokens)[r] : (long)((const int*)a.tokens)[r];
  return t >= 0 && t < a.vocab ? (int)t : -1;
}

// Elements of 16 bytes as floats.
template <typename T>
struct Vec16;
template <>
struct Vec16<bf16> {
  static constexpr int kN = 8;
  __device__ __forceinline__ static void unpack(const uint4& u, float (&x)[8]) {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static uint4 pack(const float (&x)[8]) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (bf16)x[i];
    return __builtin_bit_cast(uint4, v);
  }
};
template <>
struct Vec16<float> {
  static constexpr int kN = 4;
  __device__ __forceinline__ static void unpack(const uint4& u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x);
    x[1] = __uint_as_float(u.y);
    x[2] = __uint_as_float(u.z);
    x[3] = __uint_as_float(u.w);
  }
  __device__ __forceinline__ static uint4 pack(const float (&x)[4]) {
    return uint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};

// Elements before the first 16-byte boundary of a row (a row of fewer elements is all head).
template <typename T>
__device__ __forceinline__ int row_head(const T* p, int n) {
  const int h = (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T);
  return h < n ? h : n;
}

// Running softmax statistics in base 2: m the largest x seen, s = sum 2^(c (x - m)), w = sum 2^(c (x - m)) c (x - m).
struct SoftStat {
  float m, s, w;
};
constexpr float kFarBelow = -1e30f;  // a finite stand-in for c (x - m) of x = -inf, whose term is 0
constexpr float kFarOut = 1e36f;     // c x might overflow from here on (rows masked with the type's lowest value)

template <bool ENT, int N>
__device__ __forceinline__ void soft_add(SoftStat& a, const float (&x)[N], float c) {
  float mx = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) mx = fmaxf(mx, x[i]);
  if (mx > a.m) {
    const float z = fmaxf(c * (a.m - mx), kFarBelow), f = fast_exp2(z);
    if (ENT) a.w = f * (a.w + a.s * z);
    a.s *= f;
    a.m = mx;
  }
  if (fabsf(a.m) < kFarOut) {
    const float off = -c * a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = fmaf(c, x[i], off), e = fast_exp2(z);
      a.s += e;
      if (ENT) a.w += e * fmaxf(z, kFarBelow);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (x[i] == -INFINITY) continue;
      const float z = c * (x[i] - a.m), e = fast_exp2(z);
      a.s += e;
      if (ENT) a.w += e * fmaxf(z, kFarBelow);
    }
  }
}

__device__ __forceinline__ SoftStat soft_join(const SoftStat& a, const SoftStat& b, float c) {
  SoftStat r;
  r.m = fmaxf(a.m, b.m);
  const float za = a.m == r.m ? 0.f : fmaxf(c * (a.m - r.m), kFarBelow);
  const float zb = b.m == r.m ? 0.f : fmaxf(c * (b.m - r.m), kFarBelow);
  const float fa = fast_exp2(za), fb = fast_exp2(zb);
  r.s = a.s * fa + b.s * fb;
  r.w = fa * (a.w + a.s * za) + fb * (b.w + b.s * zb);
  return r;
}

// Row b of the logits: the groups' last prefix rows, then the response rows. `targets`: the response rows
// [first of each member m0 .. m1), or the one row `target`; none when target < 0 and m0 == m1.
struct LogitRow {
  int group, target, m0, m1;
};
__device__ __forceinline__ LogitRow logit_row(const LogprobArgs& a, long b) {
  LogitRow r{-1, -1, 0, 0};
  if (b < a.ng) {
    r.group = (int)b;
    const GroupInfoEx gi = a.ginfo[b];
    if (gi.p1 > gi.p0) {  // an empty prefix has no row that predicts
      r.m0 = gi.m0;
      r.m1 = gi.m1;
    }
  } else {
    const int row = (int)(b - a.ng), m = wave_upper_index(a.cu_s, a.ns, row);
    if (row + 1 < a.cu_s[m + 1]) r.target = row + 1;
  }
  return r;
}

// The statistics of a whole row, by the workgroup; every thread gets them. part: one entry for each wave.
template <typename T, int NT, bool ENT>
__device__ __forceinline__ SoftStat row_stats(const T* x, int vocab, float c, SoftStat* part) {
  using V = Vec16<T>;
  constexpr int kUnroll = 4;
  const int t = threadIdx.x;
  SoftStat st{-INFINITY, 0.f, 0.f};
  const int head = row_head(x, vocab), nv = (vocab - head) / V::kN, tail = head + nv * V::kN;
  if (t < head) {
    const float v[1] = {(float)x[t]};
    soft_add<ENT>(st, v, c);
  }
  if (t < vocab - tail) {
    const float v[1] = {(float)x[tail + t]};
    soft_add<ENT>(st, v, c);
  }
  const uint4* xv = (const uint4*)(x + head);
  for (int i = t; i < nv; i += kUnroll * NT) {
    uint4 u[kUnroll];
    if (i - t + kUnroll * NT <= nv) {  // the whole workgroup: no test for each piece
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) u[k] = xv[i + k * NT];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        float v[V::kN];
        V::unpack(u[k], v);
        soft_add<ENT>(st, v, c);
      }
    } else {  // what is left, its loads side by side too
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i + k * NT < nv) u[k] = xv[i + k * NT];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (i + k * NT >= nv) break;
        float v[V::kN];
        V::unpack(u[k], v);
        soft_add<ENT>(st, v, c);
      }
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    SoftStat o;
    o.m = __shfl_xor(st.m, off);
    o.s = __shfl_xor(st.s, off);
    o.w = __shfl_xor(st.w, off);
    st = soft_join(st, o, c);
  }
  if (NT > 64) {
    if ((t & 63) == 0) part[t >> 6] = st;
    __syncthreads();
    st = part[0];
    for (int k = 1; k < NT / 64; ++k) st = soft_join(st, part[k], c);
    __syncthreads();
  }
  return st;
}

template <typename T, int NT, bool ENT>
__global__ void __launch_bounds__(NT) logprob_kernel(const LogprobArgs a) {
  __shared__ SoftStat part[NT / 64];
  if (a.hdr->error) return;
  const int t = threadIdx.x;
  const float c = a.inv_temp * kLog2e;
  for (long b = blockIdx.x; b < (long)a.ng + a.ts; b += gridDim.x) {
    const LogitRow row = logit_row(a, b);
    if (row.group >= 0 && row.m0 == row.m1) {
      // no row predicts the first tokens of this group's members
      const GroupInfoEx gi = a.ginfo[row.group];
      for (int m = gi.m0 + t; m < gi.m1; m += NT) {
        const int r = a.cu_s[m];
        if (r == a.cu_s[m + 1]) continue;
        a.logp[r] = 0.f;
        a.lse[r] = -INFINITY;
        if (ENT) a.entropy[r] = 0.f;
      }
      continue;
    }
    if (row.group < 0 && row.target < 0) continue;
    const T* x = row.group >= 0 ? (const T*)a.last + row.group * a.ld_last : (const T*)a.suf + (b - a.ng) * a.ld_suf;
    const SoftStat st = row_stats<T, NT, ENT>(x, a.vocab, c, part);
    // ln sum exp(x / T), and the entropy ln s - sum p ln 2 c (x - m)
    // (a maximum passes over NaN, the sum does not: a row of NaN and -inf has s = NaN, one of -inf alone s = 0)
    const bool none = st.m == -INFINITY && st.s == 0.f;
    const float ln_s = logf(st.s);
    float lse = none ? -INFINITY : st.m * a.inv_temp + ln_s;
    if (lse == -INFINITY && !none) lse = -FLT_MAX;  // m / T is out of range: -inf is for rows with nothing left
    float ent = none ? 0.f : ln_s - kLn2 * st.w / st.s;
    if (ent < 0.f) ent = 0.f;  // by rounding only; a NaN stays
    auto put = [&](int r) {
      const int tok = token_at(a, r);
      float lp = 0.f;
      if (tok >= 0) lp = none ? -INFINITY : ((float)x[tok] - st.m) * a.inv_temp - ln_s;
      a.logp[r] = lp;
      a.lse[r] = lse;
      if (ENT) a.entropy[r] = ent;
    };
    if (row.group < 0) {
      if (t == 0) put(row.target);
    } else {
      for (int m = row.m0 + t; m < row.m1; m += NT)
        if (a.cu_s[m + 1] > a.cu_s[m]) put(a.cu_s[m]);
    }
  }
}

// dlogits = (1 / T) sum over the row's targets of dlogp (onehot - softmax). A row without a target, or whose targets
// all have dlogp = 0 or a token outside the vocabulary, or with no finite logit, gets zeros and is not read.
// The row that a group's members share has many targets. One thread a member sums what the members with its token add,
// in member order, and forms that element's gradient before the row is written (it may be written over the logits); the
// row is written as if it had no target, and the targets' elements after it. (One group, two rows a member, 32000 wide:
// 64, 256 and 1024 members 159, 811 and 3226 us when every 16 bytes with a target walked the members, 17, 20 and 74 now.)
constexpr int kStaged = 1024;  // members in LDS at a time

template <typename T, int NT>
__global__ void __launch_bounds__(NT) logprob_bwd_kernel(const LogprobArgs a) {
  using V = Vec16<T>;
  constexpr int kUnroll = 4;
  alignas(16) __shared__ int staged_tok[kStaged];  // first tokens of the group's members, -1 where there is no gradient
  alignas(16) __shared__ float staged_d[kStaged];
  __shared__ float sum_part[NT / 64], lse_part[NT / 64];
  __shared__ int any_part[NT / 64];
  __shared__ SoftStat stat_part[NT / 64];
  if (a.hdr->error) return;
  const int t = threadIdx.x;
  const float c = a.inv_temp * kLog2e;
  for (long b = blockIdx.x; b < (long)a.ng + a.ts; b += gridDim.x) {
    const LogitRow row = logit_row(a, b);
    const bool grp = row.group >= 0;
    const T* x = grp ? (const T*)a.last + row.group * a.ld_last : (const T*)a.suf + (b - a.ng) * a.ld_suf;
    T* dx = grp ? (T*)a.d_last + row.group * a.ldd_last : (T*)a.d_suf + (b - a.ng) * a.ldd_suf;
    // the gradient's head follows dx's alignment; x may have another one, then it is read element by element
    const int head = row_head(dx, a.vocab), nv = (a.vocab - head) / V::kN, tail = head + nv * V::kN;
    const bool same = (((uintptr_t)x ^ (uintptr_t)dx) & 15) == 0;
    float total = 0.f, lse = -INFINITY, d1 = 0.f;
    int tok1 = -1, any = 0;
    // the token that member m starts with and its gradient; false where there is none
    auto first_token = [&](int m, int& tok, float& d) {
      const int r = a.cu_s[m];
      if (r == a.cu_s[m + 1]) return false;
      tok = token_at(a, r);
      d = a.dlogp[r];
      return tok >= 0 && d != 0.f;
    };
    if (grp) {
      float sum = 0.f, l = -INFINITY;
      for (int m = row.m0 + t; m < row.m1; m += NT) {
        const int r = a.cu_s[m];
        if (r < a.cu_s[m + 1]) l = a.lse[r];  // the same for every member: the row's own
        int tok;
        float d;
        if (!first_token(m, tok, d)) continue;
        any = 1;
        sum += d;
      }
      // a fixed order: the members of a lane, the lanes of a wave, the waves
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) {
        sum += __shfl_xor(sum, off);
        const float o = __shfl_xor(l, off);
        l = l == -INFINITY ? o : l;
        any |= __shfl_xor(any, off);
      }
      if ((t & 63) == 0) {
        sum_part[t >> 6] = sum;
        lse_part[t >> 6] = l;
        any_part[t >> 6] = any;
      }
      __syncthreads();
      any = 0;
#pragma unroll
      for (int k = 0; k < NT / 64; ++k) {
        total += sum_part[k];
        any |= any_part[k];
        if (lse == -INFINITY) lse = lse_part[k];
      }
    } else if (row.target >= 0) {
      tok1 = token_at(a, row.target);
      d1 = a.dlogp[row.target];
      lse = a.lse[row.target];
      if (tok1 >= 0 && d1 != 0.f) {
        any = 1;
        total = d1;
      } else {
        tok1 = -1;
      }
    }
    if (lse == -INFINITY) any = 0;
    // p = 2^(c x - lse log2 e); where the log-sum-exp is too large for that it has also lost ln s (a row masked with
    // the type's lowest value throughout), and the statistics are taken again: p = 2^(c (x - m)) / s
    const bool far = any && fabsf(lse) >= kFarOut;
    float off = -lse * kLog2e, w = -total * a.inv_temp, top = 0.f;
    if (far) {
      const SoftStat st = row_stats<T, NT, false>(x, a.vocab, c, stat_part);
      top = st.m;
      off = 0.f;
      w /= st.s;
    }
    auto prob = [&](float v) { return fast_exp2(far ? c * (v - top) : fmaf(c, v, off)); };
    if (grp && any) {
      const int n = row.m1 - row.m0;
      for (int i0 = 0; i0 < n; i0 += NT) {
        int mine = -1;
        float d, add = 0.f;
        if (i0 + t < n && !first_token(row.m0 + i0 + t, mine, d)) mine = -1;
        for (int j0 = 0; j0 < n; j0 += kStaged) {
          const int here = min(kStaged, n - j0), up = (here + 3) & ~3;
          if (i0 == 0 || n > kStaged) {
            __syncthreads();
            for (int j = t; j < up; j += NT) {
              int tok = -1;
              float dj = 0.f;
              const bool has = j < here && first_token(row.m0 + j0 + j, tok, dj);
              staged_tok[j] = has ? tok : -1;
              staged_d[j] = dj;
            }
            __syncthreads();
          }
          if (mine >= 0)
#pragma unroll 4
            for (int j = 0; j < up; j += 4) {
              const int4 q = *(const int4*)(staged_tok + j);
              const f32x4 v = *(const f32x4*)(staged_d + j);
              add += q.x == mine ? v[0] : 0.f;
              add += q.y == mine ? v[1] : 0.f;
              add += q.z == mine ? v[2] : 0.f;
              add += q.w == mine ? v[3] : 0.f;
            }
        }
        if (mine >= 0) a.target[row.m0 + i0 + t] = fmaf(add, a.inv_temp, prob((float)x[mine]) * w);
      }
      __syncthreads();  // the targets' logits have been read
    }
    auto one = [&](int e) {
      float y = 0.f;
      if (any) y = fmaf(e == tok1 ? d1 : 0.f, a.inv_temp, prob((float)x[e]) * w);  // as vec() forms it, bit for bit
      dx[e] = (T)y;
    };
    if (t < head) one(t);
    if (t < a.vocab - tail) one(tail + t);
    uint4* dv = (uint4*)(dx + head);
    if (!any) {
      for (int i = t; i < nv; i += NT) dv[i] = uint4{0, 0, 0, 0};
    } else {
      auto vec = [&](int i, const float (&v)[V::kN]) {
        float y[V::kN];
#pragma unroll
        for (int k = 0; k < V::kN; ++k) y[k] = prob(v[k]) * w;
        const int e0 = head + i * V::kN;
        if ((unsigned)(tok1 - e0) < (unsigned)V::kN) {
#pragma unroll
          for (int k = 0; k < V::kN; ++k)
            if (tok1 - e0 == k) y[k] = fmaf(d1, a.inv_temp, y[k]);
        }
        dv[i] = V::pack(y);
      };
      const T* xs = x + head;
      if (same) {
        for (int i = t; i < nv; i += kUnroll * NT) {
          uint4 u[kUnroll];
          const bool whole = i - t + kUnroll * NT <= nv;
#pragma unroll
          for (int k = 0; k < kUnroll; ++k)
            if (whole || i + k * NT < nv) u[k] = ((const uint4*)xs)[i + k * NT];
#pragma unroll
          for (int k = 0; k < kUnroll; ++k) {
            if (!whole && i + k * NT >= nv) break;
            float v[V::kN];
            V::unpack(u[k], v);
            vec(i + k * NT, v);
          }
        }
      } else {
        for (int i = t; i < nv; i += NT) {
          float v[V::kN];
#pragma unroll
          for (int k = 0; k < V::kN; ++k) v[k] = (float)xs[i * V::kN + k];
          vec(i, v);
        }
      }
    }
    __syncthreads();  // the partial sums are reused by the next row; the targets' elements come after the others
    if (grp && any)
      for (int m = row.m0 + t; m < row.m1; m += NT) {
        int tok;
        float d;
        if (first_token(m, tok, d)) dx[tok] = (T)a.target[m];  // members with one token write the same
      }
  }
}

// ---------------------------------------------------------------- policy loss
// Token t of member m of group g, with r = exp(lp - lp_old), A the member's advantage, x = lp_ref - lp:
//   L_t = -min(r A, clip(r, 1 - lo, 1 + hi) A) + beta (exp(x) - x - 1),   loss = sum_t w_t L_t,
//   dL_t / dlp = -[not clipped] r A + beta (1 - exp(x)).
// w_t = 1 / (groups with members * members of g * kept tokens of m), or 1 / all kept tokens. The arithmetic is in
// fp64: a batch has at most some hundred thousand tokens of 20 bytes each, so the time is launches and latency, the
// ratio next to the clip's border is decided as the definition does, and the sums cancel.
struct PolicyArgs {
  const float *logp, *logp_old, *logp_ref, *adv;
  const unsigned char* mask;
  const int *cu_s, *gsz;
  float *stats, *dlogp;
  PlanHeader* hdr;
  double* member_w;  // [n_suffixes]: 1 / (groups * members) of each member
  int* count;        // [n_suffixes + 1]: kept tokens of each member, and of all
  double* part;      // [blocks, 4]
  int ng, ns, ts, by_token;
  double cut_lo, cut_hi, beta, grad_scale;
};
constexpr int kPolicyThreads = 1024, kPolicyTok = 256;
constexpr int kPolicyPer = 4;       // tokens a thread
constexpr int kPolicySmall = 8192;  // tokens that one workgroup takes in one launch

struct PolicySums {
  double v[4];
};

// One kept token: adds to the sums, returns its gradient.
__device__ __forceinline__ double policy_token(const PolicyArgs& a, double lp, double old, double ref, double adv,
                                               double w, PolicySums& s) {
  const double lr = a.logp_old ? lp - old : 0.0;
  const bool cut = (adv > 0.0 && lr > a.cut_hi) || (adv < 0.0 && lr < a.cut_lo);
  const double r = exp(cut ? (adv > 0.0 ? a.cut_hi : a.cut_lo) : lr);
  const double ra = adv == 0.0 ? 0.0 : r * adv;
  double kl = 0.0, grad = cut ? 0.0 : -ra;
  if (a.logp_ref) {
    const double x = ref - lp, em = expm1(x);
    kl = em - x;
    if (a.beta != 0.0) grad -= a.beta * em;
  }
  s.v[0] += w * ((a.beta != 0.0 ? a.beta * kl : 0.0) - ra);
  s.v[1] -= w * ra;
  s.v[2] += w * kl;
  s.v[3] += cut ? w : 0.0;
  return grad * w * a.grad_scale;
}

// Sums over a workgroup of NT threads in a fixed order; every thread gets them.
template <int NT>
__device__ __forceinline__ void block_sum4(PolicySums& s, double (*tmp)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s.v[k] += __shfl_xor(s.v[k], off);
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6][k] = s.v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    double x = 0.0;
    for (int w = 0; w < NT / 64; ++w) x += tmp[w][k];
    s.v[k] = x;
  }
}

// Counts the kept tokens of a wave's lanes (whole numbers: their order does not matter); all lanes of the wave come.
__device__ __forceinline__ void policy_count(bool on, int m, int* count) {
  const unsigned long long all = __ballot(on);
  if (__all(m == uniform(m))) {
    if ((threadIdx.x & 63) == 0 && all) atomicAdd(&count[m], __popcll(all));
  } else if (on) {
    atomicAdd(&count[m], 1);
  }
}

// The whole loss in one workgroup and launch, for few tokens and grouping arrays that fit LDS: five thousand tokens are
// launches and dependent loads, no work.
__global__ void __launch_bounds__(kPolicyThreads) policy_small_kernel(const PolicyArgs a) {
  __shared__ int cu[kLdsMembers + 1], cnt[kLdsMembers + 1], first[kLdsGroups + 1];
  __shared__ double mw[kLdsMembers], tmp[kPolicyThreads / 64][4];
  __shared__ int tot[1][kPlanThreads / 64];
  __shared__ int bad, groups;
  const int t = threadIdx.x;
  constexpr int kPer = kPolicySmall / kPolicyThreads;
  if (a.ng == 0) {  // nothing, and perhaps no arrays either
    if (t < 4) a.stats[t] = 0.f;
    if (t == 0) a.hdr->error = 0;
    return;
  }
  const int size = t < a.ng ? a.gsz[t] : 0;
  // the tokens are on their way while the grouping arrays are looked over
  float lp[kPer], old[kPer], ref[kPer];
  bool on[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t + k * kPolicyThreads;
    on[k] = i < a.ts && (!a.mask || a.mask[i]);
    lp[k] = i < a.ts ? a.logp[i] : 0.f;
    old[k] = i < a.ts && a.logp_old ? a.logp_old[i] : 0.f;
    ref[k] = i < a.ts && a.logp_ref ? a.logp_ref[i] : 0.f;
  }
  for (int m = t; m <= a.ns; m += kPolicyThreads) {
    cu[m] = a.cu_s[m];
    cnt[m] = 0;
  }
  if (t == 0) {
    bad = 0;
    groups = 0;
  }
  __syncthreads();
  int b = size < 0 || size > a.ns;
  for (int m = t; m <= a.ns; m += kPolicyThreads) {
    const int v = cu[m];
    if ((m == 0 && v != 0) || (m == a.ns && v != a.ts) || (m > 0 && v < cu[m - 1])) b = 1;
  }
  int start[1] = {b ? 0 : size};
  const int members = start[0];
  if (members > 0) atomicAdd(&groups, 1);
  block_exclusive_sums(start, a.ng, tot);  // fits 32 bits: at most kLdsGroups sizes of at most kLdsMembers
  if (t <= a.ng && ((t == a.ng && start[0] != a.ns) || start[0] + members > a.ns)) b = 1;
  if (b) atomicOr(&bad, 1);
  __syncthreads();
  if (t == 0) a.hdr->error = bad;
  if (bad) return;
  if (t <= a.ng) first[t] = start[0];
  __syncthreads();
  for (int m = t; m < a.ns; m += kPolicyThreads) {
    const int g = upper_index(first, 0, a.ng, m);  // of groups that start alike, the last has the members
    mw[m] = (double)groups * (double)(first[g + 1] - first[g]);
  }
  int mem[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t + k * kPolicyThreads;
    mem[k] = i < a.ts ? upper_index(cu, 0, a.ns, i) : 0;
    if (a.mask && i - (t & 63) < a.ts) policy_count(on[k], a.by_token ? a.ns : mem[k], cnt);  // whole waves
  }
  if (!a.mask)
    for (int m = t; m <= a.ns; m += kPolicyThreads) cnt[m] = m < a.ns ? cu[m + 1] - cu[m] : a.ts;
  __syncthreads();
  for (int m = t; m < a.ns; m += kPolicyThreads) mw[m] = 1.0 / (a.by_token ? (double)cnt[a.ns] : mw[m] * cnt[m]);
  __syncthreads();
  PolicySums s{{0.0, 0.0, 0.0, 0.0}};
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = t + k * kPolicyThreads;
    if (i >= a.ts) break;
    double g = 0.0;
    if (on[k]) {
      g = policy_token(a, lp[k], old[k], ref[k], a.adv[mem[k]], mw[mem[k]], s);
    }
    if (a.dlogp) a.dlogp[i] = (float)g;
  }
  block_sum4<kPolicyThreads>(s, tmp);
  if (t == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k) a.stats[k] = (float)s.v[k];
}

// Otherwise three launches, four with a mask. Checks and per-member weights; one block.
__global__ void __launch_bounds__(kPolicyThreads) policy_plan_kernel(const PolicyArgs a) {
  __shared__ long long tmp[kPolicyThreads];
  __shared__ long long members;
  __shared__ int first[kPolicyThreads + 1];
  __shared__ int bad, groups;
  const int t = threadIdx.x;
  if (t == 0) {
    members = 0;
    bad = 0;
    groups = 0;
  }
  __syncthreads();
  int b = 0;
  for (int m = t; m <= a.ns; m += kPolicyThreads) {
    const int v = a.cu_s[m], before = m > 0 ? a.cu_s[m - 1] : 0;
    if ((m == 0 && v != 0) || (m == a.ns && v != a.ts) || v < before) b = 1;
    if (a.mask) a.count[m] = 0;
    else if (m > 0) a.count[m - 1] = v - before;
  }
  if (t == 0 && !a.mask) a.count[a.ns] = a.ts;
  int full = 0;
  for (int g = t; g < a.ng; g += kPolicyThreads) {
    const int v = a.gsz[g];
    if (v < 0 || v > a.ns) b = 1;
    full += v > 0;
  }
  if (b) atomicOr(&bad, 1);
  if (full) atomicAdd(&groups, full);
  __syncthreads();
  for (int base = 0; base < a.ng && !bad; base += kPolicyThreads) {
    const int g = base + t;
    const long long v = g < a.ng ? a.gsz[g] : 0;
    const long long from = members, end = from + block_inclusive_scan<kPolicyThreads>(v, tmp);
    // first member of each group of these, past the last member where sizes add up to more
    first[t] = (int)min(end - v, (long long)a.ns);
    if (t == kPolicyThreads - 1) {
      first[kPolicyThreads] = (int)min(end, (long long)a.ns);
      members = end;
    }
    __syncthreads();
    for (int m = (int)min(from, (long long)a.ns) + t; m < first[kPolicyThreads]; m += kPolicyThreads) {
      // of groups that start alike, the last has the members
      const int k = upper_index(first, 0, min(kPolicyThreads, a.ng - base), m);
      a.member_w[m] = 1.0 / ((double)groups * (double)(first[k + 1] - first[k]));
    }
    __syncthreads();
  }
  if (t == 0) {
    a.hdr->error = bad || members != a.ns;
  }
}

// The member of token i, whose workgroup's tokens lie in members m0 .. m1.
__device__ __forceinline__ int policy_member(const PolicyArgs& a, int m0, int m1, int i) {
  return upper_index(a.cu_s, m0, m1 + 1, i);
}

// Kept tokens of each member, or of all. One atomic a wave where its lanes are in one member: an atomic for each wave
// of 64 tokens on one counter was 52 of 94 us at 266k tokens.
__global__ void __launch_bounds__(kPolicyTok) policy_count_kernel(const PolicyArgs a) {
  __shared__ int sum;
  if (a.hdr->error) return;
  const int t = threadIdx.x;
  const long first = (long)blockIdx.x * kPolicyTok * kPolicyPer;
  const int last = (int)min((long)a.ts, first + kPolicyTok * kPolicyPer) - 1;
  if (a.by_token) {
    if (t == 0) sum = 0;
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int k = 0; k < kPolicyPer; ++k) {
      const long i = first + t + k * kPolicyTok;
      n += __popcll(__ballot(i <= last && a.mask[i]));
    }
    if ((t & 63) == 0) atomicAdd(&sum, n);
    __syncthreads();
    if (t == 0) atomicAdd(&a.count[a.ns], sum);
    return;
  }
  const int m0 = wave_upper_index(a.cu_s, a.ns, (int)first), m1 = wave_upper_index(a.cu_s, a.ns, last);
  if (m0 == m1) {
    if (t == 0) sum = 0;
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int k = 0; k < kPolicyPer; ++k) {
      const long i = first + t + k * kPolicyTok;
      n += __popcll(__ballot(i <= last && a.mask[i]));
    }
    if ((t & 63) == 0) atomicAdd(&sum, n);
    __syncthreads();
    if (t == 0) atomicAdd(&a.count[m0], sum);
    return;
  }
#pragma unroll
  for (int k = 0; k < kPolicyPer; ++k) {
    const long i = first + t + k * kPolicyTok;
    policy_count(i <= last && a.mask[i], policy_member(a, m0, m1, (int)min(i, (long)last)), a.count);
  }
}

// Terms, gradients and each workgroup's sums.
__global__ void __launch_bounds__(kPolicyTok) policy_loss_kernel(const PolicyArgs a) {
  __shared__ double tmp[kPolicyTok / 64][4];
  const int t = threadIdx.x;
  const long first = (long)blockIdx.x * kPolicyTok * kPolicyPer;
  const int last = (int)min((long)a.ts, first + kPolicyTok * kPolicyPer) - 1;
  PolicySums s{{0.0, 0.0, 0.0, 0.0}};
  if (first <= last) {
    float lp[kPolicyPer], old[kPolicyPer], ref[kPolicyPer];
    bool on[kPolicyPer];
#pragma unroll
    for (int k = 0; k < kPolicyPer; ++k) {
      const long i = min(first + t + k * kPolicyTok, (long)last);
      on[k] = first + t + k * kPolicyTok <= last && (!a.mask || a.mask[i]);
      lp[k] = a.logp[i];
      old[k] = a.logp_old ? a.logp_old[i] : 0.f;
      ref[k] = a.logp_ref ? a.logp_ref[i] : 0.f;
    }
    const int m0 = wave_upper_index(a.cu_s, a.ns, (int)first), m1 = wave_upper_index(a.cu_s, a.ns, last);
    if (a.hdr->error) return;  // whole workgroups; what is above stays in bounds whatever the arrays hold
    auto weight = [&](int m) { return a.by_token ? 1.0 / a.count[a.ns] : a.member_w[m] / a.count[m]; };
    const bool one = m0 == m1 || a.by_token;  // one weight for all
    const double w0 = one ? weight(m0) : 0.0;
#pragma unroll
    for (int k = 0; k < kPolicyPer; ++k) {
      const long i = first + t + k * kPolicyTok;
      double g = 0.0;
      if (on[k]) {
        const int m = policy_member(a, m0, m1, (int)i);
        g = policy_token(a, lp[k], old[k], ref[k], a.adv[m], one ? w0 : weight(m), s);
      }
      if (a.dlogp && i <= last) a.dlogp[i] = (float)g;
    }
  }
  if (a.hdr->error) return;
  block_sum4<kPolicyTok>(s, tmp);
  if (t == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k) a.part[4 * (size_t)blockIdx.x + k] = s.v[k];
}

// The workgroups' sums, in their order. A launch of its own: that the last workgroup of the kernel above adds them up
// would need each to flush its XCD's L2 (266k tokens: 18 and 25 us with 260 and 521 workgroups, 12 us without).
__global__ void __launch_bounds__(kPolicyTok) policy_sum_kernel(const PolicyArgs a, int blocks) {
  __shared__ double tmp[kPolicyTok / 64][4];
  if (a.hdr->error) return;
  PolicySums s{{0.0, 0.0, 0.0, 0.0}};
  for (int b = threadIdx.x; b < blocks; b += kPolicyTok)
#pragma unroll
    for (int k = 0; k < 4; ++k) s.v[k] += a.part[4 * (size_t)b + k];
  block_sum4<kPolicyTok>(s, tmp);
  if (threadIdx.x == 0)
#pragma unroll
    for (int k = 0; k < 4; ++k) a.stats[k] = (float)s.v[k];
}

}  // namespace pg
