// Entry points of linear attention (included by pg_attn.hip): argument checks, workspace layout, launches.
#pragma once

namespace {

// Rows an item holds. Long items save traffic (each costs a state written, scanned and read: 16 D^2 bytes a kv head),
// short ones give more workgroups.
int linear_item_rows(int tp, int ts, int heads) {
  const long rows = (long)tp + ts;
  int L = 2048;
  while (L > 128 && rows * heads < 1024L * L) L /= 2;
  return L;
}

struct LinearLayout {
  size_t hdr, ginfo, qoff, kvoff, seg_off, items, slots, total;
  int L, max_items;
};

// Items of one walk: a segment of r rows has ceil(r / L).
long linear_max_items(int ng, int ns, int tp, int ts, int L) {
  return (long)tp / L + ng + (long)ts / L + ns;
}

LinearLayout linear_layout(int ng, int ns, int tp, int ts, int heads, int h_kv, int d) {
  LinearLayout L{};
  L.L = linear_item_rows(tp, ts, heads);
  const long items = linear_max_items(ng, ns, tp, ts, L.L);
  L.max_items = items > INT32_MAX ? -1 : (int)items;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  L.hdr = take(sizeof(pg::PlanHeader));
  L.ginfo = take(sizeof(pg::GroupInfoEx) * (size_t)(ng > 0 ? ng : 1));
  L.qoff = take(sizeof(int) * ((size_t)ng + 1));
  L.kvoff = take(sizeof(int) * ((size_t)ng + 1));
  L.seg_off = take(sizeof(int) * ((size_t)ng + ns + 1));
  L.items = take(sizeof(pg::LinItem) * (size_t)items);
  L.slots = take(sizeof(float) * (size_t)(items + ng) * h_kv * d * d);
  L.total = off;
  return L;
}

LinearLayout linear_fwd_layout(const Common& c) { return linear_layout(c.ng, c.ns, c.tp, c.ts, c.h_q, c.h_kv, c.d); }
LinearLayout linear_bwd_layout(const Common& c) { return linear_layout(c.ng, c.ns, c.tp, c.ts, c.h_kv, c.h_kv, c.d); }

// One walk's plan, item shares and scans.
template <typename T, int D, bool REV, int SPLIT>
int linear_states(const Common& c, const LinearLayout& L, char* ws, const int32_t* cu_p, const int32_t* cu_s,
                  const pg::LinArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(pg::lin_items_kernel, dim3(1), dim3(pg::kPlanThreads), 0, st, cu_p, cu_s, c.ng, c.ns, L.L,
                     L.max_items, REV ? 1 : 0, (pg::PlanHeader*)(ws + L.hdr), a.ginfo, (int*)(ws + L.seg_off),
                     (pg::LinItem*)(ws + L.items));
  const long blocks = pg::xcd_grid_blocks(L.max_items, c.h_kv, 1);
  hipLaunchKernelGGL((pg::lin_state_kernel<T, D, REV, SPLIT>), dim3((unsigned)blocks),
                     dim3(pg::kLinThreads), 0, st, a);
  for (int i = 0; i < 2; ++i) {
    const int part = REV ? 1 - i : i, segs = part ? c.ns : c.ng;
    if (segs > 0)
      hipLaunchKernelGGL((pg::lin_scan_kernel<D, REV>), dim3(D * D / 1024, c.h_kv, std::min(segs, 65535)),
                         dim3(pg::kScanThreads), 0, st, a, part);
  }
  return PG_OK;
}

template <typename T, int D, int SPLIT>
void linear_out(const Common& c, const LinearLayout& L, const pg::LinArgs& a, hipStream_t st) {
  const long blocks = pg::xcd_grid_blocks(L.max_items, c.h_q, c.h_q / c.h_kv);
  hipLaunchKernelGGL((pg::lin_out_kernel<T, D, SPLIT>), dim3((unsigned)blocks), dim3(pg::kLinThreads), 0, st,
                     a);
}

void linear_common_args(pg::LinArgs& a, const Common& c, const LinearLayout& L, char* ws, const float* log_decay) {
  a.log_decay = log_decay;
  a.slots = (float*)(ws + L.slots);
  a.seg_off = (const int*)(ws + L.seg_off);
  a.items = (const pg::LinItem*)(ws + L.items);
  a.hdr = (const pg::PlanHeader*)(ws + L.hdr);
  a.ginfo = (const pg::GroupInfoEx*)(ws + L.ginfo);
  a.ng = c.ng; a.ns = c.ns; a.h_q = c.h_q; a.h_kv = c.h_kv; a.max_items = L.max_items;
  a.scale = c.scale;
}

template <typename T, int D>
int linear_fwd_typed(const Common& c, const LinearLayout& L, char* ws, const int32_t* cu_p, const int32_t* cu_s,
                     const pg::LinArgs& a, hipStream_t st) {
  constexpr bool b16 = sizeof(T) == 2;
  const bool states = a.state_out[0] || a.state_out[1];
  {
    Timed tm(PG_K_LINEAR_STATE, st);
    if (states) linear_states<T, D, false, b16 ? 3 : 1>(c, L, ws, cu_p, cu_s, a, st);
    else linear_states<T, D, false, b16 ? 2 : 1>(c, L, ws, cu_p, cu_s, a, st);
  }
  Timed tm(PG_K_LINEAR_OUT, st);
  if (states) linear_out<T, D, b16 ? 3 : 1>(c, L, a, st);
  else linear_out<T, D, b16 ? 2 : 1>(c, L, a, st);
  return PG_OK;
}

template <typename T, int D>
int linear_bwd_typed(const Common& c, const LinearLayout& F, const LinearLayout& B, char* ws, const int32_t* cu_p,
                     const int32_t* cu_s, const pg::LinArgs& dq, const pg::LinArgs& g, hipStream_t st) {
  constexpr int SPLIT = sizeof(T) == 2 ? 2 : 1;
  {
    Timed tm(PG_K_LINEAR_STATE, st);
    linear_states<T, D, false, SPLIT>(c, F, ws, cu_p, cu_s, dq, st);
  }
  {
    Timed tm(PG_K_LINEAR_OUT, st);
    linear_out<T, D, SPLIT>(c, F, dq, st);
  }
  {
    Timed tm(PG_K_LINEAR_STATE, st);
    linear_states<T, D, true, SPLIT>(c, B, ws, cu_p, cu_s, g, st);
  }
  Timed tm(PG_K_LINEAR_GRAD, st);
  const long blocks = pg::xcd_grid_blocks(B.max_items, c.h_kv, 1);
  hipLaunchKernelGGL((pg::lin_grad_kernel<T, D, SPLIT>), dim3((unsigned)blocks), dim3(pg::kLinThreads), 0, st,
                     g);
  return PG_OK;
}

int linear_grid_check(const Common& c, const LinearLayout& L) {
  // workgroups of 256 threads, fewer than 2^32 threads a launch; item and slot numbers in 31 bits
  if (L.max_items < 0 || (long)L.max_items + c.ng > INT32_MAX || ((long)L.max_items + 8) * c.h_q * 256 > 0xffffffffL ||
      c.h_kv > 65535)
    return fail(PG_EUNSUPPORTED, "%d groups, %d members x %d heads exceed the launch grid", c.ng, c.ns, c.h_q);
  return PG_OK;
}

int plan_groups(const Common& c, char* ws, size_t hdr, size_t ginfo, size_t qoff, size_t kvoff, const int32_t* cu_p,
                const int32_t* cu_s, const int32_t* gsz, hipStream_t st) {
  Timed tp(PG_K_PLAN, st);
  return launch_rope_plan(RopeLayout{hdr, ginfo, qoff, kvoff, 0}, ws, c.ng, c.ns, c.tp, c.ts, cu_p, cu_s, gsz, st);
}

bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned16(p)) return true;
  return false;
}

}  // namespace

extern "C" {

size_t pg_linear_fwd_workspace_size(int n_groups, int n_suffixes, int total_prefix, int total_suffix, int h_q,
                                    int h_kv, int head_dim) {
  if (n_groups < 0 || n_suffixes < 0 || total_prefix < 0 || total_suffix < 0 || h_q < 0 || h_kv < 0 || head_dim < 0)
    return 0;
  return linear_layout(n_groups, n_suffixes, total_prefix, total_suffix, h_q, h_kv, head_dim).total;
}

size_t pg_linear_bwd_workspace_size(int n_groups, int n_suffixes, int total_prefix, int total_suffix, int h_q,
                                    int h_kv, int head_dim) {
  if (n_groups < 0 || n_suffixes < 0 || total_prefix < 0 || total_suffix < 0 || h_q < 0 || h_kv < 0 || head_dim < 0)
    return 0;
  return std::max(linear_layout(n_groups, n_suffixes, total_prefix, total_suffix, h_q, h_kv, head_dim).total,
                  linear_layout(n_groups, n_suffixes, total_prefix, total_suffix, h_kv, h_kv, head_dim).total);
}

int pg_linear_fwd(int dtype, int n_groups, int n_suffixes, int total_prefix, int total_suffix,
                  const int32_t* cu_prefix_lens, const int32_t* cu_suffix_lens, const int32_t* group_sizes, int h_q,
                  int h_kv, int head_dim, float scale, const float* log_decay, const void* q_pre, const void* k_pre,
                  const void* v_pre, const void* q_suf, const void* k_suf, const void* v_suf, const float* state_in,
                  void* o_pre, void* o_suf, float* state_pre, float* state_suf, void* workspace,
                  size_t workspace_bytes, void* stream) {
  g_last_error.clear();
  const Common c{dtype, n_groups, n_suffixes, total_prefix, total_suffix, h_q, h_kv, head_dim, scale};
  int rc = check_common(c, cu_prefix_lens, cu_suffix_lens, group_sizes);
  if (rc) return rc;
  if (!log_decay) return fail(PG_EINVAL, "log_decay is NULL");
  if (total_prefix > 0 && (!q_pre || !k_pre || !v_pre || !o_pre)) return fail(PG_EINVAL, "a prefix tensor pointer is NULL");
  if (total_suffix > 0 && (!q_suf || !k_suf || !v_suf || !o_suf)) return fail(PG_EINVAL, "a suffix tensor pointer is NULL");
  if (misaligned({q_pre, k_pre, v_pre, q_suf, k_suf, v_suf, state_in, o_pre, o_suf, state_pre, state_suf, workspace}))
    return fail(PG_EINVAL, "tensor pointers must be 16-byte aligned");
  const LinearLayout L = linear_fwd_layout(c);
  if ((rc = linear_grid_check(c, L))) return rc;
  if (!workspace || workspace_bytes < L.total)
    return fail(PG_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, L.total);
  if ((rc = device_ready())) return rc;
  if (c.ng == 0) return PG_OK;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  if ((rc = plan_groups(c, ws, L.hdr, L.ginfo, L.qoff, L.kvoff, cu_prefix_lens, cu_suffix_lens, group_sizes, st)))
    return rc;
  pg::LinArgs a{};
  linear_common_args(a, c, L, ws, log_decay);
  a.q[0] = q_pre; a.k[0] = k_pre; a.v[0] = v_pre; a.q[1] = q_suf; a.k[1] = k_suf; a.v[1] = v_suf;
  a.out[0] = o_pre; a.out[1] = o_suf;
  a.state_in = state_in;
  a.state_out[0] = state_pre; a.state_out[1] = state_suf;
  if (dtype == PG_BF16)
    rc = head_dim == 128 ? linear_fwd_typed<pg::bf16, 128>(c, L, ws, cu_prefix_lens, cu_suffix_lens, a, st)
                         : linear_fwd_typed<pg::bf16, 64>(c, L, ws, cu_prefix_lens, cu_suffix_lens, a, st);
  else
    rc = head_dim == 128 ? linear_fwd_typed<float, 128>(c, L, ws, cu_prefix_lens, cu_suffix_lens, a, st)
                         : linear_fwd_typed<float, 64>(c, L, ws, cu_prefix_lens, cu_suffix_lens, a, st);
  if (rc) return rc;
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "linear attention forward launch");
  return PG_OK;
}

int pg_linear_bwd(int dtype, int n_groups, int n_suffixes, int total_prefix, int total_suffix,
                  const int32_t* cu_prefix_lens, const int32_t* cu_suffix_lens, const int32_t* group_sizes, int h_q,
                  int h_kv, int head_dim, float scale, const float* log_decay, const void* q_pre, const void* k_pre,
                  const void* v_pre, const void* q_suf, const void* k_suf, const void* v_suf, const void* do_pre,
                  const void* do_suf, void* dq_pre, void* dk_pre, void* dv_pre, void* dq_suf, void* dk_suf,
                  void* dv_suf, void* workspace, size_t workspace_bytes, void* stream) {
  g_last_error.clear();
  const Common c{dtype, n_groups, n_suffixes, total_prefix, total_suffix, h_q, h_kv, head_dim, scale};
  int rc = check_common(c, cu_prefix_lens, cu_suffix_lens, group_sizes);
  if (rc) return rc;
  if (!log_decay) return fail(PG_EINVAL, "log_decay is NULL");
  if (total_prefix > 0 && (!q_pre || !k_pre || !v_pre || !do_pre || !dq_pre || !dk_pre || !dv_pre))
    return fail(PG_EINVAL, "a prefix tensor pointer is NULL");
  if (total_suffix > 0 && (!q_suf || !k_suf || !v_suf || !do_suf || !dq_suf || !dk_suf || !dv_suf))
    return fail(PG_EINVAL, "a suffix tensor pointer is NULL");
  if (misaligned({q_pre, k_pre, v_pre, q_suf, k_suf, v_suf, do_pre, do_suf, dq_pre, dk_pre, dv_pre, dq_suf, dk_suf,
                  dv_suf, workspace}))
    return fail(PG_EINVAL, "tensor pointers must be 16-byte aligned");
  const LinearLayout F = linear_fwd_layout(c), B = linear_bwd_layout(c);
  if ((rc = linear_grid_check(c, F)) || (rc = linear_grid_check(c, B))) return rc;
  const size_t need = std::max(F.total, B.total);
  if (!workspace || workspace_bytes < need)
    return fail(PG_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, need);
  if ((rc = device_ready())) return rc;
  if (c.ng == 0) return PG_OK;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  if ((rc = plan_groups(c, ws, F.hdr, F.ginfo, F.qoff, F.kvoff, cu_prefix_lens, cu_suffix_lens, group_sizes, st)))
    return rc;
  // dq_t = c sum l^(t-s) (do_t . v_s) k_s: the forward walk with do, v, k in the places of q, k, v
  pg::LinArgs dq{}, g{};
  linear_common_args(dq, c, F, ws, log_decay);
  dq.q[0] = do_pre; dq.k[0] = v_pre; dq.v[0] = k_pre; dq.q[1] = do_suf; dq.k[1] = v_suf; dq.v[1] = k_suf;
  dq.out[0] = dq_pre; dq.out[1] = dq_suf;
  linear_common_args(g, c, B, ws, log_decay);
  g.q[0] = q_pre; g.k[0] = k_pre; g.v[0] = v_pre; g.q[1] = q_suf; g.k[1] = k_suf; g.v[1] = v_suf;
  g.d_o[0] = do_pre; g.d_o[1] = do_suf;
  g.dk[0] = dk_pre; g.dk[1] = dk_suf; g.dv[0] = dv_pre; g.dv[1] = dv_suf;
  if (dtype == PG_BF16)
    rc = head_dim == 128 ? linear_bwd_typed<pg::bf16, 128>(c, F, B, ws, cu_prefix_lens, cu_suffix_lens, dq, g, st)
                         : linear_bwd_typed<pg::bf16, 64>(c, F, B, ws, cu_prefix_lens, cu_suffix_lens, dq, g, st);
  else
    rc = head_dim == 128 ? linear_bwd_typed<float, 128>(c, F, B, ws, cu_prefix_lens, cu_suffix_lens, dq, g, st)
                         : linear_bwd_typed<float, 64>(c, F, B, ws, cu_prefix_lens, cu_suffix_lens, dq, g, st);
  if (rc) return rc;
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "linear attention backward launch");
  return PG_OK;
}

int pg_linear_step(int dtype, int n, int h_q, int h_kv, int head_dim, float scale, const float* log_decay,
                   const void* q, const void* k, const void* v, const float* state, void* o, float* state_out,
                   void* stream) {
  g_last_error.clear();
  if (dtype != PG_BF16 && dtype != PG_FP32) return fail(PG_EUNSUPPORTED, "dtype %d is not PG_BF16 or PG_FP32", dtype);
  if (n < 0) return fail(PG_EINVAL, "negative number of sequences %d", n);
  if (h_q <= 0 || h_kv <= 0 || h_q % h_kv != 0)
    return fail(PG_EINVAL, "h_q=%d must be a positive multiple of h_kv=%d", h_q, h_kv);
  if (head_dim != 64 && head_dim != 128) return fail(PG_EUNSUPPORTED, "head_dim=%d (supported: 64, 128)", head_dim);
  if (!(std::isfinite(scale) && scale > 0.f)) return fail(PG_EINVAL, "scale must be finite and > 0");
  if (!log_decay || (n > 0 && (!q || !k || !v || !state || !o || !state_out)))
    return fail(PG_EINVAL, "a tensor pointer is NULL");
  if (misaligned({q, k, v, state, o, state_out})) return fail(PG_EINVAL, "tensor pointers must be 16-byte aligned");
  int rc = device_ready();
  if (rc || n == 0) return rc;
  pg::LinStepArgs a{q, k, v, log_decay, state, o, state_out, n, h_q, h_kv, scale};
  hipStream_t st = (hipStream_t)stream;
  Timed tm(PG_K_LINEAR_STEP, st);
  const long states = (long)n * h_kv;
  // few states: a state is spread over head_dim / 32 workgroups
  const bool wide = states >= 512;
  const int cols = wide ? head_dim : 32;
  const unsigned blocks = (unsigned)std::min(states * (head_dim / cols), 1L << 20);
#define PG_STEP(T, D, C) \
  hipLaunchKernelGGL((pg::lin_step_kernel<T, D, C>), dim3(blocks), dim3(pg::kStepThreads), 0, st, a)
  if (dtype == PG_BF16) {
    if (head_dim == 128) { if (wide) PG_STEP(pg::bf16, 128, 128); else PG_STEP(pg::bf16, 128, 32); }
    else { if (wide) PG_STEP(pg::bf16, 64, 64); else PG_STEP(pg::bf16, 64, 32); }
  } else {
    if (head_dim == 128) { if (wide) PG_STEP(float, 128, 128); else PG_STEP(float, 128, 32); }
    else { if (wide) PG_STEP(float, 64, 64); else PG_STEP(float, 64, 32); }
  }
#undef PG_STEP
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "linear attention step launch");
  return PG_OK;
}

}  // extern "C"
