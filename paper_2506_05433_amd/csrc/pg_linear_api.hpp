// Entry points of linear attention (included by pg_lib.hip, after the helpers of pg_attn.hip): argument checks, workspace layout, launches.
#pragma once

namespace {

// Rows an item of a prefix and of a member holds, of one walk with `heads` workgroups an item (query heads for
// outputs, kv heads for gradients). Every item but a segment's last costs a state written, scanned and read (16 D^2
// bytes a kv head) and its rows read once more; fewer items leave CUs idle.
struct ItemRows {
  int pre, suf;
  int hpw;  // query heads a workgroup of the output kernel takes
  bool members_first;
  bool alone;  // no states between workgroups: each walks the rows that its own start from as well
  int round;  // items that fill the CUs once, where they are ordered by length (pg_linear.hpp, item_place)
};

// Few rows are launches and latency: the states and scans are 3 of a call's 5 launches. Where one workgroup gets over the
// rows that its own start from faster than those kernels pass it the state, every segment is one item, and a member's
// workgroup walks its prefix first (a prefix's its members, backwards). Measured, us alone and in 32-row items, forward
// then backward: P 64, 4 x 24 rows, d 64, fp32 15, 22 and 23, 28, bf16 10, 17 and 15, 21; bf16 d 128 P 128, 4 x 16, 8/2
// heads 15, 19 and (dk, dv walk 192 rows x 4 heads) 54, 29; P 192 20, 20 and 81, 33; P 400 33, 22; fp32 d 128 P 128 36,
// 24.
constexpr int kAloneRows = 512;

bool linear_alone(int dtype, int tp, int ts, int ratio, int d, bool grad) {
  const long rows = (long)tp + ts;
  if (rows > kAloneRows) return false;
  return grad ? rows * ratio <= 384 : (long)tp * d <= (dtype == PG_BF16 ? 128 * 128 : 64 * 128);
}

ItemRows linear_item_rows(int ns, int tp, int ts, int h_q, int h_kv, int d, bool grad, bool alone) {
  ItemRows r{};
  const int ratio = h_kv > 0 ? h_q / h_kv : 1;
  const long rows = (long)tp + ts;
  r.hpw = 1;
  if (alone) {
    r.pre = r.suf = kAloneRows + 1;  // no segment is longer: no more items than segments
    r.alone = true;
    return r;
  }
  // output workgroups take all query heads of a kv head (or a divisor of their number) while there are 512 of them
  // with 64-row items, one for each member at least: they share the state's updates, keys and values. P 4096, 8 x
  // 256..1024 rows, 32/8 heads: 1, 2 and 4 heads 79, 57 and 52 us; 8100 rows, 16/4 heads, d 64: 25, 22 and 18; P 1024,
  // 256 x 1 row, 32/8 heads, the whole forward with 1 and 4: 115 and 77
  if (!grad)
    for (int n = 1; n <= ratio; ++n)
      if (ratio % n == 0 && std::max(rows, 64L * ns) * h_kv * (ratio / n) >= 512L * 64) r.hpw = n;
  const int heads = grad ? h_kv : h_q / r.hpw;
  // members: whole where there are enough of them (up to twice the mean length: a longer one is split), else about 512
  // workgroups in all; a chunk at least
  const int least = d == 128 ? 32 : 64;
  const bool many = (long)ns * heads >= 512;
  r.suf = 1024;
  if (many)
    while (r.suf < 65536 && (long)r.suf * ns < 2L * ts) r.suf *= 2;
  else
    while (r.suf > least && rows * heads < 512L * r.suf) r.suf /= 2;
  // prefixes: enough items to fill the CUs with the state kernel's workgroups (one a kv head; half the CUs where they
  // only read keys and values) and, with the members, with the output kernel's. P 16384 of 8 kv heads, 256, 512 and
  // 1024 rows: forward state and output 29 + 111, 27 + 110, 38 + 187 us, backward 99 + 152, 81 + 157, 112 + 257;
  // P 4096, 128, 256 and 512: 19 + 52, 16 + 49, 21 + 78; P 400 of 2, a whole backward with 32, 64, 128 and 256: 47, 55,
  // 77 and 123
  const long groups = many ? (long)ns * heads : (long)ts / r.suf * heads;
  r.pre = 1024;
  while (r.pre > least && ((long)tp * h_kv < (grad ? 256L : 128L) * r.pre || (long)tp / r.pre * heads + groups < 400)) r.pre /= 2;
  r.members_first = many;
  r.round = many ? (int)ceil_div_l(256, heads) : 0;
  return r;
}

struct LinearLayout {
  struct List {
    ItemRows rows;
    int max_items;
    size_t seg_off, items, slots;
  };
  size_t hdr, ginfo, qoff, kvoff, total;
  List out, grad;  // the forward walk (outputs, or dq); the backward one (dk, dv)
};

// dtype: PG_BF16 or PG_FP32, or -1 for a layout that serves both, and a call that returns states (which the scans write
// for segments without rows); it is the largest.
LinearLayout linear_layout(int dtype, int ng, int ns, int tp, int ts, int h_q, int h_kv, int d, bool bwd) {
  LinearLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  L.hdr = take(sizeof(pg::PlanHeader));
  L.ginfo = take(sizeof(pg::GroupInfoEx) * (size_t)(ng > 0 ? ng : 1));
  L.qoff = take(sizeof(int) * ((size_t)ng + 1));
  L.kvoff = take(sizeof(int) * ((size_t)ng + 1));
  auto list = [&](LinearLayout::List& l, bool grad) {
    const bool alone = dtype >= 0 && linear_alone(dtype, tp, ts, h_q / h_kv, d, grad);
    l.rows = linear_item_rows(ns, tp, ts, h_q, h_kv, d, grad, alone);
    // a segment of r rows has ceil(r / rows of an item) items
    const long items = (long)tp / l.rows.pre + ng + (long)ts / l.rows.suf + ns;
    l.max_items = items > INT32_MAX ? -1 : (int)items;
    l.seg_off = take(sizeof(int) * ((size_t)ng + ns + 1));
    l.items = take(sizeof(pg::LinItem) * (size_t)items);
    l.slots = take(sizeof(float) * (size_t)(items + ng) * h_kv * d * d);
  };
  list(L.out, false);
  if (bwd) list(L.grad, true);
  L.total = off;
  return L;
}

// Groups and items of the call's walks.
int linear_plan(const Common& c, const LinearLayout& L, char* ws, const int32_t* cu_p, const int32_t* cu_s,
                const int32_t* gsz, bool bwd, hipStream_t st) {
  Timed tm(PG_K_PLAN, st);
  auto* hdr = (pg::PlanHeader*)(ws + L.hdr);
  auto* gi = (pg::GroupInfoEx*)(ws + L.ginfo);
  auto list = [&](const LinearLayout::List& l, bool grad) {
    return pg::LinList{(int*)(ws + l.seg_off), (pg::LinItem*)(ws + l.items), grad ? &hdr->n_kvtiles : &hdr->n_qtiles,
                       l.rows.pre, l.rows.suf, l.max_items, grad ? 1 : 0, l.rows.round};
  };
  const pg::LinList out = list(L.out, false), grad = bwd ? list(L.grad, true) : out;
  if (pg::plan_fits_lds(c.ng, c.ns) && !plan_multi()) {
    hipLaunchKernelGGL(pg::lin_plan_kernel, dim3(1), dim3(pg::kPlanThreads), 0, st, cu_p, cu_s, gsz, c.ng, c.ns, c.tp,
                       c.ts, hdr, gi, (int*)(ws + L.qoff), (int*)(ws + L.kvoff), out, grad, bwd ? 2 : 1);
    return finish_plan(hdr, st);
  }
  int rc = launch_rope_plan(RopeLayout{L.hdr, L.ginfo, L.qoff, L.kvoff, 0}, ws, c.ng, c.ns, c.tp, c.ts, cu_p, cu_s, gsz,
                            st);
  if (rc) return rc;
  for (int i = 0; i < (bwd ? 2 : 1); ++i)
    hipLaunchKernelGGL(pg::lin_items_kernel, dim3(1), dim3(pg::kPlanThreads), 0, st, cu_p, cu_s, c.ng, c.ns,
                       i ? grad : out, hdr, gi);
  return PG_OK;
}

// States before the items of a forward walk and, in a backward call, of its reverse walk (either may be NULL): shares and
// scans of both side by side. The prefixes' scan of a members_first walk comes later.
template <typename T, int D, int SPLIT>
void linear_states(const Common& c, const pg::LinArgs* a, const pg::LinArgs* r, hipStream_t st) {
  if (!a && !r) return;
  Timed tm(PG_K_LINEAR_STATE, st);
  const pg::LinArgs &fa = a ? *a : *r, &fr = r ? *r : *a;
  auto blocks = [&](const pg::LinArgs* w) { return w ? (unsigned)pg::xcd_grid_blocks(w->max_items, c.h_kv, 1) : 0u; };
  hipLaunchKernelGGL((pg::lin_state_kernel<T, D, SPLIT>), dim3(blocks(a) + blocks(r)), dim3(pg::kLinStateThreads), 0, st,
                     fa, fr, blocks(r));
  const unsigned a1 = a ? pg::scan_blocks<D, 0>(*a) : 0, r1 = r ? pg::scan_blocks<D, 1>(*r) : 0;
  if (a1 + r1)
    hipLaunchKernelGGL((pg::lin_scan_kernel<D, false>), dim3(a1 + r1), dim3(pg::kScanThreads), 0, st, fa, fr, a1);
  const unsigned a2 = a ? pg::scan_blocks<D, 1>(*a) : 0, r2 = r && !r->members_first ? pg::scan_blocks<D, 0>(*r) : 0;
  if (a2 + r2)
    hipLaunchKernelGGL((pg::lin_scan_kernel<D, true>), dim3(a2 + r2), dim3(pg::kScanThreads), 0, st, fa, fr, a2);
}

unsigned linear_out_blocks(const Common& c, int hpw, const pg::LinArgs& a) {
  const int parts = c.h_q / c.h_kv / hpw;
  return (unsigned)pg::xcd_grid_blocks(a.max_items, c.h_kv * parts, parts);
}

template <typename T, int D, int SPLIT>
void linear_outputs(const Common& c, int hpw, const pg::LinArgs& a, hipStream_t st) {
  Timed tm(PG_K_LINEAR_OUT, st);
  hipLaunchKernelGGL((pg::lin_out_kernel<T, D, SPLIT>), dim3(linear_out_blocks(c, hpw, a)), dim3(pg::kLinThreads), 0, st,
                     a, hpw);
}

void linear_common_args(pg::LinArgs& a, const Common& c, const LinearLayout& L, bool grad, char* ws,
                        const float* log_decay, const int32_t* cu_p, const int32_t* cu_s) {
  const LinearLayout::List& l = grad ? L.grad : L.out;
  a.log_decay = log_decay;
  a.cu_p = cu_p; a.cu_s = cu_s;
  a.slots = (float*)(ws + l.slots);
  a.seg_off = (const int*)(ws + l.seg_off);
  a.items = (const pg::LinItem*)(ws + l.items);
  a.hdr = (const pg::PlanHeader*)(ws + L.hdr);
  a.n_items = grad ? &a.hdr->n_kvtiles : &a.hdr->n_qtiles;
  a.ginfo = (const pg::GroupInfoEx*)(ws + L.ginfo);
  a.ng = c.ng; a.ns = c.ns; a.h_q = c.h_q; a.h_kv = c.h_kv; a.max_items = l.max_items;
  a.l_pre = l.rows.pre; a.l_suf = l.rows.suf;
  a.members_first = l.rows.members_first;
  a.alone = l.rows.alone;
  a.scale = c.scale;
}

template <typename T, int D, int SPLIT>
void linear_walk(const Common& c, int hpw, const pg::LinArgs& a, hipStream_t st) {
  linear_states<T, D, SPLIT>(c, a.alone ? nullptr : &a, nullptr, st);
  linear_outputs<T, D, SPLIT>(c, hpw, a, st);
}

template <typename T, int D>
void linear_fwd_typed(const Common& c, int hpw, const pg::LinArgs& a, hipStream_t st) {
  constexpr bool b16 = sizeof(T) == 2;
  if (a.state_out[0] || a.state_out[1]) linear_walk<T, D, b16 ? 3 : 1>(c, hpw, a, st);
  else linear_walk<T, D, b16 ? 2 : 1>(c, hpw, a, st);
}

template <typename T, int D>
void linear_bwd_typed(const Common& c, int hpw, const pg::LinArgs& dq, const pg::LinArgs& g, hipStream_t st) {
  constexpr int SPLIT = sizeof(T) == 2 ? 2 : 1;
  linear_states<T, D, SPLIT>(c, dq.alone ? nullptr : &dq, g.alone ? nullptr : &g, st);
  const unsigned first = (unsigned)pg::xcd_grid_blocks(g.max_items, c.h_kv, 1);
  {
    Timed tm(PG_K_LINEAR_GRAD, st);
    hipLaunchKernelGGL((pg::lin_grads_kernel<T, D, SPLIT>), dim3(first + linear_out_blocks(c, hpw, dq)),
                       dim3(pg::kLinThreads), 0, st, dq, hpw, g, first, g.members_first ? 1 : -1);
  }
  if (!g.members_first) return;
  // the members' walks have ended with the states that the prefixes' start from: no pass over the responses for them alone
  {
    Timed tm(PG_K_LINEAR_STATE, st);
    hipLaunchKernelGGL((pg::lin_scan_kernel<D, true>), dim3(pg::scan_blocks<D, 0>(g)), dim3(pg::kScanThreads), 0, st, g, g,
                       0u);
  }
  Timed tm(PG_K_LINEAR_GRAD, st);
  hipLaunchKernelGGL((pg::lin_grad_kernel<T, D, SPLIT>), dim3(first), dim3(pg::kLinThreads), 0, st, g, 0);
}

// items: of all walks of the call
int linear_grid_check(const Common& c, long items) {
  // workgroups of 256 threads, fewer than 2^32 threads a launch; item and slot numbers in 31 bits
  if (items < 0 || items + c.ng > INT32_MAX || (items + 16) * c.h_q * 256 > 0xffffffffL)
    return fail(PG_EUNSUPPORTED, "%d groups, %d members x %d heads exceed the launch grid", c.ng, c.ns, c.h_q);
  return PG_OK;
}

bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned16(p)) return true;
  return false;
}

bool overlap(const void* p, const void* q, size_t p_bytes, size_t q_bytes) {
  return p && q && (uintptr_t)p < (uintptr_t)q + q_bytes && (uintptr_t)q < (uintptr_t)p + p_bytes;
}

}  // namespace

extern "C" {

size_t pg_linear_fwd_workspace_size(int n_groups, int n_suffixes, int total_prefix, int total_suffix, int h_q,
                                    int h_kv, int head_dim) {
  if (n_groups < 0 || n_suffixes < 0 || total_prefix < 0 || total_suffix < 0 || h_q < 0 || h_kv < 0 || head_dim < 0)
    return 0;
  return linear_layout(-1, n_groups, n_suffixes, total_prefix, total_suffix, h_q, h_kv, head_dim, false).total;
}

size_t pg_linear_bwd_workspace_size(int n_groups, int n_suffixes, int total_prefix, int total_suffix, int h_q,
                                    int h_kv, int head_dim) {
  if (n_groups < 0 || n_suffixes < 0 || total_prefix < 0 || total_suffix < 0 || h_q < 0 || h_kv < 0 || head_dim < 0)
    return 0;
  return linear_layout(-1, n_groups, n_suffixes, total_prefix, total_suffix, h_q, h_kv, head_dim, true).total;
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
  const size_t state = sizeof(float) * (size_t)h_kv * head_dim * head_dim, in = state * n_groups;
  if (overlap(state_in, state_pre, in, in) || overlap(state_in, state_suf, in, state * n_suffixes))
    return fail(PG_EINVAL, "state_in overlaps state_pre or state_suf");
  const LinearLayout L = linear_layout(state_pre || state_suf ? -1 : dtype, c.ng, c.ns, c.tp, c.ts, c.h_q, c.h_kv, c.d, false);
  if ((rc = linear_grid_check(c, L.out.max_items))) return rc;
  if (!workspace || workspace_bytes < L.total)
    return fail(PG_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, L.total);
  if ((rc = device_ready())) return rc;
  if (c.ng == 0) return PG_OK;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  if ((rc = linear_plan(c, L, ws, cu_prefix_lens, cu_suffix_lens, group_sizes, false, st))) return rc;
  pg::LinArgs a{};
  linear_common_args(a, c, L, false, ws, log_decay, cu_prefix_lens, cu_suffix_lens);
  a.q[0] = q_pre; a.k[0] = k_pre; a.v[0] = v_pre; a.q[1] = q_suf; a.k[1] = k_suf; a.v[1] = v_suf;
  a.out[0] = o_pre; a.out[1] = o_suf;
  a.state_in = state_in;
  a.state_out[0] = state_pre; a.state_out[1] = state_suf;
  const int hpw = L.out.rows.hpw;
  if (dtype == PG_BF16) {
    if (head_dim == 128) linear_fwd_typed<pg::bf16, 128>(c, hpw, a, st); else linear_fwd_typed<pg::bf16, 64>(c, hpw, a, st);
  } else {
    if (head_dim == 128) linear_fwd_typed<float, 128>(c, hpw, a, st); else linear_fwd_typed<float, 64>(c, hpw, a, st);
  }
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
  const LinearLayout L = linear_layout(dtype, c.ng, c.ns, c.tp, c.ts, c.h_q, c.h_kv, c.d, true);
  const long items = L.out.max_items < 0 || L.grad.max_items < 0 ? -1 : (long)L.out.max_items + L.grad.max_items;
  if ((rc = linear_grid_check(c, items))) return rc;
  if (!workspace || workspace_bytes < L.total)
    return fail(PG_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, L.total);
  if ((rc = device_ready())) return rc;
  if (c.ng == 0) return PG_OK;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  if ((rc = linear_plan(c, L, ws, cu_prefix_lens, cu_suffix_lens, group_sizes, true, st))) return rc;
  // dq_t = c sum l^(t-s) (do_t . v_s) k_s: the forward walk with do, v, k in the places of q, k, v
  pg::LinArgs dq{}, g{};
  linear_common_args(dq, c, L, false, ws, log_decay, cu_prefix_lens, cu_suffix_lens);
  dq.q[0] = do_pre; dq.k[0] = v_pre; dq.v[0] = k_pre; dq.q[1] = do_suf; dq.k[1] = v_suf; dq.v[1] = k_suf;
  dq.out[0] = dq_pre; dq.out[1] = dq_suf;
  linear_common_args(g, c, L, true, ws, log_decay, cu_prefix_lens, cu_suffix_lens);
  g.q[0] = q_pre; g.k[0] = k_pre; g.v[0] = v_pre; g.q[1] = q_suf; g.k[1] = k_suf; g.v[1] = v_suf;
  g.d_o[0] = do_pre; g.d_o[1] = do_suf;
  g.dk[0] = dk_pre; g.dk[1] = dk_suf; g.dv[0] = dv_pre; g.dv[1] = dv_suf;
  const int hpw = L.out.rows.hpw;
  if (dtype == PG_BF16) {
    if (head_dim == 128) linear_bwd_typed<pg::bf16, 128>(c, hpw, dq, g, st);
    else linear_bwd_typed<pg::bf16, 64>(c, hpw, dq, g, st);
  } else {
    if (head_dim == 128) linear_bwd_typed<float, 128>(c, hpw, dq, g, st);
    else linear_bwd_typed<float, 64>(c, hpw, dq, g, st);
  }
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
  const size_t states_bytes = sizeof(float) * (size_t)n * h_kv * head_dim * head_dim;
  if (state_out != state && overlap(state, state_out, states_bytes, states_bytes))
    return fail(PG_EINVAL, "state_out overlaps state without being state");
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
