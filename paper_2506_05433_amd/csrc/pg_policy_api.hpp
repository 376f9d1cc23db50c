// Entry points of the token log-probabilities and the policy loss (included by pg_lib.hip, after the helpers of pg_attn.hip).
#pragma once

namespace {

int check_logprobs(int dtype, int token_bytes, int ng, int ns, int tp, int ts, const int32_t* cu_p,
                   const int32_t* cu_s, const int32_t* gsz, int vocab, const long (&ld)[4], float temperature) {
  int rc = check_grouping(ng, ns, tp, ts, cu_p, cu_s, gsz);
  if (rc) return rc;
  if (dtype != PG_BF16 && dtype != PG_FP32) return fail(PG_EUNSUPPORTED, "dtype %d is not PG_BF16 or PG_FP32", dtype);
  if (token_bytes != 4 && token_bytes != 8) return fail(PG_EUNSUPPORTED, "tokens of %d bytes (4 or 8)", token_bytes);
  if (vocab <= 0) return fail(PG_EINVAL, "vocab=%d must be > 0", vocab);
  for (long s : ld)
    if (s < vocab) return fail(PG_EINVAL, "row stride %ld is less than vocab=%d", s, vocab);
  if (!(std::isfinite(temperature) && temperature > 0.f) || !std::isfinite(1.f / temperature))
    return fail(PG_EINVAL, "temperature must be finite and > 0");
  return PG_OK;
}

bool unaligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

struct LogprobLayout {
  RopeLayout plan;
  size_t target, total;
};

LogprobLayout logprob_layout(int ng, int ns) {
  LogprobLayout L{};
  L.plan = rope_layout(ng);
  L.target = align_up(L.plan.total);
  L.total = L.target + align_up(sizeof(float) * (size_t)(ns > 0 ? ns : 1));
  return L;
}

template <typename T, int NT>
void launch_logprobs(const pg::LogprobArgs& a, bool bwd, unsigned blocks, hipStream_t st) {
  if (bwd) {
    if constexpr (NT > 64) hipLaunchKernelGGL((pg::logprob_bwd_kernel<T, NT>), dim3(blocks), dim3(NT), 0, st, a);
  } else if (a.entropy) hipLaunchKernelGGL((pg::logprob_kernel<T, NT, true>), dim3(blocks), dim3(NT), 0, st, a);
  else hipLaunchKernelGGL((pg::logprob_kernel<T, NT, false>), dim3(blocks), dim3(NT), 0, st, a);
}

int run_logprobs(int dtype, const pg::LogprobArgs& a0, bool bwd, const int32_t* gsz, int tp, void* workspace,
                 size_t workspace_bytes, void* stream) {
  pg::LogprobArgs a = a0;
  const LogprobLayout L = logprob_layout(a.ng, a.ns);
  if (!workspace || workspace_bytes < L.total)
    return fail(PG_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, L.total);
  int rc = device_ready();
  if (rc) return rc;
  if (a.ng == 0) return PG_OK;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  a.hdr = (const pg::PlanHeader*)(ws + L.plan.hdr);
  a.ginfo = (const pg::GroupInfoEx*)(ws + L.plan.ginfo);
  a.target = (float*)(ws + L.target);
  {
    Timed tp_(PG_K_PLAN, st);
    if ((rc = launch_rope_plan(L.plan, ws, a.ng, a.ns, tp, a.ts, a.cu_p, a.cu_s, gsz, st))) return rc;
  }
  if (!bwd && a.ts == 0) return PG_OK;  // no token to predict: no logits are read, they may be NULL
  // Threads a row, by its 16-byte pieces. 64: short rows where there are many, no barriers (5k rows, bf16: 1000 wide 8.8
  // us against 15.9 with 256, 5000 wide 16.4 and 21.6, 17000 wide 36.2 and 35.4; as many waves as the card holds, each
  // takes several rows). 1024: a few long rows (6 of 131072: 15.5, 17.9), and gradients of long rows, whose reads and
  // writes then stay closer together (5k rows: 50001 wide bf16 203 us against 224, fp32 392 and 447; 17000 wide bf16
  // 93 and 73).
  const long rows = (long)a.ng + a.ts, pieces = a.vocab / (dtype == PG_BF16 ? 8 : 4);
  const bool few = rows <= 128;
  const bool wave = !bwd && pieces <= 1250 && rows >= 1024, long_rows = few ? pieces >= 2048 : bwd && pieces >= 4096;
  const unsigned blocks = (unsigned)std::min(rows, wave ? 8192L : 1L << 20);
  Timed tm(PG_K_LOGPROBS, st);
  if (dtype == PG_BF16) {
    if (wave) launch_logprobs<pg::bf16, 64>(a, bwd, blocks, st);
    else if (long_rows) launch_logprobs<pg::bf16, 1024>(a, bwd, blocks, st);
    else launch_logprobs<pg::bf16, 256>(a, bwd, blocks, st);
  } else {
    if (wave) launch_logprobs<float, 64>(a, bwd, blocks, st);
    else if (long_rows) launch_logprobs<float, 1024>(a, bwd, blocks, st);
    else launch_logprobs<float, 256>(a, bwd, blocks, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "token log-probability launch");
  return PG_OK;
}

struct PolicyLayout {
  size_t hdr, member_w, count, part, total;
  int blocks;
};

PolicyLayout policy_layout(int ns, int ts) {
  PolicyLayout L{};
  L.blocks = (int)std::max(1L, ceil_div_l(ts, pg::kPolicyTok * pg::kPolicyPer));
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  L.hdr = take(sizeof(pg::PlanHeader));
  L.member_w = take(sizeof(double) * (size_t)(ns > 0 ? ns : 1));
  L.count = take(sizeof(int) * ((size_t)ns + 1));
  L.part = take(sizeof(double) * 4 * (size_t)L.blocks);
  L.total = off;
  return L;
}

}  // namespace

extern "C" {

size_t pg_token_logprobs_workspace_size(int n_groups, int n_suffixes, int total_suffix, int vocab) {
  if (n_groups < 0 || n_suffixes < 0 || total_suffix < 0 || vocab < 0) return 0;
  return logprob_layout(n_groups, n_suffixes).total;
}

int pg_token_logprobs(int dtype, int token_bytes, int n_groups, int n_suffixes, int total_prefix, int total_suffix,
                      const int32_t* cu_prefix_lens, const int32_t* cu_suffix_lens, const int32_t* group_sizes,
                      int vocab, float temperature, const void* logits_last, int64_t stride_last,
                      const void* logits_suf, int64_t stride_suf, const void* tokens, float* logp, float* lse,
                      float* entropy, void* workspace, size_t workspace_bytes, void* stream) {
  g_last_error.clear();
  int rc = check_logprobs(dtype, token_bytes, n_groups, n_suffixes, total_prefix, total_suffix, cu_prefix_lens,
                          cu_suffix_lens, group_sizes, vocab, {stride_last, stride_suf, stride_last, stride_suf},
                          temperature);
  if (rc) return rc;
  if (total_suffix > 0 && (!logits_last || !logits_suf || !tokens || !logp || !lse))
    return fail(PG_EINVAL, "a tensor pointer is NULL");
  const size_t e = dtype == PG_BF16 ? 2 : 4;
  if (unaligned(logits_last, e) || unaligned(logits_suf, e) || unaligned(tokens, token_bytes))
    return fail(PG_EINVAL, "a tensor pointer is not aligned to its elements");
  pg::LogprobArgs a{};
  a.last = logits_last; a.suf = logits_suf; a.ld_last = stride_last; a.ld_suf = stride_suf;
  a.tokens = tokens; a.tok64 = token_bytes == 8;
  a.logp = logp; a.lse = lse; a.entropy = entropy;
  a.cu_p = cu_prefix_lens; a.cu_s = cu_suffix_lens;
  a.ng = n_groups; a.ns = n_suffixes; a.ts = total_suffix; a.vocab = vocab;
  a.inv_temp = 1.f / temperature;
  return run_logprobs(dtype, a, false, group_sizes, total_prefix, workspace, workspace_bytes, stream);
}

int pg_token_logprobs_bwd(int dtype, int token_bytes, int n_groups, int n_suffixes, int total_prefix,
                          int total_suffix, const int32_t* cu_prefix_lens, const int32_t* cu_suffix_lens,
                          const int32_t* group_sizes, int vocab, float temperature, const void* logits_last,
                          int64_t stride_last, const void* logits_suf, int64_t stride_suf, const void* tokens,
                          const float* lse, const float* dlogp, void* dlogits_last, int64_t dstride_last,
                          void* dlogits_suf, int64_t dstride_suf, void* workspace, size_t workspace_bytes,
                          void* stream) {
  g_last_error.clear();
  int rc = check_logprobs(dtype, token_bytes, n_groups, n_suffixes, total_prefix, total_suffix, cu_prefix_lens,
                          cu_suffix_lens, group_sizes, vocab, {stride_last, stride_suf, dstride_last, dstride_suf},
                          temperature);
  if (rc) return rc;
  if (n_groups > 0 && (!logits_last || !dlogits_last)) return fail(PG_EINVAL, "a tensor pointer is NULL");
  if (total_suffix > 0 && (!logits_suf || !tokens || !lse || !dlogp || !dlogits_suf))
    return fail(PG_EINVAL, "a tensor pointer is NULL");
  const size_t e = dtype == PG_BF16 ? 2 : 4;
  if (unaligned(logits_last, e) || unaligned(logits_suf, e) || unaligned(dlogits_last, e) ||
      unaligned(dlogits_suf, e) || unaligned(tokens, token_bytes))
    return fail(PG_EINVAL, "a tensor pointer is not aligned to its elements");
  // in place means element for element: the same rows
  if ((dlogits_last == logits_last && logits_last && dstride_last != stride_last) ||
      (dlogits_suf == logits_suf && logits_suf && dstride_suf != stride_suf))
    return fail(PG_EINVAL, "gradients in the place of their logits need the logits' row stride");
  pg::LogprobArgs a{};
  a.last = logits_last; a.suf = logits_suf; a.ld_last = stride_last; a.ld_suf = stride_suf;
  a.d_last = dlogits_last; a.d_suf = dlogits_suf; a.ldd_last = dstride_last; a.ldd_suf = dstride_suf;
  a.tokens = tokens; a.tok64 = token_bytes == 8;
  a.lse = (float*)lse; a.dlogp = dlogp;
  a.cu_p = cu_prefix_lens; a.cu_s = cu_suffix_lens;
  a.ng = n_groups; a.ns = n_suffixes; a.ts = total_suffix; a.vocab = vocab;
  a.inv_temp = 1.f / temperature;
  return run_logprobs(dtype, a, true, group_sizes, total_prefix, workspace, workspace_bytes, stream);
}

size_t pg_policy_loss_workspace_size(int n_groups, int n_suffixes, int total_suffix) {
  if (n_groups < 0 || n_suffixes < 0 || total_suffix < 0) return 0;
  return policy_layout(n_suffixes, total_suffix).total;
}

int pg_policy_loss(int average, int n_groups, int n_suffixes, int total_suffix, const int32_t* cu_suffix_lens,
                   const int32_t* group_sizes, double clip_low, double clip_high, double beta, double grad_scale,
                   const float* logp, const float* logp_old, const float* logp_ref, const float* advantages,
                   const uint8_t* mask, float* stats, float* dlogp, void* workspace, size_t workspace_bytes,
                   void* stream) {
  g_last_error.clear();
  int rc = check_grouping(n_groups, n_suffixes, 0, total_suffix, cu_suffix_lens, cu_suffix_lens, group_sizes);
  if (rc) return rc;
  if (average != PG_AVERAGE_GROUP && average != PG_AVERAGE_TOKEN) return fail(PG_EINVAL, "unknown average %d", average);
  if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0 && std::isfinite(clip_high)))
    return fail(PG_EINVAL, "clip_low must be in [0, 1], clip_high finite and >= 0");
  if (!std::isfinite(beta) || !std::isfinite(grad_scale)) return fail(PG_EINVAL, "beta and grad_scale must be finite");
  if (beta != 0.0 && !logp_ref) return fail(PG_EINVAL, "beta is not 0 but logp_ref is NULL");
  if (!stats) return fail(PG_EINVAL, "stats is NULL");
  if (total_suffix > 0 && (!logp || !advantages)) return fail(PG_EINVAL, "a tensor pointer is NULL");
  const PolicyLayout L = policy_layout(n_suffixes, total_suffix);
  if (!workspace || workspace_bytes < L.total)
    return fail(PG_EWORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, L.total);
  if ((rc = device_ready())) return rc;
  hipStream_t st = (hipStream_t)stream;
  char* ws = (char*)workspace;
  pg::PolicyArgs a{};
  a.logp = logp; a.logp_old = logp_old; a.logp_ref = logp_ref; a.adv = advantages; a.mask = mask;
  a.cu_s = cu_suffix_lens; a.gsz = group_sizes; a.stats = stats; a.dlogp = dlogp;
  a.hdr = (pg::PlanHeader*)(ws + L.hdr);
  a.member_w = (double*)(ws + L.member_w);
  a.count = (int*)(ws + L.count);
  a.part = (double*)(ws + L.part);
  a.ng = n_groups; a.ns = n_suffixes; a.ts = total_suffix; a.by_token = average == PG_AVERAGE_TOKEN;
  a.cut_lo = std::log1p(-clip_low); a.cut_hi = std::log1p(clip_high);
  a.beta = beta; a.grad_scale = grad_scale;
  if (total_suffix <= pg::kPolicySmall && pg::plan_fits_lds(n_groups, n_suffixes)) {
    Timed tm(PG_K_POLICY, st);
    hipLaunchKernelGGL(pg::policy_small_kernel, dim3(1), dim3(pg::kPolicyThreads), 0, st, a);
    return finish_plan(a.hdr, st);
  }
  {
    Timed tp(PG_K_PLAN, st);
    hipLaunchKernelGGL(pg::policy_plan_kernel, dim3(1), dim3(pg::kPolicyThreads), 0, st, a);
    if ((rc = finish_plan(a.hdr, st))) return rc;
  }
  Timed tm(PG_K_POLICY, st);
  if (mask && total_suffix > 0)
    hipLaunchKernelGGL(pg::policy_count_kernel, dim3((unsigned)L.blocks), dim3(pg::kPolicyTok), 0, st, a);
  hipLaunchKernelGGL(pg::policy_loss_kernel, dim3((unsigned)L.blocks), dim3(pg::kPolicyTok), 0, st, a);
  hipLaunchKernelGGL(pg::policy_sum_kernel, dim3(1), dim3(pg::kPolicyTok), 0, st, a, L.blocks);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "policy loss launch");
  return PG_OK;
}

}  // extern "C"
