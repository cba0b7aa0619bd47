// C-ABI host side of the operators around the attention: argument checks, workspace layout, launches.
// See include/sagebwd_serve.h for the contract of every entry point.
#include "sagebwd_serve.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "cache_attend_kernel.h"
#include "cache_chunk_kernel.h"
#include "cache_plan_kernels.h"
#include "rotary_kernel.h"
#include "serve_host.h"

namespace {

using namespace sage;

template <int DIM, int GROUP>
struct NibbleKernels {
  static constexpr int D = DIM, MOST_TILES = 2;      // of 16 rows, of the kernel for few
  static constexpr bool BYTES = false;      // held in 8 bits: no kernel for tiles of 64 and 128 rows
  template <int NQ>
  static void few(int grid, const AttendArgs& a, hipStream_t st) { cache_attend_kernel<D, GROUP, NQ><<<grid, 256, 0, st>>>(a); }
  template <int ROWS>
  static void join_few(dim3 grid, const AttendArgs& a, hipStream_t st) { cache_join_kernel<D, ROWS><<<grid, 256, 0, st>>>(a); }
  template <int ROWS>
  static void join_many(dim3 grid, const AttendArgs& a, hipStream_t st) { cache_join_rows_kernel<D, ROWS><<<grid, 256, 0, st>>>(a); }
  static void chunk(int grid, const AttendArgs& a, hipStream_t st) { cache_chunk_kernel<D, GROUP><<<grid, 512, 0, st>>>(a); }
  template <int RG>
  static void span(int grid, const AttendArgs& a, hipStream_t st) { cache_span_kernel<D, GROUP, RG><<<grid, 512, 0, st>>>(a); }
  static void unpack(int grid, const AttendArgs& a, hipStream_t st) { cache_unpack_kernel<D, GROUP><<<grid, 512, 0, st>>>(a); }
  static void wide(int grid, const AttendArgs& a, hipStream_t st) { cache_wide_kernel<D, GROUP><<<grid, 512, 0, st>>>(a); }
};

template <typename F>
int with_format(const sagebwd_cache_params& p, F f) {
  if (p.d == 64) return p.group == 32 ? f(std::integral_constant<int, 64>(), std::integral_constant<int, 32>())
                                      : f(std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
  return p.group == 32 ? f(std::integral_constant<int, 128>(), std::integral_constant<int, 32>())
                       : f(std::integral_constant<int, 128>(), std::integral_constant<int, 64>());
}

}  // namespace

extern "C" {

int sagebwd_cache_page_bytes(const sagebwd_cache_params* params, size_t* bytes) {
  const int rc = check_cache(params, false);
  if (rc != SAGEBWD_OK) return rc;
  if (bytes == nullptr) return SAGEBWD_INVALID_ARG;
  const CacheGeometry g = geometry(*params);
  *bytes = params->block ? (size_t)g.H * (params->d == 64 ? Bytes8<64>::head_bytes(g) : Bytes8<128>::head_bytes(g)) : g.page_bytes();
  return SAGEBWD_OK;
}

int sagebwd_cache_plan(const int32_t* held, const int32_t* added, int32_t* block_table, const int32_t* free_pages, const int32_t* free_count,
                       int32_t R, int32_t columns, int32_t page, int32_t capacity, int32_t rows, int64_t* slots, int32_t* positions,
                       int32_t* cu_new, int32_t* lengths, int32_t* granted, int32_t* free_left, void* stream) {
  if (R < 0 || rows < 0 || columns < 1 || capacity < 0) return SAGEBWD_INVALID_ARG;
  if ((R > 0 && (held == nullptr || added == nullptr || block_table == nullptr || lengths == nullptr || granted == nullptr)) ||
      (capacity > 0 && free_pages == nullptr) || free_count == nullptr || cu_new == nullptr || free_left == nullptr ||
      (rows > 0 && (slots == nullptr || positions == nullptr)))
    return SAGEBWD_INVALID_ARG;
  if (page_shift_of(page) < 0 || (int64_t)columns * page > INT32_MAX / 2 || R > 1 << 20 || (int64_t)R * columns > kMostEntries || rows > kMostRows)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  const PlanArgs a{held, added, free_pages, free_count, block_table, slots, positions, cu_new, lengths, granted, free_left,
                   R, columns, page_shift_of(page), capacity, rows};
  hipStream_t st = (hipStream_t)stream;
  // Several workgroups read what one of them writes where the lengths are updated in place; more requests than a workgroup has threads are summed
  // in several steps: many rows are then a launch of their own.
  const bool in_place = lengths == held || free_left == free_count;
  const bool several = R <= 1024 && !in_place;
  const int with_rows = several || rows <= 2048;
  if (R <= 64 && rows <= 256) cache_plan_kernel<1><<<1, 64, 0, st>>>(a, 1);
  else if (R <= 256 && rows <= 1024) cache_plan_kernel<4><<<1, 256, 0, st>>>(a, 1);
  else cache_plan_kernel<16><<<several && rows > 0 ? (rows + 1023) / 1024 : 1, 1024, 0, st>>>(a, with_rows);
  SERVE_LAUNCH_CHECK();
  if (with_rows) return SAGEBWD_OK;
  cache_plan_rows_kernel<<<(rows + 255) / 256, 256, 0, st>>>(a);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_trim(const int32_t* keep, int32_t* lengths, int32_t* block_table, int32_t* free_pages, int32_t* free_count, int32_t R,
                       int32_t columns, int32_t page, int32_t capacity, void* stream) {
  if (R < 0 || columns < 1 || capacity < 0 || free_count == nullptr || (capacity > 0 && free_pages == nullptr) ||
      (R > 0 && (keep == nullptr || lengths == nullptr || block_table == nullptr)))
    return SAGEBWD_INVALID_ARG;
  if (page_shift_of(page) < 0 || (int64_t)columns * page > INT32_MAX / 2 || R > 1 << 20 || (int64_t)R * columns > kMostEntries)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  if (R == 0) return SAGEBWD_OK;
  cache_trim_kernel<<<1, 1024, 0, (hipStream_t)stream>>>(
      TrimArgs{keep, lengths, block_table, free_pages, free_count, R, columns, page_shift_of(page), capacity});
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_append(const void* K, const void* V, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                         int64_t v_head_stride, const int64_t* slots, int32_t T, const float* k_mean, const float* v_mean,
                         const sagebwd_cache_params* params, void* pool, void* stream) {
  const int rc = check_cache(params, true);
  if (rc != SAGEBWD_OK) return rc;
  if (T < 0 || !stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) || !stride_ok(v_head_stride))
    return SAGEBWD_INVALID_ARG;
  if (T == 0) return SAGEBWD_OK;
  if (K == nullptr || V == nullptr || slots == nullptr || pool == nullptr || !aligned(K) || !aligned(V) || !aligned(pool)) return SAGEBWD_INVALID_ARG;
  const int64_t per = 256 / (params->d / 8), groups = (T + per - 1) / per;      // tokens of a workgroup, and workgroups of a head
  if (groups * params->H * 256 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  const StoreArgs a{(const __bf16*)K, (const __bf16*)V, {k_token_stride, k_head_stride}, {v_token_stride, v_head_stride}, slots, k_mean, v_mean,
                    (unsigned char*)pool, nullptr, nullptr, T, geometry(*params)};
  if (params->block) return cache8_append(a, *params, (hipStream_t)stream);
  return with_format(*params, [&](auto d, auto group) -> int {
    cache_append_kernel<decltype(d)::value, decltype(group)::value><<<dim3((unsigned)groups, params->H), 256, 0, (hipStream_t)stream>>>(a);
    SERVE_LAUNCH_CHECK();
    return SAGEBWD_OK;
  });
}

int sagebwd_cache_read(const int64_t* slots, int32_t T, const float* k_mean, const float* v_mean, const sagebwd_cache_params* params,
                       const void* pool, void* K, void* V, void* stream) {
  const int rc = check_cache(params, true);
  if (rc != SAGEBWD_OK) return rc;
  if (T < 0) return SAGEBWD_INVALID_ARG;
  if (T == 0) return SAGEBWD_OK;
  if (K == nullptr || V == nullptr || slots == nullptr || pool == nullptr || !aligned(K) || !aligned(V) || !aligned(pool)) return SAGEBWD_INVALID_ARG;
  const int64_t per = 256 / (params->d / 8), groups = (T + per - 1) / per;      // tokens of a workgroup, and workgroups of a head
  if (groups * params->H * 256 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  const StoreArgs a{nullptr, nullptr, {0, 0}, {0, 0}, slots, k_mean, v_mean, (unsigned char*)pool, (__bf16*)K, (__bf16*)V, T, geometry(*params)};
  if (params->block) return cache8_read(a, *params, (hipStream_t)stream);
  return with_format(*params, [&](auto d, auto group) -> int {
    cache_read_kernel<decltype(d)::value, decltype(group)::value><<<dim3((unsigned)groups, params->H), 256, 0, (hipStream_t)stream>>>(a);
    SERVE_LAUNCH_CHECK();
    return SAGEBWD_OK;
  });
}

int sagebwd_cache_workspace_bytes(const sagebwd_cache_params* params, const sagebwd_cache_call* call, size_t* bytes) {
  const int rc = check_call(params, call);
  if (rc != SAGEBWD_OK) return rc;
  if (bytes == nullptr) return SAGEBWD_INVALID_ARG;
  *bytes = attend_plan(*params, *call).total;
  return SAGEBWD_OK;
}

int sagebwd_cache_attention(const void* Q, const void* pool, const int32_t* block_table, const int32_t* lengths, const int32_t* cu,
                            const float* v_mean, const sagebwd_cache_params* params, const sagebwd_cache_call* call, void* O, float* LSE,
                            void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_call(params, call);
  if (rc != SAGEBWD_OK) return rc;
  if (call->R == 0 || call->T == 0) return SAGEBWD_OK;
  if (Q == nullptr || pool == nullptr || block_table == nullptr || lengths == nullptr || cu == nullptr || O == nullptr || !aligned(Q) ||
      !aligned(pool) || !aligned(O))
    return SAGEBWD_INVALID_ARG;
  const AttendPlan w = attend_plan(*params, *call);
  if (workspace_bytes < w.total) return SAGEBWD_WORKSPACE_TOO_SMALL;
  if (workspace == nullptr || !aligned(workspace, 256)) return SAGEBWD_INVALID_ARG;
  char* ws = (char*)workspace;
  AttendArgs a = {};
  a.Q = (const __bf16*)Q;
  a.pool = (const unsigned char*)pool;
  a.table = block_table;
  a.lengths = lengths;
  a.cu = cu;
  a.v_mean = v_mean;
  a.O = (__bf16*)O;
  a.LSE = LSE;
  a.g = geometry(*params);
  a.R = call->R;
  a.T = call->T;
  a.Hq = call->Hq;
  a.G = call->Hq / params->H;
  a.columns = call->columns;
  a.max_new = call->max_new;
  a.max_length = w.max_length;
  a.causal = call->causal;
  a.scale_log2 = (call->sm_scale > 0.f ? call->sm_scale : 1.f / sqrtf((float)params->d)) * 1.4426950408889634f;
  a.q_token = call->q_token_stride;
  a.q_head = call->q_head_stride;
  if (params->block) return cache8_attend(a, *params, w, ws, (hipStream_t)stream);
  return with_format(*params, [&](auto d, auto group) {
    return launch_attend<NibbleKernels<decltype(d)::value, decltype(group)::value>>(a, w, ws, (hipStream_t)stream);
  });
}

int sagebwd_rotary(const void* Q, const void* K, void* Qo, void* Ko, const void* positions, const float* inv_freq,
                   const sagebwd_rotary_params* p, void* stream) {
  if (p == nullptr || p->B < 0 || p->N < 0 || p->Hq < 1 || p->Hk < 0 || p->axes < 1 || p->axes > 4 || (p->adjacent != 0 && p->adjacent != 1) ||
      (p->inverse != 0 && p->inverse != 1) || (p->positions64 != 0 && p->positions64 != 1))
    return SAGEBWD_INVALID_ARG;
  if (p->d < 16 || p->d > 512 || p->d % 16 != 0 || p->rotary_dim < 16 || p->rotary_dim > p->d || p->rotary_dim % 16 != 0 ||
      (int64_t)p->B * p->N > INT32_MAX / 64 || (int64_t)p->Hq + p->Hk > kMostInY)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  int64_t sum = 0;
  for (int k = 0; k < p->axes; k++) {
    if (p->sections[k] < 0) return SAGEBWD_INVALID_ARG;
    sum += p->sections[k];
  }
  if (sum != p->rotary_dim / 2) return SAGEBWD_INVALID_ARG;
  for (int k = 0; k < 3; k++)
    if (!stride_ok(p->q_strides[k]) || !stride_ok(p->qo_strides[k]) || (p->Hk > 0 && (!stride_ok(p->k_strides[k]) || !stride_ok(p->ko_strides[k]))))
      return SAGEBWD_INVALID_ARG;
  if (p->B == 0 || p->N == 0) return SAGEBWD_OK;
  if (Q == nullptr || Qo == nullptr || positions == nullptr || inv_freq == nullptr || !aligned(Q) || !aligned(Qo) ||
      (p->Hk > 0 && (K == nullptr || Ko == nullptr || !aligned(K) || !aligned(Ko))))
    return SAGEBWD_INVALID_ARG;
  RotaryArgs a;
  a.x[0] = (const __bf16*)Q;
  a.x[1] = (const __bf16*)K;
  a.y[0] = (__bf16*)Qo;
  a.y[1] = (__bf16*)Ko;
  for (int k = 0; k < 3; k++) {
    a.xs[0][k] = p->q_strides[k];
    a.xs[1][k] = p->k_strides[k];
    a.ys[0][k] = p->qo_strides[k];
    a.ys[1][k] = p->ko_strides[k];
  }
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.N = p->N;
  a.tokens = p->B * p->N;
  a.d = p->d;
  a.half = p->rotary_dim / 2;
  a.heads[0] = p->Hq;
  a.heads[1] = p->Hk;
  a.axes = p->axes;
  int at = 0;
  for (int k = 0; k < 4; k++) {
    if (k < p->axes) at += p->sections[k];
    a.end[k] = at;
  }
  a.sign = p->inverse ? -1.f : 1.f;
  // Many tokens: eight frequencies a thread, for as many of up to eight heads as leave the machine 2^16 threads (of a training batch, 4109 tokens of 126
  // heads of 128, one head 74 us, eight 57; 2048 of 40 14.6 and, with two, 10.2; 8192 of 64 of 64 40 and 30; asked to leave 2^19, 16381
  // of 32 of 64 go from 122 to 134 forth and back); few: two, for one head.
  const int64_t many = (int64_t)a.tokens * (p->d / 16);
  const bool wide = many >= 4096;
  a.pieces = p->d / (wide ? 16 : 4);
  a.heads_per_thread = 1;
  for (int n = 8; n > 1 && a.heads_per_thread == 1; n /= 2)
    if (wide && many * ((p->Hq + n - 1) / n + (p->Hk + n - 1) / n) >= 1 << 16) a.heads_per_thread = n;
  for (int k = 0; k < 2; k++) a.head_groups[k] = (a.heads[k] + a.heads_per_thread - 1) / a.heads_per_thread;
  const dim3 grid((unsigned)(((int64_t)a.tokens * a.pieces + 255) / 256), a.head_groups[0] + a.head_groups[1]);
  hipStream_t st = (hipStream_t)stream;
  const auto launch = [&](auto adjacent, auto pos) {
    typedef decltype(pos) P;
    if (wide) rotary_kernel<8, decltype(adjacent)::value, P><<<grid, 256, 0, st>>>(a);
    else rotary_kernel<2, decltype(adjacent)::value, P><<<grid, 256, 0, st>>>(a);
  };
  if (p->adjacent) p->positions64 ? launch(std::true_type(), int64_t()) : launch(std::true_type(), int32_t());
  else p->positions64 ? launch(std::false_type(), int64_t()) : launch(std::false_type(), int32_t());
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

}  // extern "C"
