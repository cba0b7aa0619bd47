// Launches of the cache held in 8 bits: the calls of sagebwd_serve.h with block > 0, whose checks are in serve_api.hip.
#include "serve_host.h"

#include "cache8_attend_kernel.h"
#include "cache8_kernels.h"

namespace sage {

namespace {

template <int D, int ROWS>
__global__ __launch_bounds__(256) void cache8_join_kernel(AttendArgs a) {
  join_few<D, ROWS>(a);
}
template <int D, int ROWS>
__global__ __launch_bounds__(256) void cache8_join_rows_kernel(AttendArgs a) {
  join_many<D, ROWS>(a);
}

template <int DIM>
struct ByteKernels {
  static constexpr int D = DIM;
  template <int NQ>
  static void few(int grid, const AttendArgs& a, hipStream_t st) { cache8_attend_kernel<D, NQ><<<grid, 256, 0, st>>>(a); }
  template <int ROWS>
  static void join_few(dim3 grid, const AttendArgs& a, hipStream_t st) { cache8_join_kernel<D, ROWS><<<grid, 256, 0, st>>>(a); }
  template <int ROWS>
  static void join_many(dim3 grid, const AttendArgs& a, hipStream_t st) { cache8_join_rows_kernel<D, ROWS><<<grid, 256, 0, st>>>(a); }
  static void chunk(int grid, const AttendArgs& a, hipStream_t st) { cache8_chunk_kernel<D><<<grid, 512, 0, st>>>(a); }
  template <int RG>
  static void span(int grid, const AttendArgs& a, hipStream_t st) { cache8_span_kernel<D, RG><<<grid, 512, 0, st>>>(a); }
  static void unpack(int grid, const AttendArgs& a, hipStream_t st) { cache8_unpack_kernel<D><<<grid, 512, 0, st>>>(a); }
  static void wide(int grid, const AttendArgs& a, hipStream_t st) { cache8_wide_kernel<D><<<grid, 512, 0, st>>>(a); }
};

}  // namespace

int cache8_append(const StoreArgs& a, const sagebwd_cache_params& p, hipStream_t st) {
  // rows that a workgroup looks through
  int window = 1;
  while (window < 64 && (int64_t)a.T * p.H > 2048 * (int64_t)window) window *= 2;
  const dim3 grid((unsigned)((a.T + (int64_t)window - 1) / window), p.H);
  if ((int64_t)grid.x * p.H * 256 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  const int shift = p.block == 64 ? 6 : 5;
  if (p.d == 64) cache8_append_kernel<64><<<grid, 256, 0, st>>>(a, shift, window);
  else cache8_append_kernel<128><<<grid, 256, 0, st>>>(a, shift, window);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int cache8_read(const StoreArgs& a, const sagebwd_cache_params& p, hipStream_t st) {
  const int64_t per = 256 / (p.d / 8);      // (as many workgroups as the caller has bounded)
  const dim3 grid((unsigned)((a.T + per - 1) / per), p.H);
  if (p.d == 64) cache8_read_kernel<64><<<grid, 256, 0, st>>>(a);
  else cache8_read_kernel<128><<<grid, 256, 0, st>>>(a);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int cache8_attend(const AttendArgs& a, const sagebwd_cache_params& p, const AttendPlan& w, char* ws, hipStream_t st) {
  return p.d == 64 ? launch_attend<ByteKernels<64>>(a, w, ws, st) : launch_attend<ByteKernels<128>>(a, w, ws, st);
}

}  // namespace sage
