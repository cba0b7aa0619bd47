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
  static constexpr int D = DIM, MOST_TILES = DIM == 128 ? 4 : 2;      // of 16 rows, of the kernel for few
  static constexpr bool BYTES = true;      // held in 8 bits: no kernel for tiles of 64 and 128 rows
  template <int NQ>
  static void few(int grid, const AttendArgs& a, hipStream_t st) { cache8_attend_kernel<D, NQ><<<grid, 256, 0, st>>>(a); }
  template <int NQ>
  static void few_short(int grid, const AttendArgs& a, hipStream_t st) { cache8_short_kernel<D, NQ><<<grid, 256, 0, st>>>(a); }
  template <int ROWS>
  static void join_few(dim3 grid, const AttendArgs& a, hipStream_t st) { cache8_join_kernel<D, ROWS><<<grid, 256, 0, st>>>(a); }
  template <int ROWS>
  static void join_many(dim3 grid, const AttendArgs& a, hipStream_t st) { cache8_join_rows_kernel<D, ROWS><<<grid, 256, 0, st>>>(a); }
  static void chunk(int grid, const AttendArgs& a, hipStream_t st) { cache8_chunk_kernel<D><<<grid, 512, 0, st>>>(a); }
  static void unpack(int grid, const AttendArgs& a, hipStream_t st) { cache8_unpack_kernel<D><<<grid, 512, 0, st>>>(a); }
  static void wide(int grid, const AttendArgs& a, hipStream_t st) { cache8_wide_kernel<D><<<grid, 512, 0, st>>>(a); }
};

}  // namespace

// Rows that a workgroup looks through for runs of its own: 1024 workgroups of four waves, as an empty one costs 2 ns.  (Storing 7700 tokens of 8 heads in runs
// of 32 with windows of 4, 8, 16, 32 rows: 48, 27, 18.5, 17 us.)
static int window_of(const StoreArgs& a, const sagebwd_cache_params& p, int waves) {
  int window = 1;
  while (window < 64 && (int64_t)a.T * p.H * waves > 4096 * (int64_t)window) window *= 2;
  return window;
}
template <int D, int BLOCK, int WAVES>
static void launch_append(const StoreArgs& a, const dim3& grid, int window, hipStream_t st) {
  cache8_append_kernel<D, BLOCK, WAVES><<<grid, 64 * WAVES, 0, st>>>(a, window);
}

int cache8_append(const StoreArgs& a, const sagebwd_cache_params& p, hipStream_t st) {
  // Few tokens are mostly one of each request: two waves, which go through a whole block in up to four rounds, where else a wave has no more than one.
  // (48 tokens of 8 heads, one of each request: eight waves 6.0 us, two 4.9.)
  const bool few = a.T <= 256;
  const int waves = few ? 2 : p.block * p.d / 1024, window = window_of(a, p, 2 * waves);
  const dim3 grid((unsigned)((a.T + (int64_t)window - 1) / window), p.H, 2);
  if ((int64_t)grid.x * p.H * 1024 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  if (p.d == 64 && p.block == 32) launch_append<64, 32, 2>(a, grid, window, st);
  else if (p.d == 64) few ? launch_append<64, 64, 2>(a, grid, window, st) : launch_append<64, 64, 4>(a, grid, window, st);
  else if (p.block == 32) few ? launch_append<128, 32, 2>(a, grid, window, st) : launch_append<128, 32, 4>(a, grid, window, st);
  else few ? launch_append<128, 64, 2>(a, grid, window, st) : launch_append<128, 64, 8>(a, grid, window, st);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int cache8_read(const StoreArgs& a, const sagebwd_cache_params& p, hipStream_t st) {
  const int window = window_of(a, p, 4);
  const dim3 grid((unsigned)((a.T + (int64_t)window - 1) / window), p.H);
  if ((int64_t)grid.x * p.H * 256 > kMostThreads) return SAGEBWD_UNSUPPORTED_SHAPE;
  if (p.d == 64) cache8_read_kernel<64><<<grid, 256, 0, st>>>(a, window);
  else cache8_read_kernel<128><<<grid, 256, 0, st>>>(a, window);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int cache8_attend(const AttendArgs& a, const sagebwd_cache_params& p, const AttendPlan& w, char* ws, hipStream_t st) {
  return p.d == 64 ? launch_attend<ByteKernels<64>>(a, w, ws, st) : launch_attend<ByteKernels<128>>(a, w, ws, st);
}

}  // namespace sage
