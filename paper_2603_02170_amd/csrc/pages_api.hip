// C-ABI host side of pages that requests share: argument checks, workspaces, launches.  See include/sagebwd_serve.h for the contract.
#include "serve_host.h"

#include "cache_share_kernels.h"

namespace {

using namespace sage;

// Entries of the table up to which a call is one launch of one workgroup.
constexpr int64_t kSmallEntries = 2048;
bool small(int R, int columns) { return (int64_t)R * columns <= kSmallEntries; }
// Entries, pages and requests up to which that has four waves and not sixteen (eight requests of 18 pages, free, fork and own 16.2 -> 15.2 us).
bool smallest(int R, int columns, int pages) { return (int64_t)R * columns <= 512 && pages <= 16384; }
constexpr int kFewRequests = 256;
// Workgroups of a launch that has kColumns columns of a row each.
unsigned row_chunks(int R, int columns) { return (unsigned)(R * (int64_t)((columns + kColumns - 1) / kColumns)); }

int check_pages(const void* asked, const void* lengths, const void* table, const void* free_pages, const void* free_count, const void* shares, int32_t R,
                int32_t columns, int32_t page, int32_t capacity, int32_t pages) {
  if (R < 0 || columns < 1 || capacity < 0 || pages < 1 || free_count == nullptr || (capacity > 0 && free_pages == nullptr) || shares == nullptr ||
      (R > 0 && (asked == nullptr || lengths == nullptr || table == nullptr)))
    return SAGEBWD_INVALID_ARG;
  if (page_shift_of(page) < 0 || (int64_t)columns * page > INT32_MAX / 2 || R > 1 << 20 || (int64_t)R * columns > kMostEntries || pages > 1 << 28)
    return SAGEBWD_UNSUPPORTED_SHAPE;
  return SAGEBWD_OK;
}
int check_pool(const sagebwd_cache_params* p, const void* pool, size_t* bytes) {
  const int rc = check_cache(p, true);
  if (rc != SAGEBWD_OK) return rc;
  if (p->pages > 1 << 28) return SAGEBWD_UNSUPPORTED_SHAPE;
  if (pool == nullptr || !aligned(pool)) return SAGEBWD_INVALID_ARG;
  return sagebwd_cache_page_bytes(p, bytes);
}
unsigned pieces_of(size_t page_bytes) { return (unsigned)((page_bytes + kCopyPiece - 1) / kCopyPiece); }

struct CompactLayout {
  size_t moves, masks, before, sizes, total;
};
CompactLayout compact_layout(int pages) {
  CompactLayout l;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes); return o; };
  const size_t groups = ((size_t)pages + 63) / 64;
  l.moves = take(((size_t)pages / 2 + 1) * sizeof(int2));
  l.masks = take(groups * 8);
  l.before = take(groups * 4);
  l.sizes = take(8);
  l.total = off;
  return l;
}

}  // namespace

extern "C" {

int sagebwd_cache_free(const int32_t* keep, int32_t* lengths, int32_t* block_table, int32_t* free_pages, int32_t* free_count, int32_t* shares, int32_t R,
                       int32_t columns, int32_t page, int32_t capacity, int32_t pages, void* stream) {
  const int rc = check_pages(keep, lengths, block_table, free_pages, free_count, shares, R, columns, page, capacity, pages);
  if (rc != SAGEBWD_OK || R == 0) return rc;
  PagesArgs a = {};
  a.asked = keep;
  a.lengths = lengths;
  a.table = block_table;
  a.free_pages = free_pages;
  a.free_count = free_count;
  a.shares = shares;
  a.R = R;
  a.columns = columns;
  a.page_shift = page_shift_of(page);
  a.capacity = capacity;
  a.pages = pages;
  hipStream_t st = (hipStream_t)stream;
  if (small(R, columns)) {
    if (smallest(R, columns, pages)) cache_free_kernel<4><<<1, 256, 0, st>>>(a);
    else cache_free_kernel<16><<<1, 1024, 0, st>>>(a);
  } else {
    cache_free_rows_kernel<<<row_chunks(R, columns), 256, 0, st>>>(a);
    SERVE_LAUNCH_CHECK();
    cache_freed_kernel<<<1 + (R + 1023) / 1024, 1024, 0, st>>>(a);
  }
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_fork_workspace_bytes(int32_t R, int32_t columns, size_t* bytes) {
  if (R < 0 || columns < 1 || bytes == nullptr) return SAGEBWD_INVALID_ARG;
  if (R > 1 << 20 || (int64_t)R * columns > kMostEntries) return SAGEBWD_UNSUPPORTED_SHAPE;
  *bytes = align_up((size_t)R * columns * 4) + align_up((size_t)R * 4);
  return SAGEBWD_OK;
}

int sagebwd_cache_fork(const int32_t* parents, int32_t* lengths, int32_t* block_table, int32_t* free_pages, int32_t* free_count, int32_t* shares, int32_t R,
                       int32_t columns, int32_t page, int32_t capacity, int32_t pages, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_pages(parents, lengths, block_table, free_pages, free_count, shares, R, columns, page, capacity, pages);
  if (rc != SAGEBWD_OK || R == 0) return rc;
  size_t need = 0;
  sagebwd_cache_fork_workspace_bytes(R, columns, &need);
  if (workspace_bytes < need) return SAGEBWD_WORKSPACE_TOO_SMALL;
  if (workspace == nullptr || !aligned(workspace, 256)) return SAGEBWD_INVALID_ARG;
  PagesArgs a = {};
  a.asked = parents;
  a.lengths = lengths;
  a.table = block_table;
  a.free_pages = free_pages;
  a.free_count = free_count;
  a.shares = shares;
  a.rows = (int32_t*)workspace;
  a.new_lengths = (int32_t*)((char*)workspace + align_up((size_t)R * columns * 4));
  a.R = R;
  a.columns = columns;
  a.page_shift = page_shift_of(page);
  a.capacity = capacity;
  a.pages = pages;
  hipStream_t st = (hipStream_t)stream;
  if (small(R, columns)) {
    if (smallest(R, columns, pages)) cache_fork_kernel<4><<<1, 256, 0, st>>>(a);
    else cache_fork_kernel<16><<<1, 1024, 0, st>>>(a);
  } else {
    cache_fork_rows_kernel<<<row_chunks(R, columns), 256, 0, st>>>(a);
    SERVE_LAUNCH_CHECK();
    cache_forked_kernel<<<1 + row_chunks(R, columns), 1024, 0, st>>>(a);
  }
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_own(const int32_t* added, const int32_t* lengths, int32_t* block_table, const int32_t* free_pages, int32_t* free_count, int32_t* shares,
                      int32_t R, int32_t columns, int32_t capacity, const sagebwd_cache_params* params, void* pool, int32_t* added_out, void* workspace,
                      size_t workspace_bytes, void* stream) {
  size_t page_bytes = 0;
  int rc = check_pool(params, pool, &page_bytes);
  if (rc != SAGEBWD_OK) return rc;
  rc = check_pages(added, lengths, block_table, free_pages, free_count, shares, R, columns, params->page, capacity, params->pages);
  if (rc != SAGEBWD_OK || R == 0) return rc;
  if (added_out == nullptr) return SAGEBWD_INVALID_ARG;
  if (workspace_bytes < (size_t)R * sizeof(int2)) return SAGEBWD_WORKSPACE_TOO_SMALL;
  if (workspace == nullptr || !aligned(workspace)) return SAGEBWD_INVALID_ARG;
  if (pieces_of(page_bytes) > (unsigned)kMostInY) return SAGEBWD_UNSUPPORTED_SHAPE;
  PagesArgs a = {};
  a.asked = added;
  a.lengths = (int32_t*)lengths;
  a.table = block_table;
  a.free_pages = (int32_t*)free_pages;
  a.free_count = free_count;
  a.shares = shares;
  a.granted = added_out;
  a.moves = (int2*)workspace;
  a.R = R;
  a.columns = columns;
  a.page_shift = page_shift_of(params->page);
  a.capacity = capacity;
  a.pages = params->pages;
  hipStream_t st = (hipStream_t)stream;
  if (R <= kFewRequests) cache_own_kernel<4><<<1, 256, 0, st>>>(a);
  else cache_own_kernel<16><<<1, 1024, 0, st>>>(a);
  SERVE_LAUNCH_CHECK();
  cache_copy_pages_kernel<<<dim3(R, pieces_of(page_bytes)), 256, 0, st>>>(a.moves, (unsigned char*)pool, page_bytes);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

int sagebwd_cache_compact_workspace_bytes(int32_t pages, size_t* bytes) {
  if (pages < 1 || bytes == nullptr) return SAGEBWD_INVALID_ARG;
  if (pages > 1 << 28) return SAGEBWD_UNSUPPORTED_SHAPE;
  *bytes = compact_layout(pages).total;
  return SAGEBWD_OK;
}

int sagebwd_cache_compact(const int32_t* lengths, const int32_t* block_table, int32_t R, int32_t columns, const sagebwd_cache_params* params, void* pool,
                          int32_t* table_out, int32_t* free_pages, int32_t capacity, int32_t* free_count, int32_t* shares, int32_t* used, void* workspace,
                          size_t workspace_bytes, void* stream) {
  size_t page_bytes = 0;
  int rc = check_pool(params, pool, &page_bytes);
  if (rc != SAGEBWD_OK) return rc;
  rc = check_pages(lengths, lengths, block_table, free_pages, free_count, shares, R, columns, params->page, capacity, params->pages);
  if (rc != SAGEBWD_OK) return rc;
  if ((R > 0 && table_out == nullptr) || used == nullptr || capacity < params->pages) return SAGEBWD_INVALID_ARG;
  const CompactLayout l = compact_layout(params->pages);
  if (workspace_bytes < l.total) return SAGEBWD_WORKSPACE_TOO_SMALL;
  if (workspace == nullptr || !aligned(workspace, 256)) return SAGEBWD_INVALID_ARG;
  char* ws = (char*)workspace;
  CompactArgs c = {};
  c.p.lengths = (int32_t*)lengths;
  c.p.table = (int32_t*)block_table;
  c.p.free_pages = free_pages;
  c.p.free_count = free_count;
  c.p.shares = shares;
  c.p.moves = (int2*)(ws + l.moves);
  c.p.R = R;
  c.p.columns = columns;
  c.p.page_shift = page_shift_of(params->page);
  c.p.capacity = capacity;
  c.p.pages = params->pages;
  c.table_out = table_out;
  c.used = used;
  c.masks = (uint64_t*)(ws + l.masks);
  c.before = (int32_t*)(ws + l.before);
  c.sizes = (int32_t*)(ws + l.sizes);
  c.pool = (unsigned char*)pool;
  c.page_bytes = page_bytes;
  c.pieces = (int)pieces_of(page_bytes);
  hipStream_t st = (hipStream_t)stream;
  if (small(R, columns)) {
    cache_count_and_choose_kernel<<<1, 1024, 0, st>>>(c);
  } else {
    cache_count_kernel<<<row_chunks(R, columns), 256, 0, st>>>(c);
    SERVE_LAUNCH_CHECK();
    cache_choose_kernel<<<1, 1024, 0, st>>>(c);
  }
  SERVE_LAUNCH_CHECK();
  // (how many pages move is not known here: workgroups that step over them)
  const int64_t most = (int64_t)params->pages / 2 * c.pieces, here = most < 8 * kCus ? most : 8 * kCus;
  cache_compact_kernel<<<(unsigned)(here > 16 ? here : 16), 256, 0, st>>>(c);
  SERVE_LAUNCH_CHECK();
  return SAGEBWD_OK;
}

}  // extern "C"
