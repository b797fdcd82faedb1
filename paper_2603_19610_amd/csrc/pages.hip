// Page tables made on the device (gfx950): the pages of a batch's sequences grown
// and cut back from a stack of free ones, and the cache slots of a batch's new rows.
// Both are integer bookkeeping between two model steps, bound by the latency of one
// launch; nothing of it needs the host, so a step that does it can be a graph.
//
// Resize.  Sequence b wants need_b = ceil(len_b / P) pages.  Those past need_b go on
// the stack in order (b, then page); then sequences take need_b - held_b pages off
// its top in order, each only if all that it and those ahead of it lack are there.
// Every order is fixed by sums over the batch, so the result is the same each time.
// (64 sequences: 7.1 us, a chain of loads, scans and stores; 16 prompts that take up
// to 1040 pages each, 8.8.  Slots: 576 rows 4.4 us, 532480 rows 7.8.)
// One workgroup does it: the sums in LDS, then its waves move the entries, one or
// more waves a sequence, 256 entries of each on their way.
#include "common.h"

namespace pvlm {
namespace {

constexpr int kMaxBatch = 4096;
constexpr int kWg = 1024;

// The inclusive sum over the workgroup's threads in order, and the total.
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t* s_wave, int64_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) s_wave[w] = x;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int i = 0; i < waves; ++i) {
    if (i < w) before += s_wave[i];
    total += s_wave[i];
  }
  __syncthreads();
  return before + x;
}

struct ResizeArgs {
  const int32_t* len;
  int32_t* held;
  int32_t* table;
  int32_t* free_pages;
  int32_t* n_free;
  int32_t* granted;
  int32_t* status;
  int64_t n_pages;
  int B, page, max_pages;
};

__global__ void __launch_bounds__(kWg) pages_resize_kernel(ResizeArgs a) {
  __shared__ int s_need[kMaxBatch], s_held[kMaxBatch];
  __shared__ int64_t s_first[kMaxBatch];  // entries (given back, then taken) of the sequences ahead
  __shared__ int64_t s_wave[kWg / 64];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, waves = kWg / 64;
  if (tid == 0) s_bad = 0;
  int64_t top = *a.n_free;
  bool bad = top < 0 || top > a.n_pages;
  top = top < 0 ? 0 : top > a.n_pages ? a.n_pages : top;
  int64_t back = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWg) {
    const int b = b0 + tid;
    int need = 0, held = 0;
    if (b < a.B) {
      const int64_t most = (int64_t)a.max_pages * a.page;
      int64_t n = a.len[b];
      held = a.held[b];
      bad |= n < 0 || n > most || held < 0 || held > a.max_pages;
      n = n < 0 ? 0 : n > most ? most : n;
      held = held < 0 ? 0 : held > a.max_pages ? a.max_pages : held;
      need = (int)((n + a.page - 1) / a.page);
      s_need[b] = need;
      s_held[b] = held;
    }
    int64_t total;
    const int64_t x = held > need ? held - need : 0, upto = block_scan(x, s_wave, total);
    if (b < a.B) s_first[b] = back + upto - x;
    back += total;
  }
  __syncthreads();
  // Several waves to a sequence where there are few.
  const int per = a.B >= waves ? 1 : waves / a.B;
  const int part = w % per;
  bool bad_entry = false;
  for (int b = w / per; b < a.B; b += waves / per) {
    const int need = s_need[b], n = s_held[b] - need;
    int32_t* row = a.table + (int64_t)b * a.max_pages + need;
    int32_t* to = a.free_pages + top + s_first[b];
    const int64_t room = a.n_pages - top - s_first[b];
#pragma unroll 4
    for (int j = 64 * part + lane; j < n; j += 64 * per) {
      const int pg = row[j];
      bad_entry |= pg < 0 || pg >= a.n_pages || j >= room;
      if (j < room) to[j] = pg;
      row[j] = -1;
    }
  }
  if (bad_entry) s_bad = 1;
  bad |= bad_entry;
  __threadfence_block();
  __syncthreads();
  int64_t depth = top + back < a.n_pages ? top + back : a.n_pages;
  if (s_bad) {
    // A table held entries that name no page (or more than there are): what was given
    // back is gone through once more, and only pages stay.  One wave, 64 at a time.
    if (w == 0) {
      int64_t out = top;
      for (int64_t i0 = top; i0 < depth; i0 += 64) {
        const int pg = i0 + lane < depth ? a.free_pages[i0 + lane] : -1;
        const bool fine = pg >= 0 && pg < a.n_pages;
        const uint64_t m = __ballot(fine);
        if (fine) a.free_pages[out + __popcll(m & (((uint64_t)1 << lane) - 1))] = pg;
        out += __popcll(m);
      }
      if (lane == 0) s_first[0] = out;
    }
    __threadfence_block();
    __syncthreads();
    depth = s_first[0];
    __syncthreads();
  }
  // what is taken
  int64_t asked = 0, taken = 0;
  bool none_left = false;
  for (int b0 = 0; b0 < a.B; b0 += kWg) {
    const int b = b0 + tid;
    const int held = b < a.B ? s_held[b] : 0, need = b < a.B ? s_need[b] : 0;
    const int64_t x = need > held ? need - held : 0;
    int64_t total, total_taken;
    const int64_t upto = asked + block_scan(x, s_wave, total);
    const bool fits = x == 0 || upto <= depth;
    (void)block_scan(fits ? x : 0, s_wave, total_taken);
    if (b < a.B) {
      s_first[b] = upto - x;
      if (!fits) s_need[b] = held;  // (nothing of it)
      a.held[b] = fits ? need : held;
      if (a.granted) a.granted[b] = fits;
      none_left |= !fits;
    }
    asked += total;
    taken += total_taken;
  }
  __syncthreads();
  for (int b = w / per; b < a.B; b += waves / per) {
    const int held = s_held[b], n = s_need[b] - held;
    int32_t* row = a.table + (int64_t)b * a.max_pages + held;
    const int32_t* from = a.free_pages + depth - 1 - s_first[b];
#pragma unroll 4
    for (int j = 64 * part + lane; j < n; j += 64 * per) row[j] = from[-(int64_t)j];
  }
  if (tid == 0) *a.n_free = (int32_t)(depth - taken);
  if (bad) dev_flag(a.status, PVLM_DEV_RANGE);
  if (none_left) dev_flag(a.status, PVLM_DEV_NO_PAGES);
}

// ------------------------------------------------------------- slot map --
struct SlotArgs {
  const int32_t* ctx;
  const int32_t* n_new;
  const int32_t* table;  // NULL: a padded cache, a page a sequence
  int64_t* slots;
  int32_t* pos;
  int32_t* seq;
  int32_t* start;
  int32_t* status;
  int64_t n_pages, n_rows;
  int B, T, page, max_pages;  // T: rows of a sequence, 0 packed
};

constexpr int kSlotWg = 256, kSlotRows = 4;  // a work-item's rows

// Every workgroup adds the batch's counts up in LDS (4096 of them at most), then a
// row finds its sequence among them by bisection.
__global__ void __launch_bounds__(kSlotWg) slot_map_kernel(SlotArgs a) {
  __shared__ int s_start[kMaxBatch + 1];
  __shared__ int64_t s_wave[kSlotWg / 64];
  const int tid = threadIdx.x;
  const bool flags = blockIdx.x == 0;
  bool bad = false;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.B; b0 += kSlotWg) {
    const int b = b0 + tid;
    int64_t n = b < a.B ? a.n_new[b] : 0;
    const int64_t most = a.T ? a.T : a.n_rows;
    bad |= n < 0 || n > most;
    n = n < 0 ? 0 : n > most ? most : n;
    int64_t total;
    int64_t upto = before + block_scan(n, s_wave, total);
    before += total;
    // rows past n_rows are dropped (packed), and flagged
    if (!a.T) {
      bad |= upto > a.n_rows;
      upto = upto > a.n_rows ? a.n_rows : upto;
    }
    if (b < a.B) {
      s_start[b + 1] = (int)upto;
      if (flags && a.start) a.start[b + 1] = (int)upto;
    }
  }
  if (tid == 0) {
    s_start[0] = 0;
    if (flags && a.start) a.start[0] = 0;
  }
  if (flags && bad) dev_flag(a.status, PVLM_DEV_RANGE);
  __syncthreads();
  bad = false;
  for (int k = 0; k < kSlotRows; ++k) {
    const int64_t i = ((int64_t)blockIdx.x * kSlotRows + k) * kSlotWg + tid;
    if (i >= a.n_rows) break;
    int b, j, n;
    if (a.T) {
      b = (int)(i / a.T);
      j = (int)(i - (int64_t)b * a.T);
      n = s_start[b + 1] - s_start[b];
    } else {
      // the last sequence that begins at or before row i (of several, empty ones among them, the last)
      int lo = 0, hi = a.B;
      while (lo + 1 < hi) {
        const int mid = (lo + hi) / 2;
        if (s_start[mid] <= i) lo = mid;
        else hi = mid;
      }
      b = lo;
      j = (int)(i - s_start[b]);
      n = s_start[b + 1] - s_start[b];
    }
    const bool real = j < n;
    int64_t slot = -1;
    int row = 0;
    if (real) {
      const int ctx = a.ctx[b];
      const int64_t t = (int64_t)ctx + j;
      const int64_t page = t < 0 ? -1 : t / a.page;
      if (ctx >= 0 && page < a.max_pages && t <= INT32_MAX) {
        const int64_t pg = a.table ? a.table[(int64_t)b * a.max_pages + page] : b;
        if (pg >= 0 && pg < a.n_pages) slot = pg * a.page + (t - page * a.page);
      }
      bad |= slot < 0;
      row = slot < 0 ? 0 : (int)t;
    }
    a.slots[i] = slot;
    if (a.pos) a.pos[i] = row;
    if (a.seq) a.seq[i] = real ? b : -1;
  }
  if (bad) dev_flag(a.status, PVLM_DEV_RANGE);
}

}  // namespace
}  // namespace pvlm

using namespace pvlm;

extern "C" pvlm_status pvlm_pages_resize(int B, int page_size, int max_pages, int64_t n_pages, const int32_t* len,
                                         int32_t* n_held, int32_t* page_table, int32_t* free_pages, int32_t* n_free,
                                         int32_t* granted, int32_t* status, hipStream_t stream) {
  if (!len || !n_held || !page_table || !free_pages || !n_free) return PVLM_ERR_NULL;
  if (B < 1 || page_shift_of(page_size) < 0 || max_pages < 1 || n_pages < 1 || n_pages > INT32_MAX ||
      (int64_t)max_pages * page_size > ((int64_t)1 << 30))
    return PVLM_ERR_SHAPE;
  if (B > kMaxBatch) return PVLM_ERR_UNSUPPORTED;
  ResizeArgs a{len, n_held, page_table, free_pages, n_free, granted, status, n_pages, B, page_size, max_pages};
  hipLaunchKernelGGL(pages_resize_kernel, dim3(1), dim3(kWg), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

extern "C" pvlm_status pvlm_slot_map(int B, int64_t n_rows, int rows_per_seq, int page_size, int max_pages,
                                     int64_t n_pages, const int32_t* page_table, const int32_t* ctx_len,
                                     const int32_t* n_new, int64_t* slots, int32_t* pos, int32_t* seq,
                                     int32_t* row_start, int32_t* status, hipStream_t stream) {
  if (!ctx_len || !n_new || !slots) return PVLM_ERR_NULL;
  if (B < 1 || n_rows < 1 || rows_per_seq < 0 || page_size < 1 || page_size > (1 << 30) || max_pages < 1 || n_pages < 1 ||
      n_pages > INT32_MAX || (int64_t)max_pages * page_size > ((int64_t)1 << 30))
    return PVLM_ERR_SHAPE;
  if (page_table ? page_shift_of(page_size) < 0 : max_pages != 1) return PVLM_ERR_SHAPE;
  if (rows_per_seq && n_rows != (int64_t)B * rows_per_seq) return PVLM_ERR_SHAPE;
  if (B > kMaxBatch) return PVLM_ERR_UNSUPPORTED;
  if (n_rows > ((int64_t)1 << 30)) return PVLM_ERR_SHAPE;
  if ((uintptr_t)slots % 8 != 0) return PVLM_ERR_UNSUPPORTED;
  SlotArgs a{ctx_len, n_new, page_table, slots, pos, seq, row_start, status, n_pages, n_rows,
             B, rows_per_seq, page_size, max_pages};
  const int64_t per = kSlotWg * kSlotRows;
  hipLaunchKernelGGL(slot_map_kernel, dim3((unsigned)((n_rows + per - 1) / per)), dim3(kSlotWg), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}
