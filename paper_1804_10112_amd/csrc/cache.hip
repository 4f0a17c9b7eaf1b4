// The pages of a cache: rows that are extended, written, compacted, cut and forked. All of it is integer work on the table and
// copies of whole slots, so results do not depend on the order in which workgroups run. Nearly all of these kernels take what a launch and
// a few dependent loads take (1.3 to 5 us); copies move 16 bytes a lane: 56 forked rows whose last pages are copied in 4 layers, 27 MB
// read and written, 16.7 us.
#include "cache.hpp"

namespace spt {

namespace {

constexpr int kScanBlock = 1024;

// Gives back the pages of row s at places from .. to-1. Called by a whole wave.
__device__ __forceinline__ void release(const Cache& c, int s, int from, int to) {
  for (int j = from + lane_id(); j < to; j += kWave) {
    const int p = page_at(c, s, j);
    if (p >= 0) atomicSub(&c.refs[p], 1);
    c.table[static_cast<int64_t>(s) * c.row_pages + j] = -1;
  }
}

// ---- free -------------------------------------------------------------------------------------------------------------------

__global__ void free_kernel(Cache c, const int32_t* __restrict__ new_len) {
  const int s = blockIdx.x * (kBlock / kWave) + wave_id();
  if (s >= c.rows) return;
  const int before = row_length(c, s), after = new_len[s];
  if (after < 0 || after >= before) return;
  release(c, s, pages_held(c, after), pages_held(c, before));
  if (lane_id() == 0) c.len[s] = after;
}

// ---- fork -------------------------------------------------------------------------------------------------------------------

// A workgroup for each entry. Parents are only read (an entry whose child is a parent is skipped) and each child belongs to one
// entry, the last that names it, so entries do not meet; refs are atomic.
__global__ void fork_kernel(Cache c, int n, const int32_t* __restrict__ parents, const int32_t* __restrict__ children) {
  const int i = blockIdx.x, parent = parents[i], child = children[i];
  if (parent < 0 || parent >= c.rows || child < 0 || child >= c.rows) return;
  int barred = 0;
  for (int k = threadIdx.x; k < n; k += blockDim.x) barred |= parents[k] == child || (k > i && children[k] == child);
  if (__syncthreads_or(barred)) return;
  const int length = row_length(c, parent), held = pages_held(c, length), old = pages_held(c, row_length(c, child));
  __syncthreads();  // before the child's length changes
  for (int j = threadIdx.x; j < (held > old ? held : old); j += blockDim.x) {
    const int was = j < old ? page_at(c, child, j) : -1, is = j < held ? page_at(c, parent, j) : -1;
    if (was >= 0) atomicSub(&c.refs[was], 1);
    if (is >= 0) atomicAdd(&c.refs[is], 1);
    c.table[static_cast<int64_t>(child) * c.row_pages + j] = is;
  }
  if (threadIdx.x == 0) c.len[child] = length;
}

// ---- extend -----------------------------------------------------------------------------------------------------------------
//
// Three steps. (1) The free pages are counted, in stretches of the pool, and the rows are gone through for the running sum of the
// pages they want. (2) With both, the k-th free page finds the row and the place it goes to. (3) Copies on write, lengths, and the
// shared pages' refs, which (1) and (2) both have to find as they were. A launch each; the first two are one workgroup's where its
// threads hold the whole pool's refs in registers.

struct Wanted {
  int start, count;  // places start .. start+count-1 of the table
  bool refused;
};

// What row s wants to hold `add` tokens more; copy: its last page is partly filled and shared.
__device__ __forceinline__ Wanted wanted(const Cache& c, int length, int add, bool copy) {
  if (add <= 0) return {0, 0, false};
  if (add > (c.row_pages << c.shift) - length) return {0, 0, true};
  const int start = pages_held(c, length) - copy;
  return {start, pages_held(c, length + add) - start, false};
}

__device__ __forceinline__ int block_inclusive_scan(int v, int* lds) {
  const int lane = lane_id(), wave = wave_id();
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = v;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += lds[w];
  return v + before;
}

// What (1) leaves to (2) and (3), in the workspace.
struct Plan {
  int32_t* free_pages;  // of each stretch
  int32_t* end;         // of each row: pages wanted by the rows up to it
  int32_t* copied;      // of each row: its shared last page, or -1
  int32_t* target;      // of each row: the page that takes its place
  int32_t* fill;        // of each row: slots used of its last page, 0 = all
  int32_t* total;       // free pages in all
};

// Step (1) of the rows, by a whole workgroup.
__device__ __forceinline__ void want(const Cache& c, const int32_t* __restrict__ add, const Plan& plan, int32_t* refused, int* lds) {
  int before = 0;
  for (int base = 0; base < c.rows; base += kScanBlock) {
    const int s = base + threadIdx.x;
    int n = 0, from = -1;
    if (s < c.rows) {
      const int length = row_length(c, s), more = add[s];
      if (more > 0 && (length & ((1 << c.shift) - 1)) != 0) {
        const int p = page_at(c, s, length >> c.shift);
        if (p >= 0 && c.refs[p] > 1) from = p;
      }
      n = wanted(c, length, more, from >= 0).count;
      plan.copied[s] = from;
      plan.fill[s] = length & ((1 << c.shift) - 1);
    }
    const int sum = before + block_inclusive_scan(n, lds);
    if (s < c.rows) plan.end[s] = sum;
    __syncthreads();
    if (threadIdx.x == kScanBlock - 1) lds[0] = sum;
    __syncthreads();
    before = lds[0];
  }
  if (threadIdx.x == 0) *refused = 0;
}

// Step (2) of free page p, the k-th of `total`.
__device__ __forceinline__ void assign(const Cache& c, const int32_t* __restrict__ add, const Plan& plan, int p, int k, int total) {
  int s = 0, n = c.rows;  // the first row with end > k
  while (n > 0) {
    const int half = n >> 1;
    if (plan.end[s + half] <= k) s += half + 1, n -= half + 1;
    else n = half;
  }
  if (plan.end[s] > total) return;
  const Wanted w = wanted(c, row_length(c, s), add[s], plan.copied[s] >= 0);
  const int place = k - (plan.end[s] - w.count);
  c.table[static_cast<int64_t>(s) * c.row_pages + w.start + place] = p;
  c.refs[p] = 1;
  if (place == 0) plan.target[s] = p;
}

// Refs that a thread holds of a small pool. Pools of 1000 to 4000 pages take 11.2 us either way, with the freeing after it (replayed); one
// launch less to make is what counts. At 16 000 pages one workgroup takes 12.9 us, two launches 11.3.
constexpr int kHeld = 4;

__global__ void __launch_bounds__(kScanBlock) extend_small_kernel(Cache c, const int32_t* __restrict__ add, Plan plan,
                                                                  int32_t* refused) {
  __shared__ int lds[kScanBlock / kWave];
  // bit k: page k * kScanBlock + thread is free; pages in ascending order are ranked group by group
  uint32_t is_free = 0;
  int held[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int p = k * kScanBlock + threadIdx.x;
    held[k] = p < c.pages ? c.refs[p] : 1;
  }
#pragma unroll
  for (int k = 0; k < kHeld; ++k) is_free |= (held[k] == 0) << k;
  want(c, add, plan, refused, lds);
  __shared__ int in_wave[kHeld][kScanBlock / kWave];  // free pages of each group and wave, then of all before them
  __shared__ int sum;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int n = __popcll(__ballot(is_free >> k & 1));
    if (lane_id() == 0) in_wave[k][wave_id()] = n;
  }
  __syncthreads();
  constexpr int kCounts = kHeld * (kScanBlock / kWave);
  static_assert(kCounts <= kScanBlock, "a count a thread");
  const int mine = threadIdx.x < kCounts ? (&in_wave[0][0])[threadIdx.x] : 0, upto = block_inclusive_scan(mine, lds);
  __syncthreads();
  if (threadIdx.x < kCounts) (&in_wave[0][0])[threadIdx.x] = upto - mine;
  if (threadIdx.x == kScanBlock - 1) sum = upto;
  __syncthreads();
  const int total = sum, needed = c.rows ? plan.end[c.rows - 1] : 0;
  if (threadIdx.x == 0) *plan.total = total;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const uint64_t b = __ballot(is_free >> k & 1);
    const int rank = in_wave[k][wave_id()] + __popcll(b & ((uint64_t(1) << lane_id()) - 1));
    if ((is_free >> k & 1) && rank < needed) assign(c, add, plan, k * kScanBlock + threadIdx.x, rank, total);
  }
}

__global__ void __launch_bounds__(kScanBlock) extend_count_kernel(Cache c, const int32_t* __restrict__ add, int stretch, Plan plan,
                                                                  int32_t* refused) {
  __shared__ int lds[kScanBlock / kWave];
  if (blockIdx.x + 1 == gridDim.x) {
    want(c, add, plan, refused, lds);
    return;
  }
  const int lo = blockIdx.x * stretch, hi = c.pages - lo < stretch ? c.pages : lo + stretch;
  int n = 0;
  strided(lo, hi, threadIdx.x, kScanBlock, [&](int p) { n += c.refs[p] == 0; });
  n = block_inclusive_scan(n, lds);
  if (threadIdx.x == kScanBlock - 1) plan.free_pages[blockIdx.x] = n;
}

__global__ void __launch_bounds__(kScanBlock) extend_assign_kernel(Cache c, const int32_t* __restrict__ add, int stretch, Plan plan) {
  __shared__ int lds[kScanBlock / kWave];
  __shared__ int sums[2];
  if (threadIdx.x < 2) sums[threadIdx.x] = 0;
  __syncthreads();
  int mine = 0, all = 0;
  for (int b = threadIdx.x; b < static_cast<int>(gridDim.x); b += kScanBlock) {
    const int n = plan.free_pages[b];
    all += n;
    if (b < static_cast<int>(blockIdx.x)) mine += n;
  }
  if (mine) atomicAdd(&sums[0], mine);
  if (all) atomicAdd(&sums[1], all);
  __syncthreads();
  int rank = sums[0];
  const int total = sums[1];
  if (blockIdx.x == 0 && threadIdx.x == 0) *plan.total = total;
  const int needed = plan.end[c.rows - 1];
  const int lo = blockIdx.x * stretch;
  const uint32_t hi = c.pages - lo < stretch ? c.pages : lo + stretch;
  for (uint32_t base = lo; base < hi && rank < needed; base += kScanBlock) {  // a step past the last page may pass 2^31
    const uint32_t p = base + threadIdx.x;
    const int is_free = p < hi && c.refs[p] == 0;
    const int upto = rank + block_inclusive_scan(is_free, lds);
    if (is_free && upto <= needed) assign(c, add, plan, p, upto - 1, total);
    __syncthreads();
    if (threadIdx.x == kScanBlock - 1) lds[0] = upto;
    __syncthreads();
    rank = lds[0];
    __syncthreads();
  }
}

// Rows by blockIdx.x; the slots to copy are dealt out over blockIdx.y, the last of which does the row's numbers.
__global__ void extend_finish_kernel(Cache c, const int32_t* __restrict__ add, Plan plan, int32_t* refused) {
  const int s = blockIdx.x, from = plan.copied[s], fill = plan.fill[s];
  const int wants = plan.end[s] - (s ? plan.end[s - 1] : 0);
  const bool served = wants == 0 || plan.end[s] <= *plan.total;
  if (blockIdx.y + 1 == gridDim.y) {
    if (threadIdx.x != 0) return;
    const int length = row_length(c, s);
    if (!served || wanted(c, length, add[s], from >= 0).refused) {
      atomicAdd(refused, 1);
    } else if (add[s] > 0) {
      c.len[s] = length + add[s];
      if (wants && from >= 0) atomicSub(&c.refs[from], 1);
    }
    return;
  }
  if (from < 0 || wants == 0 || !served) return;
  const int to = plan.target[s], vecs = c.width_bytes / 16;
  const int64_t units = static_cast<int64_t>(c.layers) * fill * c.heads * vecs * 2;
  for (int64_t u = blockIdx.y * static_cast<int64_t>(blockDim.x) + threadIdx.x; u < units;
       u += static_cast<int64_t>(gridDim.y - 1) * blockDim.x) {
    int64_t r = u;
    const int v = r % vecs;
    r /= vecs;
    const int h = r % c.heads;
    r /= c.heads;
    const int o = r % fill;
    r /= fill;
    char* pool = (r & 1) ? c.V : c.K;
    pool += (r >> 1) * c.layer_bytes + o * c.slot_bytes + h * c.head_bytes + v * 16;
    *reinterpret_cast<int4*>(pool + to * c.page_bytes) = *reinterpret_cast<const int4*>(pool + from * c.page_bytes);
  }
}

// ---- write ------------------------------------------------------------------------------------------------------------------

// A wave for each token.
__global__ void write_kernel(Cache c, int layer, const int32_t* __restrict__ first, int total, const char* __restrict__ k,
                             const char* __restrict__ v, int64_t token_bytes, int64_t in_head_bytes) {
  const int i = blockIdx.x * (kBlock / kWave) + wave_id();
  if (i >= total) return;
  const int s = wave_row_of(first, c.rows, i);
  if (s < 0) return;
  const Drafted d = drafted(first, s, total);
  const int length = row_length(c, s), t = length - d.count + i - d.begin;
  if (t < 0 || t >= length) return;
  const int page = page_at(c, s, t >> c.shift);
  if (page < 0) return;
  const int64_t at = layer * c.layer_bytes + page * c.page_bytes + (t & ((1 << c.shift) - 1)) * c.slot_bytes;
  const int vecs = c.width_bytes / 16;
  for (int u = lane_id(); u < c.heads * vecs; u += kWave) {
    const int h = u / vecs, e = (u - h * vecs) * 16;
    const int64_t from = i * token_bytes + h * in_head_bytes + e, to = at + h * c.head_bytes + e;
    *reinterpret_cast<int4*>(c.K + to) = *reinterpret_cast<const int4*>(k + from);
    *reinterpret_cast<int4*>(c.V + to) = *reinterpret_cast<const int4*>(v + from);
  }
}

// ---- compact ----------------------------------------------------------------------------------------------------------------

// Entries of a row's list that name drafted tokens it has. The list ascends, so those that are none lie at its ends: a look at both ends,
// and a search (halving, by every thread for itself) only where there are some.
struct Kept {
  int begin, count;
};
__device__ __forceinline__ Kept kept(const Pattern& keep, int s, int drafts) {
  int begin = pattern_begin(keep, s), end = pattern_end(keep, s);
  if (begin < end && (keep.crd[begin] < 0 || keep.crd[end - 1] >= drafts)) {
    auto below = [&](int limit) {  // the first entry that is not below it
      int lo = begin, hi = end;
      while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (keep.crd[mid] < limit) lo = mid + 1;
        else hi = mid;
      }
      return lo;
    };
    const int from = below(0), to = below(drafts);
    begin = from, end = to;
  }
  return {begin, clamped(end - begin, 0, drafts)};
}

// A thread owns 16 bytes of each token of the row (in one layer, K or V, and head) and moves them token after token, kBatch loads at a
// time: the kept ones ascend, so a slot that is written was read before and is not read again. Where the tokens lie the workgroup
// finds out first, kMoves of them at a time. 48 rows that keep a third of up to 64 tokens in 4 layers: 8.6 us, token after token with its
// lookups 17. (Without a look at the lists' ends, which has to come before the length that is cut to, 8.3, and 2.8 instead of 3.2 for the cut.)
constexpr int kMoves = kBlock, kBatch = 8;
typedef int Bytes16 __attribute__((ext_vector_type(4)));
__global__ void __launch_bounds__(kBlock) compact_move_kernel(Cache c, const int32_t* __restrict__ first, Pattern keep) {
  __shared__ int64_t from[kMoves], to[kMoves];  // -1: stays where it is
  const int s = blockIdx.x, vecs = c.width_bytes / 16;
  const Drafted d = drafted(first, s, INT32_MAX);
  const int context = row_length(c, s) - d.count;
  const Kept k = kept(keep, s, d.count);
  const int begin = k.begin, n = k.count;
  if (context < 0 || n == 0) return;
  int r = blockIdx.y * blockDim.x + threadIdx.x;
  const bool mine = r < c.layers * 2 * c.heads * vecs;
  const int v = r % vecs;
  r /= vecs;
  const int h = r % c.heads;
  r /= c.heads;
  char* pool = ((r & 1) ? c.V : c.K) + (r >> 1) * c.layer_bytes + h * c.head_bytes + v * 16;
  for (int base = 0; base < n; base += kMoves) {
    __syncthreads();
    const int j = base + threadIdx.x;
    if (j < n) {
      const int f = keep.crd[begin + j];
      int64_t a = -1, b = -1;
      if (f > j && f < d.count) {
        const int x = context + f, y = context + j, px = page_at(c, s, x >> c.shift), py = page_at(c, s, y >> c.shift);
        const int mask = (1 << c.shift) - 1;
        if (px >= 0 && py >= 0) a = px * c.page_bytes + (x & mask) * c.slot_bytes, b = py * c.page_bytes + (y & mask) * c.slot_bytes;
      }
      from[threadIdx.x] = a;
      to[threadIdx.x] = b;
    }
    __syncthreads();
    const int count = n - base < kMoves ? n - base : kMoves;
    if (mine)
      for (int k = 0; k < count; k += kBatch) {
        Bytes16 x[kBatch];
#pragma unroll
        for (int e = 0; e < kBatch; ++e)
          if (k + e < count && from[k + e] >= 0) x[e] = *reinterpret_cast<const Bytes16*>(pool + from[k + e]);
#pragma unroll
        for (int e = 0; e < kBatch; ++e)
          if (k + e < count && from[k + e] >= 0) *reinterpret_cast<Bytes16*>(pool + to[k + e]) = x[e];
      }
  }
}

__global__ void compact_cut_kernel(Cache c, const int32_t* __restrict__ first, Pattern keep) {
  const int s = blockIdx.x * (kBlock / kWave) + wave_id();
  if (s >= c.rows) return;
  const Drafted d = drafted(first, s, INT32_MAX);
  const int before = row_length(c, s), context = before - d.count;
  if (context < 0 || d.count == 0) return;
  const int after = context + kept(keep, s, d.count).count;
  release(c, s, pages_held(c, after), pages_held(c, before));
  if (lane_id() == 0) c.len[s] = after;
}

int stretch_of(int64_t pages) {
  const int64_t s = (pages + 1023) / 1024;
  return s < kScanBlock ? kScanBlock : static_cast<int>(s);
}

}  // namespace

size_t cache_extend_workspace(const spt_cache* c) {
  return 4 * align_up(static_cast<size_t>(c->rows) * 4, 256) + align_up(1024 * 4, 256) + 256;
}

spt_status cache_extend_dispatch(const spt_cache* cache, const int32_t* add, int32_t* refused, void* ws, hipStream_t stream) {
  const Cache c = cache_view(cache);
  Workspace w(ws, cache_extend_workspace(cache));
  Plan plan;
  plan.free_pages = w.take<int32_t>(1024);
  plan.end = w.take<int32_t>(c.rows);
  plan.copied = w.take<int32_t>(c.rows);
  plan.target = w.take<int32_t>(c.rows);
  plan.fill = w.take<int32_t>(c.rows);
  plan.total = w.take<int32_t>(1);
  if (c.pages <= kHeld * kScanBlock) {
    extend_small_kernel<<<1, kScanBlock, 0, stream>>>(c, add, plan, refused);
  } else {
    const int stretch = stretch_of(c.pages), blocks = (c.pages - 1) / stretch + 1;
    extend_count_kernel<<<blocks + 1, kScanBlock, 0, stream>>>(c, add, stretch, plan, refused);
    if (c.rows > 0) extend_assign_kernel<<<blocks, kScanBlock, 0, stream>>>(c, add, stretch, plan);
  }
  if (c.rows == 0) {
    SPT_CHECK_LAUNCH("cache_extend");
    return SPT_OK;
  }
  const int64_t units = static_cast<int64_t>(c.layers) * 2 * c.heads * (c.width_bytes / 16) << c.shift;
  int64_t y = (units + 8 * kBlock - 1) / (8 * kBlock);
  const int64_t most = c.rows < 8192 ? 8192 / c.rows : 1;
  y = y > most ? most : y;
  extend_finish_kernel<<<dim3(c.rows, static_cast<unsigned>(y) + 1), kBlock, 0, stream>>>(c, add, plan, refused);
  SPT_CHECK_LAUNCH("cache_extend");
  return SPT_OK;
}

spt_status cache_free_dispatch(const spt_cache* cache, const int32_t* new_len, hipStream_t stream) {
  const Cache c = cache_view(cache);
  free_kernel<<<(c.rows + 3) / 4, kBlock, 0, stream>>>(c, new_len);
  SPT_CHECK_LAUNCH("cache_free");
  return SPT_OK;
}

spt_status cache_fork_dispatch(const spt_cache* cache, int n, const int32_t* parents, const int32_t* children, hipStream_t stream) {
  fork_kernel<<<n, kBlock, 0, stream>>>(cache_view(cache), n, parents, children);
  SPT_CHECK_LAUNCH("cache_fork");
  return SPT_OK;
}

spt_status cache_write_dispatch(const spt_cache* cache, int layer, const int32_t* first, int total, const void* k, const void* v,
                                int64_t token_stride, int64_t head_stride, hipStream_t stream) {
  const int64_t b = value_bytes(cache->dtype);
  write_kernel<<<(total + 3) / 4, kBlock, 0, stream>>>(cache_view(cache), layer, first, total, static_cast<const char*>(k),
                                                       static_cast<const char*>(v), token_stride * b, head_stride * b);
  SPT_CHECK_LAUNCH("cache_write");
  return SPT_OK;
}

spt_status cache_compact_dispatch(const spt_cache* cache, const int32_t* first, const spt_tensor* keep, hipStream_t stream) {
  const Cache c = cache_view(cache);
  const Pattern k = pattern_view(keep);
  const int64_t threads = static_cast<int64_t>(c.layers) * 2 * c.heads * (c.width_bytes / 16);
  compact_move_kernel<<<dim3(c.rows, static_cast<unsigned>((threads + kBlock - 1) / kBlock)), kBlock, 0, stream>>>(c, first, k);
  compact_cut_kernel<<<(c.rows + 3) / 4, kBlock, 0, stream>>>(c, first, k);
  SPT_CHECK_LAUNCH("cache_compact");
  return SPT_OK;
}

}  // namespace spt
