// Which pages the sequences of a paged cache have: tables reordered by parents (fork), pages given up, exchanged and taken
// (reserve), a pool moved together (compact), and the copies these leave to do (copy), with their C entry points.
#include <cooperative_groups.h>

#include <climits>

#include "paged.cuh"

namespace cg = cooperative_groups;

#define PAGES_MAX_ROWS 8192   // rows of a table: their prefix sums fit a CTA's shared memory

namespace {

struct Pool {
  int32_t *refs, *status;
  int n_pages, page_size, page_shift;
};
struct Table {
  int32_t *pages, *held, *len;
  int B, ld;
};
struct Moves {
  int32_t *list, *count;   // list: (from, to, slots)
  int capacity;
};

// entries a row holds, inside its table row
__device__ __forceinline__ int row_held(const Table& t, const Pool& p, int row) {
  const int h = t.held[row];
  if (h < 0 || h > t.ld) paged_flag(p.status, SPS_PAGED_BAD_LENGTH);
  return min(max(h, 0), t.ld);
}

// ------------------------------------------------------------------------------------------------------------------
// Fork: dst row i = src row parents[i]; a page of src row r gains children(r) - 1 references.
// Bound by latency (lengths -> entries -> references); the bytes are the tables', read once and written once.  A CTA has a
// run of 2048 entries of one row, as a row of dst and as a row of src.  Rows with exactly one child, the most of a beam step,
// touch no reference; the sums are atomic and whole, so their order does not matter.
// ------------------------------------------------------------------------------------------------------------------
constexpr int FORK_THREADS = 256, FORK_PER = 8;

struct ForkArgs {
  Pool pool;
  Table src, dst;
  const int32_t* parents;
};

__global__ void __launch_bounds__(FORK_THREADS) fork_kernel(const __grid_constant__ ForkArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x, tid = threadIdx.x, e0 = blockIdx.y * FORK_THREADS * FORK_PER + tid;
  if (row < a.dst.B) {
    const int parent = a.parents[row];
    const bool there = parent >= 0 && parent < a.src.B;
    const int held = there ? row_held(a.src, a.pool, parent) : 0;
    if (blockIdx.y == 0 && tid == 0) {
      if (parent >= a.src.B) paged_flag(a.pool.status, SPS_PAGED_BAD_ROW);
      a.dst.held[row] = held;
      a.dst.len[row] = there ? a.src.len[parent] : 0;
    }
    const int32_t* from = a.src.pages + (long long)(there ? parent : 0) * a.src.ld;
    int32_t* to = a.dst.pages + (long long)row * a.dst.ld;
    int v[FORK_PER];
#pragma unroll
    for (int i = 0; i < FORK_PER; ++i) v[i] = e0 + i * FORK_THREADS < held ? from[e0 + i * FORK_THREADS] : 0;
#pragma unroll
    for (int i = 0; i < FORK_PER; ++i)
      if (e0 + i * FORK_THREADS < held) to[e0 + i * FORK_THREADS] = v[i];
  }
  if (row < a.src.B) {
    int children = 0;
    for (int b0 = 0; b0 < a.dst.B; b0 += FORK_THREADS) children += __syncthreads_count(b0 + tid < a.dst.B && a.parents[b0 + tid] == row);
    if (children == 1) return;
    const int held = row_held(a.src, a.pool, row);
    const int32_t* from = a.src.pages + (long long)row * a.src.ld;
    int v[FORK_PER];
#pragma unroll
    for (int i = 0; i < FORK_PER; ++i) v[i] = e0 + i * FORK_THREADS < held ? from[e0 + i * FORK_THREADS] : -2;
#pragma unroll
    for (int i = 0; i < FORK_PER; ++i) {
      if (v[i] == -2 && e0 + i * FORK_THREADS >= held) continue;
      if (v[i] < 0 || v[i] >= a.pool.n_pages) paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE);
      else atomicAdd(a.pool.refs + v[i], children - 1);
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Block-wide helpers of the pool kernels (1024 threads)
// ------------------------------------------------------------------------------------------------------------------
constexpr int POOL_THREADS = 1024, POOL_WARPS = POOL_THREADS / 32;

// inclusive sum over the block's threads, in thread order; s_warp: [POOL_WARPS]; total: the block's
__device__ __forceinline__ int block_scan(int v, int* s_warp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();   // (s_warp may still be read from the last call)
  if (lane == 31) s_warp[warp] = v;
  __syncthreads();
  int w = s_warp[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += u;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return v + (warp > 0 ? before : 0);
}

// this CTA's pages of the pool, in whole tiles of 4 pages a thread
__device__ __forceinline__ void pool_part(int n_pages, unsigned rank, unsigned parts, int* lo, int* hi) {
  const long long tiles = ((long long)n_pages + POOL_THREADS * 4 - 1) / (POOL_THREADS * 4), per = (tiles + parts - 1) / parts;
  const long long a = per * rank * (POOL_THREADS * 4), b = a + per * (POOL_THREADS * 4);
  *lo = (int)(a < n_pages ? a : n_pages);
  *hi = (int)(b < n_pages ? b : n_pages);
}
// references of pages p .. p + 3, `outside` behind hi (read from L2: other CTAs changed them)
__device__ __forceinline__ int4 refs4(const int32_t* refs, int p, int hi, int outside) {
  int4 r = make_int4(outside, outside, outside, outside);
  if (p < hi) r.x = __ldcg(refs + p);
  if (p + 1 < hi) r.y = __ldcg(refs + p + 1);
  if (p + 2 < hi) r.z = __ldcg(refs + p + 2);
  if (p + 3 < hi) r.w = __ldcg(refs + p + 3);
  return r;
}

// ------------------------------------------------------------------------------------------------------------------
// Reserve.  With n = min(len, want) tokens kept in k = ceil(n / page) pages, a row (1) gives up its entries behind k, (2)
// exchanges entry k - 1 for a fresh page if it is partly filled, about to be written and held by others too -- unless all who
// hold it write to it and this row is the first of them --, and (3) takes fresh pages up to want tokens.  Fresh pages are the
// lowest free ones, handed out row after row: a prefix sum over the rows' needs and one over the pool's free pages meet.
//
// One cluster does it all (its CTAs share the pool's scan and the rows; needs are summed by every CTA for itself), the
// steps divided by cluster barriers: giving up -> marks at shared last pages -> needs and counts -> pages handed out.  What
// it costs is those steps' trips to L2, one behind the other; the references are read once or twice (4 bytes a page).
// Marks: per page the number of rows about to write to it and B - (the first of them), in the workspace, zero between calls.
// ------------------------------------------------------------------------------------------------------------------
struct ReserveArgs {
  Pool pool;
  Table t;
  const int32_t* want;
  Moves moves;
  int32_t *writers, *first;   // [n_pages], zero
};

struct RowPlan { int n, k, held, to; };   // tokens and pages kept, entries held, pages wanted
__device__ __forceinline__ RowPlan row_plan(const ReserveArgs& a, int b) {
  RowPlan r;
  const int cap = (int)min((long long)a.t.ld << a.pool.page_shift, (long long)INT_MAX - a.pool.page_size);
  const int held = a.t.held[b], len = a.t.len[b], want = a.want[b];
  r.held = min(max(held, 0), a.t.ld);
  const int room = (int)min((long long)r.held << a.pool.page_shift, (long long)cap);
  if (held != r.held || len > room || want > cap) paged_flag(a.pool.status, SPS_PAGED_BAD_LENGTH);
  const int w = min(max(want, 0), cap);
  r.n = min(min(max(len, 0), room), w);
  r.k = (r.n + a.pool.page_size - 1) >> a.pool.page_shift;
  r.to = (w + a.pool.page_size - 1) >> a.pool.page_shift;
  return r;
}
// the page of a row's last kept entry if the row is about to write into it, else -1
__device__ __forceinline__ int written_page(const ReserveArgs& a, int b, const RowPlan& r) {
  if (!(r.n & (a.pool.page_size - 1)) || a.want[b] <= r.n) return -1;
  const int q = a.t.pages[(long long)b * a.t.ld + r.k - 1];
  if (q < 0 || q >= a.pool.n_pages) { paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE); return -1; }
  return q;
}

__global__ void __launch_bounds__(POOL_THREADS) reserve_kernel(const __grid_constant__ ReserveArgs a) {
  extern __shared__ int s_rows[];
  __shared__ int s_warp[POOL_WARPS], s_free;
  int *s_end = s_rows, *s_keep = s_rows + a.t.B, *s_moves = s_keep + a.t.B, *s_page = s_moves + a.t.B;   // each [B]
  cg::cluster_group cl = cg::this_cluster();
  const unsigned rank = cl.block_rank(), parts = cl.num_blocks();
  const int tid = threadIdx.x, B = a.t.B;
  pdl_launch_dependents();
  pdl_wait();

  // (1) entries behind the kept ones, a row per warp
  for (int b = rank * POOL_WARPS + (tid >> 5); b < B; b += parts * POOL_WARPS) {
    const RowPlan r = row_plan(a, b);
    const int32_t* row = a.t.pages + (long long)b * a.t.ld;
    for (int i0 = r.k + (tid & 31); i0 < r.held; i0 += 32 * 8) {
      int p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = i0 + 32 * j < r.held ? row[i0 + 32 * j] : INT_MIN;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (i0 + 32 * j >= r.held) continue;
        if (p[j] < 0 || p[j] >= a.pool.n_pages) paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE);
        else atomicAdd(a.pool.refs + p[j], -1);
      }
    }
  }
  cl.sync();
  // (2) marks at the pages that are shared and about to be written
  for (int b = rank * POOL_THREADS + tid; b < B; b += parts * POOL_THREADS) {
    const int q = written_page(a, b, row_plan(a, b));
    if (q >= 0 && __ldcg(a.pool.refs + q) > 1) {
      atomicAdd(a.writers + q, 1);
      atomicMax(a.first + q, B - b);
    }
  }
  cl.sync();
  // (3) needs and their sums, in every CTA
  const int per = (B + POOL_THREADS - 1) / POOL_THREADS, b0 = min(tid * per, B), b1 = min(b0 + per, B);
  int need = 0, fresh = 0;
  for (int b = b0; b < b1; ++b) {
    const RowPlan r = row_plan(a, b);
    const int q = written_page(a, b, r);
    int swap = 0;
    if (q >= 0) {
      const int refs = __ldcg(a.pool.refs + q);
      swap = refs > 1 && !(__ldcg(a.writers + q) == refs && __ldcg(a.first + q) == B - b);
    }
    need += max(r.to - r.k, 0) + swap;
    fresh += swap;
    s_end[b] = need;
    s_moves[b] = fresh;
    s_keep[b] = r.k;
    s_page[b] = q;
  }
  int total_need, total_moves;
  const int need0 = block_scan(need, s_warp, &total_need) - need, fresh0 = block_scan(fresh, s_warp, &total_moves) - fresh;
  for (int b = b0; b < b1; ++b) { s_end[b] += need0; s_moves[b] += fresh0; }
  int lo, hi, mine = 0;
  pool_part(a.pool.n_pages, rank, parts, &lo, &hi);
  for (int p = lo + tid * 4; p < hi; p += POOL_THREADS * 4) {
    const int4 r = refs4(a.pool.refs, p, hi, 1);
    mine += (r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0);
  }
  int free_here;
  block_scan(mine, s_warp, &free_here);
  if (tid == 0) s_free = free_here;
  cl.sync();
  int before = 0, free_all = 0;
  for (unsigned c = 0; c < parts; ++c) {
    const int n = *cl.map_shared_rank(&s_free, c);
    if (c < rank) before += n;
    free_all += n;
  }
  // (4) rows' new state and the pages given up for fresh ones (CTA 0), then the fresh pages
  if (rank == 0) {
    for (int b = tid; b < B; b += POOL_THREADS) {
      const RowPlan r = row_plan(a, b);
      const int start = b ? s_end[b - 1] : 0, swap = s_moves[b] - (b ? s_moves[b - 1] : 0), q = s_page[b];
      const bool wants = s_end[b] > start, served = wants && s_end[b] <= free_all;
      if (wants && !served) paged_flag(a.pool.status, SPS_PAGED_NO_PAGE);
      if (q >= 0) { a.writers[q] = 0; a.first[q] = 0; }
      if (served && swap) {
        atomicAdd(a.pool.refs + q, -1);
        int32_t* m = a.moves.list + 3ll * (s_moves[b] - 1);
        m[0] = q;
        m[2] = r.n & (a.pool.page_size - 1);
      }
      a.t.held[b] = served ? max(r.to, r.k) : r.k;
      a.t.len[b] = r.n;
    }
    // moves of the rows that were served: those end with the last row whose need fits
    if (tid == 0) {
      int lo_b = 0, hi_b = B;   // the first row whose needs do not fit
      while (lo_b < hi_b) {
        const int m = (lo_b + hi_b) >> 1;
        if (s_end[m] > free_all) hi_b = m; else lo_b = m + 1;
      }
      a.moves.count[0] = lo_b ? s_moves[lo_b - 1] : 0;
    }
  }
  int at = before;
  for (int p0 = lo; p0 < hi && at < total_need; p0 += POOL_THREADS * 4) {
    const int p = p0 + tid * 4;
    const int4 r = refs4(a.pool.refs, p, hi, 1);
    const int free4[4] = {r.x == 0, r.y == 0, r.z == 0, r.w == 0};
    const int n = free4[0] + free4[1] + free4[2] + free4[3];
    int tile;
    int j = at + block_scan(n, s_warp, &tile) - n;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!free4[i]) continue;
      if (j < total_need) {
        int x = 0, y = B - 1;   // the row that the j-th free page goes to: the first whose needs end behind j
        while (x < y) {
          const int m = (x + y) >> 1;
          if (s_end[m] > j) y = m; else x = m + 1;
        }
        if (s_end[x] <= free_all) {
          const int swap = s_moves[x] - (x ? s_moves[x - 1] : 0), e = s_keep[x] - swap + j - (x ? s_end[x - 1] : 0);
          a.t.pages[(long long)x * a.t.ld + e] = p + i;
          a.pool.refs[p + i] = 1;
          if (swap && e == s_keep[x] - 1) a.moves.list[3ll * (s_moves[x] - 1) + 1] = p + i;
        }
      }
      ++j;
    }
    at += tile;
  }
  cl.sync();   // (a CTA's counts are read by the others until here)
}

// ------------------------------------------------------------------------------------------------------------------
// Compact: of U pages in use, those numbered U and above go to the free ones below U, the i-th to the i-th.
// First a cluster over the pool: U, the number of holes, then each page's place among the holes or among those that move
// (references read twice); then a grid over the table's entries and the list.  map[p]: where page p >= U stands in the list, -1 if
// it stays (nothing in use, or the list is full).
// ------------------------------------------------------------------------------------------------------------------
struct CompactArgs {
  Pool pool;
  Table src, dst;
  int32_t* refs_out;
  Moves moves;
  int32_t *map, *used;   // [n_pages], [1]
};

__global__ void __launch_bounds__(POOL_THREADS) compact_scan_kernel(const __grid_constant__ CompactArgs a) {
  __shared__ int s_warp[POOL_WARPS], s_n[2];
  cg::cluster_group cl = cg::this_cluster();
  const unsigned rank = cl.block_rank(), parts = cl.num_blocks();
  const int tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  int lo, hi, mine = 0, n_used;
  pool_part(a.pool.n_pages, rank, parts, &lo, &hi);
  for (int p = lo + tid * 4; p < hi; p += POOL_THREADS * 4) {
    const int4 r = refs4(a.pool.refs, p, hi, 0);
    mine += (r.x != 0) + (r.y != 0) + (r.z != 0) + (r.w != 0);
  }
  block_scan(mine, s_warp, &n_used);
  if (tid == 0) s_n[0] = n_used;
  cl.sync();
  int used = 0, before = 0;
  for (unsigned c = 0; c < parts; ++c) {
    const int n = *cl.map_shared_rank(&s_n[0], c);
    if (c < rank) before += n;
    used += n;
  }
  // pages in use below U: all of a part's that lies below, part of one's
  int below = hi <= used ? n_used : 0;
  if (lo < used && used < hi) {
    mine = 0;
    for (int p = lo + tid * 4; p < used; p += POOL_THREADS * 4) {
      const int4 r = refs4(a.pool.refs, p, used, 0);
      mine += (r.x != 0) + (r.y != 0) + (r.z != 0) + (r.w != 0);
    }
    block_scan(mine, s_warp, &below);
  }
  if (tid == 0) s_n[1] = below;
  cl.sync();
  int stay = 0;   // pages in use below U
  for (unsigned c = 0; c < parts; ++c) stay += *cl.map_shared_rank(&s_n[1], c);
  if (rank == 0 && tid == 0) {
    a.used[0] = used;
    a.moves.count[0] = min(used - stay, a.moves.capacity);
  }
  int at = before;
  for (int p0 = lo; p0 < hi; p0 += POOL_THREADS * 4) {
    const int p = p0 + tid * 4;
    const int4 r = refs4(a.pool.refs, p, hi, 0);
    const int ref[4] = {r.x, r.y, r.z, r.w};
    const int n = (ref[0] != 0) + (ref[1] != 0) + (ref[2] != 0) + (ref[3] != 0);
    int tile;
    int u = at + block_scan(n, s_warp, &tile) - n;   // pages in use before p
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = p + i;
      if (q >= hi) break;
      if (a.refs_out != a.pool.refs) a.refs_out[q] = ref[i];
      if (q < used) {
        if (ref[i] == 0 && q - u < a.moves.capacity) a.moves.list[3ll * (q - u) + 1] = q;
      } else {
        const int m = ref[i] != 0 && u - stay < a.moves.capacity ? u - stay : -1;
        a.map[q] = m;
        if (m >= 0) {
          a.moves.list[3ll * m] = q;
          a.moves.list[3ll * m + 2] = a.pool.page_size;
        }
      }
      u += ref[i] != 0;
    }
    at += tile;
  }
  cl.sync();
}

__global__ void __launch_bounds__(FORK_THREADS) compact_apply_kernel(const __grid_constant__ CompactArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int row = blockIdx.x, tid = threadIdx.x, e0 = blockIdx.y * FORK_THREADS * FORK_PER + tid;
  const long long all = (long long)gridDim.x * gridDim.y * FORK_THREADS, me = ((long long)blockIdx.y * gridDim.x + row) * FORK_THREADS + tid;
  const int count = a.moves.count[0], used = a.used[0];
  for (long long i = me; i < count; i += all) {   // a page's references go with it
    const int from = a.moves.list[3 * i], to = a.moves.list[3 * i + 1], r = a.pool.refs[from];
    a.refs_out[to] = r;
    a.refs_out[from] = 0;
  }
  if (row >= a.src.B) return;
  const int held = row_held(a.src, a.pool, row);
  if (blockIdx.y == 0 && tid == 0) {
    a.dst.held[row] = held;
    a.dst.len[row] = a.src.len[row];
  }
  const int32_t* from = a.src.pages + (long long)row * a.src.ld;
  int32_t* to = a.dst.pages + (long long)row * a.dst.ld;
  int v[FORK_PER];
#pragma unroll
  for (int i = 0; i < FORK_PER; ++i) v[i] = e0 + i * FORK_THREADS < held ? from[e0 + i * FORK_THREADS] : 0;
#pragma unroll
  for (int i = 0; i < FORK_PER; ++i) {
    if (e0 + i * FORK_THREADS >= held) continue;
    int p = v[i];
    if (p < 0 || p >= a.pool.n_pages) paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE);
    else if (p >= used && a.map[p] >= 0) p = a.moves.list[3ll * a.map[p] + 1];
    to[e0 + i * FORK_THREADS] = p;
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Copy: the first `slots` slots of page `from` to page `to`, of every layer's keys and values.  Bound by HBM.  An item is up
// to 32 KB of one page of one layer's keys or values (COPY_PER 16-byte pieces per thread, all on their way before the first is
// stored); items go round a grid that fills the SMs.  Pieces run along whichever of heads and slots lies closer together.
// ------------------------------------------------------------------------------------------------------------------
constexpr int COPY_THREADS = 256, COPY_PER = 8, COPY_LAYERS = 64;   // layers per launch

struct CopyArgs {
  Moves moves;
  char* base[2 * COPY_LAYERS];            // keys, values, layer after layer
  long long page, head, slot;             // strides in 16-byte pieces
  int tensors, n_pages, page_size, heads, row_shift;   // row_shift: log2 of a slot's pieces
  int slot_first, chunks;                 // heads lie closer than slots; items of a whole page
};

__global__ void __launch_bounds__(COPY_THREADS) copy_kernel(const __grid_constant__ CopyArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int count = min(max(a.moves.count[0], 0), a.moves.capacity);
  const long long items = (long long)count * a.tensors * a.chunks;
  const int pr = 1 << a.row_shift;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int chunk = (int)(it % a.chunks);
    const long long r = it / a.chunks;
    const int tensor = (int)(r % a.tensors);
    const int32_t* m = a.moves.list + 3 * (r / a.tensors);
    const int from = m[0], to = m[1], slots = min(max(m[2], 0), a.page_size);
    if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) continue;
    const long long n = (long long)slots * a.heads << a.row_shift;
    uint4* const base = reinterpret_cast<uint4*>(a.base[tensor]);
    const uint4* const src = base + (long long)from * a.page;
    uint4* const dst = base + (long long)to * a.page;
    const long long i0 = (long long)chunk * (COPY_THREADS * COPY_PER) + threadIdx.x;
    uint4 v[COPY_PER];
    long long off[COPY_PER];
#pragma unroll
    for (int j = 0; j < COPY_PER; ++j) {
      const long long i = i0 + j * COPY_THREADS;
      off[j] = -1;
      if (i >= n) continue;
      const unsigned row = (unsigned)(i >> a.row_shift), inner = a.slot_first ? (unsigned)a.heads : (unsigned)slots;
      const unsigned o = row / inner, k = row - o * inner;
      off[j] = (a.slot_first ? o * a.slot + k * a.head : o * a.head + k * a.slot) + (i & (pr - 1));
      v[j] = src[off[j]];
    }
#pragma unroll
    for (int j = 0; j < COPY_PER; ++j)
      if (off[j] >= 0) dst[off[j]] = v[j];
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Launches and entry points
// ------------------------------------------------------------------------------------------------------------------
int no(int code, const char* msg) {
  sps_set_global_error(msg);
  return code;
}
int done(cudaError_t e) { return e == cudaSuccess ? SPS_OK : no(SPS_ECUDA, cudaGetErrorString(e)); }

template <class Args>
cudaError_t launch_cluster(void (*kern)(Args), int ctas, size_t smem, cudaStream_t st, const Args& a) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(POOL_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ctas; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = sps_pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, a);
}
// CTAs for a pool: a tile of 4096 pages each, up to a portable cluster
int pool_ctas(int n_pages) {
  int c = 1;
  while (c < 8 && (long long)c * POOL_THREADS * 4 < n_pages) c *= 2;
  return c;
}

const char* bad_pool(const sps_page_pool* p) {
  if (!p) return "null pool";
  if (p->n_pages < 1) return "pool: n_pages out of range";
  if (p->page_size < 8 || p->page_size > 512 || (p->page_size & (p->page_size - 1))) return "pool: page_size must be a power of two, 8 .. 512";
  if (!p->refs) return "pool: null pointer";
  if (((uintptr_t)p->refs | (uintptr_t)p->status) & 3) return "pool: pointers must be 4-byte aligned";
  return nullptr;
}
const char* bad_table(const sps_page_table* t) {
  if (!t) return "null table";
  if (t->B < 0 || t->B > PAGES_MAX_ROWS) return "table: B must be 0 .. 8192";
  if (t->ld < 0 || (int64_t)t->B * t->ld > INT_MAX) return "table: ld negative, or B x ld not below 2^31";
  if (t->B > 0 && (!t->held || !t->len || (!t->pages && t->ld > 0))) return "table: null pointer";
  if (((uintptr_t)t->pages | (uintptr_t)t->held | (uintptr_t)t->len) & 3) return "table: pointers must be 4-byte aligned";
  return nullptr;
}
const char* bad_moves(const sps_page_moves* m) {
  if (!m) return "null moves";
  if (m->capacity < 0) return "moves: capacity out of range";
  if (!m->count || (!m->list && m->capacity > 0)) return "moves: null pointer";
  if (((uintptr_t)m->list | (uintptr_t)m->count) & 3) return "moves: pointers must be 4-byte aligned";
  return nullptr;
}
const char* bad_workspace(const void* w) { return !w || ((uintptr_t)w & 15) ? "workspace null or not 16-byte aligned" : nullptr; }

Pool pool_of(const sps_page_pool* p) {
  Pool q{p->refs, p->status, p->n_pages, p->page_size, 0};
  while ((1 << q.page_shift) < p->page_size) ++q.page_shift;
  return q;
}
Table table_of(const sps_page_table* t) { return Table{t->pages, t->held, t->len, t->B, t->ld}; }
Moves moves_of(const sps_page_moves* m) { return Moves{m->list, m->count, m->capacity}; }
dim3 table_grid(int rows, int ld) { return dim3(rows, ld > 0 ? (ld + FORK_THREADS * FORK_PER - 1) / (FORK_THREADS * FORK_PER) : 1); }

}  // namespace

extern "C" {

int64_t sps_paged_pool_workspace_bytes(int32_t n_pages) {
  if (n_pages < 1) { no(SPS_EINVAL, "n_pages must be at least 1"); return -1; }
  return 256 + 3 * 4 * (((int64_t)n_pages + 63) / 64 * 64);
}

int sps_paged_fork(const sps_page_pool* pool, const sps_page_table* src, const sps_page_table* dst, const int32_t* parents, void* stream) {
  const char* why = bad_pool(pool);
  if (!why) why = bad_table(src);
  if (!why) why = bad_table(dst);
  if (why) return no(SPS_EINVAL, why);
  if (dst->ld < src->ld) return no(SPS_EINVAL, "fork: dst's rows are shorter than src's");
  if (dst->B > 0 && src->B > 0 && (dst->held == src->held || dst->len == src->len || (src->ld > 0 && dst->pages == src->pages)))
    return no(SPS_EINVAL, "fork: src and dst must not share their arrays");
  if ((dst->B > 0 && !parents) || ((uintptr_t)parents & 3)) return no(SPS_EINVAL, "parents null or not 4-byte aligned");
  const int rows = src->B > dst->B ? src->B : dst->B;
  if (rows == 0) return SPS_OK;
  ForkArgs a{pool_of(pool), table_of(src), table_of(dst), parents};
  return done(launch_k(fork_kernel, table_grid(rows, src->ld), dim3(FORK_THREADS), 0, (cudaStream_t)stream, a));
}

int sps_paged_reserve(const sps_page_pool* pool, const sps_page_table* table, const int32_t* want, const sps_page_moves* moves, void* workspace,
                      void* stream) {
  const char* why = bad_pool(pool);
  if (!why) why = bad_table(table);
  if (!why) why = bad_moves(moves);
  if (!why) why = bad_workspace(workspace);
  if (why) return no(SPS_EINVAL, why);
  if ((table->B > 0 && !want) || ((uintptr_t)want & 3)) return no(SPS_EINVAL, "want null or not 4-byte aligned");
  if (moves->capacity < table->B) return no(SPS_EINVAL, "moves: a row may need one, capacity is smaller than the table's B");
  ReserveArgs a{};
  a.pool = pool_of(pool); a.t = table_of(table); a.want = want; a.moves = moves_of(moves);
  const int64_t n = ((int64_t)pool->n_pages + 63) / 64 * 64;
  a.writers = (int32_t*)((char*)workspace + 256);
  a.first = a.writers + n;
  const size_t smem = sizeof(int) * 4 * (size_t)table->B;
  static DevSmemCache attr;
  cudaError_t e = sps_ensure_smem(reserve_kernel, smem, attr);
  if (e == cudaSuccess) e = launch_cluster(reserve_kernel, pool_ctas(pool->n_pages), smem, (cudaStream_t)stream, a);
  return done(e);
}

int sps_paged_compact(const sps_page_pool* pool, const sps_page_table* src, const sps_page_table* dst, int32_t* refs_out, const sps_page_moves* moves,
                      void* workspace, void* stream) {
  const char* why = bad_pool(pool);
  if (!why) why = bad_table(src);
  if (!why) why = bad_table(dst);
  if (!why) why = bad_moves(moves);
  if (!why) why = bad_workspace(workspace);
  if (why) return no(SPS_EINVAL, why);
  if (dst->B != src->B || dst->ld < src->ld) return no(SPS_EINVAL, "compact: dst must have src's rows, at least as long");
  if (dst->pages == src->pages && dst->ld != src->ld) return no(SPS_EINVAL, "compact: in place, src and dst must have the same ld");
  if (!refs_out || ((uintptr_t)refs_out & 3)) return no(SPS_EINVAL, "refs_out null or not 4-byte aligned");
  CompactArgs a{};
  a.pool = pool_of(pool); a.src = table_of(src); a.dst = table_of(dst); a.refs_out = refs_out; a.moves = moves_of(moves);
  const int64_t n = ((int64_t)pool->n_pages + 63) / 64 * 64;
  a.used = (int32_t*)workspace;
  a.map = (int32_t*)((char*)workspace + 256) + 2 * n;
  cudaError_t e = launch_cluster(compact_scan_kernel, pool_ctas(pool->n_pages), 0, (cudaStream_t)stream, a);
  if (e == cudaSuccess) e = launch_k(compact_apply_kernel, table_grid(src->B > 0 ? src->B : 1, src->ld), dim3(FORK_THREADS), 0, (cudaStream_t)stream, a);
  return done(e);
}

int sps_paged_copy(const sps_paged_cache* layers, int32_t n_layers, const sps_page_moves* moves, void* stream) {
  if (n_layers < 0 || (n_layers > 0 && !layers)) return no(SPS_EINVAL, "layers null, or n_layers negative");
  const char* why = bad_moves(moves);
  for (int l = 0; l < n_layers && !why; ++l) {
    why = paged_bad_cache(layers + l);
    const sps_paged_cache &c = layers[l], &f = layers[0];
    if (!why && (c.page_stride != f.page_stride || c.head_stride != f.head_stride || c.pos_stride != f.pos_stride || c.dtype != f.dtype || c.n_pages != f.n_pages ||
                 c.page_size != f.page_size || c.n_kv_heads != f.n_kv_heads || c.d_head != f.d_head))
      why = "copy: layers of unlike shape, strides or dtype";
  }
  if (why) return no(SPS_EINVAL, why);
  if (n_layers == 0 || moves->capacity == 0) return SPS_OK;
  const sps_paged_cache& f = layers[0];
  CopyArgs a{};
  a.moves = moves_of(moves);
  const int per16 = f.dtype == 0 ? 4 : 8;
  a.page = f.page_stride / per16; a.head = f.head_stride / per16; a.slot = f.pos_stride / per16;
  a.n_pages = f.n_pages; a.page_size = f.page_size; a.heads = f.n_kv_heads;
  while ((per16 << a.row_shift) < f.d_head) ++a.row_shift;
  a.slot_first = f.n_kv_heads > 1 && f.head_stride < f.pos_stride;
  const long long pieces = (long long)f.page_size * f.n_kv_heads << a.row_shift;
  a.chunks = (int)((pieces + COPY_THREADS * COPY_PER - 1) / (COPY_THREADS * COPY_PER));
  for (int l = 0; l < n_layers; l += COPY_LAYERS) {
    const int n = n_layers - l < COPY_LAYERS ? n_layers - l : COPY_LAYERS;
    for (int i = 0; i < n; ++i) { a.base[2 * i] = (char*)layers[l + i].k; a.base[2 * i + 1] = (char*)layers[l + i].v; }
    a.tensors = 2 * n;
    const long long items = (long long)moves->capacity * a.tensors * a.chunks, most = (long long)paged_sms() * 6;
    const cudaError_t e = launch_k(copy_kernel, dim3((unsigned)(items < most ? items : most)), dim3(COPY_THREADS), 0, (cudaStream_t)stream, a);
    if (e != cudaSuccess) return done(e);
  }
  return SPS_OK;
}

}  // extern "C"
