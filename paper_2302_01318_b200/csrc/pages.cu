// Which pages the sequences of a paged cache have: tables reordered by parents (fork), pages given up, exchanged and taken
// (reserve), a pool moved together (compact), and the copies these leave to do (copy), with their C entry points.
#include <cooperative_groups.h>

#include <climits>

#include "paged.cuh"

namespace cg = cooperative_groups;

#define PAGES_MAX (1 << 20)    // pages of a pool: their bits fit the shared memory of eight CTAs
#define PAGES_MAX_ROWS 8192   // rows of a table: a thread each of a cluster of eight CTAs

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
  // as a row of src: what it gives up or hands on; as a row of dst: what it gets (both on their way before either is looked at)
  const bool is_src = row < a.src.B, is_dst = row < a.dst.B;
  const int gives = is_src ? row_held(a.src, a.pool, row) : 0, parent = is_dst ? a.parents[row] : -1;
  const bool there = parent >= 0 && parent < a.src.B;
  const int gets = there ? row_held(a.src, a.pool, parent) : 0;
  const int32_t* const mine = a.src.pages + (long long)(is_src ? row : 0) * a.src.ld;
  const int32_t* const from = a.src.pages + (long long)(there ? parent : 0) * a.src.ld;
  int v[FORK_PER], u[FORK_PER], children = 0;
#pragma unroll
  for (int i = 0; i < FORK_PER; ++i) {
    const int e = e0 + i * FORK_THREADS;
    u[i] = e < gives ? mine[e] : 0;
    v[i] = e < gets ? from[e] : 0;
  }
  if (is_src)
    for (int b0 = 0; b0 < a.dst.B; b0 += FORK_THREADS) children += __syncthreads_count(b0 + tid < a.dst.B && a.parents[b0 + tid] == row);
  if (is_dst) {
    if (blockIdx.y == 0 && tid == 0) {
      if (parent < -1 || parent >= a.src.B) paged_flag(a.pool.status, SPS_PAGED_BAD_ROW);
      a.dst.held[row] = gets;
      a.dst.len[row] = there ? a.src.len[parent] : 0;
    }
    int32_t* const to = a.dst.pages + (long long)row * a.dst.ld;
#pragma unroll
    for (int i = 0; i < FORK_PER; ++i)
      if (e0 + i * FORK_THREADS < gets) to[e0 + i * FORK_THREADS] = v[i];
  }
  unsigned top = 0;   // (what is not there is page 0; below 0 is far above)
#pragma unroll
  for (int i = 0; i < FORK_PER; ++i) top = max(top, (unsigned)u[i]);
  if (top >= (unsigned)a.pool.n_pages) paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE);
  if (is_src && children != 1) {
#pragma unroll
    for (int i = 0; i < FORK_PER; ++i)
      if (e0 + i * FORK_THREADS < gives && (unsigned)u[i] < (unsigned)a.pool.n_pages) atomicAdd(a.pool.refs + u[i], children - 1);
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Helpers of the pool kernels: one cluster, 1024 threads to a CTA
// ------------------------------------------------------------------------------------------------------------------
constexpr int POOL_THREADS = 1024, POOL_WARPS = POOL_THREADS / 32;
constexpr int POOL_WORDS = 4096;   // of 32 pages each, that a CTA may have: pools of 2^20 pages in a cluster of eight

// inclusive sums over the block's threads, in thread order; s_warp: [POOL_WARPS]; total: the block's
__device__ __forceinline__ int2 block_scan(int2 v, int2* s_warp, int2* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto scan = [&](int2 x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u0 = __shfl_up_sync(0xffffffffu, x.x, o), u1 = __shfl_up_sync(0xffffffffu, x.y, o);
      if (lane >= o) { x.x += u0; x.y += u1; }
    }
    return x;
  };
  v = scan(v);
  __syncthreads();   // (s_warp may still be read from the last call)
  if (lane == 31) s_warp[warp] = v;
  __syncthreads();
  const int2 w = scan(s_warp[lane]);
  total->x = __shfl_sync(0xffffffffu, w.x, 31);
  total->y = __shfl_sync(0xffffffffu, w.y, 31);
  const int b0 = __shfl_sync(0xffffffffu, w.x, (warp + 31) & 31), b1 = __shfl_sync(0xffffffffu, w.y, (warp + 31) & 31);
  return warp > 0 ? make_int2(v.x + b0, v.y + b1) : v;
}
__device__ __forceinline__ void block_add(int v, int* s_sum) {   // *s_sum is complete after the next barrier
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0 && v) atomicAdd(s_sum, v);
}

// The pool's references as bits in shared memory, a page's set where it is in use; a CTA has the pages lo .. hi - 1, whole words
// of them.  A warp reads 32 neighbouring references and votes; words go round the warps.
struct PoolPart { int lo, hi, words; };
__device__ __forceinline__ PoolPart pool_part(int n_pages, int rank, int parts) {
  const int per = ((n_pages + 31) / 32 + parts - 1) / parts * 32;
  PoolPart p;
  p.lo = min(per * rank, n_pages);
  p.hi = min(p.lo + per, n_pages);
  p.words = (p.hi - p.lo + 31) / 32;
  return p;
}
// references are read from L2 (other CTAs changed them), four to a lane if they are aligned, and copied to `copy` if that is given
__device__ __forceinline__ void used_bits(const int32_t* refs, const PoolPart& p, uint32_t* s_bits, int32_t* copy = nullptr) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int w0 = 0;   // words done
  if (((uintptr_t)refs & 15) == 0) {
    const int fours = (p.hi - p.lo) / 128;   // four words to a load
    for (int f0 = warp; f0 < fours; f0 += 8 * POOL_WARPS) {
      int4 r[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (f0 + i * POOL_WARPS < fours) r[i] = __ldcg(reinterpret_cast<const int4*>(refs + p.lo) + (f0 + i * POOL_WARPS) * 32 + lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int f = f0 + i * POOL_WARPS;
        if (f >= fours) break;
        uint32_t v = ((r[i].x != 0) | (r[i].y != 0) << 1 | (r[i].z != 0) << 2 | (r[i].w != 0) << 3) << (lane & 7) * 4;
        v |= __shfl_xor_sync(0xffffffffu, v, 1);
        v |= __shfl_xor_sync(0xffffffffu, v, 2);
        v |= __shfl_xor_sync(0xffffffffu, v, 4);
        if ((lane & 7) == 0) s_bits[f * 4 + (lane >> 3)] = v;
        if (copy) {
          int32_t* const c = copy + p.lo + (f * 32 + lane) * 4;
          c[0] = r[i].x; c[1] = r[i].y; c[2] = r[i].z; c[3] = r[i].w;
        }
      }
    }
    w0 = fours * 4;
  }
  for (w0 += warp; w0 < p.words; w0 += 4 * POOL_WARPS) {
    int r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int page = p.lo + (w0 + i * POOL_WARPS) * 32 + lane;
      r[i] = page < p.hi ? __ldcg(refs + page) : 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int w = w0 + i * POOL_WARPS, page = p.lo + w * 32 + lane;
      if (w >= p.words) break;
      const uint32_t v = __ballot_sync(0xffffffffu, r[i] != 0);
      if (lane == 0) s_bits[w] = v;
      if (copy && page < p.hi) copy[page] = r[i];
    }
  }
}
__device__ __forceinline__ uint32_t existing_bits(int page, int hi) {   // of the 32 pages from `page` on, those below hi
  return page + 32 <= hi ? 0xffffffffu : (page < hi ? (1u << (hi - page)) - 1u : 0u);
}
// fn(word, its bits, page, lane) for every page of this CTA's words w0 .. w0 + 1023, a warp to a word
template <class Fn>
__device__ __forceinline__ void for_pages(const PoolPart& p, const uint32_t* s_bits, int w0, Fn fn) {
  const int lane = threadIdx.x & 31, end = min(w0 + POOL_THREADS, p.words);
#pragma unroll 4
  for (int w = w0 + (threadIdx.x >> 5); w < end; w += POOL_WARPS) fn(w, s_bits[w], p.lo + w * 32 + lane, lane);
}

// use(row, i, load(row, i)) for i < count of every row of the CTA (a row per thread), by threads of a warp for neighbouring i: rows of
// one or two by their own thread, the others, listed in any order, by a warp each or, where one of them is long, in runs of
// 256 that go round the warps.  *s_rows: 0, and left so
template <class Load, class Use>
__device__ __forceinline__ void for_entries(int count, int* s_rows, int* s_end, int* s_count, int2* s_warp, Load load, Use use) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool few = count <= 2;
  if (few && count > 0) {
    const int v0 = load(tid, 0), v1 = count > 1 ? load(tid, 1) : 0;
    use(tid, 0, v0);
    if (count > 1) use(tid, 1, v1);
  }
  s_count[tid] = count;
  if (!few) s_end[atomicAdd(s_rows, 1)] = tid;
  if (!__syncthreads_or(!few)) return;
  const int rows = *s_rows;
  auto run = [&](int r, int i0, int n) {
    int v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i0 + 32 * j < n ? load(r, i0 + 32 * j) : 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i0 + 32 * j < n) use(r, i0 + 32 * j, v[j]);
  };
  const bool any_long = __syncthreads_or(count > 1024);
  if (tid == 0) *s_rows = 0;
  if (!any_long) {
    for (int x = warp; x < rows; x += POOL_WARPS) {
      const int r = s_end[x], n = s_count[r];
      for (int i0 = lane; i0 - lane < n; i0 += 256) run(r, i0, n);
    }
    return;
  }
  int2 all;
  s_end[tid] = block_scan(make_int2(few ? 0 : (count + 255) / 256, 0), s_warp, &all).x;
  __syncthreads();
  for (int u = warp; u < all.x; u += POOL_WARPS) {
    int x = 0, y = POOL_THREADS - 1;   // the row of the u-th run: the first whose runs end behind it
    while (x < y) {
      const int m = (x + y) >> 1;
      if (s_end[m] > u) y = m; else x = m + 1;
    }
    run(x, (u - (x ? s_end[x - 1] : 0)) * 256 + lane, s_count[x]);
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Reserve.  With n = min(len, want) tokens kept in k = ceil(n / page) pages, a row (1) gives up its entries behind k, (2)
// exchanges entry k - 1 for a fresh page if it is partly filled, about to be written and held by others too -- unless all who
// hold it write to it and this row is the one of them that keeps it --, and (3) takes fresh pages up to want tokens.  Fresh pages are the
// lowest free ones, handed out row after row: a prefix sum over the rows' needs and one over the pool's free pages meet in
// a list of the pages handed out.
// Who keeps it: where all rows get what they need, the first, since the others' copies are made before anyone appends.  Where
// pages are short one of the others may go without and keep its tokens there: then the one with the most tokens, the first of
// those, which writes behind what the others have.  The needs' total is the same either way, so that is known beforehand.
//
// One cluster does it all, a thread to a row (its state stays in registers), a part of the pool to a CTA, the steps divided by
// cluster barriers: giving up -> marks at shared last pages, free pages -> needs -> list -> entries.  What it costs is those
// steps' trips to L2, one behind the other; the references are read once (4 bytes a page).
// Marks: per page the number of rows about to write to it and B - (the first of them), where pages are short the one with the most
// tokens; in the workspace, zero between calls.
// ------------------------------------------------------------------------------------------------------------------
struct ReserveArgs {
  Pool pool;
  Table t;
  const int32_t* want;
  int32_t* room;              // or null
  Moves moves;
  int32_t *writers, *first;   // [n_pages], zero
  int32_t* fresh;             // [n_pages]: the pages handed out
};

// a row's claim to keep a page of which it has n tokens (above 0): the largest keeps it
__device__ __forceinline__ int keep_claim(int n, int page_size, int row) { return (n & (page_size - 1)) * PAGES_MAX_ROWS + PAGES_MAX_ROWS - 1 - row; }

struct RowPlan { int n, keep, want, to, give, q; };   // tokens and pages kept, tokens and pages wanted, entries given up, the page about to be written (-1: none)
__device__ __forceinline__ RowPlan row_plan(const ReserveArgs& a, int b) {
  RowPlan r;
  const int held0 = a.t.held[b], len0 = a.t.len[b], want0 = a.want[b];
  const int cap = (int)min((long long)a.t.ld << a.pool.page_shift, (long long)INT_MAX - a.pool.page_size);
  const int held = min(max(held0, 0), a.t.ld), room = (int)min((long long)held << a.pool.page_shift, (long long)cap), want = min(max(want0, 0), cap);
  if (held != held0 || len0 < 0 || len0 > room || want0 < 0 || want0 > cap) paged_flag(a.pool.status, SPS_PAGED_BAD_LENGTH);
  r.n = min(min(max(len0, 0), room), want);
  r.keep = (r.n + a.pool.page_size - 1) >> a.pool.page_shift;
  r.want = want;
  r.to = (want + a.pool.page_size - 1) >> a.pool.page_shift;
  r.give = held - r.keep;
  r.q = -1;
  if ((r.n & (a.pool.page_size - 1)) && want > r.n) {
    r.q = a.t.pages[(long long)b * a.t.ld + r.keep - 1];
    if (r.q < 0 || r.q >= a.pool.n_pages) { paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE); r.q = -1; }
  }
  return r;
}

__global__ void __launch_bounds__(POOL_THREADS) reserve_kernel(const __grid_constant__ ReserveArgs a) {
  __shared__ int s_end[POOL_THREADS], s_count[POOL_THREADS], s_from[POOL_THREADS], s_at[POOL_THREADS];
  __shared__ int2 s_warp[POOL_WARPS];
  __shared__ uint32_t s_bits[POOL_WORDS];
  __shared__ int s_rows, s_free, s_met, s_sums[3][8];   // this CTA's free pages; what is met where not all is; every CTA's free pages, needs and moves
  cg::cluster_group cl = cg::this_cluster();   // (at the first barrier every CTA is there to be written to)
  const int rank = (int)cl.block_rank(), parts = (int)cl.num_blocks(), tid = threadIdx.x, B = a.t.B;
  const int per = (B + parts - 1) / parts, b = rank * per + tid;
  const bool row = tid < per && b < B;
  const PoolPart part = pool_part(a.pool.n_pages, rank, parts);
  pdl_launch_dependents();
  pdl_wait();

  // (1) the row's plan, and what it gives up
  const auto [n, keep, want, to, give, q] = row ? row_plan(a, b) : RowPlan{0, 0, 0, 0, 0, -1};
  s_from[tid] = keep;
  if (tid == 0) { s_free = 0; s_rows = 0; }
  __syncthreads();
  for_entries(give, &s_rows, s_end, s_count, s_warp, [&](int r, int i) { return a.t.pages[(long long)(rank * per + r) * a.t.ld + s_from[r] + i]; }, [&](int, int, int p) {
    if (p < 0 || p >= a.pool.n_pages) paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE);
    else atomicAdd(a.pool.refs + p, -1);
  });
  cl.sync();
  // (2) marks at pages that are shared and about to be written; the free pages
  const int shared = q >= 0 ? __ldcg(a.pool.refs + q) : 0;
  if (shared > 1) {
    atomicAdd(a.writers + q, 1);
    atomicMax(a.first + q, B - b);
  }
  used_bits(a.pool.refs, part, s_bits);
  __syncthreads();
  int free_pages = 0;
  for (int w = tid; w < part.words; w += POOL_THREADS) {
    const uint32_t v = ~s_bits[w] & existing_bits(part.lo + w * 32, part.hi);
    s_bits[w] = v;   // (the free ones from here on)
    free_pages += __popc(v);
  }
  block_add(free_pages, &s_free);
  cl.sync();
  // (3) needs, summed in the rows' order, and every CTA told the others' sums
  const int more = row ? max(to - keep, 0) : 0;   // pages behind those that it has
  const bool all_write = shared > 1 && __ldcg(a.writers + q) == shared;
  bool swap = shared > 1 && !(all_write && __ldcg(a.first + q) == B - b);
  int2 sum;
  int need, end, moves_end, free_before, free_all, need_all, moves_all;
  auto add_up = [&]() {
    need = more + swap;
    const int2 ends = block_scan(make_int2(need, swap), s_warp, &sum);
    if (tid < parts) {
      int* const s = cl.map_shared_rank(&s_sums[0][0], tid);
      s[rank] = s_free; s[8 + rank] = sum.x; s[16 + rank] = sum.y;
    }
    cl.sync();
    end = ends.x; moves_end = ends.y;
    free_before = free_all = need_all = moves_all = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      if (c >= parts) break;
      const int f = s_sums[0][c], n0 = s_sums[1][c], m = s_sums[2][c];
      if (c < rank) { free_before += f; end += n0; moves_end += m; }
      free_all += f; need_all += n0; moves_all += m;
    }
  };
  add_up();
  if (need_all > free_all) {
    if (all_write) a.first[q] = 0;   // (all have read it)
    cl.sync();
    const int claim = keep_claim(n, a.pool.page_size, b);
    if (all_write) atomicMax(a.first + q, claim);
    cl.sync();
    swap = shared > 1 && !(all_write && __ldcg(a.first + q) == claim);
    add_up();
    // the rows behind the first that goes without do so too: what the ones before it need, and their moves
    if (row && need > 0 && end > free_all) paged_flag(a.pool.status, SPS_PAGED_NO_PAGE);
    s_met = 0;
    __syncthreads();
    if (row && end <= free_all) atomicMax(&s_met, end);
    cl.sync();
    need_all = 0;
    for (int c = 0; c < parts; ++c) need_all = max(need_all, *cl.map_shared_rank(&s_met, c));
    cl.sync();
    if (tid == 0) s_met = 0;
    __syncthreads();
    if (row && end <= free_all) atomicMax(&s_met, moves_end);
    cl.sync();
    moves_all = 0;
    for (int c = 0; c < parts; ++c) moves_all = max(moves_all, *cl.map_shared_rank(&s_met, c));
  }
  // (4) the rows' new state, the pages that they exchange, and the list of fresh pages
  const bool served = need > 0 && end <= need_all;
  if (row) {
    a.t.held[b] = served ? max(to, keep) : keep;
    a.t.len[b] = n;
    if (a.room) a.room[b] = served || need == 0 ? want : n;
    if (served && swap) {
      atomicAdd(a.pool.refs + q, -1);
      int32_t* m = a.moves.list + 3ll * (moves_end - 1);
      m[0] = q;
      m[2] = n & (a.pool.page_size - 1);
    }
    if (shared > 1) { a.writers[q] = 0; a.first[q] = 0; }
  }
  if (b == 0 && tid == 0) a.moves.count[0] = moves_all;
  for (int w0 = 0, at = free_before; w0 < part.words && at < need_all; w0 += POOL_THREADS) {
    const int count = w0 + tid < part.words ? __popc(s_bits[w0 + tid]) : 0;
    s_count[tid] = at - count + block_scan(make_int2(count, 0), s_warp, &sum).x;   // (for_entries is done with it)
    __syncthreads();
    at += sum.x;
    for_pages(part, s_bits, w0, [&](int w, uint32_t v, int page, int lane) {
      const int j = s_count[w - w0] + __popc(v & ((1u << lane) - 1u));
      if ((v >> lane & 1) && j < need_all) { a.fresh[j] = page; a.pool.refs[page] = 1; }
    });
    __syncthreads();
  }
  cl.sync();
  // (5) the rows' entries from the list
  const int take = served ? need : 0;
  s_from[tid] = end - need;
  s_at[tid] = keep - swap;
  for_entries(take, &s_rows, s_end, s_count, s_warp, [&](int r, int i) { return __ldcg(a.fresh + s_from[r] + i); },
              [&](int r, int i, int p) { a.t.pages[(long long)(rank * per + r) * a.t.ld + s_at[r] + i] = p; });
  if (served && swap) a.moves.list[3ll * (moves_end - 1) + 1] = __ldcg(a.fresh + end - need);
}

// The same for pools whose references fit a CTA's shared memory, and a table of a row per thread: the steps' counts, marks and
// list are kept there, and trips to L2 are only the rows, the references and the entries.  A beam step of 4 rows takes 9.5 us with
// this kernel and 12.2 with the cluster's, one of 64 rows in a pool of 700 pages 23.1 and 26.3.  64 rows with a scoring pass's room:
// 3.9 us and 5.9 in a pool of 830 pages, 5.6 and 6.8 of 16606; with half of them coming and going 6.3 and 7.9, 11.6 and 10.6.  Changes
// of references go to both places.
constexpr int SMALL_PAGES = 24576;   // two words each

__global__ void __launch_bounds__(POOL_THREADS) reserve_small_kernel(const __grid_constant__ ReserveArgs a) {
  extern __shared__ int4 s_dyn[];
  __shared__ int s_end[POOL_THREADS], s_count[POOL_THREADS], s_from[POOL_THREADS], s_at[POOL_THREADS];
  __shared__ int2 s_warp[POOL_WARPS];
  __shared__ uint32_t s_bits[SMALL_PAGES / 32];
  __shared__ int s_rows, s_free, s_need, s_moves;
  const int tid = threadIdx.x, lane = tid & 31, B = a.t.B, n_pages = a.pool.n_pages, words = (n_pages + 31) / 32;
  int* const s_refs = (int*)s_dyn;             // [words * 32]
  int* const s_first = s_refs + words * 32;    // first of those who write to a page; then the list of fresh pages
  const bool row = tid < B;
  pdl_launch_dependents();
  pdl_wait();
  if (((uintptr_t)a.pool.refs & 15) == 0) {
    for (int i = tid; i < n_pages / 4; i += POOL_THREADS) s_dyn[i] = reinterpret_cast<const int4*>(a.pool.refs)[i];
    for (int i = n_pages / 4 * 4 + tid; i < words * 32; i += POOL_THREADS) s_refs[i] = i < n_pages ? a.pool.refs[i] : 1;
  } else {
    for (int i = tid; i < words * 32; i += POOL_THREADS) s_refs[i] = i < n_pages ? a.pool.refs[i] : 1;
  }
  const auto [n, keep, want, to, give, q] = row ? row_plan(a, tid) : RowPlan{0, 0, 0, 0, 0, -1};
  s_from[tid] = keep;
  if (tid == 0) { s_rows = 0; s_free = 0; s_need = 0; s_moves = 0; }
  __syncthreads();
  for_entries(give, &s_rows, s_end, s_count, s_warp, [&](int r, int i) { return a.t.pages[(long long)r * a.t.ld + s_from[r] + i]; }, [&](int, int, int p) {
    if (p < 0 || p >= n_pages) { paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE); return; }
    atomicAdd(s_refs + p, -1);
    atomicAdd(a.pool.refs + p, -1);
  });
  __syncthreads();
  // who writes to a shared page gives it up; where nothing is left the first of them takes it back
  const bool writes = q >= 0 && s_refs[q] > 1;
  if (writes) s_first[q] = B;
  __syncthreads();
  if (writes) {
    atomicSub(s_refs + q, 1);
    atomicMin(s_first + q, tid);
  }
  __syncthreads();
  const bool all_write = writes && s_refs[q] == 0;
  bool swap = writes && !(all_write && s_first[q] == tid);
  const int more = row ? max(to - keep, 0) : 0;   // pages behind those that it has
  int need = more + swap;
  __syncthreads();
  if (writes && !swap) s_refs[q] = 1;
  int2 all;
  int2 ends = block_scan(make_int2(need, swap), s_warp, &all);   // (its barriers: s_refs is complete, s_first free)
  int free_pages = 0;
  for (int w = tid >> 5; w < words; w += POOL_WARPS) {
    const uint32_t v = __ballot_sync(0xffffffffu, s_refs[w * 32 + lane] == 0);
    if (lane == 0) s_bits[w] = v;
    free_pages += __popc(v);
  }
  if (lane == 0 && free_pages) atomicAdd(&s_free, free_pages);
  __syncthreads();
  const int free_all = s_free;
  int need_all = all.x, moves_all = all.y;
  if (need_all > free_all) {
    if (all_write) s_first[q] = 0;
    __syncthreads();
    const int claim = keep_claim(n, a.pool.page_size, tid);
    if (all_write) atomicMax(s_first + q, claim);
    __syncthreads();
    swap = writes && !(all_write && s_first[q] == claim);
    need = more + swap;
    ends = block_scan(make_int2(need, swap), s_warp, &all);
    // what the rows ahead of the first that goes without need, and their moves
    if (need > 0 && ends.x > free_all) paged_flag(a.pool.status, SPS_PAGED_NO_PAGE);
    if (row && ends.x <= free_all) { atomicMax(&s_need, ends.x); atomicMax(&s_moves, ends.y); }
    __syncthreads();
    need_all = s_need;
    moves_all = s_moves;
  }
  const bool served = need > 0 && ends.x <= need_all;
  if (row) {
    a.t.held[tid] = served ? max(to, keep) : keep;
    a.t.len[tid] = n;
    if (a.room) a.room[tid] = served || need == 0 ? want : n;
    if (served && swap) {
      atomicAdd(a.pool.refs + q, -1);
      int32_t* m = a.moves.list + 3ll * (ends.y - 1);
      m[0] = q;
      m[2] = n & (a.pool.page_size - 1);
    }
  }
  if (tid == 0) a.moves.count[0] = moves_all;
  if (need_all == 0) return;
  const int count = tid < words ? __popc(s_bits[tid]) : 0;
  s_count[tid] = block_scan(make_int2(count, 0), s_warp, &all).x - count;
  __syncthreads();
  for (int w = tid >> 5; w < words; w += POOL_WARPS) {
    const uint32_t v = s_bits[w];
    const int j = s_count[w] + __popc(v & ((1u << lane) - 1u));
    if ((v >> lane & 1) && j < need_all) { s_first[j] = w * 32 + lane; a.pool.refs[w * 32 + lane] = 1; }
  }
  s_from[tid] = ends.x - need;
  s_at[tid] = keep - swap;
  __syncthreads();
  for_entries(served ? need : 0, &s_rows, s_end, s_count, s_warp, [&](int r, int i) { return s_first[s_from[r] + i]; },
              [&](int r, int i, int p) { a.t.pages[(long long)r * a.t.ld + s_at[r] + i] = p; });
  if (served && swap) a.moves.list[3ll * (ends.y - 1) + 1] = s_first[ends.x - need];
}

// ------------------------------------------------------------------------------------------------------------------
// Compact: of U pages in use, those numbered U and above go to the free ones below U, the i-th to the i-th.
// First a cluster over the pool, its references read once: U, the holes below it, then each page's place among the holes or
// among those that move; then a grid over the table's entries and the list.  map[p]: where page p >= U stands in the list, -1 if
// it stays (nothing in use, or the list is full).
// ------------------------------------------------------------------------------------------------------------------
struct CompactArgs {
  Pool pool;
  Table src, dst;
  int32_t* refs_out;
  Moves moves;
  int32_t *map, *used;   // [n_pages], [1]
  int apply;             // by the scan's only CTA: little to carry out
};

// the moves carried out in references and table by `workers` warps, of which this is one: pages' references go with them, entries are
// renamed, 256 of a row at a time
__device__ __forceinline__ void compact_apply(const CompactArgs& a, int worker, int workers) {
  const int lane = threadIdx.x & 31, count = a.moves.count[0], used = a.used[0], chunks = max((a.src.ld + 255) / 256, 1);
  for (int i = worker * 32 + lane; i < count; i += workers * 32) {
    const int from = a.moves.list[3ll * i], to = a.moves.list[3ll * i + 1], r = a.pool.refs[from];
    a.refs_out[to] = r;
    a.refs_out[from] = 0;
  }
  for (long long u = worker; u < (long long)a.src.B * chunks; u += workers) {
    const int row = (int)(u / chunks), e0 = (int)(u - (long long)row * chunks) * 256 + lane;
    const int held = row_held(a.src, a.pool, row);
    if (e0 == 0) {
      a.dst.held[row] = held;
      a.dst.len[row] = a.src.len[row];
    }
    const int32_t* from = a.src.pages + (long long)row * a.src.ld;
    int32_t* to = a.dst.pages + (long long)row * a.dst.ld;
    int v[8], m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e0 + i * 32 < held ? from[e0 + i * 32] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = v[i] >= used && v[i] < a.pool.n_pages ? a.map[v[i]] : -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (e0 + i * 32 >= held) continue;
      if (v[i] < 0 || v[i] >= a.pool.n_pages) paged_flag(a.pool.status, SPS_PAGED_BAD_PAGE);
      to[e0 + i * 32] = m[i] >= 0 ? a.moves.list[3ll * m[i] + 1] : v[i];
    }
  }
}
__global__ void __launch_bounds__(POOL_THREADS) compact_scan_kernel(const __grid_constant__ CompactArgs a) {
  __shared__ int2 s_warp[POOL_WARPS];
  __shared__ uint32_t s_bits[POOL_WORDS];
  __shared__ int s_rank[POOL_THREADS], s_n[2], s_sums[2][8];
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), parts = (int)cl.num_blocks(), tid = threadIdx.x;
  const PoolPart part = pool_part(a.pool.n_pages, rank, parts);
  if (tid < 2) s_n[tid] = 0;
  pdl_launch_dependents();
  pdl_wait();
  cl.sync();   // (every CTA is there to be written to)
  auto tell = [&](int i) {   // this CTA's sum to all, everyone's from all
    __syncthreads();
    if (tid < parts) cl.map_shared_rank(&s_sums[i][0], tid)[rank] = s_n[i];
    cl.sync();
    int2 all = make_int2(0, 0);   // of the CTAs before this one, of all
    for (int c = 0; c < parts; ++c) {
      if (c < rank) all.x += s_sums[i][c];
      all.y += s_sums[i][c];
    }
    return all;
  };
  used_bits(a.pool.refs, part, s_bits, a.refs_out != a.pool.refs ? a.refs_out : nullptr);
  __syncthreads();
  int mine = 0;
  for (int w = tid; w < part.words; w += POOL_THREADS) mine += __popc(s_bits[w]);
  block_add(mine, &s_n[0]);
  const int2 in_use = tell(0);
  const int used = in_use.y;
  mine = 0;
  for (int w = tid; w < part.words; w += POOL_THREADS) mine += __popc(s_bits[w] & existing_bits(part.lo + w * 32, used));
  block_add(mine, &s_n[1]);
  const int stay = tell(1).y;   // pages in use below U
  if (rank == 0 && tid == 0) {
    a.used[0] = used;
    a.moves.count[0] = min(used - stay, a.moves.capacity);
  }
  for (int w0 = 0, at = in_use.x; w0 < part.words; w0 += POOL_THREADS) {
    const int count = w0 + tid < part.words ? __popc(s_bits[w0 + tid]) : 0;
    int2 sum;
    s_rank[tid] = at - count + block_scan(make_int2(count, 0), s_warp, &sum).x;   // pages in use before the word's
    __syncthreads();
    at += sum.x;
    for_pages(part, s_bits, w0, [&](int w, uint32_t v, int page, int lane) {
      if (page >= part.hi) return;
      const bool in = v >> lane & 1;
      const int before = s_rank[w - w0] + __popc(v & ((1u << lane) - 1u));
      if (page < used) {
        if (!in && page - before < a.moves.capacity) a.moves.list[3ll * (page - before) + 1] = page;
      } else {
        const int j = before - stay;
        const bool goes = in && j < a.moves.capacity;
        a.map[page] = goes ? j : -1;
        if (goes) {
          a.moves.list[3ll * j] = page;
          a.moves.list[3ll * j + 2] = a.pool.page_size;
        }
      }
    });
    __syncthreads();
  }
  if (a.apply) compact_apply(a, tid >> 5, POOL_WARPS);
}

__global__ void __launch_bounds__(FORK_THREADS) compact_apply_kernel(const __grid_constant__ CompactArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  compact_apply(a, (int)(blockIdx.x * (FORK_THREADS / 32) + (threadIdx.x >> 5)), (int)(gridDim.x * (FORK_THREADS / 32)));
}

// ------------------------------------------------------------------------------------------------------------------
// Copy: the first `slots` slots of page `from` to page `to`, of every layer's keys and values.  Bound by HBM, which likes long
// runs of reads and of writes: a thread has PER 16-byte pieces on their way before the first is stored.  805 MB in whole pages of
// 32 KB take 248 us with PER 16 and 258 with 8; a beam step with 64 rows' partly filled pages in 24 layers takes 31 us with 16 and 26
// with 4, where CTAs without an item are the cost: the list's capacity, all that the host knows, decides.  A unit is such a run at one
// place of a page of one layer's keys or values; a CTA keeps to its unit and goes from page to page.  Pieces run along
// whichever of heads and slots lies closer together.
// ------------------------------------------------------------------------------------------------------------------
constexpr int COPY_THREADS = 256, COPY_LAYERS = 64;   // layers: per launch
constexpr long long COPY_MUCH = 512ll << 20;          // bytes of a full list that are much

struct CopyArgs {
  Moves moves;
  char* base[2 * COPY_LAYERS];            // keys, values, layer after layer
  long long page, head, slot;             // strides in 16-byte pieces
  int units, chunks;                      // tensors x chunks; chunks: of a whole page
  int n_pages, page_size, heads, row_shift;   // row_shift: log2 of a slot's pieces
  int slot_first;                         // heads lie closer than slots
};

template <int PER>
__global__ void __launch_bounds__(COPY_THREADS) copy_kernel(const __grid_constant__ CopyArgs a) {
  pdl_launch_dependents();
  const int first = blockIdx.x / a.units, unit = blockIdx.x - first * a.units, step = gridDim.x / a.units;
  const int tensor = unit / a.chunks, chunk = unit - tensor * a.chunks;
  const int piece = chunk * (COPY_THREADS * PER) + threadIdx.x;
  uint4* const base = reinterpret_cast<uint4*>(a.base[tensor]) + (piece & ((1 << a.row_shift) - 1));
  pdl_wait();
  const int count = min(max(a.moves.count[0], 0), a.moves.capacity);
  int had = -1, n = 0;
  long long off[PER];   // of this thread's pieces in a page, for `had` slots
  int next[3] = {0, 0, 0};   // the next item, read while this one is copied
  auto read = [&](int i) {
    if (i < count) { next[0] = a.moves.list[3ll * i]; next[1] = a.moves.list[3ll * i + 1]; next[2] = a.moves.list[3ll * i + 2]; }
  };
  read(first);
  for (int i = first; i < count; i += step) {
    const int from = next[0], to = next[1], slots = min(max(next[2], 0), a.page_size);
    read(i + step);
    if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) continue;
    if (slots != had) {
      had = slots;
      n = slots * a.heads << a.row_shift;
      const unsigned inner = a.slot_first ? (unsigned)a.heads : (unsigned)max(slots, 1);
      const long long so = a.slot_first ? a.slot : a.head, si = a.slot_first ? a.head : a.slot;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const unsigned row = (unsigned)(piece + j * COPY_THREADS) >> a.row_shift, o = row / inner;
        off[j] = o * so + (row - o * inner) * si;
      }
    }
    const uint4* const src = base + (long long)from * a.page;
    uint4* const dst = base + (long long)to * a.page;
    uint4 v[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (piece + j * COPY_THREADS < n) v[j] = src[off[j]];
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (piece + j * COPY_THREADS < n) dst[off[j]] = v[j];
  }
}

template <int PER, int CTAS>   // CTAs: per SM
cudaError_t copy_launch(CopyArgs& a, int tensors, int num_sm, cudaStream_t st) {
  const int pieces = a.page_size * a.heads << a.row_shift;   // at most 512 x 4096 x 32
  a.chunks = (pieces + COPY_THREADS * PER - 1) / (COPY_THREADS * PER);
  a.units = tensors * a.chunks;
  int at_once = num_sm * CTAS / a.units;   // pages: as many as fill the SMs
  at_once = at_once < 1 ? 1 : (at_once < a.moves.capacity ? at_once : a.moves.capacity);
  return launch_k(copy_kernel<PER>, dim3((unsigned)(at_once * a.units)), dim3(COPY_THREADS), 0, st, a);
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
cudaError_t launch_cluster(void (*kern)(Args), int ctas, cudaStream_t st, const Args& a) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(POOL_THREADS); cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ctas; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = sps_pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, a);
}
// CTAs for a pool and a table: up to 4096 pages and a row to a thread, until the cluster has eight
int pool_ctas(int n_pages, int rows) {
  int c = 1;
  while (c < 8 && ((long long)c * 4096 < n_pages || c * POOL_THREADS < rows)) c *= 2;
  return c;
}

const char* bad_pool(const sps_page_pool* p) {
  if (!p) return "null pool";
  if (p->n_pages < 1 || p->n_pages > PAGES_MAX) return "pool: n_pages must be 1 .. 2^20";
  if (p->page_size < 8 || p->page_size > 512 || (p->page_size & (p->page_size - 1))) return "pool: page_size must be a power of two, 8 .. 512";
  if (!p->refs) return "pool: null pointer";
  if (((uintptr_t)p->refs | (uintptr_t)p->status) & 3) return "pool: pointers must be 4-byte aligned";
  return nullptr;
}
const char* bad_table(const sps_page_table* t) {
  if (!t) return "null table";
  if (t->B < 0 || t->B > PAGES_MAX_ROWS) return "table: B must be 0 .. 8192";
  if (t->ld < 0 || t->ld > PAGES_MAX || (int64_t)t->B * t->ld > INT_MAX) return "table: ld must be 0 .. 2^20, B x ld below 2^31";
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
  if (n_pages < 1 || n_pages > PAGES_MAX) { no(SPS_EINVAL, "n_pages must be 1 .. 2^20"); return -1; }
  // the number of pages in use; writers, the first of them, pages handed out (or a compaction's map), a word each
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

int sps_paged_reserve(const sps_page_pool* pool, const sps_page_table* table, const int32_t* want, int32_t* room, const sps_page_moves* moves,
                      void* workspace, void* stream) {
  const char* why = bad_pool(pool);
  if (!why) why = bad_table(table);
  if (!why) why = bad_moves(moves);
  if (!why) why = bad_workspace(workspace);
  if (why) return no(SPS_EINVAL, why);
  if ((table->B > 0 && !want) || ((uintptr_t)want & 3)) return no(SPS_EINVAL, "want null or not 4-byte aligned");
  if ((uintptr_t)room & 3) return no(SPS_EINVAL, "room not 4-byte aligned");
  if (moves->capacity < table->B) return no(SPS_EINVAL, "moves: a row may need one, capacity is smaller than the table's B");
  ReserveArgs a{};
  a.pool = pool_of(pool); a.t = table_of(table); a.want = want; a.room = room; a.moves = moves_of(moves);
  const int64_t n = ((int64_t)pool->n_pages + 63) / 64 * 64;
  a.writers = (int32_t*)((char*)workspace + 256);
  a.first = a.writers + n;
  a.fresh = a.writers + 2 * n;
  if (pool->n_pages <= SMALL_PAGES && table->B <= POOL_THREADS) {
    const size_t smem = (size_t)((pool->n_pages + 31) / 32) * 32 * 8;
    static DevSmemCache attr;
    // (with what the kernel has by itself 48 KB are passed early)
    const cudaError_t e = sps_ensure_smem(reserve_small_kernel, smem > 24 * 1024 && smem < 40 * 1024 ? 40 * 1024 : smem, attr);
    return done(e == cudaSuccess ? launch_k(reserve_small_kernel, dim3(1), dim3(POOL_THREADS), smem, (cudaStream_t)stream, a) : e);
  }
  return done(launch_cluster(reserve_kernel, pool_ctas(pool->n_pages, table->B), (cudaStream_t)stream, a));
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
  const int ctas = pool_ctas(pool->n_pages, 0);
  const long long units = (long long)(src->B > 0 ? src->B : 1) * (src->ld > 0 ? (src->ld + 255) / 256 : 1), warps = FORK_THREADS / 32, most = (long long)paged_sms() * 8;
  // one launch where a CTA scans the pool and has no more than 256 entries to a warp to rename (6 rows in a pool of 110 pages, copies
  // included: 8.1 us against 8.7; with 96 rows in 3500 pages 14 against 11)
  a.apply = ctas == 1 && units <= POOL_WARPS;
  cudaError_t e = launch_cluster(compact_scan_kernel, ctas, (cudaStream_t)stream, a);
  if (e == cudaSuccess && !a.apply) e = launch_k(compact_apply_kernel, dim3((unsigned)((units + warps - 1) / warps < most ? (units + warps - 1) / warps : most)), dim3(FORK_THREADS), 0, (cudaStream_t)stream, a);
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
  for (int l = 0; l < n_layers; l += COPY_LAYERS) {
    const int n = n_layers - l < COPY_LAYERS ? n_layers - l : COPY_LAYERS;
    for (int i = 0; i < n; ++i) { a.base[2 * i] = (char*)layers[l + i].k; a.base[2 * i + 1] = (char*)layers[l + i].v; }
    const bool much = (long long)moves->capacity * 2 * n * ((long long)a.page_size * a.heads << a.row_shift) * 16 >= COPY_MUCH;
    const cudaError_t e = much ? copy_launch<16, 3>(a, 2 * n, paged_sms(), (cudaStream_t)stream) : copy_launch<4, 8>(a, 2 * n, paged_sms(), (cudaStream_t)stream);
    if (e != cudaSuccess) return done(e);
  }
  return SPS_OK;
}

}  // extern "C"
