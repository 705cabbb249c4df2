// Shared by the paged-cache kernels: argument blocks, where a sequence's rows and tokens are, and how the attention
// kernels cut a ragged batch into equal pieces of work.
#pragma once
#include "../../include/sps.h"
#include "common.cuh"

// activations by row and head (sps_rows on the device side)
struct RowsView {
  void* p;
  long long row, head;   // strides in elements
};

struct PagedSeqs {       // sps_paged_batch, with what bounds it on the host
  const int32_t *q_start, *kv_len, *pages;
  int32_t* status;
  int B, pages_ld, rows;
  int n_pages, page_size, page_shift;   // page_size = 1 << page_shift
};

__device__ __forceinline__ void paged_flag(int32_t* status, int bit) {
  if (status) atomicOr(status, bit);
}

// tokens the page table of a sequence can hold (fits 32 bits: longer tables are cut)
__device__ __forceinline__ int paged_capacity(const PagedSeqs& s) {
  const long long c = (long long)s.pages_ld << s.page_shift;
  return c > 0x7fff0000ll ? 0x7fff0000 : (int)c;
}

// first row and rows, of those inside the call's buffers; tokens up to the last such row's own (rows behind the buffers take
// theirs with them); cut: kv_len did not fit the page table
struct SeqGeom { int row0, nq, len; bool cut; };
__device__ __forceinline__ SeqGeom paged_seq(const PagedSeqs& s, int b) {
  SeqGeom g;
  const int end = s.q_start[b + 1], r0 = min(max(s.q_start[b], 0), s.rows), r1 = min(max(end, r0), s.rows);
  const int len = s.kv_len[b], cap = paged_capacity(s);
  g.row0 = r0;
  g.nq = r1 - r0;
  g.cut = len > cap;
  g.len = max(min(max(len, 0), cap) - (max(end, r1) - r1), 0);
  return g;
}

// ------------------------------------------------------------------------------------------------------------------
// The attention kernels' work.  A sequence's queries of one key head are nq * G rows (token-major: row r is token r / G,
// head r % G of the group), taken NR at a time: an item is (sequence, key head, tile of NR rows), and its work is the
// number of tiles of KT tokens its last row sees (at least one, so that empty rows get their zeros), plus `lead` for what an
// item costs before its first tile.  All items' work in order -- sequences, key heads, row tiles -- is cut into equal runs,
// one per CTA: a ragged batch, one long sequence and a prompt chunk are balanced alike, to one tile.  A CTA whose run
// begins or ends inside an item leaves that part's
// (maximum, sum, unnormalised output) in its slot; the last CTA of the item to finish joins the parts in their order, so
// results do not depend on timing.
// ------------------------------------------------------------------------------------------------------------------
// an item cut into parts, left for the join by the CTA that has its first part
struct PartRecord { int row0, nq, hk, t, first, parts; };

struct PagedAttnArgs {
  PagedSeqs s;
  RowsView q, out;
  int q_bf16, out_bf16, q_vec, out_vec;   // vec: 16-byte accesses are aligned
  void *k, *v;
  long long page_stride, head_stride, pos_stride;
  int H, Hkv, G;
  unsigned long long g_magic;   // ceil(2^64 / G) for G > 1: row / G is a high product
  float scale_log2;         // scale * log2(e): scores are kept in base 2
  float* lse;               // [rows][H] or null
  int* counters;            // [grid] arrivals at an item, by the first CTA that works on it; zero between launches
  PartRecord* records;      // [grid] (kernels whose parts another kernel joins)
  int* gave_up;             // not 0: a wait of this call, or of an earlier one on this workspace, ran out
  uint32_t grid_magic;      // ceil(2^32 / CTAs), and the numbers below which its high product divides by them
  int grid_magic_to;
  int lead, min_run;        // set by the launcher: an item's cost ahead of its tiles, the least run, in tiles
  float* slots;             // [2 * grid] parts: [NR] maxima, [NR] sums, [NR][d_head] outputs
  unsigned long long wait_ns;
  int drop_stage;           // test hook: the half-tile that the copies of the list's first CTA leave out, -1 = none
};

// r / G for a row of a group of G heads
__device__ __forceinline__ int row_token(const PagedAttnArgs& a, int r) { return a.G == 1 ? r : (int)__umul64hi((unsigned long long)r, a.g_magic); }

// tiles of KT tokens row tile t of a sequence has to read
template <int NR, int KT>
__device__ __forceinline__ int item_tiles(const PagedAttnArgs& a, int nq, int len, int t) {
  const int last = min((t + 1) * NR, nq * a.G) - 1;
  const int pos = len - nq + row_token(a, last);
  return pos < 0 ? 1 : pos / KT + 1;
}

struct WorkCursor {       // a place in the list of items, and the run that is left
  int b, hk, t;           // item
  int row0, nq, len, nt;  // its sequence; nt = row tiles of the sequence
  int n;                  // tiles of the item
  int k0, k1;             // this CTA's tiles of it
  int b0;                 // the run's first sequence: geo[] holds it and those behind it
  long long u_end;        // the end of the run in the whole list
  long long item0;        // place of the item's first tile in the list (its lead lies before it)
  long long per;          // length of a run
  bool valid;
  int spoilt;             // not 0: the workspace holds what a call left that gave up, nothing is worked on
};
constexpr int GEO = 32;   // sequences a CTA keeps in shared memory, from its first on

// the part of item (b, hk, t) that lies in the run, which enters it at place u
template <int NR, int KT>
__device__ __forceinline__ void cursor_part(const PagedAttnArgs& a, WorkCursor& c, long long u) {
  c.n = item_tiles<NR, KT>(a, c.nq, c.len, c.t);
  c.k0 = u > c.item0 ? (int)(u - c.item0) : 0;
  c.k1 = c.u_end - c.item0 < c.n ? (int)(c.u_end - c.item0) : c.n;
  c.valid = c.k1 > c.k0;  // (a run that ends in an item's lead has no part of it)
}

template <int NR, int KT>
__device__ __forceinline__ void cursor_next(const PagedAttnArgs& a, WorkCursor& c, const SeqGeom* geo) {
  const long long u = c.item0 + c.n;
  if (u >= c.u_end) { c.valid = false; return; }
  c.item0 = u + a.lead;
  if (++c.t == c.nt) {
    c.t = 0;
    if (++c.hk == a.Hkv) {
      c.hk = 0;
      do {
        if (++c.b >= a.s.B) { c.valid = false; return; }
        const SeqGeom g = c.b - c.b0 < GEO ? geo[c.b - c.b0] : paged_seq(a.s, c.b);
        c.row0 = g.row0; c.nq = g.nq; c.len = g.len;
      } while (c.nq == 0);
      c.nt = (int)((unsigned)(c.nq * a.G + NR - 1) / NR);
    }
  }
  cursor_part<NR, KT>(a, c, u);
}

// The work of one key head of a sequence, for the sequences of one warp (lane = sequence): short sequences by
// their own lane, long ones by the whole warp.
template <int NR, int KT>
__device__ __forceinline__ long long warp_seq_units(const PagedAttnArgs& a, const SeqGeom& g, bool live) {
  const int lane = threadIdx.x & 31;
  const int nt = live ? (int)((unsigned)(g.nq * a.G + NR - 1) / NR) : 0;
  long long sum = 0;
  if (nt == 1) sum = a.lead + item_tiles<NR, KT>(a, g.nq, g.len, 0);
  else if (nt <= 4) for (int t = 0; t < nt; ++t) sum += a.lead + item_tiles<NR, KT>(a, g.nq, g.len, t);
  unsigned big = __ballot_sync(0xffffffffu, nt > 4);
  while (big) {
    const int src = __ffs(big) - 1;
    big &= big - 1;
    const int nq = __shfl_sync(0xffffffffu, g.nq, src), len = __shfl_sync(0xffffffffu, g.len, src), n = __shfl_sync(0xffffffffu, nt, src);
    long long part = 0;
    for (int t = lane; t < n; t += 32) part += a.lead + item_tiles<NR, KT>(a, nq, len, t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    if (lane == src) sum = part;
  }
  return sum;
}

__device__ __forceinline__ long long list_div(long long n, long long d) {   // n, d >= 0; almost always 32 bits wide
  if (((unsigned long long)(n | d) >> 32) == 0) return (long long)((unsigned)n / (unsigned)d);
  return n / d;
}

// Called by every warp of the CTA; the result is warp 0's, and with geo for every thread (in shared memory).  a.min_run: the
// least work a CTA takes, so that a short list is not cut into parts that cost more to join than they save.  Up to 32
// sequences are read by warp 0, once.  More of them are summed by all warps, in 32 stretches of whole blocks of 32
// (sums: shared, [32]), before warp 0 reads the stretch that this CTA's run begins in; with one warp reading all of them
// twice 512 (2048) sequences of one token took 34 (123) us, this way 18 (56).
template <int NR, int KT>
__device__ __forceinline__ WorkCursor cursor_begin(const PagedAttnArgs& a, SeqGeom* geo, long long* sums) {
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, B = a.s.B;
  WorkCursor c;
  c.valid = false;
  c.spoilt = 0;
  if (warp == 0) c.spoilt = __ldcg(a.gave_up);   // (one request a CTA: all of them ask for the same word)
  SeqGeom g{};                   // the sequences of one block of 32, a lane each; their work, and the sum up to each
  long long head = 0, units = 0, incl = 0, total = 0;   // head: of one key head
  auto block = [&](int b0) {
    const int b = b0 + lane;
    g = SeqGeom{};
    if (b < B) g = paged_seq(a.s, b);
    head = warp_seq_units<NR, KT>(a, g, b < B);
    units = head * a.Hkv;
    incl = units;
    if (__any_sync(0xffffffffu, units >= (1ll << 26))) {
#pragma unroll 1
      for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
    } else {   // the sum fits 32 bits
      int sum = (int)units;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
      }
      incl = sum;
    }
  };
  const long long stretch = 32ll * (((unsigned)B + 1023u) >> 10);   // sequences of one
  long long mine = 0, upto = 0;   // lane's stretch, and the sum up to it
  if (B <= 32) {
    if (warp != 0) return c;
    block(0);
    if (blockIdx.x == 0 && g.cut && g.nq > 0) paged_flag(a.s.status, SPS_PAGED_BAD_LENGTH);
    total = __shfl_sync(0xffffffffu, incl, 31);
  } else {
    for (int x = warp; x < 32; x += (int)(blockDim.x >> 5)) {
      long long sum = 0;
      for (long long b0 = x * stretch; b0 < (x + 1) * stretch && b0 < B; b0 += 32) {
        block((int)b0);
        if (blockIdx.x == 0 && g.cut && g.nq > 0) paged_flag(a.s.status, SPS_PAGED_BAD_LENGTH);
        sum += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (lane == 0) sums[x] = sum;
    }
    __syncthreads();
    if (warp != 0) return c;
    mine = upto = sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    total = __shfl_sync(0xffffffffu, upto, 31);
  }
  // ceil(total / CTAs): a high product for lists of up to 2^31 / CTAs tiles
  const long long up = total + gridDim.x - 1;
  c.per = up < a.grid_magic_to ? (long long)__umulhi((unsigned)up, a.grid_magic) : up / gridDim.x;
  if (c.per < a.min_run) c.per = a.min_run;
  const long long u = (long long)blockIdx.x * c.per;
  c.u_end = u + c.per < total ? u + c.per : total;
  if (u >= c.u_end) return c;
  // the sequence that place u falls into
  long long base = 0;
  int from = 0;
  if (B > 32) {
    const int x = __ffs(__ballot_sync(0xffffffffu, upto > u)) - 1;
    base = __shfl_sync(0xffffffffu, upto - mine, x);
    from = (int)(x * stretch);
  }
  for (int b0 = from; b0 < B; b0 += 32) {
    if (B > 32) block(b0);
    const unsigned hit = __ballot_sync(0xffffffffu, base + incl > u);
    if (hit) {
      const int src = __ffs(hit) - 1;
      c.b = c.b0 = b0 + src;
      c.row0 = __shfl_sync(0xffffffffu, g.row0, src);
      c.nq = __shfl_sync(0xffffffffu, g.nq, src);
      c.len = __shfl_sync(0xffffffffu, g.len, src);
      if (B <= 32) {
        if (lane >= src && lane < B) geo[lane - src] = g;
      } else if (c.b + lane < B) {
        geo[lane] = paged_seq(a.s, c.b + lane);
      }
      const long long first = base + __shfl_sync(0xffffffffu, incl - units, src), per_head = __shfl_sync(0xffffffffu, head, src);
      c.nt = (int)((unsigned)(c.nq * a.G + NR - 1) / NR);
      c.hk = (int)list_div(u - first, per_head);
      long long at = first + c.hk * per_head;   // where the key head's work begins
      c.t = 0;
      if (c.nt > 1) {
        // the row tile: 32 at a time
        for (int t0 = 0; t0 < c.nt; t0 += 32) {
          const int t = t0 + lane;
          const long long n = t < c.nt ? a.lead + item_tiles<NR, KT>(a, c.nq, c.len, t) : 0;
          long long in2 = n;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const long long up = __shfl_up_sync(0xffffffffu, in2, o);
            if (lane >= o) in2 += up;
          }
          const unsigned hit2 = __ballot_sync(0xffffffffu, at + in2 > u);
          if (hit2) {
            const int s2 = __ffs(hit2) - 1;
            c.t = t0 + s2;
            at += __shfl_sync(0xffffffffu, in2 - n, s2);
            break;
          }
          at += __shfl_sync(0xffffffffu, in2, 31);
        }
      }
      c.item0 = at + a.lead;
      cursor_part<NR, KT>(a, c, u);
      return c;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  return c;
}

// parts an item is cut into: the CTAs first .. first + parts - 1 each hold one
__device__ __forceinline__ void item_ctas(const WorkCursor& c, int& first, int& parts) {
  first = blockIdx.x;
  parts = 1;
  if (c.k0 == 0 && c.k1 == c.n) return;
  first = (int)list_div(c.item0, c.per);
  parts = (int)list_div(c.item0 + c.n - 1, c.per) - first + 1;
}
// the slot of this CTA's part: 2 c + 1 where the item begins in this CTA, else 2 c (a run holds at most one of each)
__device__ __forceinline__ int part_slot(int cta, bool begins) { return 2 * cta + (begins ? 1 : 0); }
template <int NR, int D> __host__ __device__ constexpr size_t slot_floats() { return (size_t)NR * (D + 2); }

// One thread's word that its CTA's part is out (the CTA's threads have met since): true for the last part of the item, which
// may then read the others'; the counter is left at zero for the next call.
__device__ __forceinline__ bool part_arrive(int* counter, int parts) {
  int old;
  asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
  if (old != parts - 1) return false;
  *counter = 0;
  return true;
}

__device__ __forceinline__ void store_out(const PagedAttnArgs& a, long long at, float v) {
  if (a.out_bf16) reinterpret_cast<__nv_bfloat16*>(a.out.p)[at] = __float2bfloat16_rn(v);
  else reinterpret_cast<float*>(a.out.p)[at] = v;
}

// Joins the parts of an item and writes its rows: o = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c.  Run by all THREADS
// threads that finished the item's last part to arrive (named barrier `bar` is theirs).  A part's slot is a trip to L2 away, so many loads are in
// flight at once: every thread first asks for its four-element pieces of the first AHEAD parts' outputs, then for maxima and
// sums (THREADS / NR threads to a row), and goes on four parts at a time, their weights in shared memory.  s_max, s_inv: shared
// scratch of NR floats each; w: of w_floats >= 2 * THREADS.
template <int NR, int D, int THREADS>
__device__ __forceinline__ void join_parts(const PagedAttnArgs& a, const WorkCursor& c, int first, int parts, int tid, float* s_max, float* s_inv, float* w, int w_floats, int bar = 2) {
  const int R = c.nq * a.G, r0 = c.t * NR, live = min(NR, R - r0);
  constexpr size_t SF = slot_floats<NR, D>();
  constexpr int LANES = THREADS / NR, PIECES = NR * (D / 4) / THREADS, BLOCK = PIECES < 4 ? PIECES : 4, AHEAD = 2;
  const float* slots = a.slots + SF * (size_t)(2 * first);
  auto slot = [&](int p) { return slots + SF * (size_t)(p == 0 ? 1 : 2 * p); };   // part 0 begins in its CTA: part_slot
  auto sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(THREADS) : "memory"); };
  auto row = [&](int i) { return i / (D / 4); };
  auto fetch = [&](int p, int i) { return __ldcg(reinterpret_cast<const float4*>(slot(p) + 2 * NR) + i); };
  float4 early[AHEAD][BLOCK];
#pragma unroll
  for (int p = 0; p < AHEAD; ++p)
#pragma unroll
    for (int k = 0; k < BLOCK; ++k) {
      const int i = tid + k * THREADS;
      early[p][k] = row(i) < live ? fetch(p, i) : make_float4(0.f, 0.f, 0.f, 0.f);    // (an item that is joined has at least two)
    }
  {
    const int r = tid % NR, p0 = tid / NR;
    float M = -INFINITY, L = 0.f;
    if (r < live) {
#pragma unroll 4
      for (int p = p0; p < parts; p += LANES) {
        const float m = __ldcg(slot(p) + r), l = __ldcg(slot(p) + NR + r);
        const float nm = fmaxf(M, m), base = nm == -INFINITY ? 0.f : nm;
        L = L * exp2f(M - base) + l * exp2f(m - base);      // 2^-inf = 0 on either side that has nothing
        M = nm;
      }
    }
    w[2 * tid] = M;
    w[2 * tid + 1] = L;
  }
  sync();
  if (tid < live) {
    float M = -INFINITY, L = 0.f;
    for (int i = 0; i < LANES; ++i) M = fmaxf(M, w[2 * (i * NR + tid)]);
    const float base = M == -INFINITY ? 0.f : M;
    for (int i = 0; i < LANES; ++i) L += w[2 * (i * NR + tid) + 1] * exp2f(w[2 * (i * NR + tid)] - base);
    s_max[tid] = base;
    s_inv[tid] = L == 0.f ? 0.f : 1.f / L;
    if (a.lse) {
      const int r = r0 + tid;
      a.lse[(size_t)(c.row0 + row_token(a, r)) * a.H + c.hk * a.G + r - row_token(a, r) * a.G] = L == 0.f ? -INFINITY : 0.6931471805599453f * (base + log2f(L));
    }
  }
  sync();
  const int table = w_floats / NR;                             // parts whose weights fit at once
#pragma unroll 1
  for (int kb = 0; kb < PIECES; kb += BLOCK) {
    float4 o[BLOCK];
#pragma unroll
    for (int k = 0; k < BLOCK; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int pb = 0; pb < parts; pb += table) {
      const int pn = min(table, parts - pb);
      if (kb == 0 || parts > table) {
        for (int i = tid; i < pn * NR; i += THREADS) {
          const int p = i / NR, r = i - p * NR;
          if (r < live) w[i] = exp2f(__ldcg(slot(pb + p) + r) - s_max[r]) * s_inv[r];
        }
        sync();
      }
      auto add = [&](int k, float f, const float4& v) { o[k].x += f * v.x; o[k].y += f * v.y; o[k].z += f * v.z; o[k].w += f * v.w; };
      int p = 0;
      if (kb == 0 && pb == 0) {
#pragma unroll
        for (; p < AHEAD; ++p)
#pragma unroll
          for (int k = 0; k < BLOCK; ++k) {
            const int r = row(tid + k * THREADS);
            if (r < live) add(k, w[p * NR + r], early[p][k]);
          }
      }
#pragma unroll 4
      for (; p < pn; ++p) {
#pragma unroll
        for (int k = 0; k < BLOCK; ++k) {
          const int i = tid + (kb + k) * THREADS, r = row(i);
          if (r < live) add(k, w[p * NR + r], fetch(pb + p, i));
        }
      }
      if (parts > table) sync();   // the table may be written again
    }
#pragma unroll
    for (int k = 0; k < BLOCK; ++k) {
      const int i = tid + (kb + k) * THREADS, r = row(i);
      if (r < live) {
        const int e = (i - r * (D / 4)) * 4, rr = r0 + r, tok = row_token(a, rr);
        const long long at = (long long)(c.row0 + tok) * a.out.row + (long long)(c.hk * a.G + rr - tok * a.G) * a.out.head + e;
        store_out(a, at, o[k].x); store_out(a, at + 1, o[k].y); store_out(a, at + 2, o[k].z); store_out(a, at + 3, o[k].w);
      }
    }
  }
}

// The rows of a call that gave up, or that found its workspace spoilt by one: NaN, so that no caller takes them for answers.
// Share `share` of `shares`, by all threads of a CTA.
template <int D> __device__ __forceinline__ void nan_rows(const PagedAttnArgs& a, int share, int shares) {
  const int r0 = min(max(a.s.q_start[0], 0), a.s.rows), r1 = min(max(a.s.q_start[a.s.B], r0), a.s.rows);
  const float nan = __int_as_float(0x7fffffff);
  for (int row = r0 + share; row < r1; row += shares)
    for (int head = 0; head < a.H; ++head) {
      const long long at = (long long)row * a.out.row + (long long)head * a.out.head;
      for (int e = threadIdx.x; e < D; e += blockDim.x) store_out(a, at + e, nan);
      if (threadIdx.x == 0 && a.lse) a.lse[(size_t)row * a.H + head] = nan;
    }
}

// launchers
struct RotaryArgs {
  RowsView x[3], y[3];         // queries (or the rows of sps_rotary), keys, values; y[1], y[2]: page pools
  int heads[3];
  int d_head, rot, halves, transposed;
  float gain;
  const double* freq;          // null: nothing is rotated
  const int32_t* positions;    // sps_rotary; null: from the batch
  PagedSeqs s;
  long long pos_stride;        // cache slots
  int rows;
  // set by the launcher: heads of all three, units of a head, (row, head) pairs the threads of a CTA take at once, a CTA's
  // rows and heads of each, where a head's unrotated part starts and half its length; reciprocals for divisions
  int vheads, uh, per_pass, rows_per_cta, heads_per_cta, flat0, flat_half;
  uint32_t uh_magic, span_magic;
};
cudaError_t rotary_launch(RotaryArgs a, int x_bf16, int yq_bf16, int cache_bf16, int num_sm, cudaStream_t st);
// CTAs of an attention launch on a device of num_sm SMs, at most (counters and slots are laid out for as many)
inline int paged_attn_grid(int num_sm) { return num_sm < 1024 ? num_sm : 1024; }
size_t paged_attn_slot_bytes(int dtype, int q_dtype, int d_head);
size_t paged_attn_tc_slot_bytes(int d_head);
size_t paged_attn_wide_slot_bytes(int d_head);
cudaError_t paged_attn_wide_launch(const PagedAttnArgs& a, int d_head, int num_sm, cudaStream_t st);
cudaError_t paged_attn_tc_launch(const PagedAttnArgs& a, int d_head, int max_q, int num_sm, cudaStream_t st);
cudaError_t paged_attn_launch(const PagedAttnArgs& a, int cache_bf16, int d_head, int max_q, int num_sm, cudaStream_t st);
