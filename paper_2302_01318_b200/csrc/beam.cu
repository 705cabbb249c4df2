// The selection of a beam step (sps_beam_select): the best continuations over a sequence's beams and the vocabulary.
#include <climits>
#include <cmath>

#include <cooperative_groups.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

// ------------------------------------------------------------------------------------------------------------------
// c[w, v] = s[w] + l[w, v] / T - log sum_u exp(l[w, u] / T); the N best (w, v) of each sequence, ties to the lowest w V + v.
//
// Two kernels.  The scan reads every logit once: per row running maxima and sums of exponentials, and the maximum of every
// segment of 512 bytes.  A row's order is its logits', so the N best elements lie in the N segments whose maxima score
// best (ties to the lower segment: any element outside has N better ones in them) -- whatever the numbers are.  The pick, a
// CTA per sequence, finds those segments (or a few more), reads them again (N x 512 bytes, from L2) and picks the N best elements.
// The scan is bound by HBM with many rows; the pick by latency, a chain of a dozen short steps between barriers (6 us): 256 rows of
// 131071 in bf16 (67 MB) 22.5 us, 512 of 32000 in fp32 20 us, of which the bytes' floor is 10.
// Candidates are compared in 64 bits, from exact logits and a sum of fp32 exponentials, so that a beam's far scores keep the order of
// their last bits; results are rounded to fp32 at the end.  The sum's relative error, found with scores that make c about 0: 1 - 2 10^-7
// for 1000 .. 131071 logits, at most 4.6 10^-7 = 2^-21 (5120 rows of 10^6, 2000 x 8 of 32000, 2^24 logits).
// ------------------------------------------------------------------------------------------------------------------
namespace {

constexpr int SCAN_THREADS = 256, SCAN_WARPS = 8, SCAN_SEGS = 4;       // segments of a group: a warp's load
constexpr int ONE_RUN = 2, ONE_CTAS = 8, ONE_THREADS = 1024, ONE_PICK = 512, ONE_WARPS = ONE_CTAS * ONE_THREADS / 32;   // the kernel for little work; ONE_PICK: threads that pick
constexpr int PICK_CAP = 1024, PICK_COUNTED = 128, PICK_SPLIT = 8, PICK_PER = 4, PICK_FEW = 4;   // entries of a list, of one ranked by counting, threads that rank one; segments a thread holds, to a candidate that are few
constexpr int BEAM_MAX_B = 8192, BEAM_MAX_W = 128, BEAM_MAX_N = 128;

struct BeamArgs {
  const void* logits;
  long long row_stride;
  int B, W, V, N;
  double inv_t, t;
  float c, inv_t32;          // log2(e) / T, 1 / T
  const float* scores;
  const int32_t* done;       // or null
  int end_token;
  float* out_scores;
  int32_t *out_parents, *out_tokens, *out_done;   // out_done: or null
  float* seg_max;            // [B W][n_seg]
  float2* parts;             // [B W][max_parts]: maximum, sum of exponentials
  int n_seg, groups, run, max_parts;   // segments and groups of a row, groups of a run, parts a row may have
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two fp32 operations in one instruction: (x, y) f + (g, g); (x, y) += (a, b)
__device__ __forceinline__ void fma2(float& x, float& y, float f, float g) {
  asm("{\n .reg .b64 s, t, u;\n mov.b64 s, {%0, %1};\n mov.b64 t, {%2, %2};\n mov.b64 u, {%3, %3};\n fma.rn.f32x2 s, s, t, u;\n mov.b64 {%0, %1}, s;\n}\n"
      : "+f"(x), "+f"(y) : "f"(f), "f"(g));
}
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
  asm("{\n .reg .b64 s, t;\n mov.b64 s, {%0, %1};\n mov.b64 t, {%2, %3};\n add.rn.f32x2 s, s, t;\n mov.b64 {%0, %1}, s;\n}\n" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
// numbers in the order of floats; NaN never comes here (maxima leave it out)
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }

// E logits in 16 bytes
template <typename T> struct Logit;
template <> struct Logit<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void unpack(uint4 u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float top(uint4 u) {   // NaN left out, by this one and the next
    return fmaxf(fmaxf(fmaxf(__uint_as_float(u.x), -INFINITY), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
  }
};
template <> struct Logit<__nv_bfloat16> {
  static constexpr int E = 8;
  static __device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void unpack(uint4 u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {   // (of numbers that are bf16)
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[2 * i]) >> 16 | (__float_as_uint(f[2 * i + 1]) & 0xffff0000u);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ float top(uint4 u) {
    auto two = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    const __nv_bfloat162 m = __hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w)));
    return fmaxf(fmaxf(__low2float(m), -INFINITY), __high2float(m));
  }
};

// Rows need not begin at 16 bytes: segments are counted from the 16-byte boundary at or before a row's first logit, `shift` elements
// ahead of it, so that all but the pieces at its ends are read 16 bytes at a time.
template <typename T>
__device__ __forceinline__ const T* row_begin(const BeamArgs& a, int row, int* shift) {
  const T* x = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
  *shift = (int)(((uintptr_t)x & 15) / sizeof(T));
  return x - *shift;
}
// the piece at place v of such a row (a multiple of E), -inf what is not of the row
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* x, int v, int shift, int V) {
  constexpr int E = Logit<T>::E;
  if (v >= shift && v + E <= V + shift) return *reinterpret_cast<const uint4*>(x + v);
  float f[E];
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = v + e >= shift && v + e < V + shift ? Logit<T>::get(x + v + e) : -INFINITY;
  return Logit<T>::pack(f);
}

// a beam that reads its logits: it has a score, and is not done
__device__ __forceinline__ bool beam_reads(const BeamArgs& a, int row) {
  return !(a.done && a.done[row]) && isfinite(a.scores[row]);
}

// (m, s) of the warp from its lanes': sums are relative to the maxima
__device__ __forceinline__ void warp_merge(float& m, float& s, float c) {
  const float all = unordered(__reduce_max_sync(0xffffffffu, ordered(m))), r = all == -INFINITY ? 0.f : all;
  s = warp_sum(s * ex2((m - r) * c));
  m = all;
}

// A lane's running maximum m and sum of 2^(c l - R), R = c m rounded: one fused operation per exponent, whose rounding is the
// difference's alone; what R's own rounding leaves, R - c m, is exact in one more and put right at the end.  With maxima beyond
// 2^20 / c (`far`, for the rest of the part) differences are taken first: c l might overflow.
struct Running {
  float m, R, s;
  bool far;
};
template <typename T>
__device__ __forceinline__ void running_add(Running& r, const uint4 (&u)[SCAN_SEGS], float top, float c) {
  constexpr int E = Logit<T>::E;
  const float m1 = fmaxf(r.m, top), R1 = m1 == -INFINITY ? 0.f : m1 * c;
  if (!r.far && __any_sync(0xffffffffu, !(fabsf(R1) < 1048576.f))) {
    r.far = true;
    if (r.m > -INFINITY) r.s *= ex2(-fmaf(r.m, c, -r.R));
  }
  float s0 = 0.f, s1 = 0.f;
  if (r.far) {
    const float ref = m1 == -INFINITY ? 0.f : m1;
    r.s *= ex2((r.m - ref) * c);
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j) {
      float f[E];
      Logit<T>::unpack(u[j], f);
#pragma unroll
      for (int e = 0; e < E; ++e) s0 += ex2((f[e] - ref) * c);
    }
  } else {
    r.s *= ex2(r.R - R1);
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j) {
      float f[E];
      Logit<T>::unpack(u[j], f);
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        fma2(f[e], f[e + 1], c, -R1);
        add2(s0, s1, ex2(f[e]), ex2(f[e + 1]));
      }
    }
    r.R = m1 == -INFINITY ? -INFINITY : R1;
  }
  r.s += s0 + s1;
  r.m = m1;
}

// A run of the list of `rows` rows' groups (SCAN_SEGS segments; the last of a row may be short), from group x0 of the list on, by
// one warp: its next group is under way while it works on this one, whatever the rows' number and length.  A run's share of a
// row is a part of it; beams that are done or dead are skipped.  seg_max, parts: the list's.
template <typename T>
__device__ __forceinline__ void beam_scan(const BeamArgs& a, int first_row, int rows, int me, float* seg_max, float2* parts) {
  constexpr int E = Logit<T>::E, SEG = 32 * E, GROUP = SCAN_SEGS * SEG;
  const int lane = threadIdx.x & 31;
  const long long x0 = (long long)me * a.run;
  if (x0 >= (long long)rows * a.groups) return;
  int row = (int)x0 / a.groups, g = (int)x0 - row * a.groups, left = (int)min((long long)a.run, (long long)rows * a.groups - x0);
  int shift;
  const T* x = row_begin<T>(a, first_row + row, &shift);
  uint4 u[SCAN_SEGS];
  auto fetch = [&](const T* p, int group) {
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j) u[j] = *reinterpret_cast<const uint4*>(p + (long long)group * GROUP + j * SEG + lane * E);
  };
  auto inside = [&](int group) { return (group > 0 || shift == 0) && (group + 1) * GROUP <= a.V + shift; };   // all of it in the row
  bool fetched = inside(g);
  if (fetched) fetch(x, g);   // (before its row is known to be read)
  int row0 = row;
  unsigned live = __ballot_sync(0xffffffffu, row + lane < rows && beam_reads(a, first_row + min(row + lane, rows - 1)));
  Running run{-INFINITY, -INFINITY, 0.f, false};
  while (left > 0) {
    if (row - row0 >= 32) {
      row0 = row;
      live = __ballot_sync(0xffffffffu, row + lane < rows && beam_reads(a, first_row + min(row + lane, rows - 1)));
    }
    if (!((live >> (row - row0)) & 1)) {
      left -= a.groups - g;
      ++row;
      g = 0;
      if (left <= 0) break;
      x = row_begin<T>(a, first_row + row, &shift);
      fetched = row - row0 < 32 && ((live >> (row - row0)) & 1) && inside(0);
      if (fetched) fetch(x, 0);
      continue;
    }
    uint4 now[SCAN_SEGS];
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j) now[j] = fetched ? u[j] : load_piece(x, g * GROUP + j * SEG + lane * E, shift, a.V);
    const int now_row = row, now_g = g;
    --left;
    if (++g == a.groups) {
      g = 0;
      ++row;
      if (left > 0) x = row_begin<T>(a, first_row + row, &shift);
    }
    fetched = left > 0 && row - row0 < 32 && ((live >> (row - row0)) & 1) && inside(g);
    if (fetched) fetch(x, g);
    float top = -INFINITY;
    int best = 0;
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j) {
      const float t = Logit<T>::top(now[j]);
      top = fmaxf(top, t);
      const int w = __reduce_max_sync(0xffffffffu, ordered(t));
      if (lane == j) best = w;
    }
    if (lane < SCAN_SEGS && now_g * SCAN_SEGS + lane < a.n_seg) seg_max[(long long)now_row * a.n_seg + now_g * SCAN_SEGS + lane] = unordered(best);
    running_add<T>(run, now, top, a.c);
    if (g == 0 || left == 0) {   // the end of the row, or of the run
      float m = run.m, s = run.s;
      if (!run.far && m > -INFINITY) s *= ex2(-fmaf(m, a.c, -run.R));
      warp_merge(m, s, a.c);
      if (lane == 0) parts[(long long)now_row * a.max_parts + me - now_row * a.groups / a.run] = make_float2(m, s);
      run = Running{-INFINITY, -INFINITY, 0.f, false};
    }
  }
}

// log s to 2^-25, for s >= 2^-126: the fp32 function of a number next to 1, whose logarithm is below 0.35, and the exponent's share
__device__ __forceinline__ double log_of(float s) {
  const int i = __float_as_int(s), e = (i - 0x3f3504f3) >> 23;   // s 2^-e in 0.707 .. 1.414
  return fma((double)e, 0.6931471805599453, (double)logf(__int_as_float(i - (e << 23))));
}

// Picking: candidates are (score, place) pairs, ties falling to the lowest place, so that all differ.  A list takes those that
// reach a bound which at least N reach; only where more reach it than the list holds (ties by the hundred, rising rows) is the
// stream taken in rounds, the list cut to its N best whenever it might overflow.
template <int THREADS>
__device__ __forceinline__ void pick_sync() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }   // of the threads that pick
struct Best {
  double* key;        // [PICK_CAP]
  int* at;
  double* keep_key;   // [BEAM_MAX_N]: the N best, in order
  int* keep_at;
  int* count;
  int *thread, *tops, *bound;   // [THREADS], [BEAM_MAX_N + 2 WARPS], [1]: for best_bound
};
__device__ __forceinline__ bool better(double k, int i, double k1, int i1) { return k > k1 || (k == k1 && i < i1); }
__device__ __forceinline__ void best_push(const Best& b, double k, int i) {
  const int n = atomicAdd(b.count, 1);
  if (n < PICK_CAP) { b.key[n] = k; b.at[n] = i; }
}
// a number that at least N of the threads' numbers reach (-inf: they may be fewer): the N-th of the groups' best, k from each, a
// group having one lane of 32, or two, of every warp, another one in each (a warp's numbers may all be of one beam, and only its first
// lanes have any where a beam has few segments)
template <int THREADS>
__device__ __forceinline__ float best_bound(const Best& b, float top, int N) {
  constexpr int WARPS = THREADS / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, k = (N + WARPS - 1) / WARPS + 1;
  b.thread[tid] = ordered(top);
  if (tid == 0) *b.bound = INT_MIN;
  pick_sync<THREADS>();
  int mine = b.thread[lane % WARPS * 32 + ((warp - lane) & (WARPS - 1)) + lane / WARPS * WARPS];
  for (int j = 0; j < k; ++j) {
    const int v = __reduce_max_sync(0xffffffffu, mine);
    if (lane == 0) b.tops[warp * k + j] = v;
    if (__ffs(__ballot_sync(0xffffffffu, mine == v)) - 1 == lane) mine = INT_MIN;
  }
  pick_sync<THREADS>();
  for (int i = tid; i < k * WARPS; i += THREADS) {
    const int v = b.tops[i];
    int r = 0;
#pragma unroll 8
    for (int j = 0; j < k * WARPS; ++j) r += b.tops[j] > v || (b.tops[j] == v && j < i);
    if (r == N - 1) *b.bound = v;
  }
  pick_sync<THREADS>();
  return unordered(max(*b.bound, ordered(-INFINITY)));
}

// A list of n, above PICK_COUNTED (few segments with many candidates), cut to what reaches a bound; what is long even then (ties by
// the hundred) is sorted, a bitonic network over the next power of two, of which a warp has 64 neighbours to itself.  Returns
// how many are left at its head: all of the N best, at most 2 PICK_COUNTED.  (Out of line, like all that is rarely run: the pick is a
// walk through code that has to be fetched.)
template <int THREADS>
__device__ __noinline__ int best_shorten(const Best& b, int N, int n) {
  constexpr int PER = (PICK_CAP + THREADS - 1) / THREADS;
  const int tid = threadIdx.x;
  double k[PER];
  int p[PER];
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = tid + j * THREADS;
    k[j] = i < n ? b.key[i] : -INFINITY;
    p[j] = i < n ? b.at[i] : 0;
    top = fmaxf(top, __double2float_rd(k[j]));
  }
  const float least = best_bound<THREADS>(b, top, N);
  if (tid == 0) *b.count = 0;
  pick_sync<THREADS>();
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (k[j] > -INFINITY && k[j] >= (double)least) best_push(b, k[j], p[j]);
  pick_sync<THREADS>();
  n = *b.count;
  if (n <= 2 * PICK_COUNTED) return n;
  int size = 4 * PICK_COUNTED;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += THREADS) { b.key[i] = -INFINITY; b.at[i] = INT_MAX; }
  pick_sync<THREADS>();
  for (int run = 2; run <= size; run *= 2)
    for (int step = run / 2; step > 0; step /= 2) {
      if (tid < size / 2) {
        const int i = 2 * tid - (tid & (step - 1)), j = i + step;
        const double ki = b.key[i], kj = b.key[j];
        const int ai = b.at[i], aj = b.at[j];
        if (better(kj, aj, ki, ai) == ((i & run) == 0)) { b.key[i] = kj; b.at[i] = aj; b.key[j] = ki; b.at[j] = ai; }
      }
      // the next step's pairs lie within what a warp has, unless its step is above 32
      if (step > 32 || (step == 1 && run > 32)) pick_sync<THREADS>();
      else __syncwarp();
    }
  pick_sync<THREADS>();
  return 2 * PICK_COUNTED;
}
// The list's N best to keep_key / keep_at in order; returns how many there are (every thread of the CTA calls it, the list is
// complete).  Every entry counts those before it, PICK_SPLIT threads to an entry.  Counting 1000 entries would take 50 us, sorting
// them 10, cutting them 1.
template <int THREADS>
__device__ __forceinline__ int best_rank(const Best& b, int N) {
  const int tid = threadIdx.x, sub = tid % PICK_SPLIT;
  int n = min(*b.count, PICK_CAP);
  const int found = min(n, N);
  if (n > PICK_COUNTED) n = best_shorten<THREADS>(b, N, n);
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += THREADS / PICK_SPLIT) {
    const int i = i0 + tid / PICK_SPLIT;
    const double k = i < n ? b.key[i] : 0.0;
    const int p = i < n ? b.at[i] : 0;
    int r = 0;
    if (i < n)
#pragma unroll 4
      for (int j = sub; j < n; j += PICK_SPLIT) r += better(b.key[j], b.at[j], k, p);
#pragma unroll
    for (int o = PICK_SPLIT / 2; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
    if (i < n && sub == 0 && r < N) { b.keep_key[r] = k; b.keep_at[r] = p; }
  }
  pick_sync<THREADS>();
  return found;
}
// The N best of item(0 .. all - 1) -> (key, place), -inf keys left out: those that reach a bound from the items themselves (a bound
// from segments' maxima says little where they are of one beam), or, where the list does not hold these either, in rounds.  15 x 873
// with a beam far ahead of the others, 13 candidates, took 50 us in rounds alone, 16 so; equal logits, which a bound does not
// thin, 42 and 61 (64 x 4 x 32000, 8 candidates).
template <int THREADS, class Item>
__device__ __noinline__ int best_rounds(const Best& b, int N, int all, Item item) {
  float top = -INFINITY;
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += THREADS) {
    int at;
    top = fmaxf(top, __double2float_rd(item(i, &at)));
  }
  const float least = best_bound<THREADS>(b, top, N);
  if (threadIdx.x == 0) *b.count = 0;
  pick_sync<THREADS>();
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += THREADS) {
    int at;
    const double k = item(i, &at);
    if (k > -INFINITY && k >= (double)least) best_push(b, k, at);
  }
  pick_sync<THREADS>();
  if (*b.count <= PICK_CAP) return best_rank<THREADS>(b, N);
  int have = 0;
  pick_sync<THREADS>();
  for (int i0 = 0; i0 < all; i0 += PICK_CAP - BEAM_MAX_N) {
    for (int i = threadIdx.x; i < have; i += THREADS) { b.key[i] = b.keep_key[i]; b.at[i] = b.keep_at[i]; }
    if (threadIdx.x == 0) *b.count = have;
    pick_sync<THREADS>();
    const double bound = have == N ? b.key[N - 1] : -INFINITY;
    const int bound_at = have == N ? b.at[N - 1] : 0;
    for (int i = i0 + threadIdx.x; i < min(i0 + PICK_CAP - BEAM_MAX_N, all); i += THREADS) {
      int at;
      const double k = item(i, &at);
      if (better(k, at, bound, bound_at)) best_push(b, k, at);
    }
    pick_sync<THREADS>();
    have = best_rank<THREADS>(b, N);
  }
  return have;
}
// best_bound from top(i, lane) of the segments i < segs, a warp to a segment
template <int THREADS, class Top>
__device__ __noinline__ float best_elements(const Best& b, int N, int segs, Top top) {
  float t = -INFINITY;
#pragma unroll 1
  for (int i = threadIdx.x >> 5; i < segs; i += THREADS / 32) t = fmaxf(t, top(i, threadIdx.x & 31));
  return best_bound<THREADS>(b, t, N);
}

// a sequence's beams, where the pick finds them
struct Beams {
  float score[BEAM_MAX_W];
  int done[BEAM_MAX_W];
};
template <int THREADS>
__device__ __forceinline__ void beams_load(const BeamArgs& a, int b, Beams& beams) {
  for (int w = threadIdx.x; w < a.W; w += THREADS) {
    beams.score[w] = a.scores[b * a.W + w];
    beams.done[w] = a.done ? a.done[b * a.W + w] : 0;
  }
}

// Alike beams, of one score and the same logits, tie in every candidate, and places decide.  Their sums of exponentials were added
// up in the parts that the runs and the rows' alignment made, and may differ in the last bits: the later ones take the first's.
// It is the rows that are compared, where score and maximum are the same: sums that are close say nothing.  A warp looks for each beam's
// first earlier one by the rows' first pieces, then all threads compare what was found to the end.  Rare (a search that starts from
// beams of one score), and then a second reading by one CTA: 4 alike beams of 32000 fp32 logits take 15 us, where unlike ones take 9; 64 x
// 4 of 131071 in bf16 52, else 22.  Where it is not run it and the look at the scores cost 0.1 - 0.2 us (0.2 - 0.3 with it
// out of line: the call's registers), with 128 beams 1 - 2 of 38.
// base, top, line: the beams', as in beam_pick; like, differ: scratch, [BEAM_MAX_W]
template <typename T, int THREADS>
__device__ __forceinline__ void alike_beams(const BeamArgs& a, int first_row, const Beams& beams, double* base, const float* top, float2* line, int* like, int* differ) {
  constexpr int E = Logit<T>::E, WARPS = THREADS / 32, PER = 4;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // whether two rows differ in what a thread compares: the elements below n, `step` threads sharing them (it is number t of them)
  auto unlike = [&](int w, int r, int n, int t, int step) {
    int sw, sr;
    const T *x = row_begin<T>(a, first_row + w, &sw), *y = row_begin<T>(a, first_row + r, &sr);
    bool no = false;
    int whole = 0;   // elements in 16-byte pieces, behind the first `ahead` ones
    const int ahead = sw ? E - sw : 0;
    if (sw == sr) whole = max(n - ahead, 0) / E * E;
    for (int i0 = t; i0 < whole / E; i0 += PER * step) {
      uint4 u[PER], v[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int at = sw + ahead + min(i0 + j * step, whole / E - 1) * E;
        u[j] = *reinterpret_cast<const uint4*>(x + at);
        v[j] = *reinterpret_cast<const uint4*>(y + at);
      }
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        float f[E], g[E];
        Logit<T>::unpack(u[j], f);
        Logit<T>::unpack(v[j], g);
#pragma unroll
        for (int e = 0; e < E; ++e) no |= f[e] != g[e];
      }
    }
    // the others: those ahead of the pieces and behind them, or, where the rows' alignment differs, all
    for (int i0 = t; i0 < n - whole; i0 += PER * step) {
      T f[PER], g[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int i = min(i0 + j * step, n - whole - 1), at = i < ahead ? i : i + whole;
        f[j] = x[sw + at];
        g[j] = y[sr + at];
      }
#pragma unroll
      for (int j = 0; j < PER; ++j) no |= Logit<T>::get(f + j) != Logit<T>::get(g + j);
    }
    return no;
  };
  // the first beam of r0 .. w - 1 whose score, maximum and first n logits are w's (w: none), by a warp
  auto search = [&](int w, int r0, int n) {
    for (; r0 < w; r0 += 32) {
      const int r = min(r0 + lane, w);
      unsigned may = __ballot_sync(0xffffffffu, r < w && base[w] > -INFINITY && base[r] > -INFINITY && beams.score[r] == beams.score[w] && top[r] == top[w]);
      for (; may; may &= may - 1) {
        const int at = r0 + __ffs(may) - 1;
        if (!__any_sync(0xffffffffu, unlike(w, at, n, lane, 32))) return at;
      }
    }
    return w;
  };
  const int first = a.V <= 4096 ? a.V : 32 * E;   // (short rows to their end)
  for (int w = warp; w < a.W; w += WARPS) {
    const int r = search(w, 0, first);
    if (lane == 0) { like[w] = r; differ[w] = 0; }
  }
  pick_sync<THREADS>();
  if (first < a.V) {
    for (int w = 0; w < a.W; ++w)
      if (like[w] < w && unlike(w, like[w], a.V, tid, THREADS)) differ[w] = 1;
    pick_sync<THREADS>();
    for (int w = warp; w < a.W; w += WARPS)   // (alike at first only: the next one that is so to the end)
      if (differ[w]) {
        const int r = search(w, like[w] + 1, a.V);
        if (lane == 0) like[w] = r;
      }
    pick_sync<THREADS>();
  }
  // (who is found is the first of its kind: what it has stays)
  if (tid < a.W && like[tid] < tid) { base[tid] = base[like[tid]]; line[tid] = line[like[tid]]; }
  pick_sync<THREADS>();
}

// the pick of sequence b by a CTA; first: its first row in the list that was cut into runs, seg_max and parts: from there on
template <typename T, int THREADS>
__device__ __forceinline__ void beam_pick(const BeamArgs& a, int b, int first, const Beams& beams, const float* seg_max, const float2* all_parts) {
  constexpr int E = Logit<T>::E, SEG = 32 * E, WARPS = THREADS / 32, PER = PICK_PER;
  __shared__ double s_key[PICK_CAP], s_keep[BEAM_MAX_N], s_base[BEAM_MAX_W];
  __shared__ float s_max[BEAM_MAX_W];
  __shared__ float2 s_line[BEAM_MAX_W];   // a beam's score_of as a line in fp32: what a logit of 0 would have, and what that is off by
  __shared__ int s_thread[THREADS], s_at[PICK_CAP], s_keep_at[BEAM_MAX_N], s_tops[BEAM_MAX_N + 2 * WARPS], s_count, s_bound, s_one_score;
  __shared__ int3 s_seg[BEAM_MAX_N];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, N = a.N;
  const Best best{s_key, s_at, s_keep, s_keep_at, &s_count, s_thread, s_tops, &s_bound};
  const int all = a.W * a.n_seg;
  // A warp takes the segments of one beam, 32 PER at a time; those of the first time round are on their way while the beams are
  // looked at.  (Fewer at a time where there are warps enough: 8.7 us became 9.1 for 4 x 32000.)
  const int chunks = (a.n_seg + 32 * PER - 1) / (32 * PER), units = a.W * chunks;
  float held[PER];
  auto load = [&](int unit) {
    const int w = unit / chunks, r0 = (unit - w * chunks) * 32 * PER + lane;
#pragma unroll
    for (int j = 0; j < PER; ++j) held[j] = r0 + 32 * j < a.n_seg ? seg_max[(long long)w * a.n_seg + r0 + 32 * j] : -INFINITY;
    return make_int2(w, r0);
  };
  int2 place = warp < units ? load(warp) : make_int2(0, 0);
  // a beam's part of its candidates' scores, -inf where it has none: c = base + (l - max) / T
  auto parts_of = [&](int w) { return ((first + w) * a.groups + a.groups - 1) / a.run - (first + w) * a.groups / a.run + 1; };
  float2 ahead = make_float2(-INFINITY, 0.f);   // (so is a warp's first part)
  if (warp < a.W && lane < a.max_parts) ahead = all_parts[(long long)warp * a.max_parts + lane];   // (those behind its own are not used)
  if (tid == 0) s_one_score = 0;
  pick_sync<THREADS>();   // (`beams` is there)
  // beams of one score may be alike: a thread compares one with 32 others (the last warps, which have no parts to add up, where there are few)
  if (const int w = (THREADS - 1 - tid) % BEAM_MAX_W, r0 = (THREADS - 1 - tid) / BEAM_MAX_W * 32; w < a.W && isfinite(beams.score[w])) {
    bool same = false;
#pragma unroll 4
    for (int r = r0; r < min(r0 + 32, w); ++r) same |= beams.score[r] == beams.score[w];
    if (same) s_one_score = 1;
  }
  for (int w = warp; w < a.W; w += WARPS) {
    const float2* parts = all_parts + (long long)w * a.max_parts;
    const int n_parts = parts_of(w);
    float m = -INFINITY, s = 0.f;
    for (int p0 = 0; p0 < n_parts; p0 += 32) {   // (one round, but for few rows that are long)
      float2 v = make_float2(-INFINITY, 0.f);
      if (p0 + lane < n_parts) v = w == warp && p0 == 0 ? ahead : parts[p0 + lane];
      warp_merge(v.x, v.y, a.c);
      const float t = fmaxf(m, v.x), r = t == -INFINITY ? 0.f : t;
      s = s * ex2((m - r) * a.c) + v.y * ex2((v.x - r) * a.c);
      m = t;
    }
    if (lane == 0) {
      const float score = beams.score[w];
      const bool live = !beams.done[w] && isfinite(score) && isfinite(m) && s > 0.f && s < INFINITY;   // (else its parts were not written)
      const double base = live ? (double)score - log_of(s) : -INFINITY;
      const float at0 = (float)(base - (double)m * a.inv_t);
      s_base[w] = base;
      s_max[w] = m;
      // (-inf: no beam; a start outside fp32's range: nothing is known of the scores)
      s_line[w] = !live ? make_float2(-INFINITY, 0.f) : (isfinite(at0) ? make_float2(at0, fmaf(fabsf(at0), 4.7683716e-7f, 1e-36f)) : make_float2(0.f, INFINITY));
    }
  }
  if (tid == 0) s_count = 0;
  pick_sync<THREADS>();
  if (__builtin_expect(s_one_score, 0)) alike_beams<T, THREADS>(a, b * a.W, beams, s_base, s_max, s_line, s_at, s_thread);
  auto score_of = [&](int w, float l) { return s_base[w] > -INFINITY ? s_base[w] + ((double)l - (double)s_max[w]) * a.inv_t : -INFINITY; };
  // The N best segments.  Scores are first taken in fp32, a line in the logit, with what their roundings may come to (the line's
  // start, 1 / T, one of the fused operation: 2^-24 each of numbers no larger than the score's and the start's together): at
  // least N reach the bound with the least that they may be, and only those that may reach it are scored in 64 bits
  float top = -INFINITY;
  for (int u = warp; u < units; u += WARPS) {
    if (u != warp) place = load(u);
    const float2 line = s_line[place.x];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const float v = fmaf(held[j], a.inv_t32, line.x);
      top = fmaxf(top, v - fmaf(fabsf(v), 4.7683716e-7f, line.y));   // (NaN, from a score of -inf, is left out)
    }
  }
  const float least = best_bound<THREADS>(best, top, N);
  for (int u = warp; u < units; u += WARPS) {
    if (units > WARPS) place = load(u);
    const float2 line = s_line[place.x];
    if (!(line.x > -INFINITY)) continue;
    unsigned pass = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const float v = fmaf(held[j], a.inv_t32, line.x);
      // (what left fp32's range may be anything)
      if (held[j] > -INFINITY && !(v + fmaf(fabsf(v), 4.7683716e-7f, line.y) < least)) pass |= 1u << j;
    }
#pragma unroll 1
    for (; pass; pass &= pass - 1) {
      const int i = place.x * a.n_seg + place.y + 32 * (__ffs(pass) - 1);
      best_push(best, score_of(place.x, seg_max[i]), i);
    }
  }
  pick_sync<THREADS>();
  // few more than N: all are read, else the N best
  int segs = s_count;
  const bool all_read = segs <= BEAM_MAX_N;
  double bound = least;
  if (!all_read) {
    segs = segs > PICK_CAP ? best_rounds<THREADS>(best, N, all, [&](int i, int* at) { *at = i; return score_of(i / a.n_seg, seg_max[i]); })
                           : best_rank<THREADS>(best, N);
    bound = segs == N ? s_keep[N - 1] : -INFINITY;
  }
  const int* const from = all_read ? s_at : s_keep_at;
  for (int i = tid; i < segs; i += THREADS) {   // each one's beam, and the token that it begins with (the row's first, or some before it)
    const int w = from[i] / a.n_seg;
    int shift;
    row_begin<T>(a, b * a.W + w, &shift);
    s_seg[i] = make_int3(w, (from[i] - w * a.n_seg) * SEG - shift, 0);
  }
  pick_sync<THREADS>();
  // their elements that reach the bound, and the beams that are done
  auto ended = [&](int w, int* at) {            // beam w's candidate, if it is done
    const float s = beams.done[w] ? beams.score[w] : -INFINITY;
    *at = w * a.V + a.end_token;
    return isfinite(s) ? (double)s : -(double)INFINITY;
  };
  auto row_of = [&](int w) { return reinterpret_cast<const T*>(a.logits) + (long long)(b * a.W + w) * a.row_stride; };
  // Where there are few segments to a candidate their maxima hardly thin the elements, and a bound from the elements does: 9 x 13 x 147,
  // 25 candidates 17.1 -> 10.7 us, 56 x 2 x 255, 6 candidates 13.5 -> 11.2, 20 x 15000, 127 candidates 51 -> 24, 60 drawn selections 10.45 -> 10.0 in the mean; 39 x 466, 3
  // candidates, where the maxima would have done, 8.5 -> 9.9
  if (N > 1 && all < PICK_FEW * N)
    bound = fmax(bound, (double)best_elements<THREADS>(best, N, segs, [&](int i, int lane) {
      const int3 sg = s_seg[i];
      return __double2float_rd(score_of(sg.x, Logit<T>::top(load_piece(row_of(sg.x), sg.y + lane * E, 0, a.V))));
    }));
  if (tid == 0) s_count = 0;
  for (int i = tid; i < segs; i += THREADS) {   // the least logit that may reach the bound, rounded down, by which nearly all are told
    const double base = s_base[s_seg[i].x], m = s_max[s_seg[i].x], off = (bound - base) * a.t;
    const float low = __double2float_rd(m + off - (fabs(m) + fabs(off) + fabs(base) * a.t) * 1e-12);
    s_seg[i].z = __float_as_int(fmaxf(low, -3.4028235e38f));   // (-inf is no candidate)
  }
  pick_sync<THREADS>();
#pragma unroll 1
  for (int i0 = warp; i0 < segs; i0 += 4 * WARPS) {
    uint4 u[4];
    unsigned pass = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + j * WARPS >= segs) continue;
      const int3 sg = s_seg[i0 + j * WARPS];
      u[j] = load_piece(row_of(sg.x), sg.y + lane * E, 0, a.V);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i0 + j * WARPS >= segs) continue;
      const float low = __int_as_float(s_seg[i0 + j * WARPS].z);
      float f[E];
      Logit<T>::unpack(u[j], f);
#pragma unroll
      for (int e = 0; e < E; ++e) pass |= (f[e] >= low ? 1u : 0u) << (j * E + e);
    }
#pragma unroll 1
    for (; pass; pass &= pass - 1) {
      const int bit = __ffs(pass) - 1;
      const int3 sg = s_seg[i0 + bit / E * WARPS];
      const int token = sg.y + lane * E + bit % E;
      const double v = score_of(sg.x, Logit<T>::get(row_of(sg.x) + token));
      if (v >= bound) best_push(best, v, sg.x * a.V + token);
    }
  }
  if (a.done && tid < a.W) {
    int at;
    const double v = ended(tid, &at);
    if (v >= bound && v > -INFINITY) best_push(best, v, at);
  }
  pick_sync<THREADS>();
  auto element = [&](int i, int* at) {          // element i of the segments, one behind the other, then the done beams
    if (i >= segs * SEG) return ended(i - segs * SEG, at);
    const int3 sg = s_seg[i / SEG];
    const int v = sg.y + i % SEG;
    *at = sg.x * a.V + v;
    return v >= 0 && v < a.V ? score_of(sg.x, Logit<T>::get(row_of(sg.x) + v)) : -(double)INFINITY;
  };
  const int n = s_count > PICK_CAP ? best_rounds<THREADS>(best, N, segs * SEG + (a.done ? a.W : 0), element) : best_rank<THREADS>(best, N);
  for (int i = tid; i < N; i += THREADS) {
    const bool there = i < n;
    const int at = there ? s_keep_at[i] : 0, w = at / a.V, v = at - w * a.V;
    const long long o = (long long)b * N + i;
    a.out_scores[o] = there ? (float)s_keep[i] : -INFINITY;
    a.out_parents[o] = there ? b * a.W + w : -1;
    a.out_tokens[o] = there ? v : -1;
    if (a.out_done) a.out_done[o] = there && (v == a.end_token || beams.done[w]);
  }
}

// With a CTA to each part of a row 64 x 4 rows of 131071 took 20 us, as runs 15.  Neighbouring runs go to different CTAs, so that
// beams that are skipped are spread over all.
template <typename T>
__global__ void __launch_bounds__(SCAN_THREADS, 4) beam_scan_kernel(const __grid_constant__ BeamArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  beam_scan<T>(a, 0, a.B * a.W, (threadIdx.x >> 5) * gridDim.x + blockIdx.x, a.seg_max, a.parts);
}
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) beam_pick_kernel(const __grid_constant__ BeamArgs a) {
  __shared__ Beams s_beams;
  const int row = blockIdx.x * a.W;
  pdl_launch_dependents();
  pdl_wait();
  beams_load<THREADS>(a, blockIdx.x, s_beams);
  beam_pick<T, THREADS>(a, blockIdx.x, row, s_beams, a.seg_max + (long long)row * a.n_seg, a.parts + (long long)row * a.max_parts);
}
// Both for little work, a cluster to a sequence: what the scan finds goes straight to the shared memory of the CTA that picks (half
// of its threads do: the pick's steps cost by the warp).  It saves a launch, which is the host's time: one prompt of 4 x 32000 takes 9.2
// us a call (8.9 replayed from a graph), of 8 x 32000 10.5 (10.1), eight of those 10.9 (10.5); as two launches 10.9 (8.7) and
// 11.1 (10.7), and 16 where the host is slow.
template <typename T>
__global__ void __cluster_dims__(ONE_CTAS, 1, 1) __launch_bounds__(ONE_THREADS) beam_one_kernel(const __grid_constant__ BeamArgs a) {
  __shared__ Beams s_beams;
  __shared__ float s_segs[ONE_RUN * ONE_WARPS * SCAN_SEGS];
  __shared__ float2 s_parts[ONE_WARPS + 2 * BEAM_MAX_W];
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), b = blockIdx.x / ONE_CTAS;
  pdl_launch_dependents();
  cl.sync();   // (the CTA that picks has to be there before others write to it)
  pdl_wait();
  if (rank == 0) beams_load<ONE_THREADS>(a, b, s_beams);
  beam_scan<T>(a, b * a.W, a.W, (threadIdx.x >> 5) * ONE_CTAS + rank, cl.map_shared_rank(s_segs, 0), cl.map_shared_rank(s_parts, 0));
  cl.sync();
  if (rank == 0 && threadIdx.x < ONE_PICK) beam_pick<T, ONE_PICK>(a, b, 0, s_beams, s_segs, s_parts);
}

int no(int code, const char* msg) {
  sps_set_global_error(msg);
  return code;
}
const char* bad_shape(int B, int W, int V) {
  if (B < 0 || B > BEAM_MAX_B || W < 1 || W > BEAM_MAX_W || V < 1 || V > 1 << 24) return "beams: B must be 0 .. 8192, W 1 .. 128, V 1 .. 2^24";
  if ((int64_t)W * V > INT_MAX || (int64_t)B * W * ((V + 514) / 512) > INT_MAX) return "beams: W x V must stay below 2^31, B x W x V below 2^40";
  return nullptr;
}
int64_t up(int64_t n) { return (n + 255) / 256 * 256; }

// of fp32 rows, which have the most, shifted by up to 3: segments, and parts (a run is one group at least)
int64_t most_segs(int V) { return ((int64_t)V + 3 + 127) / 128; }
int max_parts(int V) { return (int)((most_segs(V) + SCAN_SEGS - 1) / SCAN_SEGS) + 1; }
template <typename T>
cudaError_t beam_launch(BeamArgs& a, int num_sm, cudaStream_t st) {
  constexpr int E = Logit<T>::E, SEG = 32 * E;
  const bool aligned = (((uintptr_t)a.logits | (uintptr_t)(a.row_stride * (int64_t)sizeof(T))) & 15) == 0;
  a.n_seg = (a.V + (aligned ? 0 : E - 1) + SEG - 1) / SEG;
  a.groups = (a.n_seg + SCAN_SEGS - 1) / SCAN_SEGS;
  a.max_parts = max_parts(a.V);
  const long long all = (long long)a.B * a.W * a.groups, warps = (long long)num_sm * 4 * SCAN_WARPS;
  // little work, no more than ONE_RUN groups to a warp, and clusters that fit beside one another (with 18 of 8 x 32000 they do not:
  // 15.5 us against 12.6): one launch
  if ((long long)a.W * a.groups <= ONE_RUN * ONE_WARPS && a.B * ONE_CTAS <= num_sm / 2) {
    a.run = (a.W * a.groups + ONE_WARPS - 1) / ONE_WARPS;
    a.max_parts = (a.groups + a.run - 1) / a.run + 1;   // W of them: ONE_WARPS + 2 W at most
    return launch_k(beam_one_kernel<T>, dim3(a.B * ONE_CTAS), dim3(ONE_THREADS), 0, st, a);
  }
  a.run = (int)((all + warps - 1) / warps);
  const long long runs = (all + a.run - 1) / a.run;
  cudaError_t e = launch_k(beam_scan_kernel<T>, dim3((unsigned)((runs + SCAN_WARPS - 1) / SCAN_WARPS)), dim3(SCAN_THREADS), 0, st, a);
  if (e != cudaSuccess) return e;
  // a small CTA for few segments: what each warp does for itself then costs less than the walk over them
  if ((long long)a.W * a.n_seg <= 2048) return launch_k(beam_pick_kernel<T, 512>, dim3(a.B), dim3(512), 0, st, a);
  return launch_k(beam_pick_kernel<T, 1024>, dim3(a.B), dim3(1024), 0, st, a);
}
}  // namespace

extern "C" {

int64_t sps_beam_select_workspace_bytes(int32_t B, int32_t W, int32_t V) {
  if (const char* why = bad_shape(B, W, V)) { no(SPS_EINVAL, why); return -1; }
  const int64_t rows = (int64_t)B * W;
  return up(rows * most_segs(V) * 4) + up(rows * max_parts(V) * 8);
}

int sps_beam_select(const void* logits, int32_t dtype, int64_t row_stride, int32_t B, int32_t W, int32_t V, double temperature,
                    const float* scores, const int32_t* done, int32_t end_token, int32_t N, float* out_scores, int32_t* out_parents,
                    int32_t* out_tokens, int32_t* out_done, void* workspace, void* stream) {
  const char* why = bad_shape(B, W, V);
  if (why) return no(SPS_EINVAL, why);
  if (dtype != 0 && dtype != 1) return no(SPS_EINVAL, "logits: dtype must be 0 (fp32) or 1 (bf16)");
  if (N < 1 || N > BEAM_MAX_N) return no(SPS_EINVAL, "N must be 1 .. 128");
  if (row_stride < 0) return no(SPS_EINVAL, "logits: negative stride");
  const float c = (float)(1.4426950408889634 / temperature);
  if (!(temperature > 0.0) || !std::isfinite(c) || c < 1.1754944e-38f) return no(SPS_EINVAL, "temperature must be above 0 and finite, its inverse too");
  if (end_token < -1 || end_token >= V) return no(SPS_EINVAL, "end_token must be a token, or -1");
  if (done && end_token < 0) return no(SPS_EINVAL, "done needs an end_token");
  if (B == 0) return SPS_OK;
  if (!logits || !scores || !out_scores || !out_parents || !out_tokens) return no(SPS_EINVAL, "null argument");
  if (((uintptr_t)logits & (dtype == 0 ? 3 : 1)) ||
      (((uintptr_t)scores | (uintptr_t)done | (uintptr_t)out_scores | (uintptr_t)out_parents | (uintptr_t)out_tokens | (uintptr_t)out_done) & 3))
    return no(SPS_EINVAL, "pointers must be aligned to their elements");
  if (!workspace || ((uintptr_t)workspace & 15)) return no(SPS_EINVAL, "workspace null or not 16-byte aligned");
  BeamArgs a{};
  a.logits = logits; a.row_stride = row_stride; a.B = B; a.W = W; a.V = V; a.N = N;
  a.t = temperature; a.inv_t = 1.0 / temperature; a.inv_t32 = (float)a.inv_t; a.c = c; a.scores = scores; a.done = done; a.end_token = end_token;
  a.out_scores = out_scores; a.out_parents = out_parents; a.out_tokens = out_tokens; a.out_done = out_done;
  a.seg_max = (float*)workspace;
  a.parts = (float2*)((char*)workspace + up((int64_t)B * W * most_segs(V) * 4));
  const cudaError_t e = dtype == 0 ? beam_launch<float>(a, paged_sms(), (cudaStream_t)stream) : beam_launch<__nv_bfloat16>(a, paged_sms(), (cudaStream_t)stream);
  return e == cudaSuccess ? SPS_OK : no(SPS_ECUDA, cudaGetErrorString(e));
}

}  // extern "C"
