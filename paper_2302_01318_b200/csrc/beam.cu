// The selection of a beam step (sps_beam_select): the best continuations over a sequence's beams and the vocabulary.
#include <climits>
#include <cmath>

#include "paged.cuh"

// ------------------------------------------------------------------------------------------------------------------
// c[w, v] = s[w] + l[w, v] / T - log sum_u exp(l[w, u] / T); the N best (w, v) of each sequence, ties to the lowest w V + v.
//
// Two kernels.  The scan reads every logit once: per row running maxima and sums of exponentials, and the maximum of every
// segment of 512 bytes.  A row's order is its logits', so the N best elements lie in the N segments whose maxima score
// best (ties to the lower segment: any element outside has N better ones in them) -- whatever the numbers are.  The pick, a
// CTA per sequence, finds those segments, reads them again (N x 512 bytes, from L2) and picks the N best elements.
// Bound by HBM with many rows, by latency with few.
// Candidates are compared in 64 bits, from exact logits and a sum of fp32 exponentials (relative error about 2^-22), so that
// far scores keep the order of their last bits; results are rounded once.
// ------------------------------------------------------------------------------------------------------------------
namespace {

constexpr int SCAN_THREADS = 256, SCAN_WARPS = 8, SCAN_SEGS = 4;      // segments a warp loads at a time
constexpr int SCAN_PART = SCAN_WARPS * SCAN_SEGS;                     // the least segments of a part (a CTA's)
constexpr int PICK_THREADS = 256, PICK_WARPS = 8, PICK_CAP = 512;
constexpr int BEAM_MAX_W = 128, BEAM_MAX_N = 128;

struct BeamArgs {
  const void* logits;
  long long row_stride;
  int B, W, V, N;
  double inv_t;
  float c;                   // log2(e) / T
  const float* scores;
  const int32_t* done;       // or null
  int end_token;
  float* out_scores;
  int32_t *out_parents, *out_tokens, *out_done;   // out_done: or null
  float* seg_max;            // [B W][n_seg]
  float2* parts;             // [B W][n_parts]: maximum, sum of exponentials
  int n_seg, n_parts, part_segs;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// numbers in the order of floats; NaN never comes here (maxima leave it out)
__device__ __forceinline__ int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }

template <typename T> struct Logit;
template <> struct Logit<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void unpack(uint4 u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
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
};

// a beam that reads its logits: it has a score, and is not done
__device__ __forceinline__ bool beam_reads(const BeamArgs& a, int row) {
  return !(a.done && a.done[row]) && isfinite(a.scores[row]);
}

// (m, s) of a set and of another: sums are relative to the maxima
__device__ __forceinline__ void merge(float& m, float& s, float m1, float s1, float c) {
  const float t = fmaxf(m, m1), r = t == -INFINITY ? 0.f : t;
  s = s * ex2((m - r) * c) + s1 * ex2((m1 - r) * c);
  m = t;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(SCAN_THREADS) beam_scan_kernel(const __grid_constant__ BeamArgs a) {
  constexpr int E = Logit<T>::E, SEG = 32 * E;
  __shared__ float s_m[SCAN_WARPS], s_s[SCAN_WARPS];
  pdl_launch_dependents();
  const int row = blockIdx.x / a.n_parts, part = blockIdx.x - row * a.n_parts;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  if (!beam_reads(a, row)) return;
  const T* x = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
  const int s0 = part * a.part_segs, s1 = min(s0 + a.part_segs, a.n_seg);
  float m = -INFINITY, s = 0.f;
  for (int seg = s0 + warp * SCAN_SEGS; seg < s1; seg += SCAN_PART) {
    float f[SCAN_SEGS][E];
    const bool whole = (long long)(seg + SCAN_SEGS) * SEG <= a.V;
    if (VEC && whole) {
      uint4 u[SCAN_SEGS];
#pragma unroll
      for (int j = 0; j < SCAN_SEGS; ++j) u[j] = *reinterpret_cast<const uint4*>(x + (seg + j) * SEG + lane * E);
#pragma unroll
      for (int j = 0; j < SCAN_SEGS; ++j) Logit<T>::unpack(u[j], f[j]);
    } else {
#pragma unroll
      for (int j = 0; j < SCAN_SEGS; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int v = (seg + j) * SEG + e * 32 + lane;
          f[j][e] = v < a.V ? Logit<T>::get(x + v) : -INFINITY;
        }
    }
    float top = -INFINITY;
    int best = 0;
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j) {
      float t = f[j][0];
#pragma unroll
      for (int e = 1; e < E; ++e) t = fmaxf(t, f[j][e]);
      t = fmaxf(t, -INFINITY);      // (NaN left out)
      top = fmaxf(top, t);
      const int w = __reduce_max_sync(0xffffffffu, ordered(t));
      if (lane == j) best = w;
    }
    if (lane < SCAN_SEGS && seg + lane < s1) a.seg_max[(long long)row * a.n_seg + seg + lane] = unordered(best);
    const float m1 = fmaxf(m, top), r = m1 == -INFINITY ? 0.f : m1;
    s *= ex2((m - r) * a.c);
    m = m1;
#pragma unroll
    for (int j = 0; j < SCAN_SEGS; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) s += ex2((f[j][e] - r) * a.c);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m1 = __shfl_xor_sync(0xffffffffu, m, o), v1 = __shfl_xor_sync(0xffffffffu, s, o);
    merge(m, s, m1, v1, a.c);
  }
  if (lane == 0) { s_m[warp] = m; s_s[warp] = s; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < SCAN_WARPS; ++w) merge(m, s, s_m[w], s_s[w], a.c);
    a.parts[(long long)row * a.n_parts + part] = make_float2(m, s);
  }
}

// The N best of a stream of (score, place), places falling ties to the lowest: a buffer of PICK_CAP and the bound below which
// nothing is taken, the N-th best so far once there are N.
struct Best {
  double* key[2];
  int* at[2];
  int* count;
  int side;
  double bound;
  int bound_at;
};
__device__ __forceinline__ bool better(double k, int i, double k1, int i1) { return k > k1 || (k == k1 && i < i1); }
__device__ __forceinline__ void best_push(Best& b, double k, int i) {
  if (!better(k, i, b.bound, b.bound_at)) return;
  const int n = atomicAdd(b.count, 1);
  b.key[b.side][n] = k;
  b.at[b.side][n] = i;
}
// leaves the N best in order and raises the bound (every thread of the CTA calls it); the buffer's count is returned
__device__ __forceinline__ int best_prune(Best& b, int N) {
  __syncthreads();
  const int n = *b.count, keep = min(n, N);
  const double* key = b.key[b.side];
  const int* at = b.at[b.side];
  for (int i = threadIdx.x; i < n; i += PICK_THREADS) {
    const double k = key[i];
    const int p = at[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += better(key[j], at[j], k, p);
    if (r < N) { b.key[b.side ^ 1][r] = k; b.at[b.side ^ 1][r] = p; }
  }
  __syncthreads();
  if (threadIdx.x == 0) *b.count = keep;
  b.side ^= 1;
  if (n >= N) { b.bound = b.key[b.side][N - 1]; b.bound_at = b.at[b.side][N - 1]; }
  __syncthreads();
  return keep;
}
__device__ __forceinline__ void best_room(Best& b, int N) {   // room for a push by every thread
  __syncthreads();
  const int n = *b.count;
  if (n > PICK_CAP - PICK_THREADS) best_prune(b, N);
  else __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(PICK_THREADS) beam_pick_kernel(const __grid_constant__ BeamArgs a) {
  constexpr int E = Logit<T>::E, SEG = 32 * E;
  __shared__ double s_key[2][PICK_CAP], s_base[BEAM_MAX_W];
  __shared__ float s_max[BEAM_MAX_W];
  __shared__ int s_at[2][PICK_CAP], s_seg[BEAM_MAX_N], s_done[BEAM_MAX_W], s_count;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  pdl_wait();
  // a beam's part of its candidates' scores, -inf where it has none: c = base + (l - max) / T
  for (int w = warp; w < a.W; w += PICK_WARPS) {
    const int row = b * a.W + w;
    double base = -INFINITY;
    float m = -INFINITY;
    if (beam_reads(a, row)) {
      for (int p = lane; p < a.n_parts; p += 32) m = fmaxf(m, a.parts[(long long)row * a.n_parts + p].x);
      m = warp_max(m);
      const float r = m == -INFINITY ? 0.f : m;
      double s = 0.0;
      for (int p = lane; p < a.n_parts; p += 32) {
        const float2 v = a.parts[(long long)row * a.n_parts + p];
        s += (double)v.y * exp(((double)v.x - (double)r) * a.inv_t);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (isfinite(m) && s > 0.0 && s < INFINITY) base = (double)a.scores[row] - log(s);
    }
    if (lane == 0) { s_base[w] = base; s_max[w] = m; s_done[w] = a.done ? a.done[row] : 0; }   // (out_done may be done)
  }
  Best best{{s_key[0], s_key[1]}, {s_at[0], s_at[1]}, &s_count, 0, -INFINITY, 0};   // (-inf is not taken)
  if (tid == 0) s_count = 0;
  __syncthreads();
  // the N best segments
  const int all = a.W * a.n_seg;
  for (int i0 = 0; i0 < all; i0 += PICK_THREADS) {
    const int i = i0 + tid;
    best_room(best, a.N);
    if (i < all) {
      const int w = i / a.n_seg;
      if (s_base[w] > -INFINITY) best_push(best, s_base[w] + ((double)a.seg_max[(long long)b * all + i] - (double)s_max[w]) * a.inv_t, i);
    }
  }
  const int segs = best_prune(best, a.N);
  for (int i = tid; i < segs; i += PICK_THREADS) s_seg[i] = best.at[best.side][i];
  __syncthreads();
  if (tid == 0) s_count = 0;
  // their elements that reach the N-th segment's maximum, and the beams that are done
  best.bound_at = INT_MAX;
  for (int i0 = 0; i0 < segs; i0 += PICK_WARPS) {
    const int i = i0 + warp;
    const int w = i < segs ? s_seg[i] / a.n_seg : 0, v0 = i < segs ? (s_seg[i] - w * a.n_seg) * SEG : a.V;
    const T* x = reinterpret_cast<const T*>(a.logits) + (long long)(b * a.W + w) * a.row_stride;
    float f[E];
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = v0 + e * 32 + lane < a.V ? Logit<T>::get(x + v0 + e * 32 + lane) : -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      best_room(best, a.N);
      if (f[e] > -INFINITY) best_push(best, s_base[w] + ((double)f[e] - (double)s_max[w]) * a.inv_t, w * a.V + v0 + e * 32 + lane);
    }
  }
  best_room(best, a.N);
  if (tid < a.W && s_done[tid] && isfinite(a.scores[b * a.W + tid]))
    best_push(best, (double)a.scores[b * a.W + tid], tid * a.V + a.end_token);
  const int n = best_prune(best, a.N);
  for (int i = tid; i < a.N; i += PICK_THREADS) {
    const bool there = i < n;
    const int at = there ? best.at[best.side][i] : 0, w = at / a.V, v = at - w * a.V;
    const long long o = (long long)b * a.N + i;
    a.out_scores[o] = there ? (float)best.key[best.side][i] : -INFINITY;
    a.out_parents[o] = there ? b * a.W + w : -1;
    a.out_tokens[o] = there ? v : -1;
    if (a.out_done) a.out_done[o] = there && (v == a.end_token || s_done[w]);
  }
}

int no(int code, const char* msg) {
  sps_set_global_error(msg);
  return code;
}
const char* bad_shape(int B, int W, int V) {
  if (B < 0 || B > 1 << 16 || W < 1 || W > BEAM_MAX_W || V < 1 || V > 1 << 24) return "beams: B must be 0 .. 2^16, W 1 .. 128, V 1 .. 2^24";
  const int64_t parts = ((int64_t)V + 128 * SCAN_PART - 1) / (128 * SCAN_PART);
  if ((int64_t)W * V > INT_MAX || (int64_t)B * W * parts > INT_MAX) return "beams: W x V must stay below 2^31, B x W x V below 2^43";
  return nullptr;
}
int64_t up(int64_t n) { return (n + 255) / 256 * 256; }

template <typename T>
cudaError_t beam_launch(BeamArgs& a, cudaStream_t st) {
  constexpr int SEG = 32 * Logit<T>::E;
  a.n_seg = (a.V + SEG - 1) / SEG;
  const int rows = a.B * a.W;
  a.part_segs = SCAN_PART;
  a.n_parts = (a.n_seg + a.part_segs - 1) / a.part_segs;
  const bool vec = (((uintptr_t)a.logits | (uintptr_t)(a.row_stride * (int64_t)sizeof(T))) & 15) == 0;
  const dim3 grid((unsigned)((long long)rows * a.n_parts));
  cudaError_t e = vec ? launch_k(beam_scan_kernel<T, true>, grid, dim3(SCAN_THREADS), 0, st, a) : launch_k(beam_scan_kernel<T, false>, grid, dim3(SCAN_THREADS), 0, st, a);
  if (e == cudaSuccess) e = launch_k(beam_pick_kernel<T>, dim3(a.B), dim3(PICK_THREADS), 0, st, a);
  return e;
}

}  // namespace

extern "C" {

int64_t sps_beam_select_workspace_bytes(int32_t B, int32_t W, int32_t V) {
  if (const char* why = bad_shape(B, W, V)) { no(SPS_EINVAL, why); return -1; }
  const int64_t segs = ((int64_t)V + 127) / 128, parts = (segs + SCAN_PART - 1) / SCAN_PART;
  return 256 + up((int64_t)B * W * segs * 4) + up((int64_t)B * W * parts * 8);
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
  a.inv_t = 1.0 / temperature; a.c = c; a.scores = scores; a.done = done; a.end_token = end_token;
  a.out_scores = out_scores; a.out_parents = out_parents; a.out_tokens = out_tokens; a.out_done = out_done;
  const int64_t segs = ((int64_t)V + 127) / 128;
  a.seg_max = (float*)((char*)workspace + 256);
  a.parts = (float2*)((char*)workspace + 256 + up((int64_t)B * W * segs * 4));
  const cudaError_t e = dtype == 0 ? beam_launch<float>(a, (cudaStream_t)stream) : beam_launch<__nv_bfloat16>(a, (cudaStream_t)stream);
  return e == cudaSuccess ? SPS_OK : no(SPS_ECUDA, cudaGetErrorString(e));
}

}  // extern "C"
