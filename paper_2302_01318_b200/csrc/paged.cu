// Rotary positions and the append to a paged cache: one kernel for both (sps_rotary is the append's query part with given
// positions), and the C entry points of the paged-cache calls.
#include <cmath>
#include <atomic>
#include <type_traits>

#include "paged.cuh"

// ------------------------------------------------------------------------------------------------------------------
// y = gain R(p f) x on the first rot elements of every head, the rest copied; keys and values to their slots.
//
// Bound by HBM: every element is read once and written once, 6 operations per pair.  The angles would not be cheap per
// element -- a 64-bit product and reduction and a sine and cosine each --, so a CTA works them out once per row, shares
// them through shared memory, and rotates many heads of that row by them.  A unit is two 16-byte pieces of x half a head
// apart -- in the halves layout both halves of its pairs, apart by half the rotated part --; a thread keeps its place in the
// head and goes from head to head, 64 bytes of loads in flight, through queries, keys and values and the rows of its CTA.
// What a unit costs beside its bytes (where it is, what is done to it) counts: one piece to a unit took a tenth longer.
// The first units are on their way before positions, page table and angles are looked at; what is left of that latency
// hides behind the SM's other CTAs.
// E = elements per access: 16 bytes of x when addresses, strides and the rotated part allow, else single elements.
// ------------------------------------------------------------------------------------------------------------------
namespace {

constexpr int ROT_THREADS = 256;
constexpr int ROT_PASSES = 4;     // batches of loads per thread, at most
constexpr int ROT_MAX_ROWS = 32;  // rows a CTA may share (small rows)

template <typename T> struct Elem;
template <> struct Elem<float> {
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};

template <typename T, int E> struct alignas(sizeof(T) * E) Pack { T v[E]; };
template <typename T, int E> __device__ __forceinline__ Pack<T, E> load_e(const T* p) { return *reinterpret_cast<const Pack<T, E>*>(p); }
// (pairs of bf16 in one instruction each way: element by element their conversions, not HBM, bound the kernel)
template <typename T, int E> __device__ __forceinline__ void unpack(const Pack<T, E>& k, float (&f)[E]) {
  if constexpr (sizeof(T) == 2 && E % 2 == 0) {
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const uint32_t u = reinterpret_cast<const uint32_t*>(&k)[i / 2];
      f[i] = __uint_as_float(u << 16);
      f[i + 1] = __uint_as_float(u & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = Elem<T>::get(k.v[i]);
  }
}
template <typename T, int E> __device__ __forceinline__ void store_e(T* p, const float (&f)[E]) {
  Pack<T, E> k;
  if constexpr (sizeof(T) == 2 && E % 2 == 0) {
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[i], f[i + 1]);
      reinterpret_cast<uint32_t*>(&k)[i / 2] = *reinterpret_cast<const uint32_t*>(&h);
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) k.v[i] = Elem<T>::put(f[i]);
  }
  *reinterpret_cast<Pack<T, E>*>(p) = k;
}

// cos and sin of p f: the angle in 64 bits, reduced to (-pi, pi], the rest of its rounding to 32 bits put back to first
// order (positions of millions keep their phase to fp32's last bits)
__device__ __forceinline__ float2 turn(double p, double f) {
  const double a = p * f;
  const double n = rint(a * 0.15915494309189535);
  double r = fma(-n, 6.283185307179586, a);
  r = fma(-n, 2.4492935982947064e-16, r);
  const float rf = (float)r, d = (float)(r - (double)rf);
  float s, c;
  sincosf(rf, &s, &c);
  return make_float2(fmaf(-d, s, c), fmaf(d, c, s));
}

// positions and cache slots (element offsets; -1: the row is skipped) of the CTA's rows, a row per warp
__device__ __forceinline__ void row_places(const RotaryArgs& a, int row0, int nr, int* s_pos, long long* s_slot) {
  const int lane = threadIdx.x & 31;
  if (a.positions) {
    for (int i = threadIdx.x; i < nr; i += ROT_THREADS) { s_pos[i] = a.positions[row0 + i]; s_slot[i] = 0; }
    return;
  }
  for (int i = threadIdx.x >> 5; i < nr; i += ROT_THREADS / 32) {
    const int row = row0 + i;
    // the sequence: as many as end at or before this row precede it
    int before = 0;
    for (int b0 = 0; b0 < a.s.B; b0 += 32) {
      const int b = b0 + lane;
      before += __popc(__ballot_sync(0xffffffffu, b < a.s.B && a.s.q_start[min(b, a.s.B - 1) + 1] <= row));
    }
    if (lane == 0) {
      long long slot = -1, pos = 0;
      if (before < a.s.B && row >= a.s.q_start[before]) {
        pos = (long long)a.s.kv_len[before] - a.s.q_start[before + 1] + row;
        if (pos >= paged_capacity(a.s)) paged_flag(a.s.status, SPS_PAGED_BAD_LENGTH);
        else if (pos >= 0) {
          const int page = a.s.pages[(long long)before * a.s.pages_ld + (pos >> a.s.page_shift)];
          if (page < 0 || page >= a.s.n_pages) paged_flag(a.s.status, SPS_PAGED_BAD_PAGE);
          else slot = (long long)page * a.y[1].row + (pos & (a.s.page_size - 1)) * a.pos_stride;
        }
      }
      s_slot[i] = slot;
      s_pos[i] = (int)pos;
    }
  }
}

// the turns of the CTA's rows; pair k of a row at (k % PU) (hr / PU) + k / PU, PU pairs to a piece: neighbouring pieces read
// neighbouring words
template <int PU>
__device__ __forceinline__ void row_turns(const RotaryArgs& a, int nr, const int* s_pos, float2* s_turn) {
  const int hr = a.rot >> 1, units = hr / PU;
  for (int i = threadIdx.x; i < nr * hr; i += ROT_THREADS) {
    const int r = i / hr, k = i - r * hr;
    float2 t = turn((double)s_pos[r], a.freq[k]);
    t.x *= a.gain;
    t.y *= a.transposed ? -a.gain : a.gain;
    s_turn[r * hr + (k % PU) * units + k / PU] = t;
  }
}

__device__ __forceinline__ int magic_div(int n, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)n, magic) : n; }   // magic 0: by 1

// UPT: units per thread and batch.  Single-element access (E = 1) takes the two elements of a pair as a unit.
template <typename TX, typename TQ, typename TC, int E, bool HALVES, int UPT>
__global__ void __launch_bounds__(ROT_THREADS, 4) rotary_kernel(const __grid_constant__ RotaryArgs a) {
  extern __shared__ float2 s_turn[];                 // [rows_per_cta][rot / 2]
  __shared__ int s_pos[ROT_MAX_ROWS];
  __shared__ long long s_slot[ROT_MAX_ROWS];
  constexpr int PU = HALVES ? E : (E == 1 ? 1 : E / 2);   // pairs of a rotated unit (halves, single pair) or piece (pairs)
  const int tid = threadIdx.x, hr = a.rot >> 1, uh = a.uh;
  const int rot_units = a.freq ? hr / PU : 0;        // of a head's units, or pieces: the rotated ones
  const int row0 = blockIdx.x * a.rows_per_cta, nr = min(a.rows_per_cta, a.rows - row0);
  const int h_lo = blockIdx.y * a.heads_per_cta, span = min(a.heads_per_cta, a.vheads - h_lo);   // this CTA's heads of each row
  const int all = nr * span;                         // (row, head) pairs
  const int slice = magic_div(tid, a.uh_magic);      // a thread's first pair, among the per_pass that a pass takes
  const int active = slice < a.per_pass;
  pdl_launch_dependents();
  pdl_wait();
  bool ready = false;
  for (int w = tid - slice * uh; w < uh; w += ROT_THREADS) {   // (once, unless a head has more units than the CTA threads)
    const bool turned = w < rot_units, turned1 = !HALVES && E > 1 && w + uh < rot_units;   // (turned1: the second piece)
    int e0, e1;                                      // the unit's pieces
    if (HALVES) {
      e0 = turned ? w * E : a.flat0 + (w - rot_units) * E;
      e1 = e0 + (turned ? hr : a.flat_half);
    } else if (E == 1) {
      e0 = 2 * w;
      e1 = e0 + 1;
    } else {
      e0 = w * E;
      e1 = e0 + uh * E;
    }
    for (int i0 = slice; i0 - slice < all; i0 += a.per_pass * UPT) {
      Pack<TX, E> lo[UPT], hi[UPT];
      int rr[UPT], kind[UPT], head[UPT];             // row of the CTA (-1: none); 0 queries, 1 keys, 2 values; head of them
#pragma unroll
      for (int j = 0; j < UPT; ++j) {
        const int i = i0 + j * a.per_pass;
        rr[j] = -1;
        if (i >= all || !active) continue;
        rr[j] = a.rows_per_cta == 1 ? 0 : magic_div(i, a.span_magic);   // several rows: the CTA has all of their heads
        head[j] = h_lo + i - rr[j] * span;
        kind[j] = 0;
        if (head[j] >= a.heads[0]) {
          head[j] -= a.heads[0];
          kind[j] = 1;
          if (head[j] >= a.heads[1]) { head[j] -= a.heads[1]; kind[j] = 2; }
        }
        const RowsView& x = a.x[kind[j]];
        const TX* src = reinterpret_cast<const TX*>(x.p) + (long long)(row0 + rr[j]) * x.row + (long long)head[j] * x.head;
        lo[j] = load_e<TX, E>(src + e0);
        hi[j] = load_e<TX, E>(src + e1);
      }
      if (!ready) {
        ready = true;
        row_places(a, row0, nr, s_pos, s_slot);
        __syncthreads();
        if (a.freq) {
          row_turns<PU>(a, nr, s_pos, s_turn);
          __syncthreads();
        }
      }
#pragma unroll
      for (int j = 0; j < UPT; ++j) {
        if (rr[j] < 0) continue;
        const long long slot = s_slot[rr[j]];
        if (slot < 0) continue;
        float f[E], g[E];
        unpack<TX, E>(lo[j], f);
        unpack<TX, E>(hi[j], g);
        if (kind[j] < 2) {
          const float2* tr = s_turn + rr[j] * hr + w;
          if constexpr (HALVES || E == 1) {
            if (turned) {
#pragma unroll
              for (int q = 0; q < E; ++q) {
                const float2 t = tr[q * rot_units];
                const float p = f[q], s = g[q];
                f[q] = p * t.x - s * t.y;
                g[q] = p * t.y + s * t.x;
              }
            }
          } else {
            auto turn_piece = [&](float (&v)[E], const float2* at) {
#pragma unroll
              for (int q = 0; q < E; q += 2) {
                const float2 t = at[(q >> 1) * rot_units];
                const float p = v[q], s = v[q + 1];
                v[q] = p * t.x - s * t.y;
                v[q + 1] = p * t.y + s * t.x;
              }
            };
            if (turned) turn_piece(f, tr);
            if (turned1) turn_piece(g, tr + uh);
          }
        }
        auto put = [&](auto* dst) {
          using T = typename std::remove_reference<decltype(*dst)>::type;
          store_e<T, E>(dst + e0, f);
          store_e<T, E>(dst + e1, g);
        };
        if (kind[j] == 0) put(reinterpret_cast<TQ*>(a.y[0].p) + (long long)(row0 + rr[j]) * a.y[0].row + (long long)head[j] * a.y[0].head);
        else put(reinterpret_cast<TC*>(a.y[kind[j]].p) + slot + (long long)head[j] * a.y[kind[j]].head);
      }
    }
  }
}

// ceil(2^32 / d): n / d is the high word of a product for n d < 2^32
uint32_t magic_of(int d) { return d > 1 ? (uint32_t)(((1ull << 32) + (unsigned)d - 1) / (unsigned)d) : 0; }

template <typename TX, typename TQ, typename TC, int E, bool HALVES, int UPT>
cudaError_t rotary_cut(RotaryArgs& a, int num_sm, cudaStream_t st) {
  const int hr = a.rot / 2;
  // batches per thread: as many as leave every SM 8 CTAs, up to ROT_PASSES
  long long passes = (long long)a.rows * a.vheads * a.uh / ((long long)num_sm * 8 * ROT_THREADS * UPT);
  passes = passes < 1 ? 1 : (passes > ROT_PASSES ? ROT_PASSES : passes);
  const int want = a.per_pass * UPT * (int)passes;   // (row, head) pairs of a CTA
  a.heads_per_cta = a.vheads < want ? a.vheads : want;
  int rpc = want / a.heads_per_cta;
  const int fit = hr > 0 ? 2048 / hr : ROT_MAX_ROWS;   // rows whose angles fit 16 KB
  if (rpc > ROT_MAX_ROWS) rpc = ROT_MAX_ROWS;
  if (rpc > fit) rpc = fit;
  a.rows_per_cta = rpc < 1 ? 1 : rpc;
  a.span_magic = magic_of(a.heads_per_cta);          // pairs of a CTA: at most 4096
  const size_t smem = sizeof(float2) * (size_t)a.rows_per_cta * (hr > 0 ? hr : 1);
  const dim3 grid(((unsigned)a.rows + a.rows_per_cta - 1) / a.rows_per_cta, (a.vheads + a.heads_per_cta - 1) / a.heads_per_cta);
  return launch_k(rotary_kernel<TX, TQ, TC, E, HALVES, UPT>, grid, dim3(ROT_THREADS), smem, st, a);
}

template <typename TX, typename TQ, typename TC, int E, bool HALVES>
cudaError_t rotary_go(RotaryArgs& a, int num_sm, cudaStream_t st) {
  constexpr int UPT = 2;
  a.uh = a.d_head / (2 * E);
  a.uh_magic = magic_of(a.uh);
  a.flat0 = a.freq ? a.rot : 0;
  a.flat_half = (a.d_head - a.flat0) / 2;
  a.vheads = a.heads[0] + a.heads[1] + a.heads[2];
  a.per_pass = a.uh < ROT_THREADS ? ROT_THREADS / a.uh : 1;
  // few rows (a decode step) are spread thinner, one unit per thread, so that more SMs share the latency
  if ((long long)a.rows * a.vheads * a.uh < (long long)num_sm * ROT_THREADS * UPT) return rotary_cut<TX, TQ, TC, E, HALVES, 1>(a, num_sm, st);
  return rotary_cut<TX, TQ, TC, E, HALVES, UPT>(a, num_sm, st);
}

bool aligned(const RowsView& v, int heads, int bytes, int esize) {
  return (((uintptr_t)v.p | (uintptr_t)(v.row * esize) | (uintptr_t)(heads > 1 ? v.head * esize : 0)) & (uintptr_t)(bytes - 1)) == 0;
}

template <typename TX, typename TQ, typename TC>
cudaError_t rotary_types(RotaryArgs& a, int num_sm, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(TX);
  // a head must be whole units, its rotated part whole units (halves) or pieces (pairs)
  bool vec = a.d_head % (2 * E) == 0 && (!a.freq || a.rot % (a.halves ? 2 * E : E) == 0);
  for (int i = 0; i < 3 && vec; ++i) {
    if (!a.heads[i]) continue;
    vec = vec && aligned(a.x[i], a.heads[i], 16, (int)sizeof(TX));
    if (i == 0) vec = vec && aligned(a.y[0], a.heads[0], E * (int)sizeof(TQ), (int)sizeof(TQ));   // (the cache is always aligned)
  }
  if (a.halves) return vec ? rotary_go<TX, TQ, TC, E, true>(a, num_sm, st) : rotary_go<TX, TQ, TC, 1, true>(a, num_sm, st);
  return vec ? rotary_go<TX, TQ, TC, E, false>(a, num_sm, st) : rotary_go<TX, TQ, TC, 1, false>(a, num_sm, st);
}

}  // namespace

cudaError_t rotary_launch(RotaryArgs a, int x_bf16, int yq_bf16, int cache_bf16, int num_sm, cudaStream_t st) {
  if (x_bf16) return rotary_types<__nv_bfloat16, __nv_bfloat16, __nv_bfloat16>(a, num_sm, st);
  if (yq_bf16) return cache_bf16 ? rotary_types<float, __nv_bfloat16, __nv_bfloat16>(a, num_sm, st) : rotary_types<float, __nv_bfloat16, float>(a, num_sm, st);
  return cache_bf16 ? rotary_types<float, float, __nv_bfloat16>(a, num_sm, st) : rotary_types<float, float, float>(a, num_sm, st);
}

// ------------------------------------------------------------------------------------------------------------------
// C entry points
// ------------------------------------------------------------------------------------------------------------------
namespace {

int no(int code, const char* msg) {
  sps_set_global_error(msg);
  return code;
}
int sms() {
  static std::atomic<int> cached[SPS_MAX_DEVICES];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= SPS_MAX_DEVICES) return SPS_NUM_SM_FALLBACK;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = SPS_NUM_SM_FALLBACK;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}
RowsView view(const sps_rows* r) { return RowsView{r->p, (long long)r->row_stride, (long long)r->head_stride}; }

const char* bad_rows(const sps_rows* r, int rows) {
  if (!r) return "null rows";
  if (r->dtype != 0 && r->dtype != 1) return "rows: dtype must be 0 (fp32) or 1 (bf16)";
  if (r->heads < 1 || r->heads > 4096) return "rows: heads out of range";
  if (r->row_stride < 0 || r->head_stride < 0) return "rows: negative stride";
  if (rows > 0 && !r->p) return "rows: null pointer";
  if ((uintptr_t)r->p & (r->dtype == 0 ? 3 : 1)) return "rows: pointer not aligned to its elements";
  return nullptr;
}
const char* bad_plan(const sps_rotary_plan* p, int d_head) {
  if (!p) return "null rotary plan";
  if (!p->freq || ((uintptr_t)p->freq & 7)) return "rotary plan: freq null or not 8-byte aligned";
  if (p->rot_dim < 2 || (p->rot_dim & 1) || p->rot_dim > d_head) return "rotary plan: rot_dim must be even, 2 .. d_head";
  if (p->layout != SPS_ROTARY_PAIRS && p->layout != SPS_ROTARY_HALVES) return "rotary plan: unknown layout";
  if (!std::isfinite(p->gain)) return "rotary plan: gain must be finite";
  return nullptr;
}
const char* bad_cache(const sps_paged_cache* c) {
  if (!c) return "null cache";
  if (c->dtype != 0 && c->dtype != 1) return "cache: dtype must be 0 (fp32) or 1 (bf16)";
  if (c->d_head != 64 && c->d_head != 128) return "cache: d_head must be 64 or 128";
  if (c->page_size < 8 || c->page_size > 512 || (c->page_size & (c->page_size - 1))) return "cache: page_size must be a power of two, 8 .. 512";
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 4096) return "cache: n_pages or n_kv_heads out of range";
  if (!c->k || !c->v) return "cache: null pointer";
  const int64_t m = c->dtype == 0 ? 4 : 8;
  if ((((uintptr_t)c->k | (uintptr_t)c->v) & 15) || c->page_stride % m || c->head_stride % m || c->pos_stride % m)
    return "cache: k, v must be 16-byte aligned and strides multiples of 16 bytes";
  if (c->pos_stride < c->d_head || c->page_stride < c->d_head || c->head_stride < (c->n_kv_heads > 1 ? c->d_head : 0)) return "cache: strides smaller than d_head";
  return nullptr;
}
const char* bad_batch(const sps_paged_batch* b) {
  if (!b) return "null batch";
  if (b->B < 0 || b->B > 1 << 27 || b->pages_ld < 0 || b->max_q < 1) return "batch: B, pages_ld or max_q out of range";
  if (b->B > 0 && (!b->q_start || !b->kv_len || (!b->pages && b->pages_ld > 0))) return "batch: null pointer";
  if (((uintptr_t)b->q_start | (uintptr_t)b->kv_len | (uintptr_t)b->pages | (uintptr_t)b->status) & 3) return "batch: pointers must be 4-byte aligned";
  return nullptr;
}
PagedSeqs seqs(const sps_paged_cache* c, const sps_paged_batch* b, int rows) {
  PagedSeqs s{};
  s.q_start = b->q_start; s.kv_len = b->kv_len; s.pages = b->pages; s.status = b->status;
  s.B = b->B; s.pages_ld = b->pages_ld; s.rows = rows; s.n_pages = c->n_pages; s.page_size = c->page_size;
  while ((1 << s.page_shift) < c->page_size) ++s.page_shift;
  return s;
}

}  // namespace

extern "C" {

int sps_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, int32_t trained_len, double low_turns,
                           double high_turns, double* out) {
  if (!out) return no(SPS_EINVAL, "null argument");
  if (rot_dim < 2 || (rot_dim & 1) || rot_dim > 1024) return no(SPS_EINVAL, "rot_dim must be even, 2 .. 1024");
  if (!(base > 1.0) || !std::isfinite(base)) return no(SPS_EINVAL, "base must be above 1");
  if (scaling < SPS_ROTARY_PLAIN || scaling > SPS_ROTARY_BANDS) return no(SPS_EINVAL, "unknown scaling");
  if (scaling != SPS_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return no(SPS_EINVAL, "factor must be at least 1");
  if (scaling == SPS_ROTARY_BANDS && (trained_len < 1 || !(low_turns >= 0.0) || !(high_turns > low_turns) || !std::isfinite(high_turns)))
    return no(SPS_EINVAL, "bands need trained_len >= 1 and 0 <= low_turns < high_turns");
  if (scaling == SPS_ROTARY_BASE && rot_dim > 2) base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == SPS_ROTARY_LINEAR) f /= factor;
    if (scaling == SPS_ROTARY_BANDS) {
      const double turns = trained_len * f / 6.283185307179586476925;
      double w = (turns - low_turns) / (high_turns - low_turns);
      w = w < 0.0 ? 0.0 : (w > 1.0 ? 1.0 : w);
      f = w * f + (1.0 - w) * f / factor;
    }
    out[i] = f;
  }
  return SPS_OK;
}

int sps_rotary(const sps_rotary_plan* plan, const sps_rows* x, const sps_rows* y, int32_t rows, int32_t d_head, const int32_t* positions,
               int32_t transposed, void* stream) {
  if (rows < 0) return no(SPS_EINVAL, "rows must be >= 0");
  if (d_head < 2 || (d_head & 1) || d_head > 1024) return no(SPS_EINVAL, "d_head must be even, 2 .. 1024");
  const char* why = bad_plan(plan, d_head);
  if (!why) why = bad_rows(x, rows);
  if (!why) why = bad_rows(y, rows);
  if (why) return no(SPS_EINVAL, why);
  if (x->dtype != y->dtype || x->heads != y->heads) return no(SPS_EINVAL, "x and y must have the same dtype and heads");
  if (x->p == y->p && (x->row_stride != y->row_stride || x->head_stride != y->head_stride)) return no(SPS_EINVAL, "in place, x and y must have the same strides");
  if (rows == 0) return SPS_OK;
  if (!positions || ((uintptr_t)positions & 3)) return no(SPS_EINVAL, "positions null or not 4-byte aligned");
  RotaryArgs a{};
  a.x[0] = view(x); a.y[0] = view(y); a.heads[0] = x->heads;
  a.d_head = d_head; a.rot = plan->rot_dim; a.halves = plan->layout == SPS_ROTARY_HALVES; a.transposed = transposed != 0;
  a.gain = plan->gain; a.freq = plan->freq; a.positions = positions; a.rows = rows;
  const cudaError_t e = rotary_launch(a, x->dtype, x->dtype, 1, sms(), (cudaStream_t)stream);
  return e == cudaSuccess ? SPS_OK : no(SPS_ECUDA, cudaGetErrorString(e));
}

int sps_paged_append(const sps_paged_cache* cache, const sps_paged_batch* batch, const sps_rotary_plan* plan, int32_t rows,
                     const sps_rows* k, const sps_rows* v, const sps_rows* q, const sps_rows* q_out, void* stream) {
  if (rows < 0) return no(SPS_EINVAL, "rows must be >= 0");
  const char* why = bad_cache(cache);
  if (!why) why = bad_batch(batch);
  if (!why && plan) why = bad_plan(plan, cache->d_head);
  if (!why) why = bad_rows(k, rows);
  if (!why) why = bad_rows(v, rows);
  if (!why && q) why = bad_rows(q, rows);
  if (!why && q) why = bad_rows(q_out, rows);
  if (why) return no(SPS_EINVAL, why);
  if (!q && q_out) return no(SPS_EINVAL, "q_out without q");
  if (q && !plan) return no(SPS_EINVAL, "q needs a rotary plan");
  if (k->heads != cache->n_kv_heads || v->heads != cache->n_kv_heads) return no(SPS_EINVAL, "k and v must have the cache's heads");
  if (k->dtype != v->dtype || (q && q->dtype != k->dtype)) return no(SPS_EINVAL, "q, k and v must share a dtype");
  if (q && q->heads != q_out->heads) return no(SPS_EINVAL, "q and q_out must have the same heads");
  if (k->dtype == 1 && cache->dtype == 0) return no(SPS_EINVAL, "an fp32 cache takes fp32 rows");
  if (q && q->dtype == 1 && q_out->dtype == 0) return no(SPS_EINVAL, "bf16 queries go to a bf16 q_out");
  if (q && q->p == q_out->p && (q->dtype != q_out->dtype || q->row_stride != q_out->row_stride || q->head_stride != q_out->head_stride))
    return no(SPS_EINVAL, "in place, q and q_out must have the same dtype and strides");
  if (rows == 0 || batch->B == 0) return SPS_OK;
  RotaryArgs a{};
  a.x[1] = view(k); a.x[2] = view(v);
  a.heads[1] = a.heads[2] = cache->n_kv_heads;
  if (q) { a.x[0] = view(q); a.y[0] = view(q_out); a.heads[0] = q->heads; }
  a.y[1] = RowsView{cache->k, cache->page_stride, cache->head_stride};
  a.y[2] = RowsView{cache->v, cache->page_stride, cache->head_stride};
  a.pos_stride = cache->pos_stride;
  a.d_head = cache->d_head;
  if (plan) { a.rot = plan->rot_dim; a.halves = plan->layout == SPS_ROTARY_HALVES; a.gain = plan->gain; a.freq = plan->freq; }
  a.s = seqs(cache, batch, rows);
  a.rows = rows;
  const cudaError_t e = rotary_launch(a, k->dtype, q ? q_out->dtype : k->dtype, cache->dtype, sms(), (cudaStream_t)stream);
  return e == cudaSuccess ? SPS_OK : no(SPS_ECUDA, cudaGetErrorString(e));
}

static const char* bad_heads(const sps_paged_cache* c, int n_heads, int q_dtype) {
  if (n_heads < 1 || n_heads > 4096 || n_heads % c->n_kv_heads) return "heads of q must be a multiple of the cache's";
  if (q_dtype != 0 && q_dtype != 1) return "q: dtype must be 0 (fp32) or 1 (bf16)";
  if (q_dtype == 1 && c->dtype == 0) return "an fp32 cache takes fp32 queries";
  return nullptr;
}

// workspace: arrival counters of up to 1024 CTAs, a line for the word that a call leaves which gave up, records of up to 1024
// CTAs, then two part slots for each CTA
#define PAGED_COUNTER_BYTES (4096 + 128)
#define PAGED_RECORD_BYTES (1024 * sizeof(PartRecord))

int64_t sps_paged_attention_workspace_bytes(const sps_paged_cache* cache, int32_t n_heads, int32_t q_dtype) {
  const char* why = bad_cache(cache);
  if (!why) why = bad_heads(cache, n_heads, q_dtype);
  if (why) { no(SPS_EINVAL, why); return -1; }
  return (int64_t)(PAGED_COUNTER_BYTES + PAGED_RECORD_BYTES) + (int64_t)2 * paged_attn_grid(sms()) * (int64_t)paged_attn_slot_bytes(cache->dtype, q_dtype, cache->d_head);
}

int sps_paged_attention(const sps_paged_cache* cache, const sps_paged_batch* batch, int32_t rows, const sps_rows* q, const sps_rows* out,
                        float scale, float* lse, void* workspace, void* stream) {
  if (rows < 0) return no(SPS_EINVAL, "rows must be >= 0");
  const char* why = bad_cache(cache);
  if (!why) why = bad_batch(batch);
  if (!why) why = bad_rows(q, rows);
  if (!why) why = bad_rows(out, rows);
  if (!why) why = bad_heads(cache, q->heads, q->dtype);
  if (why) return no(SPS_EINVAL, why);
  if (out->heads != q->heads) return no(SPS_EINVAL, "q and out must have the same heads");
  if (out->p == q->p && rows > 0 && (out->dtype != q->dtype || out->row_stride != q->row_stride || out->head_stride != q->head_stride))
    return no(SPS_EINVAL, "in place, q and out must have the same dtype and strides");
  if (q->dtype == 0 && out->dtype == 1) return no(SPS_EINVAL, "out has q's dtype or is fp32");
  if ((int64_t)rows * q->heads > 0x7fff0000) return no(SPS_EINVAL, "rows x heads must stay below 2^31");
  if (!std::isfinite(scale * 1.4426950408889634f)) return no(SPS_EINVAL, "scale must be finite, in base 2 too");
  if (!workspace || ((uintptr_t)workspace & 15)) return no(SPS_EINVAL, "workspace null or not 16-byte aligned");
  if ((uintptr_t)lse & 3) return no(SPS_EINVAL, "lse not 4-byte aligned");
  if (rows == 0 || batch->B == 0) return SPS_OK;
  PagedAttnArgs a{};
  a.s = seqs(cache, batch, rows);
  a.q = view(q); a.out = view(out);
  a.q_bf16 = q->dtype; a.out_bf16 = out->dtype;
  a.q_vec = aligned(a.q, q->heads, 16, q->dtype ? 2 : 4);
  a.out_vec = aligned(a.out, out->heads, 16, out->dtype ? 2 : 4);
  a.k = cache->k; a.v = cache->v;
  a.page_stride = cache->page_stride; a.head_stride = cache->head_stride; a.pos_stride = cache->pos_stride;
  a.H = q->heads; a.Hkv = cache->n_kv_heads; a.G = a.H / a.Hkv;
  a.g_magic = a.G > 1 ? ~0ull / (unsigned long long)a.G + 1 : 0;   // ceil(2^64 / G), powers of two included
  a.scale_log2 = (scale == 0.f ? 1.f / std::sqrt((float)cache->d_head) : scale) * 1.4426950408889634f;
  a.lse = lse;
  a.counters = (int*)workspace;
  a.gave_up = a.counters + 1024;
  a.records = (PartRecord*)((char*)workspace + PAGED_COUNTER_BYTES);
  a.slots = (float*)((char*)workspace + PAGED_COUNTER_BYTES + PAGED_RECORD_BYTES);
  a.wait_ns = sps_wait_knobs().limit_ns;
  a.drop_stage = sps_wait_knobs().drop_stage;
  const unsigned grid = (unsigned)paged_attn_grid(sms());
  a.grid_magic = grid > 1 ? (uint32_t)(((1ull << 32) + grid - 1) / grid) : 0;   // one CTA: never used
  a.grid_magic_to = grid > 1 ? (int)((1ull << 31) / grid) : 0;
  const cudaError_t e = paged_attn_launch(a, cache->dtype, cache->d_head, batch->max_q, sms(), (cudaStream_t)stream);
  return e == cudaSuccess ? SPS_OK : no(SPS_ECUDA, cudaGetErrorString(e));
}

}  // extern "C"
