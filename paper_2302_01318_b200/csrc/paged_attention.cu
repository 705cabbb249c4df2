// Attention over a paged fp32 cache (see paged.cuh for how the work is cut; a bf16 cache runs on the tensor cores,
// paged_attention_tc.cu).
//
//   s_j = scale q . k_j,  m = max s_j,  l = sum 2^(s_j - m),  o = sum 2^(s_j - m) v_j / l     (scores in base 2)
//
// One pass over keys and values with the running maximum and sum; everything in fp32.  A CTA of 256 threads takes 16 query
// rows against tiles of 64 tokens, fetched into registers a tile ahead and staged in shared memory: scores by (token, four rows) per thread, the softmax
// by a warp per two rows, outputs by (two elements, a few rows) per thread in registers.
#include <type_traits>

#include "paged.cuh"

namespace {

constexpr int SIMT_NR = 16, SIMT_KT = 64, SIMT_THREADS = 256;

template <int D>
__global__ void __launch_bounds__(SIMT_THREADS) paged_attn_simt_kernel(const __grid_constant__ PagedAttnArgs a) {
  constexpr int NR = SIMT_NR, KT = SIMT_KT, LDK = D + 4;
  constexpr int RPT = NR / (SIMT_THREADS / (D / 2));   // rows a thread accumulates (4 or 2)
  constexpr int LOADS = KT * (D / 4) / SIMT_THREADS;   // four-element pieces of a tile's keys (and values) per thread
  extern __shared__ __align__(16) float simt_smem[];
  float* Ks = simt_smem;             // [KT][D + 4]
  float* Vs = Ks + KT * LDK;         // [KT][D]
  float* Qs = Vs + KT * D;           // [NR][D], scaled
  float* Ps = Qs + NR * D;           // [NR][KT]
  __shared__ float s_m[NR], s_l[NR], s_alpha[NR];
  __shared__ int s_lim[NR];
  __shared__ WorkCursor s_cur;
  __shared__ SeqGeom s_geo[GEO];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  pdl_wait();
  const WorkCursor c0 = cursor_begin<NR, KT>(a, s_geo, reinterpret_cast<long long*>(Ps));
  if (tid == 0) s_cur = c0;
  __syncthreads();
  WorkCursor c = s_cur;
  if (c.spoilt) {
    if (tid == 0) paged_flag(a.s.status, SPS_PAGED_TIMEOUT);
    nan_rows<D>(a, blockIdx.x, gridDim.x);
    return;
  }
  const int dp = tid % (D / 2), rg = tid / (D / 2);
  while (c.valid) {
    const int R = c.nq * a.G, r0 = c.t * NR;
    // keys and values of a tile into registers: this thread's four elements of LOADS tokens; zeros where there is no token or page
    float4 kr[LOADS], vr[LOADS];
    auto fetch = [&](int kt) {
      long long at[LOADS];
#pragma unroll
      for (int x = 0; x < LOADS; ++x) {
        const int i = tid + x * SIMT_THREADS, j = i / (D / 4), e = (i - j * (D / 4)) * 4, pos = kt * KT + j;
        at[x] = -1;
        if (pos < c.len) {
          const int page = a.s.pages[(long long)c.b * a.s.pages_ld + (pos >> a.s.page_shift)];
          if (page >= 0 && page < a.s.n_pages) at[x] = page * a.page_stride + c.hk * a.head_stride + (pos & (a.s.page_size - 1)) * a.pos_stride + e;
          else paged_flag(a.s.status, SPS_PAGED_BAD_PAGE);
        }
      }
#pragma unroll
      for (int x = 0; x < LOADS; ++x) {
        kr[x] = vr[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at[x] >= 0) {
          kr[x] = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.k) + at[x]);
          vr[x] = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.v) + at[x]);
        }
      }
    };
    fetch(c.k0);
    __syncthreads();   // the previous part's rows have been read
    for (int i = tid; i < NR * D; i += SIMT_THREADS) {
      const int r = i / D, e = i - r * D, rr = r0 + r;
      float v = 0.f;
      if (rr < R) {
        const int tok = row_token(a, rr);
        const long long at = (long long)(c.row0 + tok) * a.q.row + (long long)(c.hk * a.G + rr - tok * a.G) * a.q.head + e;
        v = reinterpret_cast<const float*>(a.q.p)[at];
      }
      Qs[i] = v * a.scale_log2;
    }
    if (tid < NR) {
      s_lim[tid] = r0 + tid < R ? c.len - c.nq + row_token(a, r0 + tid) : -1;
      s_m[tid] = -INFINITY;
      s_l[tid] = 0.f;
    }
    float o[RPT][2];
#pragma unroll
    for (int i = 0; i < RPT; ++i) o[i][0] = o[i][1] = 0.f;
    const int first_lim = c.len - c.nq + row_token(a, r0);
    for (int kt = c.k0; kt < c.k1; ++kt) {
      const int p0 = kt * KT;
      __syncthreads();
#pragma unroll
      for (int x = 0; x < LOADS; ++x) {
        const int i = tid + x * SIMT_THREADS, j = i / (D / 4), e = (i - j * (D / 4)) * 4;
        *reinterpret_cast<float4*>(Ks + j * LDK + e) = kr[x];
        *reinterpret_cast<float4*>(Vs + j * D + e) = vr[x];
      }
      __syncthreads();
      if (kt + 1 < c.k1) fetch(kt + 1);   // under way while this tile is worked on
      {
        const int j = tid & 63, g = tid >> 6;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int e = 0; e < D; e += 4) {
          const float4 k = *reinterpret_cast<const float4*>(Ks + j * LDK + e);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 q = *reinterpret_cast<const float4*>(Qs + (g * 4 + i) * D + e);
            s[i] += q.x * k.x; s[i] += q.y * k.y; s[i] += q.z * k.z; s[i] += q.w * k.w;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) Ps[(g * 4 + i) * KT + j] = p0 + j <= s_lim[g * 4 + i] ? s[i] : -INFINITY;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = warp * 2 + i;
        const float x = Ps[r * KT + lane], y = Ps[r * KT + lane + 32];
        const float m_old = s_m[r], m = fmaxf(m_old, warp_max(fmaxf(x, y)));
        const float mm = m == -INFINITY ? 0.f : m;   // nothing seen yet: every weight is 2^-inf = 0
        const float ex = exp2f(x - mm), ey = exp2f(y - mm), sum = warp_sum(ex + ey);
        Ps[r * KT + lane] = ex;
        Ps[r * KT + lane + 32] = ey;
        __syncwarp();
        if (lane == 0) {
          const float al = exp2f(m_old - mm);
          s_alpha[r] = al;
          s_l[r] = s_l[r] * al + sum;
          s_m[r] = m;
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < RPT; ++i) { const float al = s_alpha[rg * RPT + i]; o[i][0] *= al; o[i][1] *= al; }
      const bool edge = p0 + KT - 1 > first_lim;   // some row does not see all of this tile
      auto accumulate = [&](auto masked) {
#pragma unroll 4
        for (int j = 0; j < KT; j += 4) {
          float2 v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const float2*>(Vs + (j + q) * D + 2 * dp);
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const float4 p = *reinterpret_cast<const float4*>(Ps + (rg * RPT + i) * KT + j);
            const float w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (decltype(masked)::value && w[q] == 0.f) continue;   // what a row does not see stays out, NaN or not
              o[i][0] += w[q] * v[q].x;
              o[i][1] += w[q] * v[q].y;
            }
          }
        }
      };
      if (edge) accumulate(std::true_type{});
      else accumulate(std::false_type{});
    }
    __syncthreads();
    int first, parts;
    item_ctas(c, first, parts);
    if (parts == 1) {
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const int r = rg * RPT + i, rr = r0 + r;
        if (rr >= R) continue;
        const float l = s_l[r], inv = l == 0.f ? 0.f : 1.f / l;
        const int tok = row_token(a, rr);
        const long long at = (long long)(c.row0 + tok) * a.out.row + (long long)(c.hk * a.G + rr - tok * a.G) * a.out.head + 2 * dp;
        store_out(a, at, o[i][0] * inv);
        store_out(a, at + 1, o[i][1] * inv);
      }
      if (a.lse && tid < NR && r0 + tid < R) {
        const int rr = r0 + tid, tok = row_token(a, rr);
        a.lse[(size_t)(c.row0 + tok) * a.H + c.hk * a.G + rr - tok * a.G] = s_l[tid] == 0.f ? -INFINITY : 0.6931471805599453f * (s_m[tid] + log2f(s_l[tid]));
      }
    } else {
      float* slot = a.slots + slot_floats<NR, D>() * (size_t)part_slot(blockIdx.x, c.k0 == 0);
      if (tid < NR) { __stcg(slot + tid, s_m[tid]); __stcg(slot + NR + tid, s_l[tid]); }
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const int r = rg * RPT + i;
        if (r0 + r < R) __stcg(reinterpret_cast<float2*>(slot + 2 * NR + r * D + 2 * dp), make_float2(o[i][0], o[i][1]));
      }
      __syncthreads();
      if (tid == 0) {
        s_last = part_arrive(a.counters + first, parts);
      }
      __syncthreads();
      if (s_last) join_parts<NR, D, SIMT_THREADS>(a, c, first, parts, tid, s_alpha, s_m, Ps, NR * KT);
    }
    cursor_next<NR, KT>(a, c, s_geo);
  }
}

template <int D>
cudaError_t simt_go(PagedAttnArgs a, int num_sm, cudaStream_t st) {
  static DevSmemCache cached{};
  a.lead = 1;
  a.min_run = 1;
  constexpr size_t smem = sizeof(float) * (SIMT_KT * (D + 4) + SIMT_KT * D + SIMT_NR * D + SIMT_NR * SIMT_KT);
  const cudaError_t e = sps_ensure_smem(paged_attn_simt_kernel<D>, smem, cached);
  if (e != cudaSuccess) return e;
  return launch_k(paged_attn_simt_kernel<D>, dim3(paged_attn_grid(num_sm)), dim3(SIMT_THREADS), smem, st, a);
}

}  // namespace

size_t paged_attn_slot_bytes(int dtype, int q_dtype, int d_head) {
  if (dtype == 1) return q_dtype == 1 ? paged_attn_wide_slot_bytes(d_head) : paged_attn_tc_slot_bytes(d_head);
  return sizeof(float) * (d_head == 128 ? slot_floats<SIMT_NR, 128>() : slot_floats<SIMT_NR, 64>());
}

cudaError_t paged_attn_launch(const PagedAttnArgs& a, int cache_bf16, int d_head, int max_q, int num_sm, cudaStream_t st) {
  if (cache_bf16) return paged_attn_tc_launch(a, d_head, max_q, num_sm, st);
  return d_head == 128 ? simt_go<128>(a, num_sm, st) : simt_go<64>(a, num_sm, st);
}
