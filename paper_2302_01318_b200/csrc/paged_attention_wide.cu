// Attention over a paged bf16 cache on the 5th-generation tensor cores, for many bf16 query rows per key head (prompt chunks).
//
// Here the query rows are the tensor cores' 128-row operand, two tiles of them (256 rows) per CTA against the same keys and
// values:
//
//   S_w [128 rows x 128 tokens] = Q_w K^T       (Q resident in shared memory, K from the page copies; both K-major)
//   O_w [128 rows x d]         += P_w V         (P from tensor memory, V from the page copies, MN-major)
//
// A thread of the softmax owns a row: its 128 scores come from tensor memory into registers, its maximum and sum need no
// other thread, and its weights go back over the scores as bf16, where the second product reads them.
//
// Running maximum.  m is fixed at the maximum of the part's first tile and raised only when a score exceeds it by MAX_UP (in
// base 2): bf16 weights and fp32 sums keep their relative precision at any size, so this loses nothing, and O stays
// untouched in tensor memory from tile to tile.  A warp whose rows do outgrow m rescales their O itself, and takes the tile's
// raw scores from tensor memory once more: their differences to an m far below them were rounded at its size.  Until a row
// has a finite score m is the least finite number, which any such score outgrows.
//
// What bounds it: the tensor cores, 4 x 8 products of 64 clocks per pair of tiles (d = 128); they work on one tile while
// the other one's softmax runs.
//
//   warp 0       copies of keys and values (paged_tc.cuh)
//   warp 1       products, an elected lane issuing: O_0 and the next S_0, then O_1 and the next S_1
//   warps 4-7    Q of the part to come: its loads under way while the last scores of this part are multiplied
//   warps 8-15   softmax of tile 0 (8-11) and tile 1 (12-15), and their outputs
//
// Parts of an item are 256 rows x d floats each: they are joined by a kernel of its own (paged_join_kernel) that spreads every
// item's rows over several CTAs; one CTA joining all of them took 60 us for 18 parts of 64 rows.
//
// Waits are bounded and end as in paged_attention_tc.cu; the join then makes the rows that it writes NaN.
#include "paged_tc.cuh"

namespace {

constexpr float MAX_UP = 24.f;       // log2 of the largest weight that is let stand
constexpr float LEAST = -3.402823466e38f;   // the reference of a row that has seen no finite score yet
constexpr int W_ROWS = 256;          // rows of an item: two tiles
constexpr int W_THREADS = 512;

template <int D> struct WCfg {
  static constexpr uint32_t HALF = TILE * D * 2;
  static constexpr uint32_t Q_BYTES = W_ROWS * D * 2;
  static constexpr int STAGES = D == 128 ? 4 : 8;
  static constexpr uint32_t Q_AT = STAGES * HALF, HDR_AT = Q_AT + Q_BYTES;
  static constexpr uint32_t HDR = 1024 + W_ROWS * 8;
  static constexpr size_t SMEM = HDR_AT + HDR;
  // kind::f16 instruction descriptors: fp32 accumulator, bf16 x bf16, M = 128; S: both K-major, N = 128; O: B MN-major, N = d
  static constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TILE >> 3) << 17) | (8u << 24);
  static constexpr uint32_t IDESC_O = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | (8u << 24);
};

__device__ __forceinline__ void w_mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n mov.b64 b, {%2, %3};\n setp.ne.b32 p, %5, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n}\n" ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate ? 1u : 0u)
      : "memory");
}
__device__ __forceinline__ float w_max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <int D>
__global__ void __launch_bounds__(W_THREADS, 1) paged_attn_wide_kernel(const __grid_constant__ TcArgs ta) {
  using C = WCfg<D>;
  constexpr int STAGES = C::STAGES, NR = W_ROWS;
  extern __shared__ __align__(1024) unsigned char wmem[];   // the ring, Q (swizzled operands: 1024-byte aligned), header
  const PagedAttnArgs& a = ta.a;
  const uint32_t ring = p_smem(wmem), q_s = ring + C::Q_AT, hb = ring + C::HDR_AT;
  unsigned char* hdr = wmem + C::HDR_AT;
  const uint32_t full = hb, empty = hb + 64, s_full = hb + 128, p_full = hb + 144, pv_done = hb + 160, q_ready = hb + 176, q_free = hb + 184, drain = hb + 192, p_half = hb + 480;
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(hdr + 200);
  volatile int* s_abort = reinterpret_cast<volatile int*>(hdr + 204);
  int* s_poison = reinterpret_cast<int*>(hdr + 208);
  WorkCursor* s_cur = reinterpret_cast<WorkCursor*>(hdr + 216);
  SeqGeom* geo = reinterpret_cast<SeqGeom*>(hdr + 512);                 // [GEO]
  long long* s_qat = reinterpret_cast<long long*>(hdr + 1024);          // [256] where a row of Q is
  static_assert(sizeof(WorkCursor) <= 264 && sizeof(SeqGeom) * GEO <= 512, "header");
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { p_bar_init(full + 8 * i, 1); p_bar_init(empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { p_bar_init(s_full + 8 * i, 1); p_bar_init(p_full + 8 * i, 128); p_bar_init(p_half + 8 * i, 128); p_bar_init(pv_done + 8 * i, 1); }
    p_bar_init(q_ready, 128); p_bar_init(q_free, 1); p_bar_init(drain, 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&ta.tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&ta.tm_v) : "memory");
  }
  if (warp == 1) {   // S_0, S_1 and O_0, O_1: all 512 columns
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(hb + 200) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    pdl_launch_dependents();   // with the tensor memory in hand: a dependent on this SM that took it first would wait for this CTA
  }
  pdl_wait();
  const WorkCursor c0 = cursor_begin<NR, TILE>(a, geo, s_qat);
  if (tid == 0) {
    *s_cur = c0;
    if (c0.spoilt) { s_cur->valid = false; *s_abort = 2; paged_flag(a.s.status, SPS_PAGED_TIMEOUT); }
  }
  P_FENCE_BEFORE();
  __syncthreads();
  P_FENCE_AFTER();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *s_tmem, 0);
  WorkCursor c = *s_cur;

  // Registers: 512 threads were launched with 128 each; the softmax's 256 take 200, the others give them.  (Asked for
  // warpgroup by warpgroup, at the head of its branch: the compiler allots registers along the control flow.)
#define W_GIVE() asm volatile("setmaxnreg.dec.sync.aligned.u32 56;")
#define W_TAKE() asm volatile("setmaxnreg.inc.sync.aligned.u32 200;")
  if (warp < 4) {
    W_GIVE();
    if (warp == 0) {
      copy_pages<D, NR, STAGES>(ta, c, geo, ring, full, empty, s_abort);
    } else if (warp == 1) {
      // ---------------------------------------------------------------------------------------------------- products
      const bool leader = p_elect();
      bool ok = true;
      int it = 0, qn = 0;                  // half-tiles of the parts before, parts
      uint32_t pn[2] = {0, 0};             // weights taken, by tile
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok) ok = __all_sync(0xffffffffu, p_wait(bar, parity & 1u, a, s_abort));
      };
      auto score = [&](int w, int e, bool frees_k, bool frees_q) {   // S_w of the tile whose keys are half-tile e
        wait(full + 8 * (e % STAGES), (uint32_t)(e / STAGES));
        if (!ok) return;
        P_FENCE_AFTER();
        if (leader) {
          const uint32_t qa = p_desc_lo(q_s + w * (C::Q_BYTES / 2), 16), ka = p_desc_lo(ring + (uint32_t)(e % STAGES) * C::HALF, 16);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            p_mma(tmem + w * 128, qa + (k >> 2) * (128 * 128 >> 4) + (k & 3) * 2, p_desc_hi(1024, 2), ka + (k >> 2) * (TILE * 128 >> 4) + (k & 3) * 2, p_desc_hi(1024, 2),
                  C::IDESC_S, k > 0);
          if (frees_k) p_commit(empty + 8 * (e % STAGES));
          if (frees_q) p_commit(q_free);
          p_commit(s_full + 8 * w);
        }
        __syncwarp();
      };
      auto output = [&](int w, int e, bool first, bool frees_v) {    // O_w += P_w V
        wait(full + 8 * (e % STAGES), (uint32_t)(e / STAGES));
        const uint32_t va = p_desc_lo(ring + (uint32_t)(e % STAGES) * C::HALF, TILE * 128);
        wait(p_half + 8 * w, pn[w]);
        if (!ok) return;
        P_FENCE_AFTER();
        if (leader) {
#pragma unroll
          for (int k = 0; k < TILE / 32; ++k)
            w_mma_ts(tmem + 256 + w * 128, tmem + w * 128 + k * 8, va + k * (16 * 128 >> 4), p_desc_hi(1024, 2), C::IDESC_O, k > 0 || !first);
        }
        __syncwarp();
        wait(p_full + 8 * w, pn[w]);
        ++pn[w];
        if (!ok) return;
        P_FENCE_AFTER();
        if (leader) {
#pragma unroll
          for (int k = TILE / 32; k < TILE / 16; ++k)
            w_mma_ts(tmem + 256 + w * 128, tmem + w * 128 + k * 8, va + k * (16 * 128 >> 4), p_desc_hi(1024, 2), C::IDESC_O, k > 0 || !first);
          if (frees_v) p_commit(empty + 8 * (e % STAGES));
          p_commit(pv_done + 8 * w);
        }
        __syncwarp();
      };
      while (c.valid && ok) {
        const int n = c.k1 - c.k0;
        const bool two = c.nq * a.G - c.t * NR > 128;
        wait(q_ready, (uint32_t)qn);
        ++qn;
        score(0, it, !two, !two && n == 1);
        if (two) score(1, it, true, n == 1);
        for (int i = 0; i < n && ok; ++i) {
          const int e = it + 2 * i;
          output(0, e + 1, i == 0, !two);
          if (i + 1 < n) score(0, e + 2, !two, !two && i + 2 == n);
          if (two) {
            output(1, e + 1, i == 0, true);
            if (i + 1 < n) score(1, e + 2, true, i + 2 == n);
          }
        }
        it += 2 * n;
        cursor_next<NR, TILE>(a, c, geo);
      }
      // Every product issued must be done before the ring and the tensor memory go away.  After a part that was worked to its
      // end they are; but softmax warps that gave up go on to the end without waiting for them, and this warp need not notice.
      if (!ok) *s_abort = 1;
      if (leader) p_commit(drain);
      __syncwarp();
      p_drain(drain, 0u);
    }
  } else if (warp < 8) {
    W_GIVE();
    // ---------------------------------------------------------------------------------------------------- Q
    const int qt = tid - 128;
    bool ok = true;
    for (int qn = 0; c.valid && ok; ++qn) {
      const int live = c.nq * a.G - c.t * NR;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = qt + k * 128, rr = c.t * NR + r, tok = row_token(a, rr);
        s_qat[r] = (long long)(c.row0 + tok) * a.q.row + (long long)(c.hk * a.G + rr - tok * a.G) * a.q.head;
      }
      asm volatile("bar.sync 7, 128;" ::: "memory");
      // K-major: row r of tile w, 64-element block ch at ((w D / 64 + ch) * 128 + r) * 128, its 16-byte chunk k at chunk k ^ (r & 7)
      auto place = [&](int r, int k8) { return C::Q_AT + (((r >> 7) * (D / 64) + (k8 >> 3)) * 128 + (r & 127)) * 128 + (((k8 & 7) ^ (r & 7)) << 4); };
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q.p);
      if (qn > 0) {   // into L2 while the part before still needs the buffer
        for (int r = qt; r < min(live, NR); r += 128)
#pragma unroll
          for (int e = 0; e < D; e += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + s_qat[r] + e));
        ok = p_wait(q_free, (uint32_t)(qn - 1) & 1u, a, s_abort);
      }
      if (ok && a.q_vec) {
        // straight to shared memory, all of a thread's 16-byte chunks in flight; rows that do not exist become zeros
#pragma unroll 4
        for (int i = qt; i < NR * (D / 8); i += 128) {
          const int r = i / (D / 8), k8 = i - r * (D / 8);
          const __nv_bfloat16* src = r < live ? q + s_qat[r] + k8 * 8 : q;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ring + place(r, k8)), "l"(src), "r"(r < live ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
      } else if (ok) {
        for (int i = qt; i < NR * (D / 8); i += 128) {
          const int r = i / (D / 8), k8 = i - r * (D / 8);
          uint4 f = make_uint4(0u, 0u, 0u, 0u);
          if (r < live) {
            const unsigned short* u = reinterpret_cast<const unsigned short*>(q + s_qat[r] + k8 * 8);
            f = make_uint4(u[0] | (uint32_t)u[1] << 16, u[2] | (uint32_t)u[3] << 16, u[4] | (uint32_t)u[5] << 16, u[6] | (uint32_t)u[7] << 16);
          }
          *reinterpret_cast<uint4*>(wmem + place(r, k8)) = f;
        }
      }
      uint32_t all;   // (and s_qat may be written again)
      asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, 7, 128, q;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(all) : "r"(ok ? 1u : 0u) : "memory");
      if (!all) break;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      p_arrive(q_ready);
      cursor_next<NR, TILE>(a, c, geo);
    }
  } else {
    W_TAKE();
    // ---------------------------------------------------------------------------------------------------- softmax
    const int st = tid - 256, w = (warp - 8) >> 2, quarter = warp & 3;
    const int my = quarter * 32 + lane;                        // row of the tile: a lane of tensor memory
    const uint32_t t_s = tmem + w * 128 + ((uint32_t)(quarter * 32) << 16), t_o = t_s + 256;
    // After a wait that ran out the threads keep their common path and skip the waits, until they agree to stop.
    bool ok = true;
    uint32_t sn = 0, on = 0;                                   // scores taken; outputs awaited
    int it = 0;
    if (st == 0) a.records[blockIdx.x].parts = 0;
    while (c.valid) {
      const int R = c.nq * a.G, r = c.t * NR + w * 128 + my, n = c.k1 - c.k0;
      const int tok = row_token(a, r);
      const int lim = r < R ? c.len - c.nq + tok : -1;         // last position this row sees
      const int item_lim = c.len - c.nq + row_token(a, c.t * NR);   // the least of the item's rows'
      const bool work = w == 0 || R - c.t * NR > 128;          // the second tile may be empty
      if (st == 0) *s_poison = 0x7fffffff;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      float m = LEAST, l = 0.f;
      if (work) {
        const int warp_lim = __shfl_sync(0xffffffffu, lim < 0 && r >= R ? 0x7fffffff : lim, 0);   // the least of the warp's live rows' (rows ascend)
        for (int i = 0; i < n; ++i, ++sn) {
          const int p0 = (c.k0 + i) * TILE;
          if (w == 0 && p0 + TILE - 1 > item_lim) {
            // slots behind the sequence hold anything: zero (0 x NaN is NaN in a product).  New tokens some rows do not
            // see: a value that is not finite is taken out and remembered, its rows become NaN at the end.
            const int e = it + 2 * i + 1, pos = p0 + my;
            ok = ok && p_wait(full + 8 * (e % STAGES), (uint32_t)(e / STAGES) & 1u, a, s_abort);
            if (ok && pos > item_lim) {
              unsigned char* vr = wmem + (e % STAGES) * C::HALF + my * 128;
              bool clear = pos >= c.len;
              if (!clear) {
#pragma unroll 1
                for (int q = 0; q < D / 8; ++q) {
                  const uint4 u = *reinterpret_cast<const uint4*>(vr + (q >> 3) * (TILE * 128) + (((q & 7) ^ (my & 7)) << 4));
                  const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                  for (int z = 0; z < 4; ++z) clear = clear || (x[z] & 0x7f80u) == 0x7f80u || (x[z] & 0x7f800000u) == 0x7f800000u;
                }
                if (clear) atomicMin(s_poison, pos);
              }
              if (clear) {
#pragma unroll 1
                for (int q = 0; q < D / 8; ++q) *reinterpret_cast<uint4*>(vr + (q >> 3) * (TILE * 128) + ((q & 7) << 4)) = make_uint4(0, 0, 0, 0);
              }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          ok = ok && p_wait(s_full + 8 * w, sn & 1u, a, s_abort);
          __syncwarp();
          P_FENCE_AFTER();
          float x[128], up;
          bool fresh = i == 0;                                  // x is scale s, from which a new m is taken, not scale s - m
          for (;;) {
            const float ref = fresh ? 0.f : -m;
#pragma unroll
            for (int j = 0; j < 128; j += 32) p_ld32(t_s + j, x + j);
            P_WAIT_LD();
            p_landed<128>(x);
#pragma unroll
            for (int j = 0; j < 128; j += 2) p_fma2(x[j], x[j + 1], a.scale_log2, ref, ref);
            if (p0 + TILE - 1 > warp_lim || r >= R) {
              const int d = lim - p0;                             // last token of the tile this row sees
#pragma unroll
              for (int j = 0; j < 128; ++j) x[j] = j <= d ? x[j] : -INFINITY;
            }
            float u0 = x[0], u1 = x[1], u2 = x[2], u3 = x[3];
#pragma unroll
            for (int j = 4; j < 124; j += 8) {
              u0 = w_max3(u0, x[j], x[j + 1]);
              u1 = w_max3(u1, x[j + 2], x[j + 3]);
              u2 = w_max3(u2, x[j + 4], x[j + 5]);
              u3 = w_max3(u3, x[j + 6], x[j + 7]);
            }
            u0 = w_max3(u0, x[124], x[125]);
            u1 = w_max3(u1, x[126], x[127]);
            up = w_max3(w_max3(u0, u1, u2), u3, u3);
            if (fresh || !__any_sync(0xffffffffu, !(up <= MAX_UP))) break;
            fresh = true;
          }
          if (fresh) {
            const float was = m;
            m = up > m ? up : m;
#pragma unroll
            for (int j = 0; j < 128; j += 2) p_add2(x[j], x[j + 1], -m, -m);
            if (i > 0) {
              // these rows' O takes the factor too; every product so far is in it: S of this tile came after them
              const float f = p_ex2(was - m);
              l *= f;
#pragma unroll 1
              for (int j = 0; j < D; j += 16) {
                float o[16];
                p_ld16(t_o + j, o);
                P_WAIT_LD();
                p_landed<16>(o);
                uint32_t u[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) u[q] = __float_as_uint(o[q] * f);
                p_st16(t_o + j, u);
              }
            }
            if (!(up < INFINITY)) l = __int_as_float(0x7fffffff);   // an infinite or NaN score that the row sees
          }
          float l1 = 0.f, l2 = 0.f, l3 = 0.f;
#pragma unroll
          for (int b = 0; b < 128; b += 32) {
            uint32_t u[16];
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              float &x0 = x[b + j], &x1 = x[b + j + 1];
              x0 = p_ex2(x0);
              x1 = p_ex2(x1);
              if (j & 2) p_add2(l2, l3, x0, x1);
              else p_add2(l, l1, x0, x1);
              u[j >> 1] = p_pack(x0, x1);
            }
            p_st16(t_s + b / 2, u);
            if (b == 32) {
              P_WAIT_ST();
              P_FENCE_BEFORE();
              p_arrive(p_half + 8 * w);
            }
          }
          l += l1 + (l2 + l3);
          P_WAIT_ST();
          P_FENCE_BEFORE();
          p_arrive(p_full + 8 * w);
        }
        on += n;
        ok = ok && p_wait(pv_done + 8 * w, (on - 1) & 1u, a, s_abort);
        __syncwarp();
      }
      it += 2 * n;
      // ---- the part's end
      uint32_t all;
      asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, 1, 256, q;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(all) : "r"(ok ? 1u : 0u) : "memory");
      if (!all) break;
      int first, parts;
      item_ctas(c, first, parts);
      if (work) {
        P_FENCE_AFTER();
        if (lim >= *s_poison) l = __int_as_float(0x7fffffff);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const long long at = (long long)(c.row0 + tok) * a.out.row + (long long)(c.hk * a.G + r - tok * a.G) * a.out.head;
        float* slot = a.slots + slot_floats<NR, D>() * (size_t)part_slot(blockIdx.x, c.k0 == 0);
        const int sr = w * 128 + my;
#pragma unroll 1
        for (int j = 0; j < D; j += 32) {
          float o[32];
          p_ld32(t_o + j, o);
          P_WAIT_LD();
          p_landed<32>(o);
          if (r >= R) continue;
          if (parts > 1) {
#pragma unroll
            for (int q = 0; q < 32; q += 4) __stcg(reinterpret_cast<float4*>(slot + 2 * NR) + ((j + q) >> 2) * NR + sr, make_float4(o[q], o[q + 1], o[q + 2], o[q + 3]));
          } else {
#pragma unroll
            for (int q = 0; q < 32; ++q) o[q] = l == 0.f ? 0.f : o[q] * inv;
            if (a.out_vec && a.out_bf16) {
              uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.out.p) + at + j);
#pragma unroll
              for (int q = 0; q < 32; q += 8) dst[q >> 3] = make_uint4(p_pack(o[q], o[q + 1]), p_pack(o[q + 2], o[q + 3]), p_pack(o[q + 4], o[q + 5]), p_pack(o[q + 6], o[q + 7]));
            } else if (a.out_vec) {
              float4* dst = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out.p) + at + j);
#pragma unroll
              for (int q = 0; q < 32; q += 4) dst[q >> 2] = make_float4(o[q], o[q + 1], o[q + 2], o[q + 3]);
            } else {
#pragma unroll
              for (int q = 0; q < 32; ++q) store_out(a, at + j + q, o[q]);
            }
          }
        }
        P_FENCE_BEFORE();
        if (parts > 1) {
          __stcg(slot + sr, l == 0.f ? -INFINITY : m);
          __stcg(slot + NR + sr, l);
        } else if (a.lse && r < R) {
          a.lse[(size_t)(c.row0 + tok) * a.H + c.hk * a.G + r - tok * a.G] = l == 0.f ? -INFINITY : 0.6931471805599453f * (m + log2f(l));
        }
      }
      if (parts > 1 && c.k0 == 0 && st == 0) a.records[blockIdx.x] = PartRecord{c.row0, c.nq, c.hk, c.t, first, parts};
      asm volatile("bar.sync 1, 256;" ::: "memory");   // s_poison may be written again
      cursor_next<NR, TILE>(a, c, geo);
    }
    if (!ok) *s_abort = 1;
  }
  P_FENCE_BEFORE();
  __syncthreads();
  if (warp == 1) {
    P_FENCE_AFTER();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
  if (const int gave_up = *s_abort) nan_rows<D>(a, gave_up == 2 ? blockIdx.x : 0, gave_up == 2 ? gridDim.x : 1);
}

// Joins the parts of the items that the attention kernel cut: o = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c.  CTA (c, s)
// takes 32 rows of the item whose first part CTA c left, a lane per row, d / 32 pieces of four elements per warp; the pieces
// of four parts are in flight at once.  Bound by the parts' bytes, out of L2.
constexpr int JOIN_PARTS = 256;   // weights held at once
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedAttnArgs a) {
  constexpr int NR = W_ROWS, PIECES = D / 4 / 8;
  __shared__ float s_w[JOIN_PARTS][32];
  __shared__ int s_gave_up;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_launch_dependents();
  pdl_wait();
  const PartRecord rec = a.records[blockIdx.x];
  const int r = blockIdx.y * 32 + lane, rr = rec.t * NR + r, R = rec.nq * a.G;
  if (rec.parts < 2 || rec.t * NR + (int)blockIdx.y * 32 >= R) return;
  const bool live = rr < R;
  if (threadIdx.x == 0) s_gave_up = __ldcg(a.gave_up);       // some part may be missing: NaN (s_w's barriers are between)
  constexpr size_t SF = slot_floats<NR, D>();
  const float* slots = a.slots + SF * (size_t)(2 * rec.first);
  auto slot = [&](int p) { return slots + SF * (size_t)(p == 0 ? 1 : 2 * p); };   // part 0 begins in its CTA: part_slot
  float M = -INFINITY, L = 0.f;
  if (live) {
#pragma unroll 4
    for (int p = 0; p < rec.parts; ++p) {
      const float m = __ldcg(slot(p) + r), l = __ldcg(slot(p) + NR + r);
      const float nm = fmaxf(M, m), base = nm == -INFINITY ? 0.f : nm;
      L = L * exp2f(M - base) + l * exp2f(m - base);        // 2^-inf = 0 on either side that has nothing
      M = nm;
    }
  }
  const float base = M == -INFINITY ? 0.f : M, inv = L == 0.f ? 0.f : 1.f / L;
  float4 o[PIECES];
#pragma unroll
  for (int k = 0; k < PIECES; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < rec.parts; p0 += JOIN_PARTS) {
    const int n = min(JOIN_PARTS, rec.parts - p0);
    __syncthreads();
    for (int p = warp; p < n; p += 8) s_w[p][lane] = live ? exp2f(__ldcg(slot(p0 + p) + r) - base) * inv : 0.f;
    __syncthreads();
    if (live) {
#pragma unroll 4
      for (int p = 0; p < n; ++p) {
        const float w = s_w[p][lane];
        const float4* s = reinterpret_cast<const float4*>(slot(p0 + p) + 2 * NR) + (size_t)(warp * PIECES) * NR + r;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
          const float4 v = __ldcg(s + k * NR);
          o[k].x += w * v.x; o[k].y += w * v.y; o[k].z += w * v.z; o[k].w += w * v.w;
        }
      }
    }
  }
  if (!live) return;
  if (s_gave_up) {
    L = __int_as_float(0x7fffffff);
#pragma unroll
    for (int k = 0; k < PIECES; ++k) o[k] = make_float4(L, L, L, L);
  }
  const int tok = row_token(a, rr), head = rec.hk * a.G + rr - tok * a.G;
  const long long at = (long long)(rec.row0 + tok) * a.out.row + (long long)head * a.out.head + warp * PIECES * 4;
#pragma unroll
  for (int k = 0; k < PIECES; ++k) {
    if (a.out_vec && a.out_bf16) {
      *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out.p) + at + 4 * k) = make_uint2(p_pack(o[k].x, o[k].y), p_pack(o[k].z, o[k].w));
    } else if (a.out_vec) {
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out.p) + at + 4 * k) = o[k];
    } else {
      store_out(a, at + 4 * k, o[k].x); store_out(a, at + 4 * k + 1, o[k].y); store_out(a, at + 4 * k + 2, o[k].z); store_out(a, at + 4 * k + 3, o[k].w);
    }
  }
  if (a.lse && warp == 0) a.lse[(size_t)(rec.row0 + tok) * a.H + head] = L == 0.f ? -INFINITY : 0.6931471805599453f * (base + log2f(L));
}

template <int D>
cudaError_t wide_go(PagedAttnArgs a, int num_sm, cudaStream_t st) {
  static DevSmemCache cached{};
  a.lead = 1;
  a.min_run = 2;
  TcArgs t;
  cudaError_t e = tc_args(a, D, &t);
  if (e == cudaSuccess) e = sps_ensure_smem(paged_attn_wide_kernel<D>, WCfg<D>::SMEM, cached);
  if (e != cudaSuccess) return e;
  e = launch_k(paged_attn_wide_kernel<D>, dim3(paged_attn_grid(num_sm)), dim3(W_THREADS), WCfg<D>::SMEM, st, t);
  if (e != cudaSuccess) return e;
  return launch_k(paged_join_kernel<D>, dim3(paged_attn_grid(num_sm), W_ROWS / 32), dim3(256), 0, st, a);
}

}  // namespace

size_t paged_attn_wide_slot_bytes(int d_head) { return sizeof(float) * (d_head == 128 ? slot_floats<W_ROWS, 128>() : slot_floats<W_ROWS, 64>()); }

cudaError_t paged_attn_wide_launch(const PagedAttnArgs& a, int d_head, int num_sm, cudaStream_t st) {
  return d_head == 128 ? wide_go<128>(a, num_sm, st) : wide_go<64>(a, num_sm, st);
}
