// Attention over a paged bf16 cache on the 5th-generation tensor cores, for few query rows per key head (a decode step, a
// scoring pass of K + 1 rows, their grouped heads) and for fp32 queries of any number.
//
// The tokens are the tensor cores' 128-row operand in both products, the query rows their narrow one:
//
//   S^T [128 tokens x NR rows]   = K [128 x d] Q^T              (K straight from the page copies, K-major)
//   O^T [d x NR rows]           += V^T [d x 128] P^T            (V straight from the page copies, MN-major)
//
// so keys and values go from HBM to shared memory to the tensor cores and through no register, and a decode step of one
// row costs a product 16 columns wide instead of 128.  A thread owns one token of the tile (a lane of tensor memory) and
// all its rows' scores; it masks, exponentiates and stores its row of P^T.
//
// Running maximum.  The weights are 2^(s - m) with m fixed at the score of the part's first token, which every row that sees
// anything of the part sees: P is bf16 parts (8 exponent bits) of an fp32 number, sums are fp32, so m only has to keep the
// weights in range, not at most 1, and a weight of 1 is among them.  Only when a score exceeds m by MAX_UP (in base 2) do
// the threads of a column group agree (a reducing barrier) to take the new maximum and rescale what they hold.  The tile's
// differences are then taken again from its raw scores: those to a first token that scored far below the others were
// rounded at its size.  A first score of -inf leaves the least finite number as m, which any finite score outgrows.  That
// leaves a multiply-add, an exponential, an addition and the rounding per score, no
// cross-lane reduction per tile.  Sums stay per thread (its token of every tile) until the part ends.  Each tile's O^T
// is a product of its own, added to fp32 registers: the tensor cores cut the low bits of a running sum instead of rounding
// them, which over a context of 32 768 tokens cost 3.6e-5 of the result.
//
// Types.  bf16 queries: P enters as two bf16 parts (high, rest: 2^-17 relative), so that the output's own rounding is the
// only one of its size; here, bound by HBM, the second part costs nothing.  fp32 queries: Q and P enter as three bf16 parts
// (high, rest, rest of the rest: 24 bits).  Parts lie side by side as columns of one product -- a product reads its
// 128-row operand in 32 clocks however few its columns: 16 columns cost 39 and 48 cost 44 -- and a row's columns are added
// in fp32.
//
// What bounds it: HBM.  A tile of 128 tokens is 64 KB of keys and values (d = 128), 2760 clocks of an SM's share of
// 6.5 TB/s; its 16 products take 39 to 72 clocks each, the softmax a few hundred.  One CTA per SM, equal runs of tiles per
// CTA (paged.cuh), a ring of 4 to 6 half-tiles (K or V) of 32 KB in flight.
//
//   warp 0      copies: lane i asks for page i of the tile (TMA boxes of 64 elements x up to 128 slots, 128-byte swizzle)
//   warp 1      products: S of the next tile, the next part's included, goes before O of this one.  The warp runs as one
//               with an elected lane issuing and constant offsets: descriptors stay in uniform registers (40 clocks a
//               product; issued from a divergent lane they took 130)
//   warps 2, 3  Q of the parts to come, into shared memory in bf16 parts
//   warps 4..   softmax and outputs, 16 rows per group of four warps; for tiles of 16 rows two sets of four warps, each with
//               its own P, O and row arrays, that take the CTA's parts in turn, so that one part's outputs and join go on
//               beside the next part's scores (64 sequences of 300 tokens, 8 key heads: 27.7 -> 24.9 us; batches of short
//               sequences are bound by what a part costs at its ends, not by HBM)
//
// Every wait is bounded; on expiry the CTA sets SPS_PAGED_TIMEOUT, lets its copies and products finish, frees its tensor
// memory, leaves NaN in the call's rows and a word in the workspace, whose counters are part-way, and returns.
#include "paged_tc.cuh"

namespace {

constexpr float MAX_UP = 24.f;       // log2 of the largest weight that is let stand
constexpr float LEAST = -3.402823466e38f;   // the reference of rows that have seen no finite score yet

// Reduces v[c] over the 32 lanes for 16 columns, halving the columns a lane carries at every step; the lane ends up with
// column lane >> 1.
struct OpMax { static __device__ __forceinline__ float f(float a, float b) { return fmaxf(a, b); } };
struct OpAdd { static __device__ __forceinline__ float f(float a, float b) { return a + b; } };
template <class Op> __device__ __forceinline__ float fold16(float (&v)[16], int lane) {
  int off = 16;
#pragma unroll
  for (int w = 8; w >= 1; w >>= 1, off >>= 1) {
    const bool upper = (lane & off) != 0;
#pragma unroll
    for (int k = 0; k < w; ++k) {
      const float send = upper ? v[k] : v[k + w], keep = upper ? v[k + w] : v[k];
      v[k] = Op::f(keep, __shfl_xor_sync(0xffffffffu, send, off));
    }
  }
  return Op::f(v[0], __shfl_xor_sync(0xffffffffu, v[0], 1));
}

template <int D, int NR, int PARTS> struct Cfg {   // PARTS: of Q (1 or 3)
  static constexpr int PP = PARTS == 3 ? 3 : 2;                     // parts of P
  static constexpr int GROUPS = NR / 16;                            // column groups of four softmax warps each
  static constexpr int SETS = NR == 16 ? 2 : 1;                     // sets of softmax warps, taking parts in turn
  static constexpr int SOFT = 128 * GROUPS;                         // softmax threads of a set
  static constexpr int THREADS = 128 + SETS * SOFT;
  static constexpr int N = PARTS * NR, NO = PP * NR;                // columns of S and O
  static constexpr uint32_t HALF = TILE * D * 2;                    // keys or values of a tile
  static constexpr uint32_t Q_BYTES = N * D * 2, P_BYTES = TILE * NO * 2;   // (P: of a set)
  static constexpr uint32_t HDR = 4352;                             // barriers, small per-row arrays
  static constexpr int SET_BYTES = NR * 4 * 9 + 16;                 // a set's share of them
  static constexpr int BUDGET = 232448 - (int)HDR - SETS * (int)P_BYTES;
  static constexpr int QBUF = (BUDGET - 2 * (int)Q_BYTES) / (int)HALF >= 4 ? 2 : 1;
  static constexpr int STAGES_FIT = (BUDGET - QBUF * (int)Q_BYTES) / (int)HALF;
  static constexpr int STAGES = STAGES_FIT > 8 ? 8 : STAGES_FIT;
  static constexpr uint32_t Q_AT = STAGES * HALF, P_AT = Q_AT + QBUF * Q_BYTES, HDR_AT = P_AT + SETS * P_BYTES;
  static constexpr size_t SMEM = HDR_AT + HDR;
  static constexpr int COLUMNS = 2 * N + SETS * NO;                 // of tensor memory: S twice, O once for each set
  static constexpr uint32_t TMEM = COLUMNS <= 64 ? 64 : (COLUMNS <= 128 ? 128 : (COLUMNS <= 256 ? 256 : 512));
  // P^T is the B operand of O, MN-major under the 32-byte swizzle: blocks of 16 columns x 128 tokens, 32 bytes per token
  static constexpr uint32_t P_BLOCK = TILE * 32;
  // kind::f16 instruction descriptors: fp32 accumulator, bf16 x bf16; S: both K-major, M = 128; O: both MN-major, M = d
  static constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
  static constexpr uint32_t IDESC_O = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(NO >> 3) << 17) | ((uint32_t)(D >> 4) << 24);
  static_assert(STAGES >= 4 && COLUMNS <= 512 && NO <= 256 && N % 16 == 0, "shape");
};

// Q of the cursor's item into shared memory, in PARTS bf16 parts, by THREADS threads (named barrier `bar` is theirs): K-major,
// row (part, r) of 64-element block ch at (part NR + r) * 128, its 16-byte chunk k at chunk k ^ (r & 7); rows that do not
// exist are zeros.  s_at: scratch of NR places.  may_write: whether the buffer is free, asked with the first loads under way.
template <int D, int NR, int PARTS, int THREADS, class F>
__device__ __forceinline__ bool load_q(const PagedAttnArgs& a, const WorkCursor& c, unsigned char* q_mem, long long* s_at, int qt, int bar, F may_write) {
  constexpr int CHUNKS = NR * (D / 8) / THREADS, BATCH = CHUNKS % 6 == 0 ? 6 : (CHUNKS % 4 == 0 ? 4 : (CHUNKS % 2 == 0 ? 2 : 1));   // 8-element chunks per thread; in flight
  static_assert(NR * (D / 8) % THREADS == 0 && CHUNKS % BATCH == 0 && THREADS >= NR, "every chunk belongs to a row of the tile");
  const int live = c.nq * a.G - c.t * NR;
  if (qt < NR) {
    const int rr = c.t * NR + qt, tok = row_token(a, rr);
    s_at[qt] = (long long)(c.row0 + tok) * a.q.row + (long long)(c.hk * a.G + rr - tok * a.G) * a.q.head;
  }
  asm volatile("bar.sync %0, %1;" ::"r"(bar), "n"(THREADS) : "memory");
  bool ok = true;
#pragma unroll 1
  for (int b0 = 0; b0 < CHUNKS; b0 += BATCH) {
    float f[BATCH][8];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = qt + (b0 + b) * THREADS, r = i / (D / 8), k8 = i - r * (D / 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[b][j] = 0.f;
      if (r < live) {
        const long long at = s_at[r] + k8 * 8;
        if (PARTS == 3) {
          const float* p = reinterpret_cast<const float*>(a.q.p) + at;
          if (a.q_vec) {
            const float4 x = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
            f[b][0] = x.x; f[b][1] = x.y; f[b][2] = x.z; f[b][3] = x.w; f[b][4] = y.x; f[b][5] = y.y; f[b][6] = y.z; f[b][7] = y.w;
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[b][j] = p[j];
          }
        } else {
          const __nv_bfloat16* p = reinterpret_cast<const __nv_bfloat16*>(a.q.p) + at;
          if (a.q_vec) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { f[b][2 * j] = p_lo(w[j]); f[b][2 * j + 1] = p_hi(w[j]); }
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[b][j] = __bfloat162float(p[j]);
          }
        }
      }
    }
    if (b0 == 0) ok = may_write();
    if (!ok) break;
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = qt + (b0 + b) * THREADS, r = i / (D / 8), k8 = i - r * (D / 8);
      unsigned char* dst = q_mem + (k8 >> 3) * (PARTS * NR * 128) + r * 128 + (((k8 & 7) ^ (r & 7)) << 4);
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        uint32_t u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u[j] = p_pack(f[b][2 * j], f[b][2 * j + 1]);
          if (part + 1 < PARTS) { f[b][2 * j] -= p_lo(u[j]); f[b][2 * j + 1] -= p_hi(u[j]); }
        }
        *reinterpret_cast<uint4*>(dst + part * (NR * 128)) = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
  }
  uint32_t all;   // (and s_at may be written again)
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, %2, %3, q;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(all) : "r"(ok ? 1u : 0u), "r"(bar), "n"(THREADS) : "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  return all != 0;
}

template <int D, int NR, int PARTS>
__global__ void __launch_bounds__(Cfg<D, NR, PARTS>::THREADS, 1) paged_attn_tc_kernel(const __grid_constant__ TcArgs ta) {
  using C = Cfg<D, NR, PARTS>;
  constexpr int SOFT = C::SOFT, STAGES = C::STAGES, N = C::N, PP = C::PP;
  extern __shared__ __align__(1024) unsigned char mem[];   // the ring, Q, P^T (swizzled operands: 1024-byte aligned), header
  const PagedAttnArgs& a = ta.a;
  const uint32_t ring = p_smem(mem), hb = ring + C::HDR_AT;
  unsigned char* hdr = mem + C::HDR_AT;
  // s_full: by set and buffer of S; p_full, pv_done: by set
  const uint32_t full = hb, empty = hb + 64, s_full = hb + 128, s_free = hb + 160, p_full = hb + 176, pv_done = hb + 192, q_ready = hb + 208, q_free = hb + 224, drain = hb + 240, q_first = hb + 248;
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(hdr + 256);
  volatile int* s_abort = reinterpret_cast<volatile int*>(hdr + 260);
  WorkCursor* s_cur = reinterpret_cast<WorkCursor*>(hdr + 272);
  SeqGeom* geo = reinterpret_cast<SeqGeom*>(hdr + 416);                // [GEO]
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int set = C::SETS > 1 && warp >= 4 + SOFT / 32 ? 1 : 0;
  unsigned char* own = hdr + 928 + set * C::SET_BYTES;                 // the set's arrays
  int* s_lim = reinterpret_cast<int*>(own);                            // [NR] last position a row sees
  float* s_a = reinterpret_cast<float*>(own + NR * 4);                 // [NR] maxima
  float* s_b = s_a + NR;                                               // [NR] sums / factors
  float* s_red = s_b + NR;                                             // [4][NR]
  long long* s_off = reinterpret_cast<long long*>(s_red + 4 * NR);     // [NR] where a row's output goes
  int* s_poison = reinterpret_cast<int*>(s_off + NR);
  int* s_last = s_poison + 1;
  long long* s_qat = reinterpret_cast<long long*>(hdr + 928 + C::SETS * C::SET_BYTES);   // [2][NR] where a row of Q is (loader, first part)
  static_assert(928 + C::SETS * C::SET_BYTES + 16 * NR <= (int)C::HDR && sizeof(WorkCursor) <= 144 && sizeof(SeqGeom) * GEO <= 512, "header");

  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { p_bar_init(full + 8 * i, 1); p_bar_init(empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { p_bar_init(s_free + 8 * i, SOFT); p_bar_init(q_ready + 8 * i, 64); p_bar_init(q_free + 8 * i, 1); p_bar_init(p_full + 8 * i, SOFT); p_bar_init(pv_done + 8 * i, 1); }
    for (int i = 0; i < 4; ++i) p_bar_init(s_full + 8 * i, 1);
    p_bar_init(q_first, SOFT); p_bar_init(drain, 1);
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&ta.tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&ta.tm_v) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(hb + 256), "n"(C::TMEM) : "memory");
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
  const uint32_t tmem = __shfl_sync(0xffffffffu, *s_tmem, 0), tmem_o = tmem + 2 * N;
  WorkCursor c = *s_cur;

  if (warp == 0) {
    copy_pages<D, NR, STAGES>(ta, c, geo, ring, full, empty, s_abort);
  } else if (warp == 1) {
    // ---------------------------------------------------------------------------------------------------- products
    const bool leader = p_elect();
    bool ok = true;
    int e_s = 0, e_o = 1, sn = 0, qn = 0, s_i = 0;             // half-tiles of the next S and O, scores so far, parts so far, S's tile in its part
    int on = 0;                                                // parts whose O is done
    uint32_t p_phase = 0;                                      // parity of p_full, a bit for each set
    WorkCursor cs = c;                                         // the part S is at; c is the part O is at
    auto wait = [&](uint32_t bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, p_wait(bar, parity & 1u, a, s_abort));
    };
    auto score = [&]() {                                       // S of the next tile
      if (!cs.valid) return;
      const int buf = sn & 1, qb = qn % C::QBUF;
      if (s_i == 0) {
        if (qn == 0) wait(q_first, 0);
        else wait(q_ready + 8 * qb, (uint32_t)(qn / C::QBUF - (qb == 0 ? 1 : 0)));   // (the first part did not use it)
      }
      if (sn >= 2) wait(s_free + 8 * buf, (uint32_t)((sn >> 1) - 1));
      wait(full + 8 * (e_s % STAGES), (uint32_t)(e_s / STAGES));
      if (!ok) return;
      P_FENCE_AFTER();
      const bool last = ++s_i == cs.k1 - cs.k0;
      if (leader) {
        const uint32_t ka = p_desc_lo(ring + (uint32_t)(e_s % STAGES) * C::HALF, 16), qa = p_desc_lo(ring + C::Q_AT + qb * C::Q_BYTES, 16), d = tmem + buf * N;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          p_mma(d, ka + (k >> 2) * (TILE * 128 >> 4) + (k & 3) * 2, p_desc_hi(1024, 2), qa + (k >> 2) * (N * 128 >> 4) + (k & 3) * 2, p_desc_hi(1024, 2), C::IDESC_S, k > 0);
        p_commit(empty + 8 * (e_s % STAGES));
        p_commit(s_full + 16 * (qn % C::SETS) + 8 * buf);
        if (last) p_commit(q_free + 8 * qb);
      }
      __syncwarp();
      e_s += 2;
      ++sn;
      if (last) { cursor_next<NR, TILE>(a, cs, geo); s_i = 0; ++qn; }
    };
    score();
    while (c.valid && ok) {
      const int g = on % C::SETS;
      for (int n = c.k1 - c.k0; n > 0 && ok; --n) {
        score();
        wait(p_full + 8 * g, p_phase >> g);
        wait(full + 8 * (e_o % STAGES), (uint32_t)(e_o / STAGES));
        if (!ok) break;
        P_FENCE_AFTER();
        if (leader) {
          const uint32_t va = p_desc_lo(ring + (uint32_t)(e_o % STAGES) * C::HALF, TILE * 128), pa = p_desc_lo(ring + C::P_AT + g * C::P_BYTES, C::P_BLOCK);
#pragma unroll
          for (int k = 0; k < TILE / 16; ++k)
            p_mma(tmem_o + g * C::NO, va + k * (16 * 128 >> 4), p_desc_hi(1024, 2), pa + k * (16 * 32 >> 4), p_desc_hi(256, 6), C::IDESC_O, k > 0);
          p_commit(empty + 8 * (e_o % STAGES));
          p_commit(pv_done + 8 * g);
        }
        __syncwarp();
        e_o += 2;
        p_phase ^= 1u << g;
      }
      ++on;
      cursor_next<NR, TILE>(a, c, geo);
    }
    // Every product issued must be done before the ring and the tensor memory go away.  After a part that was worked to its
    // end they are; but softmax warps that gave up go on to the end without waiting for them, and this warp need not notice.
    if (!ok) *s_abort = 1;
    if (leader) p_commit(drain);
    __syncwarp();
    p_drain(drain, 0u);
  } else if (warp < 4) {
    // ---------------------------------------------------------------------------------------------------- Q
    const int qt = tid - 64;
    bool ok = true;
    if (c.valid) cursor_next<NR, TILE>(a, c, geo);   // the first part's are loaded by the softmax warps, which have nothing else to do yet
    for (int qn = 1; c.valid && ok; ++qn) {
      const int qb = qn % C::QBUF, use = qn / C::QBUF;
      ok = load_q<D, NR, PARTS, 64>(a, c, mem + C::Q_AT + qb * C::Q_BYTES, s_qat, qt, 7,
                                    [&]() { return use == 0 || p_wait(q_free + 8 * qb, (uint32_t)(use - 1) & 1u, a, s_abort); });
      if (!ok) break;
      p_arrive(q_ready + 8 * qb);
      cursor_next<NR, TILE>(a, c, geo);
    }
  } else {
    // ---------------------------------------------------------------------------------------------------- softmax
    const int st = tid - 128 - set * SOFT, quarter = warp & 3, group = C::SETS > 1 ? 0 : (warp - 4) >> 2, col0 = group * 16;
    const int my = quarter * 32 + lane;                       // token of the tile, and row of O^T (for d = 128)
    const uint32_t t_lane = (uint32_t)(quarter * 32) << 16;
    // After a wait that ran out the softmax threads keep their common path -- barriers among them always meet -- and skip
    // the waits, until they agree at the part's end to stop.
    bool ok = true;
    int pn = 0, it = 0;                                       // outputs awaited (the set's); half-tiles of the parts before (both sets')
    uint32_t s_phase = 0;                                     // parity of s_full, a bit for each buffer
    auto all_sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + 8 * set), "n"(SOFT) : "memory"); };
    auto group_sync = [&]() { asm volatile("bar.sync %0, 128;" ::"r"(3 + group + 8 * set) : "memory"); };
    if (c.valid && set == 0) {
      ok = load_q<D, NR, PARTS, SOFT>(a, c, mem + C::Q_AT, s_qat + NR, st, 1, []() { return true; });
      p_arrive(q_first);
    }
    auto next_part = [&]() {
      it += 2 * (c.k1 - c.k0);
      cursor_next<NR, TILE>(a, c, geo);
    };
    if (set == 1 && c.valid) next_part();
    while (c.valid) {
      const int R = c.nq * a.G, r0 = c.t * NR, n = c.k1 - c.k0, first_lim = c.len - c.nq + row_token(a, r0);
      if (st < NR) {
        const int rr = r0 + st, tok = row_token(a, rr);
        s_lim[st] = rr < R ? c.len - c.nq + tok : -1;
        s_off[st] = rr < R ? (long long)(c.row0 + tok) * a.out.row + (long long)(c.hk * a.G + rr - tok * a.G) * a.out.head : 0;
      }
      if (st == 0) *s_poison = 0x7fffffff;
      all_sync();
      int first, parts;
      item_ctas(c, first, parts);
      float l[16], o[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) l[j] = o[j] = 0.f;
      // o += O^T of the last tile multiplied, once that product is done
      bool held = false;
      auto collect = [&]() {
        if (!held) return;
        held = false;
        ok = ok && p_wait(pv_done + 8 * set, (uint32_t)(pn - 1) & 1u, a, s_abort);
        __syncwarp();
        P_FENCE_AFTER();
        float t[PP][16];
#pragma unroll
        for (int part = 0; part < PP; ++part) p_ld16(tmem_o + set * C::NO + t_lane + part * NR + col0, t[part]);
        P_WAIT_LD();
        p_landed<PP * 16>(t[0]);
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          if (PP == 3) p_add2(t[1][j], t[1][j + 1], t[PP - 1][j], t[PP - 1][j + 1]);
          p_add2(t[0][j], t[0][j + 1], t[1][j], t[1][j + 1]);
          p_add2(o[j], o[j + 1], t[0][j], t[0][j + 1]);
        }
      };
      for (int i = 0; i < n; ++i) {
        const int buf = ((it >> 1) + i) & 1, p0 = (c.k0 + i) * TILE, pos = p0 + my;
        const bool edge = p0 + TILE - 1 > first_lim;          // some row does not see all of this tile
        ok = ok && p_wait(s_full + 16 * set + 8 * buf, (s_phase >> buf) & 1u, a, s_abort);
        s_phase ^= 1u << buf;
        __syncwarp();
        P_FENCE_AFTER();
        float x[16];
        auto scores = [&]() {                                 // x = S of this thread's token
          float t[PARTS][16];
#pragma unroll
          for (int part = 0; part < PARTS; ++part) p_ld16(tmem + buf * N + t_lane + part * NR + col0, t[part]);
          P_WAIT_LD();
          p_landed<PARTS * 16>(t[0]);
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            if (PARTS == 3) {
              p_add2(t[PARTS / 2][j], t[PARTS / 2][j + 1], t[PARTS - 1][j], t[PARTS - 1][j + 1]);
              p_add2(t[0][j], t[0][j + 1], t[PARTS / 2][j], t[PARTS / 2][j + 1]);
            }
            x[j] = t[0][j];
            x[j + 1] = t[0][j + 1];
          }
        };
        scores();
        // ---- the reference maximum: the part's first token's score, a new one only when a score has outgrown it
        if (i == 0) {
          if (my == 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float s = x[j] * a.scale_log2;
              s_a[col0 + j] = s_lim[col0 + j] < pos ? 0.f : (fabsf(s) == INFINITY ? LEAST : s);
            }
          }
          group_sync();
        }
        // x -> scale x - m, rounded once, -inf where a row does not see the token
        auto relative = [&](const float* ref) {
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float4 m = *reinterpret_cast<const float4*>(ref + j);
            p_fma2(x[j], x[j + 1], a.scale_log2, -m.x, -m.y);
            p_fma2(x[j + 2], x[j + 3], a.scale_log2, -m.z, -m.w);
            if (edge) {
              const int4 lim = *reinterpret_cast<const int4*>(s_lim + col0 + j);
              x[j] = pos <= lim.x ? x[j] : -INFINITY;
              x[j + 1] = pos <= lim.y ? x[j + 1] : -INFINITY;
              x[j + 2] = pos <= lim.z ? x[j + 2] : -INFINITY;
              x[j + 3] = pos <= lim.w ? x[j + 3] : -INFINITY;
            }
          }
        };
        relative(s_a + col0);
        float up = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; j += 4) up = fmaxf(up, fmaxf(fmaxf(x[j], x[j + 1]), fmaxf(x[j + 2], x[j + 3])));
        uint32_t retake;
        asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, %2, 128, q;\n selp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(retake) : "r"(up > MAX_UP ? 1u : 0u), "r"(3 + group + 8 * set) : "memory");
        if (retake) {
          scores();
          {
            float y[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = !edge || pos <= s_lim[col0 + j] ? x[j] * a.scale_log2 : -INFINITY;
            const float top = fold16<OpMax>(y, lane);
            s_red[quarter * NR + col0 + (lane >> 1)] = top;
          }
          collect();
          group_sync();
          float m_new = 0.f;                                  // (of column col0 + my, for the group's first 16 threads)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int cc = col0 + j;
            const float was = s_a[cc], m = fmaxf(fmaxf(fmaxf(s_red[cc], s_red[NR + cc]), fmaxf(s_red[2 * NR + cc], s_red[3 * NR + cc])), was);
            const float al = p_ex2(was - m);
            l[j] = m == INFINITY ? __int_as_float(0x7fffffff) : l[j] * al;   // an infinite score that the row sees
            o[j] *= al;
            if (my == j) m_new = m;
          }
          group_sync();                                       // s_a has been read
          if (my < 16) s_a[col0 + my] = m_new;
          group_sync();                                       // ... written, s_red may be
          relative(s_a + col0);
        }
        P_FENCE_BEFORE();
        p_arrive(s_free + 8 * buf);
        // ---- weights
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = p_ex2(x[j]);
#pragma unroll
        for (int j = 0; j < 16; j += 2) p_add2(l[j], l[j + 1], x[j], x[j + 1]);
        // P^T is written once the previous output product has read it
        if (i > 0) collect();
        if (edge) {
          // slots behind the sequence hold anything: zero (0 x NaN is NaN in a product).  New tokens some rows do not see:
          // a value that is not finite is taken out and remembered, its rows become NaN at the end.
          const int e = it + 2 * i + 1;
          ok = ok && p_wait(full + 8 * (e % STAGES), (uint32_t)(e / STAGES) & 1u, a, s_abort);
          if (ok && group == 0 && pos > first_lim) {
            unsigned char* vr = mem + (e % STAGES) * C::HALF + my * 128;
            bool clear = pos >= c.len;
            if (!clear) {
#pragma unroll
              for (int ch = 0; ch < D / 64; ++ch)
#pragma unroll 2
                for (int q = 0; q < 8; ++q) {
                  const uint4 u = *reinterpret_cast<const uint4*>(vr + ch * (TILE * 128) + ((q ^ (my & 7)) << 4));
                  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                  for (int z = 0; z < 4; ++z) clear = clear || (w[z] & 0x7f80u) == 0x7f80u || (w[z] & 0x7f800000u) == 0x7f800000u;
                }
              if (clear) atomicMin(s_poison, pos);
            }
            if (clear) {
#pragma unroll
              for (int ch = 0; ch < D / 64; ++ch)
#pragma unroll 2
                for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(vr + ch * (TILE * 128) + (q << 4)) = make_uint4(0, 0, 0, 0);
            }
          }
        }
        unsigned char* pr = mem + C::P_AT + set * C::P_BYTES + group * C::P_BLOCK + my * 32;
        const int sw = (my >> 2) & 1;                          // 32-byte swizzle: a token's two 16-byte chunks swap in every other group of 4
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int part = 0; part < PP; ++part) {
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float &f0 = x[8 * k + 2 * j], &f1 = x[8 * k + 2 * j + 1];
              u[j] = p_pack(f0, f1);
              if (part + 1 < PP) p_add2(f0, f1, -p_lo(u[j]), -p_hi(u[j]));
            }
            *reinterpret_cast<uint4*>(pr + part * C::GROUPS * C::P_BLOCK + ((k ^ sw) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        P_FENCE_BEFORE();
        p_arrive(p_full + 8 * set);
        ++pn;
        held = true;
      }
      // ---- the part's end: sums over the tokens, then O^T
      const float sum = fold16<OpAdd>(l, lane);
      s_red[quarter * NR + col0 + (lane >> 1)] = sum;
      collect();
      {
        uint32_t all;
        asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, %2, %3, q;\n selp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(all) : "r"(ok ? 1u : 0u), "r"(1 + 8 * set), "n"(SOFT) : "memory");
        if (!all) break;
      }
      if (st < NR) {
        float t = (s_red[st] + s_red[NR + st]) + (s_red[2 * NR + st] + s_red[3 * NR + st]);
        if (s_lim[st] >= *s_poison) t = __int_as_float(0x7fffffff);
        if (t == 0.f) s_a[st] = -INFINITY;
        s_b[st] = t;
        if (parts == 1) {
          if (a.lse && r0 + st < R) {
            const int rr = r0 + st, tok = row_token(a, rr);
            a.lse[(size_t)(c.row0 + tok) * a.H + c.hk * a.G + rr - tok * a.G] = t == 0.f ? -INFINITY : 0.6931471805599453f * (s_a[st] + log2f(t));
          }
          s_b[st] = t == 0.f ? 0.f : 1.f / t;
        }
      }
      all_sync();
      const int e = D == 128 ? my : quarter * 16 + lane;      // element of the head (d = 64: 16 rows in each quarter's first 16 lanes)
      const bool live_lane = D == 128 || lane < 16;
      float* slot = a.slots + slot_floats<NR, D>() * (size_t)part_slot(blockIdx.x, c.k0 == 0);
      const int rows = min(max(R - r0 - col0, 0), live_lane ? 16 : 0);
      if (parts == 1) {
#pragma unroll
        for (int j0 = 0; j0 < 16; j0 += 4) {
          if (j0 >= rows) break;
          long long at[4];
          float f[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) { at[j] = s_off[col0 + j0 + j] + e; f[j] = s_b[col0 + j0 + j]; }
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = f[j] == 0.f ? 0.f : o[j0 + j] * f[j];
          if (a.out_bf16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (j0 + j < rows) reinterpret_cast<__nv_bfloat16*>(a.out.p)[at[j]] = __float2bfloat16_rn(f[j]);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (j0 + j < rows) reinterpret_cast<float*>(a.out.p)[at[j]] = f[j];
          }
        }
      } else {
        float* s = slot + 2 * NR + col0 * D + e;
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (j < rows) __stcg(s + j * D, o[j]);
      }
      if (parts > 1) {
        if (st < NR) { __stcg(slot + st, s_a[st]); __stcg(slot + NR + st, s_b[st]); }
        all_sync();
        if (st == 0) {
          *s_last = part_arrive(a.counters + first, parts);
        }
        all_sync();
        if (*s_last) join_parts<NR, D, SOFT>(a, c, first, parts, st, s_b, s_a, reinterpret_cast<float*>(mem + C::P_AT + set * C::P_BYTES), C::P_BYTES / 4, 2 + 8 * set);
      }
      all_sync();   // s_a, s_b, s_lim are free again
      next_part();
      if (C::SETS > 1 && c.valid) next_part();   // the other set's
    }
    if (!ok) *s_abort = 1;
  }
  P_FENCE_BEFORE();
  __syncthreads();
  if (warp == 1) {
    P_FENCE_AFTER();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::TMEM) : "memory");
  }
  // (items that this CTA leaves unfinished are never joined: what other CTAs write over these rows is whole)
  if (const int gave_up = *s_abort) nan_rows<D>(a, gave_up == 2 ? blockIdx.x : 0, gave_up == 2 ? gridDim.x : 1);
}

template <int D, int NR, int PARTS>
cudaError_t tc_go(PagedAttnArgs a, int num_sm, cudaStream_t st) {
  static DevSmemCache cached{};
  // An item costs about two tiles before its first one (Q, the first scores, its outputs): 64 ragged sequences of one token
  // took 103 / 82 / 61 / 62 / 65 us at 0 / 1 / 2 / 3 / 4 with one set of softmax warps, 57 / 60 / 64 at 1 / 2 / 3 with two;
  // longer least runs than one tile only slowed short calls down.
  a.lead = Cfg<D, NR, PARTS>::SETS == 2 ? 1 : 2;
  a.min_run = 1;
  TcArgs t;
  cudaError_t e = tc_args(a, D, &t);
  if (e == cudaSuccess) e = sps_ensure_smem(paged_attn_tc_kernel<D, NR, PARTS>, Cfg<D, NR, PARTS>::SMEM, cached);
  if (e != cudaSuccess) return e;
  return launch_k(paged_attn_tc_kernel<D, NR, PARTS>, dim3(paged_attn_grid(num_sm)), dim3(Cfg<D, NR, PARTS>::THREADS), Cfg<D, NR, PARTS>::SMEM, st, t);
}

// The narrowest tile that holds a sequence's rows of one key head (18 sequences of 4096 tokens, bf16: 24 rows 52 us in tiles of
// 32, 40 rows 54 us in tiles of 48 and 61 us in tiles of 64).  More rows than the widest: fp32 ones in several tiles of it,
// bf16 ones on the kernel for many rows (18 sequences x 64 rows x 4096 tokens: 62 us here, 73 us there).
template <int D>
cudaError_t tc_rows(const PagedAttnArgs& a, long long rows, int num_sm, cudaStream_t st) {
  if (a.q_bf16) {
    if (rows <= 16) return tc_go<D, 16, 1>(a, num_sm, st);
    if (rows <= 32) return tc_go<D, 32, 1>(a, num_sm, st);
    if (rows <= 48) return tc_go<D, 48, 1>(a, num_sm, st);
    return tc_go<D, 64, 1>(a, num_sm, st);
  }
  if (rows <= 16) return tc_go<D, 16, 3>(a, num_sm, st);
  if (rows <= 32) return tc_go<D, 32, 3>(a, num_sm, st);
  return tc_go<D, 48, 3>(a, num_sm, st);
}

}  // namespace

size_t paged_attn_tc_slot_bytes(int d_head) { return sizeof(float) * (d_head == 128 ? slot_floats<64, 128>() : slot_floats<64, 64>()); }

cudaError_t paged_attn_tc_launch(const PagedAttnArgs& a, int d_head, int max_q, int num_sm, cudaStream_t st) {
  const long long rows = (long long)max_q * a.G;
  if (a.q_bf16 && rows > 64) return paged_attn_wide_launch(a, d_head, num_sm, st);
  return d_head == 128 ? tc_rows<128>(a, rows, num_sm, st) : tc_rows<64>(a, rows, num_sm, st);
}
