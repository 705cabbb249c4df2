// Tensor-core and copy helpers of the paged attention kernels: mbarriers with bounded waits, page copies, operand
// descriptors, tcgen05 products and tensor-memory access, two-wide fp32 arithmetic, and the tensor maps of a page pool.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>

#include <mutex>

#include "paged.cuh"

constexpr int TILE = 128;            // tokens per tile

struct TcArgs {
  CUtensorMap tm_k, tm_v;
  PagedAttnArgs a;
  int box;             // slots per copy: min(page_size, 128)
  int head_first;      // the tensor maps' dimensions are (d, head, slot, page) instead of (d, slot, head, page)
};

__device__ __forceinline__ uint32_t p_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void p_bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void p_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void p_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t p_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
  return ok;
}
__device__ __forceinline__ unsigned long long p_timer() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// bounded wait: false after a.wait_ns, or as soon as another thread of the CTA gave up
__device__ __forceinline__ bool p_wait(uint32_t bar, uint32_t parity, const PagedAttnArgs& a, volatile int* abort_flag) {
  if (p_try(bar, parity)) return true;
  const unsigned long long t0 = p_timer();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i) {
      if (p_try(bar, parity)) return true;
      if (*abort_flag) return false;
    }
    if (p_timer() - t0 > a.wait_ns) {
      paged_flag(a.s.status, SPS_PAGED_TIMEOUT);
      *reinterpret_cast<volatile int*>(a.gave_up) = 1;
      *abort_flag = 1;
      return false;
    }
  }
}
// for what the hardware finishes by itself (copies, products): two seconds, however short the bound on other waits is
__device__ __forceinline__ void p_drain(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = p_timer();
  while (!p_try(bar, parity) && p_timer() - t0 <= 2000000000ull) {}
}
__device__ __forceinline__ void p_copy(uint32_t dst, const CUtensorMap* tm, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(tm),
               "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
               : "memory");
}
// shared-memory operand descriptors: the low word holds the address and, for MN-major operands, the bytes between blocks
// along the contiguous direction (lbo); the high word the bytes between groups of 8 rows (sbo), version 1 and the swizzle
// (layout 2 / 6 = 128 / 32 bytes)
__device__ __forceinline__ uint32_t p_desc_lo(uint32_t addr, uint32_t lbo) { return ((addr & 0x3ffffu) >> 4) | (lbo >> 4) << 16; }
__host__ __device__ constexpr uint32_t p_desc_hi(uint32_t sbo, uint32_t layout) { return (sbo >> 4) | 1u << 14 | layout << 29; }
__device__ __forceinline__ void p_mma(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n mov.b64 a, {%1, %2};\n mov.b64 b, {%3, %4};\n setp.ne.b32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n}\n" ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate ? 1u : 0u)
      : "memory");
}
__device__ __forceinline__ bool p_elect() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void p_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
#define P_FENCE_AFTER() asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory")
#define P_FENCE_BEFORE() asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory")

// Loads from tensor memory land in their registers on their own time: P_WAIT_LD, then p_landed on each register array, lie
// between a load and the first use (p_landed does nothing; it keeps the compiler from using a value before the wait).
__device__ __forceinline__ void p_ld16(uint32_t t, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]),
        "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(t)
      : "memory");
}
#define P_WAIT_LD() asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory")
template <int N> __device__ __forceinline__ void p_landed(float* v) {
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7]));
}

__device__ __forceinline__ float p_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two fp32 operations in one instruction
__device__ __forceinline__ void p_add2(float& x, float& y, float a, float b) {
  asm("{\n .reg .b64 s, t;\n mov.b64 s, {%0, %1};\n mov.b64 t, {%2, %3};\n add.rn.f32x2 s, s, t;\n mov.b64 {%0, %1}, s;\n}\n" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void p_fma2(float& x, float& y, float f, float a, float b) {   // (x, y) f + (a, b)
  asm("{\n .reg .b64 s, t, u;\n mov.b64 s, {%0, %1};\n mov.b64 t, {%2, %2};\n mov.b64 u, {%3, %4};\n fma.rn.f32x2 s, s, t, u;\n mov.b64 {%0, %1}, s;\n}\n"
      : "+f"(x), "+f"(y) : "f"(f), "f"(a), "f"(b));
}
// two floats rounded to bf16, the first in the low half
__device__ __forceinline__ uint32_t p_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float p_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float p_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

__device__ __forceinline__ void p_ld32(uint32_t t, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
      "%26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]),
        "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(t)
      : "memory");
}
__device__ __forceinline__ void p_st16(uint32_t t, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(t)
               : "memory");
}
#define P_WAIT_ST() asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory")

// The copy warp: keys and values of every tile of the CTA's run, half-tile after half-tile (K, V, K, V, ...), into a ring of
// STAGES of them.  Lane i asks for page i of the tile (or its only page): boxes of 64 elements x ta.box slots, 128-byte
// swizzle, so a half-tile is d / 64 blocks of 128 tokens x 128 bytes.
template <int D, int NR, int STAGES>
__device__ __forceinline__ void copy_pages(const TcArgs& ta, WorkCursor c, const SeqGeom* geo, uint32_t ring, uint32_t full, uint32_t empty, volatile int* s_abort) {
  constexpr uint32_t HALF = TILE * D * 2;
  const PagedAttnArgs& a = ta.a;
  const int lane = threadIdx.x & 31;
  bool ok = true;
  int it = 0;   // half-tiles asked for so far
  const int drop = c.valid && c.k0 == 0 && c.item0 == a.lead ? a.drop_stage : -1;   // (the CTA with the list's first tile)
  const int boxes = TILE / ta.box;
  auto page_of = [&](const WorkCursor& c, int kt) {   // this lane's page of a tile
    const int pos = kt * TILE + lane * ta.box;
    return lane < boxes && pos < c.len ? a.s.pages[(long long)c.b * a.s.pages_ld + (pos >> a.s.page_shift)] : 0;
  };
  int next = c.valid ? page_of(c, c.k0) : 0;
  while (c.valid && ok) {
    WorkCursor after = c;
    cursor_next<NR, TILE>(a, after, geo);
    for (int kt = c.k0; kt < c.k1 && ok; ++kt) {
      const int pos = kt * TILE + lane * ta.box;
      const bool mine = lane < boxes && pos < c.len;
      int page = next;
      // the next tile's page numbers, the next part's included, are under way while this tile waits
      if (kt + 1 < c.k1) next = page_of(c, kt + 1);
      else if (after.valid) next = page_of(after, after.k0);
      if (mine && (page < 0 || page >= a.s.n_pages)) { paged_flag(a.s.status, SPS_PAGED_BAD_PAGE); page = a.s.n_pages; }   // outside the map: zeros
      const int in_page = pos & (a.s.page_size - 1);
      const int n = __popc(__ballot_sync(0xffffffffu, mine));
#pragma unroll
      for (int kv = 0; kv < 2; ++kv, ++it) {
        const int slot = it % STAGES, use = it / STAGES;
        if (use > 0) {
          ok = p_wait(empty + 8 * slot, (uint32_t)(use - 1) & 1u, a, s_abort);
          ok = __all_sync(0xffffffffu, ok) && !*s_abort;
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
        }
        if (it == drop) continue;   // test hook: never asked for, the wait for it runs out
        if (lane == 0) {
          if (n > 0) p_expect(full + 8 * slot, (uint32_t)n * (uint32_t)ta.box * (uint32_t)(D * 2));
          else p_arrive(full + 8 * slot);
        }
        __syncwarp();
        if (mine) {
          const CUtensorMap* tm = kv ? &ta.tm_v : &ta.tm_k;
          const uint32_t dst = ring + slot * HALF + (uint32_t)(lane * ta.box) * 128u;
#pragma unroll
          for (int ch = 0; ch < D / 64; ++ch)
            p_copy(dst + ch * (TILE * 128), tm, ch * 64, ta.head_first ? c.hk : in_page, ta.head_first ? in_page : c.hk, page, full + 8 * slot);
        }
        __syncwarp();
      }
    }
    c = after;
  }
  if (lane == 0) {   // whatever happened, the copies in flight land before this CTA's shared memory goes away
    if (!ok) *s_abort = 1;
    for (int j = max(0, it - STAGES); j < it; ++j)
      if (j != drop) p_drain(full + 8 * (j % STAGES), (uint32_t)(j / STAGES) & 1u);
  }
}

inline PFN_cuTensorMapEncodeTiled_v12000 page_encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
  static std::mutex mu;
  std::lock_guard<std::mutex> lock(mu);
  if (!encode) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn) return nullptr;
    encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  }
  return encode;
}

// the pages as a 4-D tensor, boxes of 64 elements x `box` slots under the 128-byte swizzle; pages outside it read as zeros
inline cudaError_t page_map(PFN_cuTensorMapEncodeTiled_v12000 encode, const void* p, const PagedAttnArgs& a, int D, int box, bool head_first, CUtensorMap* out) {
  const cuuint64_t head = (cuuint64_t)(a.Hkv > 1 ? a.head_stride : D) * 2, slot = (cuuint64_t)a.pos_stride * 2;
  const cuuint64_t gdim[4] = {(cuuint64_t)D, (cuuint64_t)(head_first ? a.Hkv : a.s.page_size), (cuuint64_t)(head_first ? a.s.page_size : a.Hkv), (cuuint64_t)a.s.n_pages};
  const cuuint64_t gstride[3] = {head_first ? head : slot, head_first ? slot : head, (cuuint64_t)a.page_stride * 2};
  const cuuint32_t bx[4] = {64, (cuuint32_t)(head_first ? 1 : box), (cuuint32_t)(head_first ? box : 1), 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(p), gdim, gstride, bx, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}


inline cudaError_t tc_args(const PagedAttnArgs& a, int D, TcArgs* t) {
  PFN_cuTensorMapEncodeTiled_v12000 encode = page_encoder();
  if (!encode) return cudaErrorNotSupported;
  t->a = a;
  t->box = a.s.page_size < TILE ? a.s.page_size : TILE;
  t->head_first = a.Hkv > 1 && a.head_stride < a.pos_stride;
  const cudaError_t e = page_map(encode, a.k, a, D, t->box, t->head_first, &t->tm_k);
  return e != cudaSuccess ? e : page_map(encode, a.v, a, D, t->box, t->head_first, &t->tm_v);
}
