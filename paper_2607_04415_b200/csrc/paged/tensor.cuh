// The Blackwell pieces that the chunk kernel uses: bounded waits on mbarriers, tensor copies, and the
// fifth-generation matrix unit with its tensor memory.
#pragma once
#include <cuda.h>

#include "mma.cuh"

namespace gorio {
namespace paged {

constexpr u32 kDrainTicks = 10000000;                   // of 1024 ns: of the waits for a block's own copies and products, at its end

__device__ __forceinline__ u64 now_ns() {
  u64 t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

__device__ __forceinline__ void bar_init(u64 *bar, u32 count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(u64 *bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory"); }
__device__ __forceinline__ void bar_expect(u64 *bar, u32 bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(u64 *bar, u32 parity) {
  u32 ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
  return ok != 0;
}
// Waits of a whole warp for the phase of the given parity, with one answer for all its lanes: what follows a wait (tensor memory,
// votes) needs them together, and decided lane by lane some could see the phase end and others the limit pass.  False once a
// wait of this block has lasted longer than its limit: the warp then leaves its loops, and the block ends with its error word set.
// `anew` is asked when the limit has passed: true where the time until now does not count.
struct WaitLimit {
  u32 ticks;               // of 1024 ns
  volatile u32 *failed;    // of the block
};
__device__ __forceinline__ u32 now_ticks() { return (u32)(now_ns() >> 10); }
template <typename Anew>
__device__ __forceinline__ bool warp_wait(u64 *bar, u32 parity, const WaitLimit &limit, const Anew &anew) {
  bool ok = bar_try(bar, parity);
  if (!__all_sync(0xffffffffu, ok)) {
    u32 t0 = now_ticks();
    do {
      if (now_ticks() - t0 >= limit.ticks) {
        if (anew()) t0 = now_ticks();
        else *limit.failed = 1;
      }
      if (__any_sync(0xffffffffu, *limit.failed)) return false;
      ok = bar_try(bar, parity);
    } while (!__all_sync(0xffffffffu, ok));
  }
  return true;
}
__device__ __forceinline__ bool warp_wait(u64 *bar, u32 parity, const WaitLimit &limit) {
  return warp_wait(bar, parity, limit, [] { return false; });
}
// A wait for what this block itself has set going and nothing can hold up: no reason to give up early.
__device__ __forceinline__ void drain(u64 *bar, u32 parity) {
  const u32 t0 = now_ticks();
  while (!bar_try(bar, parity) && now_ticks() - t0 < kDrainTicks) {}
}
__device__ __forceinline__ u32 uniform(u32 v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ bool one_lane() {
  u32 yes;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(yes));
  return yes != 0;
}

// One box of a (head size, token, head, page) tensor into shared memory.
__device__ __forceinline__ void copy_box(void *to, const CUtensorMap *map, int x, int token, int head, int page, u64 *bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_addr(to)),
               "l"(map), "r"(x), "r"(token), "r"(head), "r"(page), "r"(smem_addr(bar))
               : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tmem_alloc(u32 *at, u32 columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(at)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(u32 base, u32 columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void mma_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// the barrier completes when all matrix operations that this thread has issued so far have
__device__ __forceinline__ void mma_commit(u64 *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Shared-memory operand of 128-byte rows with the 128-byte swizzle.  Rows along K (keys' or queries' head
// elements): groups of 8 rows follow each other, 1024 bytes.  Columns along K (values, whose rows are keys): 64 of
// the head's elements a row, the next 64 `lead` bytes on, the next 8 keys 1024 bytes on.
// The low word holds the address and `lead`, both in units of 16 bytes, the high word is the same for all.
__device__ __forceinline__ u32 operand(const void *p, u32 lead) { return ((smem_addr(p) & 0x3FFFF) >> 4) | ((lead >> 4) << 16); }
constexpr u32 kOperandHigh = (1024 >> 4) | (1u << 14) | (2u << 29);

template <typename T>
struct TypeCode { static constexpr u32 value = 1; };       // bfloat16
template <>
struct TypeCode<__half> { static constexpr u32 value = 0; };

// 16-bit operands, 32-bit sums, 128 rows by n columns; the second operand's rows along K or not
template <typename T>
__host__ __device__ constexpr u32 mma_shape(u32 n, bool b_columns) {
  return (1u << 4) | (TypeCode<T>::value << 7) | (TypeCode<T>::value << 10) | ((b_columns ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void mma_ss(u32 d, u32 a, u32 b, u32 shape, bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 x, y; setp.ne.u32 p, %4, 0; mov.b64 x, {%1, %5}; mov.b64 y, {%2, %5}; "
               "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }" ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"((u32)add), "n"(kOperandHigh)
               : "memory");
}
__device__ __forceinline__ void mma_ts(u32 d, u32 a, u32 b, u32 shape, bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 y; setp.ne.u32 p, %4, 0; mov.b64 y, {%2, %5}; "
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p; }" ::"r"(d), "r"(a), "r"(b), "r"(shape), "r"((u32)add), "n"(kOperandHigh)
               : "memory");
}

// 32 columns of this thread's row.  The values may be used after tmem_wait_ld() and keep() only.
__device__ __forceinline__ void tmem_ld32(float *v, u32 at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
        "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]),
        "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void keep(float *v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
               "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])::"memory");
  asm volatile("" : "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]),
               "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])::"memory");
}
__device__ __forceinline__ void tmem_st32(u32 at, const u32 *v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]),
      "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]),
      "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
// 16 columns, for where registers are short.
__device__ __forceinline__ void tmem_ld16(float *v, u32 at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
                 "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void keep16(float *v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
               "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])::"memory");
}
__device__ __forceinline__ void tmem_st16(u32 at, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]),
               "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ u32 load_acquire(const u32 *p) {
  u32 v;
  asm volatile("ld.acquire.gpu.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}

// two 32-bit numbers to an instruction
typedef u64 f32x2;
__device__ __forceinline__ f32x2 pack_f32(float lo, float hi) {
  f32x2 v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ void unpack_f32(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 fma_f32x2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ f32x2 add_f32x2(f32x2 a, f32x2 b) {
  f32x2 v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}

template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

}  // namespace paged
}  // namespace gorio
