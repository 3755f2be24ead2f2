// Pieces shared by the token operators' kernels: copies from memory that land in LDS, and their waits.
#pragma once
#include <utility>

#include "hb_device.hpp"

// On a lambda: inlined whatever its size, so that the arrays it captures stay in registers.
#define HB_INLINE __attribute__((always_inline))

namespace hb {

constexpr uint32_t kTkOutside = 0x80000000u;              // offset beyond any descriptor used here: arrives as zeros

template <int I>
struct TkInt {
    static constexpr int value = I;
};
template <class F, int... J>
__device__ __forceinline__ void tk_each(F f, std::integer_sequence<int, J...>) {
    (f(TkInt<J>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void tk_for(F f) {             // f(TkInt<0>{}) .. f(TkInt<N - 1>{})
    tk_each(f, std::make_integer_sequence<int, N>{});
}

__device__ __forceinline__ uint32_t tk_lds_addr(const void* p) {
    return (uint32_t)(size_t)(__attribute__((address_space(3))) const void*)p;
}
// A descriptor of the 2 GiB from `base` on.
__device__ __forceinline__ u32x4 tk_rsrc(const void* base) {
    const uint64_t b = (uint64_t)base;
    return u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
}
// The lanes copy 16 bytes each from the descriptor's base + voff (per lane) + soff to LDS at lds + 16 * lane.  Written as assembly so that
// the compiler does not make every LDS read wait for copies that are meant to stay in flight; the waits are explicit.  M0 is set in
// the same statement, and the build checks that nothing else in these kernels uses it.
__device__ __forceinline__ void tk_dma16(u32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(rsrc), "s"(soff), "s"(lds) : "memory");
}
// At most N memory instructions of this wave are outstanding afterwards.
template <int N>
__device__ __forceinline__ void tk_wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

}  // namespace hb
