// Direct loads from memory to LDS.
#pragma once
#include "delta_common.hpp"

namespace lrnnx {

// N times 16 bytes a lane (EACH = 4: four) from memory to LDS, a workgroup's from STEP to STEP, beside the lanes before.  Not the compiler's instruction for it: of that it takes every later read of LDS for
// one of what it brings, and waits for it (dh of 8192 x 2048, 32768 terms: 944 us so, 828); what has to be waited for is waited for where a stage changes hands.  There is no result in
// a register.  The descriptor may have come from the vector unit just now, which takes five instructions' time, m0 one.  m0 is named as written: without that the compiler takes a value of
// its own (of its LDS loads, of indexed registers) for still there.  Memory is not: other accesses of LDS may be moved over these, and only a wait and barrier that name memory, between a load and
// what reads its place or read it before, keep them apart.
template <int N, int STEP, int EACH = 16> __device__ __forceinline__ void load_lds(uint32_t to, const u32x4 &from, const uint32_t (&off)[N]) {
    static_assert(EACH == 16 ? N == 1 || N == 2 || N == 4 : EACH == 4 && N == 4, "");
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#define LOAD_FIRST_(load) "s_mov_b32 m0, %0\n\ts_nop 3\n\t" load " %2, %1, 0 offen lds"
#define LOAD_NEXT_(load, o, at) "\n\ts_add_u32 m0, m0, %" at "\n\ts_nop 0\n\t" load " %" o ", %1, 0 offen lds"
#define LOAD_FIRST LOAD_FIRST_("buffer_load_dwordx4")
#define LOAD_NEXT(o, at) LOAD_NEXT_("buffer_load_dwordx4", o, at)
#define ONE_NEXT(o, at) LOAD_NEXT_("buffer_load_dword", o, at)
    if constexpr (EACH == 4)
        asm volatile(LOAD_FIRST_("buffer_load_dword") ONE_NEXT("3", "6") ONE_NEXT("4", "6") ONE_NEXT("5", "6") ::"s"(to), "s"(from), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "n"(STEP) : "m0", "scc");
    else if constexpr (N == 1) asm volatile(LOAD_FIRST ::"s"(to), "s"(from), "v"(off[0]) : "m0");
    else if constexpr (N == 2) asm volatile(LOAD_FIRST LOAD_NEXT("3", "4") ::"s"(to), "s"(from), "v"(off[0]), "v"(off[1]), "n"(STEP) : "m0", "scc");
    else asm volatile(LOAD_FIRST LOAD_NEXT("3", "6") LOAD_NEXT("4", "6") LOAD_NEXT("5", "6") ::"s"(to), "s"(from), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "n"(STEP) : "m0", "scc");
#undef LOAD_FIRST_
#undef LOAD_NEXT_
#undef LOAD_FIRST
#undef LOAD_NEXT
#undef ONE_NEXT
#pragma clang diagnostic pop
}

}  // namespace lrnnx
