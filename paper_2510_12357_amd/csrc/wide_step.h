// One k-step of the 256 x 256 kernels (ffn_wide.hip, int8_wide.hip), as asm blocks.  A matrix instruction takes 16 bytes a lane of
// either operand, whatever the element; WIDE_MFMA, set by the includer, is its name.
#pragma once

#include "groups.h"
#include "wide_layout.h"

namespace mm {
namespace {

using namespace wide;

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int kA = 8, kB = 8;           // loads of a wave per token / weight chunk
constexpr int kLoads = (kA + kB) / 4;   // ... per k-step
constexpr int kLdsBytes = (SA + SB) * kSlotB;
constexpr int VM = kB + (SA - 2) * (kA + kB);   // loads in flight behind the awaited chunk
static_assert(SB > SA && kLdsBytes <= 163840, "ring");

// ---- one k-step: MFMAs on the current fragments, reads of the next ones, loads into LDS.  c: accumulators,
// a / b: fragments of the k-step, na / nb: of the next, at the LDS addresses pa / pb ----
struct Loads { i32x4 rs[4]; unsigned vo[4]; int so[4]; int md[4]; };

#define MF(i, j) WIDE_MFMA " %[c" #i #j "], %[a" #i "], %[b" #j "], %[c" #i #j "]\n\t"
#define RA(i) "ds_read_b128 %[na" #i "], %[pa] offset:%[oa" #i "]\n\t"
#define RB(j) "ds_read_b128 %[nb" #j "], %[pb] offset:%[ob" #j "]\n\t"
#define RQ(j) "ds_read_b128 %[nb" #j "], %[q" #j "] offset:%[ob" #j "]\n\t"
#define LD(l) "s_mov_b32 m0, %[md" #l "]\n\ts_nop 0\n\tbuffer_load_dwordx4 %[vo" #l "], %[rs" #l "], %[so" #l "] offen lds\n\t"
#define BAR "s_waitcnt vmcnt(%[vm])\n\ts_barrier\n\t"
// the compiler does not see what the block holds: wait states between its vector instructions and the
// matrix instructions (2), and between its scalar results and the loads that use them (5)
#define START "s_nop 4\n\t"
#define END "s_waitcnt lgkmcnt(0)"
#define C1(i, j) [c##i##j] "+a"(c[i][j])
#define C4(i) C1(i, 0), C1(i, 1), C1(i, 2), C1(i, 3)
#define NA(i) [na##i] "=&v"(na[i])
#define NB_(j) [nb##j] "=&v"(nb[j])
#define IA(i) [a##i] "v"(fa[i])
#define IB(j) [b##j] "v"(fb[j])
#define LOADS4 [rs0] "s"(L.rs[0]), [rs1] "s"(L.rs[1]), [rs2] "s"(L.rs[2]), [rs3] "s"(L.rs[3]), \
  [vo0] "v"(L.vo[0]), [vo1] "v"(L.vo[1]), [vo2] "v"(L.vo[2]), [vo3] "v"(L.vo[3]), \
  [so0] "s"(L.so[0]), [so1] "s"(L.so[1]), [so2] "s"(L.so[2]), [so3] "s"(L.so[3]), \
  [md0] "s"(L.md[0]), [md1] "s"(L.md[1]), [md2] "s"(L.md[2]), [md3] "s"(L.md[3])
#define OFFS [oa0] "n"(0), [oa1] "n"(kBlock * kRowB), [oa2] "n"(2 * kBlock * kRowB), [oa3] "n"(3 * kBlock * kRowB)
#define OB(j) [ob##j] "n"(b_frag_row(GU, j) * kRowB)
#define OFFB OB(0), OB(1), OB(2), OB(3)
// addresses of the weight fragments of the next tile's first k-step: pq for those that a narrow tile has no use for
#define QB(j) [q##j] "v"(j == 0 || j == second_frag(GU) ? pb : pq)
#define NEXT QB(0), QB(1), QB(2), QB(3), [vm] "n"(VM)
#define NALL NA(0), NA(1), NA(2), NA(3), NB_(0), NB_(1), NB_(2), NB_(3)
#define IN4 IA(0), IA(1), IA(2), IA(3), IB(0), IB(1), IB(2), IB(3)
#define REST [pa] "v"(pa), [pb] "v"(pb), LOADS4, OFFS, OFFB
// the reads behind the barrier fetch all eight fragments, whatever shape the next tile has (b_row_of)
#define RDALL RQ(0) RQ(1) RQ(2) RQ(3) RA(0) RA(1) RA(2) RA(3)

#define C2J(i, J) C1(i, 0), C1(i, J)
#define NARROW_STEPS(J)                                                                                                  \
  if constexpr (NB == 4) {                                                                                               \
    if constexpr (!BARRIER)                                                                                              \
      asm volatile(START MF(0,0) RB(0) RB(J) MF(0,J) RA(0) LD(0) MF(1,0) RA(1) RA(2) MF(1,J) RA(3) LD(1) MF(2,0) MF(2,J) LD(2) MF(3,0) LD(3) MF(3,J) END \
                   : C2J(0, J), C2J(1, J), C2J(2, J), C2J(3, J), NA(0), NA(1), NA(2), NA(3), NB_(0), NB_(J)                \
                   : IA(0), IA(1), IA(2), IA(3), IB(0), IB(J), REST : "memory");                                          \
    else                                                                                                                 \
      asm volatile(START MF(0,0) MF(0,J) BAR MF(1,0) RDALL MF(1,J) LD(0) MF(2,0) LD(1) MF(2,J) LD(2) MF(3,0) LD(3) MF(3,J) END \
                   : C2J(0, J), C2J(1, J), C2J(2, J), C2J(3, J), NALL                                                     \
                   : IA(0), IA(1), IA(2), IA(3), IB(0), IB(J), REST, NEXT : "memory");                            \
  } else if constexpr (NB == 3) {                                                                                        \
    if constexpr (!BARRIER)                                                                                              \
      asm volatile(START MF(0,0) RB(0) RB(J) MF(0,J) RA(0) LD(0) MF(1,0) RA(1) RA(2) MF(1,J) LD(1) MF(2,0) LD(2) LD(3) MF(2,J) END \
                   : C2J(0, J), C2J(1, J), C2J(2, J), NA(0), NA(1), NA(2), NB_(0), NB_(J)                                  \
                   : IA(0), IA(1), IA(2), IB(0), IB(J), REST : "memory");                                                 \
    else                                                                                                                 \
      asm volatile(START MF(0,0) MF(0,J) BAR MF(1,0) RDALL MF(1,J) LD(0) LD(1) MF(2,0) LD(2) LD(3) MF(2,J) END           \
                   : C2J(0, J), C2J(1, J), C2J(2, J), NALL                                                                \
                   : IA(0), IA(1), IA(2), IB(0), IB(J), REST, NEXT : "memory");                                   \
  } else if constexpr (NB == 2) {                                                                                        \
    if constexpr (!BARRIER)                                                                                              \
      asm volatile(START MF(0,0) RB(0) RB(J) MF(0,J) RA(0) RA(1) LD(0) MF(1,0) LD(1) LD(2) MF(1,J) LD(3) END             \
                   : C2J(0, J), C2J(1, J), NA(0), NA(1), NB_(0), NB_(J)                                                   \
                   : IA(0), IA(1), IB(0), IB(J), REST : "memory");                                                        \
    else                                                                                                                 \
      asm volatile(START MF(0,0) MF(0,J) BAR MF(1,0) RDALL MF(1,J) LD(0) LD(1) LD(2) LD(3) END                           \
                   : C2J(0, J), C2J(1, J), NALL                                                                           \
                   : IA(0), IA(1), IB(0), IB(J), REST, NEXT : "memory");                                          \
  } else {                                                                                                               \
    if constexpr (!BARRIER)                                                                                              \
      asm volatile(START MF(0,0) RB(0) RB(J) RA(0) MF(0,J) LD(0) LD(1) LD(2) LD(3) END                                   \
                   : C2J(0, J), NA(0), NB_(0), NB_(J)                                                                     \
                   : IA(0), IB(0), IB(J), REST : "memory");                                                               \
    else                                                                                                                 \
      asm volatile(START MF(0,0) MF(0,J) BAR RDALL LD(0) LD(1) LD(2) LD(3) END                                           \
                   : C2J(0, J), NALL                                                                                      \
                   : IA(0), IB(0), IB(J), REST, NEXT : "memory");                                                 \
  }

// GU: gate/up.  Tiles of more than 128 tokens: waves in a 2 x 2 grid, NB x 4 matrix tiles each.  Narrower
// ones: the waves split the weight rows four ways, NB x 2 tiles each (weight fragments 0 and
// second_frag).  pq: as pb, from the row b_row_of of the other two fragments on.
template <bool TALL, int NB, bool GU, bool BARRIER, typename Acc, typename Frag>
__device__ __forceinline__ void kstep(Acc (&c)[4][4], const Frag (&fa)[4], const Frag (&fb)[4], Frag (&na)[4],
                                      Frag (&nb)[4], unsigned pa, unsigned pb, unsigned pq, const Loads& L) {
  if constexpr (TALL && NB == 4) {
    if constexpr (!BARRIER)
      asm volatile(START MF(0,0) RB(0) MF(0,1) RB(1) MF(0,2) RB(2) LD(0) MF(0,3) RB(3) MF(1,0) RA(0) MF(1,1) RA(1) LD(1) MF(1,2) RA(2) MF(1,3) RA(3)
                   MF(2,0) LD(2) MF(2,1) MF(2,2) MF(2,3) MF(3,0) LD(3) MF(3,1) MF(3,2) MF(3,3) END
                   : C4(0), C4(1), C4(2), C4(3), NALL : IN4, REST : "memory");
    else
      asm volatile(START MF(0,0) MF(0,1) MF(0,2) MF(0,3) BAR MF(1,0) RQ(0) RQ(1) MF(1,1) RQ(2) RQ(3) MF(1,2) RA(0) RA(1) MF(1,3) RA(2) RA(3)
                   MF(2,0) LD(0) MF(2,1) MF(2,2) LD(1) MF(2,3) MF(3,0) LD(2) MF(3,1) MF(3,2) LD(3) MF(3,3) END
                   : C4(0), C4(1), C4(2), C4(3), NALL : IN4, REST, NEXT : "memory");
  } else if constexpr (TALL && NB == 3) {
    if constexpr (!BARRIER)
      asm volatile(START MF(0,0) RB(0) MF(0,1) RB(1) MF(0,2) RB(2) LD(0) MF(0,3) RB(3) MF(1,0) RA(0) MF(1,1) RA(1) LD(1) MF(1,2) RA(2) MF(1,3)
                   MF(2,0) LD(2) MF(2,1) MF(2,2) LD(3) MF(2,3) END
                   : C4(0), C4(1), C4(2), NA(0), NA(1), NA(2), NB_(0), NB_(1), NB_(2), NB_(3)
                   : IA(0), IA(1), IA(2), IB(0), IB(1), IB(2), IB(3), REST : "memory");
    else
      asm volatile(START MF(0,0) MF(0,1) MF(0,2) MF(0,3) BAR MF(1,0) RQ(0) RQ(1) MF(1,1) RQ(2) RQ(3) MF(1,2) RA(0) RA(1) MF(1,3) RA(2) RA(3)
                   MF(2,0) LD(0) MF(2,1) LD(1) MF(2,2) LD(2) MF(2,3) LD(3) END
                   : C4(0), C4(1), C4(2), NALL : IA(0), IA(1), IA(2), IB(0), IB(1), IB(2), IB(3), REST, NEXT : "memory");
  } else if constexpr (second_frag(GU) == 2) {
    NARROW_STEPS(2)
  } else {
    NARROW_STEPS(1)
  }
}
#undef NARROW_STEPS

// first fragments: nothing to multiply yet
template <bool GU, typename Frag>
__device__ __forceinline__ void first_frags(Frag (&na)[4], Frag (&nb)[4], unsigned pa, unsigned pb, unsigned pq) {
  asm volatile(BAR RDALL END : NALL : [pa] "v"(pa), OFFS, OFFB, NEXT : "memory");
}
__device__ __forceinline__ void load_one(i32x4 rs, unsigned vo, int so, int md) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" :: "v"(vo), "s"(rs), "s"(so), "s"(md) : "memory");
}

__device__ __forceinline__ i32x4 rsrc4(const void* p, unsigned bytes) {
  const uint64_t v = (uint64_t)p;
  return i32x4{uniform((int)(unsigned)v), uniform((int)(unsigned)(v >> 32)), uniform((int)bytes), 0x00020000};
}

// one accumulator out of the matrix registers: read where it is used, so that no more than the
// few values being stored sit in ordinary registers
template <typename Acc>
__device__ __forceinline__ auto acc_read(const Acc& c, int v) -> decltype(c[0] + c[0]) {
  decltype(c[0] + c[0]) x;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c[v]));
  return x;
}

}  // namespace
}  // namespace mm
