// The 8-bit product on tiles of up to 256 tokens x 256 weight rows, for many tokens.  4096 x 131072 x 4096 1745 - 1870 us (2.35 - 2.5 POP/s, by the card),
// 4096 x 14336 x 4096 201 - 215 (3.5 rounds of tiles, which take four), 333 x 50257 x 1971 61 - 65.
//
// What bounds it: the matrix cores (random codes draw so much power that the matrix instructions alone reach 3.3 of their 4.9 POP/s; LDS reads take a
// seventh of the cycles by the counters).  Four waves of 128 x 128 outputs, one per SIMD, so that nothing hides a stall:
// a chunk of 128 k is one asm block, in which matrix instructions, fragment reads of the next k-step, loads into LDS and the arithmetic of
// their addresses alternate; between blocks there is what it takes to step one cursor.
//   * LDS (all 160 KB): two slots of 256 token rows x 128 k, three of weight rows, which come from further away; rows of 128 bytes, the 16-byte
//     column c of row r at c ^ (r / 2) % 8.  Block kt loads chunk kt + 2 of the weights under its first three k-steps, and of the tokens behind its
//     barrier, which says that chunk kt + 1 has landed and that the tokens' slot of chunk kt has been read.
//   * The chunks of all tiles of a workgroup form one stream: the cursor is in the next tile while the last two chunks of a tile are multiplied.
//   * Weight row n of a wave's 128 sits in LDS row (n % 4) 32 + n / 4: a lane then ends up with four neighbouring outputs of a token, one store
//     instead of four.
//   * An XCD has a contiguous range of the tiles, ordered so that the 32 that run at a time are about 8 token tiles x 4 panels: the operands
//     that its L2 has to fetch are the fewest so.
//   * Codes behind K: whole vectors of 16 bytes are not loaded.  The rest of K % 16 codes is added by one k-step of its own, masked.
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "groups.h"
#include "int8_device.h"
#include "unaligned.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(16))) int i32x16;

constexpr int kThreadsW = 256;
constexpr int kPanelGroup = 4;          // panels that are run side by side
constexpr int kRowB = 128, kSlotB = 256 * kRowB;
constexpr int kTokenSlots = 2, kWeightSlots = 3, kLds = (kTokenSlots + kWeightSlots) * kSlotB;
static_assert(kLds == 163840, "all of a CU's LDS");
constexpr int kIns = 8;                 // loads of a wave per chunk and operand
constexpr int kMinChunks = 3;           // of a tile, so that the cursor never runs past the next one

struct Tile { int valid, m0, rows, n0, cols; };
struct Frags { i32x4 a[4], b[4]; };     // of one k-step: token rows, weight rows

// What a block needs beside the accumulators and fragments.  *_row: LDS addresses of the wave's first rows in the slots of this chunk and the next;
// to_*: of this wave's part of the slots that are loaded; k: bytes from a row's start to the loaded chunk.
struct Block { i32x4 rs_a, rs_b; unsigned a_row, b_row, a_next, b_next, to_a, to_b, k; };

#define MF(i, j, A, B) "v_mfma_i32_32x32x32_i8 %[c" #i #j "], %[" #A #i "], %[" #B #j "], %[c" #i #j "]\n\t"
#define MF4(i, A, B) MF(i, 0, A, B) MF(i, 1, A, B) MF(i, 2, A, B) MF(i, 3, A, B)
// the fragment addresses of k-step k of the chunk whose rows lie at RA / RB
#define AT(k, RA, RB) "v_add_u32 %[pa], %[" #RA "], %[col" #k "]\n\tv_add_u32 %[pb], %[" #RB "], %[col" #k "]\n\t"
#define RA(X, i) "ds_read_b128 %[" #X #i "], %[pa] offset:%[o" #i "]\n\t"
#define RB(Y, j) "ds_read_b128 %[" #Y #j "], %[pb] offset:%[o" #j "]\n\t"
#define LA(l) "s_add_u32 m0, %[ta], " #l "*1024\n\ts_nop 0\n\tbuffer_load_dwordx4 %[ao" #l "], %[ra], %[k] offen lds\n\t"
#define LB(l) "s_add_u32 m0, %[tb], " #l "*1024\n\ts_nop 0\n\tbuffer_load_dwordx4 %[bo" #l "], %[rb], %[k] offen lds\n\t"
#define DONE "s_waitcnt lgkmcnt(0)\n\t"
// in flight behind chunk kt + 1: the weights of chunk kt + 2
#define BARRIER "s_waitcnt vmcnt(8)\n\ts_barrier\n\t"
// the compiler does not see what a block holds: wait states between its vector instructions and matrix instructions
#define START "s_nop 4\n\t"

// k-step on fragments A, B; X, Y get those of k-step k; three loads
#define STEP4(A, B, X, Y, k, L0, L1, L2) AT(k, ra0, rb0) MF(0, 0, A, B) RB(Y, 0) MF(0, 1, A, B) RB(Y, 1) MF(0, 2, A, B) RB(Y, 2) L0 MF(0, 3, A, B) RB(Y, 3) \
  MF(1, 0, A, B) RA(X, 0) MF(1, 1, A, B) RA(X, 1) L1 MF(1, 2, A, B) RA(X, 2) MF(1, 3, A, B) RA(X, 3) MF(2, 0, A, B) L2 MF(2, 1, A, B) MF(2, 2, A, B) MF(2, 3, A, B) MF4(3, A, B) DONE
#define STEP3(A, B, X, Y, k, L0, L1, L2) AT(k, ra0, rb0) MF(0, 0, A, B) RB(Y, 0) MF(0, 1, A, B) RB(Y, 1) MF(0, 2, A, B) RB(Y, 2) L0 MF(0, 3, A, B) RB(Y, 3) \
  MF(1, 0, A, B) RA(X, 0) MF(1, 1, A, B) RA(X, 1) L1 MF(1, 2, A, B) RA(X, 2) MF(1, 3, A, B) L2 MF4(2, A, B) DONE
#define STEP2(A, B, X, Y, k, L0, L1, L2) AT(k, ra0, rb0) MF(0, 0, A, B) RB(Y, 0) RB(Y, 1) MF(0, 1, A, B) RB(Y, 2) RB(Y, 3) MF(0, 2, A, B) RA(X, 0) L0 MF(0, 3, A, B) RA(X, 1) \
  MF(1, 0, A, B) L1 MF(1, 1, A, B) L2 MF(1, 2, A, B) MF(1, 3, A, B) DONE
// the last k-step of a chunk; X, Y get the first of the next chunk
#define LAST4(A, B, X, Y) AT(0, ran, rbn) MF4(0, A, B) BARRIER MF(1, 0, A, B) RB(Y, 0) RB(Y, 1) MF(1, 1, A, B) RB(Y, 2) RB(Y, 3) MF(1, 2, A, B) RA(X, 0) RA(X, 1) MF(1, 3, A, B) \
  RA(X, 2) RA(X, 3) MF(2, 0, A, B) LA(0) MF(2, 1, A, B) LA(1) MF(2, 2, A, B) LA(2) MF(2, 3, A, B) LA(3) MF(3, 0, A, B) LA(4) MF(3, 1, A, B) LA(5) MF(3, 2, A, B) LA(6) MF(3, 3, A, B) LA(7) DONE
#define LAST3(A, B, X, Y) AT(0, ran, rbn) MF4(0, A, B) BARRIER MF(1, 0, A, B) RB(Y, 0) RB(Y, 1) MF(1, 1, A, B) RB(Y, 2) RB(Y, 3) MF(1, 2, A, B) RA(X, 0) RA(X, 1) MF(1, 3, A, B) \
  RA(X, 2) LA(0) LA(1) MF(2, 0, A, B) LA(2) LA(3) MF(2, 1, A, B) LA(4) MF(2, 2, A, B) LA(5) MF(2, 3, A, B) LA(6) LA(7) DONE
#define LAST2(A, B, X, Y) AT(0, ran, rbn) MF4(0, A, B) BARRIER MF(1, 0, A, B) RB(Y, 0) RB(Y, 1) RB(Y, 2) RB(Y, 3) MF(1, 1, A, B) RA(X, 0) RA(X, 1) LA(0) LA(1) MF(1, 2, A, B) \
  LA(2) LA(3) LA(4) MF(1, 3, A, B) LA(5) LA(6) LA(7) DONE
#define CHUNK(N) START STEP##N(p, q, u, w, 1, LB(0), LB(1), LB(2)) STEP##N(u, w, p, q, 2, LB(3), LB(4), LB(5)) STEP##N(p, q, u, w, 3, LB(6), LB(7), "") LAST##N(u, w, p, q)

#define C1(i, j) [c##i##j] "+a"(c[i][j])
#define C4(i) C1(i, 0), C1(i, 1), C1(i, 2), C1(i, 3)
#define FA(i) [p##i] "+v"(f.a[i]), [u##i] "=&v"(g.a[i])
#define FB(j) [q##j] "+v"(f.b[j]), [w##j] "=&v"(g.b[j])
#define ADDRESSES [pa] "=&v"(pa), [pb] "=&v"(pb)
#define OFFS [o0] "n"(0), [o1] "n"(32 * kRowB), [o2] "n"(64 * kRowB), [o3] "n"(96 * kRowB)
#define COLS [col0] "v"(col[0]), [col1] "v"(col[1]), [col2] "v"(col[2]), [col3] "v"(col[3])
#define ROWS [ra0] "s"(s.a_row), [rb0] "s"(s.b_row), [ran] "s"(s.a_next), [rbn] "s"(s.b_next), [ta] "s"(s.to_a), [tb] "s"(s.to_b), [k] "s"(s.k), [ra] "s"(s.rs_a), [rb] "s"(s.rs_b)
#define AO(l) [ao##l] "v"(ao[l]), [bo##l] "v"(bo[l])
#define INPUTS COLS, ROWS, OFFS, AO(0), AO(1), AO(2), AO(3), AO(4), AO(5), AO(6), AO(7)

// One chunk: f holds the fragments of its first k-step and gets those of the next chunk's.
template <int NB>
__device__ __forceinline__ void chunk(i32x16 (&c)[4][4], Frags& f, const unsigned (&col)[4], const unsigned (&ao)[kIns], const unsigned (&bo)[kIns], const Block& s) {
  Frags g;
  unsigned pa, pb;
  if constexpr (NB == 4)
    asm volatile(CHUNK(4) : C4(0), C4(1), C4(2), C4(3), FA(0), FA(1), FA(2), FA(3), FB(0), FB(1), FB(2), FB(3), ADDRESSES : INPUTS : "memory", "scc");
  else if constexpr (NB == 3)
    asm volatile(CHUNK(3) : C4(0), C4(1), C4(2), FA(0), FA(1), FA(2), FB(0), FB(1), FB(2), FB(3), ADDRESSES : INPUTS : "memory", "scc");
  else
    asm volatile(CHUNK(2) : C4(0), C4(1), FA(0), FA(1), FB(0), FB(1), FB(2), FB(3), ADDRESSES : INPUTS : "memory", "scc");
}
// Matrix results are readable behind this, and the compiler moves none of them in front of it.
template <int NB>
__device__ __forceinline__ void settle(i32x16 (&c)[4][4]) {
#define SETTLE "s_nop 15\n\ts_nop 7"
  if constexpr (NB == 4) asm volatile(SETTLE : C4(0), C4(1), C4(2), C4(3));
  else if constexpr (NB == 3) asm volatile(SETTLE : C4(0), C4(1), C4(2));
  else asm volatile(SETTLE : C4(0), C4(1));
#undef SETTLE
}
// The first fragments: nothing to multiply yet.  In flight behind chunk 0: the weights of chunk 1.
template <int NB>
__device__ __forceinline__ void first_frags(Frags& f, unsigned pa, unsigned pb) {
#define READS BARRIER RB(q, 0) RB(q, 1) RB(q, 2) RB(q, 3)
#define QB [q0] "=&v"(f.b[0]), [q1] "=&v"(f.b[1]), [q2] "=&v"(f.b[2]), [q3] "=&v"(f.b[3])
#define PA(i) [p##i] "=&v"(f.a[i])
#define FROM [pa] "v"(pa), [pb] "v"(pb), OFFS
  if constexpr (NB == 4) asm volatile(READS RA(p, 0) RA(p, 1) RA(p, 2) RA(p, 3) DONE : QB, PA(0), PA(1), PA(2), PA(3) : FROM : "memory");
  else if constexpr (NB == 3) asm volatile(READS RA(p, 0) RA(p, 1) RA(p, 2) DONE : QB, PA(0), PA(1), PA(2) : FROM : "memory");
  else asm volatile(READS RA(p, 0) RA(p, 1) DONE : QB, PA(0), PA(1) : FROM : "memory");
}
__device__ __forceinline__ void load_one(i32x4 rs, unsigned vo, unsigned so, unsigned md) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" :: "v"(vo), "s"(rs), "s"(so), "s"(md) : "memory");
}
// one k-step without reads and loads
template <int NB>
__device__ __forceinline__ void multiply(i32x16 (&c)[4][4], const i32x4 (&fa)[4], const i32x4 (&fb)[4]) {
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      asm volatile("s_nop 4\n\tv_mfma_i32_32x32x32_i8 %0, %1, %2, %0" : "+a"(c[i][j]) : "v"(fa[i]), "v"(fb[j]));
}
__device__ __forceinline__ int acc_read(const i32x16& c, int v) {
  int x;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c[v]));
  return x;
}
__device__ __forceinline__ i32x4 rsrc4(const void* p, unsigned bytes) {
  const uint64_t v = (uint64_t)p;
  return i32x4{uniform((int)(unsigned)v), uniform((int)(unsigned)(v >> 32)), uniform((int)bytes), 0x00020000};
}
// Size that a descriptor states.  The hardware takes the scalar offset from it before it compares, and the cursor's goes on behind a row that is
// shorter than its chunks, by up to kMinChunks of them; that difference must not go below zero.  Lanes with data lie inside the tensor by
// themselves (rows and columns are checked), so stating more than a short tensor has lets nothing through.
constexpr unsigned stated(unsigned bytes) { return bytes < kMinChunks * kRowB ? kMinChunks * kRowB : bytes; }

// Waves in a 2 x 2 grid, each NB (2, 3 or 4) blocks of 32 tokens x 128 weight rows: tiles of 64 NB tokens.
template <typename S, int NB>
__global__ __launch_bounds__(kThreadsW) __attribute__((amdgpu_waves_per_eu(1, 1))) void int8_wide_kernel(const Int8Args a, const int mt, const int panels) {
  constexpr int kHeight = 64 * NB;
  extern __shared__ __attribute__((aligned(1024))) char s_ring[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), h = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  const unsigned lds0 = (unsigned)(size_t)s_ring;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, nslots = gridDim.x >> 3;
  const int total = mt * panels;
  const int first_tile = (int)((int64_t)total * xcd / 8), end_tile = (int)((int64_t)total * (xcd + 1) / 8);
  const int K16 = a.K16;
  const int nk = max((K16 + kRowB - 1) / kRowB, kMinChunks);

  auto tile_at = [&](int i) -> Tile {
    Tile T = {};
    const int v = first_tile + i * nslots + slot;
    T.valid = v < end_tile;
    if (!T.valid) return T;
    const int g = v / (kPanelGroup * mt), r = v - g * (kPanelGroup * mt), pg = min(kPanelGroup, panels - g * kPanelGroup);
    const int m = r / pg;
    T.m0 = uniform(m * kHeight);
    T.rows = uniform(min(a.T - T.m0, kHeight));
    T.n0 = uniform((g * kPanelGroup + r - m * pg) * 256);
    T.cols = uniform(min(a.N - T.n0, 256));
    return T;
  };
  int ord = 0;
  Tile cur = tile_at(ord++);
  if (!cur.valid) return;
  Tile nx = tile_at(ord++);

  // ---- the cursor: chunk k / 128 of a tile, or of the next ----
  Block s;
  unsigned ao[kIns], bo[kIns];
  int left = 0;
  const int pc = lane & 7, sub = lane >> 3;
  auto col_of = [&](int p) { return (unsigned)(pc ^ (((p & 1) * 4 + (lane >> 4)) & 7)) * 16u; };
  auto tail = [&]() {                                      // columns behind K16; kOob is the top bit
#pragma unroll
    for (int p = 0; p < kIns; ++p) {
      const unsigned out = (unsigned)((int)s.k + (int)col_of(p) >= K16) << 31;
      ao[p] |= out;
      bo[p] |= out;
    }
  };
  auto open = [&](const Tile& T) {
    s.rs_a = rsrc4(a.x + (T.valid ? (int64_t)T.m0 * a.ldx : 0), stated(T.valid ? (unsigned)((T.rows - 1) * (int)a.ldx + K16) : 0u));
    s.rs_b = rsrc4(a.w + (T.valid ? (int64_t)T.n0 * a.ldw : 0), stated(T.valid ? (unsigned)((T.cols - 1) * (int)a.ldw + K16) : 0u));
    s.k = 0;
    left = T.valid ? nk : 0x7fffffff;
#pragma unroll
    for (int p = 0; p < kIns; ++p) {
      const int r = wave * 64 + 8 * p + sub, n = (r & 128) + 4 * (r & 31) + ((r >> 5) & 3);
      ao[p] = ((unsigned)r * (unsigned)a.ldx + col_of(p)) | ((unsigned)(!T.valid || r >= T.rows) << 31);
      bo[p] = ((unsigned)n * (unsigned)a.ldw + col_of(p)) | ((unsigned)(!T.valid || n >= T.cols) << 31);
    }
    if (K16 < kRowB) tail();
  };
  auto step = [&]() {
    left = uniform(left - 1);
    if (left == 0) open(nx);
    else { s.k = uniform(s.k + kRowB); if (uniform(K16 - (int)s.k) < kRowB) tail(); }
  };
  open(cur);

  // LDS addresses of this wave's rows and of its part of a load; the slots of chunks kt, kt + 1, kt + 2
  const unsigned a_at = uniform(lds0 + wm * NB * 32 * kRowB), b_at = uniform(lds0 + kTokenSlots * kSlotB + wn * 128 * kRowB);
  const unsigned a_to = uniform(lds0 + wave * kIns * 1024), b_to = uniform(lds0 + kTokenSlots * kSlotB + wave * kIns * 1024);
  unsigned slot_a = 0, b0 = 0, b1 = kSlotB, b2 = 2 * kSlotB;
  // ---- fill: chunk 0; of chunk 1 the weights, then, behind the first fragments, the tokens ----
#pragma unroll
  for (int l = 0; l < kIns; ++l) load_one(s.rs_b, bo[l], s.k, b_to + b0 + l * 1024);
#pragma unroll
  for (int l = 0; l < kIns; ++l) load_one(s.rs_a, ao[l], s.k, a_to + l * 1024);
  step();
#pragma unroll
  for (int l = 0; l < kIns; ++l) load_one(s.rs_b, bo[l], s.k, b_to + b1 + l * 1024);

  const unsigned fkey = (unsigned)((lane & 31) >> 1) & 7u;
  unsigned col[4];                                         // of a lane's 16 bytes of k-step k, behind the wave's first row
#pragma unroll
  for (int k = 0; k < 4; ++k) col[k] = (unsigned)((lane & 31) * kRowB) + ((unsigned)(2 * k + h) ^ fkey) * 16u;
  Frags f;
  i32x16 acc[4][4];
  first_frags<NB>(f, col[0] + a_at, col[0] + b_at);
#pragma unroll
  for (int l = 0; l < kIns; ++l) load_one(s.rs_a, ao[l], s.k, a_to + kSlotB + l * 1024);
  step();

  // Scales of this lane's outputs and of the wave's token rows (rows lane and lane + 64).  Loads end in order, so those of the next tile are issued in
  // front of this tile's stores and awaited behind them: nowhere does a wait for them stop the loads into LDS.
  const int n_l = wn * 128 + 4 * (lane & 31);
  struct Scales { float w[4], bias[4], x[2]; };
  auto scales_of = [&](const Tile& T) {
    Scales c;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = min(T.n0 + n_l + j, a.N - 1);
      c.w[j] = a.w_scale[n];
      c.bias[j] = a.bias ? a.bias[n] : kNoBias;
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) c.x[q] = a.x_scale[min(T.m0 + wm * NB * 32 + q * 64 + lane, a.T - 1)];
    asm volatile("" ::: "memory");
    return c;
  };
  auto await = [&](Scales& c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(c.w[j]), "+v"(c.bias[j]));
    asm volatile("" : "+v"(c.x[0]), "+v"(c.x[1]));
  };
  Scales sc = scales_of(cur);
  await(sc);
  for (;;) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    for (int kt = 0; kt < nk; ++kt) {
      s.a_row = a_at + slot_a; s.b_row = b_at + b0;
      s.to_a = a_to + slot_a; s.to_b = b_to + b2;
      slot_a ^= kSlotB;
      s.a_next = a_at + slot_a; s.b_next = b_at + b1;
      chunk<NB>(acc, f, col, ao, bo, s);
      const unsigned b = b0;
      b0 = b1; b1 = b2; b2 = b;
      step();
    }
    if (a.k_tail) {
      // the last K % 16 codes, in the lanes of the first half
      i32x4 ta[4], tb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ta[i] = tb[i] = i32x4{0, 0, 0, 0};
        if (i < NB && h == 0) ta[i] = masked_codes(a.x + (int64_t)min(cur.m0 + (wm * NB + i) * 32 + (lane & 31), a.T - 1) * a.ldx + K16, a.k_tail);
        if (h == 0) tb[i] = *reinterpret_cast<const i32x4*>(a.w + (int64_t)min(cur.n0 + n_l + i, a.N - 1) * a.ldw + K16);
      }
      multiply<NB>(acc, ta, tb);
    }
    settle<NB>(acc);
    // ---- epilogue: accumulator v of lane l is row 8*(v/4) + 4*(l/32) + v%4, output 4*(l%32) + j ----
    Scales next = scales_of(nx);
    const int row_w = wm * NB * 32;
    const bool whole = cur.cols == 256 && cur.rows == kHeight;
    char* out_r = static_cast<char*>(a.out) + ((int64_t)(cur.m0 + row_w) * a.ldo + cur.n0) * sizeof(S);
    const unsigned lane_off = ((unsigned)(4 * h) * (unsigned)a.ldo + (unsigned)n_l) * (unsigned)sizeof(S);
    auto store = [&](auto whole_tag) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          __builtin_amdgcn_sched_barrier(0);
          const int r = i * 32 + 8 * (v >> 2) + (v & 3);   // + 4 h
          const float s0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc.x[r >> 6]), r & 63));
          const float s1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sc.x[r >> 6]), (r & 63) + 4));
          const float xs = h ? s1 : s0;
          Unaligned<S, 4> o;
#pragma unroll
          for (int j = 0; j < 4; ++j) o.v[j] = to_out<S>(scaled(acc_read(acc[i][j], v), xs, sc.w[j], sc.bias[j]));
          S* const p = reinterpret_cast<S*>(out_r + (int64_t)r * a.ldo * (int)sizeof(S) + lane_off);
          if constexpr (decltype(whole_tag)::value) {
            *reinterpret_cast<Unaligned<S, 4>*>(p) = o;
          } else if (row_w + r + 4 * h < cur.rows) {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (n_l + j < cur.cols) p[j] = o.v[j];
          }
        }
    };
    if (whole) { store(std::true_type{}); await(next); } else { store(std::false_type{}); await(next); }
    sc = next;
    cur = nx;
    if (!cur.valid) break;
    nx = tile_at(ord++);
  }
  // the loads behind the last chunk only fill LDS with zeros; they end before the workgroup does
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <typename S, int NB>
int launch_t(const Int8Args& a, hipStream_t s) {
  static std::atomic<int> ready{0};
  if (!ready.load(std::memory_order_relaxed)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_wide_kernel<S, NB>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess)
      return hip_fail(hipGetLastError(), "int8_wide_kernel: LDS size attribute");
    ready.store(1, std::memory_order_relaxed);
  }
  int grid = device_cu_count() / 8 * 8;
  if (grid < 8) grid = 8;                                   // a multiple of the 8 XCDs
  hipLaunchKernelGGL((int8_wide_kernel<S, NB>), dim3((unsigned)grid), dim3(kThreadsW), kLds, s, a, (a.T + 64 * NB - 1) / (64 * NB), (a.N + 255) / 256);
  return hip_fail(hipGetLastError(), "int8_wide_kernel launch");
}
template <typename S>
int launch_n(const Int8Args& a, int blocks, hipStream_t s) {
  if (blocks == 4) return launch_t<S, 4>(a, s);
  return blocks == 3 ? launch_t<S, 3>(a, s) : launch_t<S, 2>(a, s);
}

}  // namespace

int launch_int8_wide(const Int8Args& a, int blocks, hipStream_t s) { return a.out_dtype == MOE_FP32 ? launch_n<float>(a, blocks, s) : launch_n<uint16_t>(a, blocks, s); }

}  // namespace mm
