// The 8-bit product on tiles of 64 tokens x 64 or 128 weight rows: more tokens than the streaming kernel takes, and too few tiles of
// 256 x 256 to fill the chip.
//
// Four waves in a 2 x 2 grid; chunks of 128 k in a ring of LDS, filled past the registers.  One workgroup per CU of eight waves: two groups with
// a ring each share K, and their sums of integers are joined in LDS, exactly; 64 x 64 in five stages, 64 x 128 in three.  Or several workgroups per CU of
// four: three of 64 x 64 in three stages, two of 64 x 128 in three, five of 64 x 64 in two stages where K is short.
// What bounds it is the way of a chunk from memory: a CU has as much of it under way as its LDS holds, so that small tiles beat the lower traffic of
// larger ones as long as all tiles are under way at once (65 x 2048 x 2048: 64 columns 7.2 us, 128 columns 9.3; 500 x 2048 x 2048 8.4 and
// 11.0), and two groups halve the number of chunks that follow each other.
// A chunk is one asm block: matrix instructions, the fragment reads of the next k-steps and the loads of a later chunk alternate, and the
// last k-step is multiplied while the first fragments of the next chunk are read (all reads in front of a chunk's multiplications, behind its
// barrier: 700 x 2048 x 5632 21.1 us, 128 x 2048 x 8192 24.0; so 20.0 and 21.6, with 128 columns).
// Rows of LDS and their swizzle as in int8_wide.hip, and so is the order of 128 weight rows in them (two neighbouring outputs per lane).
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "groups.h"
#include "int8_device.h"
#include "unaligned.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(16))) int i32x16;
constexpr int kRowBytes = 128, kTileRows = 64;
// NJ: blocks of 32 weight rows of a wave, 1 or 2: tiles of 64 NJ weight rows.
constexpr int stage_bytes(int nj) { return (kTileRows + 64 * nj) * kRowBytes; }

constexpr int kInsA = 2;                // loads of a wave per chunk: token rows; 2 NJ of weight rows

struct Frags { i32x4 a, b, d; };        // of a k-step: 32 token rows, 32 weight rows, 32 more (NJ == 2)
// What a block needs beside them.  a_row, b_row: LDS addresses of the wave's first rows in the stage of this chunk, *_next: of the next;
// to_*: of this wave's part of the stage that is loaded; k: bytes from a row's start to the loaded chunk.
struct Block { i32x4 rs_a, rs_b; unsigned a_row, b_row, a_next, b_next, to_a, to_b, k; };

// fragments of k-step k: a block of tokens, one or two of weight rows, 4 KB apart
#define AT(k, RA, RB) "v_add_u32 %[pa" #k "], %[" #RA "], %[col" #k "]\n\tv_add_u32 %[pb" #k "], %[" #RB "], %[col" #k "]\n\t"
#define RD(f, p, o) "ds_read_b128 %[" #f "], %[" #p "] offset:" #o "\n\t"
#define READ1(k) RD(a##k, pa##k, 0) RD(b##k, pb##k, 0)
#define READ2(k) READ1(k) RD(d##k, pb##k, 4096)
#define MUL(c, a, b) "v_mfma_i32_32x32x32_i8 %[" #c "], %[" #a "], %[" #b "], %[" #c "]\n\t"
#define LA(l) "s_add_u32 m0, %[ta], " #l "*1024\n\ts_nop 0\n\tbuffer_load_dwordx4 %[ao" #l "], %[ra], %[k] offen lds\n\t"
#define LB(l) "s_add_u32 m0, %[tb], " #l "*1024\n\ts_nop 0\n\tbuffer_load_dwordx4 %[bo" #l "], %[rb], %[k] offen lds\n\t"
#define WAIT(n) "s_waitcnt lgkmcnt(" #n ")\n\t"
// in flight behind chunk kt + 1: all later ones, ST - 2 of them
#define BARRIER "s_waitcnt vmcnt(%[later])\n\ts_barrier\n\t"
#define LATER [later] "n"((ST - 2) * (kInsA + 2 * NJ))
// wait states between the compiler's vector instructions and matrix instructions, and behind the last of these: the compiler, which does
// not see what a block holds, may read or move their results right behind it
#define START "s_nop 4\n\t"
#define DONE "s_nop 15\n\ts_nop 1"

// One chunk: f holds the fragments of its first k-step and gets those of the next chunk's.  The chunk that is loaded goes where the one
// before this was.  NJ == 1: c[0] gets the even k-steps and c[1] the odd ones, so that no matrix instruction waits for the one before.
#define ADDRESSES START AT(1, row_a, row_b) AT(2, row_a, row_b) AT(3, row_a, row_b) AT(0, next_a, next_b)
#define OUT1 [c00] "+v"(c[0]), [c01] "+v"(c[1]), [a0] "+v"(f.a), [b0] "+v"(f.b), [a1] "=&v"(f1.a), [b1] "=&v"(f1.b), [a2] "=&v"(f2.a), [b2] "=&v"(f2.b), \
  [a3] "=&v"(f3.a), [b3] "=&v"(f3.b), [pa0] "=&v"(pa[0]), [pa1] "=&v"(pa[1]), [pa2] "=&v"(pa[2]), [pa3] "=&v"(pa[3]), [pb0] "=&v"(pb[0]), \
  [pb1] "=&v"(pb[1]), [pb2] "=&v"(pb[2]), [pb3] "=&v"(pb[3])
#define OUT2 OUT1, [d0] "+v"(f.d), [d1] "=&v"(f1.d), [d2] "=&v"(f2.d), [d3] "=&v"(f3.d)
#define LOADS1 [ta] "s"(s.to_a), [tb] "s"(s.to_b), [k] "s"(s.k), [ra] "s"(s.rs_a), [rb] "s"(s.rs_b), [ao0] "v"(ao[0]), [ao1] "v"(ao[1]), [bo0] "v"(bo[0]), [bo1] "v"(bo[1])
#define LOADS2 LOADS1, [bo2] "v"(bo[2]), [bo3] "v"(bo[3])
#define IN [col0] "v"(col[0]), [col1] "v"(col[1]), [col2] "v"(col[2]), [col3] "v"(col[3]), [row_a] "s"(s.a_row), [row_b] "s"(s.b_row), [next_a] "s"(s.a_next), [next_b] "s"(s.b_next)
template <int NJ, int ST>
__device__ __forceinline__ void chunk(i32x16 (&c)[2], Frags& f, const unsigned (&col)[4], const unsigned (&ao)[kInsA], const unsigned (&bo)[2 * NJ], const Block& s) {
  Frags f1, f2, f3;
  unsigned pa[4], pb[4];
  if constexpr (NJ == 2)
    asm volatile(ADDRESSES READ2(1) MUL(c00, a0, b0) READ2(2) MUL(c01, a0, d0) READ2(3) LA(0) LA(1) WAIT(6) MUL(c00, a1, b1) LB(0) LB(1) MUL(c01, a1, d1) LB(2) LB(3)
                 WAIT(3) MUL(c00, a2, b2) MUL(c01, a2, d2) WAIT(0) BARRIER READ2(0) MUL(c00, a3, b3) MUL(c01, a3, d3) WAIT(0) DONE : OUT2 : IN, LATER, LOADS2 : "memory", "scc");
  else
    asm volatile(ADDRESSES READ1(1) MUL(c00, a0, b0) READ1(2) READ1(3) LA(0) LA(1) WAIT(4) MUL(c01, a1, b1) LB(0) LB(1) WAIT(2) MUL(c00, a2, b2) WAIT(0) BARRIER
                 READ1(0) MUL(c01, a3, b3) WAIT(0) DONE : OUT1 : IN, LATER, LOADS1 : "memory", "scc");
}
// The first fragments; in flight behind chunk 0: the others that were loaded.
template <int NJ, int ST>
__device__ __forceinline__ void first_frags(Frags& f, unsigned pa, unsigned pb) {
  if constexpr (NJ == 2)
    asm volatile(BARRIER READ2(0) WAIT(0) : [a0] "=&v"(f.a), [b0] "=&v"(f.b), [d0] "=&v"(f.d) : [pa0] "v"(pa), [pb0] "v"(pb), LATER : "memory");
  else
    asm volatile(BARRIER READ1(0) WAIT(0) : [a0] "=&v"(f.a), [b0] "=&v"(f.b) : [pa0] "v"(pa), [pb0] "v"(pb), LATER : "memory");
}
// one chunk into LDS without anything beside it
template <int NJ>
__device__ __forceinline__ void load(const unsigned (&ao)[kInsA], const unsigned (&bo)[2 * NJ], const Block& s) {
  if constexpr (NJ == 2) asm volatile("s_nop 4\n\t" LA(0) LA(1) LB(0) LB(1) LB(2) LB(3) :: LOADS2 : "memory", "scc");
  else asm volatile("s_nop 4\n\t" LA(0) LA(1) LB(0) LB(1) :: LOADS1 : "memory", "scc");
}
__device__ __forceinline__ i32x4 rsrc4(const void* p, unsigned bytes) {
  const uint64_t v = (uint64_t)p;
  return i32x4{uniform((int)(unsigned)v), uniform((int)(unsigned)(v >> 32)), uniform((int)bytes), 0x00020000};
}
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ i32x4 quarter(const i32x16& c, int q) { return i32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]}; }

// KG: groups of four waves that share K.  ST: stages of a ring
template <typename S, int KG, int NJ, int ST>
__global__ __launch_bounds__(256 * KG) void int8_tile_kernel(const Int8Args a, const int mt, const int total) {
  extern __shared__ __attribute__((aligned(1024))) char s_tiles[];
  constexpr int BM = kTileRows, BN = 64 * NJ, kStages = ST, kStageBytes = stage_bytes(NJ), kInsB = 2 * NJ;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6) & 3, group = uniform(tid >> 8), h = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  // an XCD has a contiguous range of the tiles; the token tiles of a panel follow each other
  const int xcd = blockIdx.x & 7;
  const int v = (int)((int64_t)total * xcd / 8) + (blockIdx.x >> 3);
  if (v >= (int)((int64_t)total * (xcd + 1) / 8)) return;
  const int panel = v / mt, m0 = uniform((v - panel * mt) * BM), n0 = uniform(panel * BN);
  const int rows = min(a.T - m0, BM), cols = min(a.N - n0, BN), K16 = a.K16;

  // scales of this lane's outputs and of the wave's token rows
  float ws[NJ], bias[NJ];
  const int n_l = wn * 32 * NJ + NJ * (lane & 31);
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int n = min(n0 + n_l + j, a.N - 1);
    ws[j] = a.w_scale[n];
    bias[j] = a.bias ? a.bias[n] : kNoBias;
  }
  const float xs = a.x_scale[min(m0 + wm * 32 + lane, a.T - 1)];

  // this group's chunks; the last group may have fewer, and zeros in the place of the others
  const int nk = ((K16 + kRowBytes - 1) / kRowBytes + KG - 1) / KG, k_first = group * nk * kRowBytes;
  // The hardware takes the scalar offset k from the size that a descriptor states before it compares, and k runs kStages - 1 chunks past the end; that
  // difference must not go below zero.  Lanes with data lie inside the tensor by themselves (rows and columns are checked), so stating more than a
  // short tensor has lets nothing through.
  const int k_end = k_first + (nk + kStages - 1) * kRowBytes;
  Block s;
  s.rs_a = rsrc4(a.x + (int64_t)m0 * a.ldx, (unsigned)max((rows - 1) * (int)a.ldx + K16, k_end));
  s.rs_b = rsrc4(a.w + (int64_t)n0 * a.ldw, (unsigned)max((cols - 1) * (int)a.ldw + K16, k_end));
  s.k = (unsigned)uniform(k_first);
  const unsigned ring = (unsigned)uniform((int)(unsigned)(size_t)s_tiles + group * (kStages * kStageBytes));
  const int pc = lane & 7, sub = lane >> 3;
  unsigned aoff[kInsA], boff[kInsB];
  auto col_of = [&](int r) { return (unsigned)(pc ^ ((r >> 1) & 7)) * 16u; };
  auto tail = [&]() {                                      // columns behind K16; kOob is the top bit
#pragma unroll
    for (int p = 0; p < kInsA; ++p) aoff[p] |= (unsigned)((int)(s.k + col_of((wave * kInsA + p) * 8 + sub)) >= K16) << 31;
#pragma unroll
    for (int p = 0; p < kInsB; ++p) boff[p] |= (unsigned)((int)(s.k + col_of((wave * kInsB + p) * 8 + sub)) >= K16) << 31;
  };
#pragma unroll
  for (int p = 0; p < kInsA; ++p) {
    const int r = (wave * kInsA + p) * 8 + sub;
    aoff[p] = ((unsigned)r * (unsigned)a.ldx + col_of(r)) | (unsigned)(r >= rows) << 31;
  }
#pragma unroll
  for (int p = 0; p < kInsB; ++p) {
    const int r = (wave * kInsB + p) * 8 + sub, n = NJ == 1 ? r : (r & 64) + 2 * (r & 31) + ((r >> 5) & 1);
    boff[p] = ((unsigned)n * (unsigned)a.ldw + col_of(r)) | (unsigned)(n >= cols) << 31;
  }
  if (K16 - (int)s.k < kRowBytes) tail();
  auto step = [&]() {
    s.k = (unsigned)uniform((int)s.k + kRowBytes);
    if (K16 - (int)s.k < kRowBytes) tail();
  };
  // LDS addresses of this wave's rows and of its part of a load
  const unsigned a_at = uniform((int)ring + wm * 32 * kRowBytes), b_at = uniform((int)ring + (BM + wn * 32 * NJ) * kRowBytes);
  const unsigned a_to = uniform((int)ring + wave * (kInsA * 1024)), b_to = uniform((int)ring + BM * kRowBytes + wave * (kInsB * 1024));
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    s.to_a = a_to + i * kStageBytes; s.to_b = b_to + i * kStageBytes;
    load<NJ>(aoff, boff, s);
    step();
  }
  const unsigned fkey = (unsigned)((lane & 31) >> 1) & 7u;
  unsigned col[4];                                         // of a lane's 16 bytes of k-step k, behind the wave's first row
#pragma unroll
  for (int k = 0; k < 4; ++k) col[k] = (unsigned)((lane & 31) * kRowBytes) + ((unsigned)(2 * k + h) ^ fkey) * 16u;
  Frags f;
  first_frags<NJ, ST>(f, col[0] + a_at, col[0] + b_at);
  i32x16 acc[2] = {};
  unsigned here = 0, next = kStageBytes, free = (kStages - 1) * kStageBytes;   // stages of chunks kt, kt + 1, kt - 1
  for (int kt = 0; kt < nk; ++kt) {
    s.a_row = a_at + here; s.b_row = b_at + here;
    s.a_next = a_at + next; s.b_next = b_at + next;
    s.to_a = a_to + free; s.to_b = b_to + free;
    chunk<NJ, ST>(acc, f, col, aoff, boff, s);
    free = here;
    here = next;
    next = next == (kStages - 1) * kStageBytes ? 0 : next + kStageBytes;
    step();
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // the loads behind the last chunk, zeros; LDS is used again or given back
  if (a.k_tail && group == 0) {
    // the last K % 16 codes, in the lanes of the first half
    const i32x4 zero = {0, 0, 0, 0};
    const i32x4 ta = h ? zero : masked_codes(a.x + (int64_t)min(m0 + wm * 32 + (lane & 31), a.T - 1) * a.ldx + K16, a.k_tail);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const i32x4 tb = h ? zero : *reinterpret_cast<const i32x4*>(a.w + (int64_t)min(n0 + n_l + j, a.N - 1) * a.ldw + K16);
      acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(ta, tb, acc[j], 0, 0, 0);
    }
  }
  if constexpr (NJ == 1) acc[0] += acc[1];
  if constexpr (KG == 2) {
    lds_barrier();                                         // the rings have been read
    i32x4* const sums = reinterpret_cast<i32x4*>(s_tiles) + wave * (4 * NJ * 64) + lane;
    if (group == 1) {
#pragma unroll
      for (int i = 0; i < 4 * NJ; ++i) sums[i * 64] = quarter(acc[i >> 2], i & 3);
    }
    lds_barrier();
    if (group == 1) return;
#pragma unroll
    for (int i = 0; i < 4 * NJ; ++i) {
      const i32x4 v = sums[i * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i >> 2][4 * (i & 3) + e] += v[e];
    }
  }
  S* const out0 = static_cast<S*>(a.out) + (int64_t)(m0 + wm * 32) * a.ldo + n0;
  const unsigned lane_off = (unsigned)(4 * h) * (unsigned)a.ldo + (unsigned)n_l;
  const bool whole = rows == BM && cols == BN;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int r = 8 * (e >> 2) + (e & 3);                  // + 4 h
    const float s = __shfl(xs, r + 4 * h);
    Unaligned<S, NJ> o;
#pragma unroll
    for (int j = 0; j < NJ; ++j) o.v[j] = to_out<S>(scaled(acc[j][e], s, ws[j], bias[j]));
    S* const p = out0 + (int64_t)r * a.ldo + lane_off;
    if (whole) {
      *reinterpret_cast<Unaligned<S, NJ>*>(p) = o;
    } else if (wm * 32 + r + 4 * h < rows) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) if (n_l + j < cols) p[j] = o.v[j];
    }
  }
}

template <typename S, int KG, int NJ, int ST>
int launch_t(const Int8Args& a, hipStream_t s) {
  constexpr int kLds = KG * ST * stage_bytes(NJ);
  static_assert(kLds <= 163840, "LDS of a CU");
  static std::atomic<int> ready{0};
  if (!ready.load(std::memory_order_relaxed)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_tile_kernel<S, KG, NJ, ST>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess)
      return hip_fail(hipGetLastError(), "int8_tile_kernel: LDS size attribute");
    ready.store(1, std::memory_order_relaxed);
  }
  const int64_t mt = (a.T + 63) / 64, total = mt * ((a.N + 64 * NJ - 1) / (64 * NJ));
  if (total >= (int64_t)1 << 23) return fail(MOE_E_UNSUPPORTED, "8-bit product: %lld tiles", (long long)total);   // of 2^32 threads in a grid
  hipLaunchKernelGGL((int8_tile_kernel<S, KG, NJ, ST>), dim3((unsigned)(((total + 7) / 8) * 8)), dim3(256 * KG), kLds, s, a, (int)mt, (int)total);
  return hip_fail(hipGetLastError(), "int8_tile_kernel launch");
}

template <typename S>
int launch_s(const Int8Args& a, Int8Tile tile, hipStream_t s) {
  switch (tile) {
    case Int8Tile::k64Shared: return launch_t<S, 2, 1, 5>(a, s);
    case Int8Tile::k64: return launch_t<S, 1, 1, 3>(a, s);
    case Int8Tile::k64Short: return launch_t<S, 1, 1, 2>(a, s);
    case Int8Tile::k128Shared: return launch_t<S, 2, 2, 3>(a, s);
    default: return launch_t<S, 1, 2, 3>(a, s);
  }
}

}  // namespace

int launch_int8_tile(const Int8Args& a, Int8Tile tile, hipStream_t s) {
  return a.out_dtype == MOE_FP32 ? launch_s<float>(a, tile, s) : launch_s<uint16_t>(a, tile, s);
}

}  // namespace mm
