// The 8-bit product on tiles of up to 256 tokens x 256 weight rows, for many tokens.
//
// What bounds it: the matrix cores (random codes draw so much power that the matrix instructions alone reach 3.3 of their 4.9 POP/s), and
// beside them LDS: 48 KB per 512 cycles of a k-step, as in ffn_wide.hip.  Its k-step serves here with the 8-bit instruction: 32 k where
// bf16 has 16, a chunk of 128 bytes is 128 k.  So do its LDS ring, its two wave layouts and the stream of chunks that runs on through
// the tiles of a workgroup; here all tiles have one height, and where the token tiles and panels lie is arithmetic.
//   * Weight row n of a wave's 128 sits in LDS row (n % 4) 32 + n / 4 (narrow tiles: 64, (n % 2) 32 + n / 2): a lane then ends up with four (two)
//     neighbouring outputs of a token, one store instead of four.
//   * An XCD has a contiguous range of the tiles, ordered so that the 32 that run at a time are about 8 token tiles x 4 panels: the operands
//     that its L2 has to fetch are the fewest so.
//   * Codes behind K: whole vectors of 16 bytes are not loaded.  The rest of K % 16 codes is added by one k-step of its own, masked.
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "int8_device.h"
#include "unaligned.h"
#define WIDE_MFMA "v_mfma_i32_32x32x32_i8"
#include "wide_step.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(16))) int i32x16;

constexpr int kThreadsW = 256;
constexpr int kPanelGroup = 4;          // panels that are run side by side

struct Tile { int valid, m0, rows, n0, cols; };

// one k-step without reads and loads
template <bool TALL, int NB>
__device__ __forceinline__ void multiply(i32x16 (&c)[4][4], const i32x4 (&fa)[4], const i32x4 (&fb)[4]) {
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < (TALL ? 4 : 2); ++j)
      asm volatile("s_nop 4\n\tv_mfma_i32_32x32x32_i8 %0, %1, %2, %0" : "+a"(c[i][j]) : "v"(fa[i]), "v"(fb[j]));
}

// Matrix results are readable behind this, and the compiler moves none of them in front of it.
template <bool TALL, int NB>
__device__ __forceinline__ void settle(i32x16 (&c)[4][4]) {
#define SETTLE "s_nop 15\n\ts_nop 7"
  if constexpr (TALL && NB == 4) asm volatile(SETTLE : C4(0), C4(1), C4(2), C4(3));
  else if constexpr (TALL) asm volatile(SETTLE : C4(0), C4(1), C4(2));
  else if constexpr (NB == 4) asm volatile(SETTLE : C1(0, 0), C1(0, 1), C1(1, 0), C1(1, 1), C1(2, 0), C1(2, 1), C1(3, 0), C1(3, 1));
  else if constexpr (NB == 3) asm volatile(SETTLE : C1(0, 0), C1(0, 1), C1(1, 0), C1(1, 1), C1(2, 0), C1(2, 1));
  else if constexpr (NB == 2) asm volatile(SETTLE : C1(0, 0), C1(0, 1), C1(1, 0), C1(1, 1));
  else asm volatile(SETTLE : C1(0, 0), C1(0, 1));
#undef SETTLE
}

template <typename S>
__global__ __launch_bounds__(kThreadsW) __attribute__((amdgpu_waves_per_eu(1, 1))) void int8_wide_kernel(const Int8Args a, const int mt, const int height,
                                                                                                        const int panels) {
  extern __shared__ __attribute__((aligned(1024))) char s_ring[];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), h = lane >> 5;
  const unsigned lds0 = (unsigned)(size_t)s_ring;
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, nslots = gridDim.x >> 3;
  const int total = mt * panels;
  const int first_tile = (int)((int64_t)total * xcd / 8), end_tile = (int)((int64_t)total * (xcd + 1) / 8);
  const bool tall = height > 128;
  const int K16 = a.K16;

  auto tile_at = [&](int i) -> Tile {
    Tile T = {};
    const int v = first_tile + i * nslots + slot;
    T.valid = v < end_tile;
    if (!T.valid) return T;
    const int g = v / (kPanelGroup * mt), r = v - g * (kPanelGroup * mt), pg = min(kPanelGroup, panels - g * kPanelGroup);
    const int m = r / pg;
    T.m0 = uniform(m * height);
    T.rows = uniform(min(a.T - T.m0, height));
    T.n0 = uniform((g * kPanelGroup + r - m * pg) * 256);
    T.cols = uniform(min(a.N - T.n0, 256));
    return T;
  };
  int ord = 0;
  Tile cur = tile_at(ord++);
  if (!cur.valid) return;
  Tile nx = tile_at(ord++);

  // ---- load cursors ----
  i32x4 rsA, rsB;
  unsigned aoff[kA], boff[kB];
  int ka = 0, kb = 0, na_left = 0, nb_left = 0;
  int slA = 0, slB = 0;                                    // slots of the next token / weight chunk
  const int pc = lane & 7, sub = lane >> 3;
  auto col_of = [&](int p) { return (unsigned)(pc ^ (((p & 1) * 4 + (lane >> 4)) & 7)) * 16u; };
  auto tail_a = [&]() {
#pragma unroll
    for (int p = 0; p < kA; ++p) aoff[p] |= (unsigned)(ka + (int)col_of(p) >= K16) << 31;   // kOob is the top bit
  };
  auto tail_b = [&]() {
#pragma unroll
    for (int p = 0; p < kB; ++p) boff[p] |= (unsigned)(kb + (int)col_of(p) >= K16) << 31;
  };
  auto open_a = [&](const Tile& T) {
    rsA = rsrc4(a.x + (T.valid ? (int64_t)T.m0 * a.ldx : 0), buffer_bytes(T.valid ? (unsigned)((T.rows - 1) * (int)a.ldx + K16) : 0u));
    ka = 0; na_left = T.valid ? tile_chunks((K16 + 1) / 2) : 0x7fffffff;
#pragma unroll
    for (int p = 0; p < kA; ++p) {
      const int r = wave * 64 + 8 * p + sub;
      aoff[p] = ((unsigned)r * (unsigned)a.ldx + col_of(p)) | ((unsigned)(!T.valid || r >= T.rows) << 31);
    }
    if (K16 < 128) tail_a();
  };
  auto open_b = [&](const Tile& T) {
    rsB = rsrc4(a.w + (T.valid ? (int64_t)T.n0 * a.ldw : 0), buffer_bytes(T.valid ? (unsigned)((T.cols - 1) * (int)a.ldw + K16) : 0u));
    kb = 0; nb_left = T.valid ? tile_chunks((K16 + 1) / 2) : 0x7fffffff;
#pragma unroll
    for (int p = 0; p < kB; ++p) {
      const int r = wave * 64 + 8 * p + sub;               // LDS row
      const int n = tall ? (r & 128) + 4 * (r & 31) + ((r >> 5) & 3) : (r & 192) + 2 * (r & 31) + ((r >> 5) & 1);
      boff[p] = ((unsigned)n * (unsigned)a.ldw + col_of(p)) | ((unsigned)(!T.valid || n >= T.cols) << 31);
    }
    if (K16 < 128) tail_b();
  };
  auto step_a = [&]() {
    slA = slA + 1 == SA ? 0 : slA + 1;
    na_left = uniform(na_left - 1);
    if (na_left == 0) open_a(nx);
    else { ka = uniform(ka + kRowB); if (uniform(K16 - ka) < 128) tail_a(); }
  };
  auto step_b = [&]() {
    slB = slB + 1 == SB ? 0 : slB + 1;
    nb_left = uniform(nb_left - 1);
    if (nb_left == 0) open_b(nx);
    else { kb = uniform(kb + kRowB); if (uniform(K16 - kb) < 128) tail_b(); }
  };
  const int ldsA = uniform((int)lds0 + wave * kA * 1024), ldsB = uniform((int)lds0 + SA * kSlotB + wave * kB * 1024);
  // load l of a period: the token chunk's first, then the weight chunk's
  auto put = [&](Loads& L, int d, int l) {
    if (l < kA) { L.rs[d] = rsA; L.vo[d] = aoff[l]; L.so[d] = uniform(ka); L.md[d] = uniform(ldsA + slA * kSlotB + l * 1024); }
    else { L.rs[d] = rsB; L.vo[d] = boff[l - kA]; L.so[d] = uniform(kb); L.md[d] = uniform(ldsB + slB * kSlotB + (l - kA) * 1024); }
  };
  open_a(cur);
  open_b(cur);
  // ---- fill: periods 1 - SB .. -1 ----
#pragma unroll
  for (int i = 1 - SB; i < 0; ++i) {
    if (i - 1 + SA >= 0) {
#pragma unroll
      for (int l = 0; l < kA; ++l) load_one(rsA, aoff[l], ka, ldsA + slA * kSlotB + l * 1024);
      step_a();
    }
#pragma unroll
    for (int l = 0; l < kB; ++l) load_one(rsB, boff[l], kb, ldsB + slB * kSlotB + l * 1024);
    step_b();
  }

  // ---- fragment addresses: a lane's 16 bytes of k-step k, without the slot and the wave's rows ----
  const unsigned fkey = (unsigned)((lane & 31) >> 1) & 7u;
  unsigned col[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) col[k] = lds0 + (unsigned)((lane & 31) * kRowB) + ((unsigned)(2 * k + h) ^ fkey) * 16u;

  auto run = [&](auto tall_tag, auto nb_tag) {
    constexpr bool TALL = decltype(tall_tag)::value;
    constexpr int NB = decltype(nb_tag)::value, TN = TALL ? 4 : 2;
    const int wm = TALL ? wave >> 1 : 0, wn = TALL ? wave & 1 : wave;
    const int arow = uniform(a_row(TALL, NB, wave) * kRowB), brow = uniform(SA * kSlotB + b_row(false, TALL, wave) * kRowB);
    const int qrow = uniform(SA * kSlotB + b_row_of(false, TALL, wave, 3) * kRowB);
    i32x4 fa[2][4], fb[2][4];
    i32x16 acc[4][4];
    int cA = 0, cB = 0;                                    // slots of the chunk being multiplied
    first_frags<false>(fa[0], fb[0], col[0] + arow, col[0] + brow, col[0] + qrow);
    // loads 0 .. kLoads-1 of period 0
#pragma unroll
    for (int l = 0; l < kLoads; ++l) load_one(rsA, aoff[l], ka, ldsA + slA * kSlotB + l * 1024);
    const int nk = uniform(tile_chunks((K16 + 1) / 2));
    // Scales of this lane's outputs and of the wave's token rows (rows lane and lane + 64).  Loads end in order, so those of the next tile are issued in
    // front of this tile's stores and awaited behind them: nowhere does a wait for them stop the loads into LDS.
    const int n_l = (TALL ? wn * 128 : wn * 64) + TN * (lane & 31);
    struct Scales { float w[TN], bias[TN], x[2]; };
    auto scales_of = [&](const Tile& T) {
      Scales s;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int n = min(T.n0 + n_l + j, a.N - 1);
        s.w[j] = a.w_scale[n];
        s.bias[j] = a.bias ? a.bias[n] : kNoBias;
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) s.x[q] = a.x_scale[min(T.m0 + wm * NB * 32 + q * 64 + lane, a.T - 1)];
      asm volatile("" ::: "memory");
      return s;
    };
    auto await = [&](Scales& s) {
#pragma unroll
      for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(s.w[j]), "+v"(s.bias[j]));
      asm volatile("" : "+v"(s.x[0]), "+v"(s.x[1]));
    };
    Scales sc = scales_of(cur);
    await(sc);
    for (;;) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
      for (int kt = 0; kt < nk; ++kt) {
        const unsigned oA = (unsigned)(cA * kSlotB + arow), oB = (unsigned)(cB * kSlotB + brow);
        Loads L;
#pragma unroll
        for (int d = 0; d < kLoads; ++d) put(L, d, kLoads + d);
        kstep<TALL, NB, false, false>(acc, fa[0], fb[0], fa[1], fb[1], col[1] + oA, col[1] + oB, 0u, L);
#pragma unroll
        for (int d = 0; d < kLoads; ++d) put(L, d, 2 * kLoads + d);
        kstep<TALL, NB, false, false>(acc, fa[1], fb[1], fa[0], fb[0], col[2] + oA, col[2] + oB, 0u, L);
        step_a();
#pragma unroll
        for (int d = 0; d < kLoads; ++d) put(L, d, 3 * kLoads + d);
        kstep<TALL, NB, false, false>(acc, fa[0], fb[0], fa[1], fb[1], col[3] + oA, col[3] + oB, 0u, L);
        step_b();
        cA = cA + 1 == SA ? 0 : cA + 1;
        cB = cB + 1 == SB ? 0 : cB + 1;
#pragma unroll
        for (int d = 0; d < kLoads; ++d) put(L, d, d);
        kstep<TALL, NB, false, true>(acc, fa[1], fb[1], fa[0], fb[0], col[0] + (unsigned)(cA * kSlotB + arow),
                                     col[0] + (unsigned)(cB * kSlotB + brow), col[0] + (unsigned)(cB * kSlotB + qrow), L);
      }
      if (a.k_tail) {
        // the last K % 16 codes, in the lanes of the first half
        i32x4 ta[4], tb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ta[i] = tb[i] = i32x4{0, 0, 0, 0};
          if (i < NB && h == 0) ta[i] = masked_codes(a.x + (int64_t)min(cur.m0 + (wm * NB + i) * 32 + (lane & 31), a.T - 1) * a.ldx + K16, a.k_tail);
          if (i < TN && h == 0) tb[i] = *reinterpret_cast<const i32x4*>(a.w + (int64_t)min(cur.n0 + n_l + i, a.N - 1) * a.ldw + K16);
        }
        multiply<TALL, NB>(acc, ta, tb);
      }
      settle<TALL, NB>(acc);
      // ---- epilogue: accumulator v of lane l is row 8*(v/4) + 4*(l/32) + v%4, output TN*(l%32) + j ----
      Scales next = scales_of(nx);
      const int row_w = wm * NB * 32;
      const bool whole = cur.cols == 256 && cur.rows == (TALL ? 2 : 1) * NB * 32;
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
            const float s = h ? s1 : s0;
            Unaligned<S, TN> o;
#pragma unroll
            for (int j = 0; j < TN; ++j) o.v[j] = to_out<S>(scaled(acc_read(acc[i][j], v), s, sc.w[j], sc.bias[j]));
            S* const p = reinterpret_cast<S*>(out_r + (int64_t)r * a.ldo * (int)sizeof(S) + lane_off);
            if constexpr (decltype(whole_tag)::value) {
              *reinterpret_cast<Unaligned<S, TN>*>(p) = o;
            } else if (row_w + r + 4 * h < cur.rows) {
#pragma unroll
              for (int j = 0; j < TN; ++j) if (n_l + j < cur.cols) p[j] = o.v[j];
            }
          }
      };
      if (whole) { store(std::true_type{}); await(next); } else { store(std::false_type{}); await(next); }
      sc = next;
      cur = nx;
      if (!cur.valid) break;
      nx = tile_at(ord++);
    }
  };
  using std::integral_constant;
  if (tall) {
    if (height > 192) run(std::true_type{}, integral_constant<int, 4>{});
    else run(std::true_type{}, integral_constant<int, 3>{});
  } else {
    if (height > 96) run(std::false_type{}, integral_constant<int, 4>{});
    else if (height > 64) run(std::false_type{}, integral_constant<int, 3>{});
    else if (height > 32) run(std::false_type{}, integral_constant<int, 2>{});
    else run(std::false_type{}, integral_constant<int, 1>{});
  }
  // the loads behind the last chunk only fill LDS with zeros; they end before the workgroup does
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <typename S>
int launch_t(const Int8Args& a, int mt, int height, hipStream_t s) {
  static std::atomic<int> ready{0};
  if (!ready.load(std::memory_order_relaxed)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_wide_kernel<S>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytes) != hipSuccess)
      return hip_fail(hipGetLastError(), "int8_wide_kernel: LDS size attribute");
    ready.store(1, std::memory_order_relaxed);
  }
  int grid = device_cu_count() / 8 * 8;
  if (grid < 8) grid = 8;                                   // a multiple of the 8 XCDs
  hipLaunchKernelGGL(int8_wide_kernel<S>, dim3((unsigned)grid), dim3(kThreadsW), kLdsBytes, s, a, mt, height, (a.N + 255) / 256);
  return hip_fail(hipGetLastError(), "int8_wide_kernel launch");
}

}  // namespace

int launch_int8_wide(const Int8Args& a, int mt, int height, hipStream_t s) {
  return a.out_dtype == MOE_FP32 ? launch_t<float>(a, mt, height, s) : launch_t<uint16_t>(a, mt, height, s);
}

}  // namespace mm
