// The 8-bit product on tiles of 64 tokens x 128 weight rows: more tokens than the streaming kernel takes, and too few tiles of 256 x 256
// to fill the chip.
//
// Four waves in a 2 x 2 grid, three stages of 128 k in LDS, filled past the registers two chunks ahead; two workgroups per CU, so that
// one multiplies while the other waits.  Where the tiles are fewer than the CUs, eight waves: two groups with a ring each share K, and
// their sums of integers are joined in LDS, exactly.  A chunk is one asm block: all its fragment reads are issued at once and the matrix
// instructions of a k-step wait for those of that k-step only.  Rows of LDS, their swizzle and the order of the weight rows in them
// as in int8_wide.hip (two neighbouring outputs per lane).
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "groups.h"
#include "int8_device.h"
#include "unaligned.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kRowBytes = 128, kTileCols = 128, kStages = 3;

#define MM_WAIT_VMCNT(n) __builtin_amdgcn_s_waitcnt(0x0f70 | ((n) & 15) | (((n) >> 4) << 14))

#define RD(f, p, o) "ds_read_b128 %[" #f "], %[" #p "] offset:" #o "\n\t"
#define MUL(c, a, b) "v_mfma_i32_32x32x32_i8 %[" #c "], %[" #a "], %[" #b "], %[" #c "]\n\t"
// fragments of k-step k: a block of tokens, two of weight rows, 4 KB apart
#define READ(k) RD(a##k, pa##k, 0) RD(b##k, pb##k, 0) RD(d##k, pb##k, 4096)
#define MULS(k) MUL(c00, a##k, b##k) MUL(c01, a##k, d##k)
#define WAIT(n) "s_waitcnt lgkmcnt(" #n ")\n\t"
#define ADDR(k) [pa##k] "v"(pa + col[k]), [pb##k] "v"(pb + col[k])

// matrix results can be read or moved: the compiler, which does not see what a block holds, may do so right behind it
#define DONE "s_nop 15\n\ts_nop 1"

// One chunk: tokens at LDS address pa, weight rows at pb, k-step k's 16 bytes of a lane at col[k].
__device__ __forceinline__ void chunk(i32x16 (&c)[2], unsigned pa, unsigned pb, const unsigned (&col)[4]) {
  i32x4 a0, a1, a2, a3, b0, b1, b2, b3, d0, d1, d2, d3;
  asm volatile("s_nop 4\n\t" READ(0) READ(1) READ(2) READ(3) WAIT(9) MULS(0) WAIT(6) MULS(1) WAIT(3) MULS(2) WAIT(0) MULS(3) DONE
               : [c00] "+v"(c[0]), [c01] "+v"(c[1]), [a0] "=&v"(a0), [a1] "=&v"(a1), [a2] "=&v"(a2), [a3] "=&v"(a3), [b0] "=&v"(b0), [b1] "=&v"(b1),
                 [b2] "=&v"(b2), [b3] "=&v"(b3), [d0] "=&v"(d0), [d1] "=&v"(d1), [d2] "=&v"(d2), [d3] "=&v"(d3)
               : ADDR(0), ADDR(1), ADDR(2), ADDR(3) : "memory");
}
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ i32x4 quarter(const i32x16& c, int q) { return i32x4{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]}; }

// KG: groups of four waves that share K
template <typename S, int KG>
__global__ __launch_bounds__(256 * KG) void int8_tile_kernel(const Int8Args a, const int mt, const int total) {
  extern __shared__ __attribute__((aligned(1024))) char s_tiles[];
  constexpr int BM = 64, kStageBytes = (BM + kTileCols) * kRowBytes, kInsA = 2, kInsB = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6) & 3, group = uniform(tid >> 8), h = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  // an XCD has a contiguous range of the tiles; the token tiles of a panel follow each other
  const int xcd = blockIdx.x & 7;
  const int v = (int)((int64_t)total * xcd / 8) + (blockIdx.x >> 3);
  if (v >= (int)((int64_t)total * (xcd + 1) / 8)) return;
  const int panel = v / mt, m0 = uniform((v - panel * mt) * BM), n0 = uniform(panel * kTileCols);
  const int rows = min(a.T - m0, BM), cols = min(a.N - n0, kTileCols), K16 = a.K16;

  // scales of this lane's outputs and of the wave's token rows
  float ws[2], bias[2];
  const int n_l = wn * 64 + 2 * (lane & 31);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int n = min(n0 + n_l + j, a.N - 1);
    ws[j] = a.w_scale[n];
    bias[j] = a.bias ? a.bias[n] : kNoBias;
  }
  const float xs = a.x_scale[min(m0 + wm * 32 + lane, a.T - 1)];

  const __amdgpu_buffer_rsrc_t ra = make_rsrc(a.x + (int64_t)m0 * a.ldx, (unsigned)((rows - 1) * (int)a.ldx + K16));
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.w + (int64_t)n0 * a.ldw, (unsigned)((cols - 1) * (int)a.ldw + K16));
  // this group's chunks; the last group may have fewer, and zeros in the place of the others
  const int nk = ((K16 + kRowBytes - 1) / kRowBytes + KG - 1) / KG, k_first = group * nk * kRowBytes;
  char* const ring = s_tiles + group * (kStages * kStageBytes);
  const int pc = lane & 7, sub = lane >> 3;
  unsigned aoff[kInsA], boff[kInsB];
  auto col_of = [&](int r) { return (unsigned)(pc ^ ((r >> 1) & 7)) * 16u; };
#pragma unroll
  for (int p = 0; p < kInsA; ++p) {
    const int r = (wave * kInsA + p) * 8 + sub;
    aoff[p] = r < rows ? (unsigned)r * (unsigned)a.ldx + col_of(r) + (unsigned)k_first : kOob;
  }
#pragma unroll
  for (int p = 0; p < kInsB; ++p) {
    const int r = (wave * kInsB + p) * 8 + sub, n = (r & 64) + 2 * (r & 31) + ((r >> 5) & 1);
    boff[p] = n < cols ? (unsigned)n * (unsigned)a.ldw + col_of(r) + (unsigned)k_first : kOob;
  }
  auto issue = [&](int kt) {
    char* const st = ring + kt % kStages * kStageBytes;
    const int left = K16 - k_first - kt * kRowBytes;                 // columns from here on are not there
#pragma unroll
    for (int p = 0; p < kInsA; ++p) {
      const unsigned off = (int)col_of((wave * kInsA + p) * 8 + sub) < left ? aoff[p] : kOob;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(st + (wave * kInsA + p) * 1024), 16, (int)off, 0, 0, 0);
      aoff[p] += kRowBytes;
    }
#pragma unroll
    for (int p = 0; p < kInsB; ++p) {
      const unsigned off = (int)col_of((wave * kInsB + p) * 8 + sub) < left ? boff[p] : kOob;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)(st + BM * kRowBytes + (wave * kInsB + p) * 1024), 16, (int)off, 0, 0, 0);
      boff[p] += kRowBytes;
    }
  };
  const unsigned fkey = (unsigned)((lane & 31) >> 1) & 7u;
  unsigned col[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) col[k] = (unsigned)((lane & 31) * kRowBytes) + ((unsigned)(2 * k + h) ^ fkey) * 16u;
  const unsigned lds0 = (unsigned)(size_t)ring;
  const unsigned pa = lds0 + wm * 32 * kRowBytes, pb = lds0 + (BM + wn * 64) * kRowBytes;
  i32x16 acc[2] = {};
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) if (i < nk) issue(i);
  for (int kt = 0; kt < nk; ++kt) {
    // chunk kt has landed: the loads behind it are those of chunk kt + 1
    if (kt + 1 < nk) MM_WAIT_VMCNT(kInsA + kInsB); else MM_WAIT_VMCNT(0);
    asm volatile("s_barrier" ::: "memory");                // ... in all waves, and all have read chunk kt - 1, whose stage chunk kt + 2 takes
    if (kt + kStages - 1 < nk) issue(kt + kStages - 1);
    const unsigned st = (unsigned)(kt % kStages * kStageBytes);
    chunk(acc, pa + st, pb + st, col);
  }
  if (a.k_tail && group == 0) {
    // the last K % 16 codes, in the lanes of the first half
    const i32x4 zero = {0, 0, 0, 0};
    const i32x4 ta = h ? zero : masked_codes(a.x + (int64_t)min(m0 + wm * 32 + (lane & 31), a.T - 1) * a.ldx + K16, a.k_tail);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const i32x4 tb = h ? zero : *reinterpret_cast<const i32x4*>(a.w + (int64_t)min(n0 + n_l + j, a.N - 1) * a.ldw + K16);
      acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(ta, tb, acc[j], 0, 0, 0);
    }
  }
  if constexpr (KG == 2) {
    lds_barrier();                                         // the rings have been read
    i32x4* const sums = reinterpret_cast<i32x4*>(s_tiles) + wave * (8 * 64) + lane;
    if (group == 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[i * 64] = quarter(acc[i >> 2], i & 3);
    }
    lds_barrier();
    if (group == 1) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const i32x4 v = sums[i * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i >> 2][4 * (i & 3) + e] += v[e];
    }
  }
  S* const out0 = static_cast<S*>(a.out) + (int64_t)(m0 + wm * 32) * a.ldo + n0;
  const unsigned lane_off = (unsigned)(4 * h) * (unsigned)a.ldo + (unsigned)n_l;
  const bool whole = rows == BM && cols == kTileCols;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int r = 8 * (e >> 2) + (e & 3);                  // + 4 h
    const float s = __shfl(xs, r + 4 * h);
    Unaligned<S, 2> o;
#pragma unroll
    for (int j = 0; j < 2; ++j) o.v[j] = to_out<S>(scaled(acc[j][e], s, ws[j], bias[j]));
    S* const p = out0 + (int64_t)r * a.ldo + lane_off;
    if (whole) {
      *reinterpret_cast<Unaligned<S, 2>*>(p) = o;
    } else if (wm * 32 + r + 4 * h < rows) {
#pragma unroll
      for (int j = 0; j < 2; ++j) if (n_l + j < cols) p[j] = o.v[j];
    }
  }
}

template <typename S, int KG>
int launch_t(const Int8Args& a, hipStream_t s) {
  constexpr int kLds = KG * kStages * (64 + kTileCols) * kRowBytes;
  static std::atomic<int> ready{0};
  if (!ready.load(std::memory_order_relaxed)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_tile_kernel<S, KG>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess)
      return hip_fail(hipGetLastError(), "int8_tile_kernel: LDS size attribute");
    ready.store(1, std::memory_order_relaxed);
  }
  const int64_t mt = (a.T + 63) / 64, total = mt * ((a.N + kTileCols - 1) / kTileCols);
  if (total >= (int64_t)1 << 30) return fail(MOE_E_UNSUPPORTED, "8-bit product: %lld tiles", (long long)total);
  hipLaunchKernelGGL((int8_tile_kernel<S, KG>), dim3((unsigned)(((total + 7) / 8) * 8)), dim3(256 * KG), kLds, s, a, (int)mt, (int)total);
  return hip_fail(hipGetLastError(), "int8_tile_kernel launch");
}

}  // namespace

int launch_int8_tile(const Int8Args& a, bool share_k, hipStream_t s) {
  if (a.out_dtype == MOE_FP32) return share_k ? launch_t<float, 2>(a, s) : launch_t<float, 1>(a, s);
  return share_k ? launch_t<uint16_t, 2>(a, s) : launch_t<uint16_t, 1>(a, s);
}

}  // namespace mm
