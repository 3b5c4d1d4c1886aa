// A user's history in 8 bits, and softmax attention over it.
//
// The cache: rows K, V [B,H,capacity,d] in e4m3, and for every block of 64 rows of a head a scale that is a power of
// two: the smallest 2^e (e >= -100) with max|x| <= 448 * 2^e over the block.  e4m3 has the same relative precision
// at every magnitude down to 2^-6, so a scale between two powers of two would gain nothing; and with whole powers a scale
// comes out of a sum as an exact factor, and a block whose exponent grows when a later row comes in is moved to the
// new exponent without another rounding (but for values under 2^-14 of the block's largest, which e4m3 holds as
// fractions of 2^-9).  A block that another program filled may have any positive scale; the append rounds its rows to a
// power of two, from what they stand for.
//
// history_append_kernel: a CTA per block of the cache that the new rows touch, head and K or V.
//
// history_attention_kernel: o = softmax(scale q K^T) V over the rows that a user has, for 16 (query, head of the
// group) rows per CTA, so that the query heads of a cached head share its rows.  Warps take blocks of 64 rows in
// turn, each with its own running maximum and sum, and add up at the end; where the queries alone do not fill the
// GPU, the rows are split over the CTAs of a cluster, which add up through distributed shared memory: one launch, no
// workspace.  A warp brings its rows to shared memory itself, the keys of the next block and the values of this one while
// it works on the keys of this one, and reads them as 8-bit fragments: a lane takes 16 bytes of a key, and the order of
// the products' inner index is whatever those bytes are (queries are laid out to match); of the values it takes the bytes
// of two rows that a fragment pairs, interleaved by one byte permutation.  All MMAs are fp16 x fp16 with fp32
// sums, e4m3 being exact in fp16:
//   q    each row by a power of two to below 2, then fp16 (bf16 storage: exact down to 2^-14 of the row's largest) or a
//        high and a low fp16 half (fp32 storage: 22 bits)
//   p    2^(s - m + 15), so that fp16 holds weights down to 2^-39 of the largest; fp32 storage: high and low halves
// The sums of a block's p V are fp32 and are scaled by the block's 2^e as they join the row's.
//
// 64 users, 8 query heads over 2 x 128: 92 us a launch where each has 16384 rows, 5.8 TB/s; 87 us, 4.6 TB/s, where they have 8192
// to 16384 (90 with the append), since every user gets the same number of CTAs and the SMs are then active three quarters of
// the time; d = 64, all of 16384, 54 us, 5.0 TB/s.  No pipe is full (issue slots 34 %, ALU 30 %, tensor 34 % of the active time):
// latency, with two warps a scheduler at 255 registers, of about 1200 instructions for a warp's 64 rows of d = 128, a fifth of them
// conversions (by shifts and masks in their place 171 us); products, exponentials and sums are made for 16 query rows, of which
// a group of four heads has four.  Hence packed arithmetic, plain copies of whole blocks and products of eight tiles in flight
// (140 us with rows straight from global memory, 107, 94).
#include <cuda_fp16.h>

#include "sm100_ptx.cuh"
#include "solar_internal.cuh"

namespace solar {
namespace {

constexpr int kBlock = SOLAR_CACHE_BLOCK;          // rows that share a scale
constexpr int kMinExp = -100, kMaxExp = 120;       // of a scale that the append writes: 448 * 2^120 is past what fp32 holds

__device__ __forceinline__ float two_to(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127
// a * f without a second rounding to come: cut off, and its last bit set where something was (24 bits before the four of e4m3)
__device__ __forceinline__ float mul_odd(float a, float f) {
  const float p = __fmul_rz(a, f);
  return fmaf(a, f, -p) == 0.f ? p : __uint_as_float(__float_as_uint(p) | 1u);
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 0xffu) - 127; }
// Two floats to e4m3, nearest even; what is not finite becomes NaN.
__device__ __forceinline__ uint32_t to_e4m3x2(float a, float b) {
  const float nan = __int_as_float(0x7fffffff);
  a = fabsf(a) == INFINITY ? nan : a;
  b = fabsf(b) == INFINITY ? nan : b;
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}

__device__ __forceinline__ uint2 e4m3x4_to_half4(uint32_t w) {
  uint2 r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
      : "=r"(r.x), "=r"(r.y) : "r"(w));
  return r;
}

// ---- append -------------------------------------------------------------------------------------------
template <typename T, int D>
__global__ void __launch_bounds__(D == 32 ? 128 : 256)
history_append_kernel(LinearOperand k, LinearOperand v, int T_new, int N, const int* start, const int* counts,
                      uint8_t* k8, uint8_t* v8, float* k_scale, float* v_scale) {
  constexpr int NT = D == 32 ? 128 : 256, PIECES = D / 16, CH = kBlock * PIECES / NT;
  __shared__ float top[NT / 32];
  const int tid = threadIdx.x, H = gridDim.y >> 1, h = blockIdx.y >> 1, b = blockIdx.z;
  const bool value = blockIdx.y & 1;
  pdl_wait();
  const int first = ld_dep(start + b);
  int n = T_new;
  if (counts != nullptr) n = min(max(ld_dep(counts + b), 0), T_new);
  if (first < 0 || first >= N) return;
  const int end = min((long long)first + n, (long long)N);       // rows past the capacity are dropped
  const int blk = first / kBlock + blockIdx.x;
  if (blk * (long long)kBlock >= end) return;
  const LinearOperand& src = value ? v : k;
  const T* rows = static_cast<const T*>(src.p) + (long long)b * src.sb + (long long)h * src.sh;
  uint8_t* cache = (value ? v8 : k8) + (((size_t)b * H + h) * N + (size_t)blk * kBlock) * D;
  float* scale = (value ? v_scale : k_scale) + ((size_t)b * H + h) * (N / kBlock) + blk;
  const int lo = max(first - blk * kBlock, 0), hi = min(end - blk * kBlock, kBlock);      // the new rows of this block
  if (lo >= hi) return;                                           // (no new row: nothing of the block changes)
  const float before = lo > 0 ? ld_dep(scale) : 0.f;

  float x[CH][16], m = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int i = tid + c * NT, row = i / PIECES, piece = i % PIECES;
    if (row >= lo && row < hi) {
      const T* p = rows + (long long)(blk * kBlock + row - first) * src.st + piece * 16;
#pragma unroll
      for (int e = 0; e < 16; e += Vec16<T>::kElems) Vec16<T>::load(p + e, &x[c][e]);
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[c][e]) < INFINITY ? fabsf(x[c][e]) : 0.f);
    }
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, s));
  if ((tid & 31) == 0) top[tid >> 5] = m;
  __syncthreads();                                                // (and every thread has read the old scale)
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) m = fmaxf(m, top[w]);
  // 448 = 1.75 * 2^8
  int e = exponent_of(m) - 8 + ((__float_as_uint(m) & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = max(e, kMinExp);
  if (lo > 0) {                                                   // at least the smallest power at or above the old scale
    const int old = exponent_of(before) + ((__float_as_uint(before) & 0x7fffffu) != 0 ? 1 : 0);
    e = max(e, min(max(old, kMinExp), kMaxExp));
  }
  const float inv = two_to(-e), moved = lo > 0 ? before * inv : 1.f;        // what the older rows' bytes are multiplied by
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int i = tid + c * NT, row = i / PIECES, piece = i % PIECES;
    uint4* at = reinterpret_cast<uint4*>(cache + row * D + piece * 16);
    uint32_t w[4];
    if (row >= lo && row < hi) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        w[q] = to_e4m3x2(x[c][4 * q] * inv, x[c][4 * q + 1] * inv) | (to_e4m3x2(x[c][4 * q + 2] * inv, x[c][4 * q + 3] * inv) << 16);
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    } else if (row < lo && moved != 1.f) {                        // older rows of the block, to the new scale
      const uint4 o = ld_dep(at);
      const uint32_t u[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t a = e4m3x2_to_half2(u[q] & 0xffffu), d = e4m3x2_to_half2(u[q] >> 16);
        const float2 fa = __half22float2(*reinterpret_cast<const __half2*>(&a)), fd = __half22float2(*reinterpret_cast<const __half2*>(&d));
        w[q] = to_e4m3x2(mul_odd(fa.x, moved), mul_odd(fa.y, moved)) | (to_e4m3x2(mul_odd(fd.x, moved), mul_odd(fd.y, moved)) << 16);
      }
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  if (tid == 0) *scale = two_to(e);
}

// ---- attention ----------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// (a, b) as NP pairs of fp16 whose sums are a and b
template <int NP> __device__ __forceinline__ void split_half(float a, float b, uint32_t (&w)[NP]) {
  w[0] = pack_half(a, b);
  if constexpr (NP == 2) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[0]));
    w[1] = pack_half(a - f.x, b - f.y);
  }
}

// (x, y) *= f, and (x, y) = (x, y) * f + (a, b), each in one instruction
__device__ __forceinline__ void mul2(float& x, float& y, float f) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %2};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(x), "+f"(y) : "f"(f));
}
__device__ __forceinline__ void fma2(float& x, float& y, float f, float a, float b) {
  asm("{\n\t.reg .b64 u, v, w;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %2};\n\tmov.b64 w, {%3, %4};\n\tfma.rn.f32x2 u, u, v, w;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "+f"(x), "+f"(y) : "f"(f), "f"(a), "f"(b));
}

constexpr int kRowsPerCta = 16, kWarps = 4, kMaxSplits = 16;
// CTAs that an SM is to hold, by registers
template <typename T, int D> constexpr int kPerSm = D == 128 ? 2 : D == 64 || sizeof(T) == 4 ? 3 : 4;
constexpr float kLift = 15.f;                      // log2 of the largest weight as fp16 holds it
constexpr float kUnlift = 0x1p-15f;

template <int D> struct HistShared {
  // A warp's rows on their way: keys of two blocks, values of one.
  struct Ring { uint8_t k[2][kBlock * D], v[kBlock * D]; };
  union {
    Ring ring[kWarps];
    struct {
      float o[kWarps][kRowsPerCta][D];             // the warps' sums; the first is the CTA's after they have joined
      float m[kWarps][kRowsPerCta], l[kWarps][kRowsPerCta];
    };
  };
};
// Which row of eight a column of the score fragment is (lane groups read keys by it, and values in its order), and
// where a row's 16-byte pieces lie, so that no two lanes of a read meet in a bank.  d = 128: a row is all banks; the four
// values' rows of a read, and the two keys' rows of eight lanes, each differ by the exclusive or.  d = 64: a row is half
// of the banks, so that even and odd rows have to take turns as well.  d = 32: values meet in pairs.
template <int D> __device__ __forceinline__ int row_of(int col) { return D == 64 ? col ^ ((col >> 1) & 1) : col; }
template <int D> __device__ __forceinline__ uint32_t piece_at(int row, int piece) {
  const int x = D == 128 ? (row & 6) ^ ((row & 1) << 2) : D == 64 ? (row >> 1) & 2 : 0;
  return (uint32_t)row * D + (uint32_t)((piece ^ x) << 4);
}
// One block's rows of 8 bits to shared memory, zeros for those that do not exist.  A turn of the warp is 512 bytes; the
// place of a lane's piece repeats with every turn (d = 128: with every second one, four rows further on).
template <int D> __device__ __forceinline__ void fetch_rows(uint8_t* dst, const uint8_t* src, int left, int lane) {
  const uint32_t to = ptx::smem_u32(dst) + piece_at<D>(lane / (D / 16), lane % (D / 16));
  const uint32_t to1 = D == 128 ? ptx::smem_u32(dst) + (piece_at<D>(lane / (D / 16), lane % (D / 16)) ^ 64) : to;
  src += lane * 16;
  if (left >= kBlock) {
#pragma unroll
    for (int i = 0; i < kBlock * D / 512; ++i)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((i & 1 ? to1 : to) + i * 512), "l"(src + i * 512) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < kBlock * D / 512; ++i) {
      const bool held = lane / (D / 16) + i * (512 / D) < left;
      const int n = held ? 16 : 0;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((i & 1 ? to1 : to) + i * 512), "l"(held ? src + i * 512 : src), "r"(n) : "memory");
    }
  }
}
__device__ __forceinline__ void rows_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void rows_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32, kPerSm<T, D>)
history_attention_kernel(LinearOperand q, T* O, long long ob, long long ot, long long oh, int M, int G, int N, int splits,
                         const uint8_t* k8, const uint8_t* v8, const float* k_scale, const float* v_scale,
                         const int* lengths, float scale, int causal) {
  constexpr int NP = sizeof(T) == 2 ? 1 : 2;       // fp16 terms of q and p
  constexpr int KS = D / 16, HALF = D < 64 ? D : 64, HALVES = D / HALF, NI = HALF / 8, KW = D < 64 ? 2 : 4;
  constexpr int KC = D < 64 ? 1 : D / 64;          // loads of a key: 8 or 16 bytes a lane
  extern __shared__ __align__(16) uint8_t smem[];
  HistShared<D>& sh = *reinterpret_cast<HistShared<D>*>(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, j = lane & 3;
  const int rt = blockIdx.x / splits, split = blockIdx.x % splits, hk = blockIdx.y, b = blockIdx.z, H = gridDim.y;
  const long long rows = (long long)M * G;

  pdl_wait();
  const int told = ld_dep(lengths + b), len = min(max(told, 0), N);
  // the row of lane group g, and the one eight below: queries r / G, head r % G of the group
  long long row[2];
  int limit[2];                                    // cached rows that it sees
  uint32_t qa[NP][KS][4];
  float qs[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    row[i] = (long long)rt * kRowsPerCta + g + 8 * i;
    const bool real = row[i] < rows;
    const long long mq = real ? row[i] / G : 0;
    const int hq = real ? (int)(row[i] - mq * G) : 0;
    limit[i] = real && causal ? (int)max(min((long long)len, (long long)told - M + mq + 1), 0ll) : len;
    const T* p = static_cast<const T*>(q.p) + (long long)b * q.sb + mq * q.st + (long long)(hk * G + hq) * q.sh;
    float x[KS][4], top = 0.f;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const int at = D < 64 ? j * 8 + kk * 4 : (kk / 4) * 64 + j * 16 + (kk % 4) * 4;
      if constexpr (sizeof(T) == 2) {
        const uint2 w = ld_dep(reinterpret_cast<const uint2*>(p + at));
        x[kk][0] = __uint_as_float(w.x << 16); x[kk][1] = __uint_as_float(w.x & 0xffff0000u);
        x[kk][2] = __uint_as_float(w.y << 16); x[kk][3] = __uint_as_float(w.y & 0xffff0000u);
      } else {
        const float4 w = ld_dep(reinterpret_cast<const float4*>(p + at));
        x[kk][0] = w.x; x[kk][1] = w.y; x[kk][2] = w.z; x[kk][3] = w.w;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[kk][e]));
    }
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
    const int e = min(max(exponent_of(top), -126), 126);
    const float f = two_to(-e);
    qs[i] = scale * 1.4426950408889634f * two_to(e);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      uint32_t a[NP], c[NP];
      split_half<NP>(x[kk][0] * f, x[kk][1] * f, a);
      split_half<NP>(x[kk][2] * f, x[kk][3] * f, c);
#pragma unroll
      for (int t = 0; t < NP; ++t) { qa[t][kk][i] = a[t]; qa[t][kk][2 + i] = c[t]; }
    }
  }
  // blocks of the cache that the tile's last row reaches, this CTA's share of them
  int reach = len;
  if (causal) {
    const long long last = min((long long)(rt + 1) * kRowsPerCta, rows) - 1;
    reach = (int)max(min((long long)len, (long long)told - M + last / G + 1), 0ll);
  }
  const int blocks = (reach + kBlock - 1) / kBlock, per = (blocks + splits - 1) / splits;
  const int b0 = min(split * per, blocks), b1 = min(b0 + per, blocks);
  const uint8_t* kc = k8 + ((size_t)b * H + hk) * N * D;
  const uint8_t* vc = v8 + ((size_t)b * H + hk) * N * D;
  const float* ksc = k_scale + ((size_t)b * H + hk) * (N / kBlock);
  const float* vsc = v_scale + ((size_t)b * H + hk) * (N / kBlock);

  float o[HALVES][NI][4], m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
  for (int x = 0; x < HALVES; ++x)
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[x][i][e] = 0.f;

  typename HistShared<D>::Ring& ring = sh.ring[warp];
  float ks = 0.f, vs = 0.f;
  auto fetch_k = [&](int blk, int slot) {
    if (blk < b1) fetch_rows<D>(ring.k[slot], kc + (size_t)blk * kBlock * D, len - blk * kBlock, lane);
    rows_commit();
  };
  auto fetch_v = [&](int blk) {
    if (blk < b1) fetch_rows<D>(ring.v, vc + (size_t)blk * kBlock * D, len - blk * kBlock, lane);
    rows_commit();
  };
  if (b0 + warp < b1) { ks = ld_dep(ksc + b0 + warp); vs = ld_dep(vsc + b0 + warp); }
  fetch_k(b0 + warp, 0);
  fetch_v(b0 + warp);
  int slot = 0;
  for (int blk = b0 + warp; blk < b1; blk += kWarps, slot ^= 1) {
    fetch_k(blk + kWarps, slot ^ 1);
    float ks_next = 0.f, vs_next = 0.f;
    if (blk + kWarps < b1) { ks_next = ld_dep(ksc + blk + kWarps); vs_next = ld_dep(vsc + blk + kWarps); }
    const uint8_t* kp = ring.k[slot];
    const uint8_t* vp = ring.v;
    const int left = len - blk * kBlock;           // rows of the block that exist
    rows_wait<2>();                                // this block's keys (its values and the next keys may be on their way)
    __syncwarp();
    float s[8][4];
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      uint32_t w[8][KW];                           // 16 (8) bytes of eight keys: the tiles' products are independent
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        if constexpr (D < 64) {
          const uint2 u = *reinterpret_cast<const uint2*>(kp + piece_at<D>(n * 8 + row_of<D>(g), j >> 1) + (j & 1) * 8);
          w[n][0] = u.x; w[n][1] = u.y;
        } else {
          const uint4 u = *reinterpret_cast<const uint4*>(kp + piece_at<D>(n * 8 + row_of<D>(g), c * 4 + j));
          w[n][0] = u.x; w[n][1] = u.y; w[n][KW - 2] = u.z; w[n][KW - 1] = u.w;
        }
      }
#pragma unroll
      for (int kk = 0; kk < KW; ++kk)
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const uint2 y = e4m3x4_to_half4(w[n][kk]);
#pragma unroll
          for (int t = 0; t < NP; ++t) mma_f16(s[n], qa[t][c * KW + kk], y.x, y.y);
        }
    }
    // scores in log2 units, masked by position (whatever lies behind the history does not count, NaN neither)
    float top[2] = {-INFINITY, -INFINITY};
    const float f[2] = {qs[0] * ks, qs[1] * ks};
    const bool whole = __all_sync(~0u, (blk + 1) * kBlock <= min(limit[0], limit[1]));
#pragma unroll
    for (int n = 0; n < 8; ++n) { mul2(s[n][0], s[n][1], f[0]); mul2(s[n][2], s[n][3], f[1]); }
    if (!whole) {
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (blk * kBlock + n * 8 + row_of<D>(2 * j + (e & 1)) >= limit[e >> 1]) s[n][e] = -INFINITY;
    }
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; e += 2) top[e >> 1] = fmaxf(fmaxf(top[e >> 1], s[n][e]), s[n][e + 1]);
    float corr[2], ref[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 1));
      top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 2));
      const float m = fmaxf(m_run[i], top[i]);
      ref[i] = m == -INFINITY ? 0.f : m - kLift;   // a row that sees nothing yet: all its weights are 2^-inf = 0
      corr[i] = m_run[i] == -INFINITY ? 0.f : exp2f(m_run[i] - m);
      m_run[i] = m;
      l_run[i] *= corr[i];
    }
    uint32_t pa[NP][4][4];
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = NP == 1 ? ptx::fast_exp2(s[n][e] - ref[e >> 1]) : exp2f(s[n][e] - ref[e >> 1]);
        l_run[e >> 1] += x[e];
      }
      uint32_t a[NP], c[NP];
      split_half<NP>(x[0], x[1], a);
      split_half<NP>(x[2], x[3], c);
#pragma unroll
      for (int t = 0; t < NP; ++t) { pa[t][n >> 1][2 * (n & 1)] = a[t]; pa[t][n >> 1][2 * (n & 1) + 1] = c[t]; }
    }
    // a block that some of the tile's queries do not see may hold nothing yet, and its scale be anything
    if (!whole && !(fabsf(vs) < INFINITY)) vs = 0.f;
    vs *= kUnlift;                                 // the weights' lift ends here: sums over large values need the exponents
    rows_wait<1>();                                // this block's values
    __syncwarp();
    bool odd = false;                              // a value of the block that is not finite
#pragma unroll
    for (int x = 0; x < HALVES; ++x) {
      uint32_t w[4][4][HALF / 32];                 // the rows of columns 2j and 2j + 1 of two tiles; bytes g * HALF / 8 ..
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = t * 16 + (r >> 1) * 8 + row_of<D>(2 * j + (r & 1));
          if constexpr (HALF == 64) {
            const uint2 u = *reinterpret_cast<const uint2*>(vp + piece_at<D>(at, x * 4 + (g >> 1)) + (g & 1) * 8);
            w[t][r][0] = u.x; w[t][r][HALF / 32 - 1] = u.y;
          } else {
            w[t][r][0] = *reinterpret_cast<const uint32_t*>(vp + piece_at<D>(at, g >> 2) + (g & 3) * 4);
          }
        }
      if (!whole) {
        // rows that only some of the tile's queries see: a NaN among them must not reach the others through 0 * NaN
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < HALF / 32; ++c) {
              const uint32_t nan = __vcmpeq4(w[t][r][c] & 0x7f7f7f7fu, 0x7f7f7f7fu);
              odd |= nan != 0;
              w[t][r][c] &= ~nan;
            }
      }
      float c[NI][4];
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[i][e] = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < NI; i += 2) {
          const uint32_t sel = (i & 2) ? 0x7362u : 0x5140u;
          const uint2 y = e4m3x4_to_half4(__byte_perm(w[t][0][i >> 2], w[t][1][i >> 2], sel));
          const uint2 z = e4m3x4_to_half4(__byte_perm(w[t][2][i >> 2], w[t][3][i >> 2], sel));
#pragma unroll
          for (int n = 0; n < NP; ++n) { mma_f16(c[i], pa[n][t], y.x, z.x); mma_f16(c[i + 1], pa[n][t], y.y, z.y); }
        }
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          mul2(c[i][e], c[i][e + 1], vs);
          fma2(o[x][i][e], o[x][i][e + 1], corr[e >> 1], c[i][e], c[i][e + 1]);
        }
    }
    if (__any_sync(~0u, odd)) {
      for (int at = 0; at < min(left, kBlock); ++at)
#pragma unroll
        for (int x = 0; x < HALVES; ++x)
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (blk * kBlock + at < limit[e >> 1]) {
                const int d = x * 64 + (2 * j + (e & 1)) * (HALF / 8) + i;
                if ((vp[piece_at<D>(at, d >> 4) + (d & 15)] & 0x7f) == 0x7f) o[x][i][e] = __int_as_float(0x7fffffff);
              }
    }
    __syncwarp();                                  // everybody has read the values
    fetch_v(blk + kWarps);
    ks = ks_next; vs = vs_next;
  }
  rows_wait<0>();
  __syncthreads();                                 // the sums come to lie over the rows

  // ---- the warps' sums -----------------------------------------------------------------------------------
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l_run[i] += __shfl_xor_sync(~0u, l_run[i], 1);
    l_run[i] += __shfl_xor_sync(~0u, l_run[i], 2);
    if (j == 0) { sh.m[warp][g + 8 * i] = m_run[i]; sh.l[warp][g + 8 * i] = l_run[i]; }
  }
#pragma unroll
  for (int x = 0; x < HALVES; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < NI; i += 4)
        *reinterpret_cast<float4*>(&sh.o[warp][g + 8 * (e >> 1)][x * 64 + (2 * j + (e & 1)) * (HALF / 8) + i]) =
            make_float4(o[x][i][e], o[x][i + 1][e], o[x][i + 2][e], o[x][i + 3][e]);
  __syncthreads();
  constexpr int QUADS = kRowsPerCta * D / 4;
  auto weight = [](float m, float top) { return m == -INFINITY ? 0.f : exp2f(m - top); };
  if (splits > 1) {
    float4 acc[QUADS / (kWarps * 32)];
    float mm = 0.f, ll = 0.f;
#pragma unroll
    for (int c = 0; c < QUADS / (kWarps * 32); ++c) {
      const int at = tid + c * kWarps * 32, r = at / (D / 4), piece = at % (D / 4);
      float top = sh.m[0][r];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) top = fmaxf(top, sh.m[w][r]);
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = weight(sh.m[w][r], top);
        const float4 y = *reinterpret_cast<const float4*>(&sh.o[w][r][piece * 4]);
        a.x = fmaf(f, y.x, a.x); a.y = fmaf(f, y.y, a.y); a.z = fmaf(f, y.z, a.z); a.w = fmaf(f, y.w, a.w);
      }
      acc[c] = a;
    }
    if (tid < kRowsPerCta) {
      mm = sh.m[0][tid];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, sh.m[w][tid]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) ll = fmaf(weight(sh.m[w][tid], mm), sh.l[w][tid], ll);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < QUADS / (kWarps * 32); ++c) {
      const int at = tid + c * kWarps * 32;
      *reinterpret_cast<float4*>(&sh.o[0][at / (D / 4)][(at % (D / 4)) * 4]) = acc[c];
    }
    // m and l of a row side by side where one 16-byte load brings both
    if (tid < kRowsPerCta) *reinterpret_cast<float4*>(&sh.o[1][0][0] + 4 * tid) = make_float4(mm, ll, 0.f, 0.f);
    ptx::cluster_sync();
  }
  // ---- the splits' sums, a share of the tile's outputs per CTA; then the quotient ---------------------------
  const int sets = splits > 1 ? splits : kWarps;
  for (int at = tid + split * kWarps * 32; at < QUADS; at += splits * kWarps * 32) {
    const int r = at / (D / 4), piece = at % (D / 4);
    float top = -INFINITY, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float ms[kMaxSplits], ls[kMaxSplits];
#pragma unroll
    for (int w = 0; w < kMaxSplits; ++w) {
      ms[w] = -INFINITY; ls[w] = 0.f;
      if (w < sets) {
        if (splits > 1) {
          const float4 y = ptx::ld_cluster_f4(&sh.o[1][0][0] + 4 * r, w);
          ms[w] = y.x; ls[w] = y.y;
        } else {
          ms[w] = sh.m[w & (kWarps - 1)][r]; ls[w] = sh.l[w & (kWarps - 1)][r];
        }
      }
      top = fmaxf(top, ms[w]);
    }
#pragma unroll
    for (int w = 0; w < kMaxSplits; ++w) {
      if (w >= sets) break;
      const float f = weight(ms[w], top);
      const float4 y = splits > 1 ? ptx::ld_cluster_f4(&sh.o[0][r][piece * 4], w) : *reinterpret_cast<const float4*>(&sh.o[w & (kWarps - 1)][r][piece * 4]);
      l = fmaf(f, ls[w], l);
      a.x = fmaf(f, y.x, a.x); a.y = fmaf(f, y.y, a.y); a.z = fmaf(f, y.z, a.z); a.w = fmaf(f, y.w, a.w);
    }
    const long long out = (long long)rt * kRowsPerCta + r;
    if (out < rows) {
      const long long mq = out / G;
      T* p = O + (long long)b * ob + mq * ot + (long long)(hk * G + (int)(out - mq * G)) * oh + piece * 4;
      // l = 0: a query that sees no row at all (a NaN in l or m is none: it goes on to the output)
      const float inv = l == 0.f ? 0.f : 0x1p15f / l;            // (l has the lift, the sums have not)
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(p) = make_uint2(ptx::pack_bf16(a.x * inv, a.y * inv), ptx::pack_bf16(a.z * inv, a.w * inv));
      else
        *reinterpret_cast<float4*>(p) = make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
    }
  }
  if (splits > 1) ptx::cluster_sync();             // nobody leaves while its sums are read
}

template <typename T, int D>
cudaError_t launch_append_td(int B, int T_new, int H, int N, const LinearOperand& k, const LinearOperand& v, const int* start,
                             const int* counts, uint8_t* k8, uint8_t* v8, float* k_scale, float* v_scale, cudaStream_t st) {
  const int most = T_new < N ? T_new : N;          // rows past the capacity touch nothing
  const dim3 grid((most + kBlock - 2) / kBlock + 1, 2 * H, B);
  return launch_pdl(history_append_kernel<T, D>, grid, dim3(D == 32 ? 128 : 256), 0, st, k, v, T_new, N, start, counts, k8, v8, k_scale, v_scale);
}

template <typename T, int D>
cudaError_t launch_attention_td(const HistoryCall& c, cudaStream_t st) {
  const size_t smem = sizeof(HistShared<D>);
  static bool limits_set[kMaxDevicesCached] = {};
  const cudaError_t e = set_kernel_limits(reinterpret_cast<const void*>(&history_attention_kernel<T, D>), smem, limits_set);
  if (e != cudaSuccess) return e;
  const long long tiles = ((long long)c.M * c.G + kRowsPerCta - 1) / kRowsPerCta, ctas = tiles * c.H * c.B;
  static bool wide[kMaxDevicesCached] = {};        // clusters of sixteen
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return cudaErrorInvalidDevice;
  if (dev >= kMaxDevicesCached || !wide[dev]) {
    const cudaError_t w = cudaFuncSetAttribute(reinterpret_cast<const void*>(&history_attention_kernel<T, D>), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (w != cudaSuccess) return w;
    if (dev < kMaxDevicesCached) wide[dev] = true;
  }
  // The rows are split while the CTAs still run at once and each warp has a block.  Clusters of sixteen only where half
  // of the GPU's CTAs are enough: they need sixteen SMs of one group at the same time (256 queries of one user over
  // 10240 x 128: 31 us in sixteens, 21 in eights).
  const long long room = (long long)kNumSMs * kPerSm<T, D>;
  int splits = 1;
  while (splits < kMaxSplits && ctas * splits * 2 <= (splits == 8 ? room / 2 : room) && c.N / kBlock >= splits * 2 * kWarps) splits *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * splits), c.H, c.B);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, history_attention_kernel<T, D>, c.q, static_cast<T*>(c.o), c.ob, c.ot, c.oh, c.M, c.G, c.N, splits,
                            c.k8, c.v8, c.k_scale, c.v_scale, c.lengths, c.scale, c.causal);
}

}  // namespace

cudaError_t launch_history_append(int B, int T_new, int H, int N, int d, solar_dtype_t dt, const LinearOperand& k, const LinearOperand& v,
                                  const int* start, const int* counts, uint8_t* k8, uint8_t* v8, float* k_scale, float* v_scale,
                                  cudaStream_t st) {
#define SOLAR_APPEND(TT, DD) return launch_append_td<TT, DD>(B, T_new, H, N, k, v, start, counts, k8, v8, k_scale, v_scale, st)
  if (dt == SOLAR_BF16) {
    if (d == 32) SOLAR_APPEND(__nv_bfloat16, 32);
    if (d == 64) SOLAR_APPEND(__nv_bfloat16, 64);
    SOLAR_APPEND(__nv_bfloat16, 128);
  }
  if (d == 32) SOLAR_APPEND(float, 32);
  if (d == 64) SOLAR_APPEND(float, 64);
  SOLAR_APPEND(float, 128);
#undef SOLAR_APPEND
}

cudaError_t launch_history_attention(int d, solar_dtype_t dt, const HistoryCall& c, cudaStream_t st) {
  if (dt == SOLAR_BF16) {
    if (d == 32) return launch_attention_td<__nv_bfloat16, 32>(c, st);
    if (d == 64) return launch_attention_td<__nv_bfloat16, 64>(c, st);
    return launch_attention_td<__nv_bfloat16, 128>(c, st);
  }
  if (d == 32) return launch_attention_td<float, 32>(c, st);
  if (d == 64) return launch_attention_td<float, 64>(c, st);
  return launch_attention_td<float, 128>(c, st);
}

}  // namespace solar
