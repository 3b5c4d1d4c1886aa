// Softmax attention of many queries over the 8-bit history cache (bf16 storage, d = 64 or 128), on tcgen05:
//   O = softmax(scale Q (ks k8)^T) (vs v8)
// A CTA takes 256 (query, head of the group) rows of one cached head in two groups of 128, and walks through the cache in
// tiles of 128 rows (d = 64) or 64 rows (d = 128: tensor memory holds scores, weights and sums of both groups).
//   warps 0-7   a row per thread: the softmax
//   warps 8-13  bring the tiles: bulk copies of the 8-bit rows three tiles ahead, then to fp16 in shared memory
//               (e4m3 is exact in fp16), once for both groups
//   warps 14,15 issue a group's MMAs: S = Q K^T of the next tile, as soon as the row warps hold the present one in
//               registers, then Y += P V of the present one
// Scales.  A query row is brought below 2 by a power of two and to fp16 (exact down to 2^-14 of its largest).  With
// a = (that row's scores), z = a * (scale log2e 2^e ks) + log2 vs is the log of weight times value scale, and
//   P = 2^(z - m + 3) as fp16,   Y = sum P v8,   l = sum 2^(z - m) / vs,   O = 2^-3 Y / l
// where m is the largest z of some tile before or of this one: P is then exact to fp16's 11 bits wherever the product of weight and value
// scale is within 2^-17 of the row's largest (and to 2^-28 of that largest below), which is what the output is rounded by.  m is
// raised (Y and l rescaled) only when the weights of a block add up to more than 2^15, and so before one of them is too large
// for fp16.
// The weights of a block whose value scale lies 2^64 or more below the largest one so far (one of zeros, whose scale is 2^-100,
// beside values of any size) may vanish from 2^(z - m) although they count in l: such a block is added to l by exponentials
// of its own, relative to its own maximum, and l is rescaled in two steps where m rises by more than fp32 has exponents.
// Where the queries alone do not fill the GPU the cache's rows are split over the CTAs of a cluster, which add up through
// distributed shared memory.  Every wait is bounded; if one runs out the tile's output rows are written as NaN.
//
// 16 x 2048 queries over 10240 rows: d = 64 170 us a launch (505 TFLOP/s; 3.4e8 exponentials would take the special-function units
// 72), d = 128 235 us (730).  Bound by the row warps' chain of a tile, 2.2 us of wait, load, exponentials and store with two
// warps a scheduler to hide it: without the exponentials 113, without the conversion 170, without the products 186 us
// (d = 64, at 210 us).  Hence as little as possible in it: no maximum, no division, one fused multiplication a pair.
#include <cuda_fp16.h>

#include <climits>

#include "sm100_ptx.cuh"
#include "solar_internal.cuh"

namespace solar {
namespace {

constexpr int kBlock = SOLAR_CACHE_BLOCK;
constexpr int kGroupRows = 128, kGroups = 2, kRows = kGroupRows * kGroups;
constexpr int kConvWarp = 8, kConvWarps = 6, kMmaWarp = 14, kThreads = 512, kConvThreads = kConvWarps * 32;
constexpr int kRowRegs = 192, kOtherRegs = 64;     // 256 threads each: together what the block is launched with, 512 x 128
constexpr int kScaleWarp = kConvWarp + kConvWarps - 1;
constexpr int kStages = 3, kMaxSplits = 8;
constexpr int kBatch = 32;                         // blocks whose scales are looked at together, one a lane
constexpr float kLift = 3.f;
constexpr float kFar = 64.f;                       // a weight lost to fp32's range is then under 2^-65 of l
constexpr int kErrKv = 0x41, kErrFree = 0x42, kErrS = 0x43, kErrSf = 0x44, kErrP = 0x45, kErrY = 0x46, kErrRaw = 0x47;

template <int D> struct HfCfg {
  static constexpr int NTOK = D == 64 ? 128 : 64;               // cache rows of a tile
  static constexpr int NB = NTOK / kBlock;                      // scales of a tile
  static constexpr int KB = D / 64;                             // boxes of 64 columns
  static constexpr int Q_BYTES = kRows * D * 2, Q_BOX = kGroupRows * 128, Q_GROUP = KB * Q_BOX;
  static constexpr int BOX = NTOK * 128, OPER = KB * BOX, STAGE = 2 * OPER;
  static constexpr int MERGE = kRows * (D + 2) * 4;             // sums for the other CTAs of the cluster
  static constexpr int RAW = 2 * NTOK * D;                      // the tile as it is in the cache
  static constexpr int TILES = Q_BYTES + kStages * (STAGE + RAW);
  static constexpr size_t SMEM = (TILES > MERGE ? TILES : MERGE) + 1024;
  static constexpr int COL_S = 0, COL_P = kGroups * NTOK, COL_O = COL_P + kGroups * NTOK / 2 <= 256 ? 256 : 384;
  static constexpr int PIECES = 2 * NTOK * D / 16, PER = (PIECES + kConvThreads - 1) / kConvThreads;
  static_assert(COL_O + kGroups * D <= 512, "tensor memory");
};

__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint2 e4m3x4_to_half4(uint32_t w) {
  uint2 r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
      : "=r"(r.x), "=r"(r.y) : "r"(w));
  return r;
}

// An untiled copy of a multiple of 16 bytes, counted on `bar`
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(ptx::smem_u32(bar)) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
history_flash_kernel(const __grid_constant__ HistoryCall c, int splits) {
  using F = HfCfg<D>;
  constexpr int NTOK = F::NTOK, NB = F::NB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = base;                              // [2 groups][KB][128][128 B]
  uint8_t* sKV = base + F::Q_BYTES;                // [stages][K, V][KB][NTOK][128 B]
  uint8_t* sRaw = sKV + kStages * F::STAGE;        // [stages][K, V][NTOK][D B]
  __shared__ __align__(8) uint64_t raw_full[kStages], kv_full[kStages], kv_free[kStages], s_full[kGroups], s_free[kGroups], p_full[kGroups], y_done[kGroups], bar_end;
  // Of the blocks of this CTA's range, the last 64 looked at: ks, log2 vs, 2^-3 / vs (0 where far), 2 where vs is far below the largest
  __shared__ float4 s_scale[2 * kBatch];
  __shared__ float s_next[2][kBatch];              // ks and vs of the next 32 blocks, on their way
  __shared__ int s_odd[kStages];                   // a value that some of the tile's queries do not see is not finite
  __shared__ uint32_t s_tmem;
  __shared__ int s_err;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int split = blockIdx.x % splits, tiles = gridDim.x / splits;
  // causal: the tiles that see most come first
  const int rt = c.causal ? tiles - 1 - blockIdx.x / splits : blockIdx.x / splits;
  const int hk = blockIdx.y, b = blockIdx.z;
  const long long rows = (long long)c.M * c.G, row0 = (long long)rt * kRows;

  if (tid == 0) {
    s_err = 0;
    for (int i = 0; i < kStages; ++i) { ptx::mbar_init(&raw_full[i], 1); ptx::mbar_init(&kv_full[i], kConvWarps); ptx::mbar_init(&kv_free[i], kGroups); }
    for (int i = 0; i < kGroups; ++i) {
      ptx::mbar_init(&s_full[i], 1); ptx::mbar_init(&s_free[i], 4); ptx::mbar_init(&p_full[i], 4); ptx::mbar_init(&y_done[i], 1);
    }
    ptx::mbar_init(&bar_end, kGroups);
    ptx::fence_mbar_init();
  }
  if (warp == kMmaWarp) ptx::tmem_alloc(&s_tmem, 512);
  pdl_wait();
  const int told = ld_dep(c.lengths + b), len = min(max(told, 0), c.N);
  auto limit_of = [&](long long row) {             // cache rows that a query row sees
    if (!c.causal) return len;
    return (int)max(min((long long)len, (long long)told - c.M + row / c.G + 1), 0ll);
  };
  const int reach = limit_of(min(row0 + kRows, rows) - 1), least = c.causal ? limit_of(row0) : INT_MAX;      // rows that every query sees
  const int all = (reach + NTOK - 1) / NTOK, per = (all + splits - 1) / splits;
  const int t0 = min(split * per, all), nt = min(per, all - t0);
  const uint8_t* kc = c.k8 + ((size_t)b * c.H + hk) * c.N * D;
  const uint8_t* vc = c.v8 + ((size_t)b * c.H + hk) * c.N * D;

  // ---- this thread's query row, to fp16 in shared memory ---------------------------------------------------
  const int grp = warp >> 2, slot = tid & (kGroupRows - 1);
  const long long row = row0 + tid;
  const bool real = warp < kConvWarp && row < rows;
  const long long mq = real ? row / c.G : 0;
  const int hq = real ? hk * c.G + (int)(row - mq * c.G) : 0;
  float qs = 1.f;
  int limit = len;
  if (warp < kConvWarp) {
    uint32_t w[D / 2];
    float top = 0.f;
    if (real) {
      limit = limit_of(row);
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(c.q.p) + (long long)b * c.q.sb + mq * c.q.st + (long long)hq * c.q.sh);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint4 u = ld_dep(p + i);
        w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < D / 2; ++i) w[i] = 0;
    }
#pragma unroll
    for (int i = 0; i < D / 2; ++i)
      top = fmaxf(top, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
    const int e = top == 0.f ? 0 : min(max((int)((__float_as_uint(top) >> 23) & 0xffu) - 127, -126), 126);
    // a negative scale goes to the queries, so that a larger product is a larger score
    const float f = c.scale < 0.f ? -__int_as_float((127 - e) << 23) : __int_as_float((127 - e) << 23);
    qs = fabsf(c.scale) * 1.4426950408889634f * __int_as_float((e + 127) << 23);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      uint32_t u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        u[q] = half_pair(__uint_as_float(w[4 * i + q] << 16) * f, __uint_as_float(w[4 * i + q] & 0xffff0000u) * f);
      *reinterpret_cast<uint4*>(sQ + grp * F::Q_GROUP + (i / 8) * F::Q_BOX + ptx::swz128(slot, i % 8)) = make_uint4(u[0], u[1], u[2], u[3]);
    }
    ptx::fence_proxy_async_smem();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  volatile int* err = &s_err;
  const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
  float m_ref = -INFINITY, l_run = 0.f;

  if (warp >= kConvWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp < kMmaWarp) {
    // ---- the cache's rows: 8 bits by bulk copies, kStages tiles ahead, then to fp16 ------------------------------
    const int ct = tid - kConvWarp * 32;
    const float* ksc = c.k_scale + ((size_t)b * c.H + hk) * (c.N / kBlock);
    const float* vsc = c.v_scale + ((size_t)b * c.H + hk) * (c.N / kBlock);
    auto copy = [&](int t) {                       // (a tile may reach past the capacity, which ends with a block)
      const int first = (t0 + t) * NTOK;
      const uint32_t bytes = (uint32_t)min(NTOK, c.N - first) * D;
      ptx::mbar_arrive_expect_tx(&raw_full[t % kStages], 2 * bytes);
      bulk_load(sRaw + (t % kStages) * F::RAW, kc + (size_t)first * D, bytes, &raw_full[t % kStages]);
      bulk_load(sRaw + (t % kStages) * F::RAW + F::RAW / 2, vc + (size_t)first * D, bytes, &raw_full[t % kStages]);
    };
    // Scales are brought and looked at by the last of these warps (which converts least), 32 blocks at a time.  A tile's own ones at a
    // time, in the path of its conversion: d = 128 250 us in the place of 235.
    float lv_top = -INFINITY;                      // log2 of the largest value scale so far
    auto fetch_scales = [&](int from) {            // blocks of this CTA's range from .. from + 31
      const int blk = t0 * NB + from + lane;
      const bool held = from < nt * NB && blk * kBlock < len;
      const uint32_t n = held ? 4 : 0;             // (zeros in the place of those that are not read)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(ptx::smem_u32(&s_next[0][lane])), "l"(ksc + (held ? blk : 0)), "r"(n) : "memory");
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(ptx::smem_u32(&s_next[1][lane])), "l"(vsc + (held ? blk : 0)), "r"(n) : "memory");
    };
    auto take_scales = [&](int from) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      float ks = s_next[0][lane], vs = s_next[1][lane];         // (a lane reads what it has brought itself)
      // a block that some queries do not see may hold nothing yet, and its scale be anything
      const bool part = (t0 * NB + from + lane + 1) * kBlock > least;
      if (part && !(fabsf(ks) < INFINITY)) ks = 1.f;
      if (part && !(fabsf(vs) < INFINITY)) vs = 0.f;
      const float lv = vs < 1.1754944e-38f ? -126.f : log2f(vs);
      // the largest scale up to this block's tile, the tile's other block included
      float top = fmaxf(lv_top, NB == 2 ? fmaxf(lv, __shfl_xor_sync(0xffffffffu, lv, 1)) : lv);
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const float other = __shfl_up_sync(0xffffffffu, top, d);
        if (lane >= d) top = fmaxf(top, other);
      }
      lv_top = __shfl_sync(0xffffffffu, top, 31);
      const bool held = (t0 * NB + from + lane) * kBlock < len;
      const bool far = held && lv < top - kFar && !(part && vs == 0.f);
      s_scale[(from & kBatch) + lane] = make_float4(ks, lv, far ? 0.f : exp2f(-lv - kLift), __int_as_float(far ? 2 : 0));
    };
    int issued = 0;
    if (ct == 0)
      for (; issued < min(nt, kStages); ++issued) copy(issued);
    if (warp == kScaleWarp) fetch_scales(0);
    for (int t = 0; t < nt; ++t) {
      const int st = t % kStages, first = (t0 + t) * NTOK;
      const uint8_t* raw = sRaw + st * F::RAW;
      ptx::mbar_wait(&raw_full[st], (t / kStages) & 1, err, kErrRaw);
      if (t >= kStages) ptx::mbar_wait(&kv_free[st], (t / kStages - 1) & 1, err, kErrFree);
      __syncwarp();
      // (every row warp is past tile t - kStages: the place of the blocks 64 before is free)
      if (warp == kScaleWarp && t % (kBatch / NB) == 0) {
        take_scales(t * NB);
        fetch_scales(t * NB + kBatch);
      }
      const bool mixed = first + NTOK > least;     // some queries do not see all of the tile's rows
      bool odd = false;
#pragma unroll
      for (int i = 0; i < F::PER; ++i) {
        const int piece = ct + i * kConvThreads, at = piece % (F::PIECES / 2), r = at / (D / 16), p = at % (D / 16);
        if (piece >= F::PIECES) break;
        uint4 w = *reinterpret_cast<const uint4*>(raw + piece * 16);
        if (first + r >= len) w = make_uint4(0, 0, 0, 0);       // rows that do not exist: zeros, whatever the memory holds
        uint32_t x[4] = {w.x, w.y, w.z, w.w};
        if (mixed && piece >= F::PIECES / 2) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t nan = __vcmpeq4(x[q] & 0x7f7f7f7fu, 0x7f7f7f7fu);
            odd |= nan != 0;
            x[q] &= ~nan;
          }
        }
        uint8_t* box = sKV + st * F::STAGE + (piece < F::PIECES / 2 ? 0 : F::OPER) + (p / 4) * F::BOX;
        const uint2 a = e4m3x4_to_half4(x[0]), d = e4m3x4_to_half4(x[1]), f = e4m3x4_to_half4(x[2]), g = e4m3x4_to_half4(x[3]);
        *reinterpret_cast<uint4*>(box + ptx::swz128(r, 2 * (p % 4))) = make_uint4(a.x, a.y, d.x, d.y);
        *reinterpret_cast<uint4*>(box + ptx::swz128(r, 2 * (p % 4) + 1)) = make_uint4(f.x, f.y, g.x, g.y);
      }
      if (ct == 0) s_odd[st] = 0;
      asm volatile("bar.sync 1, %0;" ::"n"(kConvThreads) : "memory");
      if (ct == 0 && issued < nt && *err == 0) copy(issued++);  // everybody has read the tile's bytes
      if (odd) s_odd[st] = 1;
      ptx::fence_proxy_async_smem();
      ptx::mbar_arrive_warp(&kv_full[st], lane);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (ct == 0 && *err != 0)                      // a wait ran out: the copies land before the CTA leaves
      for (int t = max(0, issued - kStages); t < issued; ++t) {
        int dummy = 0;
        ptx::mbar_wait(&raw_full[t % kStages], (t / kStages) & 1, &dummy, 0);
      }
    } else if (lane == 0 && nt > 0) {
      const int x = warp - kMmaWarp;
      const uint32_t idesc_s = idesc_f16(kGroupRows, NTOK, false), idesc_y = idesc_f16(kGroupRows, D, true);
      const uint32_t q = ptx::smem_u32(sQ + x * F::Q_GROUP);
      auto scores = [&](int t) {
        const uint32_t k = ptx::smem_u32(sKV + (t % kStages) * F::STAGE);
        if (!ptx::mbar_wait(&kv_full[t % kStages], (t / kStages) & 1, err, kErrKv)) return false;
        ptx::tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          ptx::umma_bf16_ss(s_tmem + F::COL_S + x * NTOK, ptx::umma_smem_desc(q + (kk / 4) * F::Q_BOX + (kk % 4) * 32, 0, 1024),
                            ptx::umma_smem_desc(k + (kk / 4) * F::BOX + (kk % 4) * 32, 0, 1024), idesc_s, kk != 0);
        ptx::umma_commit(&s_full[x]);
        return true;
      };
      bool ok = scores(0);
      for (int t = 0; ok && t < nt; ++t) {
        if (t + 1 < nt) ok = ptx::mbar_wait(&s_free[x], t & 1, err, kErrSf) && scores(t + 1);
        ok = ok && ptx::mbar_wait(&p_full[x], t & 1, err, kErrP);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t v = ptx::smem_u32(sKV + (t % kStages) * F::STAGE + F::OPER);
#pragma unroll
        for (int kk = 0; kk < NTOK / 16; ++kk)
          // V rows are the inner index: 16 of them are two groups of 8 rows of 128 B; its columns come in blocks of 64
          ptx::umma_bf16_ts(s_tmem + F::COL_O + x * D, s_tmem + F::COL_P + x * (NTOK / 2) + kk * 8,
                            ptx::umma_smem_desc(v + kk * 2048, F::BOX, 1024), idesc_y, (t | kk) != 0);
        ptx::umma_commit(&y_done[x]);
        ptx::umma_commit(&kv_free[t % kStages]);
      }
      ptx::umma_commit(&bar_end);
    }
  } else {
    // ---- row warps ---------------------------------------------------------------------------------------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRowRegs));
    const uint32_t tm_s = s_tmem + lane_base + F::COL_S + grp * NTOK, tm_p = s_tmem + lane_base + F::COL_P + grp * (NTOK / 2),
                   tm_y = s_tmem + lane_base + F::COL_O + grp * D;
    for (int t = 0; t < nt; ++t) {
      const int st = t % kStages, first = (t0 + t) * NTOK;
      ptx::mbar_wait(&s_full[grp], t & 1, err, kErrS);
      __syncwarp();
      ptx::tc_fence_after_sync();
      float s[NTOK];
#pragma unroll
      for (int q = 0; q < NTOK / 32; ++q) {
        uint32_t v[32];
        ptx::tmem_ld_32x32(tm_s + q * 32, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) s[q * 32 + i] = __uint_as_float(v[i]);
      }
      ptx::tmem_ld_wait();
      ptx::mbar_wait(&kv_full[st], (t / kStages) & 1, err, kErrKv);           // long since done: the scales are read here
      float4 sc[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) sc[n] = *const_cast<const float4*>(&s_scale[(t * NB + n) & (2 * kBatch - 1)]);
      int odd = *(volatile int*)&s_odd[st];
#pragma unroll
      for (int n = 0; n < NB; ++n) odd |= __float_as_int(sc[n].w) << n;
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive_warp(&s_free[grp], lane);
      if (__any_sync(0xffffffffu, first + NTOK > limit)) {
#pragma unroll
        for (int j = 0; j < NTOK; ++j) s[j] = first + j < limit ? s[j] : -INFINITY;
      }
      float f[NB], off[NB], add;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        f[n] = qs * sc[n].x;
        f[n] = f[n] < 1.1754944e-38f ? 1.1754944e-38f : f[n];         // so that -inf stays -inf
      }
      if (t > 0) {                                 // the weights before have been read, and Y is up to date
        ptx::mbar_wait(&y_done[grp], (t - 1) & 1, err, kErrY);
        __syncwarp();
        ptx::tc_fence_after_sync();
      }
      // The weights, with the reference that the tiles before have left; only where a block's sum shows that one may be
      // too large for fp16 (or there is no reference yet) is the tile's maximum looked for, and the weights made again.
      bool look = t == 0 || __any_sync(0xffffffffu, m_ref == -INFINITY);
#pragma unroll 1
      for (int round = 0; round < 3; ++round) {
#pragma unroll
        for (int n = 0; n < NB; ++n) off[n] = sc[n].y - (m_ref == -INFINITY ? 0.f : m_ref) + kLift;
        if (look) {
          float m_tile = -INFINITY;
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            float mx[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) mx[q] = s[n * kBlock + q];
#pragma unroll
            for (int j = 4; j < kBlock; ++j) mx[j % 4] = fmaxf(mx[j % 4], s[n * kBlock + j]);
            m_tile = fmaxf(m_tile, fmaf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), f[n], sc[n].y));
          }
          const float m_new = fmaxf(m_ref, m_tile), alpha = m_ref == -INFINITY ? 0.f : ptx::fast_exp2(m_ref - m_new);
          const float root = m_ref == -INFINITY ? 0.f : ptx::fast_exp2(0.5f * (m_ref - m_new));
          m_ref = m_new;
          l_run = l_run * root * root;             // (l is up to 2^100 and more where value scales are small)
          if (t > 0) {
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 16) {
              uint32_t v[16];
              ptx::tmem_ld_32x16(tm_y + c0, v);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
              ptx::tmem_st_32x16(tm_y + c0, v);
            }
            ptx::tmem_st_wait();
          }
          const float ref = m_ref == -INFINITY ? 0.f : m_ref;
#pragma unroll
          for (int n = 0; n < NB; ++n) off[n] = sc[n].y - ref + kLift;
          if (__any_sync(0xffffffffu, fabsf(ref) > 65536.f)) {
            // scores so large that a product's rounding, which m has and the fused product below has not, is itself a factor
#pragma unroll
            for (int j = 0; j < NTOK; ++j) s[j] = fmaf(s[j], f[j / kBlock], sc[j / kBlock].y) - ref;
#pragma unroll
            for (int n = 0; n < NB; ++n) { f[n] = 1.f; off[n] = kLift; }
          }
        }
        add = 0.f;
        float most = 0.f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 f2 = make_float2(f[n], f[n]), off2 = make_float2(off[n], off[n]);
#pragma unroll
          for (int c0 = 0; c0 < kBlock; c0 += 32) {
            uint32_t w[16];
#pragma unroll
            for (int j = c0; j < c0 + 32; j += 2) {
              const float2 x = fma2(make_float2(s[n * kBlock + j], s[n * kBlock + j + 1]), f2, off2);
              const float2 e = make_float2(ptx::fast_exp2(x.x), ptx::fast_exp2(x.y));
              sum2[(j / 2) % 2] = ptx::add2(sum2[(j / 2) % 2], e);
              w[(j - c0) / 2] = half_pair(e.x, e.y);
            }
            ptx::tmem_st_32x16(tm_p + (n * kBlock + c0) / 2, w);
          }
          const float sum = (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
          most = fmaxf(most, sum);
          add = fmaf(sum, sc[n].z, add);
        }
        look = __any_sync(0xffffffffu, most > 32768.f);
        if (!look) break;
      }
      l_run += add;
      if (odd != 0) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {             // blocks whose value scale is far below the largest
          if ((odd >> (n + 1) & 1) == 0) continue;
          float top = -INFINITY, sum = 0.f;
#pragma unroll
          for (int j = 0; j < kBlock; ++j) top = fmaxf(top, fmaf(s[n * kBlock + j], f[n], off[n]));
          if (top == -INFINITY) continue;
#pragma unroll
          for (int j = 0; j < kBlock; ++j) sum += ptx::fast_exp2(fmaf(s[n * kBlock + j], f[n], off[n]) - top);
          l_run = fmaf(sum, exp2f(top - kLift - *(volatile float*)&s_scale[(t * NB + n) & (2 * kBatch - 1)].y), l_run);
        }
        if (odd & 1)                               // a value that is not finite, for the queries that see it
          for (int j = first; j < min(limit, first + NTOK); ++j)
            for (int i = 0; i < D; ++i)
              if ((vc[(size_t)j * D + i] & 0x7f) == 0x7f) l_run = __int_as_float(0x7fffffff);
      }
      ptx::tmem_st_wait();
      ptx::tc_fence_before_sync();
      ptx::mbar_arrive_warp(&p_full[grp], lane);
    }
    if (nt > 0) {
      ptx::mbar_wait(&y_done[grp], (nt - 1) & 1, err, kErrY);
      __syncwarp();
      ptx::tc_fence_after_sync();
    }
    if (*err != 0) l_run = __int_as_float(0x7fffffff);
    const float inv = l_run == 0.f ? 0.f : exp2f(-kLift) / l_run;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(c.o) + (long long)b * c.ob + mq * c.ot + (long long)hq * c.oh;
    float4* merge = reinterpret_cast<float4*>(base);          // [D / 4][256 rows] sums, then m and l: over the tiles
    if (splits > 1) asm volatile("bar.sync 2, 256;" ::: "memory");            // both groups' MMAs have read the tiles
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += 16) {
      uint32_t v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = 0;
      if (nt > 0) { ptx::tmem_ld_32x16(tm_y + c0, v); ptx::tmem_ld_wait(); }
      if (splits > 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          merge[(c0 / 4 + q) * kRows + tid] = make_float4(__uint_as_float(v[4 * q]), __uint_as_float(v[4 * q + 1]), __uint_as_float(v[4 * q + 2]), __uint_as_float(v[4 * q + 3]));
      } else if (real) {
        uint32_t x[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = ptx::pack_bf16(__uint_as_float(v[2 * q]) * inv, __uint_as_float(v[2 * q + 1]) * inv);
        *reinterpret_cast<uint4*>(out + c0) = make_uint4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<uint4*>(out + c0 + 8) = make_uint4(x[4], x[5], x[6], x[7]);
      }
    }
    if (splits > 1) reinterpret_cast<float2*>(merge + (D / 4) * kRows)[tid] = make_float2(m_ref, l_run);
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (splits > 1) {
    // ---- the splits' sums in their order, a share of the rows per CTA ------------------------------------------
    ptx::cluster_sync();
    const float2* ml = reinterpret_cast<const float2*>(reinterpret_cast<const float4*>(base) + (D / 4) * kRows);
    const int share = kRows / splits;
    for (int at = tid; at < share * (D / 8); at += kThreads) {
      const int r = split * share + at % share, piece = at / share;
      const long long out_row = row0 + r;
      if (out_row >= rows) continue;
      float ms[kMaxSplits], ls[kMaxSplits], top = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < kMaxSplits; ++w) {
        ms[w] = -INFINITY; ls[w] = 0.f;
        if (w < splits) {
          const float4 y = ptx::ld_cluster_f4(reinterpret_cast<const float4*>(ml) + r / 2, w);
          ms[w] = r & 1 ? y.z : y.x; ls[w] = r & 1 ? y.w : y.y;
        }
        top = fmaxf(top, ms[w]);
      }
      float a[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kMaxSplits; ++w) {
        if (w >= splits) break;
        const float f = ms[w] == -INFINITY ? 0.f : exp2f(ms[w] - top);
        const float root = ms[w] == -INFINITY ? 0.f : exp2f(0.5f * (ms[w] - top));
        l = fmaf(ls[w] * root, root, l);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float4 y = ptx::ld_cluster_f4(reinterpret_cast<const float4*>(base) + (2 * piece + q) * kRows + r, w);
          a[4 * q] = fmaf(f, y.x, a[4 * q]); a[4 * q + 1] = fmaf(f, y.y, a[4 * q + 1]);
          a[4 * q + 2] = fmaf(f, y.z, a[4 * q + 2]); a[4 * q + 3] = fmaf(f, y.w, a[4 * q + 3]);
        }
      }
      const float inv = l == 0.f ? 0.f : exp2f(-kLift) / l;
      const long long m = out_row / c.G;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(c.o) + (long long)b * c.ob + m * c.ot + (long long)(hk * c.G + (int)(out_row - m * c.G)) * c.oh;
      *reinterpret_cast<uint4*>(out + piece * 8) = make_uint4(ptx::pack_bf16(a[0] * inv, a[1] * inv), ptx::pack_bf16(a[2] * inv, a[3] * inv),
                                                              ptx::pack_bf16(a[4] * inv, a[5] * inv), ptx::pack_bf16(a[6] * inv, a[7] * inv));
    }
    ptx::cluster_sync();
  }
  if (warp == kMmaWarp) {
    if (nt > 0) {                                  // every MMA has ended before its tensor memory goes
      int dummy = 0;
      ptx::mbar_wait(&bar_end, 0, &dummy, 0);
      __syncwarp();
    }
    ptx::tmem_dealloc(s_tmem, 512);
  }
}

// One CTA per SM: the cache's rows are split while all CTAs still run at once (in clusters fewer do), four tiles at least
// to each.
int flash_splits(long long ctas, int tiles) {
  constexpr int kAtOnce[] = {0, 0, kNumSMs, 0, 132, 0, 0, 0, 112};
  int splits = 1;
  while (splits < kMaxSplits && ctas * splits * 2 <= kAtOnce[splits * 2] && tiles >= splits * 2 * 4) splits *= 2;
  return splits;
}

template <int D> cudaError_t launch_d(const HistoryCall& c, cudaStream_t st) {
  using F = HfCfg<D>;
  static bool limits_set[kMaxDevicesCached] = {};
  const cudaError_t e = set_kernel_limits(reinterpret_cast<const void*>(&history_flash_kernel<D>), F::SMEM, limits_set);
  if (e != cudaSuccess) return e;
  const long long tiles = ((long long)c.M * c.G + kRows - 1) / kRows;
  const int splits = flash_splits(tiles * c.H * c.B, (c.N + F::NTOK - 1) / F::NTOK);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * splits), c.H, c.B);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = F::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, history_flash_kernel<D>, c, splits);
}

}  // namespace

// Which of the two kernels a call gets: the one with the shorter estimate.  This one works on 256 rows at a time, 2.2 us a
// tile of 128 cache rows (d = 128: 1.5 us, 64 rows) wherever a CTA runs, and about 14 us to start and end; the other takes
// 1.35 ns (2.5 ns) of the GPU for 16 rows and 64 cache rows, and 6 us.  us a call, measured, the other kernel and this one:
//   d = 64    1 x 512 queries, 10240 rows      13 and 37      16 x 256, 10240    57 and 56     16 x 512, 10240   111 and 57
//             64 x 128, 2048                   29 and 29      64 x 256, 2048     46 and 32     16 x 512, 256      11 and 14
//   d = 128   16 x 128, 10240                  57 and 69      16 x 192, 10240   106 and 73     64 x 128, 2048     53 and 39
bool history_flash_supported(int d, solar_dtype_t dt, const HistoryCall& c) {
  if (dt != SOLAR_BF16 || (d != 64 && d != 128)) return false;
  const int per_tile = d == 64 ? HfCfg<64>::NTOK : HfCfg<128>::NTOK;
  const long long heads = (long long)c.H * c.B, rows = (long long)c.M * c.G;
  const long long ctas = (rows + kRows - 1) / kRows * heads;
  const int tiles = (c.N + per_tile - 1) / per_tile, splits = flash_splits(ctas, tiles);
  const double here = 14. + (double)((ctas * splits + kNumSMs - 1) / kNumSMs) * ((tiles + splits - 1) / splits) * (d == 64 ? 2.2 : 1.5);
  const double other = 6. + (double)((rows + 15) / 16) * heads * (c.N / kBlock) * (d == 64 ? 1.35e-3 : 2.5e-3);
  return here < other;
}
cudaError_t launch_history_flash(int d, const HistoryCall& c, cudaStream_t st) {
  return d == 64 ? launch_d<64>(c, st) : launch_d<128>(c, st);
}

}  // namespace solar
