// Linear attention with a decay per head (the paper's Table 1 column beside SVD-attention, with the recency weight
// that a state carried from event to event needs):
//   S_t = g S_{t-1} + k_t v_t^T   [d,d],   o_t = scale q_t S_t,   g = exp(log_decay[h])
// in chunks of C tokens, so that the products run on the tensor cores: with S the state before a chunk,
//   o_t  = scale ( sum_{s <= t} g^(t-s) (q_t . k_s) v_s  +  g^(t+1) q_t S )        t, s within the chunk
//   S   <- g^n S + sum_s g^(n-1-s) k_s v_s^T                                        n tokens in the chunk
//
// The backward pass is the same kernel in three roles.  With R_t = g R_{t+1} + scale q_t do_t^T (R_{T} from the
// gradient of the last state),
//   dq_t = scale S_t do_t              = forward(q := do, k := v, v := k), the state being S^T
//   dk_t = R_t v_t                     = forward in reversed time (q := v, k := do, v := q), the state R^T
//   dv_t = R_t^T k_t                   = forward in reversed time (q := k, k := q, v := do), the state R
// and the gradient of the first state is g R_0.  In reversed time the state that comes in has no step of its own:
// its weight is g^x, not g^(x+1) (`off`), and the same power goes into what a chunk adds.
//
// Long histories of few heads are cut into up to kMaxSegments segments whose CTAs form a cluster: each sums up its own
// segment's state first (keys and values only), reads the others' through distributed shared memory, and then makes
// its outputs.  So there is no workspace, no second launch and no order that changes between runs.
//
// Arithmetic: warp-level bf16 MMAs, fp32 accumulators; the state lives in fp32 accumulators over the whole segment.
//   bf16 storage: q, k, v enter as they are; g^(n-1-s) k is split into two or three bf16 terms (16 or 24 bits: the state is
//   returned in fp32); the scores behind their decay and the state as an operand of q S are rounded to bf16, as the
//   output will be.
//   fp32 storage: every operand is split into three bf16 terms (24 bits), six products each: fp32's own rounding.
//
// Half of the warps (state_warp) carry the state, the others make the outputs of a chunk from the operand that those have
// left: the two chains of a chunk run side by side, one barrier a chunk.  16 x 10240 events, 4 heads of 64: 159 us
// (2.1 TB/s); where segments are not needed (8 x 2560, 37 heads) 104 us, 3.7 TB/s.  Bound by those chains, about 3000 cycles
// each for 400 instructions of a warp alone on its scheduler (a CTA alone on an SM takes 1.9 us a chunk, two 2.6): mma.sync
// is busy 41 %, shared memory 40 %, neither fewer products (-25 %) nor earlier loads moved it.  d = 128: 16 warps an SM, 3.5 to
// 4.3 us a chunk, of which the products need 2.2 (16 x 10240, 4 heads: 510 us).  fp32 storage, 16 x 10240, 4 heads of 32, 64, 128: 273,
// 631, 2102 us; its tiles go through registers and none is on its way while one is worked on.
#include <cuda_bf16.h>

#include <type_traits>

#include "sm100_ptx.cuh"
#include "solar_internal.cuh"

namespace solar {
namespace {

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t (&x)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&x)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// zeros where `real` is false (the address is then not read)
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool real) {
  const int n = real ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// (a, b) as NP pairs of bf16 whose sums are a and b, to 8 NP bits
template <int NP> __device__ __forceinline__ void split(float a, float b, uint32_t (&w)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    w[p] = ptx::pack_bf16(a, b);
    a -= lo_f(w[p]);
    b -= hi_f(w[p]);
  }
}

// (x, y) *= f in one instruction
__device__ __forceinline__ void mul2(float& x, float& y, float f) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %2};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}" : "+f"(x), "+f"(y) : "f"(f));
}

// (x, y) = (x, y) f + (a, b)
__device__ __forceinline__ void fma2(float& x, float& y, float f, float a, float b) {
  asm("{\n\t.reg .b64 u, v, w;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %2};\n\tmov.b64 w, {%3, %4};\n\tfma.rn.f32x2 u, u, v, w;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "+f"(x), "+f"(y) : "f"(f), "f"(a), "f"(b));
}
__device__ __forceinline__ void add4(float (&x)[4], const float (&t)[4]) {
  const float2 u = ptx::add2(make_float2(x[0], x[1]), make_float2(t[0], t[1])), v = ptx::add2(make_float2(x[2], x[3]), make_float2(t[2], t[3]));
  x[0] = u.x; x[1] = u.y; x[2] = v.x; x[3] = v.y;
}
// A 16 x 16 tile of the product of split operands: the smallest terms first, in
// accumulators of its own.  The tensor cores cut a sum off rather than round it, every time and at the size of what it
// has come to, so long sums are made of these tiles by ordinary additions.  Relative to 64 bits: fp32 outputs 1.4e-6 to
// 4e-6 with the sums in the tensor cores' accumulators, 1.2e-7 to 2.5e-7 so; states of 10240 events 3.2e-6 and 3.5e-7.
template <int NA, int NB>
__device__ __forceinline__ void tile_product(float (&t0)[4], float (&t1)[4], const uint32_t (&a)[NA][4], const uint32_t (&y)[NB][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) t0[i] = t1[i] = 0.f;
#pragma unroll
  for (int order = NA - 1; order >= 0; --order) {
#pragma unroll
    for (int pb = NB - 1; pb >= 0; --pb) {
      const int pa = order - pb;
      if (pa < 0) continue;
      mma(t0, a[pa], y[pb][0], y[pb][1]);
      mma(t1, a[pa], y[pb][2], y[pb][3]);
    }
  }
}

template <typename T, int D> struct LaCfg {
  static constexpr int NP = sizeof(T) == 2 ? 1 : 3;            // bf16 terms of an element
  static constexpr int C = (NP == 3 && D == 128) ? 32 : 64;    // tokens of a chunk (fp32, d = 128: by shared memory)
  static constexpr int NW = D == 128 ? 8 : 4, NTS = NW * 32, NT = 2 * NTS;      // warps of the state, and as many of the outputs
  static constexpr int RW = C / 16, CW = NW / RW, OC = D / CW; // warps over rows and over columns of the output tile
  static constexpr int MT = D / 16, NH = NW / MT, SC = D / NH; // warps over rows and over columns of the state
  static constexpr int PITCH = 2 * D + 16;                     // bytes of a row: 16-byte pieces, no bank conflicts
  static constexpr int TILE = C * PITCH, OPER = NP * TILE;     // one plane, one operand
  static constexpr int STAGES = NP == 1 ? 2 : 1;
  static constexpr int SBUF = NP == 1 ? 2 : 1;                 // copies of the state as an operand
  static constexpr int STATE = NP * D * PITCH;
  static constexpr int SLOTS = NP == 1 ? 8 : 4;                // keys and values of two pairs of chunks, or of one
  static constexpr int OFF_S = STAGES * 3 * OPER, OFF_W = SLOTS * OPER > OFF_S + SBUF * STATE ? SLOTS * OPER : OFF_S + SBUF * STATE;
  static constexpr int OFF_K = OFF_W + (C + 4) * 4;            // the keys' weights
  static constexpr size_t SMEM = OFF_K + 2 * C * 4;
  static constexpr int PER_SM = D == 32 && NP == 1 ? 3 : D < 128 ? 2 : 1;
  static_assert(PER_SM * (SMEM + 1024) <= 228 * 1024, "shared memory");
  static_assert(STAGES * 3 * OPER >= D * D * 4, "the segments' states lie over the tiles");
};

template <typename T, int D>
__global__ void __launch_bounds__(LaCfg<T, D>::NT, LaCfg<T, D>::PER_SM)
linear_attention_kernel(const __grid_constant__ LinearParams prm) {
  using F = LaCfg<T, D>;
  constexpr int C = F::C, NP = F::NP, NT = F::NT, PITCH = F::PITCH;
  extern __shared__ __align__(16) uint8_t smem[];
  const uint32_t sbase = ptx::smem_u32(smem);
  float* sw = reinterpret_cast<float*>(smem + F::OFF_W);       // g^0 .. g^C
  float* swk = reinterpret_cast<float*>(smem + F::OFF_K);      // what a chunk's keys enter the state with, then zeros
  const int tid = threadIdx.x, warp = (tid >> 5) % F::NW, lane = tid & 31, g = lane >> 2, j = lane & 3;
  const bool state_warp = tid < F::NTS;
  const int seg = blockIdx.x, segs = gridDim.x;
  const int h = blockIdx.y / prm.roles, b = blockIdx.z;
  const LinearRole& R = prm.role[blockIdx.y % prm.roles];
  const int rev = R.reverse;

  pdl_wait();
  const float l2 = ld_dep(prm.log_decay + h) * 1.4426950408889634f;
  int len = prm.T;
  if (prm.lengths != nullptr) len = min(max(ld_dep(prm.lengths + b), 0), prm.T);
  auto power = [&](int n) { return n == 0 ? 1.f : exp2f((float)n * l2); };      // (0 * -inf: a head that forgets at once)
  for (int i = tid; i <= C; i += NT) sw[i] = power(i);
  for (int i = tid; i < 2 * C; i += NT) swk[i] = i < C ? R.ak * power(C - 1 - i + rev) : 0.f;

  const int chunks = (len + C - 1) / C, per = (chunks + segs - 1) / segs;
  const int c0 = min(seg * per, chunks), c1 = min(c0 + per, chunks);
  const T* qp = static_cast<const T*>(R.q.p) + (long long)b * R.q.sb + (long long)h * R.q.sh;
  const T* kp = static_cast<const T*>(R.k.p) + (long long)b * R.k.sb + (long long)h * R.k.sh;
  const T* vp = static_cast<const T*>(R.v.p) + (long long)b * R.v.sb + (long long)h * R.v.sh;
  T* op = static_cast<T*>(R.o) + (long long)b * R.ob + (long long)h * R.oh;

  // chunk c of an operand to shared memory: rows behind the sequence are zeros
  auto load = [&](const T* p, long long st, int c, uint32_t dst) {
    if constexpr (NP == 1) {
      constexpr int PIECES = D / 8, ROWS = NT / PIECES;            // rows of 16-byte pieces per turn
      const int x0 = tid / PIECES, piece = tid % PIECES, at0 = c * C + x0;
      const long long step = rev ? -st : st;
      const T* from = p + (long long)(rev ? len - 1 - at0 : at0) * st + piece * 8;
      const uint32_t to = dst + x0 * PITCH + piece * 16;
      if ((c + 1) * C <= len) {
#pragma unroll
        for (int i = 0; i < C / ROWS; ++i) cp_async16(to + i * ROWS * PITCH, from + i * ROWS * step);
      } else {
#pragma unroll
        for (int i = 0; i < C / ROWS; ++i) {
          const bool real = at0 + i * ROWS < len;
          cp_async16_or_zero(to + i * ROWS * PITCH, real ? from + i * ROWS * step : p, real);
        }
      }
    } else {
      constexpr int PIECES = D / 4;
#pragma unroll 4
      for (int i = tid; i < C * PIECES; i += NT) {
        const int x = i / PIECES, piece = i % PIECES, at = c * C + x;
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at < len) f = ld_dep(reinterpret_cast<const float4*>(p + (long long)(rev ? len - 1 - at : at) * st + piece * 4));
        uint32_t w0[NP], w1[NP];
        split<NP>(f.x, f.y, w0);
        split<NP>(f.z, f.w, w1);
#pragma unroll
        for (int n = 0; n < NP; ++n)
          *reinterpret_cast<uint2*>(smem + (dst - sbase) + n * F::TILE + x * PITCH + piece * 8) = make_uint2(w0[n], w1[n]);
      }
    }
  };

  const uint32_t tile0 = sbase;
  auto oper = [&](int stage, int which) { return tile0 + (uint32_t)(stage * 3 + which) * F::OPER; };
  auto all = [&] { asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory"); };     // every warp of the CTA, wherever it stands
  auto load_kv = [&](int c, int stage) { load(kp, R.k.st, c, oper(stage, 1)); load(vp, R.v.st, c, oper(stage, 2)); };
  const int ldm_r = lane & 7, ldm_m = lane >> 3;
  const uint32_t off_mn = (uint32_t)((((ldm_m >> 1) * 8 + ldm_r) * PITCH) + (ldm_m & 1) * 16);   // rows by bit 1, columns by bit 0
  const uint32_t off_nm = (uint32_t)((((ldm_m & 1) * 8 + ldm_r) * PITCH) + (ldm_m >> 1) * 16);   // rows by bit 0, columns by bit 1
  // The chunks of a loop: `before` a chunk's tiles are needed, and `after` they have been read (bf16: the next chunk is on
  // its way meanwhile).  Both kinds of warps walk through them with the same barriers.
  auto start = [&](int c) {
    if (NP != 1 || c >= c1) return;
    load(qp, R.q.st, c, oper(0, 0));
    load_kv(c, 0);
    cp_async_commit();
  };
  auto before = [&](int c) {
    const int stage = NP == 1 ? (c - c0) & 1 : 0;
    if constexpr (NP == 1) {
      cp_async_wait<0>();
      all();
      if (c + 1 < c1) {
        load(qp, R.q.st, c + 1, oper(stage ^ 1, 0));
        load_kv(c + 1, stage ^ 1);
        cp_async_commit();
      }
    } else {
      load(qp, R.q.st, c, oper(0, 0));
      load_kv(c, 0);
      all();
    }
    return stage;
  };
  auto after = [&] { if constexpr (NP != 1) all(); };
  all();                                                           // the powers

  // ---- the state: this warp's 16 rows x SC columns ---------------------------------------------------
  const int mt = warp % F::MT, nh = warp / F::MT;
  float st[F::SC / 8][4];
#pragma unroll
  for (int n = 0; n < F::SC / 8; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) st[n][i] = 0.f;
  // bf16 storage: three terms of a decayed key, and sums outside of the state's accumulators (of the chunk, d = 128: of
  // 16 events, by registers), go in where they count, in the state that is returned.  A chunk with events behind it, whose
  // own last event they let decay to less than 2^-3, gets two terms straight into the accumulators (2.4e-6 of its sum, which
  // is an eighth of that in a state of events of one size), as all do where no state is returned.
  auto update_as = [&](uint32_t sk, uint32_t sv, int n_real, auto kind) {
    constexpr int TERMS = decltype(kind)::value;
    constexpr bool NEAR = NP == 1 && TERMS == 3 && D < 128, EXACT = NP == 3 || (TERMS == 3 && D == 128);
    const float gn = sw[n_real];
    float t[NEAR ? F::SC / 8 : 1][4];   // bf16, the chunk's own sum
    if constexpr (NEAR) {
#pragma unroll
      for (auto& x : t) x[0] = x[1] = x[2] = x[3] = 0.f;
    }
    if constexpr (!NEAR) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n) { mul2(st[n][0], st[n][1], gn); mul2(st[n][2], st[n][3], gn); }
    }
    const float* wk = swk + (C - n_real) + 2 * j;
#pragma unroll(EXACT || D == 128 ? 1 : C / 16)
    for (int ks = 0; ks < C / 16; ++ks) {          // (one after the other where registers are short)
      const float w[4] = {wk[ks * 16], wk[ks * 16 + 1], wk[ks * 16 + 8], wk[ks * 16 + 9]};   // of tokens 2j, 2j+1, 2j+8, 2j+9
      uint32_t a[TERMS][4];
      {
        uint32_t x[NP][4];
#pragma unroll
        for (int p = 0; p < NP; ++p) ldsm_t(x[p], sk + p * F::TILE + ks * 16 * PITCH + mt * 32 + off_mn);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float u = lo_f(x[NP - 1][i]), v = hi_f(x[NP - 1][i]);
#pragma unroll
          for (int p = NP - 2; p >= 0; --p) { u += lo_f(x[p][i]); v += hi_f(x[p][i]); }
          uint32_t y[TERMS];
          split<TERMS>(u * w[(i >> 1) * 2], v * w[(i >> 1) * 2 + 1], y);
#pragma unroll
          for (int p = 0; p < TERMS; ++p) a[p][i] = y[p];
        }
      }
      if constexpr (EXACT) {
#pragma unroll
        for (int n2 = 0; n2 < F::SC / 16; ++n2) {
          uint32_t y[NP][4];
          float t[2][4];
#pragma unroll
          for (int pb = 0; pb < NP; ++pb) ldsm_t(y[pb], sv + pb * F::TILE + ks * 16 * PITCH + (nh * F::SC + n2 * 16) * 2 + off_nm);
          tile_product<TERMS, NP>(t[0], t[1], a, y);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            add4(st[2 * n2 + x], t[x]);
          }
        }
      } else {
        uint32_t y[F::SC / 16][4];
#pragma unroll
        for (int n2 = 0; n2 < F::SC / 16; ++n2) ldsm_t(y[n2], sv + ks * 16 * PITCH + (nh * F::SC + n2 * 16) * 2 + off_nm);
#pragma unroll
        for (int pa = TERMS - 1; pa >= 0; --pa)    // (an accumulator's next product is SC / 8 products away)
#pragma unroll
          for (int n2 = 0; n2 < F::SC / 16; ++n2) {
            mma(NEAR ? t[NEAR ? 2 * n2 : 0] : st[2 * n2], a[pa], y[n2][0], y[n2][1]);
            mma(NEAR ? t[NEAR ? 2 * n2 + 1 : 0] : st[2 * n2 + 1], a[pa], y[n2][2], y[n2][3]);
          }
      }
    }
    if constexpr (NEAR) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n) { fma2(st[n][0], st[n][1], gn, t[n][0], t[n][1]); fma2(st[n][2], st[n][3], gn, t[n][2], t[n][3]); }
    }
  };
  auto update = [&](uint32_t sk, uint32_t sv, int c) {
    const int n_real = min(C, len - c * C);
    if constexpr (NP == 1) {
      const int after = len - (c + 1) * C;         // events behind the chunk; the last one is the state as it is returned
      if (R.s1 == nullptr || (after > 0 && (float)after * l2 < -3.f)) {
        update_as(sk, sv, n_real, std::integral_constant<int, 2>{});
        return;
      }
    }
    update_as(sk, sv, n_real, std::integral_constant<int, 3>{});
  };

  // ---- the segment's own state, where somebody needs it: both kinds of warps, a chunk of a pair each ------------
  if (segs > 1 && seg < segs - 1) {
    const int pairs = (c1 - c0 + 1) / 2;
    auto slot = [&](int pair, int half, int which) { return tile0 + (uint32_t)((NP == 1 ? (pair & 1) * 4 : 0) + half * 2 + which) * F::OPER; };
    auto load_pair = [&](int pair) {
      for (int half = 0; half < 2 && c0 + 2 * pair + half < c1; ++half) {
        load(kp, R.k.st, c0 + 2 * pair + half, slot(pair, half, 0));
        load(vp, R.v.st, c0 + 2 * pair + half, slot(pair, half, 1));
      }
      if (NP == 1) cp_async_commit();
    };
    auto fade = [&](float f) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n) { mul2(st[n][0], st[n][1], f); mul2(st[n][2], st[n][3], f); }
    };
    if (NP == 1) load_pair(0);
    for (int pair = 0; pair < pairs; ++pair) {
      if constexpr (NP == 1) {
        cp_async_wait<0>();
        all();
        if (pair + 1 < pairs) load_pair(pair + 1);
      } else {
        load_pair(pair);
        all();
      }
      const int at = (c0 + 2 * pair) * C, n0 = min(C, len - at), n1 = c0 + 2 * pair + 1 < c1 ? min(C, len - at - C) : 0;
      if (!state_warp) fade(sw[n0]);
      const int mine = state_warp ? n0 : n1;
      if (mine > 0) update(slot(pair, state_warp ? 0 : 1, 0), slot(pair, state_warp ? 0 : 1, 1), c0 + 2 * pair + (state_warp ? 0 : 1));
      if (state_warp) fade(sw[n1]);
      if (NP != 1) all();
    }
    // one sum of the two: this CTA's, for the cluster
    all();
    float4* own = reinterpret_cast<float4*>(smem) + tid % F::NTS;
    if (!state_warp) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n) own[n * F::NTS] = make_float4(st[n][0], st[n][1], st[n][2], st[n][3]);
    }
    all();
    if (state_warp) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n) {
        const float4 e = own[n * F::NTS];
        own[n * F::NTS] = make_float4(st[n][0] + e.x, st[n][1] + e.y, st[n][2] + e.z, st[n][3] + e.w);
      }
    }
  }

  if (state_warp) {
    // ---- the state before this segment ----------------------------------------------------------------
    const size_t state_at = ((size_t)b * prm.H + h) * D * D;
    auto state_row = [&](int i) { return mt * 16 + g + (i >> 1) * 8; };
    auto state_col = [&](int n, int i) { return nh * F::SC + n * 8 + 2 * j + (i & 1); };
    if (segs > 1) {
      ptx::cluster_sync();
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) st[n][i] = 0.f;
      const int rows = min(c0 * C, len);
      for (int m = 0; m < seg; ++m) {                              // in the segments' order
        const int end = min(min((m + 1) * per, chunks) * C, len);
        const float f = power(rows - end);
        if (m * per >= chunks) break;
#pragma unroll
        for (int n = 0; n < F::SC / 8; ++n) {
          const float4 e = ptx::ld_cluster_f4(reinterpret_cast<const float4*>(smem) + n * F::NTS + tid, m);
          st[n][0] = fmaf(f, e.x, st[n][0]); st[n][1] = fmaf(f, e.y, st[n][1]);
          st[n][2] = fmaf(f, e.z, st[n][2]); st[n][3] = fmaf(f, e.w, st[n][3]);
        }
      }
      ptx::cluster_sync();                                         // the tiles may be written again
    }
    if (R.s0 != nullptr) {
      const float f = power(min(c0 * C, len));
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          st[n][i] = fmaf(f, ld_dep(R.s0 + state_at + (size_t)state_row(i) * R.s0_r + (size_t)state_col(n, i) * R.s0_c), st[n][i]);
    }
    // The state as an operand: its accumulators rounded to NP bf16 terms
    auto put_state = [&](int buf) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t y[NP];
          split<NP>(st[n][2 * half], st[n][2 * half + 1], y);
#pragma unroll
          for (int p = 0; p < NP; ++p)
            *reinterpret_cast<uint32_t*>(smem + F::OFF_S + buf * F::STATE + p * D * PITCH + state_row(2 * half) * PITCH + state_col(n, 0) * 2) = y[p];
        }
    };
    put_state(0);
    start(c0);
    for (int c = c0; c < c1; ++c) {
      const int stage = before(c);
      update(oper(stage, 1), oper(stage, 2), c);
      after();
      if (c + 1 < c1) put_state(F::SBUF == 2 ? (c + 1 - c0) & 1 : 0);
    }
    if (R.s1 != nullptr && seg == segs - 1) {
#pragma unroll
      for (int n = 0; n < F::SC / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) R.s1[state_at + (size_t)state_row(i) * D + state_col(n, i)] = st[n][i];
    }
  } else {
    // ---- outputs, chunk by chunk ----------------------------------------------------------------------
    if (segs > 1) {
      ptx::cluster_sync();
      ptx::cluster_sync();
    }
    const int cw = warp / F::RW, rw0 = warp % F::RW, rw = F::CW > 1 ? (cw & 1 ? F::RW - 1 - rw0 : rw0) : (warp + seg + h) % F::RW;
    // What this thread's eight scores of a 16 x 16 tile are multiplied by: on the diagonal (zero above it), and, but for a
    // power of g^16, below it.
    float near[8], far[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int gap = g + ((i >> 1) & 1) * 8 - (2 * j + (i & 1) + (i >> 2) * 8);
      near[i] = gap >= 0 ? R.ap * power(gap) : 0.f;
      far[i] = R.ap * power(16 + gap);
    }
    start(c0);
    for (int c = c0; c < c1; ++c) {
      const int stage = before(c), buf = F::SBUF == 2 ? (c - c0) & 1 : 0;
      const uint32_t sq = oper(stage, 0), sk = oper(stage, 1), sv = oper(stage, 2), ss = sbase + F::OFF_S + buf * F::STATE;

      float o[F::OC / 8][4];
#pragma unroll
      for (int n = 0; n < F::OC / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
      uint32_t q[NP == 1 ? D / 16 : 1][4];           // (three terms: read where they are used)
      auto query = [&](int ks, uint32_t (&x)[NP][4]) {
#pragma unroll
        for (int p = 0; p < NP; ++p) ldsm(x[p], sq + p * F::TILE + rw * 16 * PITCH + ks * 32 + off_nm);
      };
      if constexpr (NP == 1) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) ldsm(q[ks], sq + rw * 16 * PITCH + ks * 32 + off_nm);
      }
      // q S, then its rows' powers
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t qa[NP][4];
        if constexpr (NP != 1) query(ks, qa);
#pragma unroll
        for (int n2 = 0; n2 < F::OC / 16; ++n2) {
          uint32_t y[NP][4];
#pragma unroll
          for (int pb = 0; pb < NP; ++pb) ldsm_t(y[pb], ss + pb * D * PITCH + ks * 16 * PITCH + (cw * F::OC + n2 * 16) * 2 + off_nm);
          if constexpr (NP == 1) {
            mma(o[2 * n2], q[ks], y[0][0], y[0][1]);
            mma(o[2 * n2 + 1], q[ks], y[0][2], y[0][3]);
          } else {
            float t[2][4];
            tile_product<NP, NP>(t[0], t[1], qa, y);
            add4(o[2 * n2], t[0]);
            add4(o[2 * n2 + 1], t[1]);
          }
        }
      }
      const int t0 = rw * 16 + g, t1 = t0 + 8;
      {
        const float f0 = R.aq * sw[t0 + 1 - rev], f1 = R.aq * sw[t1 + 1 - rev];
#pragma unroll
        for (int n = 0; n < F::OC / 8; ++n) { mul2(o[n][0], o[n][1], f0); mul2(o[n][2], o[n][3], f1); }
      }
      // Scores of 16 keys at a time, decayed, times their values.  bf16: straight-line code for each number of tiles that
      // a warp's rows have, so that the products of all of them are in flight together.
      if constexpr (NP == 1) {
        auto tiles = [&](auto number) {
          constexpr int KT = decltype(number)::value;
          float z[KT][2][4];
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[kt][0][i] = z[kt][1][i] = 0.f;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
              uint32_t y[4];
              ldsm(y, sk + kt * 16 * PITCH + ks * 32 + off_mn);
              mma(z[kt][0], q[ks], y[0], y[1]);
              mma(z[kt][1], q[ks], y[2], y[3]);
            }
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            uint32_t a[4];
            if (kt == KT - 1) {
#pragma unroll
              for (int i = 0; i < 4; ++i) { z[kt][0][i] *= near[i]; z[kt][1][i] *= near[4 + i]; }
            } else {
              const float f = sw[16 * (KT - 2 - kt)];
#pragma unroll
              for (int i = 0; i < 4; ++i) { z[kt][0][i] *= f * far[i]; z[kt][1][i] *= f * far[4 + i]; }
            }
            a[0] = ptx::pack_bf16(z[kt][0][0], z[kt][0][1]); a[1] = ptx::pack_bf16(z[kt][0][2], z[kt][0][3]);
            a[2] = ptx::pack_bf16(z[kt][1][0], z[kt][1][1]); a[3] = ptx::pack_bf16(z[kt][1][2], z[kt][1][3]);
#pragma unroll
            for (int n2 = 0; n2 < F::OC / 16; ++n2) {
              uint32_t y[4];
              ldsm_t(y, sv + kt * 16 * PITCH + (cw * F::OC + n2 * 16) * 2 + off_nm);
              mma(o[2 * n2], a, y[0], y[1]);
              mma(o[2 * n2 + 1], a, y[2], y[3]);
            }
          }
        };
        static_assert(F::RW == 4, "rows of a chunk over four warps");
        if (rw == 0) tiles(std::integral_constant<int, 1>{});
        else if (rw == 1) tiles(std::integral_constant<int, 2>{});
        else if (rw == 2) tiles(std::integral_constant<int, 3>{});
        else tiles(std::integral_constant<int, 4>{});
      } else {
#pragma unroll
      for (int kt = 0; kt < C / 16; ++kt) {
        if (kt > rw) break;
        float p0[4] = {0.f, 0.f, 0.f, 0.f}, p1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t qa[NP][4], y[NP][4];
          float t[2][4];
          query(ks, qa);
#pragma unroll
          for (int pb = 0; pb < NP; ++pb) ldsm(y[pb], sk + pb * F::TILE + kt * 16 * PITCH + ks * 32 + off_mn);
          tile_product<NP, NP>(t[0], t[1], qa, y);
          add4(p0, t[0]);
          add4(p1, t[1]);
        }
        if (kt == rw) {
#pragma unroll
          for (int i = 0; i < 4; ++i) { p0[i] *= near[i]; p1[i] *= near[4 + i]; }
        } else {
          const float f = sw[16 * (rw - kt - 1)];
#pragma unroll
          for (int i = 0; i < 4; ++i) { p0[i] *= f * far[i]; p1[i] *= f * far[4 + i]; }
        }
        uint32_t a[NP][4];
        {
          uint32_t y[NP];
          split<NP>(p0[0], p0[1], y);
#pragma unroll
          for (int p = 0; p < NP; ++p) a[p][0] = y[p];
          split<NP>(p0[2], p0[3], y);
#pragma unroll
          for (int p = 0; p < NP; ++p) a[p][1] = y[p];
          split<NP>(p1[0], p1[1], y);
#pragma unroll
          for (int p = 0; p < NP; ++p) a[p][2] = y[p];
          split<NP>(p1[2], p1[3], y);
#pragma unroll
          for (int p = 0; p < NP; ++p) a[p][3] = y[p];
        }
#pragma unroll
        for (int n2 = 0; n2 < F::OC / 16; ++n2) {
          uint32_t y[NP][4];
          float t[2][4];
#pragma unroll
          for (int pb = 0; pb < NP; ++pb) ldsm_t(y[pb], sv + pb * F::TILE + kt * 16 * PITCH + (cw * F::OC + n2 * 16) * 2 + off_nm);
          tile_product<NP, NP>(t[0], t[1], a, y);
          add4(o[2 * n2], t[0]);
          add4(o[2 * n2 + 1], t[1]);
        }
      }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int at = c * C + (half ? t1 : t0);
        if (at < len) {
          T* row = op + (long long)(rev ? len - 1 - at : at) * R.ot + cw * F::OC + 2 * j;
#pragma unroll
          for (int n = 0; n < F::OC / 8; ++n) {
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(row + n * 8) = ptx::pack_bf16(o[n][2 * half], o[n][2 * half + 1]);
            else *reinterpret_cast<float2*>(row + n * 8) = make_float2(o[n][2 * half], o[n][2 * half + 1]);
          }
        }
      }
      after();
    }
  }

  // ---- the rows behind the sequence -------------------------------------------------------------------
  constexpr int PIECES = D * (int)sizeof(T) / 16;
  for (long long i = (long long)seg * NT + tid; i < (long long)(prm.T - len) * PIECES; i += (long long)segs * NT)
    *reinterpret_cast<uint4*>(op + (len + i / PIECES) * R.ot + (i % PIECES) * (16 / sizeof(T))) = make_uint4(0, 0, 0, 0);
}

constexpr int kMaxSegments = 16;     // CTAs of a cluster

// Segments per (user, head): the shortest estimate, waves x time of a CTA in tenths of a microsecond: 31 to start and end and 16 a
// chunk; where the history is segmented 25 a chunk, the sums of its keys and values coming first, and 11 more for every CTA
// of the cluster.  Sixteen CTAs only where all clusters find their SMs at once.  us a launch, 4 heads of 64 of one user: 200
// events 9.6 whole, 10.2 in four; 1000 events 29, 25, 17.5, 16.4 in one, two, four, eight; 3000 events 26 in eight, 28 in
// sixteen; 10240 events 99 in four, 46 in sixteen.  These are the times of d = 64 in bf16; d = 128 and fp32 storage take two to
// four times as long for a chunk, segmented or not, so that the start and the cluster count for less there than they are taken for.
template <typename F> int linear_segments(long long ctas, int T) {
  const int chunks = (T + F::C - 1) / F::C;
  const long long slots = (long long)kNumSMs * F::PER_SM;
  long long best = -1;
  int segs = 1;
  for (int s = 1; s <= kMaxSegments && s <= chunks; s += s < 8 ? 1 : 8) {
    if (s == 16 && ctas * s > kNumSMs) break;
    const long long waves = (ctas * s + slots - 1) / slots;
    const long long per = (chunks + s - 1) / s, cost = waves * (31 + (s > 1 ? 25 * per + 11 * s : 16 * per));
    if (best < 0 || cost < best) { best = cost; segs = s; }
  }
  return segs;
}

template <typename T, int D> cudaError_t launch_td(const LinearParams& prm, int B, cudaStream_t st) {
  using F = LaCfg<T, D>;
  static bool limits_set[kMaxDevicesCached] = {};
  const cudaError_t e = set_kernel_limits(reinterpret_cast<const void*>(&linear_attention_kernel<T, D>), F::SMEM, limits_set);
  if (e != cudaSuccess) return e;
  static bool wide[kMaxDevicesCached] = {};        // clusters of sixteen
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return cudaErrorInvalidDevice;
  if (dev >= kMaxDevicesCached || !wide[dev]) {
    const cudaError_t w = cudaFuncSetAttribute(reinterpret_cast<const void*>(&linear_attention_kernel<T, D>), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (w != cudaSuccess) return w;
    if (dev < kMaxDevicesCached) wide[dev] = true;
  }
  const int segs = linear_segments<F>((long long)B * prm.H * prm.roles, prm.T);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(segs, prm.H * prm.roles, B);
  cfg.blockDim = dim3(F::NT);
  cfg.dynamicSmemBytes = F::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = segs; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = segs > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, linear_attention_kernel<T, D>, prm);
}

// ---- one event ------------------------------------------------------------------------------------------
// S <- g S + k v^T, o = scale q S: 32 columns of one state per CTA, 256 threads as 32 row threads x 8 pieces of four
// columns.  Bound by the state's bytes, once in and once out; every thread's rows are loaded before the first is used.
template <typename T, int D>
__global__ void __launch_bounds__(256)
linear_step_kernel(LinearOperand q, LinearOperand k, LinearOperand v, const float* __restrict__ log_decay, float scale,
                   float* state, T* o, long long ob, long long oh, int H) {
  constexpr int ROWS = D / 32;
  __shared__ float4 part[8][8];
  const int tid = threadIdx.x, col = tid & 7, row = tid >> 3, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y, b = blockIdx.z, c0 = blockIdx.x * 32 + col * 4;
  pdl_wait();
  float4* S = reinterpret_cast<float4*>(state + ((size_t)b * H + h) * D * D + c0) ;
  float4 s[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) s[i] = ld_dep(S + (size_t)(row + 32 * i) * (D / 4));
  const T* qp = static_cast<const T*>(q.p) + (long long)b * q.sb + (long long)h * q.sh;
  const T* kp = static_cast<const T*>(k.p) + (long long)b * k.sb + (long long)h * k.sh;
  const T* vp = static_cast<const T*>(v.p) + (long long)b * v.sb + (long long)h * v.sh;
  const float gm = expf(ld_dep(log_decay + h));
  const float v0 = to_f32(vp[c0]), v1 = to_f32(vp[c0 + 1]), v2 = to_f32(vp[c0 + 2]), v3 = to_f32(vp[c0 + 3]);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const float kk = to_f32(kp[row + 32 * i]), qq = to_f32(qp[row + 32 * i]);
    s[i].x = fmaf(kk, v0, gm * s[i].x); s[i].y = fmaf(kk, v1, gm * s[i].y);
    s[i].z = fmaf(kk, v2, gm * s[i].z); s[i].w = fmaf(kk, v3, gm * s[i].w);
    acc.x = fmaf(qq, s[i].x, acc.x); acc.y = fmaf(qq, s[i].y, acc.y);
    acc.z = fmaf(qq, s[i].z, acc.z); acc.w = fmaf(qq, s[i].w, acc.w);
    S[(size_t)(row + 32 * i) * (D / 4)] = s[i];
  }
#pragma unroll
  for (int m = 8; m < 32; m <<= 1) {
    acc.x += __shfl_xor_sync(~0u, acc.x, m); acc.y += __shfl_xor_sync(~0u, acc.y, m);
    acc.z += __shfl_xor_sync(~0u, acc.z, m); acc.w += __shfl_xor_sync(~0u, acc.w, m);
  }
  if (lane < 8) part[warp][lane] = acc;
  __syncthreads();
  if (tid < 32) {
    const float* p = reinterpret_cast<const float*>(part) + tid;
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) x += p[w * 32];
    o[(long long)b * ob + (long long)h * oh + blockIdx.x * 32 + tid] = from_f32<T>(scale * x);
  }
}

template <typename T, int D>
cudaError_t launch_step_td(int B, int H, const LinearOperand& q, const LinearOperand& k, const LinearOperand& v,
                           const float* log_decay, float scale, float* state, void* o, long long ob, long long oh, cudaStream_t st) {
  return launch_pdl(linear_step_kernel<T, D>, dim3(D / 32, H, B), dim3(256), 0, st, q, k, v, log_decay, scale, state,
                    static_cast<T*>(o), ob, oh, H);
}

}  // namespace

cudaError_t launch_linear_attention(int B, int d, solar_dtype_t dt, const LinearParams& prm, cudaStream_t st) {
  if (dt == SOLAR_BF16) {
    if (d == 32) return launch_td<__nv_bfloat16, 32>(prm, B, st);
    if (d == 64) return launch_td<__nv_bfloat16, 64>(prm, B, st);
    return launch_td<__nv_bfloat16, 128>(prm, B, st);
  }
  if (d == 32) return launch_td<float, 32>(prm, B, st);
  if (d == 64) return launch_td<float, 64>(prm, B, st);
  return launch_td<float, 128>(prm, B, st);
}

cudaError_t launch_linear_step(int B, int H, int d, solar_dtype_t dt, const LinearOperand& q, const LinearOperand& k,
                               const LinearOperand& v, const float* log_decay, float scale, float* state, void* o,
                               long long ob, long long oh, cudaStream_t st) {
#define SOLAR_STEP(TT, DD) return launch_step_td<TT, DD>(B, H, q, k, v, log_decay, scale, state, o, ob, oh, st)
  if (dt == SOLAR_BF16) {
    if (d == 32) SOLAR_STEP(__nv_bfloat16, 32);
    if (d == 64) SOLAR_STEP(__nv_bfloat16, 64);
    SOLAR_STEP(__nv_bfloat16, 128);
  }
  if (d == 32) SOLAR_STEP(float, 32);
  if (d == 64) SOLAR_STEP(float, 64);
  SOLAR_STEP(float, 128);
#undef SOLAR_STEP
}

}  // namespace solar
