// The optimizer of what is not projected (embedding, head, norm weights, biases): AdamW over many tensors at once with moments in fp32
// or in 8 bits, and the global gradient norm with its clip coefficient.
//
//   k_adamw            t <- t + 1; u <- b1 u + (1 - b1) s g; v <- b2 v + (1 - b2)(s g)^2; W <- W - lr ((u / c1) / (sqrt(v / c2) + eps) + wd W)
//                      and, by its last workgroup, step count and bias corrections of the next step
//   k_moments          8-bit moments <-> the fp32 array [u | v]
//   k_norm_part, k_norm_sum   sqrt(sum g^2) and min(1, max / norm)
#include "fullrank.h"

#include <algorithm>
#include <cmath>
#include <memory>
#include <vector>

namespace lordo {

// Elements of one tensor that a workgroup takes: 4096, or 1024 where those would be less than 1024 workgroups (four a compute unit).  In us, 1024 and 4096, at 128, 512,
// 1024 and 8192 chunks of 4096 with bf16 gradients: 8-bit moments 6.0 and 8.0, 10.3 and 11.0, 16.2 and 15.1, 101 and 87; fp32 ones, which either suits (within 4 %),
// 5.5 and 5.8, 11.0 and 10.5, 19.5 and 18.8, 144 and 145.
constexpr int64_t ADAMW_CHUNK = 4096, ADAMW_SMALL_CHUNK = 1024, ADAMW_MANY = 1024;
constexpr int Q8_BLOCK = 128;            // elements that share an exponent
constexpr int GROUP = 200;               // tensors of one launch, and gradients by rows among them: their pointers travel in the kernel arguments (below 4 KiB)
constexpr int GROUP_ROWS = 8;
// Elements of a workgroup of the norm at a time: 16384, or 2048 where those would be less than 320 (256 compute units).  In us, 2048 and 16384: one tensor of 500000 fp32
// elements 5.7 and 6.4, 4000000 7.7 and 7.1, 16000000 18.0 and 15.0; bf16 5.7 and 6.1, 8.5 and 6.3, 17.2 and 8.8; 150 tensors of 10000 6.2 and 6.0, of 20000 13.4 and 6.7;
// short rows, the last to gain: of 768, 128 chunks of 16384 7.6 and 10.3, 256 9.8 and 10.5, 512 14.1 and 11.0.
constexpr int64_t NORM_CHUNK = 16384, NORM_SMALL_CHUNK = 2048, NORM_MANY = 320;
constexpr int NORM_BLOCKS = 1024;
// Chunks of 16384 of dense gradients, at least one a tensor, that one workgroup takes without a second launch.  It takes them one after the other, 1.0 us each (short
// ones) to 1.2.  Calls in a row in us: to 5 chunks 7.1, 6 8.2, 7 9.1, 8 10.0, 49 49, 200 vectors of 400 190; two launches 9.2 to 10.7.  In a recorded graph, without the
// host, two launches are 5.3 to 5.6 and ahead from 4 chunks on (4 6.3, 6 8.2).
constexpr int64_t NORM_ALONE = 6;
constexpr int COUNTERS = 16;             // of finished workgroups, 128 bytes apart, behind them the one of finished counters

// What the plan knows of a tensor (device memory, written once).
struct AdamwTensor {
  int64_t n, cols;
  int64_t off;             // first element in the flat state arrays, a multiple of Q8_BLOCK
  int32_t decay, pad_;
};
// Step count and what the next step takes from its bias corrections c_i = 1 - beta_i^(t + 1), kept on the device, so that a recorded step counts its replays:
//   (u / c1) / (sqrt(v / c2) + eps) = ratio u / (sqrt(v) + eps root),   ratio = sqrt(c2) / c1, root = sqrt(c2), inverse = 1 / ratio.
struct AdamwStep {
  int64_t t;
  float ratio, root, inverse, pad_;
};
__device__ inline void adamw_step_write(AdamwStep* s, int64_t t, double beta1, double beta2, int bias_correction) {
  double c1 = 1.0, c2 = 1.0;
  if (bias_correction) {
    c1 = 1.0 - int_pow(beta1, t + 1);
    c2 = 1.0 - int_pow(beta2, t + 1);
  }
  s->t = t;
  s->ratio = (float)(sqrt(c2) / c1);
  s->root = (float)sqrt(c2);
  s->inverse = (float)(c1 / sqrt(c2));
}
__global__ void k_adamw_set(AdamwStep* s, double beta1, double beta2, int bias_correction, int64_t t) {
  adamw_step_write(s, t, beta1, beta2, bias_correction);
}
hipError_t launch_adamw_set(AdamwStep* s, double beta1, double beta2, int bias_correction, int64_t t, hipStream_t stream) {
  hipLaunchKernelGGL(k_adamw_set, dim3(1), dim3(1), 0, stream, s, beta1, beta2, bias_correction, t);
  return hipGetLastError();
}

struct AdamwState {
  float *u, *v;            // moments in fp32, or
  uint8_t *cu, *cv;        // their codes and
  uint8_t *eu, *ev;        // the exponents of the blocks
};
// A gradient by rows of a launch.
struct RowsOf {
  const int32_t* index;                   // row of the tensor -> row of the data, or none if outside [0, slots); behind them row of the data -> of the tensor
  int32_t slots;
};
constexpr uint8_t G_BF16 = 1, G_ROWS = 2;  // bits of what a gradient is; above them its entry of `rows`
struct AdamwArgs {
  void* w[GROUP];
  const void* g[GROUP];
  uint8_t kind[GROUP];
  RowsOf rows[GROUP_ROWS];
  int32_t count, advance, bias_correction; // advance: the last launch of the step moves its count on
  float b1, omb1, b2, omb2, eps, lr, wd;
  double b1d, omb1d, b2d, omb2d, scale;
  const float* coef;                      // clip coefficient on the device (null: 1)
  AdamwStep* step;
  int32_t* flag;                          // latch of steps left out, and the counters 128 bytes behind it
  const AdamwTensor* tensors;             // of this group
  const int32_t* first;                   // chunks before each
  AdamwState st;
};

// ---------------------------------------------------------------------------------------
// Moments in 8 bits: 128 elements share an exponent E, 2^E >= their largest magnitude; a value is held as the exponent of |x| 2^-E and three bits of its
// mantissa, val(a) = 2^floor(a / 8) (1 + (a mod 8) / 8), a <= 0.  These are the leading bits of the number itself, so that a code is made by one addition and one
// shift of the upper half of the double, without a product: adding w 2^-17 of a step before the bits behind are cut off rounds up if the part cut off plus w 2^-17
// reaches a step.  The moments are formed in double: in fp32 their own rounding would decide codes next to a border.  Codes: u has its sign in bit 7 and
// a = code - 127, v has a = code - 255; zero is zero.
// A moment changes by 1 - beta of itself a step (1e-3 of v), far less than half a step of the grid (6 %): rounding to nearest would freeze it.  w is
// 17 mixed bits of step and element, so that a value goes up in the right share of the steps and the changes add up: over 2000 steps of pure decay the mean
// of 4096 elements is within 1 % of beta^2000.  (Turning w by a fixed fraction from step to step instead was 17 % low: which steps round up then
// depends on the step before.)
// ---------------------------------------------------------------------------------------
constexpr uint32_t Q8_STEP = 0x9E3779B1u, Q8_ELEMENT = 0xBB67AE85u;
__device__ __forceinline__ uint32_t q8_mix(uint32_t x) {       // x = step Q8_STEP + element Q8_ELEMENT
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 14);
}
constexpr int Q8_NAN = 255;              // exponent of a block that holds an infinity or a NaN (or more than 2^127): all its values are NaN

// The value of a code in units of 2^E, as the upper half of a double (the lower is zero); not of NaN blocks, which the callers see to by the exponent.
template <bool SIGNED>
__device__ __forceinline__ uint32_t q8_value(uint32_t code) {
  const uint32_t c = SIGNED ? code & 0x7f : code;
  const uint32_t hi = c ? (c - (SIGNED ? 127 : 255) + 8 * 1023) << 17 : 0;
  return SIGNED ? hi | (code & 0x80) << 24 : hi;
}
// 2^E of a block, or NaN
__device__ __forceinline__ double q8_unit(int exponent) { return __hiloint2double(exponent == Q8_NAN ? 0x7ff80000 : (exponent - 127 + 1023) << 20, 0); }

// Largest of 32 lanes, by the bits of magnitudes: integers order a NaN above everything, so it is not lost.
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t max32(uint32_t v) {
  v = max_dpp<0xB1>(v);
  v = max_dpp<0x4E>(v);
  v = max_dpp<0x141>(v);
  v = max_dpp<0x140>(v);
  const uint32_t o = (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x401F);      // lane ^ 16
  return v > o ? v : o;
}
// Exponent of the least power of two not below the magnitude with these bits, biased; 0 where all are zero.
__device__ __forceinline__ int q8_exponent(uint32_t bits) { return bits == 0 ? 0 : (int)min(((bits - 1) >> 23) + 1, (uint32_t)Q8_NAN); }

// Four moments of a thread (32 lanes are a block) -> codes; x32 are the moments in fp32, whose largest sets the exponent; w(e) the thresholds.  A wave
// with no value of u below the least one, nearly every wave, skips what such values need; v below it takes it whatever the threshold, a maximum.
template <bool SIGNED, class W>
__device__ __forceinline__ uint32_t q8_encode(const double (&x)[4], const float (&x32)[4], W w, int& exponent) {
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) most = max(most, __float_as_uint(x32[e]) & (SIGNED ? 0x7fffffffu : 0xffffffffu));
  exponent = q8_exponent(max32(most));
  const int top = 8 * (exponent + 1023 - 127) - (SIGNED ? 127 : 255);
  const uint32_t some = exponent == 0 ? 0 : SIGNED ? 0x7f7f7f7fu : 0xffffffffu;  // nothing that fp32 holds: zeros
  int code[4];
  uint32_t least = 0xffffffffu;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t m = (uint32_t)__double2hiint(x[e]) & (SIGNED ? 0x7fffffffu : 0xffffffffu);
    code[e] = (int)((m + w(e)) >> 17) - top;           // far below 0 for a zero
    if constexpr (SIGNED) {
      code[e] = max(code[e], 0);
      least = min(least, m - 1);                       // (a zero is above all)
    } else {
      code[e] = min(max(code[e], 1), (int)m);
    }
  }
  if constexpr (SIGNED) {
    // 1.25 2^-16 of 2^E in the upper half of a double
    if (__any(least < (((uint32_t)(exponent + 1023 - 127 - 16) << 20) | 2u << 17) - 1)) {
      constexpr double LEAST = 1.25 / 65536.0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double y = fabs(x[e]) * __hiloint2double((1023 + 127 - exponent) << 20, 0);
        if (y < LEAST) code[e] = (int)(((uint32_t)(int)(y * (131072.0 / LEAST)) + w(e)) >> 17);
      }
    }
  }
  // the lowest byte of each, and the signs from the highest bytes of the moments
  uint32_t codes = __builtin_amdgcn_perm(__builtin_amdgcn_perm(code[3], code[2], 0x0c0c0400), __builtin_amdgcn_perm(code[1], code[0], 0x0c0c0400), 0x05040100) & some;
  if constexpr (SIGNED) {
    const uint32_t h01 = __builtin_amdgcn_perm(__double2hiint(x[1]), __double2hiint(x[0]), 0x0c0c0703);
    const uint32_t h23 = __builtin_amdgcn_perm(__double2hiint(x[3]), __double2hiint(x[2]), 0x0c0c0703);
    codes |= __builtin_amdgcn_perm(h23, h01, 0x05040100) & 0x80808080u;
  }
  return codes;
}

// Gradient of four elements, `cnt` of them there, of a tensor whose gradient is held by rows: from (row0, col0) + ahead on.
template <bool BF16>
__device__ __forceinline__ void load_rows(const void* g, const RowsOf& rows, int64_t cols, int64_t row0, int64_t col0, uint32_t ahead, int cnt, float (&x)[4]) {
  const uint64_t c = (uint64_t)(col0 + ahead);
  int64_t row, col;
  if (cols < (int64_t(1) << 31)) {                     // then c is below 2^32
    const uint32_t q = (uint32_t)c / (uint32_t)cols;
    row = row0 + q; col = (int64_t)((uint32_t)c - q * (uint32_t)cols);
  } else {
    row = row0 + (int64_t)(c / (uint64_t)cols); col = (int64_t)(c % (uint64_t)cols);
  }
  if (cnt == 4 && col + 4 <= cols) {
    const int32_t slot = rows.index[row];
    if ((uint32_t)slot < (uint32_t)rows.slots) {
      load_quad<BF16, true>(g, slot * cols + col, x);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (e >= cnt) break;
    const int32_t slot = rows.index[row];
    if ((uint32_t)slot < (uint32_t)rows.slots) x[e] = load_element<BF16>(g, slot * cols + col);
    if (++col == cols) { col = 0; ++row; }
  }
}

// What a thread holds of four elements of W, G, u and v.
template <bool Q8> struct Quad;
template <> struct Quad<false> {
  float x[4], g[4];
  f32x4a u, v;
};
template <> struct Quad<true> {
  float x[4], g[4];
  uint32_t cu, cv;
  int eu, ev;
};
// A chunk of a tensor: addresses of its first element, so that a thread adds 32 bits.
struct Chunk {
  void* w;
  const void* g;
  const RowsOf* rows;
  float *u, *v;
  uint8_t *cu, *cv, *eu, *ev;
  int64_t cols, row0, col0;
  int32_t n;               // elements there
  uint32_t element;        // the first, of the tensor (lower 32 bits)
};
enum GradKind : int { DENSE_F32 = 0, DENSE_BF16 = G_BF16, ROWS_F32 = G_ROWS, ROWS_BF16 = G_ROWS | G_BF16 };

template <bool WBF, bool Q8, bool WHOLE, int KIND>
__device__ __forceinline__ void load_step(Quad<Q8>& q, const Chunk& c, uint32_t i) {
  constexpr bool BF16 = KIND & G_BF16;
  const int cnt = WHOLE || c.n - (int)i >= 4 ? 4 : c.n > (int)i ? c.n - (int)i : 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) q.x[e] = q.g[e] = 0.f;
  if constexpr (Q8) { q.cu = q.cv = 0; q.eu = q.ev = 0; }
  else q.u = q.v = f32x4a{0.f, 0.f, 0.f, 0.f};
  if (cnt == 0) return;
  if constexpr (Q8) {
    q.cu = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(c.cu + i));
    q.cv = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(c.cv + i));
    q.eu = c.eu[i / Q8_BLOCK];
    q.ev = c.ev[i / Q8_BLOCK];
  } else {                                             // (the state is padded to whole blocks)
    q.u = __builtin_nontemporal_load(reinterpret_cast<const f32x4a*>(c.u + i));
    q.v = __builtin_nontemporal_load(reinterpret_cast<const f32x4a*>(c.v + i));
  }
  if (cnt == 4) load_quad<WBF, true>(c.w, i, q.x);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) q.x[e] = load_element<WBF>(c.w, i + e);
  if constexpr (KIND & G_ROWS) {
    load_rows<BF16>(c.g, *c.rows, c.cols, c.row0, c.col0, i, cnt, q.g);
  } else if (cnt == 4) {
    load_quad<BF16, true>(c.g, i, q.g);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) q.g[e] = load_element<BF16>(c.g, i + e);
  }
}

struct StepScalars {
  float scale, lr, wd, eps;            // lr ratio, wd / ratio and eps root (AdamwStep)
  double omb1_scale, omb2_scale2;      // (1 - beta1) s and (1 - beta2) s^2
  uint32_t turn;
};

// u / (sqrt(v) + eps) by the approximate root and reciprocal (one unit in the last place each).  The root does not take subnormal numbers, and gives 0 or what
// it should, at most 2^-63: nothing beside an eps from 2^-38 on.  Below that the argument is scaled, and a sum of 0 (eps = 0, no gradient so far), or one that the
// reciprocal does not take, gives 0.
__device__ __forceinline__ void updates_of(const float (&u)[4], const float (&v)[4], float eps, float (&n)[4]) {
  if (eps >= 0x1p-38f) {                               // (uniform)
#pragma unroll
    for (int e = 0; e < 4; ++e) n[e] = u[e] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[e]) + eps);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool small = v[e] < 0x1p-96f;
      const float den = fmaf(__builtin_amdgcn_sqrtf(small ? v[e] * 0x1p64f : v[e]), small ? 0x1p-32f : 1.f, eps);
      n[e] = den < 0x1p-126f ? 0.f : u[e] * __builtin_amdgcn_rcpf(den);
    }
  }
}

template <bool WBF, bool Q8, bool WHOLE>
__device__ __forceinline__ void store_step(Quad<Q8>& q, const AdamwArgs& a, const Chunk& c, const StepScalars& s, const uint32_t* values, uint32_t i) {
  const int cnt = WHOLE || c.n - (int)i >= 4 ? 4 : c.n > (int)i ? c.n - (int)i : 0;
  float u[4], v[4];
  if constexpr (!Q8) {
    if (cnt == 0) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float g = s.scale * q.g[e];
      u[e] = fmaf(a.b1, q.u[e], a.omb1 * g);
      v[e] = fmaf(a.b2, q.v[e], a.omb2 * g * g);
    }
    const f32x4a nu = {u[0], u[1], u[2], u[3]}, nv = {v[0], v[1], v[2], v[3]};
    __builtin_nontemporal_store(nu, reinterpret_cast<f32x4a*>(c.u + i));
    __builtin_nontemporal_store(nv, reinterpret_cast<f32x4a*>(c.v + i));
  } else {
    // every product and sum is rounded by itself, so that codes do not depend on which of them a compiler joins
#pragma clang fp contract(off)
    double du[4], dv[4];
    const double b1 = a.b1d * q8_unit(q.eu), b2 = a.b2d * q8_unit(q.ev);
    const uint32_t mix0 = s.turn + (c.element + i) * Q8_ELEMENT;
    uint32_t mix[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double g = (double)q.g[e], g2 = g * g;
      const double ou = __hiloint2double(values[(q.cu >> (8 * e)) & 0xff], 0), ov = __hiloint2double(values[256 + ((q.cv >> (8 * e)) & 0xff)], 0);
      const double pu = b1 * ou, qu = s.omb1_scale * g, pv = b2 * ov, qv = s.omb2_scale2 * g2;
      du[e] = WHOLE || e < cnt ? pu + qu : 0.0;
      dv[e] = WHOLE || e < cnt ? pv + qv : 0.0;
      u[e] = (float)du[e]; v[e] = (float)dv[e];
      mix[e] = q8_mix(mix0 + e * Q8_ELEMENT);
    }
    int eu, ev;
    const uint32_t cu = q8_encode<true>(du, u, [&](int e) { return mix[e] >> 15; }, eu);
    const uint32_t cv = q8_encode<false>(dv, v, [&](int e) { return mix[e] & 0x1ffffu; }, ev);
    if (cnt > 0) {
      __builtin_nontemporal_store(cu, reinterpret_cast<uint32_t*>(c.cu + i));
      __builtin_nontemporal_store(cv, reinterpret_cast<uint32_t*>(c.cv + i));
      if ((threadIdx.x & 31) == 0) {
        c.eu[i / Q8_BLOCK] = (uint8_t)eu;
        c.ev[i / Q8_BLOCK] = (uint8_t)ev;
      }
    }
  }
  float n[4];
  updates_of(u, v, s.eps, n);
  // the decay joins the update, so that the weight is rounded once: W - lr ratio (n + (wd / ratio) W)
#pragma unroll
  for (int e = 0; e < 4; ++e) q.x[e] = fmaf(-s.lr, fmaf(s.wd, q.x[e], n[e]), q.x[e]);
  if (cnt == 4) store_quad<WBF, true>(c.w, i, q.x);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < cnt) store_element<WBF>(c.w, i + e, q.x[e]);
}

// The workgroup that is the last of its launch to come here.  Counters for a sixteenth of the workgroups each, so that few wait for one address; the last of each
// counts on the one behind them, and every counter is left at zero.
__device__ __forceinline__ bool last_workgroup(int32_t* counters) {
  if (gridDim.x <= 64) {                               // few: one counter
    if (atomicAdd(counters, 1) != (int32_t)gridDim.x - 1) return false;
    atomicExch(counters, 0);
    return true;
  }
  const int32_t k = (int32_t)blockIdx.x % COUNTERS, all = ((int32_t)gridDim.x - k + COUNTERS - 1) / COUNTERS;
  if (atomicAdd(counters + 32 * k, 1) != all - 1) return false;
  atomicExch(counters + 32 * k, 0);
  if (atomicAdd(counters + 32 * COUNTERS, 1) != COUNTERS - 1) return false;
  atomicExch(counters + 32 * COUNTERS, 0);
  return true;
}

template <bool WBF, bool Q8, int64_t CHUNK, int KIND>
__device__ __forceinline__ void step_chunk(const AdamwArgs& a, const Chunk& c, const StepScalars& s, const uint32_t* values) {
  // Quads requested together.  fp32 moments: bound by memory, all four of a chunk (embedding and head of a 1B model in us: 1 518, 2 507, 4 497; with
  // chunks of 2048, 2 498).  8 bits: bound by instructions, and with the registers of more of them fewer waves fit (with the export 1 974, 2 997).
  constexpr int REPS = (int)(CHUNK / 1024), AHEAD = Q8 ? 1 : REPS;
  if (c.n == CHUNK) {
#pragma unroll
    for (int rep = 0; rep < REPS; rep += AHEAD) {
      Quad<Q8> q[AHEAD];
#pragma unroll
      for (int r = 0; r < AHEAD; ++r) load_step<WBF, Q8, true, KIND>(q[r], c, (rep + r) * 1024 + threadIdx.x * 4);
#pragma unroll
      for (int r = 0; r < AHEAD; ++r) store_step<WBF, Q8, true>(q[r], a, c, s, values, (rep + r) * 1024 + threadIdx.x * 4);
    }
  } else {
    for (int rep = 0; rep < REPS && rep * 1024 < c.n; ++rep) {
      Quad<Q8> q;
      load_step<WBF, Q8, false, KIND>(q, c, rep * 1024 + threadIdx.x * 4);
      store_step<WBF, Q8, false>(q, a, c, s, values, rep * 1024 + threadIdx.x * 4);
    }
  }
}

// One pass over W, G and the moments; a workgroup a chunk of one tensor, found by its number among the chunks of all.
// fp32 moments: HBM, 24 or 20 bytes an element and its gradient.  30011 x 1023 in fp32 with vectors, bf16 gradients: 136 us, 5.9 TB/s; 2 x 32000 x 2048 in bf16:
// 497 us, 5.8 TB/s; an in-place addition of 1 GiB reaches 5.93.
// 8 bits: vector instructions.  2 x 32000 x 4096 in bf16, 10 bytes an element: 533 us, 5.0 TB/s, at 67 instructions an element that keep the vector units busy for 97 %
// of the time.  Eight elements of a block to a thread, a table of doubles or requests of the next round ahead of this one need
// fewer instructions or wait less, but 90 to 140 registers in place of 70: 560 to 605 us.
// 25 vectors of 768: 5.3 us, a chain of four loads (which tensor, its record, its elements, the count of finished workgroups).
template <bool WBF, bool Q8, int64_t CHUNK>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a) {
  // what the codes of u and v stand for, read from there at an instruction a code instead of six
  __shared__ uint32_t values[Q8 ? 512 : 1];
  if constexpr (Q8) {
    values[threadIdx.x] = q8_value<true>(threadIdx.x);
    values[256 + threadIdx.x] = q8_value<false>(threadIdx.x);
    __syncthreads();
  }
  const int32_t chunk = a.first[0] + (int32_t)blockIdx.x;
  const int k = find_tensor(a.first, a.count, chunk);
  const AdamwTensor t = a.tensors[k];
  const double scale = a.scale * (double)(a.coef ? *a.coef : 1.f);
  if (!(fabsf((float)scale) < INFINITY)) {             // the norm was not finite, or the two factors together are not: this step is left out
    if (a.advance && blockIdx.x == 0 && threadIdx.x == 0) *a.flag = 1;
    return;
  }
  StepScalars s;
  s.scale = (float)scale;
  s.omb1_scale = a.omb1d * scale;
  s.omb2_scale2 = a.omb2d * (scale * scale);
  s.lr = a.lr * a.step->ratio;
  s.wd = t.decay ? a.wd * a.step->inverse : 0.f;
  s.eps = a.eps * a.step->root;
  const int64_t steps = a.step->t;
  s.turn = (uint32_t)(steps + 1) * Q8_STEP;
  const int64_t base = (int64_t)(chunk - a.first[k]) * CHUNK, at = t.off + base;
  const uint8_t kind = a.kind[k];
  const int dense = kind & G_ROWS ? 0 : kind & G_BF16 ? 2 : 4;         // bytes of an element of a dense gradient
  Chunk c;
  c.w = reinterpret_cast<char*>(a.w[k]) + base * (WBF ? 2 : 4);
  c.g = reinterpret_cast<const char*>(a.g[k]) + base * dense;
  c.rows = &a.rows[kind >> 2];
  c.u = a.st.u + at; c.v = a.st.v + at;
  c.cu = a.st.cu + at; c.cv = a.st.cv + at;
  c.eu = a.st.eu + at / Q8_BLOCK; c.ev = a.st.ev + at / Q8_BLOCK;
  c.cols = t.cols; c.row0 = c.col0 = 0;
  c.n = (int32_t)std::min(t.n - base, CHUNK);
  c.element = (uint32_t)base;
  if (kind & G_ROWS) {
    c.row0 = base / t.cols;
    c.col0 = base - c.row0 * t.cols;
    if (kind & G_BF16) step_chunk<WBF, Q8, CHUNK, ROWS_BF16>(a, c, s, values);
    else step_chunk<WBF, Q8, CHUNK, ROWS_F32>(a, c, s, values);
  } else if (kind & G_BF16) {
    step_chunk<WBF, Q8, CHUNK, DENSE_BF16>(a, c, s, values);
  } else {
    step_chunk<WBF, Q8, CHUNK, DENSE_F32>(a, c, s, values);
  }
  if (!a.advance) return;
  // t <- t + 1, once every workgroup has read what belongs to t
  __syncthreads();
  if (threadIdx.x == 0 && last_workgroup(a.flag + 32)) adamw_step_write(a.step, steps + 1, a.b1d, a.b2d, a.bias_correction);
}

// TO_STATE: moments <- [u | v], in 8 bits with thresholds of one half (a value of the grid stays itself); else [u | v] <- moments.  What lies
// between the tensors is written as zero.  HBM: 2 x 32000 x 4096 out of 8 bits 471 us, 5.6 TB/s (2 bytes read, 8 written an element).
template <bool Q8, bool TO_STATE>
__global__ __launch_bounds__(256) void k_moments(AdamwState st, const AdamwTensor* tensors, const int32_t* first, int32_t count, int32_t chunk_elements, float* plain,
                                                 int64_t total) {
  const int32_t chunk = first[0] + (int32_t)blockIdx.x;
  const int k = find_tensor(first, count, chunk);
  const AdamwTensor t = tensors[k];
  const int64_t base = (int64_t)(chunk - first[k]) * chunk_elements, at = t.off + base;
  const int32_t n = (int32_t)std::min<int64_t>(t.n - base, chunk_elements), padded = (n + Q8_BLOCK - 1) / Q8_BLOCK * Q8_BLOCK;
  float* const pu = plain + at;
  float* const pv = plain + total + at;
  for (int rep = 0; rep * 1024 < padded; ++rep) {
    const int i = rep * 1024 + (int)threadIdx.x * 4, cnt = std::min(std::max(n - i, 0), 4);
    const bool any = i < padded;
    float u[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    if constexpr (TO_STATE) {
      if (cnt == 4) {
        load_quad<false, true>(pu, i, u);
        load_quad<false, true>(pv, i, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < cnt) { u[e] = pu[i + e]; v[e] = pv[i + e]; }
      }
      if constexpr (Q8) {
        double du[4], dv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) { du[e] = (double)u[e]; v[e] = fabsf(v[e]); dv[e] = (double)v[e]; }
        int eu, ev;
        auto half = [](int) { return 1u << 16; };
        const uint32_t cu = q8_encode<true>(du, u, half, eu), cv = q8_encode<false>(dv, v, half, ev);
        if (any) {
          *reinterpret_cast<uint32_t*>(st.cu + at + i) = cu;
          *reinterpret_cast<uint32_t*>(st.cv + at + i) = cv;
          if ((threadIdx.x & 31) == 0) {
            st.eu[(at + i) / Q8_BLOCK] = (uint8_t)eu;
            st.ev[(at + i) / Q8_BLOCK] = (uint8_t)ev;
          }
        }
      } else if (any) {
        *reinterpret_cast<f32x4a*>(st.u + at + i) = f32x4a{u[0], u[1], u[2], u[3]};
        *reinterpret_cast<f32x4a*>(st.v + at + i) = f32x4a{v[0], v[1], v[2], v[3]};
      }
    } else if (any) {
      if constexpr (Q8) {
        const int eu = st.eu[(at + i) / Q8_BLOCK], ev = st.ev[(at + i) / Q8_BLOCK];
        const uint32_t cu = *reinterpret_cast<const uint32_t*>(st.cu + at + i), cv = *reinterpret_cast<const uint32_t*>(st.cv + at + i);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < cnt) {
            u[e] = (float)(__hiloint2double(q8_value<true>((cu >> (8 * e)) & 0xff), 0) * q8_unit(eu));
            v[e] = (float)(__hiloint2double(q8_value<false>((cv >> (8 * e)) & 0xff), 0) * q8_unit(ev));
          }
      } else {
        const f32x4a x = *reinterpret_cast<const f32x4a*>(st.u + at + i), y = *reinterpret_cast<const f32x4a*>(st.v + at + i);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < cnt) { u[e] = x[e]; v[e] = y[e]; }
      }
      store_quad<false, true>(pu, i, u);
      store_quad<false, true>(pv, i, v);
    }
  }
}

// ---------------------------------------------------------------------------------------
// Global norm.  Squares of fp32 numbers overflow from 1.8e19 on and vanish below 1e-23, and a sum of 1e9 of them in fp32 would lose the small ones:
// products and sums are in double, in an order that the sizes alone fix (each thread's elements, the lanes of a wave, the waves, the workgroups).
// ---------------------------------------------------------------------------------------
struct NormArgs {
  const void* g[GROUP];
  int32_t first[GROUP];                   // chunks before each
  uint16_t missing[GROUP];                // elements that its last chunk lacks
  uint8_t kind[GROUP];
  RowsOf rows[GROUP_ROWS];
  int64_t rows_cols[GROUP_ROWS], rows_of[GROUP_ROWS];
  int32_t count, chunks, chunk, add;      // chunk: elements of one
  double max_norm;
  double* part;
  float* out;                             // one workgroup is all: it writes the result itself
};

static_assert(sizeof(NormArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ double wave_sum(double x) {
  for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
  return x;
}
// The sum over the threads of a workgroup, in thread 0.
__device__ __forceinline__ double block_sum(double x, double* sums) {
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = x;
  __syncthreads();
  if (threadIdx.x == 0) {
    x = 0.0;
    for (int k = 0; k < (int)blockDim.x / 64; ++k) x += sums[k];
  }
  return x;
}
__device__ __forceinline__ void norm_result(double sum, double max_norm, float* out) {
  const double norm = sqrt(sum);
  const float held = (float)norm;                      // (a norm above what fp32 holds is infinite: what the caller sees decides)
  out[0] = held;
  out[1] = !(held < INFINITY) ? __uint_as_float(0x7fc00000u) : norm > max_norm ? (float)(max_norm / norm) : 1.f;
}

// Squares of the elements from `base` to `end`, sixteen bytes a thread at a time, four times requested together; the last few one a thread.
template <bool BF>
__device__ __forceinline__ double squares(const void* g, int64_t base, int64_t end, int threads) {
  constexpr int VEC = BF ? 8 : 4, AHEAD = 4;
  double sum[2] = {0.0, 0.0};
  const int64_t step = (int64_t)threads * VEC, whole = end - (end - base) % VEC;
  for (int64_t i = base + (int64_t)threadIdx.x * VEC; i < whole; i += AHEAD * step) {
    Piece<BF, VEC> p[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      p[q].clear();
      if (i + q * step < whole) p[q].load(g, i + q * step);
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e & 1] = fma((double)p[q].value(e), (double)p[q].value(e), sum[e & 1]);
  }
  if (whole + threadIdx.x < end) {
    const double x = (double)load_element<BF>(g, whole + threadIdx.x);
    sum[0] = fma(x, x, sum[0]);
  }
  return sum[0] + sum[1];
}
// The same of a gradient by rows: rows that belong to no row of the tensor hold nothing.  Long rows are taken one by one, so that whether a row is there is
// asked once; of short ones each thread asks for its own.  33.5e6 elements, a third of the rows there, in us, one by one and each thread for its own: 512 columns fp32 32.4
// and 25.8, bf16 29.5 and 22.0; 1000 23.1 and 26.5, 23.2 and 22.7; 1024 22.3 and 25.6, 21.0 and 21.8; 4096 14.5 and 24.2, 12.7 and 21.5.
template <bool BF>
__device__ __forceinline__ double squares_of_rows(const void* g, const int32_t* owner, int64_t cols, int64_t base, int64_t end, int threads) {
  if (cols >= 1024) {
    double sum = 0.0;
    int64_t row = base / cols;
    for (int64_t at = base; at < end; ++row) {
      const int64_t to = std::min((row + 1) * cols, end);
      if (owner[row] >= 0) sum += squares<BF>(g, at, to, threads);
      at = to;
    }
    return sum;
  }
  // quads of columns, four a thread requested together; cols < 1024 here, so a chunk's rows and columns are 32-bit numbers
  constexpr int AHEAD = 4;
  double sum = 0.0;
  const int64_t row0 = base / cols;
  const uint32_t width = (uint32_t)cols, col0 = (uint32_t)(base - row0 * cols), n = (uint32_t)(end - base), step = (uint32_t)threads * 4;
  const int32_t* const own = owner + row0;
  for (uint32_t i = threadIdx.x * 4; i < n; i += AHEAD * step) {
    Piece<BF, 4> p[AHEAD];
    bool there[AHEAD];
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      const uint32_t c = col0 + i + q * step, row = c / width, col = c - row * width;
      there[q] = i + q * step + 4 <= n && col + 4 <= width && own[row] >= 0;
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      p[q].clear();
      if (there[q]) p[q].load(g, base + i + q * step);
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      for (int e = 0; e < 4; ++e) sum = fma((double)p[q].value(e), (double)p[q].value(e), sum);
      const uint32_t at = i + q * step, c = col0 + at;
      if (there[q] || at >= n || (at + 4 <= n && c % width + 4 <= width)) continue;
      for (uint32_t e = 0; e < 4 && at + e < n; ++e)   // over the end of a row or of the chunk: one by one
        if (own[(c + e) / width] >= 0) {
          const double x = (double)load_element<BF>(g, base + at + e);
          sum = fma(x, x, sum);
        }
    }
  }
  return sum;
}

// HBM: 1.3e9 bf16 elements in 218 tensors 425 us with the launch of k_norm_sum (5 us), 6.1 TB/s (with one request of 8 bytes in flight a thread and 64 tensors a
// launch 975).  Few chunks are one launch of one workgroup: see NORM_ALONE.
__global__ __launch_bounds__(1024) void k_norm_part(NormArgs a) {
  __shared__ double sums[16];
  double sum = 0.0;
  const int threads = (int)blockDim.x;
  int k = find_tensor(a.first, a.count, (int32_t)blockIdx.x);
  for (int32_t c = (int32_t)blockIdx.x; c < a.chunks; c += (int32_t)gridDim.x) {
    while (k + 1 < a.count && a.first[k + 1] <= c) ++k;
    const int32_t chunks = (k + 1 < a.count ? a.first[k + 1] : a.chunks) - a.first[k];
    const int64_t base = (int64_t)(c - a.first[k]) * a.chunk, end = std::min(base + a.chunk, (int64_t)chunks * a.chunk - a.missing[k]);
    const uint8_t kind = a.kind[k];
    if (kind & G_ROWS) {
      const int r = kind >> 2;
      const int32_t* owner = a.rows[r].index + a.rows_of[r];
      sum += kind & G_BF16 ? squares_of_rows<true>(a.g[k], owner, a.rows_cols[r], base, end, threads)
                           : squares_of_rows<false>(a.g[k], owner, a.rows_cols[r], base, end, threads);
    } else {
      sum += kind & G_BF16 ? squares<true>(a.g[k], base, end, threads) : squares<false>(a.g[k], base, end, threads);
    }
  }
  sum = block_sum(sum, sums);
  if (threadIdx.x != 0) return;
  if (a.out) norm_result(sum, a.max_norm, a.out);
  else a.part[blockIdx.x] = a.add ? a.part[blockIdx.x] + sum : sum;
}

__global__ __launch_bounds__(256) void k_norm_sum(const double* part, int32_t count, double max_norm, float* out) {
  __shared__ double sums[4];
  double sum = 0.0;
#pragma unroll
  for (int q = 0; q < NORM_BLOCKS / 256; ++q) sum += (int)threadIdx.x + 256 * q < count ? part[threadIdx.x + 256 * q] : 0.0;
  sum = block_sum(sum, sums);
  if (threadIdx.x == 0) norm_result(sum, max_norm, out);
}

}  // namespace lordo

using namespace lordo;

// ---------------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------------
struct lordo_adamw {
  lordo_adamw_hparams hp{};
  std::vector<lordo_tensor> shapes;
  std::vector<AdamwTensor> tensors;
  std::vector<int32_t> first;            // chunks before each tensor; the total at the end
  int64_t total = 0;                     // elements of a flat state array
  int64_t chunk = ADAMW_CHUNK;           // elements of a workgroup
  size_t bytes = 0;
  int64_t flag = 0, step = 0, table = 0, prefix = 0, u = 0, v = 0, eu = 0, ev = 0;     // byte offsets in the arena
  char* arena = nullptr;
  int device = 0;
  int64_t t = 0;
  bool step_dirty = false;

  AdamwState state() const {
    AdamwState s{};
    if (hp.state_dtype == LORDO_Q8) {
      s.cu = reinterpret_cast<uint8_t*>(arena + u); s.cv = reinterpret_cast<uint8_t*>(arena + v);
      s.eu = reinterpret_cast<uint8_t*>(arena + eu); s.ev = reinterpret_cast<uint8_t*>(arena + ev);
    } else {
      s.u = reinterpret_cast<float*>(arena + u); s.v = reinterpret_cast<float*>(arena + v);
    }
    return s;
  }
  AdamwStep* step_dev() const { return reinterpret_cast<AdamwStep*>(arena + step); }
  bool on_its_device() const {
    int cur = -1;
    return hipGetDevice(&cur) == hipSuccess && cur == device;
  }
};

namespace {

bool unit(double b) { return b >= 0 && b < 1; }

int plan_adamw(const lordo_tensor* tensors, int32_t n, const lordo_adamw_hparams* hp, lordo_adamw& c) {
  if (!tensors || !hp || n <= 0) return LORDO_EINVAL;
  if (!unit(hp->beta1) || !unit(hp->beta2) || !(hp->eps >= 0) || !std::isfinite(hp->eps) || !(hp->weight_decay >= 0) || !(hp->weight_decay <= 0x1p64))
    return LORDO_EINVAL;
  if (hp->eps > 0 && hp->eps < 0x1p-100) return LORDO_EINVAL;           // (see updates_of)
  if (hp->bias_correction != 0 && hp->bias_correction != 1) return LORDO_EINVAL;
  if (hp->param_dtype != LORDO_F32 && hp->param_dtype != LORDO_BF16) return LORDO_EINVAL;
  if ((hp->state_dtype != LORDO_F32 && hp->state_dtype != LORDO_Q8) || hp->reserved != 0) return LORDO_EINVAL;
  c.hp = *hp;
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    const lordo_tensor& s = tensors[i];
    if (s.rows <= 0 || s.cols <= 0 || s.rows > (int64_t(1) << 38) || s.cols > (int64_t(1) << 38) / s.rows) return LORDO_EINVAL;
    if ((s.decay != 0 && s.decay != 1) || s.reserved != 0) return LORDO_EINVAL;
    chunks += (s.rows * s.cols + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
    if (chunks >= int64_t(1) << 24) return LORDO_EINVAL;           // (a launch has less than 2^32 threads)
  }
  c.chunk = chunks >= ADAMW_MANY ? ADAMW_CHUNK : ADAMW_SMALL_CHUNK;
  chunks = 0;
  for (int i = 0; i < n; ++i) {
    const lordo_tensor& s = tensors[i];
    AdamwTensor t{};
    t.n = s.rows * s.cols; t.cols = s.cols; t.off = c.total; t.decay = s.decay;
    c.first.push_back((int32_t)chunks);
    c.tensors.push_back(t);
    c.total += (t.n + Q8_BLOCK - 1) / Q8_BLOCK * Q8_BLOCK;
    chunks += (t.n + c.chunk - 1) / c.chunk;
  }
  c.first.push_back((int32_t)chunks);
  c.shapes.assign(tensors, tensors + n);
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t r = at; at += (bytes + 255) & ~int64_t(255); return r; };
  c.flag = take(128 + 128 * (COUNTERS + 1));
  c.step = take(sizeof(AdamwStep));
  c.table = take((int64_t)sizeof(AdamwTensor) * n);
  c.prefix = take((int64_t)sizeof(int32_t) * (n + 1));
  if (hp->state_dtype == LORDO_Q8) {
    c.u = take(c.total); c.v = take(c.total);
    c.eu = take(c.total / Q8_BLOCK); c.ev = take(c.total / Q8_BLOCK);
  } else {
    c.u = take(8 * c.total);             // [u | v] without a gap
    c.v = c.u + 4 * c.total;
  }
  c.bytes = (size_t)at;
  return LORDO_OK;
}

bool good_grad(const lordo_grad& g) {
  if ((!g.data && !(g.index && g.slots == 0)) || g.rows <= 0 || g.cols <= 0 || g.rows > (int64_t(1) << 38) || g.cols > (int64_t(1) << 38) / g.rows) return false;
  if ((g.dtype != LORDO_F32 && g.dtype != LORDO_BF16) || g.reserved != 0) return false;
  if (g.index) {
    if (g.slots < 0 || g.slots > LORDO_MAX_TOKENS || g.rows > LORDO_MAX_VOCAB || (g.slots > 0 && g.cols > (int64_t(1) << 38) / g.slots)) return false;
  } else if (g.slots != 0) {
    return false;
  }
  return (reinterpret_cast<uintptr_t>(g.data) & (g.dtype == LORDO_F32 ? 3 : 1)) == 0 && (reinterpret_cast<uintptr_t>(g.index) & 3) == 0;
}

template <bool Q8, int64_t CHUNK>
void launch_step(bool w_bf16, dim3 grid, hipStream_t s, const AdamwArgs& a) {
  if (w_bf16) hipLaunchKernelGGL((k_adamw<true, Q8, CHUNK>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_adamw<false, Q8, CHUNK>), grid, dim3(256), 0, s, a);
}

uint8_t grad_kind(const lordo_grad& g, int rows) { return (uint8_t)((g.dtype == LORDO_BF16 ? G_BF16 : 0) | (g.index ? G_ROWS | rows << 2 : 0)); }

#define ADAMW_CHK(expr, what)                                                                     \
  do {                                                                                            \
    if ((expr) != hipSuccess) {                                                                   \
      (void)hipGetLastError();                                                                    \
      fprintf(stderr, "lordo: %s failed\n", what);                                                \
      return LORDO_EHIP;                                                                          \
    }                                                                                             \
  } while (0)

int moments(lordo_adamw* c, float* plain, bool to_state, hipStream_t s) {
  const int n = (int)c->shapes.size();
  const AdamwState st = c->state();
  for (int at = 0; at < n; at += 256) {
    const AdamwTensor* tensors = reinterpret_cast<const AdamwTensor*>(c->arena + c->table) + at;
    const int32_t* first = reinterpret_cast<const int32_t*>(c->arena + c->prefix) + at;
    const int count = std::min(256, n - at);
    const dim3 grid((unsigned)(c->first[at + count] - c->first[at])), block(256);
    if (c->hp.state_dtype == LORDO_Q8) {
      if (to_state) hipLaunchKernelGGL((k_moments<true, true>), grid, block, 0, s, st, tensors, first, count, (int32_t)c->chunk, plain, c->total);
      else hipLaunchKernelGGL((k_moments<true, false>), grid, block, 0, s, st, tensors, first, count, (int32_t)c->chunk, plain, c->total);
    } else {
      if (to_state) hipLaunchKernelGGL((k_moments<false, true>), grid, block, 0, s, st, tensors, first, count, (int32_t)c->chunk, plain, c->total);
      else hipLaunchKernelGGL((k_moments<false, false>), grid, block, 0, s, st, tensors, first, count, (int32_t)c->chunk, plain, c->total);
    }
    const int rc = launched("k_moments");
    if (rc != LORDO_OK) return rc;
  }
  return LORDO_OK;
}

}  // namespace

extern "C" {

int lordo_adamw_workspace_bytes(const lordo_tensor* tensors, int32_t n, const lordo_adamw_hparams* hp, size_t* out_bytes) {
  if (!out_bytes) return LORDO_EINVAL;
  return guarded([&] {
    lordo_adamw c;
    const int rc = plan_adamw(tensors, n, hp, c);
    if (rc == LORDO_OK) *out_bytes = c.bytes;
    return rc;
  });
}

int lordo_adamw_init(lordo_adamw** out, const lordo_tensor* tensors, int32_t n, const lordo_adamw_hparams* hp, void* arena, size_t arena_bytes, void* stream) {
  if (!out) return LORDO_EINVAL;
  *out = nullptr;
  return guarded([&]() -> int {
    std::unique_ptr<lordo_adamw> c(new lordo_adamw());
    const int rc = plan_adamw(tensors, n, hp, *c);
    if (rc != LORDO_OK) return rc;
    if (!arena || (reinterpret_cast<uintptr_t>(arena) & 255) != 0) return LORDO_EINVAL;
    if (arena_bytes < c->bytes) return LORDO_ENOMEM;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || ndev <= 0) {
      fprintf(stderr, "lordo: no HIP device available\n");
      return LORDO_EHIP;
    }
    ADAMW_CHK(hipGetDevice(&c->device), "hipGetDevice");
    c->arena = reinterpret_cast<char*>(arena);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    ADAMW_CHK(hipStreamSynchronize(s), "hipStreamSynchronize");
    ADAMW_CHK(hipMemcpy(c->arena + c->table, c->tensors.data(), sizeof(AdamwTensor) * n, hipMemcpyHostToDevice), "hipMemcpy");
    ADAMW_CHK(hipMemcpy(c->arena + c->prefix, c->first.data(), sizeof(int32_t) * (n + 1), hipMemcpyHostToDevice), "hipMemcpy");
    ADAMW_CHK(launch_fill_zero(c->arena + c->flag, c->step - c->flag, s), "fill");
    ADAMW_CHK(launch_fill_zero(c->arena + c->u, (int64_t)c->bytes - c->u, s), "fill");
    ADAMW_CHK(launch_adamw_set(c->step_dev(), hp->beta1, hp->beta2, hp->bias_correction, 0, s), "k_adamw_set");
    ADAMW_CHK(hipStreamSynchronize(s), "hipStreamSynchronize");
    *out = c.release();
    return LORDO_OK;
  });
}

int lordo_adamw_step(lordo_adamw* c, void* const* W, const lordo_grad* G, double lr, double grad_scale, const float* clip, void* stream) {
  if (!c || !W || !G || !finite_in_fp32(lr) || !finite_in_fp32(lr * c->hp.weight_decay) || !finite_in_fp32(grad_scale)) return LORDO_EINVAL;
  if (!c->on_its_device()) return LORDO_ESTATE;
  const int n = (int)c->shapes.size();
  const uintptr_t w_mask = c->hp.param_dtype == LORDO_BF16 ? 1 : 3;
  for (int i = 0; i < n; ++i) {
    if (!W[i] || (reinterpret_cast<uintptr_t>(W[i]) & w_mask) != 0 || !good_grad(G[i])) return LORDO_EINVAL;
    if (G[i].rows != c->shapes[i].rows || G[i].cols != c->shapes[i].cols) return LORDO_EINVAL;
  }
  if ((reinterpret_cast<uintptr_t>(clip) & 3) != 0) return LORDO_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (c->step_dirty) {
    // not into a recording, where every replay would set the count again
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &capture) != hipSuccess || capture != hipStreamCaptureStatusNone) {
      (void)hipGetLastError();
      return LORDO_ESTATE;
    }
    ADAMW_CHK(launch_adamw_set(c->step_dev(), c->hp.beta1, c->hp.beta2, c->hp.bias_correction, c->t, s), "k_adamw_set");
    c->step_dirty = false;      // (a call that fails below leaves the device count right: the last launch alone moves it on)
  }
  const float* const coef = clip ? clip + 1 : nullptr;
  AdamwArgs a;
  a.b1 = (float)c->hp.beta1; a.omb1 = (float)(1.0 - c->hp.beta1);
  a.b2 = (float)c->hp.beta2; a.omb2 = (float)(1.0 - c->hp.beta2);
  a.b1d = c->hp.beta1; a.omb1d = 1.0 - c->hp.beta1; a.b2d = c->hp.beta2; a.omb2d = 1.0 - c->hp.beta2;
  a.eps = (float)c->hp.eps; a.lr = (float)lr; a.wd = (float)c->hp.weight_decay;
  a.scale = grad_scale;
  a.coef = coef;
  a.step = c->step_dev();
  a.st = c->state();
  a.flag = reinterpret_cast<int32_t*>(c->arena + c->flag);
  a.bias_correction = c->hp.bias_correction;
  for (int at = 0; at < n;) {
    a.count = 0;
    for (int rows = 0; at + a.count < n && a.count < GROUP; ++a.count) {
      const lordo_grad& g = G[at + a.count];
      if (g.index && rows == GROUP_ROWS) break;
      a.w[a.count] = W[at + a.count];
      a.g[a.count] = g.data;
      a.kind[a.count] = grad_kind(g, rows);
      if (g.index) a.rows[rows++] = RowsOf{g.index, (int32_t)g.slots};
    }
    a.tensors = reinterpret_cast<const AdamwTensor*>(c->arena + c->table) + at;
    a.first = reinterpret_cast<const int32_t*>(c->arena + c->prefix) + at;
    const dim3 grid((unsigned)(c->first[at + a.count] - c->first[at]));
    at += a.count;
    a.advance = at == n;
    const bool bf = c->hp.param_dtype == LORDO_BF16;
    const bool small = c->chunk == ADAMW_SMALL_CHUNK;
    if (c->hp.state_dtype == LORDO_Q8) small ? launch_step<true, ADAMW_SMALL_CHUNK>(bf, grid, s, a) : launch_step<true, ADAMW_CHUNK>(bf, grid, s, a);
    else small ? launch_step<false, ADAMW_SMALL_CHUNK>(bf, grid, s, a) : launch_step<false, ADAMW_CHUNK>(bf, grid, s, a);
    const int rc = launched("k_adamw");
    if (rc != LORDO_OK) return rc;
  }
  ++c->t;
  return LORDO_OK;
}

int lordo_adamw_sync_payload(lordo_adamw* c, void** dev_ptr, size_t* count) {
  if (!c || !dev_ptr || !count) return LORDO_EINVAL;
  *count = 2 * (size_t)c->total;
  *dev_ptr = c->hp.state_dtype == LORDO_F32 ? c->arena + c->u : nullptr;
  return LORDO_OK;
}

int lordo_adamw_export_moments(lordo_adamw* c, float* dst, void* stream) {
  if (!c || !dst || (reinterpret_cast<uintptr_t>(dst) & 3) != 0) return LORDO_EINVAL;
  if (!c->on_its_device()) return LORDO_ESTATE;
  return moments(c, dst, false, reinterpret_cast<hipStream_t>(stream));
}

int lordo_adamw_import_moments(lordo_adamw* c, const float* src, void* stream) {
  if (!c || !src || (reinterpret_cast<uintptr_t>(src) & 3) != 0) return LORDO_EINVAL;
  if (!c->on_its_device()) return LORDO_ESTATE;
  return moments(c, const_cast<float*>(src), true, reinterpret_cast<hipStream_t>(stream));
}

int lordo_adamw_get_step(lordo_adamw* c, int64_t* t) {
  if (!c || !t) return LORDO_EINVAL;
  *t = c->t;
  return LORDO_OK;
}

int lordo_adamw_steps_taken(lordo_adamw* c, int64_t* t, void* stream) {
  if (!c || !t) return LORDO_EINVAL;
  if (!c->on_its_device()) return LORDO_ESTATE;
  ADAMW_CHK(hipStreamSynchronize(reinterpret_cast<hipStream_t>(stream)), "hipStreamSynchronize");
  int64_t taken = c->t;                                // (set, and not yet on the device)
  if (!c->step_dirty) ADAMW_CHK(hipMemcpy(&taken, &c->step_dev()->t, sizeof(taken), hipMemcpyDeviceToHost), "hipMemcpy");
  *t = taken;
  return LORDO_OK;
}

int lordo_adamw_set_step(lordo_adamw* c, int64_t t) {
  if (!c || t < 0 || t > (int64_t(1) << 62)) return LORDO_EINVAL;
  c->t = t;
  c->step_dirty = true;
  return LORDO_OK;
}

int lordo_adamw_poll_status(lordo_adamw* c, void* stream) {
  if (!c) return LORDO_EINVAL;
  if (!c->on_its_device()) return LORDO_ESTATE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ADAMW_CHK(hipStreamSynchronize(s), "hipStreamSynchronize");
  int32_t flag = 0;
  ADAMW_CHK(hipMemcpy(&flag, c->arena + c->flag, sizeof(flag), hipMemcpyDeviceToHost), "hipMemcpy");
  if (flag == 0) return LORDO_OK;
  ADAMW_CHK(launch_fill_zero(c->arena + c->flag, 16, s), "fill");
  ADAMW_CHK(hipStreamSynchronize(s), "hipStreamSynchronize");
  return LORDO_ENUMERIC;
}

void lordo_adamw_destroy(lordo_adamw* c) { delete c; }

int lordo_grad_norm(const lordo_grad* G, int32_t n, double max_norm, float* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!G || n <= 0 || !(max_norm > 0) || !out || !workspace) return LORDO_EINVAL;
  if ((reinterpret_cast<uintptr_t>(out) & 3) != 0 || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return LORDO_EINVAL;
  if (workspace_bytes < LORDO_NORM_WORKSPACE_BYTES) return LORDO_ENOMEM;
  auto elements = [](const lordo_grad& g) { return g.index ? g.slots * g.cols : g.rows * g.cols; };
  int64_t chunk = NORM_CHUNK, chunks = 0;
  bool by_rows = false;
  for (int i = 0; i < n; ++i) {
    if (!good_grad(G[i])) return LORDO_EINVAL;
    by_rows |= G[i].index != nullptr;
    chunks += (elements(G[i]) + chunk - 1) / chunk;
    if (chunks > (int64_t(1) << 30)) return LORDO_EINVAL;
  }
  const bool one = chunks <= NORM_ALONE && !by_rows;             // (so no more tensors than a launch takes)
  if (chunks < NORM_MANY && !one) {
    chunk = NORM_SMALL_CHUNK;
    chunks = 0;
    for (int i = 0; i < n; ++i) chunks += (elements(G[i]) + chunk - 1) / chunk;
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int blocks = (int)std::min<int64_t>(std::max<int64_t>(chunks, 1), NORM_BLOCKS);      // of every launch: each adds to the sums of the one before
  NormArgs a;
  a.part = reinterpret_cast<double*>(workspace);
  a.max_norm = max_norm;
  a.chunk = (int32_t)chunk;
  a.out = nullptr;
  for (int at = 0; at < n;) {
    a.count = 0;
    a.chunks = 0;
    a.add = at > 0;
    for (int rows = 0; at + a.count < n && a.count < GROUP; ++a.count) {
      const lordo_grad& g = G[at + a.count];
      if (g.index && rows == GROUP_ROWS) break;
      const int64_t m = elements(g), mine = (m + chunk - 1) / chunk;
      a.g[a.count] = g.data;
      a.first[a.count] = a.chunks;
      a.missing[a.count] = (uint16_t)(mine * chunk - m);
      a.kind[a.count] = grad_kind(g, rows);
      if (g.index) {
        a.rows[rows] = RowsOf{g.index, (int32_t)g.slots};
        a.rows_cols[rows] = g.cols;
        a.rows_of[rows++] = g.rows;
      }
      a.chunks += (int32_t)mine;
    }
    at += a.count;
    if (one) {
      a.out = out;
      hipLaunchKernelGGL(k_norm_part, dim3(1), dim3(1024), 0, s, a);
      return launched("k_norm_part");
    }
    hipLaunchKernelGGL(k_norm_part, dim3((unsigned)blocks), dim3(256), 0, s, a);
    const int rc = launched("k_norm_part");
    if (rc != LORDO_OK) return rc;
  }
  hipLaunchKernelGGL(k_norm_sum, dim3(1), dim3(256), 0, s, a.part, blocks, max_norm, out);
  return launched("k_norm_sum");
}

}  // extern "C"
