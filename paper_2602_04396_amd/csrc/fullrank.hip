// The optimizer of what is not projected (embedding, head, norm weights, biases): AdamW over many tensors at once with moments in fp32
// or in 8 bits, and the global gradient norm with its clip coefficient.
//
//   k_adamw<WBF, Q8>   t <- t + 1; u <- b1 u + (1 - b1) s g; v <- b2 v + (1 - b2)(s g)^2; W <- W - lr ((u / c1) / (sqrt(v / c2) + eps) + wd W)
//   k_adamw_advance    step count and bias corrections of the next step
//   k_moments          8-bit moments <-> the fp32 array [u | v]
//   k_norm_part, k_norm_sum   sqrt(sum g^2) and min(1, max / norm)
#include "fullrank.h"

#include <algorithm>
#include <cmath>
#include <memory>
#include <vector>

namespace lordo {

constexpr int64_t ADAMW_CHUNK = 4096;    // elements of one tensor that a workgroup takes
constexpr int Q8_BLOCK = 128;            // elements that share a scale
constexpr int ADAMW_GROUP = 120;         // tensors of one launch: their pointers travel in the kernel arguments (below 4 KiB)
constexpr int NORM_GROUP = 64;
constexpr int64_t NORM_CHUNK = 8192;
constexpr int NORM_BLOCKS = 1024;

// What the plan knows of a tensor (device memory, written once).
struct AdamwTensor {
  int64_t n, cols;
  int64_t off;             // first element in the flat state arrays, a multiple of Q8_BLOCK
  int32_t decay, pad_;
};
struct AdamwState {
  float *u, *v;            // moments in fp32, or
  uint8_t *cu, *cv;        // their codes and
  uint8_t *eu, *ev;        // the exponents of the blocks
};
struct AdamwArgs {
  void* w[ADAMW_GROUP];
  const void* g[ADAMW_GROUP];
  const int32_t* index[ADAMW_GROUP];      // row of the vocabulary -> row of g, or -1 (null: g is dense)
  int32_t slots[ADAMW_GROUP];             // rows of g
  uint8_t g_bf16[ADAMW_GROUP];
  int32_t count;
  float b1, omb1, b2, omb2, eps, lr, wd;
  double b1d, omb1d, b2d, omb2d, scale;
  const float* coef;                      // clip coefficient on the device (null: 1)
  const StepDev* step;
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
__device__ __forceinline__ uint32_t q8_mix(uint32_t of_step, uint32_t element) {       // of_step: t times the first constant
  uint32_t x = of_step + element * 0xBB67AE85u;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 14);
}
constexpr uint32_t STEP_TURN = 0x9E3779B1u;
constexpr uint32_t Q8_HALF = 1u << 16;
constexpr int Q8_NAN = 255;              // exponent of a block that holds an infinity or a NaN (or more than 2^127): all its values are NaN

// `exponent` is biased as in fp32; code without sign, top = 127 or 255
__device__ __forceinline__ double q8_value(int code, int top, int exponent) {
  if (exponent == Q8_NAN) return __longlong_as_double(0x7ff8000000000000ll);
  return code == 0 ? 0.0 : __hiloint2double((code - top + 8 * (exponent + 1023 - 127)) << 17, 0);
}
template <bool SIGNED>
__device__ __forceinline__ uint32_t q8_code(double x, int exponent, uint32_t w) {
  constexpr int TOP = SIGNED ? 127 : 255;
  constexpr double LEAST = SIGNED ? 1.25 / 65536.0 : 1.25 / 4294967296.0;
  const double m = fabs(x);
  int code = min((int)(((uint32_t)__double2hiint(m) + w) >> 17) - 8 * (exponent + 1023 - 127) + TOP, TOP);
  const double y = m * __hiloint2double((1023 + 127 - exponent) << 20, 0);
  if (y < LEAST) code = SIGNED ? (int)(((uint32_t)(int)(fmin(y, LEAST) * (131072.0 / LEAST)) + w) >> 17) : 1;
  if (!(y > 0.0)) code = 0;
  if constexpr (SIGNED) return (uint32_t)code | (x < 0.0 && code ? 0x80u : 0u);
  else return (uint32_t)code;
}

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

// Codes of four elements a thread holds (32 lanes a block) from the moments in double; w of u is the upper, of v the lower 17 bits of mix, or 2^16 of both (HALF).
template <bool HALF>
__device__ __forceinline__ void q8_store(const AdamwState& st, int64_t at, bool any, const double (&u)[4], const double (&v)[4], const uint32_t (&mix)[4]) {
  uint32_t mu = 0, mv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    mu = max(mu, __float_as_uint(fabsf((float)u[e])));
    mv = max(mv, __float_as_uint(fabsf((float)v[e])));
  }
  const int eu = q8_exponent(max32(mu)), ev = q8_exponent(max32(mv));
  uint32_t pu = 0, pv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    pu |= q8_code<true>(u[e], eu, HALF ? Q8_HALF : mix[e] >> 15) << (8 * e);
    pv |= q8_code<false>(v[e], ev, HALF ? Q8_HALF : mix[e] & 0x1ffffu) << (8 * e);
  }
  if (!any) return;
  *reinterpret_cast<uint32_t*>(st.cu + at) = pu;
  *reinterpret_cast<uint32_t*>(st.cv + at) = pv;
  if ((threadIdx.x & 31) == 0) {
    st.eu[at / Q8_BLOCK] = (uint8_t)eu;
    st.ev[at / Q8_BLOCK] = (uint8_t)ev;
  }
}

// Gradient of four elements from i on, `cnt` of them there: dense, or by rows of a vocabulary of which few are there.
__device__ __forceinline__ void load_gradient(const void* g, const int32_t* index, int32_t slots, bool bf16, int64_t cols, int64_t row0, int64_t col0,
                                              int64_t i, int64_t ahead, int cnt, float (&x)[4]) {
  x[0] = x[1] = x[2] = x[3] = 0.f;
  if (index == nullptr) {
    if (cnt == 4) {
      if (bf16) load_quad<true, true>(g, i, x);
      else load_quad<false, true>(g, i, x);
    } else {
      for (int e = 0; e < cnt; ++e) x[e] = bf16 ? load_element<true>(g, i + e) : load_element<false>(g, i + e);
    }
    return;
  }
  // i = (row0, col0) + ahead, ahead < ADAMW_CHUNK: 32-bit arithmetic once col0 + ahead is below 2^32
  const uint64_t c = (uint64_t)(col0 + ahead);
  int64_t row, col;
  if (cols < (int64_t(1) << 31)) {
    const uint32_t q = (uint32_t)c / (uint32_t)cols;
    row = row0 + q; col = (int64_t)((uint32_t)c - q * (uint32_t)cols);
  } else {
    row = row0 + (int64_t)(c / (uint64_t)cols); col = (int64_t)(c % (uint64_t)cols);
  }
  if (cnt == 4 && col + 4 <= cols) {
    const int32_t slot = index[row];
    if ((uint32_t)slot < (uint32_t)slots) {
      if (bf16) load_quad<true, true>(g, slot * cols + col, x);
      else load_quad<false, true>(g, slot * cols + col, x);
    }
    return;
  }
  for (int e = 0; e < cnt; ++e) {
    const int32_t slot = index[row];
    if ((uint32_t)slot < (uint32_t)slots) x[e] = bf16 ? load_element<true>(g, slot * cols + col) : load_element<false>(g, slot * cols + col);
    if (++col == cols) { col = 0; ++row; }
  }
}

template <bool WBF, bool Q8>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a) {
  const int32_t c = a.first[0] + (int32_t)blockIdx.x;
  const int k = __builtin_amdgcn_readfirstlane(find_tensor(a.first, a.count, c));
  const AdamwTensor t = a.tensors[k];
  const float coef = a.coef ? *a.coef : 1.f;
  if (!(fabsf(coef) < INFINITY)) return;             // the norm was not finite: this step is left out (k_adamw_advance latches it)
  const double scale_d = a.scale * (double)coef;
  const float scale = (float)scale_d;
  const int64_t base = (int64_t)(c - a.first[k]) * ADAMW_CHUNK;
  void* const w = a.w[k];
  const void* const g = a.g[k];
  const int32_t* const index = a.index[k];
  const int32_t slots = a.slots[k];
  const bool g_bf16 = a.g_bf16[k] != 0;
  const float inv_c1 = a.step->next_inv_c1, inv_c2 = a.step->next_inv_c2, wd = t.decay ? a.wd : 0.f;
  const uint32_t turn = (uint32_t)(a.step->t + 1) * STEP_TURN;
  int64_t row0 = 0, col0 = 0;
  if (index) { row0 = base / t.cols; col0 = base - row0 * t.cols; }
#pragma unroll
  for (int rep = 0; rep < (int)(ADAMW_CHUNK / 1024); ++rep) {
    const int64_t ahead = rep * 1024 + (int64_t)threadIdx.x * 4, i = base + ahead;
    if (base + rep * 1024 >= t.n) break;             // uniform
    const int cnt = t.n - i >= 4 ? 4 : t.n > i ? (int)(t.n - i) : 0;
    float x[4] = {0.f, 0.f, 0.f, 0.f}, gr[4], u[4], v[4];
    if (cnt == 4) load_quad<WBF, true>(w, i, x);
    else
      for (int e = 0; e < cnt; ++e) x[e] = load_element<WBF>(w, i + e);
    if constexpr (!Q8) {
      if (cnt == 0) continue;
      const f32x4a ou = __builtin_nontemporal_load(reinterpret_cast<const f32x4a*>(a.st.u + t.off + i));     // (the state is padded to whole blocks)
      const f32x4a ov = __builtin_nontemporal_load(reinterpret_cast<const f32x4a*>(a.st.v + t.off + i));
      load_gradient(g, index, slots, g_bf16, t.cols, row0, col0, i, ahead, cnt, gr);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = scale * gr[e];
        u[e] = fmaf(a.b1, ou[e], a.omb1 * s);
        v[e] = fmaf(a.b2, ov[e], a.omb2 * s * s);
      }
      const f32x4a nu = {u[0], u[1], u[2], u[3]}, nv = {v[0], v[1], v[2], v[3]};
      __builtin_nontemporal_store(nu, reinterpret_cast<f32x4a*>(a.st.u + t.off + i));
      __builtin_nontemporal_store(nv, reinterpret_cast<f32x4a*>(a.st.v + t.off + i));
    } else {
      // every product and sum is rounded by itself, so that codes do not depend on which of them a compiler joins
#pragma clang fp contract(off)
      const int64_t at = t.off + i;
      const bool any = cnt > 0;
      uint32_t cu = 0, cv = 0;
      int eu = 0, ev = 0;
      if (any) {
        cu = *reinterpret_cast<const uint32_t*>(a.st.cu + at);
        cv = *reinterpret_cast<const uint32_t*>(a.st.cv + at);
        eu = a.st.eu[at / Q8_BLOCK];
        ev = a.st.ev[at / Q8_BLOCK];
      }
      load_gradient(g, index, slots, g_bf16, t.cols, row0, col0, i, ahead, cnt, gr);
      double du[4], dv[4];
      uint32_t mix[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int bu = (cu >> (8 * e)) & 0x7f, bv = (cv >> (8 * e)) & 0xff;
        const double s = scale_d * (double)gr[e];
        double ou = q8_value(bu, 127, eu);
        if ((cu >> (8 * e)) & 0x80) ou = -ou;
        const double ov = q8_value(bv, 255, ev);
        const double pu = a.b1d * ou, qu = a.omb1d * s, s2 = s * s, pv = a.b2d * ov, qv = a.omb2d * s2;
        du[e] = e < cnt ? pu + qu : 0.0;
        dv[e] = e < cnt ? pv + qv : 0.0;
        u[e] = (float)du[e]; v[e] = (float)dv[e];
        mix[e] = q8_mix(turn, (uint32_t)(i + e));
      }
      q8_store<false>(a.st, at, any, du, dv, mix);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float den = sqrtf(v[e] * inv_c2) + a.eps;
      const float n = den == 0.f ? 0.f : u[e] * inv_c1 / den;        // den = 0: eps = 0 and no gradient so far
      x[e] = fmaf(-a.lr, fmaf(wd, x[e], n), x[e]);
    }
    if (cnt == 4) store_quad<WBF, true>(w, i, x);
    else
      for (int e = 0; e < cnt; ++e) store_element<WBF>(w, i + e, x[e]);
  }
}

__global__ void k_adamw_advance(StepDev* sd, const float* coef, int32_t* flag) {
  if (coef && !(fabsf(*coef) < INFINITY)) *flag = 1;
  else step_write(sd, sd->t + 1);
}

// TO_STATE: moments <- [u | v], in 8 bits with thresholds of one half (a value of the grid stays itself); else [u | v] <- moments.  What lies
// between the tensors is written as zero.
template <bool Q8, bool TO_STATE>
__global__ __launch_bounds__(256) void k_moments(AdamwState st, const AdamwTensor* tensors, const int32_t* first, int32_t count, float* plain, int64_t total) {
  const int32_t c = (int32_t)blockIdx.x;
  int k = 0;                                          // (any number of tensors: search by halves)
  for (int lo = 0, hi = count; hi - lo > 1;) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= c) lo = mid; else hi = mid;
    k = lo;
  }
  const AdamwTensor t = tensors[k];
  const int64_t base = (int64_t)(c - first[k]) * ADAMW_CHUNK, padded = (t.n + Q8_BLOCK - 1) / Q8_BLOCK * Q8_BLOCK;
  for (int rep = 0; rep < (int)(ADAMW_CHUNK / 1024); ++rep) {
    const int64_t i = base + rep * 1024 + (int64_t)threadIdx.x * 4, at = t.off + i;
    if (base + rep * 1024 >= padded) break;
    const bool any = i < padded;
    float u[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    if (any && (TO_STATE || !Q8)) {
      for (int e = 0; e < 4; ++e)
        if (i + e < t.n) {
          u[e] = TO_STATE ? plain[at + e] : st.u[at + e];
          v[e] = TO_STATE ? plain[total + at + e] : st.v[at + e];
        }
    }
    if constexpr (Q8 && TO_STATE) {
      const double du[4] = {u[0], u[1], u[2], u[3]}, dv[4] = {v[0], v[1], v[2], v[3]};
      const uint32_t none[4] = {};
      q8_store<true>(st, at, any, du, dv, none);
    } else if (any) {
      if constexpr (Q8) {
        const uint32_t cu = *reinterpret_cast<const uint32_t*>(st.cu + at), cv = *reinterpret_cast<const uint32_t*>(st.cv + at);
        const int eu = st.eu[at / Q8_BLOCK], ev = st.ev[at / Q8_BLOCK];
        for (int e = 0; e < 4; ++e)
          if (i + e < t.n) {
            const double x = q8_value((cu >> (8 * e)) & 0x7f, 127, eu);
            u[e] = (float)((cu >> (8 * e)) & 0x80 ? -x : x);
            v[e] = (float)q8_value((cv >> (8 * e)) & 0xff, 255, ev);
          }
      }
      float* du = TO_STATE ? st.u + at : plain + at;
      float* dv = TO_STATE ? st.v + at : plain + total + at;
      for (int e = 0; e < 4; ++e) { du[e] = u[e]; dv[e] = v[e]; }
    }
  }
}

// ---------------------------------------------------------------------------------------
// Global norm.  Squares of fp32 numbers overflow from 1.8e19 on and vanish below 1e-23, and a sum of 1e9 of them in fp32 would lose the small ones:
// products and sums are in double, in an order that the sizes alone fix (each thread's elements, the lanes of a wave, the waves, the workgroups).
// ---------------------------------------------------------------------------------------
struct NormArgs {
  const void* g[NORM_GROUP];
  const int32_t* owner[NORM_GROUP];      // of rows: the row of the vocabulary that a row of g belongs to, or -1 (null: g is dense)
  int64_t n[NORM_GROUP], cols[NORM_GROUP];
  int32_t first[NORM_GROUP];
  uint8_t bf16[NORM_GROUP];
  int32_t count, chunks, add;
  double* part;
};

__device__ __forceinline__ double wave_sum(double x) {
  for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

__global__ __launch_bounds__(256) void k_norm_part(NormArgs a) {
  __shared__ double sums[4];
  double sum = 0.0;
  for (int32_t c = (int32_t)blockIdx.x; c < a.chunks; c += (int32_t)gridDim.x) {
    const int k = __builtin_amdgcn_readfirstlane(find_tensor(a.first, a.count, c));
    const void* const g = a.g[k];
    const int32_t* const owner = a.owner[k];
    const int64_t n = a.n[k], base = (int64_t)(c - a.first[k]) * NORM_CHUNK, cols = a.cols[k];
    const bool bf16 = a.bf16[k] != 0;
    for (int rep = 0; rep < (int)(NORM_CHUNK / 1024); ++rep) {
      const int64_t i = base + rep * 1024 + (int64_t)threadIdx.x * 4;
      if (i >= n) break;
      const int cnt = n - i >= 4 ? 4 : (int)(n - i);
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (owner == nullptr || (owner[i / cols] >= 0 && i % cols + cnt <= cols)) {
        if (cnt == 4) {
          if (bf16) load_quad<true, true>(g, i, x);
          else load_quad<false, true>(g, i, x);
        } else {
          for (int e = 0; e < cnt; ++e) x[e] = bf16 ? load_element<true>(g, i + e) : load_element<false>(g, i + e);
        }
      } else {
        for (int e = 0; e < cnt; ++e)
          if (owner[(i + e) / cols] >= 0) x[e] = bf16 ? load_element<true>(g, i + e) : load_element<false>(g, i + e);
      }
      for (int e = 0; e < 4; ++e) sum = fma((double)x[e], (double)x[e], sum);
    }
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    a.part[blockIdx.x] = a.add ? a.part[blockIdx.x] + sum : sum;
  }
}

__global__ __launch_bounds__(1024) void k_norm_sum(const double* part, int32_t count, double max_norm, float* out) {
  __shared__ double sums[16];
  double sum = (int)threadIdx.x < count ? part[threadIdx.x] : 0.0;
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int k = 0; k < 16; ++k) sum += sums[k];
    const double norm = sqrt(sum);
    out[0] = (float)norm;
    out[1] = !(norm < (double)INFINITY) ? __uint_as_float(0x7fc00000u) : norm > max_norm ? (float)(max_norm / norm) : 1.f;
  }
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
  StepDev* step_dev() const { return reinterpret_cast<StepDev*>(arena + step); }
  bool on_its_device() const {
    int cur = -1;
    return hipGetDevice(&cur) == hipSuccess && cur == device;
  }
};

namespace {

bool unit(double b) { return b >= 0 && b < 1; }

int plan_adamw(const lordo_tensor* tensors, int32_t n, const lordo_adamw_hparams* hp, lordo_adamw& c) {
  if (!tensors || !hp || n <= 0) return LORDO_EINVAL;
  if (!unit(hp->beta1) || !unit(hp->beta2) || !(hp->eps >= 0) || !std::isfinite(hp->eps) || !(hp->weight_decay >= 0) || !std::isfinite(hp->weight_decay))
    return LORDO_EINVAL;
  if (hp->bias_correction != 0 && hp->bias_correction != 1) return LORDO_EINVAL;
  if (hp->param_dtype != LORDO_F32 && hp->param_dtype != LORDO_BF16) return LORDO_EINVAL;
  if ((hp->state_dtype != LORDO_F32 && hp->state_dtype != LORDO_Q8) || hp->reserved != 0) return LORDO_EINVAL;
  c.hp = *hp;
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    const lordo_tensor& s = tensors[i];
    if (s.rows <= 0 || s.cols <= 0 || s.rows > (int64_t(1) << 38) || s.cols > (int64_t(1) << 38) / s.rows) return LORDO_EINVAL;
    if ((s.decay != 0 && s.decay != 1) || s.reserved != 0) return LORDO_EINVAL;
    AdamwTensor t{};
    t.n = s.rows * s.cols; t.cols = s.cols; t.off = c.total; t.decay = s.decay;
    c.first.push_back((int32_t)chunks);
    c.tensors.push_back(t);
    c.total += (t.n + Q8_BLOCK - 1) / Q8_BLOCK * Q8_BLOCK;
    chunks += (t.n + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
    if (chunks > (int64_t(1) << 30)) return LORDO_EINVAL;
  }
  c.first.push_back((int32_t)chunks);
  c.shapes.assign(tensors, tensors + n);
  int64_t at = 0;
  auto take = [&](int64_t bytes) { const int64_t r = at; at += (bytes + 255) & ~int64_t(255); return r; };
  c.flag = take(256);
  c.step = take(sizeof(StepDev));
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

#define ADAMW_CHK(expr, what)                                                                     \
  do {                                                                                            \
    if ((expr) != hipSuccess) {                                                                   \
      (void)hipGetLastError();                                                                    \
      fprintf(stderr, "lordo: %s failed\n", what);                                                \
      return LORDO_EHIP;                                                                          \
    }                                                                                             \
  } while (0)

int moments(lordo_adamw* c, float* plain, bool to_state, hipStream_t s) {
  const AdamwTensor* tensors = reinterpret_cast<const AdamwTensor*>(c->arena + c->table);
  const int32_t* first = reinterpret_cast<const int32_t*>(c->arena + c->prefix);
  const int32_t n = (int32_t)c->shapes.size();
  const dim3 grid((unsigned)c->first.back()), block(256);
  const AdamwState st = c->state();
  if (c->hp.state_dtype == LORDO_Q8) {
    if (to_state) hipLaunchKernelGGL((k_moments<true, true>), grid, block, 0, s, st, tensors, first, n, plain, c->total);
    else hipLaunchKernelGGL((k_moments<true, false>), grid, block, 0, s, st, tensors, first, n, plain, c->total);
  } else {
    if (to_state) hipLaunchKernelGGL((k_moments<false, true>), grid, block, 0, s, st, tensors, first, n, plain, c->total);
    else hipLaunchKernelGGL((k_moments<false, false>), grid, block, 0, s, st, tensors, first, n, plain, c->total);
  }
  return launched("k_moments");
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
    ADAMW_CHK(launch_fill_zero(c->arena + c->flag, 256, s), "fill");
    ADAMW_CHK(launch_fill_zero(c->arena + c->u, (int64_t)c->bytes - c->u, s), "fill");
    ADAMW_CHK(launch_step_set(c->step_dev(), hp->beta1, hp->beta2, hp->bias_correction, 0, s), "k_step_set");
    ADAMW_CHK(hipStreamSynchronize(s), "hipStreamSynchronize");
    *out = c.release();
    return LORDO_OK;
  });
}

int lordo_adamw_step(lordo_adamw* c, void* const* W, const lordo_grad* G, double lr, double grad_scale, const float* clip, void* stream) {
  if (!c || !W || !G || !std::isfinite(lr) || !std::isfinite(grad_scale)) return LORDO_EINVAL;
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
    ADAMW_CHK(launch_step_set(c->step_dev(), c->hp.beta1, c->hp.beta2, c->hp.bias_correction, c->t, s), "k_step_set");
  }
  c->step_dirty = true;         // until the whole step is enqueued: a call that fails below leaves the device count to be set back from `t`
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
  for (int at = 0; at < n; at += ADAMW_GROUP) {
    a.count = std::min(ADAMW_GROUP, n - at);
    for (int k = 0; k < a.count; ++k) {
      a.w[k] = W[at + k];
      a.g[k] = G[at + k].data;
      a.index[k] = G[at + k].index;
      a.slots[k] = (int32_t)G[at + k].slots;
      a.g_bf16[k] = G[at + k].dtype == LORDO_BF16;
    }
    a.tensors = reinterpret_cast<const AdamwTensor*>(c->arena + c->table) + at;
    a.first = reinterpret_cast<const int32_t*>(c->arena + c->prefix) + at;
    const dim3 grid((unsigned)(c->first[at + a.count] - c->first[at])), block(256);
    const bool bf = c->hp.param_dtype == LORDO_BF16;
    if (c->hp.state_dtype == LORDO_Q8) {
      if (bf) hipLaunchKernelGGL((k_adamw<true, true>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((k_adamw<false, true>), grid, block, 0, s, a);
    } else {
      if (bf) hipLaunchKernelGGL((k_adamw<true, false>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((k_adamw<false, false>), grid, block, 0, s, a);
    }
    const int rc = launched("k_adamw");
    if (rc != LORDO_OK) return rc;
  }
  hipLaunchKernelGGL(k_adamw_advance, dim3(1), dim3(1), 0, s, c->step_dev(), coef, reinterpret_cast<int32_t*>(c->arena + c->flag));
  const int rc = launched("k_adamw_advance");
  if (rc != LORDO_OK) return rc;
  ++c->t;
  c->step_dirty = false;
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

int lordo_adamw_set_step(lordo_adamw* c, int64_t t) {
  if (!c || t < 0) return LORDO_EINVAL;
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
  ADAMW_CHK(launch_fill_zero(c->arena + c->flag, 256, s), "fill");
  ADAMW_CHK(hipStreamSynchronize(s), "hipStreamSynchronize");
  return LORDO_ENUMERIC;
}

void lordo_adamw_destroy(lordo_adamw* c) { delete c; }

int lordo_grad_norm(const lordo_grad* G, int32_t n, double max_norm, float* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!G || n <= 0 || !(max_norm > 0) || !out || !workspace) return LORDO_EINVAL;
  if ((reinterpret_cast<uintptr_t>(out) & 3) != 0 || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return LORDO_EINVAL;
  if (workspace_bytes < LORDO_NORM_WORKSPACE_BYTES) return LORDO_ENOMEM;
  auto elements = [](const lordo_grad& g) { return g.index ? g.slots * g.cols : g.rows * g.cols; };
  int64_t most = 1;
  for (int at = 0; at < n; at += NORM_GROUP) {
    int64_t chunks = 0;
    for (int i = at; i < std::min(n, at + NORM_GROUP); ++i) {
      if (!good_grad(G[i])) return LORDO_EINVAL;
      chunks += (elements(G[i]) + NORM_CHUNK - 1) / NORM_CHUNK;
    }
    if (chunks > (int64_t(1) << 30)) return LORDO_EINVAL;
    most = std::max(most, chunks);
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const int blocks = (int)std::min<int64_t>(most, NORM_BLOCKS);      // the same for every launch: each adds to the sums of the one before
  NormArgs a;
  a.part = reinterpret_cast<double*>(workspace);
  for (int at = 0; at < n; at += NORM_GROUP) {
    a.count = std::min(NORM_GROUP, n - at);
    a.chunks = 0;
    for (int k = 0; k < a.count; ++k) {
      const lordo_grad& g = G[at + k];
      a.g[k] = g.data;
      a.owner[k] = g.index ? g.index + g.rows : nullptr;
      a.n[k] = elements(g);
      a.cols[k] = g.cols;
      a.bf16[k] = g.dtype == LORDO_BF16;
      a.first[k] = a.chunks;
      a.chunks += (int32_t)((a.n[k] + NORM_CHUNK - 1) / NORM_CHUNK);
    }
    a.add = at > 0;
    hipLaunchKernelGGL(k_norm_part, dim3((unsigned)blocks), dim3(256), 0, s, a);
    const int rc = launched("k_norm_part");
    if (rc != LORDO_OK) return rc;
  }
  hipLaunchKernelGGL(k_norm_sum, dim3(1), dim3(1024), 0, s, a.part, blocks, max_norm, out);
  return launched("k_norm_sum");
}

}  // extern "C"
