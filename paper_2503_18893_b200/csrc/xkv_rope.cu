// Rotary positions (xkv_rope): y_a = g (x_a cos - x_b sin), y_b = g (x_b cos + x_a sin) for every pair (a, b) of a head, the angle
// being position times the pair's frequency.
//
// Angles.  A plan holds turns per position as 64-bit fractions, so position * turns modulo 2^64 is the angle modulo one turn, exact
// but for the fraction's own 2^-64 per position.  What is left of it beyond the nearest quarter turn goes through sincospi; a product
// of a position and a frequency in 32 bits would be off by 0.01 at position 10^5.
//
// A CTA takes up to eight rows: it forms their cosines and sines once, in shared memory, for all heads of both tensors, while the first
// elements are on their way.  A thread has one place in the head and goes over heads and rows, two at a time in flight.  Bound by memory:
// each element is read and written once.  8189 tokens of 40 heads of 128: bf16 28.9 us (5.8 TB/s; four at a time 30.4), fp32 53 (6.3); 64
// tokens 3.4, one launch.
#include <math.h>

#include <cuda_fp16.h>

#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kRopeThreads = 256, kRopeMaxRows = 8;

struct RopeTensor {
  const void* x;
  void* y;
  long long x_row, x_head, y_row, y_head;
};
struct RopeArgs {
  xkv_rope_plan plan;
  RopeTensor t[2];
  int heads0, heads;                           // of the first tensor, of both
  int rows_per_cta;
  int units;                                   // places of a thread in a head
  float gain, sign;                            // factor on cosine and sine; -1: the other way round
  long long rows, n_pos;
  const int32_t* pos;
};

// P elements side by side, in 16-byte pieces where P of them make one.
template <typename T, int P>
struct Piece {
  alignas(P * sizeof(T)) T v[P];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (P * sizeof(T) == 16) *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(p);
    else v[0] = *p;
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (P * sizeof(T) == 16) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(v);
    else *p = v[0];
  }
};
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float x, float* y) { *y = x; }
__device__ __forceinline__ void from_float(float x, __half* y) { *y = __float2half_rn(x); }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16* y) { *y = __float2bfloat16_rn(x); }

// Cosine and sine of `phase` / 2^64 turns: the nearest quarter turn is taken off (its sine and cosine are 0 and +-1), so that the rest
// keeps its bits when it becomes fp32.
__device__ __forceinline__ float2 cos_sin(uint64_t phase) {
  const uint64_t quarter = (phase + (1ull << 61)) >> 62;
  float s, c;
  sincospif((float)(long long)(phase - (quarter << 62)) * 0x1p-63f, &s, &c);
  if (quarter & 1) { const float x = c; c = -s; s = x; }
  return (quarter & 2) ? make_float2(-c, -s) : make_float2(c, s);
}

template <typename T, int P, bool HALF>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs a) {
  // Cosine and sine of a row's pairs, those of one unit in pieces of 16 bytes a whole row of units apart: lanes side by side meet all banks.
  __shared__ __align__(16) float2 turn_s[kRopeMaxRows * (XKV_ROPE_MAX_ROT / 2)];
  const int pairs = a.plan.rot >> 1, turning = pairs / P, tid = threadIdx.x;
  const long long row0 = (long long)blockIdx.x * a.rows_per_cta;
  const int rows = (int)min((long long)a.rows_per_cta, a.rows - row0);
  constexpr int U = 2;
  const int width = min(a.units, kRopeThreads), step = kRopeThreads / width;     // threads of a head, heads at a time
  const bool works = tid < width * step;
  int u = tid % width, r = 0, h = tid / width;
  auto settle = [&] { while (h >= a.heads && r < rows) { h -= a.heads; ++r; } };
  settle();
  Piece<T, P> xa[U], xb[U];
  T* y[U];
  int row[U], n = 0;
  // a unit is 2 P elements of the head's pairs, or of what is copied behind them
  auto place_a = [&] { return HALF && u < turning ? u * P : u * 2 * P; };
  auto place_b = [&] { return HALF && u < turning ? u * P + pairs : u * 2 * P + P; };
  auto load = [&] {                            // the next U rows or heads of this thread's place
    n = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (works && r < rows) {
        const RopeTensor& t = a.t[h < a.heads0 ? 0 : 1];
        const long long ht = h < a.heads0 ? h : h - a.heads0;
        const T* x = (const T*)t.x + (row0 + r) * t.x_row + ht * t.x_head;
        y[i] = (T*)t.y + (row0 + r) * t.y_row + ht * t.y_head;
        xa[i].load(x + place_a());
        xb[i].load(x + place_b());
        row[i] = r;
        n = i + 1;
        h += step;
        settle();
      }
    }
  };
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  load();                                      // (under way while the turns are formed)
  for (int i = tid; i < rows * pairs; i += kRopeThreads) {
    const int ri = i / pairs, p = i - ri * pairs, k = p % P;
    const long long at = row0 + ri;
    const float2 t = cos_sin((uint64_t)(long long)a.pos[a.rows == a.n_pos ? at : at % a.n_pos] * a.plan.turns[p]);
    turn_s[ri * pairs + (P == 1 ? p : ((k >> 1) * turning + p / P) * 2 + (k & 1))] = make_float2(t.x * a.gain, t.y * a.gain * a.sign);
  }
  __syncthreads();
  if (!works) return;
  while (true) {
    while (n > 0) {
      const int ea = place_a(), eb = place_b();
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (i >= n) break;
        if (u < turning) {
          const float2* t = turn_s + row[i] * pairs;
          float2 cs[P];
          if constexpr (P == 1) {
            cs[0] = t[u];
          } else {
#pragma unroll
            for (int k = 0; k < P; k += 2) *reinterpret_cast<float4*>(cs + k) = *reinterpret_cast<const float4*>(t + ((k >> 1) * turning + u) * 2);
          }
#pragma unroll
          for (int k = 0; k < P; ++k) {
            // pair k: the k-th element of both pieces, or two neighbours of the 2 P elements
            T& va = HALF ? xa[i].v[k] : (2 * k < P ? xa[i].v[2 * k % P] : xb[i].v[2 * k % P]);
            T& vb = HALF ? xb[i].v[k] : (2 * k + 1 < P ? xa[i].v[(2 * k + 1) % P] : xb[i].v[(2 * k + 1) % P]);
            const float fa = to_float(va), fb = to_float(vb);
            from_float(fa * cs[k].x - fb * cs[k].y, &va);
            from_float(fb * cs[k].x + fa * cs[k].y, &vb);
          }
        }
        xa[i].store(y[i] + ea);
        xb[i].store(y[i] + eb);
      }
      load();
    }
    u += width;                                // (heads of more units than threads)
    if (u >= a.units) break;
    r = 0;
    h = tid / width;
    settle();
    load();
  }
}

template <typename T, int P>
cudaError_t launch_as(const RopeArgs& a, dim3 grid, cudaStream_t s) {
  return a.plan.layout == XKV_ROPE_HALF ? launch_pdl(rope_kernel<T, P, true>, grid, dim3(kRopeThreads), 0, s, a)
                                        : launch_pdl(rope_kernel<T, P, false>, grid, dim3(kRopeThreads), 0, s, a);
}

// 16-byte pieces, where places, distances and sizes allow them; else element by element.
template <typename T>
cudaError_t launch_type(RopeArgs a, bool in_place, cudaStream_t s) {
  constexpr int P = 16 / sizeof(T);
  bool wide = a.plan.rot % (2 * P) == 0 && a.plan.d_h % (2 * P) == 0;
  for (int i = 0; i < 2; ++i) {
    const RopeTensor& t = a.t[i];
    if (i == 0 ? a.heads0 > 0 : a.heads > a.heads0)
      wide = wide && ((((uintptr_t)t.x | (uintptr_t)t.y) & 15u) == 0) && ((t.x_row | t.x_head | t.y_row | t.y_head) % P) == 0;
  }
  const int p = wide ? P : 1;
  a.units = (in_place ? a.plan.rot : a.plan.d_h) / (2 * p);    // (in place there is nothing to copy)
  // Few rows: a CTA each.  Many: as many as make a thread's loads worth its way, as long as there are twelve CTAs an SM (six: 55.9 us for 8189 tokens of 40 heads in fp32, twelve 53.0).
  a.rows_per_cta = 1;
  while (a.rows_per_cta < kRopeMaxRows && a.rows / (2 * a.rows_per_cta) >= kPlanSms * 12) a.rows_per_cta *= 2;
  const dim3 grid((unsigned)((a.rows + a.rows_per_cta - 1) / a.rows_per_cta));
  return wide ? launch_as<T, P>(a, grid, s) : launch_as<T, 1>(a, grid, s);
}

}  // namespace

#pragma nv_diag_suppress 20208                 // (long double: this is host code)
int rope_plan_init(const xkv_rope_config* c, xkv_rope_plan* plan) {
  if (!c || !plan || c->struct_size != sizeof(xkv_rope_config)) return XKV_ERR_INVALID_ARG;
  if (c->d_h < 2 || c->d_h > 1024 || c->d_h % 2 || c->rot < 2 || c->rot % 2 || c->rot > c->d_h || c->rot > XKV_ROPE_MAX_ROT) return XKV_ERR_INVALID_ARG;
  if (c->layout != XKV_ROPE_HALF && c->layout != XKV_ROPE_INTERLEAVED) return XKV_ERR_INVALID_ARG;
  const bool yarn = c->scaling == XKV_ROPE_SCALE_YARN, llama3 = c->scaling == XKV_ROPE_SCALE_LLAMA3, ntk = c->scaling == XKV_ROPE_SCALE_NTK;
  if (c->scaling < XKV_ROPE_SCALE_NONE || c->scaling > XKV_ROPE_SCALE_YARN) return XKV_ERR_INVALID_ARG;
  auto positive = [](double x) { return x > 0.0 && isfinite(x); };
  if (!positive(c->base) || !(c->gain == 0.0 || positive(c->gain))) return XKV_ERR_INVALID_ARG;
  if (c->scaling != XKV_ROPE_SCALE_NONE && !positive(c->factor)) return XKV_ERR_INVALID_ARG;
  if ((yarn || llama3) && !positive(c->original)) return XKV_ERR_INVALID_ARG;
  if (llama3 && !(positive(c->low) && positive(c->high) && c->high > c->low)) return XKV_ERR_INVALID_ARG;
  if (yarn && !(c->base > 1.0 && positive(c->beta_fast) && positive(c->beta_slow))) return XKV_ERR_INVALID_ARG;
  if (ntk && c->rot < 4) return XKV_ERR_INVALID_ARG;

  constexpr long double two_pi = 6.283185307179586476925286766559005768L;
  const int n = c->rot;
  const long double factor = c->factor, base = ntk ? c->base * powl(factor, (long double)n / (n - 2)) : (long double)c->base;
  long double lo = 0, hi = 0;
  if (yarn) {
    auto pair = [&](long double beta) { return n * logl(c->original / (beta * two_pi)) / (2 * logl(base)); };
    lo = fmaxl(floorl(pair(c->beta_fast)), 0);
    hi = fminl(ceill(pair(c->beta_slow)), n - 1);
  }
  plan->struct_size = sizeof(xkv_rope_plan);
  plan->d_h = c->d_h;
  plan->rot = n;
  plan->layout = c->layout;
  plan->reserved = 0;
  plan->gain = (float)(c->gain > 0.0 ? c->gain : yarn ? 0.1L * logl(factor) + 1.0L : 1.0L);
  if (!(plan->gain > 0.0f) || isinf(plan->gain) || isinf(1.0f / plan->gain)) return XKV_ERR_INVALID_ARG;     // (the inverse divides by it)
  for (int i = 0; i < XKV_ROPE_MAX_ROT / 2; ++i) {
    plan->turns[i] = 0;
    if (i >= n / 2) continue;
    long double f = powl(base, -2.0L * i / n);
    if (c->scaling == XKV_ROPE_SCALE_LINEAR) f /= factor;
    if (llama3) {
      const long double s = fminl(fmaxl((c->original * f / two_pi - c->low) / ((long double)c->high - c->low), 0), 1);
      f = (1 - s) * f / factor + s * f;
    }
    if (yarn) {
      const long double r = fminl(fmaxl((i - lo) / fmaxl(hi - lo, 0.001L), 0), 1);
      f = r * f / factor + (1 - r) * f;
    }
    if (!isfinite(f)) return XKV_ERR_INVALID_ARG;
    long double turn = f / two_pi;
    turn -= floorl(turn);
    const long double scaled = roundl(turn * 0x1p64L);
    plan->turns[i] = scaled >= 0x1p64L ? 0 : (uint64_t)scaled;
  }
  return XKV_OK;
}

cudaError_t launch_rope(const xkv_rope_plan* plan, int direction, int type, const xkv_rope_tensor* tensors, int n_tensors, int64_t rows,
                        const int32_t* pos, int64_t n_pos, cudaStream_t s) {
  RopeArgs a;
  a.plan = *plan;
  bool in_place = true;
  for (int i = 0; i < 2; ++i) {
    const xkv_rope_tensor& t = tensors[i < n_tensors ? i : 0];
    a.t[i] = {t.x, t.y, t.x_row, t.x_head, t.y_row, t.y_head};
    if (t.heads > 0 && t.x != t.y) in_place = false;
  }
  a.heads0 = tensors[0].heads;
  a.heads = a.heads0 + (n_tensors == 2 ? tensors[1].heads : 0);
  if (rows == 0 || a.heads == 0) return cudaSuccess;
  a.gain = direction == XKV_ROPE_INVERSE ? 1.0f / plan->gain : plan->gain;
  a.sign = direction == XKV_ROPE_FORWARD ? 1.0f : -1.0f;
  a.rows = rows; a.n_pos = n_pos; a.pos = pos;
  const cudaError_t e = type == XKV_FP32 ? launch_type<float>(a, in_place, s) : type == XKV_FP16 ? launch_type<__half>(a, in_place, s) : launch_type<__nv_bfloat16>(a, in_place, s);
  count_launch(kFamRope);
  return e;
}

}  // namespace xkv
