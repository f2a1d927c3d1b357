// Rotary positions: pair i of a head's first rot_dim elements, (a, b), becomes
//   mu (a cos t - b sin t),  mu (a sin t + b cos t),   t = pos * freqs[i]   (back: -t, the transposed map),
// the rest of the head stays as it is.  asl_rotate_write also puts keys and values into the pages.  Bound by memory: 32768 tokens of 40 heads
// of 128 in 116 us = 5.8 TB/s; 4085 tokens of 36 into pages 15.4; the smallest calls 3.5 to 4.8 (position, angles, heads one after the other).
//
// Angles: a position of a million times a radian needs 64 bits to leave anything of the turn.  The product is taken in turns, what is left
// of a turn is cut to an eighth either side of a quarter turn's multiple, and only that is rounded to 32 bits; sine and cosine are then
// their power series (the first terms left out: 2^-29 and 2^-33).
#include "paged.h"

#include "asl_internal.h"

namespace asl {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kUnroll = 4;                 // heads that a lane has on their way

// Sine and cosine of `turns` whole turns.
__device__ __forceinline__ float2 sine_cosine(double turns) {
  const double part = turns - rint(turns), quarter = rint(part * 4.);
  const float x = (float)((part - quarter * .25) * 6.283185307179586);       // |x| <= pi / 4
  const float y = x * x;
  const float s = __builtin_fmaf(x * y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float c = __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -.5f), 1.f);
  const int q = (int)quarter & 3;
  const float sn = (q & 1) ? c : s, cs = (q & 1) ? s : c;
  return make_float2((q & 2) ? -sn : sn, q == 1 || q == 2 ? -cs : cs);
}

// W bytes of a row, as elements of type T.  Those narrower than 16 bytes are for rows of any alignment.
template <typename T, int W>
struct Chunk {
  static constexpr int E = W / (int)sizeof(T);
  typedef T Elements __attribute__((ext_vector_type(E), aligned(W == 16 ? 16 : sizeof(T))));
  Elements x;

  // STREAM: past the caches (transfers that do not fit them anyway).
  template <bool STREAM>
  __device__ __forceinline__ void load(const char* p) {
    x = STREAM ? __builtin_nontemporal_load((const Elements*)p) : *(const Elements*)p;
  }
  template <bool STREAM>
  __device__ __forceinline__ void store(char* p) const {
    if (STREAM) __builtin_nontemporal_store(x, (Elements*)p); else *(Elements*)p = x;
  }
};

// A wavefront has some heads of a token: a lane has unit u of every so many-th head, so that the angles of its pairs, which the lanes
// work out together once, stay in its registers.  Units of a head (E elements in W bytes): rotated ones, with halves E pairs in two
// pieces, with neighbours E / 2 pairs in one; then the pieces of the rest.  A head of values (WRITE) is copied by the same units.
template <typename T, int W, bool HALVES, bool WRITE, bool STREAM>
__global__ void __launch_bounds__(kThreads) rotate_kernel(RotateArgs a) {
  typedef Chunk<T, W> C;
  constexpr int E = C::E, PAIRS = HALVES ? E : E / 2;
  extern __shared__ float2 lds[];          // [kWaves][rot / 2] (cos, sin)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = (int64_t)blockIdx.x * kWaves + wave;
  const int tok = (int)(job / a.parts), part = (int)(job - (int64_t)tok * a.parts);
  float2* turn = lds + wave * (a.rot / 2);
  const bool there = tok < a.n;
  if (there) {
    const double pos = (double)a.pos[tok];
    for (int i = lane; i < a.rot / 2; i += 64) {
      const float2 sc = sine_cosine(pos * (a.freqs[i] * 0.15915494309189535));
      turn[i] = make_float2(sc.y * a.cos_by, sc.x * a.sin_by);
    }
  }
  __syncthreads();
  if (!there) return;
  int64_t place = -1;                      // byte offset of the token in the pages
  if (WRITE) {
    const int64_t slot = a.slot[tok];
    if (slot < -1 || (slot >> a.map.ps_shift) >= a.map.n_pages) {
      if (lane == 0 && part == 0) atomicOr(a.map.fault, kFaultPaged);
    } else if (slot >= 0) {
      place = (slot >> a.map.ps_shift) * a.map.page + (slot & (a.map.ps - 1)) * a.map.tok;
    }
  }
  const int H = a.Hq + a.Hk + (WRITE ? a.Hk : 0);
  const int h0 = part * a.heads, h1 = min(H, h0 + a.heads);
  const int width = min(a.units, 64), side = 64 / width;    // lanes of a head, heads at once
  if (lane >= side * width) return;
  for (int u = lane % width; u < a.units; u += width) {
    const bool turned = u < a.turned;
    // first byte of the unit's piece, and of its second one (-1: none), in a head that is rotated, and in one of values
    const int at = !HALVES || turned ? u * W : a.rot * (int)sizeof(T) + (u - a.turned) * W;
    const int at2 = HALVES && turned ? a.rot / 2 * (int)sizeof(T) + u * W : -1;
    const int v2 = HALVES && (u + a.units) * W < a.d * (int)sizeof(T) ? (u + a.units) * W : -1;
    float2 t[PAIRS];
#pragma unroll
    for (int e = 0; e < PAIRS; ++e) t[e] = turned ? turn[u * PAIRS + e] : make_float2(1.f, 0.f);
    for (int hb = h0 + lane / width; hb < h1; hb += side * kUnroll) {
      C x[kUnroll], y[kUnroll];
      char* to[kUnroll];
      int first[kUnroll], second[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int h = hb + k * side;
        to[k] = nullptr;
        if (h >= h1) continue;
        const char* from;
        first[k] = at;
        second[k] = at2;
        if (h < a.Hq) {
          from = a.q + tok * a.qt + h * a.qh;
          to[k] = a.q_out + tok * a.qot + h * a.qoh;
        } else if (h < a.Hq + a.Hk) {
          from = a.k + tok * a.kt + (h - a.Hq) * a.kh;
          to[k] = WRITE ? (place < 0 ? nullptr : a.k_out + place + (h - a.Hq) * a.map.head) : a.k_out + tok * a.kot + (h - a.Hq) * a.koh;
        } else {
          from = a.v + tok * a.vt + (h - a.Hq - a.Hk) * a.vh;
          to[k] = place < 0 ? nullptr : a.v_out + place + (h - a.Hq - a.Hk) * a.map.head;
          first[k] = u * W;
          second[k] = v2;
        }
        if (to[k] == nullptr) continue;
        x[k].template load<STREAM>(from + first[k]);
        if (second[k] >= 0) y[k].template load<STREAM>(from + second[k]);
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (to[k] == nullptr) continue;
        if (turned && (!WRITE || hb + k * side < a.Hq + a.Hk)) {
          if constexpr (HALVES) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float p = (float)x[k].x[e], q = (float)y[k].x[e];
              x[k].x[e] = (T)__builtin_fmaf(p, t[e].x, -(q * t[e].y));
              y[k].x[e] = (T)__builtin_fmaf(p, t[e].y, q * t[e].x);
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              const float p = (float)x[k].x[e], q = (float)x[k].x[e + 1];
              x[k].x[e] = (T)__builtin_fmaf(p, t[e / 2].x, -(q * t[e / 2].y));
              x[k].x[e + 1] = (T)__builtin_fmaf(p, t[e / 2].y, q * t[e / 2].x);
            }
          }
        }
        x[k].template store<STREAM>(to[k] + first[k]);
        if (second[k] >= 0) y[k].template store<STREAM>(to[k] + second[k]);
      }
    }
  }
}

// Bytes read and written from which a rotation goes past the caches (32768 tokens, 40 heads of 128, 671 MB: 134 us, so 117 = 5.8 TB/s; 4085
// tokens, 36 heads of 128, 75 MB that the caches hold: 16.3, 20.1).
constexpr int64_t kRotateStreamBytes = int64_t(100) << 20;

template <typename T, int W, bool HALVES>
void launch(const RotateArgs& a, bool write, bool stream, dim3 grid, size_t lds, hipStream_t st) {
  if constexpr (W == 16) {
    if (stream) {
      if (write)
        hipLaunchKernelGGL((rotate_kernel<T, W, HALVES, true, true>), grid, dim3(kThreads), lds, st, a);
      else
        hipLaunchKernelGGL((rotate_kernel<T, W, HALVES, false, true>), grid, dim3(kThreads), lds, st, a);
      return;
    }
  }
  if (write)
    hipLaunchKernelGGL((rotate_kernel<T, W, HALVES, true, false>), grid, dim3(kThreads), lds, st, a);
  else
    hipLaunchKernelGGL((rotate_kernel<T, W, HALVES, false, false>), grid, dim3(kThreads), lds, st, a);
}

template <typename T>
void launch_type(const RotateArgs& a, int width, bool halves, bool write, dim3 grid, size_t lds, hipStream_t st) {
  const bool stream = 2 * (int64_t)a.n * (a.Hq + a.Hk * (write ? 2 : 1)) * a.d * (int64_t)sizeof(T) >= kRotateStreamBytes;
  if (halves) {
    if (width == 16) launch<T, 16, true>(a, write, stream, grid, lds, st);
    else if (width == 4) launch<T, 4, true>(a, write, stream, grid, lds, st);
    else if constexpr (sizeof(T) < 4) launch<T, 2, true>(a, write, stream, grid, lds, st);
  } else {
    if (width == 16) launch<T, 16, false>(a, write, stream, grid, lds, st);
    else launch<T, 2 * sizeof(T), false>(a, write, stream, grid, lds, st);
  }
}

}  // namespace

// Tokens of one launch: a wavefront each, so 2^31 threads.  A launch of 2^32 or more in x does not fail: it runs with their number modulo 2^32.
constexpr int kRotateTokens = 1 << 25;

hipError_t launch_rotate(const RotateArgs& args, int dtype, bool halves, bool write, int width, hipStream_t st) {
  RotateArgs a = args;
  if (a.n == 0) return hipSuccess;
  const int eb = dtype == ASL_BF16 ? 2 : 4, E = width / eb;
  a.turned = halves ? a.rot / 2 / E : a.rot / E;
  a.units = a.turned + (a.in_place ? 0 : (a.d - a.rot) / E);
  const int H = a.Hq + a.Hk * (write ? 2 : 1), side = 64 / (a.units < 64 ? a.units : 64);
  // a token is a wavefront's, but for calls too small to fill the card: then some heads of it
  const int least = side < H ? side : H;
  a.parts = 1;
  while (a.parts * 2 * least <= H && (int64_t)a.n * a.parts < 2048) a.parts *= 2;
  a.heads = (H + a.parts - 1) / a.parts;
  const size_t lds = (size_t)kWaves * (a.rot / 2) * sizeof(float2);
  for (int32_t left = args.n; left > 0; left -= a.n) {
    a.n = left < kRotateTokens ? left : kRotateTokens;
    const int64_t jobs = (int64_t)a.n * a.parts;
    const dim3 grid((unsigned)((jobs + kWaves - 1) / kWaves));
    if (dtype == ASL_BF16) launch_type<__bf16>(a, width, halves, write, grid, lds, st);
    else launch_type<float>(a, width, halves, write, grid, lds, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (left == a.n) break;
    a.pos += a.n;
    if (a.Hq > 0) {
      a.q += a.n * a.qt;
      a.q_out += a.n * a.qot;
    }
    if (a.Hk > 0) a.k += a.n * a.kt;
    if (a.Hk > 0 && !write) a.k_out += a.n * a.kot;
    if (write) {
      a.v += a.n * a.vt;
      a.slot += a.n;
    }
  }
  return hipSuccess;
}

}  // namespace asl
