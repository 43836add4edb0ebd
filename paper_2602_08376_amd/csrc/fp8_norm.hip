// Root-mean-square norm of a residual stream with its output in 8 bits
// (ojbkq_rmsnorm_fp8).
#include "fp8_pack.h"

namespace ojbkq {
namespace {

struct Root {
  double inv, rest;   // 1 / sqrt(mean + eps), to twice float64's bits
};

template <class E>
__device__ __forceinline__ void widen(const Eight<E>& x, float (&h)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (float)x.v[e];
}

// One workgroup of NT threads to a token.  A thread holds NV runs of eight
// neighbouring features of h in registers (NT * 8 * NV >= m), so x and the
// residual are read once: bound by memory.  The squares are summed in float64
// (no finite h overflows), and y is formed and rounded from float64, which
// memory leaves time for where there is a residual.
// NV = 0: longer rows, read twice.
// 8192 x 8192, bfloat16, with a residual: 91 to 95 us, 5.1 to 4.9 TB/s (a large
// copy: 5.2); float16 without one 63 to 67 us, 3.2 to 3.0 TB/s, bound by the
// vector ALU and the wait for the token's sum; 1 x 4096: 3.3 us, latency.
template <int XT, int RT, int NT, int NV>
__global__ __launch_bounds__(NT) void rmsnorm_kernel(Norm8Args a) {
  typedef typename Number<XT>::type X;
  typedef typename Number<RT < 0 ? 0 : RT>::type R;
  constexpr bool kRes = RT >= 0;
  constexpr int kRuns = NV ? NV : 1, kWaves = NT / 64;
  __shared__ double part[kRuns * kWaves];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const X* const x = static_cast<const X*>(a.x) + row * a.ldx;
  const R* const rin = kRes ? static_cast<const R*>(a.r_in) + row * a.ldr : nullptr;
  R* const rout = kRes ? static_cast<R*>(a.r_out) + row * a.ldr : nullptr;
  uint8_t* const dst = a.X8 + row * a.ld8;
  const int64_t m16 = (a.m + 15) / 16 * 16;

  // h of the eight features from k on (0 past the last one)
  auto read = [&](int64_t k, float (&h)[8]) {
    Eight<X> vx;
    vx.load(x + k, a.m - k);
    if constexpr (kRes) {
      Eight<R> vr;
      vr.load(rin + k, a.m - k);
      float r[8];
      widen(vr, r);
      widen(vx, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] += r[e];
    } else {
      widen(vx, h);
    }
  };
  auto squares = [&](const float (&h)[8]) {
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fma((double)h[e], (double)h[e], s);
    return s;
  };
  // The token's sum, in every thread: runs of 512 features by themselves (a
  // wave's), then these in a fixed order, so that it does not go by how many
  // threads and registers share the features.
  auto total = [&](double (&s)[kRuns]) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
      for (int i = 0; i < kRuns; ++i) s[i] += __shfl_xor(s[i], d);
    if ((tid & 63) == 0)
#pragma unroll
      for (int i = 0; i < kRuns; ++i) part[kWaves * i + (tid >> 6)] = s[i];
    __syncthreads();
    constexpr int kParts = kRuns * kWaves, kLanes = kParts <= 4 ? 4 : kParts <= 8 ? 8 : kParts <= 16 ? 16 : 32;
    static_assert(kParts <= 32, "a lane to each");
    const int lane = tid & (kLanes - 1);
    double all = lane < kParts ? part[lane] : 0.0;
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) all += __shfl_xor(all, d);
    return all;
  };
  auto finish = [&](int64_t k, const float (&h)[8], Root root) {
    if constexpr (kRes) {
      Eight<R> o;
#pragma unroll
      for (int e = 0; e < 8; ++e) o.v[e] = (R)h[e];
      o.store(rout + k, a.m - k);
    }
    float g[8];
    if (a.gain) {
      Eight<float> vg;
      vg.load(a.gain + k, a.m - k);
      widen(vg, g);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = 1.f;
    }
    uint32_t hi[8], most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // h gain is exact in float64, and the reciprocal's second part makes the
      // product the quotient rounded once: a y that lies on a border of e4m3
      // stays there.  (NaN for a token with one; past the last feature h is 0.)
      float v = h[e];
      asm volatile("" : "+v"(v));   // (or the squares' float64 forms are kept in registers)
      const double hg = (double)v * (double)g[e];
      const double y = __builtin_fma(hg, root.inv, hg * root.rest);
      hi[e] = k + e < a.m ? sticky_high(y) : 0u;
      const uint32_t s = size_key64(hi[e]);
      most = most > s ? most : s;
    }
    const uint32_t code = scale_code64(max16(most));
    if (k < m16) *reinterpret_cast<u2*>(dst + k) = to_e4m3(hi, code);
    if ((tid & 15) == 0 && k < a.m) a.scales[row * a.lds + (k >> 7)] = (uint8_t)code;
  };
  // infinite sums (an infinity in h) give NaN for the whole token
  auto root_of = [&](double s) {
    const double v = __builtin_sqrt(s / (double)a.m + a.eps);
    const double inv = s < __builtin_huge_val() ? 1.0 / v : __builtin_nan("");
    return Root{inv, __builtin_fma(-v, inv, 1.0) * inv};
  };

  if constexpr (NV > 0) {
    float h[kRuns][8];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) read(8 * ((int64_t)tid + NT * i), h[i]);
    double s[kRuns];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) s[i] = squares(h[i]);
    const Root root = root_of(total(s));
#pragma unroll
    for (int i = 0; i < kRuns; ++i) finish(8 * ((int64_t)tid + NT * i), h[i], root);
  } else {
    // every thread reads the same features both times, so the residual may be
    // updated in place
    double s[1] = {0.0};
    float h[8];
    const int64_t whole = (a.m + 127) / 128 * 128;   // whole rows of 16 lanes for max16
    for (int64_t k = 8 * tid; k < a.m; k += 8 * NT) {
      read(k, h);
      s[0] += squares(h);
    }
    const Root root = root_of(total(s));
    for (int64_t k = 8 * tid; k < whole; k += 8 * NT) {
      read(k, h);
      finish(k, h, root);
    }
  }
}

template <int XT, int RT>
hipError_t launch_slice(const Norm8Args& a, hipStream_t s) {
  const dim3 grid((unsigned)a.T);
#define OJBKQ_NORM(NT, NV) rmsnorm_kernel<XT, RT, NT, NV><<<grid, dim3(NT), 0, s>>>(a)
  // Few tokens leave CUs idle: more threads to each, for latency; otherwise
  // fewer threads with several loads each under way, as long as their
  // registers leave a CU two workgroups.  us, bfloat16 x and residual:
  //   1 x 4096       (512, 1) 3.3   (256, 2) 3.8   (1024, 1) 4.2
  //   512 x 4096     (512, 1) 5.9   (256, 2) 6.2
  //   8192 x 4096    (512, 1) 55.4  (256, 2) 51.5
  //   1 x 8192       (1024, 1) 4.5  (512, 2) 4.6   (256, 4) 5.8
  //   512 x 8192     (1024, 1) 10.4 (512, 2) 10.5  (256, 4) 11.3
  //   8192 x 8192    (1024, 1) 112  (512, 2) 97    (256, 4) 96, float32 81.9 against 85.1 (4096 x 8192)
  //   5000 x 12000   (512, 3) 92.5  (1024, 2) 111  (512, 0) 107
  //   4096 x 16384   (512, 4) 100   (1024, 2) 107  (512, 0) 115, (1024, 0) 120
  //   2048 x 32768   (1024, 0) 121
  // Without a residual less is read and fewer registers are held, so a workgroup's
  // threads may be fewer still: 8192 x 8192 float16 (256, 4) 66, (512, 2) 73; 8192 x
  // 6144 bfloat16 (256, 3) 49, (256, 4) 61, (512, 2) 63.
  if constexpr (RT < 0)
    if (a.T > 512 && a.m > 4096 && a.m <= 8192) {
      if (a.m <= 6144) OJBKQ_NORM(256, 3);
      else OJBKQ_NORM(256, 4);
      return hipGetLastError();
    }
  if (a.m <= 2048) OJBKQ_NORM(256, 1);
  else if (a.m <= 4096 && a.T <= 512) OJBKQ_NORM(512, 1);
  else if (a.m <= 4096) OJBKQ_NORM(256, 2);
  else if (a.m <= 8192 && a.T <= 512) OJBKQ_NORM(1024, 1);
  else if (a.m <= 8192) OJBKQ_NORM(512, 2);
  else if (a.m <= 12288) OJBKQ_NORM(512, 3);
  else if (a.m <= 16384) OJBKQ_NORM(512, 4);
  else OJBKQ_NORM(1024, 0);
#undef OJBKQ_NORM
  return hipGetLastError();
}

// A grid holds 2^32 - 1 threads along a dimension.
template <int XT, int RT>
hipError_t launch(const Norm8Args& a, hipStream_t s) {
  const int64_t step = (int64_t)1 << 21;
  for (int64_t t = 0; t < a.T; t += step) {
    Norm8Args b = a;
    b.T = a.T - t < step ? a.T - t : step;
    b.x = static_cast<const typename Number<XT>::type*>(a.x) + t * a.ldx;
    if (a.r_in) {
      typedef typename Number<RT < 0 ? 0 : RT>::type R;
      b.r_in = static_cast<const R*>(a.r_in) + t * a.ldr;
      b.r_out = static_cast<R*>(a.r_out) + t * a.ldr;
    }
    b.X8 = a.X8 + t * a.ld8;
    b.scales = a.scales + t * a.lds;
    if (hipError_t e = launch_slice<XT, RT>(b, s); e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int XT>
hipError_t launch_x(const Norm8Args& a, int rtype, hipStream_t s) {
  if (!a.r_in) return launch<XT, -1>(a, s);
  switch (rtype) {
    case 0: return launch<XT, 0>(a, s);
    case 1: return launch<XT, 1>(a, s);
    case 2: return launch<XT, 2>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_rmsnorm_fp8(const Norm8Args& a, int xtype, int rtype, hipStream_t stream) {
  switch (xtype) {
    case 0: return launch_x<0>(a, rtype, stream);
    case 1: return launch_x<1>(a, rtype, stream);
    case 2: return launch_x<2>(a, rtype, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ojbkq
