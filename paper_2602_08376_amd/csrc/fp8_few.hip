// Products with 8-bit activations for few tokens: a decoding step, a small
// batch, a narrow layer.
#include "fp8_product.h"

namespace ojbkq {
namespace {

// Y for few tokens.  Bound by reading the weights (for the fewest tokens by
// latency), so a workgroup takes few channels, 16 RB, for all features, and its
// eight waves split the features: chunks of 128 go round the waves, which meet
// at the end in LDS, where their sums are added in wave order.  Lane l holds
// features 32 (l / 16) .. + 31 of a chunk, of channel l % 16 and of token l %
// 16, both brought to bf16 in registers (which holds an e4m3 value times its
// power-of-two scale, and a code less its zero point, exactly): product s of
// the chunk's four v_mfma_f32_16x16x32_bf16 takes its features 8 s .. + 7.
// (The matrix cores' 8-bit products keep about 17 bits beside the largest of
// eight neighbours; these keep float32's.)  The activations are the A operand,
// so a lane's four sums belong to one channel and take its scale.
template <int SRC, int RB, int NB>
__global__ __launch_bounds__(512) void product_few8_kernel(Product8Args a) {
  constexpr int kTok = 16 * NB, kChan = 16 * RB, kRed = kChan * kTok;
  constexpr int kDepth = RB * NB == 1 ? 4 : RB * NB <= 4 ? 2 : 1;   // chunks under way
  __shared__ float red[8 * kRed];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int64_t J0 = (int64_t)blockIdx.x * kChan, T0 = (int64_t)blockIdx.y * kTok;
  const int nch = (int)((a.m + 127) / 128);

  // rows past the last one repeat it: they feed only sums that are not stored
  int64_t j[RB], t[NB];
#pragma unroll
  for (int x = 0; x < RB; ++x) j[x] = J0 + 16 * x + i16 < a.n ? J0 + 16 * x + i16 : a.n - 1;
#pragma unroll
  for (int y = 0; y < NB; ++y) t[y] = T0 + 16 * y + i16 < a.T ? T0 + 16 * y + i16 : a.T - 1;

  struct Stage {
    uint32_t w[RB][SRC ? SRC : 8];   // 32 e4m3 values (SRC = 0) or codes of SRC bits
    float s[RB], z[RB];
    u4 x[NB][2];
    uint32_t xs[NB];
  };
  // 32 e4m3 values of a row from feature k on, in pieces of 16 (of which one
  // with any feature below m is readable)
  auto run = [&](const uint8_t* row, int64_t k, u4 (&v)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[h] = k + 16 * h < a.m ? *reinterpret_cast<const u4*>(row + k + 16 * h) : u4{0u, 0u, 0u, 0u};
  };
  auto fetch = [&](int c, Stage& st) {
    const int64_t k = 128 * (int64_t)c + 32 * g4;
#pragma unroll
    for (int x = 0; x < RB; ++x) {
      if constexpr (SRC == 0) {
        u4 v[2];
        run(a.W8 + j[x] * a.ldw, k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) st.w[x][e] = v[e >> 2][e & 3];
      } else {
        const uint32_t* p = a.P + j[x] * a.wpr;
        const int64_t wi = k / 32 * SRC;
#pragma unroll
        for (int e = 0; e < SRC; ++e) st.w[x][e] = p[wi + e < a.wpr ? wi + e : a.wpr - 1];
        st.z[x] = a.Z[j[x] * a.ws_ld + c / a.ws_div];
      }
      st.s[x] = weight_scale(a, j[x], c);
    }
#pragma unroll
    for (int y = 0; y < NB; ++y) {
      run(a.X8 + t[y] * a.ldx, k, st.x[y]);
      st.xs[y] = a.xs[t[y] * a.lds + c];
    }
  };

  v4 acc[RB][NB];
#pragma unroll
  for (int x = 0; x < RB; ++x)
#pragma unroll
    for (int y = 0; y < NB; ++y) acc[x][y] = v4{0.f, 0.f, 0.f, 0.f};
  auto products = [&](int c, Stage& st) {
    const int64_t k = 128 * (int64_t)c + 32 * g4;
    const bool whole = 128 * (int64_t)(c + 1) <= a.m;
    if (!whole) {
      // what stands behind a row's last value is not used
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          st.x[y][e >> 2][e & 3] = features_below(st.x[y][e >> 2][e & 3], k + 4 * e, a.m);
      if constexpr (SRC == 0) {
#pragma unroll
        for (int x = 0; x < RB; ++x)
#pragma unroll
          for (int e = 0; e < 8; ++e) st.w[x][e] = features_below(st.w[x][e], k + 4 * e, a.m);
      }
    }
    v4 d[RB][NB];
#pragma unroll
    for (int x = 0; x < RB; ++x)
#pragma unroll
      for (int y = 0; y < NB; ++y) d[x][y] = v4{0.f, 0.f, 0.f, 0.f};
    float power[RB];
    if constexpr (SRC == 0) {
#pragma unroll
      for (int x = 0; x < RB; ++x) {
        const SplitScale sp = split_scale(st.s[x]);
        power[x] = sp.power;
        st.s[x] = sp.rest;
      }
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      b8 fx[NB];
#pragma unroll
      for (int y = 0; y < NB; ++y)
        fx[y] = to_bf16(st.x[y][s >> 1][2 * (s & 1)], st.x[y][s >> 1][2 * (s & 1) + 1],
                        from_e8m0(st.xs[y]));
#pragma unroll
      for (int x = 0; x < RB; ++x) {
        b8 fw;
        if constexpr (SRC == 0) {
          fw = to_bf16(st.w[x][2 * s], st.w[x][2 * s + 1], power[x]);
        } else {
          // (codes past the last one are zero bits; their activations are 0)
          const float z = whole_zero<SRC>(st.z[x]);
#pragma unroll
          for (int e = 0; e < 8; ++e) fw[e] = (__bf16)((float)code_of<SRC>(st.w[x], 8 * s + e) - z);
        }
#pragma unroll
        for (int y = 0; y < NB; ++y)
          d[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[y], fw, d[x][y], 0, 0, 0);
      }
    }
#pragma unroll
    for (int x = 0; x < RB; ++x)
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[x][y][r] = __builtin_fmaf(d[x][y][r], st.s[x], acc[x][y][r]);
  };

  Stage st[kDepth];
#pragma unroll
  for (int d = 0; d < kDepth; ++d)
    if (wave + 8 * d < nch) fetch(wave + 8 * d, st[d]);
  for (int c = wave; c < nch; c += 8 * kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      const int cd = c + 8 * d;
      if (cd >= nch) break;
      Stage cur = st[d];
      if (cd + 8 * kDepth < nch) fetch(cd + 8 * kDepth, st[d]);
      products(cd, cur);
    }
  }

  // the waves' sums, in wave order: lane l holds tokens 4 (l / 16) + r of
  // channel l % 16
#pragma unroll
  for (int x = 0; x < RB; ++x)
#pragma unroll
    for (int y = 0; y < NB; ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        red[wave * kRed + (16 * x + i16) * kTok + 16 * y + 4 * g4 + r] = acc[x][y][r];
  __syncthreads();
  for (int e = tid; e < kRed; e += 512) {
    const int jj = a.tokens_first ? e % kChan : e / kTok, tt = a.tokens_first ? e / kChan : e % kTok;
    float v = red[jj * kTok + tt];
#pragma unroll
    for (int w = 1; w < 8; ++w) v += red[w * kRed + jj * kTok + tt];
    if (J0 + jj < a.n && T0 + tt < a.T) store_y(a, J0 + jj, T0 + tt, v);
  }
}

template <int SRC, int NB>
hipError_t launch_rb(const Product8Args& a, hipStream_t s) {
  // as many channels per workgroup as leave one for every CU
  const int64_t gy = (a.T + 16 * NB - 1) / (16 * NB);
  auto grid = [&](int rb) { return dim3((unsigned)((a.n + 16 * rb - 1) / (16 * rb)), (unsigned)gy); };
  if ((a.n + 63) / 64 * gy >= 256)
    product_few8_kernel<SRC, 4, NB><<<grid(4), dim3(512), 0, s>>>(a);
  else if ((a.n + 31) / 32 * gy >= 256)
    product_few8_kernel<SRC, 2, NB><<<grid(2), dim3(512), 0, s>>>(a);
  else
    product_few8_kernel<SRC, 1, NB><<<grid(1), dim3(512), 0, s>>>(a);
  return hipGetLastError();
}

template <int SRC>
hipError_t launch(const Product8Args& a, hipStream_t s) {
  if (a.T <= 16) return launch_rb<SRC, 1>(a, s);
  if (a.T <= 32) return launch_rb<SRC, 2>(a, s);
  return launch_rb<SRC, 4>(a, s);
}

}  // namespace

hipError_t launch_product_few8(const Product8Args& a, int bits, hipStream_t stream) {
  // (the second dimension of a grid holds 65535)
  const int64_t step = (int64_t)65535 * 64;
  for (int64_t t = 0; t < a.T; t += step) {
    Product8Args b = a;
    const size_t size = a.ytype == 0 ? 4 : 2;
    b.T = a.T - t < step ? a.T - t : step;
    b.X8 = a.X8 + t * a.ldx;
    b.xs = a.xs + t * a.lds;
    b.Y = static_cast<char*>(a.Y) + (a.tokens_first ? t * a.ldy : t) * size;
    hipError_t e;
    switch (bits) {
      case 0: e = launch<0>(b, stream); break;
      case 1: e = launch<1>(b, stream); break;
      case 2: e = launch<2>(b, stream); break;
      case 3: e = launch<3>(b, stream); break;
      case 4: e = launch<4>(b, stream); break;
      default: return hipErrorInvalidValue;
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ojbkq
