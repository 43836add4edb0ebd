// Products with 8-bit activations for few tokens: a decoding step, a small
// batch, a narrow layer.
#include "fp8_product.h"

namespace ojbkq {
namespace {

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// Y for few tokens.  Bound by reading the weights (for the fewest tokens by
// latency), so a workgroup takes few channels, 16 RB, for all features, and its
// eight waves split the features: chunks of 128 go round the waves, which meet
// at the end in LDS, where their sums are added in wave order.  A lane's
// operands are 32 features of channel l % 16 and of token l % 16, both brought to
// 16 bits in registers, a quarter of them to each of the chunk's four products of
// 16 x 16 x 32.  (The matrix cores' 8-bit products keep about 13 bits beside the
// largest of eight neighbours; these keep float32's.)  The activations are the A
// operand, so a lane's four sums belong to one channel and take its scale.
//   e4m3 weights: both in bf16, which holds a value times a power of two.
//   Codes: both in fp16, without the scales.  A code q set into the low bits of
//   fp16's 1024 is 1024 + q, from which a packed subtraction takes 1024 + z: of
//   two 4-bit codes a shift (but for the lowest ones), a mask, an or and the
//   subtraction, against six operations by way of float32 (some 410 vector
//   instructions beside the 32 products of a chunk of 64 channels and 32 tokens,
//   240 of them for the codes).
//
// Read from memory that way, neighbouring lanes would be rows apart, and every
// lane's 16 bytes an access of the cache by itself (690 accesses a chunk of 32
// channels and tokens; they were the bound).  So a wave's rows come straight to
// LDS, neighbouring lanes along a row, into a ring of kDepth chunks of its own;
// no barrier is needed until the end.
//
// 4096 x 4096, one token, kernels in a graph: e4m3 6.0 us, 4-bit codes 6.6, of
// which the latency of a launch, of the first loads and of the sums' meeting is the
// larger part (its 16.8 or 8.4 MB would pass in 3.2 or 1.6); 24 tokens, codes of
// 14336 x 4096: 16 us, bound by the vector instructions that bring both operands
// to 16 bits.  Of 33 to 1000 tokens every 32 read and convert the weights anew:
// 4096 x 4096, 256 tokens 28 us, some seven times the transfer.
template <int SRC, int RB, int NB>
struct Few {
  static constexpr int kTok = 16 * NB, kChan = 16 * RB, kWaves = 8;
  static constexpr int kPitch = kChan + 4, kRed = kTok * kPitch;   // floats of a wave's sums, by tokens
  static constexpr int kRow = SRC ? 16 * SRC : 128;                      // bytes of a chunk's row of weights
  static constexpr int kW = (kChan * kRow + 1023) / 1024 * 1024, kX = kTok * 128;
  // then a word for every channel and token with its scale, and of codes one
  // with the zero point; lane i's from 4 i on
  static constexpr int kS = kW + kX, kXs = kS + 256, kZ = kXs + 256, kStage = SRC ? kZ + 256 : kZ;
  static constexpr int kDepth = kWaves * 4 * kStage <= 160 * 1024 ? 4 : 2;
  static constexpr int kWide = kW / 1024;
  static constexpr int kLoads = kWide + kX / 1024 + (kStage - kS) / 256;   // of a chunk, at least
  static constexpr int kRing = kWaves * kDepth * kStage, kSums = kWaves * kRed * 4;
};

template <int SRC, int RB, int NB>
__global__ __launch_bounds__(512) void product_few8_kernel(Product8Args a) {
  typedef Few<SRC, RB, NB> F;
  constexpr int kTok = F::kTok, kChan = F::kChan, kWaves = F::kWaves, kDepth = F::kDepth;
  __shared__ __align__(16) uint8_t lds[F::kRing > F::kSums ? F::kRing : F::kSums];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int64_t J0 = (int64_t)blockIdx.x * kChan, T0 = (int64_t)blockIdx.y * kTok;
  const int nch = (int)((a.m + 127) >> 7);
  uint8_t* const ring = lds + wave * (kDepth * F::kStage);

  // rows past the last one repeat it: they feed only sums that are not stored
  auto channel = [&](int r) { return J0 + r < a.n ? J0 + r : a.n - 1; };
  auto token = [&](int r) { return T0 + r < a.T ? T0 + r : a.T - 1; };
  const uint32_t* const P = a.P;

  // ---- memory to LDS --------------------------------------------------------
  // A row of 128 bytes in LDS has its 16-byte piece p at place p ^ (row % 8),
  // one of 64 bytes (4-bit codes) at p ^ (row / 4 % 4), which spreads the reads
  // below over the banks; load h of a wave fills 1 KB, lane i its 16 bytes from
  // 16 i on.
  const int r8 = lane >> 3, p8 = (lane & 7) ^ r8;
  // whole pieces behind the last feature are read from the row's first one
  auto load_rows = [&](const uint8_t* row, int64_t k, uint8_t* to) {
    load_to_lds16_at(row + k + (k + 16 * p8 < a.m ? 16 * p8 : 0), to);
  };
  const bool wide = SRC == 0 || (a.wpr % 4 == 0 && reinterpret_cast<uintptr_t>(P) % 16 == 0);
  auto load_chunk = [&](int c, int slot) {
    uint8_t* const w = ring + slot * F::kStage;
    const int64_t k = 128 * (int64_t)c;
#pragma unroll
    for (int h = 0; h < F::kWide; ++h) {
      if constexpr (SRC == 0) {
        load_rows(a.W8 + channel(8 * h + r8) * a.ldw, k, w + 1024 * h);
      } else if (wide && k + 128 <= a.m) {
        constexpr int kPieces = kChan * SRC;
        const int u = 64 * h + lane < kPieces ? 64 * h + lane : kPieces - 1;
        const int r = u / SRC, p = SRC == 4 ? (u % SRC) ^ ((r >> 2) & 3) : u % SRC;
        load_to_lds16_at(P + channel(r) * a.wpr + 4 * SRC * (int64_t)c + 4 * p, w + 1024 * h);
      } else {
        // word by word (words behind the row's last one: its activations are 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          constexpr int kWords = kChan * SRC * 4;
          int u = 256 * h + 64 * e + lane;
          u = u < kWords ? u : kWords - 1;
          const int r = u / (4 * SRC), v = u % (4 * SRC);
          const int64_t at = 4 * SRC * (int64_t)c + (SRC == 4 ? v ^ ((r & 12)) : v);
          load_to_lds4_at(P + channel(r) * a.wpr + (at < a.wpr ? at : a.wpr - 1), w + 1024 * h + 256 * e);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2 * NB; ++h) load_rows(a.X8 + token(8 * h + r8) * a.ldx, k, w + F::kW + 1024 * h);
  };
  // scales: a lane to each row (of the e8m0 ones a word, that of four chunks)
  const bool bytes = SRC == 0 && a.ws_e8m0;
  const int64_t srow = (channel(lane & (kChan - 1)) >> a.ws_shift) * a.ws_ld;
  const uint8_t* const s_at = static_cast<const uint8_t*>(a.ws) + (bytes ? srow : 4 * srow);
  const uint8_t* const xs_at = a.xs + token(lane & (kTok - 1)) * a.lds;
  auto load = [&](int i) {
    const int c = wave + kWaves * i, c0 = c & ~3;
    uint8_t* const to = ring + (i & (kDepth - 1)) * F::kStage;
    const uint32_t b = a.ws_div == 1 ? (uint32_t)c : (uint32_t)c / a.ws_div;
    load_to_lds4_at(s_at + (bytes ? (uint32_t)c0 : 4 * b), to + F::kS);
    if constexpr (SRC != 0) load_to_lds4_at(a.Z + srow + b, to + F::kZ);
    load_to_lds4_at(xs_at + c0, to + F::kXs);
    load_chunk(c, i & (kDepth - 1));
  };
  const int count = wave < nch ? (nch - wave + kWaves - 1) / kWaves : 0;   // this wave's chunks

  v4 acc[RB][NB];
#pragma unroll
  for (int x = 0; x < RB; ++x)
#pragma unroll
    for (int y = 0; y < NB; ++y) acc[x][y] = v4{0.f, 0.f, 0.f, 0.f};

#pragma unroll 1
  for (int i = 0; i < kDepth && i < count; ++i) load(i);
#pragma unroll 1
  for (int i = 0; i < count; ++i) {
    // chunk i has arrived when no more loads are under way than the chunks
    // behind it have (at least kLoads each)
    const int behind = count - 1 - i < kDepth - 1 ? count - 1 - i : kDepth - 1;
    if (behind == 3) wait_loads<3 * F::kLoads>();
    else if (behind == 2) wait_loads<2 * F::kLoads>();
    else if (behind == 1) wait_loads<F::kLoads>();
    else wait_loads<0>();

    const int c = wave + kWaves * i, q = c & 3;
    const uint8_t* const w = ring + (i & (kDepth - 1)) * F::kStage;
    auto word = [&](int at, int n) { return *reinterpret_cast<const uint32_t*>(w + at + 4 * n); };
    uint32_t cw[RB][SRC ? SRC : 8], cx[NB][8], cs[RB], cz[RB];
    u4 cxs[NB];
    // pieces g4 and 4 + g4 of a row of 128 bytes
    auto row32 = [&](const uint8_t* rows, int r, uint32_t (&v)[8]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u4 p = *reinterpret_cast<const u4*>(rows + 128 * r + 16 * ((4 * h + g4) ^ (r & 7)));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = p[e];
      }
    };
#pragma unroll
    for (int x = 0; x < RB; ++x) {
      const int r = 16 * x + i16;
      if constexpr (SRC == 0) {
        row32(w, r, cw[x]);
      } else {
        // pieces and features as the activations': 16 codes from each of two
        // places, SRC half words; word e takes half word e of both
        const uint8_t* const at = w + F::kRow * r;
        if constexpr (SRC == 4) {
          u2v h[2];
#pragma unroll
          for (int f = 0; f < 2; ++f)
            h[f] = *reinterpret_cast<const u2v*>(at + 16 * ((2 * f + (g4 >> 1)) ^ ((r >> 2) & 3)) + 8 * (g4 & 1));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            cw[x][e] = __builtin_amdgcn_perm(h[1][e >> 1], h[0][e >> 1], (e & 1) ? 0x07060302u : 0x05040100u);
        } else {
          const uint16_t* const h = reinterpret_cast<const uint16_t*>(at) + SRC * g4;
#pragma unroll
          for (int e = 0; e < SRC; ++e) cw[x][e] = h[e] | ((uint32_t)h[4 * SRC + e] << 16);
        }
        cz[x] = word(F::kZ, r);
      }
      cs[x] = word(F::kS, r);
    }
#pragma unroll
    for (int y = 0; y < NB; ++y) {
      row32(w + F::kW, 16 * y + i16, cx[y]);
      // (the scales of four chunks) of this lane's token, or of its four sums'
      if constexpr (SRC == 0) cxs[y][0] = word(F::kXs, 16 * y + i16);
      else cxs[y] = *reinterpret_cast<const u4*>(w + F::kXs + 4 * (16 * y + 4 * g4));
    }
    // whether every token's scale is 2^-100 to 2^100, a lane to each token
    const uint32_t mine = SRC ? word(F::kXs, lane & (kTok - 1)) >> (8 * q) : 0u;
    wait_lds();
    const bool usual = !__any((mine & 0xffu) - 27u > 200u);
    if (i + kDepth < count) load(i + kDepth);

    if (128 * (int64_t)(c + 1) > a.m) {
      // what stands behind a row's last value is not used
      const int64_t k = 128 * (int64_t)c + 16 * g4;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t ke = k + 64 * (e >> 2) + 4 * (e & 3);
#pragma unroll
        for (int y = 0; y < NB; ++y) cx[y][e] = features_below(cx[y][e], ke, a.m);
        if constexpr (SRC == 0)
#pragma unroll
          for (int x = 0; x < RB; ++x) cw[x][e] = features_below(cw[x][e], ke, a.m);
      }
    }

    v4 d[RB][NB];
#pragma unroll
    for (int x = 0; x < RB; ++x)
#pragma unroll
      for (int y = 0; y < NB; ++y) d[x][y] = v4{0.f, 0.f, 0.f, 0.f};
    if constexpr (SRC == 0) {
      SplitScale s[RB];
      float sx[NB];
#pragma unroll
      for (int y = 0; y < NB; ++y) sx[y] = from_e8m0((cxs[y][0] >> (8 * q)) & 0xffu);
#pragma unroll
      for (int x = 0; x < RB; ++x)
        s[x] = split_scale(bytes ? from_e8m0((cs[x] >> (8 * q)) & 0xffu) : __uint_as_float(cs[x]));
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        b8 fx[NB];
#pragma unroll
        for (int y = 0; y < NB; ++y) fx[y] = to_bf16(cx[y][2 * p], cx[y][2 * p + 1], sx[y]);
#pragma unroll
        for (int x = 0; x < RB; ++x) {
          const b8 fw = to_bf16(cw[x][2 * p], cw[x][2 * p + 1], s[x].power);
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
          for (int r = 0; r < 4; ++r)
            acc[x][y][r] = __builtin_fmaf(d[x][y][r], s[x].rest, acc[x][y][r]);
    } else {
      h2 less[RB];   // 1024 + z
#pragma unroll
      for (int x = 0; x < RB; ++x) {
        const _Float16 z = (_Float16)(1024.f + whole_zero<SRC>(__uint_as_float(cz[x])));
        less[x] = h2{z, z};
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        // features 4 p .. + 3 of both halves, in turn
        h8 fx[NB];
#pragma unroll
        for (int y = 0; y < NB; ++y) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t v = __builtin_amdgcn_perm(cx[y][4 + p], cx[y][p], h ? 0x07030602u : 0x05010400u);
            const h2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.f, false);
            const h2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.f, true);
            fx[y][4 * h] = lo.x;
            fx[y][4 * h + 1] = lo.y;
            fx[y][4 * h + 2] = hi.x;
            fx[y][4 * h + 3] = hi.y;
          }
        }
#pragma unroll
        for (int x = 0; x < RB; ++x) {
          h8 fw;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            constexpr uint32_t kMask = 0x00010001u * ((1u << SRC) - 1u);
            const int b = (4 * p + e) * SRC, at = b >> 4, sh = b & 15;
            uint32_t v = (cw[x][at] >> sh) & kMask;
            if (sh + SRC > 16)   // a code that goes on in the next half word
              v = ((cw[x][at] >> sh) & (0x00010001u * ((1u << (16 - sh)) - 1u))) |
                  ((cw[x][at + 1 < SRC ? at + 1 : at] << (16 - sh)) & kMask &
                   ~(0x00010001u * ((1u << (16 - sh)) - 1u)));
            const h2 f = __builtin_bit_cast(h2, v | 0x64006400u) - less[x];
            fw[2 * e] = f.x;
            fw[2 * e + 1] = f.y;
          }
#pragma unroll
          for (int y = 0; y < NB; ++y)
            d[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fx[y], fw, d[x][y], 0, 0, 0);
        }
      }
      // A block's sums d are multiples of 2^-9 below 2^20, so with the scales of
      // the usual tokens they are float32's normal numbers.  For the others, the
      // weight scale's power of two joins theirs in one exponent and the rest, 1
      // to 2, comes last: only a sum that is beyond float32 as a result too
      // overflows.  (That for all tokens costs some 6% at 14336 x 4096, 24 tokens.)
      if (__builtin_expect(!usual, 0)) {
#pragma unroll
        for (int x = 0; x < RB; ++x) {
          const SplitScale s = split_scale(__uint_as_float(cs[x]));
          const int power = (int)(__float_as_uint(s.power) >> 23) - 254;   // (less the bias of both)
          cs[x] = __float_as_uint(s.rest);
#pragma unroll
          for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int code = (int)((cxs[y][r] >> (8 * q)) & 0xffu);
              d[x][y][r] = code == 255 ? __builtin_nanf("") : __builtin_ldexpf(d[x][y][r], code + power);
            }
        }
#pragma unroll
        for (int y = 0; y < NB; ++y) cxs[y] = u4{0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};   // 1
      }
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float sx = __uint_as_float(((cxs[y][r] >> (8 * q)) & 0xffu) << 23);
#pragma unroll
          for (int x = 0; x < RB; ++x)
            acc[x][y][r] = __builtin_fmaf(d[x][y][r] * sx, __uint_as_float(cs[x]), acc[x][y][r]);
        }
    }
  }

  // the waves' sums, in wave order: lane l holds tokens 4 (l / 16) + r of
  // channel l % 16
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int x = 0; x < RB; ++x)
#pragma unroll
    for (int y = 0; y < NB; ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        red[wave * F::kRed + (16 * y + 4 * g4 + r) * F::kPitch + 16 * x + i16] = acc[x][y][r];
  __syncthreads();
  for (int e = tid; e < kChan * kTok; e += 64 * kWaves) {
    const int jj = a.tokens_first ? e % kChan : e / kTok, tt = a.tokens_first ? e / kChan : e % kTok;
    float v = red[tt * F::kPitch + jj];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += red[w * F::kRed + tt * F::kPitch + jj];
    if (J0 + jj < a.n && T0 + tt < a.T) store_y(a, J0 + jj, T0 + tt, v);
  }
}

template <int SRC, int NB>
hipError_t launch_rb(const Product8Args& a, hipStream_t s) {
  const int64_t gy = (a.T + 16 * NB - 1) / (16 * NB);
  auto grid = [&](int rb) { return dim3((unsigned)((a.n + 16 * rb - 1) / (16 * rb)), (unsigned)gy); };
  // As many channels as leave work for 160 of the 256 CUs: fewer bring a second
  // round of workgroups, each of which reads the activations again (us for 64 /
  // 32 / 16 channels: codes 14336 x 4096, 24 tokens 16.5 / 19.1 / 27.4, 11008 x
  // 4096 16.1 / 19.1 / 21.5; for 32 / 16: codes 4096 x 11008, 32 tokens, 128
  // and 256 workgroups, 20.3 / 15.9; e4m3, m = 4096, 24 tokens: 4096 channels, 128
  // and 256 workgroups, 8.1 / 6.9, 5120, 160 and 320, 8.6 / 11.3, 14336 16.9 /
  // 21.6; one token 6.4 / 5.9, 7.1 / 9.5, 14.3 / 18.1).  64 e4m3 channels do not
  // fit in LDS twice.
  if constexpr (SRC != 0)
    if ((a.n + 63) / 64 * gy >= 160) {
      product_few8_kernel<SRC, 4, NB><<<grid(4), dim3(512), 0, s>>>(a);
      return hipGetLastError();
    }
  if ((a.n + 31) / 32 * gy >= 160)
    product_few8_kernel<SRC, 2, NB><<<grid(2), dim3(512), 0, s>>>(a);
  else
    product_few8_kernel<SRC, 1, NB><<<grid(1), dim3(512), 0, s>>>(a);
  return hipGetLastError();
}

template <int SRC>
hipError_t launch(const Product8Args& a, hipStream_t s) {
  return a.T <= 16 ? launch_rb<SRC, 1>(a, s) : launch_rb<SRC, 2>(a, s);
}

}  // namespace

hipError_t launch_product_few8(const Product8Args& a, int bits, hipStream_t stream) {
  // (the second dimension of a grid holds 65535)
  const int64_t step = (int64_t)65535 * 32;
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
