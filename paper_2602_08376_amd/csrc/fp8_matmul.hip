// Products with 8-bit activations for many tokens, and the choice of the kernel
// for the sizes at hand.
//
//   expand_codes_kernel  packed codes -> e4m3 values q - z, once
//   product8_kernel      Y of e4m3 weights and activations, in tiles
#include "fp8_product.h"
#include "kernels.h"

namespace ojbkq {
namespace {

typedef int i8 __attribute__((ext_vector_type(8)));

// ---- codes in e4m3 ---------------------------------------------------------

// W8 [n, ldw] e4m3 = q - z of the packed codes: whole numbers of at most 15,
// exact in e4m3's 4 significant bits.  One thread to 32 codes (BITS words) of
// a row, and of others below it.  Bound by memory: it writes a byte for every
// code.  4096 x 4096, 4 bits: 9.6 us; 4096 x 11008, 3 bits: 15.4 us, 4.0 TB/s.
template <int BITS>
__global__ __launch_bounds__(256) void expand_codes_kernel(Product8Args a, uint8_t* W8, int64_t ldw) {
  const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;   // 32 codes of a row
  if (32 * u >= ldw) return;
  // (runs past the last feature: any group will do, they are not used)
  const uint32_t grp = 32 * u < a.m ? (uint32_t)(u / 4) / a.ws_div : 0u;
  const bool whole = (u + 1) * BITS <= a.wpr;
  for (int64_t j = blockIdx.y; j < a.n; j += gridDim.y) {
    const uint32_t* const row = a.P + j * a.wpr + u * BITS;
    uint32_t w[BITS];
    if (whole) {
      typedef uint32_t Any __attribute__((ext_vector_type(BITS), aligned(4)));
      const Any v = *reinterpret_cast<const Any*>(row);
#pragma unroll
      for (int q = 0; q < BITS; ++q) w[q] = v[q];
    } else {
#pragma unroll
      for (int q = 0; q < BITS; ++q) w[q] = u * BITS + q < a.wpr ? row[q] : 0u;
    }
    const float z = whole_zero<BITS>(a.Z[j * a.ws_ld + grp]);
    u4 out[2];
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      float v[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = (float)code_of<BITS>(w, 4 * d + c) - z;
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
      p = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], p, true);
      out[d >> 2][d & 3] = (uint32_t)p;
    }
    *reinterpret_cast<u4*>(W8 + j * ldw + 32 * u) = out[0];
    *reinterpret_cast<u4*>(W8 + j * ldw + 32 * u + 16) = out[1];
  }
}

// ---- tiles -----------------------------------------------------------------

// Output tile of this workgroup: each XCD (of eight, dealt workgroups round
// robin) takes a contiguous run of tiles, walked in groups of 8 channel tiles
// with the token tiles outer, so that the workgroups it runs at once share
// their panels in its L2.
__device__ __forceinline__ void tile_of(int64_t tiles_n, int64_t& tj, int64_t& tt) {
  constexpr int64_t kGroup = 8;
  const int64_t nb = gridDim.x, tiles_t = nb / tiles_n;
  int64_t t = blockIdx.x;
  if ((nb & 7) == 0) t = (t & 7) * (nb >> 3) + (t >> 3);
  const int64_t per = kGroup * tiles_t, first = (t / per) * kGroup;
  const int64_t rows = tiles_n - first < kGroup ? tiles_n - first : kGroup;
  const int64_t r = t % per;
  tj = first + r % rows;
  tt = r / rows;
}

// Sums are formed where they stand (the compiler moves them, with the products
// they come from, behind the branches and barriers that follow, and has to hold
// all operands until then).
__device__ __forceinline__ void pin(v4& v) { asm volatile("" : "+v"(v)); }

template <class E, int N>
__device__ __forceinline__ void store_run(E* p, const float (&v)[N], int64_t left) {
  typedef E Any __attribute__((ext_vector_type(N), aligned(sizeof(E))));
  if (left >= N) {
    Any o;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = (E)v[e];
    *reinterpret_cast<Any*>(p) = o;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) p[e] = (E)v[e];
  }
}

// Tiles of TT tokens x TC channels, a block of 128 features to a stage, BUFS
// stages in LDS; WR x WC waves, each of 16 NX tokens x 64 channels: its weights
// of a stage stay in registers while its activations pass.  Both operands go
// straight from memory to LDS in lines of 128 bytes, 16-byte chunk c of line l
// at slot c ^ (l % 8), which spreads the operand reads of 16 lines x 4 chunks
// over all banks (the conflicts that a profile counts, 0.2 to 0.3 for each LDS
// instruction of kScaled and kExact, are some 8 cycles a stage and wave, and kPowers,
// which does without the reads of the weight scales' rests, has none).
// Line 16 x + i of the activations holds token 32 (x / 2) + 8 (i / 4) + 4 (x %
// 2) + i % 4, line 16 y + i of a wave's 64 of weights channel 4 i + y: a lane
// then ends up with runs of 8 tokens and of 4 channels, whichever is contiguous
// in Y.
// kExact: operands brought to bf16, with the activations' scales and the powers
// of two of the weights', exactly, and multiplied there.  Otherwise
// v_mfma_scale_f32_16x16x128_f8f6f4 takes them as they are, with these scales,
// at twice the rate; kPowers: the weights' scales are powers of two, so it takes
// the sums so far as well.
// 256 tokens x 256 channels, a wave 128 x 64, reads least from LDS for its
// products (1536 of a stage's cycles, beside 2048 of the matrix cores); it leaves
// a CU one workgroup, so 128 x 128, two to a CU, does better on few tiles.
// Float32 results need bf16 operands in registers (twice the size) and so smaller
// ones: a wave 64 x 64 in both, 256 x 128 with three stages in LDS.
// 4096 x 4096 x 32768, float32 scales, bfloat16 results: 543 to 585 us, 2.0 to 1.9
// PFLOP/s (matrix cores busy 45% of the time; beside each product stand four
// FMAs that scale its sums); 4096 x 11008, 1999 tokens, e8m0: 88 us, 2.05; with
// float32 results 163, 1.10 (bf16 products; 43%).  What is left is the waves
// waiting for each other at a stage's barrier, and power: zeros for operands are
// 13% faster (502 us; at 1999 tokens 5%, 83 us).  Three stages of 256 x 128 or 128 x 256 for 16-bit results: 98.9
// against 97.7 us and, where 256 x 256 serves, 667 against 538.
enum { kPowers, kScaled, kExact };
template <int TT, int TC, int WR, int WC, int BUFS, int HOW>
__global__ __launch_bounds__(64 * WR * WC, 2) void product8_kernel(Product8Args a, int64_t tiles_n) {
  constexpr int NX = TT / WR / 16, kWaves = WR * WC, kLines = TT + TC;
  static_assert(TC == 64 * WC && NX % 2 == 0 && kLines <= 64 * kWaves && TT <= 256 && TC <= 256, "");
  __shared__ __align__(16) uint8_t sX[BUFS][TT * 128], sW[BUFS][TC * 128];
  // scales of four stages: of a line of activations (a byte each), of a channel
  // of weights (a float32 each, or e8m0 bytes in the first)
  __shared__ __align__(16) uint32_t sxs[2][TT], sws[2][4][TC];
  __shared__ __align__(16) uint8_t swp[2][4][TC];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int wr = wave % WR, wc = wave / WR;
  int64_t tj, tt;
  tile_of(tiles_n, tj, tt);
  const int64_t J0 = tj * TC, T0 = tt * TT;
  const int nst = (int)((a.m + 127) / 128);

  auto token_of = [](int line) {
    const int i = line & 15;
    return (line & ~31) + 8 * (i >> 2) + 4 * ((line >> 4) & 1) + (i & 3);
  };
  auto channel_of = [](int line) { return (line & ~63) + 4 * (line & 15) + ((line >> 4) & 3); };

  // ---- memory to LDS --------------------------------------------------------
  // Load q of a wave fills lines 8 (QX wave + q) .. + 7; rows past the last one
  // repeat it (they feed only results that are not stored).
  constexpr int QX = TT / 8 / kWaves, QW = TC / 8 / kWaves;
  const int last_t = (int)(a.T - 1 - T0 < TT - 1 ? a.T - 1 - T0 : TT - 1);
  const int last_j = (int)(a.n - 1 - J0 < TC - 1 ? a.n - 1 - J0 : TC - 1);
  const uint32_t piece = 16 * ((lane & 7) ^ (lane >> 3));
  uint32_t xoff[QX], woff[QW];
#pragma unroll
  for (int q = 0; q < QX; ++q) {
    const int t = token_of(8 * (QX * wave + q) + (lane >> 3));
    xoff[q] = (uint32_t)(t < last_t ? t : last_t) * (uint32_t)a.ldx + piece;
  }
#pragma unroll
  for (int q = 0; q < QW; ++q) {
    const int j = channel_of(8 * (QW * wave + q) + (lane >> 3));
    woff[q] = (uint32_t)(j < last_j ? j : last_j) * (uint32_t)a.ldw + piece;
  }
  const uint8_t* const xbase = a.X8 + T0 * a.ldx;
  const uint8_t* const wbase = a.W8 + J0 * a.ldw;
  const bool ragged = (a.m & 127) != 0;
  auto load = [&](int st) {
    const int64_t k0 = 128 * (int64_t)st;
    const int buf = st % BUFS;
    // a piece past the last feature reads the row's first one; mask_tail clears it
    const uint32_t back = ragged && st == nst - 1 && k0 + piece >= a.m ? piece : 0u;
#pragma unroll
    for (int q = 0; q < QW; ++q) load_to_lds16(wbase + k0, woff[q] - back, sW[buf] + 1024 * (QW * wave + q));
#pragma unroll
    for (int q = 0; q < QX; ++q) load_to_lds16(xbase + k0, xoff[q] - back, sX[buf] + 1024 * (QX * wave + q));
  };
  // the last stage of a ragged row: everything from feature m on cleared
  auto mask_tail = [&](int st) {
    if (tid >= kLines) return;
    const int left = (int)(a.m - 128 * (int64_t)st), buf = st % BUFS;
    uint8_t* const line = tid < TT ? sX[buf] + 128 * tid : sW[buf] + 128 * (tid - TT);
    for (int c = left / 16; c < 8; ++c) {
      u4* const p = reinterpret_cast<u4*>(line + 16 * (c ^ (tid & 7)));
      u4 v = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = features_below(v[e], 16 * c + 4 * e, left);
      *p = v;
    }
  };
  // a wave to 64 lines or channels (their addresses formed anew every time, not
  // held in registers)
  const bool bytes = a.ws_e8m0 != 0;
  auto load_scales = [&](int quad) {
    int w = wave;
    __asm__("" : "+s"(w));
    const int buf = quad & 1;
    if (w < TT / 64) {
      const int t = token_of(64 * w + lane);
      load_to_lds4_at(a.xs + (T0 + (t < last_t ? t : last_t)) * a.lds + 4 * quad, &sxs[buf][64 * w]);
    } else if (w < kLines / 64) {
      const int c0 = 64 * (w - TT / 64), j = c0 + lane;
      const int64_t at = ((J0 + (j < last_j ? j : last_j)) >> a.ws_shift) * a.ws_ld;
      const uint8_t* const S = static_cast<const uint8_t*>(a.ws);
      if (bytes) {
        load_to_lds4_at(S + at + 4 * quad, &sws[buf][0][c0]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t b = (uint32_t)(4 * quad + e < nst ? 4 * quad + e : nst - 1);
          load_to_lds4_at(S + 4 * (at + (a.ws_div == 1 ? b : b / a.ws_div)), &sws[buf][e][c0]);
        }
      }
    }
  };
  // Stage st, of which every wave has loaded a share, has arrived (the youngest
  // loads are those of the stages behind it); at the end of the stage before.
  auto arrived = [&](int st) {
    if (BUFS > 2 && st + 1 < nst) wait_loads<(BUFS - 2) * (QX + QW)>();
    else wait_loads<0>();
    __syncthreads();
    if (ragged && st == nst - 1) {
      mask_tail(st);
      __syncthreads();
    }
  };

  // ---- LDS to registers -----------------------------------------------------
  // Pieces g4 and 4 + g4 of a line: any order of the features will do, if it is
  // the same for both operands.
  const int slot0 = 16 * (g4 ^ (i16 & 7));
  const int xline = 16 * NX * wr + i16, wline = 64 * wc + i16;
  auto operand = [&](const uint8_t* lines, int line, u4 (&v)[2]) {
    v[0] = *reinterpret_cast<const u4*>(lines + 128 * line + slot0);
    v[1] = *reinterpret_cast<const u4*>(lines + 128 * line + (slot0 ^ 64));
  };
  auto xscales = [&](int st, int x) { return sxs[(st >> 2) & 1][xline + 16 * x]; };   // of four stages
  // The scales of four stages parted in place (split_scale), a thread to a
  // channel, well before the first of them.
  auto part_scales = [&](int quad) {
    if (tid < TT || tid >= kLines) return;
    const int c = tid - TT, buf = quad & 1;
    const uint32_t first = sws[buf][0][c];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (HOW == kPowers) {
        swp[buf][e][c] = (uint8_t)(first >> (8 * e));
        continue;
      }
      const uint32_t w = sws[buf][e][c];
      const SplitScale sp = split_scale(bytes ? from_e8m0((first >> (8 * e)) & 0xffu) : __uint_as_float(w));
      sws[buf][e][c] = __float_as_uint(sp.rest);
      swp[buf][e][c] = (uint8_t)(__float_as_uint(sp.power) >> 23);
    }
  };
  // of a lane's four channels
  auto rests = [&](int st) {
    return *reinterpret_cast<const v4*>(&sws[(st >> 2) & 1][st & 3][64 * wc + 4 * i16]);
  };
  auto powers = [&](int st) {
    return *reinterpret_cast<const uint32_t*>(&swp[(st >> 2) & 1][st & 3][64 * wc + 4 * i16]);
  };

  v4 acc[NX][4];
#pragma unroll
  for (int x = 0; x < NX; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[x][y] = v4{0.f, 0.f, 0.f, 0.f};

  load_scales(0);
#pragma unroll
  for (int st = 0; st < BUFS - 1; ++st)
    if (st < nst) load(st);
  wait_loads<0>();
  arrived(0);
  part_scales(0);
  __syncthreads();
  if constexpr (HOW == kExact) {
    // The sums take their scale beside the products of the next line of
    // activations (the last one's beside the next stage's first); the barrier
    // stands before a stage's last line, behind it the weights of the next stage
    // are read and brought to bf16 as the last products leave them.
    b8 fw[4][4];
    u4 next[2], wnext[4];
    uint32_t nsx;
    v4 s = rests(0), last_s = {0.f, 0.f, 0.f, 0.f}, wait[4];
    uint32_t power = powers(0);
    auto read_x = [&](int st, int x) {
      operand(sX[st % BUFS], xline + 16 * x, next);
      nsx = xscales(st, x);
    };
    // half h of the weights of a stage (products 2 h and 2 h + 1)
    auto read_w = [&](int st, int h) {
#pragma unroll
      for (int y = 0; y < 4; ++y)
        wnext[y] = *reinterpret_cast<const u4*>(sW[st % BUFS] + 128 * (wline + 16 * y) + (slot0 ^ (64 * h)));
    };
    auto bring_w = [&](uint32_t codes, int k) {
#pragma unroll
      for (int y = 0; y < 4; ++y)
        fw[y][k] = to_bf16(wnext[y][2 * (k & 1)], wnext[y][2 * (k & 1) + 1],
                           __uint_as_float(((codes >> (8 * y)) & 0xffu) << 23));
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      read_w(0, h);
      bring_w(power, 2 * h);
      bring_w(power, 2 * h + 1);
    }
    read_x(0, 0);
#pragma unroll
    for (int y = 0; y < 4; ++y) wait[y] = v4{0.f, 0.f, 0.f, 0.f};
    for (int st = 0; st < nst; ++st) {
      if ((st & 3) == 0 && st + 4 < nst) load_scales(st / 4 + 1);
      if ((st & 3) == 1 && (st | 3) + 1 < nst) part_scales(st / 4 + 1);
      if (st + BUFS - 1 < nst) load(st + BUFS - 1);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const u4 v[2] = {next[0], next[1]};
        const float sx = from_e8m0((nsx >> (8 * (st & 3))) & 0xffu);
        if (x + 1 < NX) {
          read_x(st, x + 1);
        } else {
          // (behind the last stage these read what stands there, unused)
          __builtin_amdgcn_s_setprio(1);
          if (st + 1 < nst) arrived(st + 1);
          read_w(st + 1, 0);
          read_x(st + 1, 0);
          power = powers(st + 1);
        }
        v4 d[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const b8 fx = to_bf16(v[k >> 1][2 * (k & 1)], v[k >> 1][2 * (k & 1) + 1], sx);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            d[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx, fw[y][k], k ? d[y] : v4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          if (x + 1 == NX) {
            bring_w(power, k);
            if (k == 1) read_w(st + 1, 1);
          }
          constexpr int kLast = NX - 1;
          const int px = x ? x - 1 : kLast;
          const float ps = x ? s[k] : last_s[k];
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[px][k][r] = __builtin_fmaf(wait[k][r], ps, acc[px][k][r]);
          pin(acc[px][k]);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) wait[y] = d[y];
      }
      last_s = s;
      s = rests(st + 1);
    }
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[NX - 1][y][r] = __builtin_fmaf(wait[y][r], last_s[y], acc[NX - 1][y][r]);
  } else {
    // A product's sums take their scale two products later, beside the matrix
    // cores; the last two of a stage in the next one.  A stage's last line of
    // activations is read ahead, so the barrier stands before its products:
    // behind it the stage's buffers take the stage after the next, and the next
    // stage's first operands are read.
    auto eight = [](const u4 (&v)[2]) {
      return __builtin_bit_cast(i8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    i8 fw[4];
    u4 next[2];
    v4 s = rests(0);
    uint32_t power = powers(0), next_power = 0;   // four e8m0 codes
    float last_s[2] = {0.f, 0.f};
    v4 wait[2] = {v4{0.f, 0.f, 0.f, 0.f}, v4{0.f, 0.f, 0.f, 0.f}};
    uint32_t nsx;
    auto read_w = [&](int st, int y) {
      u4 v[2];
      operand(sW[st % BUFS], wline + 16 * y, v);
      fw[y] = eight(v);
    };
    auto read_x = [&](int st, int x) {
      operand(sX[st % BUFS], xline + 16 * x, next);
      nsx = xscales(st, x);
    };
#pragma unroll
    for (int y = 0; y < 4; ++y) read_w(0, y);
    read_x(0, 0);
    for (int st = 0; st < nst; ++st) {
      if ((st & 3) == 0 && st + 4 < nst) load_scales(st / 4 + 1);
      if ((st & 3) == 1 && (st | 3) + 1 < nst) part_scales(st / 4 + 1);
      if (st + BUFS - 1 < nst) load(st + BUFS - 1);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const i8 fx = eight(next);
        const int sx = (int)(nsx >> (8 * (st & 3)));
        if (x + 1 < NX) {
          read_x(st, x + 1);
        } else {
          // (behind the last stage these read what stands there, unused)
          __builtin_amdgcn_s_setprio(1);
          if (st + 1 < nst) arrived(st + 1);
          read_x(st + 1, 0);
        }
        if (x == NX / 2) next_power = powers(st + 1);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          constexpr v4 kZero = {0.f, 0.f, 0.f, 0.f};
          v4 d = HOW == kPowers ? acc[x][y] : kZero;
          if (y == 0) d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[0], d, 0, 0, 0, sx, 0, (int)power);
          else if (y == 1) d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[1], d, 0, 0, 0, sx, 1, (int)power);
          else if (y == 2) d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[2], d, 0, 0, 0, sx, 2, (int)power);
          else d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[3], d, 0, 0, 0, sx, 3, (int)power);
          if (x + 1 == NX) read_w(st + 1, y);
          if (HOW == kPowers) {
            acc[x][y] = d;
            pin(acc[x][y]);
            __builtin_amdgcn_sched_barrier(0);
            continue;
          }
          // (the product before the one before)
          const int px = y >= 2 ? x : (x + NX - 1) % NX, py = (y + 2) & 3;
          const float ps = x == 0 && y < 2 ? last_s[y] : s[py];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            acc[px][py][r] = __builtin_fmaf(wait[y & 1][r], ps, acc[px][py][r]);
          pin(acc[px][py]);
          wait[y & 1] = d;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      last_s[0] = s[2];
      last_s[1] = s[3];
      s = rests(st + 1);
      power = next_power;
    }
#pragma unroll
    for (int y = 0; y < (HOW == kPowers ? 0 : 2); ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        acc[NX - 1][2 + y][r] = __builtin_fmaf(wait[y][r], last_s[y], acc[NX - 1][2 + y][r]);
  }

  // lane l holds tokens 4 g4 + r (lines) of channel i16 of each 16 x 16 block
  auto store = [&](auto* Y) {
    const int64_t j0 = J0 + 64 * wc + 4 * i16, t0 = T0 + 16 * NX * wr + 8 * g4;
#pragma unroll
    for (int p = 0; p < NX / 2; ++p) {
      const int64_t t = t0 + 32 * p;
      if (a.tokens_first) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) v[y] = acc[2 * p + (e >> 2)][y][e & 3];
          if (t + e < a.T) store_run(Y + (t + e) * a.ldy + j0, v, a.n - j0);
        }
      } else {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = acc[2 * p + (e >> 2)][y][e & 3];
          if (j0 + y < a.n) store_run(Y + (j0 + y) * a.ldy + t, v, a.T - t);
        }
      }
    }
  };
  if (a.ytype == 0) store(static_cast<float*>(a.Y));
  else if (a.ytype == 1) store(static_cast<_Float16*>(a.Y));
  else store(static_cast<__bf16*>(a.Y));
}

template <int TT, int TC, int WR, int WC, int BUFS, int HOW>
hipError_t launch_tiles(const Product8Args& a, hipStream_t s) {
  const int64_t tiles_n = (a.n + TC - 1) / TC, tiles = tiles_n * ((a.T + TT - 1) / TT);
  // (a grid holds 2^32 - 1 threads: a result beyond that is one of over 500 GB)
  if (tiles * (64 * WR * WC) >> 32) return hipErrorInvalidValue;
  product8_kernel<TT, TC, WR, WC, BUFS, HOW>
      <<<dim3((unsigned)tiles), dim3(64 * WR * WC), 0, s>>>(a, tiles_n);
  return hipGetLastError();
}

// A CU holds one workgroup of the larger tiles or two of 128 x 128, so the chip
// takes them in rounds of 256 or 512 tiles.
// kExact: 256 x 128 while their rounds are full to 15/16 (us for 256 x 128 / 128
// x 128 at m = 4096, 4096 channels: 2048 tokens, one round, 70.9 / 73.0, 4096
// 136.7 / 140.0, 8192 270 / 279; 1024, half a round, 62.7 / 49.4; 5000, 2.5
// rounds, 189 / 177; 14336 channels, 600 tokens, 1.3 rounds, 122 / 106, 2048, 3.5
// rounds, 257 / 250).
// 16-bit results: a round of 256 x 256 does twice the work of one of 128 x 128
// in 1.6 times the time (us for 256 x 256 / 128 x 128: 4096 channels, 2048 tokens, half
// a round, 61 / 49; 4096 74 / 95; 5000, 1.25 rounds, 125 / 118; 8192 142 / 174;
// 14336 channels, 600 tokens 61 / 73, 2048 134 / 162; the rule misses up to 8%
// where a last round is half full: 6144 125 / 137).
template <int HOW>
hipError_t launch_how(const Product8Args& a, hipStream_t s) {
  auto tiles = [&](int64_t tt, int64_t tc) { return (a.n + tc - 1) / tc * ((a.T + tt - 1) / tt); };
  if constexpr (HOW == kExact) {
    const int64_t big = tiles(256, 128);
    return 16 * big >= 15 * ((big + 255) / 256 * 256) ? launch_tiles<256, 128, 4, 2, 3, HOW>(a, s)
                                                      : launch_tiles<128, 128, 2, 2, 2, HOW>(a, s);
  } else {
    return 100 * ((tiles(256, 256) + 255) / 256) <= 62 * ((tiles(128, 128) + 511) / 512)
               ? launch_tiles<256, 256, 2, 4, 2, HOW>(a, s)
               : launch_tiles<128, 128, 2, 2, 2, HOW>(a, s);
  }
}

// The kernel for few tokens takes up to 32 of them, and more while blocks of 32
// channels x 32 tokens are few (its workgroups take 16 to 64 channels of them):
// 28 us for 1000 blocks at m = 4096, where a round of 128-wide tiles takes 35 us
// however full, 48 us with float32 results, and 13 or 20 us more expand the codes
// of 4096 and 14336 channels.  us for few tokens' kernel / tiles, 4096 channels:
//                   e4m3, 16 bits   float32       codes, 16 bits  float32
//   m = 1024,  256  12.5 / 11.8     12.9 / 15.9   13.8 / 18.5     14.2 / 21.8
//              512  23.5 / 12.7     24.0 / 16.9   25.6 / 18.6     26.2 / 22.8
//   m = 4096,  256  28.2 / 34.7     27.9 / 47.0   28.5 / 48.5     28.6 / 60.0
//              512  52.8 / 35.5     53.1 / 47.9   55.0 / 47.9     55.4 / 60.0
//   m = 14336, 256  65.4 / 108      64.4 / 150    73.2 / 132      73.4 / 171
//              512  127 / 109       127 / 153     144 / 132       144 / 172
// The limits are those of m = 4096.  Tiles' times grow faster with m, so near the
// limits the slower kernel is taken elsewhere: up to 1.3 times the other's time at
// m = 1024 (14336 channels, 128 tokens, float32, 21.9 / 16.7), 1.2 at 14336.
bool few(int64_t n, int64_t T, bool codes, bool f32) {
  const int64_t most = codes ? (f32 ? 2304 : 1792) : (f32 ? 1792 : 1280);
  return T <= 32 || (n + 31) / 32 * ((T + 31) / 32) <= most;
}
int64_t expanded_row(int64_t m) { return (m + 127) / 128 * 128; }

}  // namespace

size_t product8_workspace_bytes(int64_t n, int64_t m, int64_t T) {
  return few(n, T, true, false) ? 0 : (size_t)n * (size_t)expanded_row(m);
}

hipError_t launch_product8(const Product8Args& a, int bits, void* workspace, hipStream_t stream) {
  // (tiles address their rows with 32 bits)
  if (few(a.n, a.T, bits != 0, a.ytype == 0) || a.ldx > (1 << 23) || (bits == 0 && a.ldw > (1 << 23)))
    return launch_product_few8(a, bits, stream);
  Product8Args b = a;
  if (bits) {
    uint8_t* const W8 = static_cast<uint8_t*>(workspace);
    b.W8 = W8;
    b.ldw = expanded_row(a.m);
    // about eight rows to a workgroup where that leaves enough of them
    const int64_t across = (b.ldw / 32 + 255) / 256, down = a.n * across >= 16384 ? (a.n + 7) / 8 : a.n;
    const dim3 grid((unsigned)across, (unsigned)(down < 65535 ? down : 65535)), block(256);
    switch (bits) {
      case 1: expand_codes_kernel<1><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      case 2: expand_codes_kernel<2><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      case 3: expand_codes_kernel<3><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      case 4: expand_codes_kernel<4><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      default: return hipErrorInvalidValue;
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (b.ytype == 0) return launch_how<kExact>(b, stream);
  return b.ws_e8m0 ? launch_how<kPowers>(b, stream) : launch_how<kScaled>(b, stream);
}

}  // namespace ojbkq
