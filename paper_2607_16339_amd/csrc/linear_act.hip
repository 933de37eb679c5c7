// The bf16 projection with its epilogue: out = act(a W^T + bias) + residual, or
// silu(gate) up of two products (kGlu: weight rows n and Nw/2 + n, which a wavefront
// holds as slabs of 16 gate rows and the same 16 up rows). Calls of few rows that are
// one stream of weights go to the first layer's kernel, which has the same epilogue.
//
// Each output is one chain of 16x16x32 bf16 MFMAs over K in order, the same bits
// whatever the tile.
//
// K-steps of 64 elements (128 bytes of a row) come by direct copies into an LDS
// ring, [rows][128 B] with the 16-byte chunk c of row r at c ^ ((r / 2) mod 8):
// the 16 rows of an operand read touch every bank once. Rows past M and columns
// past the weight's rows fetch the last one and are not stored.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "activation.h"
#include "device.h"
#include "launch.h"

namespace lacache {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

struct LinCall {
  const uint16_t* a;
  const uint16_t* w;
  uint16_t* out;
  ActArgs act;
  int64_t M, K;
  int64_t Nw;  // weight rows
  int R, C;    // row and column tiles
};

// Copies of the rows of a K-step: copy u of wavefront v of W fills rows 8 (v + W u) ..
// of the tile's activation or weight rows, lane l row l / 8, chunk (l mod 8) ^ swizzle.
struct CopyPlan {
  int crow;
  uint32_t chunk;  // of even groups of 8 rows; odd ones flip bit 6
};
__device__ __forceinline__ CopyPlan copy_plan(int lane) {
  return {lane >> 3, static_cast<uint32_t>(((lane & 7) ^ (lane >> 4)) << 4)};
}
// Byte offset from a (row 0 of the tile) of the lane's chunk of rows 8 g ..; last: the last row that exists.
__device__ __forceinline__ uint32_t row_off(const CopyPlan& p, int g, uint32_t K2, int64_t last) {
  const int row = 8 * g + p.crow;
  return static_cast<uint32_t>(row < last ? row : last) * K2 + (p.chunk ^ ((g & 1) << 6));
}
// The weight row of row 8 g + r of a tile of BN rows from column tile ct (kGlu: bands of
// 16 NT rows, NT/2 slabs of gate rows and then the up rows of the same columns).
template <bool kGlu, int BN, int NT>
__device__ __forceinline__ int64_t weight_row(int64_t Nw, int ct, int row) {
  if (!kGlu) {
    const int64_t n = static_cast<int64_t>(ct) * BN + row;
    return n < Nw ? n : Nw - 1;
  }
  const int slab = row >> 4, j = slab % NT;
  const int64_t n = static_cast<int64_t>(ct) * (BN / 2) + ((slab / NT) * (NT / 2) + j % (NT / 2)) * 16 + (row & 15);
  return (n < Nw / 2 ? n : Nw / 2 - 1) + (j < NT / 2 ? 0 : Nw / 2);
}

// The sums acc[MT][NT] of a wavefront (rows row0 .., band of 16 NT weight rows wn of
// column tile ct) to the output, through LDS of the wavefront's own, kSlabs slabs of
// 16 rows at a time, so that the residual is read and the output written 16 bytes a
// lane, a row's columns together. A lane keeps its 8 columns; the residual's loads
// of a part are all in flight before its sums go through LDS, and the activation is
// chosen once per 8 values (chosen per value, with a load between, a 256 x 256 tile's
// epilogue took 18 us).
template <bool kGlu, int BN, int MT, int NT, int kSlabs>
struct Epilogue {
  static constexpr int kCols = 16 * NT, kPitch = kCols + 4;  // fp32; 4: rows apart by 16 bytes of the banks
  static constexpr int kRows = 16 * kSlabs, kBytes = kRows * kPitch * 4;
  static constexpr int kOut = kGlu ? kCols / 2 : kCols, kVec = kOut / 8, kIters = (kRows * kVec + 63) / 64;
  static_assert(MT % kSlabs == 0 && kOut % 8 == 0 && 64 % kVec == 0, "epilogue");

  static __device__ __forceinline__ void unpack(const uint16_t* p, float (&v)[8]) {
    const uint4 w4 = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
    for (int x = 0; x < 4; ++x) v[2 * x] = bf16lo(w[x]), v[2 * x + 1] = bf16hi(w[x]);
  }
  static __device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const v4f a = *reinterpret_cast<const v4f*>(p), b = *reinterpret_cast<const v4f*>(p + 4);
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = a[x], v[4 + x] = b[x];
  }

  static __device__ __forceinline__ void store(const LinCall& c, const v4f (&acc)[MT][NT], float* tile, int64_t row0,
                                               int ct, int wn, int lane) {
    const int q = lane >> 4, lr = lane & 15;
    const int64_t no = kGlu ? c.Nw / 2 : c.Nw;
    const int rl = lane / kVec, c8 = 8 * (lane % kVec);  // this lane's first row and its columns
    const int64_t col = static_cast<int64_t>(ct) * (kGlu ? BN / 2 : BN) + kOut * wn + c8;
    const bool bias = c.act.bias != nullptr && col < no;
    float b1[8] = {}, b2[8] = {};
    if (bias) {
      unpack(c.act.bias + col, b1);
      if (kGlu) unpack(c.act.bias + no + col, b2);
    }
#pragma unroll
    for (int part = 0; part < MT / kSlabs; ++part) {
      uint4 res[kIters];
      bool live[kIters];
#pragma unroll
      for (int it = 0; it < kIters; ++it) {
        const int rr = rl + it * (64 / kVec);
        const int64_t row = row0 + part * kRows + rr;
        live[it] = rr < kRows && row < c.M && col < no;
        res[it] = make_uint4(0u, 0u, 0u, 0u);
        if (c.act.residual != nullptr && live[it])
          res[it] = *reinterpret_cast<const uint4*>(c.act.residual + row * no + col);
      }
#pragma unroll
      for (int i = 0; i < kSlabs; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          *reinterpret_cast<v4f*>(tile + (16 * i + lr) * kPitch + 16 * j + 4 * q) = acc[part * kSlabs + i][j];
      wait_lds();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int it = 0; it < kIters; ++it) {
        if (!live[it]) continue;
        const int rr = rl + it * (64 / kVec);
        const float* src = tile + rr * kPitch + c8;
        float v[8];
        load8(src, v);
        if (bias) {
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] += b1[x];
        }
        if (kGlu) {
          float u[8];
          load8(src + kOut, u);
          if (bias) {
#pragma unroll
            for (int x = 0; x < 8; ++x) u[x] += b2[x];
          }
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = silu(v[x]) * u[x];
        } else {
          activate(c.act.act, v);
        }
        if (c.act.residual != nullptr) {
          const uint32_t rw[4] = {res[it].x, res[it].y, res[it].z, res[it].w};
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] += x & 1 ? bf16hi(rw[x >> 1]) : bf16lo(rw[x >> 1]);
        }
        uint32_t ow[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          ow[x] = cvt_pk_bf16(v[2 * x], v[2 * x + 1]);
          if (__builtin_isunordered(v[2 * x], v[2 * x + 1])) ow[x] = bf16x2_quiet(ow[x]);
        }
        *reinterpret_cast<uint4*>(c.out + (row0 + part * kRows + rr) * no + col) = make_uint4(ow[0], ow[1], ow[2], ow[3]);
      }
      wait_lds();
      asm volatile("" ::: "memory");
    }
  }
};

// WR x WC wavefronts, each MT x NT slabs of a BM x BN tile, a ring of S steps.
template <bool kGlu, int BM, int BN, int WR, int WC, int S>
__global__ __launch_bounds__(64 * WR * WC) void linear_act_tile_kernel(LinCall c) {
  constexpr int W = WR * WC, MT = BM / WR / 16, NT = BN / WC / 16, kStep = (BM + BN) * 128;
  constexpr int PA = BM / 8 / W, PB = BN / 8 / W, P = PA + PB;
  using Epi = Epilogue<kGlu, BN, MT, NT, 1>;
  static_assert(BM % (8 * W) == 0 && BN % (8 * W) == 0 && S >= 3 && W * Epi::kBytes <= S * kStep && S * kStep <= 163840,
                "tile shape");
  __shared__ __align__(16) uint8_t ring[S * kStep];
  const int t = threadIdx.x, lane = t & 63, wave = wave_uniform(t >> 6);
  const int q = lane >> 4, lr = lane & 15, wm = wave / WC, wn = wave % WC;
  const int KS = static_cast<int>(c.K / 64);
  const uint32_t K2 = static_cast<uint32_t>(c.K) * 2u;
  int rt, ct;
  xcd_grouped_tile(static_cast<int>(blockIdx.x), c.R, c.C, rt, ct);
  const int64_t m0 = static_cast<int64_t>(rt) * BM;
  const CopyPlan cp = copy_plan(lane);
  uint32_t ao[PA], bo[PB];
#pragma unroll
  for (int u = 0; u < PA; ++u) ao[u] = row_off(cp, wave + W * u, K2, c.M - 1 - m0);
#pragma unroll
  for (int u = 0; u < PB; ++u) {
    const int g = wave + W * u;
    bo[u] = static_cast<uint32_t>(weight_row<kGlu, BN, NT>(c.Nw, ct, 8 * g + cp.crow) -
                                  (kGlu ? 0 : static_cast<int64_t>(ct) * BN)) * K2 + (cp.chunk ^ ((g & 1) << 6));
  }
  const uint8_t* ab = reinterpret_cast<const uint8_t*>(c.a + m0 * c.K);
  const uint8_t* wb = reinterpret_cast<const uint8_t*>(kGlu ? c.w : c.w + static_cast<int64_t>(ct) * BN * c.K);
  const uint32_t lds = lds_u32(ring);
  auto issue = [&](int ks, int slot) {
    // (past the end the last step again, never read)
    const int64_t kb = static_cast<int64_t>(ks < KS ? ks : KS - 1) * 128;
    const uint32_t dst = lds + slot * kStep;
#pragma unroll
    for (int u = 0; u < PA; ++u) dma16s(ab + kb, ao[u], wave_uniform(static_cast<int>(dst + (wave + W * u) * 1024)));
#pragma unroll
    for (int u = 0; u < PB; ++u)
      dma16s(wb + kb, bo[u], wave_uniform(static_cast<int>(dst + BM * 128 + (wave + W * u) * 1024)));
  };
  const int frag[2] = {lr * 128 + ((q ^ (lr >> 1)) << 4), lr * 128 + (((4 + q) ^ (lr >> 1)) << 4)};
  bf8 af[2][MT], bf[2][NT];
  auto read = [&](int slot, int h) {
    const uint8_t* pa = ring + slot * kStep + MT * wm * 2048 + frag[h];
    const uint8_t* pb = ring + slot * kStep + BM * 128 + NT * wn * 2048 + frag[h];
#pragma unroll
    for (int i = 0; i < MT; ++i) af[h][i] = *reinterpret_cast<const bf8*>(pa + i * 2048);
#pragma unroll
    for (int j = 0; j < NT; ++j) bf[h][j] = *reinterpret_cast<const bf8*>(pb + j * 2048);
  };
  v4f acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](int h) {
    // weight rows first: a lane's four results are four consecutive columns of one row
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MT; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[h][j], af[h][i], acc[i][j], 0, 0, 0);
  };

#pragma unroll
  for (int s = 0; s < S - 1; ++s) issue(s, s);
  wait_vm<(S - 2) * P>();
  bar();
  read(0, 0);
  int cur = 0;
  for (int ks = 0; ks < KS; ++ks) {
    const int nxt = cur + 1 == S ? 0 : cur + 1;
    __builtin_amdgcn_sched_barrier(0);
    read(cur, 1);
    multiply(0);
    __builtin_amdgcn_sched_barrier(0);
    wait_vm<(S - 3) * P>();  // this wavefront's copies of the next step have landed ...
    bar();                   // ... and everyone's; step ks - 1 has been read
    issue(ks + S - 1, cur == 0 ? S - 1 : cur - 1);
    read(nxt, 0);
    multiply(1);
    cur = nxt;
  }
  wait_vm<0>();
  bar();
  Epi::store(c, acc, reinterpret_cast<float*>(ring + wave * Epi::kBytes), m0 + 16 * MT * wm, ct, wn, lane);
}

// 256 x 256 or 128 x 256 tiles, 8 wavefronts of 64 x 128 or 64 x 64, walked by at most
// one workgroup per CU. Two wavefronts share a SIMD and alternate: one reads its operands and issues
// copies while the other multiplies, a barrier between the phases. Wavefronts 0-3
// copy the activation rows (ring of DA steps), 4-7 the weight rows (of DB).
template <bool kGlu, int BM, int BN, int DA, int DB>
__global__ __launch_bounds__(512) void linear_act_pairs_kernel(LinCall c) {
  constexpr int WC = 8 / (BM / 64), MT = 4, NT = BN / WC / 16, kA = BM * 128, kB = BN * 128;
  constexpr int PA = BM / 32, PB = BN / 32, P = PA > PB ? PA : PB;
  using Epi = Epilogue<kGlu, BN, MT, NT, 2>;
  static_assert(DA * kA + DB * kB <= 163840 && 8 * Epi::kBytes <= DA * kA + DB * kB, "tile shape");
  __shared__ __align__(16) uint8_t ring[DA * kA + DB * kB];
  uint8_t* const sB = ring + DA * kA;
  const int t = threadIdx.x, lane = t & 63, wave = wave_uniform(t >> 6);
  const int q = lane >> 4, lr = lane & 15, wm = wave / WC, wn = wave % WC;
  const bool late = wave >= 4;  // copies weights, half a phase behind the others
  const int KS = static_cast<int>(c.K / 64);
  const uint32_t K2 = static_cast<uint32_t>(c.K) * 2u;
  const CopyPlan cp = copy_plan(lane);
  const int frag[2] = {lr * 128 + ((q ^ (lr >> 1)) << 4), lr * 128 + (((4 + q) ^ (lr >> 1)) << 4)};

  for (int item = blockIdx.x; item < c.R * c.C; item += gridDim.x) {
    int rt, ct;
    xcd_grouped_tile(item, c.R, c.C, rt, ct);
    const int64_t m0 = static_cast<int64_t>(rt) * BM;
    const uint8_t* base = late ? reinterpret_cast<const uint8_t*>(kGlu ? c.w : c.w + static_cast<int64_t>(ct) * BN * c.K)
                               : reinterpret_cast<const uint8_t*>(c.a + m0 * c.K);
    uint32_t off[P];
#pragma unroll
    for (int u = 0; u < P; ++u) {
      const int g = (wave & 3) + 4 * u;  // (up to PA or PB of them are used)
      const uint32_t x = cp.chunk ^ ((g & 1) << 6);
      off[u] = late ? static_cast<uint32_t>(weight_row<kGlu, BN, NT>(c.Nw, ct, 8 * g + cp.crow) -
                                            (kGlu ? 0 : static_cast<int64_t>(ct) * BN)) * K2 + x
                    : row_off(cp, g, K2, c.M - 1 - m0);
    }
    auto issue = [&](int ks, uint8_t* dst) {
      const uint8_t* g = base + static_cast<int64_t>(ks < KS ? ks : KS - 1) * 128;
      const int l = static_cast<int>(lds_u32(dst)) + (wave & 3) * 1024;
#pragma unroll
      for (int u = 0; u < P; ++u)
        if (u < (late ? PB : PA)) dma16s(g, off[u], wave_uniform(l + u * 4096));
    };
    auto landed = [&]() {
      if (late)
        wait_vm<(DB - 2) * PB>();
      else
        wait_vm<(DA - 2) * PA>();
    };
    v4f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < (DA > DB ? DA : DB) - 1; ++s) {
      if (late && s < DB - 1) issue(s, sB + s * kB);
      if (!late && s < DA - 1) issue(s, ring + s * kA);
    }
    landed();
    bar();  // step 0 is in LDS
    if (late) bar();
    int ca = 0, cb = 0;
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* pa = ring + ca * kA + frag[h] + MT * wm * 2048;
        const uint8_t* pb = sB + cb * kB + frag[h] + NT * wn * 2048;
        bf8 af[MT], bf[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) af[i] = *reinterpret_cast<const bf8*>(pa + i * 2048);
#pragma unroll
        for (int j = 0; j < NT; ++j) bf[j] = *reinterpret_cast<const bf8*>(pb + j * 2048);
        if (h == 0) {  // into the stages of step ks - 1, which every wavefront has read
          if (late)
            issue(ks + DB - 1, sB + (cb == 0 ? DB - 1 : cb - 1) * kB);
          else
            issue(ks + DA - 1, ring + (ca == 0 ? DA - 1 : ca - 1) * kA);
        }
        if (h == 1 && late) landed();
        wait_lds();
        bar();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < MT; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[j], af[i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if (h == 1 && !late) landed();
        bar();
      }
      ca = ca + 1 == DA ? 0 : ca + 1;
      cb = cb + 1 == DB ? 0 : cb + 1;
    }
    if (!late) bar();
    wait_vm<0>();  // the trailing repeat copies
    bar();         // every wavefront is done with the ring
    Epi::store(c, acc, reinterpret_cast<float*>(ring + wave * Epi::kBytes), m0 + 16 * MT * wm, ct, wn, lane);
    bar();  // the next item's copies overwrite the ring
  }
}

// The tiles, and a cost that ranks them: rounds (of `fit` workgroups per CU) of a
// start and K/64 steps, a step's part in the traffic of the whole chip, and a part
// for every workgroup that shares a CU. (The constants are fitted to the order of the
// times, not to the times: M = 32, N = K = 4096 costs 7.6 on the streaming kernel and 9.9
// on 32 x 64 tiles.) Up to 128 rows the weight-streaming kernel of
// the first layer (K over four wavefronts, 16 or 48 weight rows) competes. Weighed on
// 376 sizes with weights from HBM, M = 1..8192, N x K = 128 x 4096 to 24576 x 4096, K
// from 128 to 16384, all kernels in turn in one process: the choice is on average 0.2 %
// slower than the best, 7 % at most (on 76 more, of other N and K, 0.9 % and 12 %);
// without one of the two 128 x 256 tiles 1 % and 27 %, without 64 x 64 or 64 x 128 more.
// Times in us, weights from HBM, on the streaming kernel, 32 x 64, 64 x 64, 64 x 128, 128 x 128, 128 x 256 (16
// wavefronts, 8 in pairs) and 256 x 256:
//   N = K = 4096       M =   32  11, 17, 19, 27, 30, 67, 58, 80
//                           128  24, 17, 21, 29, 38, 75, 59, 83
//                           512   -, 49, 35, 30, 39, 71, 58, 84
//                          1024   -, 91, 66, 57, 39, 70, 58, 85
//                          2048   -, 157, 120, 108, 75, 74, 66, 91
//                          8192   -, 567, 396, 360, 275, 241, 252, 210
//   N = 12288, K = 4096      48  36, 30, 25, 34, 35, 71, 61, 82
//   N = 8192, K = 256      3000   -, 63, 44, 47, 32, 27, 31, 33
// More wavefronts of less work each were better for the small tiles, a step of a lone
// workgroup being a chain of barrier, LDS reads and products (128 x 128 on 4, 8 and 16
// wavefronts, M = 512: 43, 36, 33); 256 x 256 on 4 wavefronts of 128 x 128 took 288 us
// where these take 218, on 16 of 64 x 64 the same, with 32x32x16 MFMAs 231.
struct Shape {
  int bm, bn, waves, fit;
  double start, step, chip, shared;
};
constexpr Shape kShapes[7] = {{32, 64, 4, 2, 0.739, 0.080, 0.078, 0.043},  {64, 64, 8, 2, 1.117, 0.040, 0.114, 0.103},
                              {64, 128, 8, 1, 1.517, 0.174, 0.203, 0.0},   {128, 128, 16, 1, 1.499, 0.342, 0.235, 0.0},
                              {128, 256, 16, 1, 0.832, 0.868, 0.302, 0.0},
                              {128, 256, 8, 1, 4.854, 0.638, 0.337, 0.0},  // in pairs, a workgroup per CU, as
                              {256, 256, 8, 1, 5.993, 1.301, 0.297, 0.0}};
constexpr int kFirstPairs = 5;
constexpr int kStream = -1;

int best_shape(int64_t M, int64_t Nw, int64_t K) {
  const double cus = static_cast<double>(device_cu_count()), ks = static_cast<double>(K) / 64.0;
  int pick = kStream;
  double best = HUGE_VAL;
  if (linear_streams_rows(M)) {
    int tile[2];
    linear_tile(M, Nw, K, tile);
    const double items = static_cast<double>(Nw / tile[1] * ((M + 63) / 64));
    const double kb = static_cast<double>(2 * std::min<int64_t>(4, (M + 15) / 16) + tile[1] / 8);  // of a wavefront's step
    best = 2.704 + std::ceil(items / cus) * ks / 4 * (0.047 + 0.013 * kb) + 0.03 * ks * items * kb / (4 * cus);
  }
  for (int t = 0; t < 7; ++t) {
    const Shape& s = kShapes[t];
    const double items = static_cast<double>(((M + s.bm - 1) / s.bm) * ((Nw + s.bn - 1) / s.bn));
    const double per_cu = std::ceil(items / cus);
    const double cost = std::ceil(per_cu / s.fit) * (s.start + s.step * ks) + s.chip * ks * items / cus + s.shared * ks * per_cu;
    if (cost < best) pick = t, best = cost;
  }
  return pick;
}

template <bool kGlu>
hipError_t launch_shape(hipStream_t st, LinCall c, int shape) {
  c.R = static_cast<int>((c.M + kShapes[shape].bm - 1) / kShapes[shape].bm);
  c.C = static_cast<int>((c.Nw + kShapes[shape].bn - 1) / kShapes[shape].bn);
  const int64_t items = static_cast<int64_t>(c.R) * c.C, cus = device_cu_count();
  const dim3 all(static_cast<unsigned>(items)), round(static_cast<unsigned>(items < cus ? items : cus));
#define LT(I_, WR_, WC_, S_)                                                                                             \
  case I_:                                                                                                               \
    static_assert(WR_ * WC_ == kShapes[I_].waves, "wavefronts");                                                         \
    hipLaunchKernelGGL((linear_act_tile_kernel<kGlu, kShapes[I_].bm, kShapes[I_].bn, WR_, WC_, S_>), all,                \
                       dim3(64 * WR_ * WC_), 0, st, c);                                                                  \
    break
  switch (shape) {
    LT(0, 2, 2, 6);
    LT(1, 4, 2, 5);
    LT(2, 2, 4, 6);
    LT(3, 4, 4, 5);
    LT(4, 4, 4, 3);
    case 5: hipLaunchKernelGGL((linear_act_pairs_kernel<kGlu, 128, 256, 3, 3>), round, dim3(512), 0, st, c); break;
    default: hipLaunchKernelGGL((linear_act_pairs_kernel<kGlu, 256, 256, 2, 3>), round, dim3(512), 0, st, c);
  }
#undef LT
  return hipGetLastError();
}

}  // namespace

// The threads of a launch are counted in 32 bits.
bool linear_act_launches(int64_t M, int64_t N, int64_t K, int act) {
  const int64_t Nw = act == LACACHE_ACT_SWIGLU ? 2 * N : N;
  if (M * Nw < int64_t(1) << 32) return true;  // (a thread has at least 8 products)
  const int shape = best_shape(M, Nw, K);
  if (shape == kStream || shape >= kFirstPairs) return true;
  const Shape& s = kShapes[shape];
  return (M + s.bm - 1) / s.bm * ((Nw + s.bn - 1) / s.bn) * 64 * s.waves <= UINT32_MAX;
}

hipError_t launch_linear_act(hipStream_t st, const uint16_t* a, const uint16_t* w, const uint16_t* bias,
                             const uint16_t* residual, uint16_t* out, int64_t M, int64_t N, int64_t K, int act) {
  const bool glu = act == LACACHE_ACT_SWIGLU;
  const ActArgs aa{bias, residual, act};
  const LinCall c{a, w, out, aa, M, K, glu ? 2 * N : N, 0, 0};
  const int shape = best_shape(M, c.Nw, K);
  if (shape == kStream) return launch_linear_act_rows(st, a, w, aa, out, M, N, K);
  return glu ? launch_shape<true>(st, c, shape) : launch_shape<false>(st, c, shape);
}

void linear_act_tile(int64_t M, int64_t N, int64_t K, int act, int* tile, int* waves) {
  const int64_t Nw = act == LACACHE_ACT_SWIGLU ? 2 * N : N;
  const int shape = best_shape(M, Nw, K);
  int t[2];
  if (shape == kStream)
    linear_tile(M, Nw, K, t), *waves = kStreamWaves;
  else
    t[0] = kShapes[shape].bm, t[1] = kShapes[shape].bn, *waves = kShapes[shape].waves;
  tile[0] = t[0], tile[1] = t[1];
}

}  // namespace lacache
