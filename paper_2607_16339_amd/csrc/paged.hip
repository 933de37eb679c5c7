// Paged key/value cache: rotation and append of new tokens, and their
// attention over the cache.
#include <algorithm>

#include "device.h"
#include "launch.h"

namespace lacache {
namespace {

// Rotation and append. A group of D/8 lanes holds one head's vector of one token, 8
// dims per lane; in the rotated part lane c meets its partner c +- r/16 by shuffles.
// A workgroup takes a token's heads, kBatch vectors of each group in flight at a
// time (the cosines of the token's position are loaded once for all of them), or
// several tokens of few heads (kTokens: T of them in all).
template <int D, bool kFp8, bool kTokens>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppend a, int64_t T) {
  constexpr int L = D / 8, G = 256 / L, kBatch = 3;
  const int lane = threadIdx.x & 63, c = threadIdx.x % L, group = threadIdx.x / L;
  const int HT = a.heads + 2 * a.kv_heads;
  int64_t t = blockIdx.x;
  int first = blockIdx.y * G + group, step = gridDim.y * G;
  if (kTokens) {
    t = (t * G + group) >> a.groups_log2;
    step = 1 << a.groups_log2, first = group & (step - 1);
    if (t >= T) return;  // (whole groups, and only lanes of a group shuffle)
  }
  const uint4* src = reinterpret_cast<const uint4*>(a.qkv + t * HT * D) + c;
  uint4 x[kBatch];
  auto load = [&](int hs0) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int hs = hs0 + b * step;
      x[b] = make_uint4(0u, 0u, 0u, 0u);
      if (hs < HT) x[b] = src[static_cast<int64_t>(hs) * L];
    }
  };
  load(first);
  const int seq = a.seq_ids[t], pos = a.positions[t];
  if (seq < 0 || seq >= a.S || pos < 0 || pos >= a.max_pos) return;
  const int page = a.table[static_cast<int64_t>(seq) * a.max_pages + (pos >> a.page_log2)];
  if (page < 0 || page >= a.num_pages) return;
  const int slot = pos & ((1 << a.page_log2) - 1);
  const int hc = a.rope_dim >> 4;  // chunks of half the rotated part
  const bool rot = c < 2 * hc, low = c < hc;
  const int partner = rot ? (low ? lane + hc : lane - hc) : lane;
  float cs[8], sn[8];
  if (rot) {
    const int64_t o = static_cast<int64_t>(pos) * (8 * hc) + 8 * (low ? c : c - hc);
    const v4f* pc = reinterpret_cast<const v4f*>(a.cs + o);
    const v4f* ps = reinterpret_cast<const v4f*>(a.sn + o);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cs[e] = pc[e >> 2][e & 3];
      sn[e] = low ? -ps[e >> 2][e & 3] : ps[e >> 2][e & 3];  // (x - y and x + (-y) are the same bits)
    }
  }
  for (int hs0 = first; hs0 < HT; hs0 += kBatch * step) {
    if (hs0 != first) load(hs0);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int hs = hs0 + b * step;
      const uint32_t xw[4] = {x[b].x, x[b].y, x[b].z, x[b].w};
      uint32_t pw[4];  // (every lane of the group shuffles)
#pragma unroll
      for (int e = 0; e < 4; ++e) pw[e] = static_cast<uint32_t>(__shfl(static_cast<int>(xw[e]), partner, 64));
      if (hs >= HT) continue;
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[2 * e] = bf16lo(xw[e]), y[2 * e + 1] = bf16hi(xw[e]);
      const bool turn = rot && hs < a.heads + a.kv_heads;
      if (turn) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float o = e & 1 ? bf16hi(pw[e >> 1]) : bf16lo(pw[e >> 1]);
          y[e] = y[e] * cs[e] + o * sn[e];
        }
      }
      const bool to_cache = hs >= a.heads, is_v = hs >= a.heads + a.kv_heads;
      const int h = is_v ? hs - a.heads - a.kv_heads : hs - a.heads;
      const int64_t row = ((static_cast<int64_t>(page) * a.kv_heads + h) << a.page_log2) + slot;
      if (kFp8 && to_cache) {
        // the largest magnitude by its bits, so that infinities and NaNs win
        uint32_t top = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[e]) & 0x7FFFFFFFu);
#pragma unroll
        for (int o = L / 2; o >= 1; o >>= 1)
          top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, 64)));
        const float s = __uint_as_float(top) / kE4M3Max;
        uint32_t lo = 0x7F7F7F7Fu, hi = 0x7F7F7F7Fu;  // a vector that is not finite reads as NaN
        if (top < 0x7F800000u) quant8(y, s, lo, hi);
        reinterpret_cast<uint2*>(is_v ? a.v_cache : a.k_cache)[row * L + c] = make_uint2(lo, hi);
        if (c == 0) (is_v ? a.v_scale : a.k_scale)[row] = s;
        continue;
      }
      const uint4 o = turn ? make_uint4(cvt_pk_bf16(y[0], y[1]), cvt_pk_bf16(y[2], y[3]), cvt_pk_bf16(y[4], y[5]),
                                        cvt_pk_bf16(y[6], y[7]))
                           : x[b];
      if (to_cache)
        reinterpret_cast<uint4*>(is_v ? a.v_cache : a.k_cache)[row * L + c] = o;
      else
        reinterpret_cast<uint4*>(a.q)[(t * a.heads + hs) * L + c] = o;
    }
  }
}

// ---------------------------------------------------------------------------
// Attention of the new tokens.
//
// The nq heads / kv_heads query rows of a KV head share its keys and values, so
// they are the columns of one product: S^T = K Q^T, O^T = V^T P^T with 16x16x32
// bf16 MFMAs, RT tiles of 16 rows. What a call of up to 64 rows per KV head cannot
// do without is one read of the sequences' keys and values, and every choice serves
// that stream (for more rows see paged_attention_rows_kernel):
//
// A wavefront works alone on a run of key tiles (of 32 or 64 keys, see PagedTile)
// through two LDS slots of its own, one of keys and one of values, each
// refilled by direct copies as soon as it has been read: the next keys fly
// during softmax and P V, the next values during the next scores, without a
// barrier. Eight wavefronts per CU, in one workgroup or two (paged_plan), keep 64 to
// 128 KB in flight.
//
// Work is cut on the device, where the lengths are: a sequence's tiles into
// ceil(nt / C) pieces, C (piece_tiles) from all lengths of the call; a piece's tiles
// are divided over the wavefronts, whose states meet in LDS. A sequence of one
// piece is finished there; those of others are joined by paged_join_kernel, in
// piece order. With sum nt <= 2 C Wq there are at most 2 Wq + S pieces, and fewer
// than 4 Wq in sequences of several (of more than C tiles, so n < 2 nt / C).
//
// Softmax in base 2 with the state (m, l, O) in fp32; P enters the second
// product as two bf16 terms (p = hi + lo, 2^-17 relative: one term would double
// the error of the rounded output, and the products are not what bounds the
// call). e4m3 keys and values become bf16 exactly; a key's scale multiplies its
// scores, a value's its P, both in fp32.
//
// Places that no row may see: keys behind the end or on no page get scores of
// -inf and value rows of zeros in LDS (0 times a NaN would be one); in the tiles
// where causal rows differ, values that are not finite send the tile through one
// product per number of keys that a row sees, with zeros for the values behind.
//
// Measured (32 heads over 8 KV heads, D = 128; a large copy moves 5.05 TB/s): 48
// sequences of 1..8191 keys, bf16, 155 us = 5.4 TB/s; 64 of 12000..16384, e4m3, 64
// heads, 364 us = 5.3 TB/s; one of 131072, e4m3, 58 us = 4.8 TB/s; one of 500, 8.6 us
// with the call's way through the host, the chain of loads length - page - keys -
// values being what its kernel waits for.
// ---------------------------------------------------------------------------
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef int i2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s4 lds_s4;
typedef __attribute__((address_space(3))) i2 lds_i2;

constexpr float kInf = __builtin_inff(), kSlack = 8.0f;

// Sum over lanes 0 .. l of a wavefront.
__device__ __forceinline__ int wave_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of rows 0 and 2 to the rows above
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
  return x;
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

__device__ __forceinline__ int seq_len(const PagedAttn& a, int s) {
  const int len = a.seq_lens[s];
  return len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
}

// Key tiles of all sequences (in every lane); first: those of sequence `lane`.
template <int kKeys>
__device__ __forceinline__ int total_tiles(const PagedAttn& a, int lane, int first) {
  int n = first;
  for (int s = 64 + lane; s < a.S; s += 64) n += ceil_div(seq_len(a, s), kKeys);
  return __builtin_amdgcn_readlane(wave_prefix(n), 63);
}

// The most tiles of a piece, for all sequences of a call. Wq pieces per KV head and
// row tile fill the chip once. Pieces of kLong tiles and more hide their start:
// twice Wq of them, for balance. Shorter ones: the least length, from kLeast, at
// which all pieces run at once, if one below kLong does that. A sequence of at most
// kWhole tiles stays whole: a second kernel costs more than its few steps.
// kWays: wavefronts that split a piece's keys. 1: they split its rows, every tile is a
// step of 2 us for each, and shorter pieces pay although a piece's state is 128 rows:
// with the least 8 and whole up to 12 tiles, against 2 and 4, 72 rows over 8 sequences of
// 1..899 keys (D = 64) take 39 us against 18.6, 224 rows of 300 keys 18.0 / 13.7, over 8
// sequences of 200..1024 27 / 24 (128 rows over 2 of 4096 24.5 / 26.5).
template <int kWays>
struct PieceRule {
  static constexpr int kLeast = kWays > 1 ? 8 : 2, kWhole = kWays > 1 ? 32 : 4, kLong = 64;
};
template <int kKeys, int kWays>
__device__ __forceinline__ int piece_tiles(const PagedAttn& a, int lane, int first) {
  using P = PieceRule<kWays>;
  if (a.wq <= 1) return 1 << 30;  // (enough heads: every sequence whole)
  const int tot = total_tiles<kKeys>(a, lane, first);
  const int two = ceil_div(tot, 2 * a.wq);
  if (two >= P::kLong) return two;
  if (a.wq <= a.S) return P::kLong;  // (as many sequences as fill the chip)
  int lo = max(P::kLeast, ceil_div(tot, a.wq)), hi = P::kLong;
  hi = min(hi, max(lo, ceil_div(tot, a.wq - a.S)));  // (enough: a piece more per sequence)
  if (a.S <= 64) {
    while (lo < hi) {  // (six rounds at most)
      const int c = (lo + hi) / 2;
      if (__builtin_amdgcn_readlane(wave_prefix(ceil_div(first, c)), 63) <= a.wq)
        hi = c;
      else
        lo = c + 1;
    }
  }
  return hi;
}

// Pieces of a sequence of nt tiles.
template <int kWays>
__device__ __forceinline__ int pieces(int nt, int most) {
  return nt <= PieceRule<kWays>::kWhole ? 1 : ceil_div(nt, most);
}

// A workgroup's piece: tiles p0 .. p1 - 1 of sequence s (of n pieces, the first of
// which is kept at `slot` where n > 1), KV head h, row tile rt.
struct Piece {
  int s, n, unit, slot, len, p0, p1, h, rt;
};
template <int kKeys, int kWays>
__device__ __forceinline__ bool find_piece(const PagedAttn& a, int lane, Piece& p) {
  // row tiles of one (piece, KV head) together on an XCD
  const int rt_n = a.row_tiles, per = 8 * rt_n;
  const int q8 = blockIdx.x / per, rem = blockIdx.x - q8 * per, pair = q8 * 8 + (rem & 7);
  p.rt = rem >> 3;
  p.h = pair % a.kv_heads;
  int unit = pair / a.kv_heads, slot = 0;
  if (a.whole) {
    if (unit >= a.S) return false;
    p.s = unit, p.n = 1, p.unit = 0, p.slot = 0;
    p.len = seq_len(a, unit), p.p0 = 0, p.p1 = ceil_div(p.len, kKeys);
    return true;
  }
  // (the lengths of the first 64 sequences are loaded once: a short call is a chain of loads)
  const int len0 = lane < a.S ? seq_len(a, lane) : 0;
  const int most = piece_tiles<kKeys, kWays>(a, lane, ceil_div(len0, kKeys));
  for (int b = 0; b < a.S; b += 64) {
    const int lenb = b == 0 ? len0 : (b + lane < a.S ? seq_len(a, b + lane) : 0);
    const int mine = b + lane < a.S ? pieces<kWays>(ceil_div(lenb, kKeys), most) : 0;
    const int upto = wave_prefix(mine), kept = wave_prefix(mine > 1 ? mine : 0);
    const uint64_t behind = __ballot(upto > unit);
    if (behind != 0) {
      const int at = __builtin_ctzll(behind);
      p.s = b + at;
      p.n = __builtin_amdgcn_readlane(mine, at);
      p.len = __builtin_amdgcn_readlane(lenb, at);
      p.unit = unit - (__builtin_amdgcn_readlane(upto, at) - p.n);
      p.slot = slot + __builtin_amdgcn_readlane(kept, at) - p.n;
      const int nt = ceil_div(p.len, kKeys);
      // (below 2^32: n <= 2 Wq <= 4 CUs as C >= nt / (2 Wq), and nt <= 2^17)
      p.p0 = static_cast<int>(static_cast<uint32_t>(p.unit) * static_cast<uint32_t>(nt) / p.n);
      p.p1 = static_cast<int>(static_cast<uint32_t>(p.unit + 1) * static_cast<uint32_t>(nt) / p.n);
      // what the join needs to know
      if (p.unit == 0 && p.h == 0 && p.rt == 0 && threadIdx.x == 0) a.cuts[p.s] = make_int2(p.n, p.slot);
      return true;
    }
    unit -= __builtin_amdgcn_readlane(upto, 63);
    slot += __builtin_amdgcn_readlane(kept, 63);
  }
  return false;  // (fewer pieces than the grid has room for)
}

// Keys of a tile, of rt tiles of 16 rows: 64, or 32 where 64 would not fit the LDS or the registers.
constexpr int tile_keys(int d, bool fp8, int rt) {
  return d * (fp8 ? 1 : 2) == 256 || (d == 128 && rt == 2) ? 32 : 64;
}
template <int D, bool kFp8, int RT>
struct PagedTile {
  static constexpr int RB = D * (kFp8 ? 1 : 2);       // bytes of a key
  static constexpr int kKeys = tile_keys(D, kFp8, RT);
  static constexpr int kBytes = kKeys * RB;           // of an LDS slot
  static constexpr int CPR = RB / 16;                 // 16-byte chunks of a key
  static constexpr int KPI = 1024 / RB;               // keys of a copy instruction
  static constexpr int UPS = 16 / KPI;                // copies of 16 keys
  static constexpr int kSub = kKeys / 16;
  static constexpr int kCopies = kBytes / 1024 + (kFp8 ? 1 : 0);  // of keys or values, with their scales
  static constexpr int kSlot = 2 * kBytes + (kFp8 ? 2 * 64 * 4 : 0);  // a wavefront's LDS
};
// A key's 16-byte chunk c lies at c ^ swizzle: keys are read 16 at a time, one
// chunk of each, values (transposed) in 8 or 16 keys by 32 or 16 bytes, and both
// then touch every bank once. (The swizzle of a sum of key numbers without common
// bits is the xor of theirs.)
template <int RB>
__device__ __forceinline__ int kswz(int key) {
  return RB == 256 ? key & 15 : (RB == 128 ? (key >> 1) & 7 : (key >> 2) & 3);
}
template <int RB, bool kFp8>
__device__ __forceinline__ int vswz(int key) {
  if (RB == 256) return 2 * (key & 7);
  if (RB == 128 && !kFp8) return 2 * ((key >> 1) & 3);
  if (RB == 128) return ((key >> 1) & 3) | ((key >> 2) & 4);
  return ((key >> 2) & 1) | ((key >> 3) & 2);
}

__device__ __forceinline__ bf8 cvt_fp8x8(uint32_t lo, uint32_t hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const b2 x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const b2 x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const b2 x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const b2 x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return bf8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}

__device__ __forceinline__ v4f mfma16(bf8 a, bf8 b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float finite_max(float m) { return m == -kInf ? 0.0f : m; }

// The output row (an index of [S x nq x heads]) of row rr of KV head h.
__device__ __forceinline__ int64_t out_row(const PagedAttn& a, int s, int h, int rr) {
  const int G = a.heads / a.kv_heads, t = rr / G;
  return (static_cast<int64_t>(s) * a.nq + t) * a.heads + h * G + (rr - t * G);
}

// (a row without any weight is 0 also where its O is no number: 0 times an infinite value)
__device__ __forceinline__ void store_out(const PagedAttn& a, int64_t row, int D, int c4, v4f o, float m, float l) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (l == 0.0f) o = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  *reinterpret_cast<uint2*>(a.o + row * D + 4 * c4) =
      make_uint2(cvt_pk_bf16(o[0] * inv, o[1] * inv), cvt_pk_bf16(o[2] * inv, o[3] * inv));
  if (a.lse != nullptr && c4 == 0) a.lse[row] = (m + __log2f(l)) * 0.69314718055994531f;
}

// Keeps the compiler from holding what is derived from v in registers across a loop.
template <typename V>
__device__ __forceinline__ V fresh(V v) {
  asm volatile("" : "+v"(v));
  return v;
}

// A wavefront's way to the pages of a sequence: lane x holds the page of keys
// 16 (sb + x) ..; -1: not to be read.
template <int D, bool kFp8>
struct PagedCopy {
  static constexpr int RB = D * (kFp8 ? 1 : 2), CPR = RB / 16, KPI = 1024 / RB, UPS = 16 / KPI;
  const int32_t* table;
  int sb, pages, len, h, lane;
  uint32_t koff, voff;

  __device__ __forceinline__ void init(const PagedAttn& a, const Piece& p, int lane_) {
    lane = lane_, len = p.len, h = p.h;
    table = a.table + static_cast<int64_t>(p.s) * a.max_pages;
    const int key = lane / CPR, ch = lane % CPR;
    koff = key * RB + ((ch ^ kswz<RB>(key)) << 4);
    voff = key * RB + ((ch ^ vswz<RB, kFp8>(key)) << 4);
  }
  __device__ __forceinline__ void load_pages(const PagedAttn& a, int first) {
    sb = first;
    const int key = (first + lane) * 16;
    const int page = table[(key < a.max_len ? key : a.max_len - 1) >> a.page_log2];
    pages = key < len && page < static_cast<int>(a.num_pages) ? page : -1;
    // (known to the compiler, which would else wait for every copy at each use)
    wait_vm<0>();
  }
  // Keys of 16 sub .. + 15 that exist (a prefix), by the pages from 16 sb_ on.
  __device__ __forceinline__ int count(int pages_, int sb_, int sub) const {
    const int left = len - 16 * sub;
    return __builtin_amdgcn_readlane(pages_, sub - sb_) < 0 ? 0 : (left > 16 ? 16 : (left < 0 ? 0 : left));
  }
  // Copies those 16 keys (or values) to lds; odd: the tile's second 16, fourth, ...
  __device__ __forceinline__ void copy16(const PagedAttn& a, bool values, int sub, bool odd, uint32_t lds) const {
    const int page = __builtin_amdgcn_readlane(pages, sub - sb);
    const int in = (sub * 16) & ((1 << a.page_log2) - 1);
    // (16 keys of no page: any that exist; they are not used)
    const int64_t row = page < 0 ? 0 : ((static_cast<int64_t>(page) * a.kv_heads + h) << a.page_log2) + in;
    // (the same in every lane, and the copies take it from scalar registers)
    const int64_t urow = static_cast<int64_t>(static_cast<uint32_t>(wave_uniform(static_cast<int>(row)))) |
                         (static_cast<int64_t>(wave_uniform(static_cast<int>(row >> 32))) << 32);
    const uint8_t* src = static_cast<const uint8_t*>(values ? a.v_cache : a.k_cache) + urow * RB;
    const uint32_t off = fresh(values ? voff : koff) ^
                         (odd ? static_cast<uint32_t>(values ? vswz<RB, kFp8>(16) : kswz<RB>(16)) << 4 : 0u);
#pragma unroll
    for (int u = 0; u < UPS; ++u) {
      const uint32_t x = static_cast<uint32_t>(values ? vswz<RB, kFp8>(KPI * u) : kswz<RB>(KPI * u)) << 4;
      dma16s(src + u * 1024, off ^ x, wave_uniform(static_cast<int>(lds + u * 1024)));
    }
  }
  // The scales of 64 keys from 16 sub on, a lane each; subs: how many 16s there are (of 2: twice).
  template <int kSubs>
  __device__ __forceinline__ void copy_scales(const PagedAttn& a, bool values, int sub, uint32_t lds) const {
    const int page = __shfl(pages, sub - sb + ((lane >> 4) & (kSubs - 1)), 64);
    const int in = (sub * 16 + (lane & (16 * kSubs - 1))) & ((1 << a.page_log2) - 1);
    const int64_t row = page < 0 ? lane & 15 : ((static_cast<int64_t>(page) * a.kv_heads + h) << a.page_log2) + in;
    dma4((values ? a.v_scale : a.k_scale) + row, wave_uniform(static_cast<int>(lds)));
  }
};

// A wavefront's RT tiles of 16 query rows, and what it does with a tile of keys in LDS.
template <int D, bool kFp8, int RT>
struct PagedRows {
  using T = PagedTile<D, kFp8, RT>;
  static constexpr int RB = T::RB, kKeys = T::kKeys, kSub = T::kSub, kSteps = D / 32, kDims = D / 16;
  bf8 qf[RT][kSteps];
  int limit[RT];  // keys that this lane's row sees
  int seen;       // keys that every row sees
  float m[RT], l[RT];
  v4f ot[RT][kDims];  // O~^T: dims 16 d + 4 g .. of row r
  int lane, g, r, k_base, v_base;

  // Rows row0 .. of KV head h; Q^T with the dims that the K operand's lanes read together.
  __device__ __forceinline__ void init(const PagedAttn& a, const Piece& p, int row0, int lane_) {
    lane = lane_, g = lane >> 4, r = lane & 15;
    const int G = a.heads / a.kv_heads, R = a.nq * G;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      const int rr = row0 + 16 * x + r;
      limit[x] = a.causal ? p.len - a.nq + rr / G + 1 : p.len;
      const uint16_t* src = a.q + out_row(a, p.s, p.h, rr < R ? rr : 0) * D;
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        const int dim = kFp8 ? 64 * (ks >> 1) + 16 * g + 8 * (ks & 1) : 32 * ks + 8 * g;
        qf[x][ks] = *reinterpret_cast<const bf8*>(src + dim);
      }
      m[x] = -kInf, l[x] = 0.0f;
#pragma unroll
      for (int d = 0; d < kDims; ++d) ot[x][d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
    seen = a.causal ? p.len - a.nq + 1 : p.len;
    // per-lane LDS offsets: K operand chunk 4 step + g of key r; V^T operand (transposing
    // reads) of keys 4 g .. + 3 and 16 + 4 g .. + 3, dims 16 d ..
    k_base = r * RB + ((g ^ kswz<RB>(r)) << 4);
    const int vkey = kFp8 ? ((r >> 1) < 4 ? 4 * g + (r >> 1) : 12 + 4 * g + (r >> 1)) : 4 * g + (r >> 2);
    v_base = vkey * RB + (vswz<RB, kFp8>(vkey) << 4) +
             (kFp8 ? 8 * (r & 1) : ((((r & 3) >> 1) << 4) | (8 * (r & 1))));
  }

  __device__ __forceinline__ bf8 value_operand(const uint8_t* Vt, int vb, int step, int d) const {
    if constexpr (kFp8) {
      const i2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2*)(Vt + 32 * step * RB + (vb ^ (d << 4))));
      return cvt_fp8x8(static_cast<uint32_t>(w[0]), static_cast<uint32_t>(w[1]));
    } else {
      const uint8_t* p = Vt + 32 * step * RB + (vb ^ (d << 5));
      const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p));
      const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + 16 * RB));
      return __builtin_bit_cast(bf8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }

  // S^T = K Q^T in base 2: sc[x][tt] holds keys 16 tt + 4 g .. of row r. Ks: the keys' scales.
  __device__ __forceinline__ void scores(const PagedAttn& a, const uint8_t* Kt, const float* Ks,
                                         v4f (&sc)[RT][kSub]) const {
    const int kb = fresh(k_base);
#pragma unroll
    for (int tt = 0; tt < kSub; ++tt) {
#pragma unroll
      for (int x = 0; x < RT; ++x) sc[x][tt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (kFp8) {
#pragma unroll
        for (int ks = 0; ks < kSteps; ks += 2) {
          const uint4 w = *reinterpret_cast<const uint4*>(Kt + 16 * tt * RB + (kb ^ (ks << 5)));
          const bf8 k0 = cvt_fp8x8(w.x, w.y), k1 = cvt_fp8x8(w.z, w.w);
#pragma unroll
          for (int x = 0; x < RT; ++x) sc[x][tt] = mfma16(k1, qf[x][ks + 1], mfma16(k0, qf[x][ks], sc[x][tt]));
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
          const bf8 kf = *reinterpret_cast<const bf8*>(Kt + 16 * tt * RB + (kb ^ (ks << 6)));
#pragma unroll
          for (int x = 0; x < RT; ++x) sc[x][tt] = mfma16(kf, qf[x][ks], sc[x][tt]);
        }
      }
    }
#pragma unroll
    for (int tt = 0; tt < kSub; ++tt) {
      v4f f = {a.scale_log2, a.scale_log2, a.scale_log2, a.scale_log2};
      if (kFp8) f = *reinterpret_cast<const v4f*>(Ks + 16 * tt + 4 * g) * a.scale_log2;
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[x][tt][e] *= f[e];
    }
  }

  // Does no row see key 16 tt + 4 g + e of the tile (from key0 on), or this lane's row not?
  __device__ __forceinline__ bool hidden(const int (&cnt)[kSub], int key0, int x, int tt, int e) const {
    return 4 * g + e >= cnt[tt] || key0 + 16 * tt + 4 * g + e >= limit[x];
  }

  // The online softmax: sc becomes P, the state follows. masked: not every row sees every key.
  // The base m of a row is its greatest score so far, or up to kSlack less: only a
  // greater one moves it (P stays below 2^kSlack), so that the tiles after the first
  // few take no maximum over lanes and leave O alone (3 to 5 % of calls of more than 64
  // rows). D = 64 moves it with every tile: O is half as wide there, and the branch cost
  // 3 to 4 %.
  __device__ __forceinline__ void weigh(v4f (&sc)[RT][kSub], const int (&cnt)[kSub], bool masked, int key0) {
    if (masked) {
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int tt = 0; tt < kSub; ++tt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (hidden(cnt, key0, x, tt, e)) sc[x][tt][e] = -kInf;
    }
    float mx[RT];
    bool above = false;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      mx[x] = sc[x][0][0];
#pragma unroll
      for (int tt = 0; tt < kSub; ++tt)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[x] = __builtin_fmaxf(mx[x], sc[x][tt][e]);
      above |= mx[x] > m[x] + kSlack;
    }
    if (D == 64 || __any(above)) {
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        mx[x] = __builtin_fmaxf(mx[x], __shfl_xor(mx[x], 16, 64));
        mx[x] = __builtin_fmaxf(mx[x], __shfl_xor(mx[x], 32, 64));
        const float mn = __builtin_fmaxf(m[x], mx[x]);
        const float alpha = __builtin_amdgcn_exp2f(m[x] - finite_max(mn));
        m[x] = mn;
        l[x] *= alpha;
#pragma unroll
        for (int d = 0; d < kDims; ++d) ot[x][d] *= alpha;
      }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      const float ms = finite_max(m[x]);
      float sum = 0.0f;
#pragma unroll
      for (int tt = 0; tt < kSub; ++tt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(sc[x][tt][e] - ms);
          sc[x][tt][e] = p;
          sum += p;
        }
      l[x] += sum;
    }
  }

  // O~^T += V^T P^T. whole: every key of the tile exists; differ: some row does not see all of them.
  __device__ __forceinline__ void values(const PagedAttn& a, uint8_t* Vt, const float* Vs, v4f (&sc)[RT][kSub],
                                         const int (&cnt)[kSub], bool whole, bool differ, int key0) {
    if (kFp8) {
#pragma unroll
      for (int tt = 0; tt < kSub; ++tt) {
        const v4f vs = *reinterpret_cast<const v4f*>(Vs + 16 * tt + 4 * g);
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[x][tt][e] *= vs[e];
      }
      if (!whole || differ) {
        // A hidden key's scale may be no number. (One branch around all of it, which the
        // statement keeps: as a branch per value these cost e4m3 calls 5 to 12 %.)
        asm volatile("" ::: "memory");
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
          for (int tt = 0; tt < kSub; ++tt)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[x][tt][e] = hidden(cnt, key0, x, tt, e) ? 0.0f : sc[x][tt][e];
      }
    }
    bf8 ph[RT][kKeys / 32], pl[RT][kKeys / 32];
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
      for (int st = 0; st < kKeys / 32; ++st) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const v4f& p = sc[x][2 * st + (e >> 1)];
          const float p0 = p[2 * (e & 1)], p1 = p[2 * (e & 1) + 1];
          hi[e] = cvt_pk_bf16(p0, p1);
          lo[e] = cvt_pk_bf16(p0 - bf16lo(hi[e]), p1 - bf16hi(hi[e]));
        }
        ph[x][st] = __builtin_bit_cast(bf8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        pl[x][st] = __builtin_bit_cast(bf8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
      }
    if (!whole) {
      // values of keys that do not exist: zeros (every wavefront that reads the tile writes them)
      uint8_t* const mine = Vt + fresh(lane * 16);
#pragma unroll
      for (int u = 0; u < T::kBytes / 1024; ++u) {
        const int key = T::KPI * u + lane / T::CPR;  // (one 16 of the tile per copy)
        if ((key & 15) >= cnt[(T::KPI * u) >> 4]) *reinterpret_cast<uint4*>(mine + u * 1024) = make_uint4(0u, 0u, 0u, 0u);
      }
      asm volatile("" ::: "memory");
    }
    bool odd = false;
    if (a.causal && differ) {
      // is every value finite?
      uint32_t bad = 0u;
      const uint8_t* const mine = Vt + fresh(lane * 16);
#pragma unroll 1
      for (int u = 0; u < T::kBytes / 1024; ++u) {
        const uint4 w4 = *reinterpret_cast<const uint4*>(mine + u * 1024);
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          bad |= kFp8 ? (((w[e] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u)
                      : (((w[e] & 0x7F807F80u) + 0x00800080u) & 0x80008000u);
      }
      odd = __any(bad != 0u);
    }
    const int vb = fresh(v_base);
    if (!odd) {
#pragma unroll
      for (int st = 0; st < kKeys / 32; ++st)
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
          const bf8 vf = value_operand(Vt, vb, st, d);
#pragma unroll
          for (int x = 0; x < RT; ++x) ot[x][d] = mfma16(vf, pl[x][st], mfma16(vf, ph[x][st], ot[x][d]));
        }
    } else {
      // For each number n of the tile's keys that a row may see: the products above with zeros
      // for the values behind, which only the rows that see n take. In those rows P is zero
      // there, so every bit is as with values that are finite. (8 tokens of 8 sequences of 1024
      // keys, d = 64: 55 us against 12 where the last tiles hold no such value.)
#pragma unroll 1
      for (int n = 1; n <= kKeys; ++n) {
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
          __builtin_amdgcn_sched_barrier(0);  // (one at a time: few registers are left)
          v4f sum[RT];
#pragma unroll
          for (int x = 0; x < RT; ++x) sum[x] = ot[x][d];
#pragma unroll
          for (int st = 0; st < kKeys / 32; ++st) {
            const uint4 w = __builtin_bit_cast(uint4, value_operand(Vt, vb, st, d));
            uint32_t ww[4] = {w.x, w.y, w.z, w.w};
            const int left = fresh(n - 4 * g) - 32 * st;  // (words e / 2: keys 16 (e / 2) + 2 (e % 2) and the next)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = 16 * (e >> 1) + 2 * (e & 1);
              ww[e] = k + 1 < left ? ww[e] : (k < left ? ww[e] & 0xFFFFu : 0u);
            }
            const bf8 vf = __builtin_bit_cast(bf8, make_uint4(ww[0], ww[1], ww[2], ww[3]));
#pragma unroll
            for (int x = 0; x < RT; ++x) sum[x] = mfma16(vf, pl[x][st], mfma16(vf, ph[x][st], sum[x]));
          }
#pragma unroll
          for (int x = 0; x < RT; ++x) ot[x][d] = fresh(min(limit[x] - key0, kKeys)) == n ? sum[x] : ot[x][d];
        }
      }
    }
  }

  // The lanes that share a row add their parts of l.
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      l[x] += __shfl_xor(l[x], 16, 64);
      l[x] += __shfl_xor(l[x], 32, 64);
    }
  }
};

// Up to 64 rows per KV head, 16 or 32 per workgroup: its kWaves wavefronts split a
// piece's keys.
template <int D, bool kFp8, int RT, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_kernel(PagedAttn a) {
  using W = PagedRows<D, kFp8, RT>;
  using T = typename W::T;
  constexpr int kKeys = T::kKeys, kSub = T::kSub, kRows = 16 * RT;
  constexpr int kState = kRows * D * 4;  // a wavefront's O at the end
  constexpr int kSlot = T::kSlot > kState ? T::kSlot : kState;
  __shared__ __align__(16) uint8_t smem[kWaves * kSlot];
  __shared__ float sml[2][kWaves][kRows];
  const int t = threadIdx.x, lane = t & 63, wave = wave_uniform(t >> 6);
  const int g = lane >> 4, r = lane & 15;
  Piece p;
  if (!find_piece<kKeys, kWaves>(a, lane, p)) return;
  const int i0 = p.p0 + wave * (p.p1 - p.p0) / kWaves, i1 = p.p0 + (wave + 1) * (p.p1 - p.p0) / kWaves;
  W w;
  w.init(a, p, kRows * p.rt, lane);

  uint8_t* const Kt = smem + wave * kSlot;
  uint8_t* const Vt = Kt + T::kBytes;
  const float* const Ks = reinterpret_cast<const float*>(Vt + T::kBytes);
  const float* const Vs = Ks + 64;
  const uint32_t lds = lds_u32(Kt);
  PagedCopy<D, kFp8> c;
  c.init(a, p, lane);
  auto issue = [&](int i, bool values) {
    const uint32_t dst = lds + (values ? T::kBytes : 0);
#pragma unroll
    for (int tt = 0; tt < kSub; ++tt) c.copy16(a, values, i * kSub + tt, tt & 1, dst + tt * 16 * T::RB);
    if (kFp8) c.template copy_scales<kSub>(a, values, i * kSub, lds + 2 * T::kBytes + (values ? 256 : 0));
  };

  // (of a short table all of them, without waiting for the length)
  c.load_pages(a, a.max_len <= 1024 ? 0 : i0 * kSub);
  if (i0 < i1) {
    issue(i0, false);
    issue(i0, true);
  }
  for (int i = i0; i < i1; ++i) {
    const bool more = i + 1 < i1;
    int cnt[kSub];
    bool whole = true;
#pragma unroll
    for (int tt = 0; tt < kSub; ++tt) cnt[tt] = c.count(c.pages, c.sb, i * kSub + tt), whole &= cnt[tt] == 16;
    const bool differ = (i + 1) * kKeys > w.seen;
    wait_vm<T::kCopies>();  // the keys have landed
    v4f sc[RT][kSub];
    w.scores(a, Kt, Ks, sc);
    wait_lds();
    if (more) {
      if ((i + 1) * kSub - c.sb >= 64) c.load_pages(a, (i + 1) * kSub);
      issue(i + 1, false);
    }
    w.weigh(sc, cnt, !whole || differ, i * kKeys);
    if (more)
      wait_vm<T::kCopies>();  // the values have landed (the next keys may be in flight)
    else
      wait_vm<0>();
    w.values(a, Vt, Vs, sc, cnt, whole, differ, i * kKeys);
    wait_lds();
    if (more) issue(i + 1, true);
  }

  // the wavefronts' states meet: O of row x at 16-byte chunk c ^ row
  w.finish();
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    if (g == 0) sml[0][wave][16 * x + r] = w.m[x], sml[1][wave][16 * x + r] = w.l[x];
#pragma unroll
    for (int d = 0; d < W::kDims; ++d)
      *reinterpret_cast<v4f*>(Kt + (16 * x + r) * D * 4 + (((4 * d + g) ^ r) << 4)) = w.ot[x][d];
  }
  __syncthreads();
  constexpr int C4 = D / 4;
  const int R = a.nq * (a.heads / a.kv_heads);
  float* part = a.part + (static_cast<int64_t>(p.slot + p.unit) * a.kv_heads * a.row_tiles + p.h * a.row_tiles + p.rt) *
                             (kRows * (D + 2));
#pragma unroll
  for (int e = t; e < kRows * C4; e += 64 * kWaves) {
    const int row = e / C4, c4 = e - row * C4, rr = kRows * p.rt + row;
    if (rr >= R) continue;
    float mm = -kInf;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) mm = __builtin_fmaxf(mm, sml[0][v][row]);
    const float ms = finite_max(mm);
    float ll = 0.0f;
    v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float f = __builtin_amdgcn_exp2f(sml[0][v][row] - ms);
      ll += f * sml[1][v][row];
      const v4f x = *reinterpret_cast<const v4f*>(smem + v * kSlot + row * D * 4 + ((c4 ^ (row & 15)) << 4));
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] += f * x[k];
    }
    if (p.n == 1) {
      store_out(a, out_row(a, p.s, p.h, rr), D, c4, o, mm, ll);
    } else {
      *reinterpret_cast<v4f*>(part + 2 * kRows + row * D + 4 * c4) = o;
      if (c4 == 0) part[row] = mm, part[kRows + row] = ll;
    }
  }
}

// More than 64 rows: four wavefronts of 32 rows each share every tile of keys, which
// comes in stages of kTiles tiles (16 KB of keys, 16 of values) through two LDS
// buffers, each wavefront copying its share; one barrier per stage. The stream does not
// bound these calls, nor is a unit full: the matrix cores are busy 30 % of the time (P's
// second term counted), the vector units 50 % (256 rows over 8 sequences of 4000 keys,
// 350 TFLOP/s); a wavefront's steps wait for each other, and two wavefronts per SIMD
// overlap little more than that.
// Against row tiles of 32 whose wavefronts split the keys (8 sequences of 1000..4096
// keys, 8 KV heads, D = 128): 72 rows 35.7 us against 42.9, 96 37.8 / 43.7, 128 41.1 /
// 46.1, 256 76 / 86; one sequence of 65536 and 96 rows 90 / 118; 64 sequences of 128
// rows and 500..1024 keys 70 / 88. For up to 64 rows two row tiles of 32 are the better
// choice: 16.0 us against 21.7 for 8 sequences of 1000 keys, 67.9 / 70.7 for one of
// 65536, 96 / 104 for 32 of 1000..4096; two wavefronts of 32 rows were no better
// (22.2, 92 and 86).
template <int D, bool kFp8>
__global__ __launch_bounds__(256, 2) void paged_attention_rows_kernel(PagedAttn a) {
  constexpr int RG = 4;
  using W = PagedRows<D, kFp8, 2>;
  using T = typename W::T;
  constexpr int kKeys = T::kKeys, kSub = T::kSub, kRows = 32 * RG;
  constexpr int kTiles = RG * 4096 / T::kBytes, kSubs = kTiles * kSub, kStageKeys = 16 * kSubs;
  constexpr int kHalf = kTiles * T::kBytes;  // a stage's keys (or values)
  constexpr int kStage = 2 * kHalf + (kFp8 ? 2 * kStageKeys * 4 : 0);
  static_assert(kTiles >= 1 && kSubs % RG == 0 && kSubs <= 64 && (!kFp8 || 2 * kStageKeys / 64 % RG == 0), "stage");
  __shared__ __align__(16) uint8_t smem[2 * kStage];
  const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
  Piece p;
  if (!find_piece<kKeys, 1>(a, lane, p)) return;
  const int R = a.nq * (a.heads / a.kv_heads), row0 = kRows * p.rt + 32 * wave;
  W w;
  w.init(a, p, row0, lane);
  PagedCopy<D, kFp8> c;
  c.init(a, p, lane);
  const uint32_t lds = lds_u32(smem);
  // this wavefront's share of the stage from tile i on
  auto issue = [&](int i, int buf) {
    if ((i + kTiles) * kSub - c.sb > 64) c.load_pages(a, i * kSub);
    const uint32_t dst = lds + buf * kStage;
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int b = 0; b < kSubs / RG; ++b) {
        const int sub = wave + RG * b;
        c.copy16(a, v != 0, i * kSub + sub, wave & 1, dst + v * kHalf + sub * 16 * T::RB);
      }
    if (kFp8) {
#pragma unroll
      for (int b = 0; b < 2 * kStageKeys / 64 / RG; ++b) {
        const int q = wave + RG * b, v = q >= kStageKeys / 64 ? 1 : 0, k = q - v * (kStageKeys / 64);
        c.template copy_scales<4>(a, v != 0, i * kSub + 4 * k, dst + 2 * kHalf + v * kStageKeys * 4 + k * 256);
      }
    }
  };
  c.load_pages(a, p.p0 * kSub);
  if (p.p0 < p.p1) issue(p.p0, 0);
  for (int i = p.p0, buf = 0; i < p.p1; i += kTiles, buf ^= 1) {
    const int pages = c.pages, sb = c.sb;  // (the next stage's may be other ones)
    wait_vm<0>();  // this wavefront's copies of the stage have landed ...
    bar();         // ... and everyone's; the other buffer has been read
    if (i + kTiles < p.p1) issue(i + kTiles, buf ^ 1);
    if (row0 < R) {
      uint8_t* const K = smem + buf * kStage;
      const float* const S = reinterpret_cast<const float*>(K + 2 * kHalf);
#pragma unroll 1
      for (int q = 0; q < kTiles && i + q < p.p1; ++q) {
        int cnt[kSub];
        bool whole = true;
#pragma unroll
        for (int tt = 0; tt < kSub; ++tt) cnt[tt] = c.count(pages, sb, (i + q) * kSub + tt), whole &= cnt[tt] == 16;
        const int key0 = (i + q) * kKeys;
        const bool differ = key0 + kKeys > w.seen;
        v4f sc[2][kSub];
        w.scores(a, K + q * T::kBytes, S + q * kKeys, sc);
        w.weigh(sc, cnt, !whole || differ, key0);
        w.values(a, K + kHalf + q * T::kBytes, S + kStageKeys + q * kKeys, sc, cnt, whole, differ, key0);
      }
    }
    wait_lds();
  }
  w.finish();
  float* part = a.part + (static_cast<int64_t>(p.slot + p.unit) * a.kv_heads * a.row_tiles + p.h * a.row_tiles + p.rt) *
                             (kRows * (D + 2));
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int row = 32 * wave + 16 * x + w.r, rr = kRows * p.rt + row;
    if (rr >= R) continue;
    const int64_t dst = out_row(a, p.s, p.h, rr);
#pragma unroll
    for (int d = 0; d < W::kDims; ++d) {
      const int c4 = 4 * d + w.g;
      if (p.n == 1) {
        store_out(a, dst, D, c4, w.ot[x][d], w.m[x], w.l[x]);
      } else {
        *reinterpret_cast<v4f*>(part + 2 * kRows + row * D + 4 * c4) = w.ot[x][d];
        if (c4 == 0) part[row] = w.m[x], part[kRows + row] = w.l[x];
      }
    }
  }
}

// Joins the pieces of a (sequence, KV head, row tile), 32 dims of join_rows rows per
// workgroup: 8 threads per (row, share of the pieces), the shares (every pg-th
// piece, in order) joined through LDS in order. Each thread has kAhead pieces'
// loads in flight, and a long sequence's pieces are spread over up to 32 shares:
// one thread per 4 dims walking 128 pieces took 95 us (one row of 131072 keys); with
// one share for 28 rows' 256 pieces the call took 65 us, with 8 of them 27.
template <int D, int kRows>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttn a) {
  constexpr int kPart = kRows * (D + 2), kAhead = 4;
  __shared__ __align__(16) float so[32][8][4];
  __shared__ float sm[32], sl[32];
  const int t = threadIdx.x;
  const int hrs = a.kv_heads * a.row_tiles;
  const int hr = blockIdx.x % hrs, s = blockIdx.x / hrs;
  const int2 cut = a.cuts[s];
  const int n = cut.x;
  if (n == 1) return;
  const int h = hr / a.row_tiles, rt = hr - h * a.row_tiles;
  const int row0 = a.join_rows * (blockIdx.y / (D / 32));
  const int left = min(kRows, a.nq * (a.heads / a.kv_heads) - kRows * rt) - row0, rows = min(left, a.join_rows);
  if (rows <= 0) return;
  const int rows2 = rows <= 1 ? 1 : 1 << (32 - __builtin_clz(rows - 1)), pg = 32 / rows2;
  const int64_t stride = static_cast<int64_t>(hrs) * kPart;
  const float* part = a.part + cut.y * stride + static_cast<int64_t>(hr) * kPart + row0;
  const int c = t & 7, u = t >> 3, row = u & (rows2 - 1), share = u / rows2;
  const int c4 = 8 * (blockIdx.y % (D / 32)) + c;
  float m = -kInf, l = 0.0f;
  v4f o = {0.0f, 0.0f, 0.0f, 0.0f};
  if (row < rows) {
    for (int p = share; p < n; p += kAhead * pg) {
      float pm[kAhead], pl[kAhead];
      v4f po[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int q = p + k * pg;
        const float* x = part + (q < n ? q : p) * stride;
        pm[k] = q < n ? x[row] : -kInf;
        pl[k] = x[kRows + row];
        po[k] = *reinterpret_cast<const v4f*>(x + 2 * kRows + row0 * (D - 1) + row * D + 4 * c4);  // (x is row0 on)
      }
      float mn = m;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) mn = __builtin_fmaxf(mn, pm[k]);
      const float ms = finite_max(mn), f = __builtin_amdgcn_exp2f(m - ms);
      m = mn;
      l *= f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (p + k * pg >= n) break;
        const float fk = __builtin_amdgcn_exp2f(pm[k] - ms);
        l += fk * pl[k];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += fk * po[k][e];
      }
    }
  }
  *reinterpret_cast<v4f*>(so[u][c]) = o;
  if (c == 0) sm[u] = m, sl[u] = l;
  __syncthreads();
  if (share != 0 || row >= rows) return;
  float mm = m;
  for (int k = 1; k < pg; ++k) mm = __builtin_fmaxf(mm, sm[row + k * rows2]);
  const float ms = finite_max(mm), f = __builtin_amdgcn_exp2f(m - ms);
  l *= f;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] *= f;
  for (int k = 1; k < pg; ++k) {
    const int w = row + k * rows2;
    const float fk = __builtin_amdgcn_exp2f(sm[w] - ms);
    l += fk * sl[w];
    const v4f x = *reinterpret_cast<const v4f*>(so[w][c]);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += fk * x[e];
  }
  store_out(a, out_row(a, s, h, kRows * rt + row0 + row), D, c4, o, mm, l);
}

// Rows of a workgroup: 16 or 32 where its wavefronts split the keys, 128 where they
// split the rows (the times of both stand at that kernel).
// Where the wavefronts split the keys: one workgroup of 8 per CU while the sequences,
// uncut, are too few for two of 4. Shorter runs per wavefront cost less than a cut
// with its join (times of one state's calls in a row): 8 blocks of 32 tokens, 700..1024
// keys and 32 heads 25.6 us against 30.6, 32 tokens with 200..1024 keys 17.8 / 22.9, 8
// with 100..1000 12.2 / 14.4, 48 with 1..8191 154.7 / 156.6 (longer sequences that have to be cut are even, 1 to
// 131072 keys, or lose to their longer pieces, 8 of 1000..4096 23.9 / 22.0). With more
// sequences two workgroups of 4 per CU hide each other's start and end: 128 of
// 50..500 keys 31.2 us against 39.0, of 100..2000 in e4m3 66.9 / 77.0 (of 250..2500 in
// bf16 145 / 138, but their lengths are not known here).
struct PagedPlan {
  int rows, ways;
  int64_t row_tiles, wq, parts;  // parts: piece states that a call may keep
};
PagedPlan paged_plan(int64_t S, int64_t nq, int64_t heads, int64_t kv_heads) {
  const int64_t R = nq * (heads / kv_heads);
  PagedPlan p;
  p.rows = R <= 16 ? 16 : (R <= 64 ? 32 : 128);
  p.row_tiles = (R + p.rows - 1) / p.rows;
  const int64_t hr = kv_heads * p.row_tiles;
  p.wq = (2 * device_cu_count() + hr - 1) / hr;
  p.ways = R > 64 ? 1 : (S < p.wq ? 8 : 4);
  if (p.ways == 8) p.wq = (device_cu_count() + hr - 1) / hr;
  p.parts = p.wq == 1 ? 0 : 4 * p.wq * hr;
  return p;
}

}  // namespace

hipError_t launch_paged_append(hipStream_t st, PagedAppend a, int64_t T, int64_t d, bool fp8) {
  const int G = static_cast<int>(256 / (d / 8));
  const int HT = a.heads + 2 * a.kv_heads;
  const int per = (HT + G - 1) / G;
  // Few tokens: a workgroup for every G vectors of a token, the chip not being full
  // otherwise (48 vectors of 128 dims: 16 tokens 3.0 us against 3.3, 64 in e4m3 3.7
  // against 4.2); from then on one for 3 G, whose loads are in flight together (512
  // tokens 4.5 us against 4.8).
  const bool few = T * per <= 2 * device_cu_count();
  const int ny = few ? per : (per + 2) / 3;
  // Heads that leave half the groups idle: several tokens per workgroup (6 vectors of 64
  // dims in e4m3, 97024 tokens: 31 us against 90).
  const int need = few ? HT : (HT + 2) / 3;
  a.groups_log2 = 0;
  while ((1 << a.groups_log2) < need) ++a.groups_log2;
  const bool tokens = (1 << a.groups_log2) < G;
  const int64_t at_once = tokens ? G >> a.groups_log2 : 1;
  const dim3 grid(static_cast<unsigned>((T + at_once - 1) / at_once), static_cast<unsigned>(tokens ? 1 : ny)), block(256);
#define PP(D_, F_)                                                                                  \
  if (tokens) hipLaunchKernelGGL((paged_append_kernel<D_, F_, true>), grid, block, 0, st, a, T);    \
  else hipLaunchKernelGGL((paged_append_kernel<D_, F_, false>), grid, block, 0, st, a, T)
  if (d == 128 && fp8) {
    PP(128, true);
  } else if (d == 128) {
    PP(128, false);
  } else if (fp8) {
    PP(64, true);
  } else {
    PP(64, false);
  }
#undef PP
  return hipGetLastError();
}

// The workspace: [S] (pieces, first kept piece), then the kept pieces' states.
static size_t ws_bytes(int64_t S, int64_t parts, int64_t rows, int64_t d) {
  const size_t cuts = (static_cast<size_t>(S) * 8 + 255) / 256 * 256;
  return (cuts + static_cast<size_t>(parts) * rows * (d + 2) * 4 + 255) / 256 * 256;
}
size_t paged_attention_ws_bytes(int64_t S, int64_t nq, int64_t heads, int64_t kv_heads, int64_t d) {
  const PagedPlan p = paged_plan(S, nq, heads, kv_heads);
  return ws_bytes(S, p.parts, p.rows, d);
}

namespace {
// What the capacity of the table's pages leaves of a plan.
struct PagedRoom {
  int64_t pieces;  // of all sequences, at most; S: none can be cut
  int64_t kept;    // piece states, at most
};
PagedRoom paged_room(const PagedPlan& p, const PagedAttn& a, int64_t d, bool fp8) {
  using Keys = PieceRule<8>;
  using Rows = PieceRule<1>;
  const int keys = tile_keys(static_cast<int>(d), fp8, p.rows == 16 ? 1 : 2);
  const int64_t nt = (a.max_len + keys - 1) / keys;
  const int64_t whole = p.wq <= a.S ? Keys::kLong : (p.ways > 1 ? Keys::kWhole : Rows::kWhole);
  const int64_t least = p.ways > 1 ? Keys::kLeast : Rows::kLeast;
  if (p.wq == 1 || nt <= whole) return {a.S, 0};
  const int64_t by_table = a.S * ((nt + least - 1) / least);  // (piece_tiles is never below kLeast)
  return {std::min(2 * p.wq + a.S, by_table), std::min(p.parts, by_table * a.kv_heads * p.row_tiles)};
}
}  // namespace

size_t paged_attention_need_bytes(const PagedAttn& a, int64_t d, bool fp8) {
  const PagedPlan p = paged_plan(a.S, a.nq, a.heads, a.kv_heads);
  const PagedRoom r = paged_room(p, a, d, fp8);
  return r.pieces == a.S ? 0 : ws_bytes(a.S, r.kept, p.rows, d);
}

hipError_t launch_paged_attention(hipStream_t st, PagedAttn a, int64_t d, bool fp8, void* ws) {
  const PagedPlan p = paged_plan(a.S, a.nq, a.heads, a.kv_heads);
  const int64_t n = paged_room(p, a, d, fp8).pieces;
  a.whole = n == a.S;
  if (!a.whole) {
    a.cuts = static_cast<int2*>(ws);
    a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + ws_bytes(a.S, 0, 0, 0));
  }
  a.row_tiles = static_cast<int>(p.row_tiles);
  a.wq = static_cast<int>(p.wq);
  auto launch = [&](auto kernel, auto join) {
    const dim3 grid(static_cast<unsigned>((n * a.kv_heads + 7) / 8 * 8 * p.row_tiles));
    hipLaunchKernelGGL(kernel, grid, dim3(p.ways == 8 ? 512 : 256), 0, st, a);
    if (a.whole) return;  // (no sequence of several pieces: nothing to join)
    // the join: as few rows per workgroup (as many shares of the pieces) as fill the chip
    const int64_t R = static_cast<int64_t>(a.nq) * (a.heads / a.kv_heads), rows = std::min<int64_t>(R, p.rows);
    const int64_t joins = static_cast<int64_t>(a.S) * a.kv_heads * p.row_tiles, dims = d / 32;
    a.join_rows = 4;  // (more shares than 8 take longer to meet than they save)
    while (a.join_rows < 32 && a.join_rows < rows &&
           joins * dims * ((rows + a.join_rows - 1) / a.join_rows) > 4 * device_cu_count())
      a.join_rows *= 2;
    const dim3 jgrid(static_cast<unsigned>(joins), static_cast<unsigned>(dims * ((rows + a.join_rows - 1) / a.join_rows)));
    hipLaunchKernelGGL(join, jgrid, dim3(256), 0, st, a);
  };
#define PA(D_, F_)                                                              \
  if (p.rows == 128)                                                            \
    launch(paged_attention_rows_kernel<D_, F_>, paged_join_kernel<D_, 128>);    \
  else if (p.rows == 32 && p.ways == 8)                                         \
    launch(paged_attention_kernel<D_, F_, 2, 8>, paged_join_kernel<D_, 32>);    \
  else if (p.rows == 32)                                                        \
    launch(paged_attention_kernel<D_, F_, 2, 4>, paged_join_kernel<D_, 32>);    \
  else if (p.ways == 8)                                                         \
    launch(paged_attention_kernel<D_, F_, 1, 8>, paged_join_kernel<D_, 16>);    \
  else                                                                          \
    launch(paged_attention_kernel<D_, F_, 1, 4>, paged_join_kernel<D_, 16>);
  if (d == 128 && fp8) {
    PA(128, true)
  } else if (d == 128) {
    PA(128, false)
  } else if (fp8) {
    PA(64, true)
  } else {
    PA(64, false)
  }
#undef PA
  return hipGetLastError();
}

}  // namespace lacache
