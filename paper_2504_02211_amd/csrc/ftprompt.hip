// Attention over packed prompts with grouped heads: the kernel and the C ABI of ../include/ftprompt.h.
//
// One pass over the keys with a running maximum and sum (the weights never leave the registers).  A workgroup owns 128 rows of one
// (sequence, key / value head); a ROW is one (query, head of the group), numbered query-major, so that the heads of a group share
// the key and value tiles in LDS, short prompts fill a row tile with heads, and the rows of a tile end within 128 / group keys of each other:
// little is computed only to be masked.  Wave w owns rows 32w .. 32w+31.
//
// Scores are computed transposed, S^T = K Q^T with the 32x32x16 MFMA: lane l owns row l % 32 and, with h = l / 32, the keys
// 8g + 4h + r (g, r in 0..3) of a block of 32.  A maximum or sum over keys is in-lane work and one exchange between lane and lane^32.
// The weights then are the right-hand operand of O^T = V^T P^T as they lie, where contraction slot (h, 4s + r) stands for key 16i + 8s + 4h + r;
// V^T in that order comes from row-major LDS tiles by transposing reads of four keys each.
//
// Bound: 16,384 tokens of 32 heads on 4 of 128 (2.2e12 operations) take 1.97 to 2.15 ms by card, 1020 to 1115 TFLOP/s where a large library product reaches 1222;
// the clock falls to 1.64 GHz under it with the matrix pipe 63 % busy.  With fewer rows it is the time of a key tile in one workgroup, 1.0 us at head_dim 128 and
// 0.7 at 64, of which a row tile needs one after the other: 24 prompts of up to 1531 tokens, 12 heads of 64, take 26 to 28 us.  Four waves of 32 rows, two
// workgroups to a CU: waves of 64 rows would read half as much from LDS, but came out of the compiler with their accumulators copied (3.6 ms); three workgroups to a CU at
// head_dim 64 have too few registers (one prompt of 16,000 tokens, 4 heads on 1: 205 us, 259 with three).
#include "ftprompt.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>
#include <type_traits>

namespace ftprompt {
using namespace ftserve;

constexpr int BM = 128, BN = 64, NW = 4, STAGES = 2;      // rows of a workgroup, keys of a tile; waves; stages in LDS
// Long row tiles are divided by their keys where there are too few of them to keep the chip busy to the end: into shares of equal length, about `piece` key tiles
// long, so that a call has about SHARES workgroups of as much to do.  A share costs its state through memory beside its keys, together about the time of ten
// tiles: pieces have LEAST tiles, or FEW where row tiles leave half of the CUs idle, and a row tile a third longer than a piece stays whole.  Measured (us; whole,
// divided): 3 x 20 queries over 8000 keys, 32 heads on 8: 135, 38; 6 chunks of up to 509 over 3000, 16 on 4: 70, 55; 1 x 4000, 8 on 2: 79, 58;
// 2 x 9090, 5 on 1, of 64: 120, 99.  With pieces of 10: 1 x 2000, 32 on 8: 53, 60; 24 of up to 1531, 12, of 64: 29, 36.
constexpr int SHARES = 512, LEAST = 24, FEW = 12, STATES = 2 * SHARES, MANY = 64;

struct Rows { char* data; int64_t token, head; };         // strides in bytes

struct Args {
  Rows q, k, v, o;
  const int32_t *cu_q, *cu_k;
  int32_t batch, total_q, total_k, kv_heads, group;
  int32_t divide;          // 0: no row tile is divided
  float scale_log2;
  float* ws;               // states of shares, STATES of them
  uint32_t* done;          // shares of a row tile that are there, by its first state; 0 between calls
};

template <int D> constexpr int tile_bytes() { return BN * D * 2; }
template <int D> constexpr int lds_bytes() { return STAGES * 2 * tile_bytes<D>(); }

// N times 16 bytes per lane from (uniform base + per-lane byte offsets) straight into LDS, 1 KB apart from the uniform LDS address on.
// (Opaque to the compiler, which would wait for the tile in flight before it reads another; ordering against barriers and counted waits is kept because all of
// them are side-effecting instructions.  The first wait covers a base that a vector instruction has moved to its scalar registers just before: five states.)
template <int N> __device__ __forceinline__ void load_lds16(const void* base, const uint32_t (&off)[N], uint32_t lds_addr) {
  static_assert(N == 2 || N == 4, "loads of a wave for a tile");
#define FTPROMPT_NEXT(r) "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %" #r ", %[base]\n\t"
  if constexpr (N == 4)
    asm volatile("s_mov_b32 m0, %[lds]\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %[base]\n\t" FTPROMPT_NEXT(1) FTPROMPT_NEXT(2) FTPROMPT_NEXT(3)
                 ::"v"(off[0]), "v"(off[1]), "v"(off[2 % N]), "v"(off[3 % N]), [base] "s"(base), [lds] "s"(lds_addr) : "memory", "scc", "m0");
  else
    asm volatile("s_mov_b32 m0, %[lds]\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %[base]\n\t" FTPROMPT_NEXT(1)
                 ::"v"(off[0]), "v"(off[1]), [base] "s"(base), [lds] "s"(lds_addr) : "memory", "scc", "m0");
#undef FTPROMPT_NEXT
}

template <bool BF> __device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c) {
  if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}
// c plus the lane's own four values (sixteen products of 4x4 with ones side by side): a sum on the matrix pipe
template <bool BF> __device__ __forceinline__ float4v add4(uint2v x, float4v c) {
  if constexpr (BF) return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(short4v{0x3F80, 0x3F80, 0x3F80, 0x3F80}, __builtin_bit_cast(short4v, x), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_4x4x4f16(half4v{1, 1, 1, 1}, __builtin_bit_cast(half4v, x), c, 0, 0, 0);
}

__device__ __forceinline__ float max32(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
  return __builtin_fmaxf(as_f(r[0]), as_f(r[1]));
}
__device__ __forceinline__ float sum32(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
  return as_f(r[0]) + as_f(r[1]);
}

__device__ __forceinline__ bool is_finite(float x) { return __builtin_fabsf(x) <= 3.4028235e38f; }

// Sums over the lanes up to this one.
__device__ __forceinline__ int plus(int a, int b) { return a + b; }
__device__ __forceinline__ int plus_float(int a, int b) { return (int)as_u(as_f((uint32_t)a) + as_f((uint32_t)b)); }
template <int (*ADD)(int, int)> __device__ __forceinline__ int scan(int x) {
  x = ADD(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));      // row_shr 1, 2, 4, 8
  x = ADD(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
  x = ADD(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
  x = ADD(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
  x = ADD(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));      // row_bcast 15, 31
  return ADD(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
}
__device__ __forceinline__ int sum_upto(int x) { return scan<plus>(x); }

// A sequence: its first rows, its queries and keys, its rows and row tiles; row r sees nk - nq + r / G + 1 keys.
struct Sequence {
  int q0, k0, nq, nk, rows, tiles;
  __device__ __forceinline__ int seen_by(int r, int G) const { return nk - nq + (r < rows ? r : rows - 1) / G + 1; }
  __device__ __forceinline__ int key_tiles(int tile, int G) const {
    const int keys = seen_by(tile * BM + BM - 1, G);
    return keys > 0 ? (keys + BN - 1) / BN : 0;
  }
  // the first row tile of more than `part` shares (part >= 1), `tiles` if there is none: one that sees more than part * piece key tiles, for a second share a third more
  __device__ __forceinline__ int first_with(int part, int piece, int G) const {
    const int64_t more = part == 1 ? piece + piece / 3 : (int64_t)part * piece;
    const int64_t at = (more * BN - (nk - nq)) * G;      // the first row that sees more
    return at <= 0 ? 0 : at > rows - 1 ? tiles : (int)(at / BM);
  }
};
__device__ __forceinline__ Sequence sequence(const Args& a, int b) {
  Sequence s{0, 0, 0, 0, 0, 0};
  if (b >= a.batch) return s;
  s.q0 = clamped(a.cu_q[b], a.total_q);
  s.k0 = clamped(a.cu_k[b], a.total_k);
  const int q1 = clamped(a.cu_q[b + 1], a.total_q), k1 = clamped(a.cu_k[b + 1], a.total_k);
  s.nq = q1 > s.q0 ? q1 - s.q0 : 0;
  s.nk = k1 > s.k0 ? k1 - s.k0 : 0;
  s.rows = s.nq * a.group;
  s.tiles = (s.rows + BM - 1) / BM;
  return s;
}

// Share `id` of a key / value head: first all row tiles' first shares, longest tiles of a sequence first, then the second shares of those that have one, and
// so on.  Lane l looks after sequences l * per ..; all waves come to the same result.
struct Share {
  Sequence s;
  int tile, part, parts, slot;      // slot: number of the row tile's first state
};
__device__ __forceinline__ bool share_of(const Args& a, int id, Share& x) {
  const int lane = threadIdx.x & 63, G = a.group;
  if (!a.divide) {
    // sequence b owns the numbers from cu_q[b] * G / BM + b on: at least as many as it has row tiles, whatever the others have
    auto before = [&](int b) { return (int64_t)clamped(a.cu_q[b], a.total_q) * G / BM + b; };
    const int last = (int)((int64_t)a.total_q * G / BM) + a.batch - 1 - id;
    if (last < 0) return false;
    const int b = sequence_of(a.batch, last, before);
    x.s = sequence(a, b);
    x.tile = last - (int)before(b);
    x.part = x.slot = 0;
    x.parts = 1;
    return x.tile >= 0 && x.tile < x.s.tiles;
  }
  // lane b looks after sequence b
  const Sequence mine = sequence(a, lane);
  // bounds that fall: more rows than there are, and not a workgroup for each; nothing is divided then
  const bool fall = lane < a.batch && a.cu_q[lane + 1] < a.cu_q[lane];
  // key tiles of all row tiles, not too few: they rise evenly from one to the next
  const float work = mine.tiles ? (0.5f * (float)(mine.key_tiles(0, G) + mine.key_tiles(mine.tiles - 1, G)) + 1.f) * (float)mine.tiles : 0.f;
  const int tiles_upto = sum_upto(mine.tiles), least = __builtin_amdgcn_readlane(tiles_upto, 63) < 128 / a.kv_heads ? FEW : LEAST;
  const float fair = as_f((uint32_t)__builtin_amdgcn_readlane(scan<plus_float>((int)as_u(work)), 63)) * (float)a.kv_heads * (1.001f / SHARES);
  const int piece = __builtin_amdgcn_readfirstlane(__any(fall) || fair > 1e8f ? 100000000 : fair < (float)least ? least : (int)fair + 1);
  for (int part = 0;; ++part) {
    const int n = part == 0 ? mine.tiles : mine.tiles - mine.first_with(part, piece, G), upto = part == 0 ? tiles_upto : sum_upto(n);
    const int all = __builtin_amdgcn_readlane(upto, 63);
    if (all == 0) return false;
    if (id >= all) {
      id -= all;
      continue;
    }
    const int owner = __ffsll((unsigned long long)__ballot(upto > id)) - 1;
    auto from_owner = [&](int v) { return __builtin_amdgcn_readlane(v, owner); };
    x.s = Sequence{from_owner(mine.q0), from_owner(mine.k0), from_owner(mine.nq), from_owner(mine.nk), from_owner(mine.rows), from_owner(mine.tiles)};
    x.tile = x.s.tiles - 1 - (id - from_owner(upto - n));
    x.part = part;
    const int length = x.s.key_tiles(x.tile, G);
    x.parts = length > piece + piece / 3 ? (length + piece - 1) / piece : 1;
    x.slot = 0;
    if (x.parts > 1)      // states of the divided row tiles before this one: of each q, the tiles of more than q shares; those of more than 0 are those of more than 1
      for (int q = 1;; ++q) {
        const int m = mine.tiles - mine.first_with(q, piece, G), m_upto = sum_upto(m);
        if (__builtin_amdgcn_readlane(m_upto, 63) == 0) break;
        const int first = x.s.first_with(q, piece, G), here = x.tile > first ? x.tile - first : 0;
        x.slot += (q == 1 ? 2 : 1) * (from_owner(m_upto - m) + here);
      }
    return true;
  }
}

typedef __attribute__((address_space(3))) char lds_char;

__device__ __forceinline__ void put(float* p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)as_u(a) | (uint64_t)as_u(b) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int D, bool BF, bool F32OUT>
__global__ __launch_bounds__(NW * 64, 2) void ftprompt_main(const Args a) {
  extern __shared__ uint4v lds[];
  constexpr int NF = D / 32, TILE = tile_bytes<D>();
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int hk = blockIdx.x % a.kv_heads, G = a.group;
  Share x;
  if (!share_of(a, blockIdx.x / a.kv_heads, x)) return;
  const int tile = x.tile, q0 = x.s.q0, k0 = x.s.k0, nq = x.s.nq, nk = x.s.nk, rows = x.s.rows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;

  // keys that row r of the sequence sees (may be <= 0); rows behind the last count as it
  auto seen_by = [&](int r) { return x.s.seen_by(r, G); };
  const int row0 = tile * BM + wave * 32, length = x.s.key_tiles(tile, G);
  const int all_seen = seen_by(row0), any_seen = seen_by(row0 + 31);
  // key tiles of this share; of this wave; that every row of it sees whole (counted from the beginning of the sequence)
  const int begin = (int)((int64_t)length * x.part / x.parts), tiles = (int)((int64_t)length * (x.part + 1) / x.parts);
  auto at_most = [&](int n) { return n < tiles ? n : tiles; };
  const int steps = at_most(any_seen > 0 ? (any_seen + BN - 1) / BN : 0), full = at_most(all_seen > 0 ? all_seen / BN : 0);

  const int row = row0 + n, rowc = row < rows ? row : rows - 1;
  const int query = rowc / G, head = hk * G + rowc - query * G, seen = nk - nq + query + 1;
  uint4v qf[D / 16];
  const char* const qp = a.q.data + (int64_t)(q0 + query) * a.q.token + (int64_t)head * a.q.head + 16 * h;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const uint4v*>(qp + 32 * i);

  // Tiles: row r of keys has its 16-byte chunk c at place c ^ (r & 15) (head_dim 64: c ^ (r / 2 & 7)), a row of values its 64 bytes f at f ^ (r & 3) (f ^ (r / 2 & 1)).
  // Sixteen lanes that read 16 bytes of as many rows of keys then meet all banks once, and so do 32 that read 32 bytes of four rows of values, twice.
  constexpr int CH = D / 8, LOADS = TILE / 1024 / NW, RPL = 64 / CH;      // chunks of a row; loads of a wave for a tile; rows of a load
  uint32_t koff[LOADS], voff[LOADS];
  const char* kbase = a.k.data + (int64_t)k0 * a.k.token + (int64_t)hk * a.k.head;
  const char* vbase = a.v.data + (int64_t)k0 * a.v.token + (int64_t)hk * a.v.head;
  auto chunk_k = [&](int r) { return (uint32_t)((lane % CH) ^ (D == 128 ? r & 15 : r >> 1 & 7)) * 16; };
  auto chunk_v = [&](int r) { return (uint32_t)((lane % CH) ^ (D == 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2)) * 16; };
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = (wave * LOADS + i) * RPL + lane / CH;
    koff[i] = (uint32_t)r * (uint32_t)a.k.token + chunk_k(r);
    voff[i] = (uint32_t)r * (uint32_t)a.v.token + chunk_v(r);
  }
  auto issue_one = [&](const char* base, int64_t stride, const uint32_t (&off)[LOADS], auto chunk, int t, uint32_t to) __attribute__((always_inline)) {
    const char* const p = base + (int64_t)t * BN * stride;
    to += (uint32_t)wave * (LOADS * 1024);
    if ((int64_t)(t + 1) * BN <= nk) {
      load_lds16<LOADS>(p, off, to);
    } else {           // rows behind the last key: the last one again (no row sees them)
      uint32_t held[LOADS];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = (wave * LOADS + i) * RPL + lane / CH, rc = r < nk - 1 - t * BN ? r : nk - 1 - t * BN;
        held[i] = (uint32_t)rc * (uint32_t)stride + chunk(r);
      }
      load_lds16<LOADS>(p, held, to);
    }
  };
  auto issue_k = [&](int t, uint32_t to) __attribute__((always_inline)) { issue_one(kbase, a.k.token, koff, chunk_k, t, to); };
  auto issue_v = [&](int t, uint32_t to) __attribute__((always_inline)) { issue_one(vbase, a.v.token, voff, chunk_v, t, to); };

  // operands from LDS.  k_at / v_at: address of a step's first row
  const uint32_t klane = (uint32_t)n * (2 * D) + (uint32_t)(h ^ (D == 128 ? n & 15 : n >> 1 & 7)) * 16;
  const int rr = (lane & 15) >> 2;
  const uint32_t vlane = (uint32_t)(4 * h + rr) * (2 * D) + (uint32_t)((lane >> 4 & 1) * 32 + (lane & 3) * 8) + (uint32_t)(D == 128 ? rr : rr >> 1) * 64;
  uint32_t kplace[D / 16], vplace[NF];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) kplace[i] = lds0 + (klane ^ (32u * i));
#pragma unroll
  for (int f = 0; f < NF; ++f) vplace[f] = lds0 + (vlane ^ (64u * f));
  auto key = [&](uint32_t k_at, int i) { return *(__attribute__((address_space(3))) uint4v*)(uintptr_t)(kplace[i] + k_at); };
  auto value = [&](uint32_t v_at, int i, int f) {      // V^T: elements 32f + lane % 32, keys 16i + 4h + 0..3 and 8 on
    const uint32_t at = vplace[f] + v_at + (uint32_t)i * (32 * D);
    const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)at));
    const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)(at + 16 * D)));
    return uint4v{x[0], x[1], y[0], y[1]};
  };

  float16v o[NF];
  float4v sums = (float4v)0.f;
  float ref = -3.4028234e38f;
#pragma unroll
  for (int f = 0; f < NF; ++f) o[f] = (float16v)0.f;

  // scores of a tile, transposed
  auto scores = [&](uint32_t k_at, float16v (&to)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      to[t] = (float16v)0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) to[t] = mfma32<BF>(key(k_at + t * (64 * D), i), qf[i], to[t]);
    }
  };
  auto mask = [&](int t, float16v (&x)[2]) __attribute__((always_inline)) {
    const int limit = seen - t * BN - 4 * h;
#pragma unroll
    for (int v = 0; v < 32; ++v)
      if (limit <= 8 * (v >> 2) + (v & 3)) x[v >> 4][v & 15] = -__builtin_inff();
  };
  // The reference lies UP below the largest score that it was made from, and weights reach 2^(ROOM + UP).  fp16: 2^14, so that those far below the largest keep their
  // bits.  bf16: 1, so that sums of weights and values stay finite where those of the formula do.
  constexpr float ROOM = 8.f, UP = BF ? -8.f : 6.f;
  auto largest = [&](const float16v (&x)[2]) __attribute__((always_inline)) {
    float m = __builtin_fmaxf(x[0][0], x[1][0]);
#pragma unroll
    for (int v = 1; v < 16; ++v) m = __builtin_fmaxf(__builtin_fmaxf(m, x[0][v]), x[1][v]);
    return max32(m) * a.scale_log2;
  };
  // a row's reference moves when a score exceeds it by more than there is room for: rarely after the first step
  auto renew = [&](float m) __attribute__((always_inline)) {
    if (__any(m > ref + (ROOM + UP))) {
      const float next = __builtin_fmaxf(m - UP, ref), f = ex2(ref - next);
      ref = next;
      sums *= f;
#pragma unroll
      for (int x = 0; x < NF; ++x) o[x] *= f;
    }
  };
  auto weight_pair = [&](const float16v (&x)[2], int v, uint4v (&p)[4]) __attribute__((always_inline)) {
    p[v >> 3][(v & 7) >> 1] = pack2<BF>(ex2(__builtin_fmaf(x[v >> 4][v & 15], a.scale_log2, -ref)), ex2(__builtin_fmaf(x[v >> 4][(v & 15) + 1], a.scale_log2, -ref)));
  };
  auto add_up = [&](const uint4v (&p)[4], int i) __attribute__((always_inline)) {        // the i-th four weights
    sums = add4<BF>(i & 1 ? uint2v{p[i >> 1][2], p[i >> 1][3]} : uint2v{p[i >> 1][0], p[i >> 1][1]}, sums);
  };
  auto weights = [&](const float16v (&x)[2], uint4v (&p)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 32; v += 2) weight_pair(x, v, p);
#pragma unroll
    for (int i = 0; i < 8; ++i) add_up(p, i);
  };
  // clean: values that are not finite count as 0, and are found
  short2v finite = {-1, -1};
  auto products = [&](uint32_t v_at, const uint4v (&p)[4], auto clean) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        uint4v av = value(v_at, i, f);
        if constexpr (decltype(clean)::value) {
          constexpr short E = BF ? 0x7F80 : 0x7C00;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const short2v is = (__builtin_bit_cast(short2v, av[w] & 0x7FFF7FFFu) - short2v{E, E}) >> 15;      // -1 where the exponent is not all ones
            finite &= is;
            av[w] &= __builtin_bit_cast(uint32_t, is);
          }
        }
        o[f] = mfma32<BF>(av, p[i], o[f]);
      }
  };

  // A value that a row does not see must not reach it, and 0 times infinity would: in steps that some row does not see whole, values that are not finite are
  // left out of the products, and added behind the loop to the rows that see them.
  // Stage t & 1 holds what iteration t reads: the values of tile t and the keys of tile t + 1.  An iteration computes the scores of the next tile beside the
  // exponentials of its own (vector instructions in the shadow of the wave's own matrix instructions are nearly free), then its products beside the maxima of the next.
  auto arrive = [&](int t) __attribute__((always_inline)) {
    // what iteration t reads is there, and nobody reads what t - 1 did any more: it makes room for t + 1
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const uint32_t next = lds0 + ((t + 1) & 1) * (2 * TILE);
    if (t + 1 < tiles) issue_v(t + 1, next + TILE);
    if (t + 2 < tiles) issue_k(t + 2, next);
    return (uint32_t)(t & 1) * (2 * TILE);      // (from the beginning of LDS)
  };
  float16v s[2];
  if (tiles > begin) {
    const uint32_t first = (uint32_t)(begin & 1) * (2 * TILE), other = 2 * TILE - first;
    issue_k(begin, lds0 + other);
    issue_v(begin, lds0 + first + TILE);
    if (tiles > begin + 1) issue_k(begin + 1, lds0 + first);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (steps > begin) {
      scores(other, s);
      if (full <= begin) mask(begin, s);
      renew(largest(s));
    }
  }
  int t = begin;
  for (; t + 1 < full; ++t) {              // this tile and the next one are seen whole by every row of the wave
    const uint32_t at = arrive(t);
    // Written out in the order that it runs in: every matrix instruction with the operand that was requested AHEAD instructions before, the request of
    // another, and the vector instructions that fit beside it.
    constexpr int NK = D / 8, NV = 4 * NF, N = NK + NV, AHEAD = 4, PER = 32 / NK, MAXIMA = 16 / NV;
    auto operand = [&](int x) __attribute__((always_inline)) { return x < NK ? key(at + (x & 1) * (64 * D), x >> 1) : value(at + TILE, (x - NK) / NF, (x - NK) % NF); };
    uint4v ring[AHEAD], p[4];
    float16v then[2];
    float m = 0.f;
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) ring[x] = operand(x);
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const uint4v mine = ring[x % AHEAD];
      if (x < NK) then[x & 1] = mfma32<BF>(mine, qf[x >> 1], x < 2 ? (float16v)0.f : then[x & 1]);
      else o[(x - NK) % NF] = mfma32<BF>(mine, p[(x - NK) / NF], o[(x - NK) % NF]);
      if (x + AHEAD < N) ring[x % AHEAD] = operand(x + AHEAD);
      if (x < NK) {
#pragma unroll
        for (int v = x * PER; v < (x + 1) * PER; v += 2) weight_pair(s, v, p);
      } else {
        constexpr int SUMS = 8 * 2 / NV;
        const int y = x - NK;
        if ((y & 1) == 0)
#pragma unroll
          for (int i = y / 2 * SUMS; i < (y / 2 + 1) * SUMS; ++i) add_up(p, i);
#pragma unroll
        for (int v = y * MAXIMA; v < (y + 1) * MAXIMA; ++v) m = v == 0 ? __builtin_fmaxf(then[0][0], then[1][0]) : __builtin_fmaxf(__builtin_fmaxf(m, then[0][v]), then[1][v]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    m = max32(m) * a.scale_log2;
    s[0] = then[0];
    s[1] = then[1];
    renew(m);
  }
  const int t0 = t;
#pragma unroll 1
  for (; t < tiles; ++t) {
    const uint32_t at = arrive(t);
    if (t >= steps) continue;
    uint4v p[4];
    weights(s, p);
    products(at + TILE, p, std::true_type{});
    if (t + 1 < steps) {
      scores(at, s);
      mask(t + 1, s);
      renew(largest(s));
    }
  }
  // In whole tiles they enter the products, with weights that may have fallen to 0 in 16 bits: an element that has seen one is not finite, but may be NaN where the
  // formula gives infinity.  A wave that holds such an element looks through the values of all its tiles, and an element that has seen any gets their sum.
  // (16,384 tokens of 32 heads on 4 of 128: 2.4 ms, with one infinite value 7.5, with NaN everywhere 2.0, with nothing but infinities 230.)
  float l = sum32(sums[0]);
  float4v check = (float4v)0.f;
  if (t0 > begin)
#pragma unroll
    for (int i = 0; i < NF * 16; ++i) check[i & 3] = __builtin_fmaf(o[i >> 4][i & 15], 0.f, check[i & 3]);
  const bool open = l == l;                    // (a row whose sum is NaN is NaN whatever its values are)
  const bool whole = __any(open && check[0] + check[1] + check[2] + check[3] != 0.f);      // (0 or NaN)
  if (__builtin_expect(whole || __any(__builtin_bit_cast(uint32_t, finite) != 0xFFFFFFFFu), 0)) {
    uint32_t spoilt[NF / 2];                // elements to be replaced, 32 of them a word
#pragma unroll
    for (int i = 0; i < NF / 2; ++i) {
      spoilt[i] = 0;
#pragma unroll
      for (int j = 0; j < 32; ++j) spoilt[i] |= is_finite(o[2 * i + (j >> 4)][j & 15]) ? 0u : 1u << j;
    }
    const int upto = any_seen < tiles * BN ? any_seen : tiles * BN;
    for (int j0 = (whole ? begin : t0) * BN; j0 < upto; j0 += RPL) {      // RPL rows at a time, 16 bytes of them a lane
      const int mine = j0 + lane / CH;
      uint4v x = (uint4v)0u;
      if (mine < upto) x = *reinterpret_cast<const uint4v*>(vbase + (int64_t)mine * a.v.token + lane % CH * 16);
      bool strange = false;
#pragma unroll
      for (int w = 0; w < 4; ++w) strange |= !is_finite(low_of<BF>(x[w])) || !is_finite(high_of<BF>(x[w]));
      const uint64_t found = __ballot(strange);
      if (!found) continue;
#pragma unroll 1
      for (int j = j0 + __builtin_ctzll(found) / CH; j <= j0 + (63 - __builtin_clzll(found)) / CH; ++j)
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(vbase + (int64_t)j * a.v.token + 2 * (32 * f + 8 * (r >> 2) + 4 * h + (r & 3)));
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const float value = z ? high_of<BF>(w) : low_of<BF>(w);
              const uint32_t bit = 1u << (16 * (f & 1) + r + z);
              if (j < seen && !is_finite(value)) {
                o[f][r + z] = spoilt[f >> 1] & bit ? value : o[f][r + z] + value;
                spoilt[f >> 1] &= ~bit;
              }
            }
          }
      // NaN stays NaN: nothing is left to be found where every row has come to it
      bool done = true;
#pragma unroll
      for (int i = 0; i < NF * 16; ++i) done = done && o[i >> 4][i & 15] != o[i >> 4][i & 15] && !(spoilt[i >> 5] >> (i & 31) & 1);
      if (__all(done || !open)) break;
    }
  }
  if (x.parts > 1) {
    // The state of a share: its rows' references and sums, then the output before its division, as the lanes hold it.  Written through to memory, since the
    // workgroup that reads it may lie on another XCD; the one that comes last puts all shares together, in their order.  Stores that the compiler knows: it keeps
    // the registers of a store from what overwrites them, which takes two states here, and waits for the matrix instructions.  (Two stores of 8 bytes where one of 16
    // would do: 6 chunks over 3000 keys 54.5 us against 53.5.)
    constexpr int ROWS = NW * 64 * 2, STATE = ROWS + NW * NF * 16 * 64;
    const int64_t next = (int64_t)a.kv_heads * STATE;
    float* const first = a.ws + ((int64_t)x.slot * a.kv_heads + hk) * STATE;
    float* const mine = first + x.part * next;
    const bool used = row0 < rows;               // (waves without rows have no state)
    if (used) {
      put(mine + (wave * 64 + lane) * 2, ref, l);
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float* const to = mine + ROWS + ((wave * NF + f) * 4 + g) * 256 + lane * 4;
          put(to, o[f][4 * g], o[f][4 * g + 1]);
          put(to + 2, o[f][4 * g + 2], o[f][4 * g + 3]);
        }
    }
    // (the wait itself is nothing to the compiler that stores have to stand before)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);          // (vmcnt(0): the state is where every XCD sees it)
    __syncthreads();
    uint32_t* const last = reinterpret_cast<uint32_t*>(lds);
    if (threadIdx.x == 0) {
      uint32_t* const done = a.done + (int64_t)x.slot * a.kv_heads + hk;
      *last = atomicAdd(done, 1u) + 1 == (uint32_t)x.parts;
      if (*last) *done = 0;
    }
    __syncthreads();
    if (!*last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    if (!used) return;
    ref = -3.4028234e38f;
    for (int i = 0; i < x.parts; ++i) ref = __builtin_fmaxf(ref, first[i * next + (wave * 64 + lane) * 2]);
    l = 0.f;
#pragma unroll
    for (int f = 0; f < NF; ++f) o[f] = (float16v)0.f;
    for (int i = 0; i < x.parts; ++i) {
      const float* const from = first + i * next;
      const float2v head = *reinterpret_cast<const float2v*>(from + (wave * 64 + lane) * 2);
      float4v y[NF * 4];
#pragma unroll
      for (int g = 0; g < NF * 4; ++g) y[g] = *reinterpret_cast<const float4v*>(from + ROWS + (wave * NF * 4 + g) * 256 + lane * 4);
      const float scale = __builtin_fmaxf(ex2(head[0] - ref), 1.17549435e-38f);      // (not 0: what is infinite stays so)
      l += scale * head[1];
#pragma unroll
      for (int g = 0; g < NF * 4; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[g >> 2][4 * (g & 3) + r] += scale * y[g][r];
    }
  }
  // (a row that saw nothing but scores of -infinity: infinite values among its elements count for nothing either)
  if (__builtin_expect(l == 0.f, 0))
#pragma unroll
    for (int f = 0; f < NF; ++f) o[f] = (float16v)0.f;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (row >= rows) return;
  char* op = a.o.data + (int64_t)(q0 + query) * a.o.token + (int64_t)head * a.o.head;
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float x0 = o[f][4 * g] * inv, x1 = o[f][4 * g + 1] * inv, x2 = o[f][4 * g + 2] * inv, x3 = o[f][4 * g + 3] * inv;
      const int e = 32 * f + 8 * g + 4 * h;
      if constexpr (F32OUT) *reinterpret_cast<float4v*>(op + 4 * e) = float4v{x0, x1, x2, x3};
      else *reinterpret_cast<uint2v*>(op + 2 * e) = uint2v{pack2<BF>(x0, x1), pack2<BF>(x2, x3)};
    }
}

typedef void (*kernel_fn)(const Args);
template <int D, bool BF> static kernel_fn kernel_of(bool f32) { return f32 ? ftprompt_main<D, BF, true> : ftprompt_main<D, BF, false>; }
constexpr int64_t state_floats(int d) { return NW * 64 * 2 + NW * 32 * d; }

}  // namespace ftprompt

using namespace ftprompt;

struct ftprompt_ctx {
  ftprompt_config cfg;
  kernel_fn fn = nullptr;
  int lds = 0;
  void* scratch = nullptr;       // STATES counters, then as many states
  std::string err;
};

static thread_local std::string g_prompt_create_err;

static int pfail(ftprompt_ctx* c, int code, const char* msg) {
  try {
    (c ? c->err : g_prompt_create_err) = msg;
  } catch (...) {
  }
  return code;
}
static int pfail_hip(ftprompt_ctx* c, const char* what, hipError_t e) {
  try {
    (c ? c->err : g_prompt_create_err) = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return e == hipErrorOutOfMemory ? FTPROMPT_ENOMEM : FTPROMPT_EHIP;
}

extern "C" int ftprompt_create(const ftprompt_config* cfg, ftprompt_ctx** out) {
  if (!cfg || !out) return pfail(nullptr, FTPROMPT_EINVAL, "null argument");
  *out = nullptr;
  if (cfg->struct_size != sizeof(ftprompt_config)) return pfail(nullptr, FTPROMPT_EINVAL, "struct_size mismatch");
  if (cfg->heads < 1 || cfg->kv_heads < 1 || cfg->heads % cfg->kv_heads) return pfail(nullptr, FTPROMPT_EINVAL, "heads must be a positive multiple of kv_heads");
  if (cfg->heads > 65536) return pfail(nullptr, FTPROMPT_EUNSUPPORTED, "more than 65536 heads");
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return pfail(nullptr, FTPROMPT_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (cfg->in_dtype != FTPROMPT_F16 && cfg->in_dtype != FTPROMPT_BF16) return pfail(nullptr, FTPROMPT_EINVAL, "in_dtype must be F16 or BF16");
  if (cfg->out_dtype != FTPROMPT_F32 && cfg->out_dtype != cfg->in_dtype) return pfail(nullptr, FTPROMPT_EINVAL, "out_dtype must be F32 or the input type");
  if (!(std::fabs(cfg->softmax_scale) <= 3.0e38f) || cfg->softmax_scale * LOG2E > 3.4e38f) return pfail(nullptr, FTPROMPT_EINVAL, "softmax_scale is not finite, or too large");
  ftprompt_ctx* c = new (std::nothrow) ftprompt_ctx();
  if (!c) return pfail(nullptr, FTPROMPT_ENOMEM, "out of host memory");
  c->cfg = *cfg;
  if (!(c->cfg.softmax_scale > 0.f)) c->cfg.softmax_scale = 1.0f / std::sqrt((float)cfg->head_dim);
  const bool bf = cfg->in_dtype == FTPROMPT_BF16, f32 = cfg->out_dtype == FTPROMPT_F32;
  c->fn = cfg->head_dim == 128 ? (bf ? kernel_of<128, true>(f32) : kernel_of<128, false>(f32)) : (bf ? kernel_of<64, true>(f32) : kernel_of<64, false>(f32));
  c->lds = cfg->head_dim == 128 ? lds_bytes<128>() : lds_bytes<64>();
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) {
    he = hipFuncSetAttribute((const void*)c->fn, hipFuncAttributeMaxDynamicSharedMemorySize, c->lds);
    if (he == hipSuccess) he = hipMalloc(&c->scratch, STATES * (sizeof(uint32_t) + state_floats(cfg->head_dim) * sizeof(float)));
    if (he == hipSuccess) he = hipMemset(c->scratch, 0, STATES * sizeof(uint32_t));
    if (he == hipSuccess) he = hipDeviceSynchronize();
    if (he != hipSuccess && c->scratch) (void)hipFree(c->scratch);
    (void)hipSetDevice(before);
  }
  if (he != hipSuccess) {
    const int rc = pfail_hip(nullptr, "device", he);
    delete c;
    return rc;
  }
  *out = c;
  return FTPROMPT_OK;
}

extern "C" int ftprompt_get_config(const ftprompt_ctx* ctx, ftprompt_config* effective) {
  if (!ctx || !effective) return FTPROMPT_EINVAL;
  *effective = ctx->cfg;
  return FTPROMPT_OK;
}

extern "C" int ftprompt_forward(ftprompt_ctx* c, const ftprompt_rows* q, const ftprompt_rows* k, const ftprompt_rows* v, const ftprompt_rows* o,
                                const int32_t* cu_q, const int32_t* cu_k, int32_t batch, int32_t total_q, int32_t total_k, void* hip_stream) {
  if (!c) return FTPROMPT_EINVAL;
  if (!q || !k || !v || !o || !cu_q || !cu_k) return pfail(c, FTPROMPT_EINVAL, "null argument");
  if (batch < 1 || total_q < 0 || total_k < 0) return pfail(c, FTPROMPT_EINVAL, "batch must be >= 1 and the totals >= 0");
  const ftprompt_config& e = c->cfg;
  const ftprompt_rows* all[4] = {q, k, v, o};
  Rows r[4];
  for (int i = 0; i < 4; ++i) {
    const int size = i == 3 && e.out_dtype == FTPROMPT_F32 ? 4 : 2, unit = 16 / size;
    const bool none = (i == 1 || i == 2 ? total_k : total_q) == 0;
    if ((!all[i]->data && !none) || ((uintptr_t)all[i]->data & 15)) return pfail(c, FTPROMPT_EINVAL, "tensors must be 16-byte aligned device pointers");
    if (((uintptr_t)all[i]->token_stride | (uintptr_t)all[i]->head_stride) % unit) return pfail(c, FTPROMPT_EINVAL, "strides must be whole 16-byte words");
    if (all[i]->token_stride < 0 || all[i]->head_stride < 0 || all[i]->token_stride > (1 << 24) || all[i]->head_stride > (1ll << 40))
      return pfail(c, FTPROMPT_EUNSUPPORTED, "strides must be >= 0, and those of tokens at most 2^24 elements");
    r[i] = Rows{static_cast<char*>(all[i]->data), all[i]->token_stride * size, all[i]->head_stride * size};
  }
  if (total_q == 0) return FTPROMPT_OK;
  const int group = e.heads / e.kv_heads;
  // A lane of share_of looks after one sequence, so more than MANY are not divided.  With several key heads or rows there are workgroups enough all the same; without, the
  // step shows: sequences of 1 query over 8000 keys, 8 heads on 1 of 128, bf16: 64 of them 55 us, 65 134, 256 212; of 20 queries: 102, 137, 405; on 8 key heads, 32 heads: 379, 504, 1626;
  // of 20 queries over 2000 keys, 8 heads on 1: 43, 43, 118.
  const int32_t divide = total_k > (FEW + FEW / 3) * BN && batch <= MANY;
  // row tiles at most, and as many shares again as they are divided into at most
  const int64_t shares = (int64_t)total_q * group / BM + batch + (divide ? (SHARES + e.kv_heads - 1) / e.kv_heads : 0);
  if ((int64_t)total_q * group > 0x7FFFFF00ll || shares * e.kv_heads > MOST_GROUPS) return pfail(c, FTPROMPT_EUNSUPPORTED, "too many rows");
  Args a{r[0], r[1], r[2], r[3], cu_q, cu_k, batch, total_q, total_k, e.kv_heads, group, divide, e.softmax_scale * LOG2E,
         reinterpret_cast<float*>(static_cast<char*>(c->scratch) + STATES * sizeof(uint32_t)), static_cast<uint32_t*>(c->scratch)};
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess && before != e.device) he = hipSetDevice(e.device);
  if (he != hipSuccess) return pfail_hip(c, "device", he);
  hipLaunchKernelGGL(c->fn, dim3((uint32_t)(shares * e.kv_heads)), dim3(NW * 64), c->lds, (hipStream_t)hip_stream, a);
  he = hipGetLastError();
  if (before != e.device) (void)hipSetDevice(before);
  return he == hipSuccess ? FTPROMPT_OK : pfail_hip(c, "launch", he);
}

extern "C" int ftprompt_destroy(ftprompt_ctx* c) {
  if (!c) return FTPROMPT_OK;
  int before = 0;
  const bool moved = hipGetDevice(&before) == hipSuccess && before != c->cfg.device && hipSetDevice(c->cfg.device) == hipSuccess;
  (void)hipFree(c->scratch);
  if (moved) (void)hipSetDevice(before);
  delete c;
  return FTPROMPT_OK;
}

extern "C" const char* ftprompt_last_error(const ftprompt_ctx* c) { return c ? c->err.c_str() : g_prompt_create_err.c_str(); }
