// Paged key / value cache in 4 bits: the kernels and the C ABI of ../include/ftcache.h.
//
//   ftcache_put     rotates the new tokens' queries and keys, writes both, and puts keys and values into their pages
//   ftcache_get     the reverse of the second half: cached tokens as 16-bit rows
//   ftcache_one     attention of one token per sequence over the cache
//
// Bound of all three: memory.  A token of a key / value head is head_dim + 8 bytes of cache, 136 at head_dim 128 where 16 bits
// would be 512.
#include "ftcache.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>
#include <type_traits>

namespace ftcache {
using namespace ftserve;

struct Rows { char* data; int64_t token, head; };       // strides in bytes

struct Places {
  const int32_t *cu, *starts, *table;
  int64_t table_stride;
  int32_t batch, tokens, width;
};

struct Pool {
  char* data;
  int32_t pages, kv_heads, page_shift;
  int32_t head_bytes;                // of one head of a page
  __device__ __forceinline__ char* head(int page, int hk) const { return data + ((int64_t)page * kv_heads + hk) * head_bytes; }
};

struct Args {
  Pool pool;
  Places at;
  Rows q, k, v, q_out, k_out;
  const float* rotation;
  int32_t positions, heads, rotary;
  unsigned long long* refused;       // [0] tokens, [1] sequences
};

// Tokens of 8 consecutive places of a sequence (a block of the page layout), one of them per lane group of 8.
struct Block {
  int b;                   // sequence
  int place, row;          // of this lane's token; packed row
  bool real;               // the block holds a new token for this lane
  bool whole;              // all 8 places are new tokens (uniform)
  bool sound;              // the sequence does not begin before its first place, nor does the block lie behind the last one
  char* page;              // the page, or nullptr where the table names none
};

// Sequence b owns the blocks from cu[b] / 8 + 2b on, at least as many as n new tokens can touch: (n + 6) / 8 + 1.
__device__ __forceinline__ bool block_of(const Places& p, const Pool& pool, int id, Block& x) {
  auto before = [&](int b) { return (int64_t)(clamped(p.cu[b], p.tokens) / 8 + 2 * b); };
  x.b = sequence_of(p.batch, id, before);
  const int r0 = clamped(p.cu[x.b], p.tokens), r1 = clamped(p.cu[x.b + 1], p.tokens), start = p.starts[x.b];
  const int64_t from = start < 0 ? 0 : start, first = (from / 8 + (id - before(x.b))) * 8;
  if (r1 <= r0 || id < before(x.b) || first >= from + (r1 - r0)) return false;
  const int64_t place = first + ((threadIdx.x & 63) >> 3);
  x.place = (int)place;
  x.real = place >= from && place < from + (r1 - r0);
  x.row = r0 + (int)(place - from);
  x.whole = first >= from && first + 8 <= from + (r1 - r0);
  x.page = nullptr;
  x.sound = start >= 0 && first < 0x7FFFFFF0;
  const int entry = (int)first >> pool.page_shift;
  if (x.sound && entry < p.width) {
    const int page = p.table[x.b * p.table_stride + entry];
    if (page >= 0 && page < pool.pages) x.page = pool.head(page, 0);
  }
  return true;
}


// over the 8 lanes of a token
__device__ __forceinline__ float lanes8(float x, bool largest) {
  auto step = [&](auto moved) { x = largest ? __builtin_fmaxf(x, moved) : __builtin_fminf(x, moved); };
  step(as_f((uint32_t)__builtin_amdgcn_update_dpp((int)as_u(x), (int)as_u(x), 0xB1, 0xF, 0xF, false)));        // lane ^ 1
  step(as_f((uint32_t)__builtin_amdgcn_update_dpp((int)as_u(x), (int)as_u(x), 0x4E, 0xF, 0xF, false)));        // lane ^ 2
  step(as_f((uint32_t)__builtin_amdgcn_update_dpp((int)as_u(x), (int)as_u(x), 0x141, 0xF, 0xF, false)));       // 7 - lane
  return x;
}
__device__ __forceinline__ uint32_t lanes8_max(uint32_t x) {
  auto step = [&](uint32_t moved) { x = moved > x ? moved : x; };
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0xB1, 0xF, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x4E, 0xF, 0xF, false));
  step((uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x141, 0xF, 0xF, false));
  return x;
}

// N elements of a lane, 16-bit, as they lie in memory
template <int N> struct Elements { uint32_t w[N / 2]; };

template <int N> __device__ __forceinline__ Elements<N> load(const char* p) {
  Elements<N> x;
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    const uint4v y = *reinterpret_cast<const uint4v*>(p + 16 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) x.w[4 * i + j] = y[j];
  }
  return x;
}
template <int N> __device__ __forceinline__ void store(char* p, const Elements<N>& x) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i) *reinterpret_cast<uint4v*>(p + 16 * i) = uint4v{x.w[4 * i], x.w[4 * i + 1], x.w[4 * i + 2], x.w[4 * i + 3]};
}

// The rotation of a lane's elements e0 .. e0 + N of a token, in chunks of 8: cosines and sines, which are the same for every head.  Halves: an element
// and its partner rotary/2 away, sines with the sign that the element's product with its partner has.  Pairs: elements side by side, four of each in a chunk.
template <int N, bool PAIRS> struct Turn {
  static constexpr int PER = PAIRS ? 4 : 8;
  float c[N / 8 * PER], s[N / 8 * PER];
  int partner[N / 8];      // bytes from the chunk to its partners
  bool turned[N / 8];
};
template <int N, bool PAIRS> __device__ __forceinline__ void turn_of(Turn<N, PAIRS>& t, const float* row, int e0, int rotary) {
  const int half = rotary / 2;
  constexpr int PER = Turn<N, PAIRS>::PER;
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    const int e = e0 + 8 * i;
    const bool first = e < half;
    t.turned[i] = e < rotary;
    t.partner[i] = PAIRS || !t.turned[i] ? 0 : first ? 2 * half : -2 * half;
    const int at = !t.turned[i] ? 0 : PAIRS ? e / 2 : first ? e : e - half;
#pragma unroll
    for (int j = 0; j < PER; j += 4) {
      const float4v c = *reinterpret_cast<const float4v*>(row + at + j), s = *reinterpret_cast<const float4v*>(row + half + at + j);
#pragma unroll
      for (int x = 0; x < 4; ++x) { t.c[PER * i + j + x] = c[x]; t.s[PER * i + j + x] = !PAIRS && first ? -s[x] : s[x]; }
    }
  }
}

// What a rotation reads: the lane's elements, and their partners (every lane of a token has read them before any stores).
template <int N, bool PAIRS> struct Loaded2 {
  Elements<N> x, partners;
};
template <int N, bool PAIRS> __device__ __forceinline__ Loaded2<N, PAIRS> load(const char* p, const Turn<N, PAIRS>& t) {
  Loaded2<N, PAIRS> y;
  y.x = load<N>(p);
  if constexpr (!PAIRS) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const uint4v z = *reinterpret_cast<const uint4v*>(p + 16 * i + t.partner[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) y.partners.w[4 * i + j] = z[j];
    }
  }
  return y;
}
template <int N, bool BF, bool PAIRS> __device__ __forceinline__ Elements<N> rotated(const Loaded2<N, PAIRS>& in, const Turn<N, PAIRS>& t) {
#pragma clang fp contract(off)
  Elements<N> y;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const uint32_t w = in.x.w[i];
    const float a = low_of<BF>(w), b = high_of<BF>(w);
    float u, v;
    if constexpr (PAIRS) {
      const float c = t.c[i], s = t.s[i];
      u = a * c - b * s;
      v = b * c + a * s;
    } else {
      const uint32_t z = in.partners.w[i];
      u = a * t.c[2 * i] + low_of<BF>(z) * t.s[2 * i];
      v = b * t.c[2 * i + 1] + high_of<BF>(z) * t.s[2 * i + 1];
    }
    y.w[i] = t.turned[i / 4] ? pack2<BF>(u, v) : w;
  }
  return y;
}

template <int N> struct Codes { uint32_t w[N / 8]; uint32_t params; };      // 8 codes a word, lowest bits first; scale and minimum (in_dtype)

template <int N, bool BF> __device__ __forceinline__ Codes<N> coded(const Elements<N>& x) {
#pragma clang fp contract(off)
  Codes<N> r;
  float lo = low_of<BF>(x.w[0]), hi = lo;
  ushort2v most = {0, 0};
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float a = low_of<BF>(x.w[i]), b = high_of<BF>(x.w[i]);
    lo = __builtin_fminf(lo, __builtin_fminf(a, b));
    hi = __builtin_fmaxf(hi, __builtin_fmaxf(a, b));
    most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, x.w[i] & 0x7FFF7FFFu));
  }
  lo = lanes8(lo, false);
  hi = lanes8(hi, true);
  const uint32_t top = lanes8_max(most[0] > most[1] ? most[0] : most[1]);
  const bool fine = top < largest_finite_plus_one<BF>();
  const uint32_t params = pack2<BF>(hi / 15.f - lo / 15.f, lo);
  const float step = low_of<BF>(params) * 0.5f, base = lo * 0.5f;
  r.params = fine ? params : 0x7FFF7FFFu;
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float e = j & 1 ? high_of<BF>(x.w[4 * i + j / 2]) : low_of<BF>(x.w[4 * i + j / 2]);
      const float c = __builtin_rintf((e * 0.5f - base) / step);
      w |= (uint32_t)__builtin_fminf(__builtin_fmaxf(c, 0.f), 15.f) << (4 * j);
    }
    r.w[i] = fine && step != 0.f ? w : 0u;
  }
  return r;
}

// A wave takes 8 places of a sequence, two query heads, or the key and value of a head, at a time: lane 8t + c has elements c * D/8 .. of token t.
// Bound by memory: 20,278 tokens of 32 + 8 heads of 128 in 101 us, 484 MB at 4.8 TB/s (a copy reaches 4.9); with one head at a time and its partners' sign by
// branches it took 147.
template <int D, bool BF, bool PAIRS>
__global__ __launch_bounds__(256) void ftcache_put(const Args a) {
  constexpr int N = D / 8;
  __shared__ uint16_t turned[4][D / 4][8];            // value codes of 8 tokens, to be written 16 bytes at a time
  Block x;
  if (!block_of(a.at, a.pool, blockIdx.x, x)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane >> 3, c = lane & 7, e0 = c * N;
  const bool known = x.sound && x.place < a.positions, kept = x.real && known && x.page;
  if (blockIdx.y == 0 && wave == 0) {
    const uint64_t refused = __ballot(x.real && !kept && c == 0);
    if (refused && lane == 0) atomicAdd(a.refused, (unsigned long long)__popcll(refused));
  }
  const bool whole = x.whole && __all(kept);
  Turn<N, PAIRS> turn;
  turn_of<N, PAIRS>(turn, a.rotation + (int64_t)(known ? x.place : 0) * a.rotary, e0, a.rotary);
  const int kv = a.pool.kv_heads, step = gridDim.y * 4;
  // heads of keys and values first: they take longer
  const int64_t row = x.real ? x.row : 0;
  auto finish = [&](Elements<N> y, char* out, bool store_it) __attribute__((always_inline)) {
    if (!known)
#pragma unroll
      for (int i = 0; i < N / 2; ++i) y.w[i] = 0x7FFF7FFFu;
    if (store_it && x.real) store<N>(out, y);
    return y;
  };
  const int ps = 1 << a.pool.page_shift, in_page = x.place & (ps - 1);
  const char* const krow = a.k.data + row * a.k.token + 2 * e0;
  const char* const vrow = a.v.data + row * a.v.token + 2 * e0;
  char* const kout = a.k_out.data + row * a.k_out.token + 2 * e0;
  int item = blockIdx.y * 4 + wave;
  for (; item < kv; item += step) {
    // (a lane without a token reads the first row: a call has one)
    const Loaded2<N, PAIRS> in = load<N, PAIRS>(krow + item * a.k.head, turn);
    const Elements<N> v = load<N>(vrow + item * a.v.head);
    const Elements<N> k = finish(rotated<N, BF, PAIRS>(in, turn), kout + item * a.k_out.head, a.k_out.data != nullptr);
    const Codes<N> zk = coded<N, BF>(k), zv = coded<N, BF>(v);
    char* const page = x.page + (int64_t)item * a.pool.head_bytes;      // (used where kept only)
    if (kept) {
      if (c == 0) {
        uint16_t* par = reinterpret_cast<uint16_t*>(page + ps * D) + (in_page >> 3) * 32 + t;
        par[0] = (uint16_t)zk.params;
        par[8] = (uint16_t)(zk.params >> 16);
        par[16] = (uint16_t)zv.params;
        par[24] = (uint16_t)(zv.params >> 16);
      }
      if constexpr (N == 16) *reinterpret_cast<uint2v*>(page + in_page * (D / 2) + e0 / 2) = uint2v{zk.w[0], zk.w[1]};
      else *reinterpret_cast<uint32_t*>(page + in_page * (D / 2) + e0 / 2) = zk.w[0];
    }
    char* const block = page + ps * (D / 2) + (in_page >> 3) * (4 * D);
    if (whole) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) turned[wave][c * (N / 4) + i][t] = (uint16_t)(zv.w[i / 2] >> (16 * (i & 1)));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (lane < D / 4) *reinterpret_cast<uint4v*>(block + lane * 16) = *reinterpret_cast<const uint4v*>(turned[wave][lane]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else if (kept) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i)
        *reinterpret_cast<uint16_t*>(block + (c * (N / 4) + i) * 16 + t * 2) = (uint16_t)(zv.w[i / 2] >> (16 * (i & 1)));
    }
  }
  if (!a.q.data) return;
  const char* const qrow = a.q.data + row * a.q.token + 2 * e0;
  char* const qout = a.q_out.data + row * a.q_out.token + 2 * e0;
  for (item -= kv; item < a.heads; item += 2 * step) {
    const int64_t other = item + step < a.heads ? item + step : item;
    const Loaded2<N, PAIRS> in = load<N, PAIRS>(qrow + item * a.q.head, turn), in2 = load<N, PAIRS>(qrow + other * a.q.head, turn);
    finish(rotated<N, BF, PAIRS>(in, turn), qout + item * a.q_out.head, true);
    if (other != item) finish(rotated<N, BF, PAIRS>(in2, turn), qout + other * a.q_out.head, true);
  }
}

// the type's finite numbers: a scale that was rounded up can take the largest code of the largest element beyond them (NaN stays)
template <bool BF> constexpr float LARGEST = BF ? 3.38953139e38f : 65504.f;
template <bool BF> __device__ __forceinline__ float held(float x) {
  constexpr float top = LARGEST<BF>;
  return x > top ? top : x < -top ? -top : x;
}

template <int D, bool BF>
__global__ __launch_bounds__(256) void ftcache_get(const Args a) {
#pragma clang fp contract(off)
  constexpr int N = D / 8;
  Block x;
  if (!block_of(a.at, a.pool, blockIdx.x, x)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = lane >> 3, c = lane & 7, e0 = c * N;
  if (blockIdx.y == 0 && wave == 0 && !x.page) {
    const uint64_t refused = __ballot(x.real && c == 0);
    if (refused && lane == 0) atomicAdd(a.refused, (unsigned long long)__popcll(refused));
  }
  if (!x.real) return;
  const int kv = a.pool.kv_heads, in_page = x.place & ((1 << a.pool.page_shift) - 1), ps = 1 << a.pool.page_shift;
  for (int item = blockIdx.y * 4 + wave; item < 2 * kv; item += gridDim.y * 4) {
    const bool is_v = item >= kv;
    const int head = is_v ? item - kv : item;
    Elements<N> y;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) y.w[i] = 0x7FFF7FFFu;
    if (x.page) {
      const char* const page = x.page + (int64_t)head * a.pool.head_bytes;
      uint32_t w[N / 8];
      if (is_v) {
        const char* const block = page + ps * (D / 2) + (in_page >> 3) * (4 * D) + t * 2;
#pragma unroll
        for (int i = 0; i < N / 8; ++i)
          w[i] = (uint32_t)*reinterpret_cast<const uint16_t*>(block + (c * (N / 4) + 2 * i) * 16) |
                 (uint32_t)*reinterpret_cast<const uint16_t*>(block + (c * (N / 4) + 2 * i + 1) * 16) << 16;
      } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) w[i] = *reinterpret_cast<const uint32_t*>(page + in_page * (D / 2) + e0 / 2 + 4 * i);
      }
      const uint16_t* par = reinterpret_cast<const uint16_t*>(page + ps * D) + (in_page >> 3) * 32 + (is_v ? 16 : 0) + t;
      const float scale = low_of<BF>(par[0]), low = low_of<BF>(par[8]);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const uint32_t v = w[i / 4] >> (8 * (i & 3));
        y.w[i] = pack2<BF>(held<BF>((float)(v & 15) * scale + low), held<BF>((float)(v >> 4 & 15) * scale + low));
      }
    }
    const Rows& out = is_v ? a.v : a.k;
    store<N>(out.data + (int64_t)x.row * out.token + (int64_t)head * out.head + 2 * e0, y);
  }
}

// ------------------------------------------------------------------ attention of single tokens
//
// The query heads of a group are rows of the matrix instructions (16 a pass): scores transposed, S^T = K q^T with 16x16x32, keys down and
// heads across, so that lane l owns row l % 16 and, of a step of 32 tokens, the 8 tokens 8g .. 8g + 7 (g = l / 16) whose weights are its
// operand of O^T = V^T P^T as they lie.  Neither codes nor weights pass through LDS.
//
// Codes enter the products as they are.  A key code's bits alone are the number c * 2^-24 in fp16, c * 2^-133 in bf16 (and 16 c of them four
// bits higher): subnormal or next to it, which the matrix instructions take like any other, and one AND gives two of them.  The query's row is scaled up by a
// power of two, which the score loses again.  Value codes lie under the bits of 128 in bf16, 128 + c; the offset leaves through the sum of the weights.
// Scale and minimum of a token are applied to its scores and to its weights, in 32 bits:
//     score = ks (q . c) + kz (sum q),   O = sum (p vs) (c' - 8) + sum p (vz + 8 vs)
// (about the middle of the codes, so that rounding p vs costs half of what it would).  Bound: loads under way where there is enough to read, 1.25 M tokens of 96 sequences,
// 32 heads on 8 of 128, 1.36 GB in 266 us: 5.1 TB/s, where a kernel that does nothing but read reaches 7.1 (waves wait for 63 % of their time; vector instructions take
// half of the cycles, the matrix pipe 13 %).  Below that the start of a piece (3 us) and putting parts together (3 us a level): 131,072
// tokens of one sequence 23 us, 35,000 of 32 sequences 16.  Three workgroups of four waves to a CU; two, by
// more registers, took 314 us for the first, four, with registers spilled, 384.
struct OneArgs {
  Pool pool;
  Rows q, o;
  const int32_t *lengths, *table;
  int64_t table_stride;
  int32_t batch, most, group, row_tiles;        // most: tokens that a row of the table holds; row_tiles: passes of 16 heads for a group
  int32_t chunks, one_round, most_parts;        // pieces over all sequences: at most about, at a time; at most of one
  float scale_log2;
  float* ws;                                    // states of divided sequences
  uint32_t* done;                               // [level][state]: parts that are there, and behind the last level whether a sequence has been refused; 0 between calls
  int64_t done_level;
  unsigned long long* refused;
};

constexpr int ONE_WAVES = 4, ONE_STEP = 32, ONE_UNIT = ONE_WAVES * ONE_STEP;      // tokens of a step of a wave, of a workgroup
constexpr int CUS = 256, ONE_GROUPS = 8 * CUS, ROUND = 3 * CUS;      // workgroups that a call is divided among (more where sequences are many), and that fit side by side
constexpr int SPLIT_TO = 4 * CUS;                    // workgroups of append and read, where heads give as many
constexpr int MOST_PARTS = 2 * CUS, JOIN = 16, LEVELS = 3;      // of one sequence, where there is one head; put together at a time
static_assert(JOIN * JOIN * JOIN >= MOST_PARTS, "levels");
constexpr int LONG = 8, SOME = 6;                    // units of a piece, see piece_of
constexpr int SHORT = 8;                             // units of a sequence that is not divided: joining two parts takes about 3 us, the time of some steps

template <bool BF> __device__ __forceinline__ float4v mfma16(uint4v a, uint4v b, float4v c) {
  if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// 8 codes of a word as an operand: words (c0, c4), (16 c1, 16 c5), (c2, c6), (16 c3, 16 c7)
__device__ __forceinline__ uint4v key_operand(uint32_t w) {
  const uint32_t u = w >> 8;
  return uint4v{w & 0x000F000Fu, w & 0x00F000F0u, u & 0x000F000Fu, u & 0x00F000F0u};
}
// (bits128: those of 128, twice, in a vector register: with two constants it is an AND and an OR)
__device__ __forceinline__ uint32_t value_codes(uint32_t w, uint32_t bits128) { return (w & 0x000F000Fu) | bits128; }

// sum over the lanes up to this one: register moves within rows of 16 lanes, then from row to row
__device__ __forceinline__ int sum_upto(int x) {
  auto step = [&](int moved) { x += moved; };
  step(__builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));      // row_shr 1, 2, 4, 8
  step(__builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));      // row_bcast 15, 31
  step(__builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
  return x;
}

__device__ __forceinline__ int max_upto(int x) {      // of values >= 0
  auto step = [&](int moved) { x = moved > x ? moved : x; };
  step(__builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));
  step(__builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
  return x;
}

struct Piece { int b, first, count, part, parts, slot; };      // tokens first .. first + count of sequence b, part of parts; place of part 0's state

// Sequences are divided into pieces of one length, the same for all, chosen so that there are about `chunks` pieces in all: the last of a sequence is
// shorter.  Lengths count in units of ONE_UNIT tokens (all of them together below 2^31, see ftcache_attend).  A wave looks at 64 sequences at a time.
__device__ __forceinline__ bool piece_of(const OneArgs& a, int id, Piece& p, bool& known) {
  const int lane = threadIdx.x & 63, most = a.most;
  auto length = [&](int b) { return b < a.batch ? a.lengths[b] : 0; };
  auto sound = [&](int n) { return n < 0 || n > most ? 0 : n; };
  auto units = [&](int n) { return (int)(((uint32_t)sound(n) + ONE_UNIT - 1) / ONE_UNIT); };
  const int mine = length(lane);
  int total = units(mine), longest = total;
#pragma unroll 4
  for (int b = lane + 64; b < a.batch; b += 64) {
    const int u = units(a.lengths[b]);
    total += u;
    longest = u > longest ? u : longest;
  }
  total = __builtin_amdgcn_readlane(sum_upto(total), 63);
  longest = __builtin_amdgcn_readlane(max_upto(longest), 63);
  // Pieces that leave every CU several are best where there is enough to read (1.25 M tokens of 96 sequences and 8 heads: 297 us in 3 workgroups a CU,
  // 265 in 8), one round of what fits side by side where there is not (35,000 tokens of 32: 15.9 us in 3, 17.4 in 8), and few enough parts to be put together
  // at once where that makes them no longer than some steps (4 sequences of 8000: 18.0 us with more than 16 parts, 13.7 with 16).
  auto of = [&](int n, int chunks) { return (n + chunks - 1) / chunks; };
  auto larger = [](int x, int y) { return x > y ? x : y; };
  auto smaller = [](int x, int y) { return x < y ? x : y; };
  const int size = larger(larger(larger(of(total, a.chunks), of(longest, a.most_parts)), 1), larger(smaller(of(total, a.one_round), LONG), smaller(of(longest, JOIN), SOME)));
  auto parts_of = [&](int n) { const int u = units(n); return u > size && u > SHORT ? (u + size - 1) / size : 1; };
  int slot = 0;                       // states of the divided sequences so far
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int n = b0 ? length(b0 + lane) : mine, parts = b0 + lane < a.batch ? parts_of(n) : 0, states = parts > 1 ? parts : 0;
    const int upto = sum_upto(parts), states_upto = sum_upto(states), all = __builtin_amdgcn_readlane(upto, 63);
    if (id >= all) {
      id -= all;
      slot += __builtin_amdgcn_readlane(states_upto, 63);
      continue;
    }
    const int owner = __ffsll((unsigned long long)__ballot(upto > id)) - 1;
    auto from_owner = [&](int v) { return __builtin_amdgcn_readlane(v, owner); };
    const int raw = from_owner(n), part = id - from_owner(upto - parts), count = from_owner(parts), first = part * size * ONE_UNIT, rest = sound(raw) - first;
    known = raw == sound(raw);
    p = Piece{b0 + owner, first, count == 1 || rest < size * ONE_UNIT ? rest : size * ONE_UNIT, part, count, slot + from_owner(states_upto - states)};
    return true;
  }
  return false;
}

// What a piece leaves of its 16 rows: reference and sum of weights of each, then the output before its division.
template <int D> constexpr int STATE = 16 * 2 + 16 * D;

// States go from workgroup to workgroup, whose XCDs may differ, past the L2 caches: written through to memory, and read behind an
// invalidation by the one workgroup that reads them.  (A fence for the whole device writes back an L2 at a time: with one in every workgroup 35,000 tokens of
// 32 sequences took 94 us.)
__device__ __forceinline__ void put_state(float* p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)as_u(a) | (uint64_t)as_u(b) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// What a wave has loaded of a step: two tokens' key codes a lane, the value codes of its 8 tokens, and one of the 16 words of their parameters.
template <int D> struct Loaded {
  uint32_t k[2][D / 32];
  uint4v v[D / 64];
  uint32_t par;
};
// what lane I of each 16 holds: part of the instruction that uses it
template <int I> __device__ __forceinline__ float of_lane(float x) { return as_f((uint32_t)__builtin_amdgcn_mov_dpp((int)as_u(x), 0x150 + I, 0xF, 0xF, true)); }

template <int D, bool BF, bool F32OUT>
__global__ __launch_bounds__(ONE_WAVES * 64, 3) void ftcache_one(const OneArgs a) {
  constexpr int KW = D / 32;              // words of key codes per lane and token = matrix instructions over the head
  constexpr int NO = D / 16;              // accumulators of the output
  constexpr int THREADS = ONE_WAVES * 64;
  constexpr int PITCH = D + 4;
  __shared__ __attribute__((aligned(16))) float merged[ONE_WAVES * 16 * PITCH];      // the waves' outputs
  __shared__ float refs[ONE_WAVES][16], sums[ONE_WAVES][16];
  __shared__ int last, wrong[ONE_WAVES];
  const int heads = a.pool.kv_heads * a.row_tiles, hr = blockIdx.x % heads, hk = hr / a.row_tiles, tile = hr % a.row_tiles;
  Piece p;
  bool known;
  if (!piece_of(a, blockIdx.x / heads, p, known)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, n = lane & 15;
  const int rows = a.group - 16 * tile < 16 ? a.group - 16 * tile : 16, head0 = hk * a.group + 16 * tile;

  // the row's query as an operand, scaled by a power of two so that its largest element lies in [2^10, 2^11) (fp16), at 2^126 or as far up as one
  // factor brings it (bf16): the products with codes are then far from both ends of 32 bits, and sixteenths of small elements keep their bits
  uint4v qf[KW];
  float alpha, qsum;       // what a score of products with codes still lacks; the sum of the query's elements, in the same measure
  {
    const char* qp = a.q.data + (int64_t)p.b * a.q.token + (int64_t)(head0 + (n < rows ? n : 0)) * a.q.head + 2 * (8 * KW * g);
    uint32_t w[4 * KW];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < KW; ++i) {
      const uint4v y = *reinterpret_cast<const uint4v*>(qp + 16 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[4 * i + j] = y[j];
        const uint32_t lo = as_u(low_of<BF>(y[j])) & 0x7FFFFFFFu, hi = as_u(high_of<BF>(y[j])) & 0x7FFFFFFFu;
        most = lo > most ? lo : most;
        most = hi > most ? hi : most;
      }
    }
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) { const uint32_t x = __shfl_xor(most, d); most = x > most ? x : most; }
    const int e = (int)(most >> 23) - 127;
    int up_by = (BF ? 126 : 10) - e;
    up_by = up_by > 126 ? 126 : up_by < -126 ? -126 : up_by;
    const float up = as_f((uint32_t)(127 + up_by) << 23);
    float plain = 0.f;
#pragma unroll
    for (int i = 0; i < KW; ++i) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        plain += low_of<BF>(w[4 * i + j]);
        plain += high_of<BF>(w[4 * i + j]);
        f[2 * j] = low_of<BF>(w[4 * i + j]) * up;
        f[2 * j + 1] = high_of<BF>(w[4 * i + j]) * up;
      }
      const float odd = 0.0625f;
      qf[i] = uint4v{pack2<BF>(f[0], f[4]), pack2<BF>(f[1] * odd, f[5] * odd), pack2<BF>(f[2], f[6]), pack2<BF>(f[3] * odd, f[7] * odd)};
    }
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) plain += __shfl_xor(plain, d);
    alpha = __builtin_ldexpf(a.scale_log2, (BF ? 133 : 24) - up_by);
    qsum = __builtin_ldexpf(plain, up_by - (BF ? 133 : 24));
  }

  float4v o[NO], ones = (float4v)0.f;
#pragma unroll
  for (int i = 0; i < NO; ++i) o[i] = (float4v)0.f;
  float ref = -3.4028234e38f, l = 0.f, z = 0.f;
  bool bad = !known;
  uint32_t bits128 = 0x43004300u;
  asm("" : "+v"(bits128));
  const int ps = 1 << a.pool.page_shift, end = p.first + p.count;
  const int32_t* const table = a.table + p.b * a.table_stride;
  // entries of the table for the blocks of 8 tokens that a lane reads in a step, keys' and values' (the last block's behind the end)
  struct Entries { uint32_t k, v; };
  const int last_block = (end - 1) & ~7, my_k = 8 * (n >> 2), my_v = 8 * g;
  const char* const kpool = a.pool.head(0, hk) + (n & 3) * (D / 2) + g * (4 * KW);
  const char* const vpool = a.pool.head(0, hk) + ps * (D / 2) + n * (D / 4);
  const char* const ppool = a.pool.head(0, hk) + ps * D + 4 * n;
  const uint32_t page_bytes = (uint32_t)a.pool.kv_heads * (uint32_t)a.pool.head_bytes, in_page = (uint32_t)ps - 1, pages = (uint32_t)a.pool.pages;
  uint32_t highest = 0;                   // entry met
  auto block = [&](int t) { return t < last_block ? t : last_block; };
  auto entries_of = [&](int t0) {
    return Entries{(uint32_t)table[block(t0 + my_k) >> a.pool.page_shift], (uint32_t)table[block(t0 + my_v) >> a.pool.page_shift]};
  };
  auto page_at = [&](uint32_t entry) {
    highest = entry > highest ? entry : highest;
    return (uint64_t)(entry < pages ? entry : pages - 1) * page_bytes;
  };
  auto load = [&](int t0, Entries at) {
    Loaded<D> x;
    const uint64_t kpage = page_at(at.k), vpage = page_at(at.v);
    const uint32_t kin = (uint32_t)block(t0 + my_k) & in_page, vin = (uint32_t)block(t0 + my_v) & in_page;
    const char* const kp = kpool + (kpage + kin * (D / 2));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (KW == 4) { const uint4v y = *reinterpret_cast<const uint4v*>(kp + t * (2 * D)); x.k[t][0] = y[0]; x.k[t][1] = y[1]; x.k[t][2] = y[2]; x.k[t][3] = y[3]; }
      else { const uint2v y = *reinterpret_cast<const uint2v*>(kp + t * (2 * D)); x.k[t][0] = y[0]; x.k[t][1] = y[1]; }
    }
    const char* const vp = vpool + (vpage + vin * (D / 2));
#pragma unroll
    for (int i = 0; i < D / 64; ++i) x.v[i] = *reinterpret_cast<const uint4v*>(vp + 16 * i);
    x.par = *reinterpret_cast<const uint32_t*>(ppool + (vpage + vin * 8));
    return x;
  };
  // The reference lies DOWN above the largest score that it was made from, and weights reach 2^(8 - DOWN).  bf16: a weight times its value's scale meets 128 + c, up to
  // 143 of 15 steps that span at most twice the largest |v|; at 2^-5 of weight their sums stay finite where those of the formula do.
  constexpr float DOWN = BF ? 13.f : 0.f;
  auto step = [&](int t0, const Loaded<D>& y) __attribute__((always_inline)) {
    float4v s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = (float4v)0.f;
#pragma unroll
      for (int i = 0; i < KW; ++i) s[t] = mfma16<BF>(key_operand(y.k[t][i]), qf[i], s[t]);
    }
    // scores before softmax_scale * log2(e), from the words that the 16 lanes of a block hold together
    float x[8];
    const float plo = low_of<BF>(y.par), phi = high_of<BF>(y.par);
    auto scores = [&](auto i) __attribute__((always_inline)) {            // tokens 2i and 2i + 1
      constexpr int I = decltype(i)::value;
      x[2 * I] = __builtin_fmaf(of_lane<I>(plo), s[I >> 1][2 * (I & 1)], of_lane<4 + I>(plo) * qsum);
      x[2 * I + 1] = __builtin_fmaf(of_lane<I>(phi), s[I >> 1][2 * (I & 1) + 1], of_lane<4 + I>(phi) * qsum);
    };
    scores(std::integral_constant<int, 0>{});
    scores(std::integral_constant<int, 1>{});
    scores(std::integral_constant<int, 2>{});
    scores(std::integral_constant<int, 3>{});
    float vlo = plo, vhi = phi;
    if (t0 + ONE_STEP > end) {
      asm volatile("; the last step of a sequence");         // (a branch, not selections in every step)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (t0 + 8 * g + j >= end) x[j] = -__builtin_inff();
      // scales and minima of values behind the end
      if (t0 + 8 * g + 2 * (n & 3) >= end) vlo = 0.f;
      if (t0 + 8 * g + 2 * (n & 3) + 1 >= end) vhi = 0.f;
    }
    float m = __builtin_fmaxf(x[0], x[1]);
#pragma unroll
    for (int j = 2; j < 8; ++j) m = __builtin_fmaxf(m, x[j]);
    m *= alpha;
    if (__any(m > ref + (8.f - DOWN))) {
      m = __builtin_fmaxf(m, __shfl_xor(m, 16));
      m = __builtin_fmaxf(m, __shfl_xor(m, 32));
      const float next = __builtin_fmaxf(m + DOWN, ref), f = ex2(ref - next);
      ref = next;
      l *= f;
      z *= f;
      ones *= f;
#pragma unroll
      for (int i = 0; i < NO; ++i) o[i] *= f;
    }
    float w[8];
    auto weights = [&](auto i) __attribute__((always_inline)) {
      constexpr int I = decltype(i)::value;
      const float e0 = ex2(__builtin_fmaf(x[2 * I], alpha, -ref)), e1 = ex2(__builtin_fmaf(x[2 * I + 1], alpha, -ref));
      l += e0;
      l += e1;
      z = __builtin_fmaf(of_lane<12 + I>(vlo), e0, z);
      z = __builtin_fmaf(of_lane<12 + I>(vhi), e1, z);
      w[2 * I] = of_lane<8 + I>(vlo) * e0;
      w[2 * I + 1] = of_lane<8 + I>(vhi) * e1;
      z = __builtin_fmaf(w[2 * I], 8.f, z);
      z = __builtin_fmaf(w[2 * I + 1], 8.f, z);
    };
    weights(std::integral_constant<int, 0>{});
    weights(std::integral_constant<int, 1>{});
    weights(std::integral_constant<int, 2>{});
    weights(std::integral_constant<int, 3>{});
    // weights in bf16; for fp16 tokens in two words, the second what the first leaves, so that they are no coarser than the tokens
    // (for bf16 tokens two would bring the error from 2.3e-3 to that of the rounded result, 1.7e-3, in 1.5 to 9 % more time)
    uint4v ph, pl;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      ph[j] = pack2<true>(w[2 * j], w[2 * j + 1]);
      if constexpr (!BF) pl[j] = pack2<true>(w[2 * j] - low_of<true>(ph[j]), w[2 * j + 1] - high_of<true>(ph[j]));
    }
    const uint4v one = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    ones = mfma16<true>(one, ph, ones);
    if constexpr (!BF) ones = mfma16<true>(one, pl, ones);
#pragma unroll
    for (int i = 0; i < NO; ++i) {
      const uint4v v = y.v[i / 4];
      const int by = 4 * (i & 3);
      const uint4v c = {value_codes(v[0] >> by, bits128), value_codes(v[1] >> by, bits128), value_codes(v[2] >> by, bits128), value_codes(v[3] >> by, bits128)};
      o[i] = mfma16<true>(c, ph, o[i]);
      if constexpr (!BF) o[i] = mfma16<true>(c, pl, o[i]);
    }
  };
  // the loads of the next AHEAD steps are under way while a step is computed, and the entries of the one after those
  constexpr int AHEAD = 1;
  const int t0 = p.first + wave * ONE_STEP;
  if (t0 < end) {
    Loaded<D> ring[AHEAD + 1];
    Entries next = entries_of(t0);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (t0 + i * ONE_UNIT < end) ring[i] = load(t0 + i * ONE_UNIT, next);
      next = entries_of(t0 + (i + 1) * ONE_UNIT);
    }
    for (int t = t0; t < end;) {
#pragma unroll
      for (int i = 0; i <= AHEAD; ++i) {
        if (t + AHEAD * ONE_UNIT < end) ring[(i + AHEAD) % (AHEAD + 1)] = load(t + AHEAD * ONE_UNIT, next);
        next = entries_of(t + (AHEAD + 1) * ONE_UNIT);
        __builtin_amdgcn_sched_barrier(0);
        step(t, ring[i]);
        t += ONE_UNIT;
        if (t >= end) break;
      }
    }
  }
  bad = __any(bad || highest >= pages);
#pragma unroll
  for (int d = 16; d < 64; d <<= 1) { l += __shfl_xor(l, d); z += __shfl_xor(z, d); }
  const float shift = z - 136.f * ones[0];
  if (bad) l = __builtin_nanf("");
  if (g == 0) { refs[wave][n] = ref; sums[wave][n] = l; }
  if (lane == 0) wrong[wave] = bad;
#pragma unroll
  for (int i = 0; i < NO; ++i)
#pragma unroll
    for (int v = 0; v < 4; ++v) merged[(wave * 16 + n) * PITCH + (4 * g + v) * NO + i] = o[i][v] + shift;
  __syncthreads();

  const int tid = threadIdx.x;
  auto finish = [&](int row, int e, float4v value, float sum) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    char* op = a.o.data + (int64_t)p.b * a.o.token + (int64_t)(head0 + row) * a.o.head;
    value *= inv;
    if constexpr (F32OUT) *reinterpret_cast<float4v*>(op + 4 * e) = value;
    else {
      const float most = __builtin_fmaxf(__builtin_fmaxf(__builtin_fabsf(value[0]), __builtin_fabsf(value[1])), __builtin_fmaxf(__builtin_fabsf(value[2]), __builtin_fabsf(value[3])));
      if (__builtin_expect(__any(most > LARGEST<BF>), 0))      // (as values read back are held; rare)
        value = float4v{held<BF>(value[0]), held<BF>(value[1]), held<BF>(value[2]), held<BF>(value[3])};
      *reinterpret_cast<uint2v*>(op + 2 * e) = uint2v{pack2<BF>(value[0], value[1]), pack2<BF>(value[2], value[3])};
    }
  };
  constexpr int CD = D / 4;               // columns of four elements of a row
  for (int x = tid; x < rows * CD; x += THREADS) {
    const int row = x / CD, e = x % CD * 4;
    float most = refs[0][row];
#pragma unroll
    for (int w = 1; w < ONE_WAVES; ++w) most = __builtin_fmaxf(most, refs[w][row]);
    float4v value = (float4v)0.f;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < ONE_WAVES; ++w) {
      const float f = ex2(refs[w][row] - most);
      value += f * *reinterpret_cast<const float4v*>(&merged[(w * 16 + row) * PITCH + e]);
      sum += f * sums[w][row];
    }
    if (p.parts == 1) finish(row, e, value, sum);
    else {
      float* const ws = a.ws + ((int64_t)(p.slot + p.part) * heads + hr) * STATE<D>;
      put_state(ws + 32 + row * D + e, value[0], value[1]);
      put_state(ws + 32 + row * D + e + 2, value[2], value[3]);
      if (e == 0) put_state(ws + 2 * row, most, sum);
    }
  }
  // a sequence counts once: of its parts, the first that finds something wrong says so for all
  uint32_t* const told = a.done + LEVELS * a.done_level + (int64_t)p.slot * heads;      // (of a divided sequence)
  bool any_bad = false;
#pragma unroll
  for (int w = 0; w < ONE_WAVES; ++w) any_bad |= wrong[w] != 0;
  if (any_bad && tid == 0 && hr == 0 && (p.parts == 1 || atomicExch(told, 1u) == 0)) atomicAdd(a.refused + 1, 1ull);
  // Parts are put together by sixteens: the workgroup that comes last of sixteen leaves their sum where the first of them had its state and goes on as one part of
  // the next sixteen.  (One workgroup for 128 parts took 11 us for them.)
  int parts = p.parts, part = p.part, apart = 1;                   // of this level; a part's states lie `apart` pieces from the next one's
  for (uint32_t* level = a.done; parts > 1; level += a.done_level) {
    const int first = part / JOIN * JOIN, members = parts - first < JOIN ? parts - first : JOIN;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);          // (vmcnt(0): the state is where every XCD sees it)
    __syncthreads();
    if (tid == 0) {
      uint32_t* const done = level + (int64_t)(p.slot + first * apart) * heads + hr;
      last = atomicAdd(done, 1u) + 1 == (uint32_t)members;
      if (last) *done = 0;
      if (last && parts <= JOIN && hr == 0) *told = 0;
    }
    __syncthreads();
    if (!last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    float* const at = a.ws + ((int64_t)(p.slot + first * apart) * heads + hr) * STATE<D>;
    // (byte offsets in 32 bits: all states together are less, see ftcache_create)
    const uint32_t next = (uint32_t)apart * (uint32_t)heads * (STATE<D> * 4);
    const bool whole = parts <= JOIN;
    for (int x = tid; x < rows * CD; x += THREADS) {
      const int row = x / CD, e = x % CD * 4;
      float2v head[JOIN];
      float4v part_of[JOIN];
      uint32_t from = 0;
#pragma unroll
      for (int i = 0; i < JOIN; ++i) {
        head[i] = *reinterpret_cast<const float2v*>(reinterpret_cast<const char*>(at) + (from + 8 * row));
        part_of[i] = *reinterpret_cast<const float4v*>(reinterpret_cast<const char*>(at) + (from + 4 * (32 + row * D + e)));
        from += i + 1 < members ? next : 0;        // (the last one again behind it)
      }
      float most = head[0][0];
#pragma unroll
      for (int i = 1; i < JOIN; ++i) most = __builtin_fmaxf(most, head[i][0]);
      float4v value = (float4v)0.f;
      float sum = 0.f;
      int left = members;
      asm volatile("" : "+v"(left));               // (compared where it is used: sixteen conditions do not lie in scalar registers for the whole loop)
#pragma unroll
      for (int i = 0; i < JOIN; ++i) {
        const float f = ex2(head[i][0] - most);
        const bool there = i < left;
#pragma unroll
        for (int j = 0; j < 4; ++j) value[j] = there ? __builtin_fmaf(f, part_of[i][j], value[j]) : value[j];
        sum = there ? __builtin_fmaf(f, head[i][1], sum) : sum;
      }
      if (whole) finish(row, e, value, sum);
      else {
        // (a row's reference and sum are read by all of its lanes, which lie in one wave or, at head_dim 128, half of one: they have all read them)
        put_state(at + 32 + row * D + e, value[0], value[1]);
        put_state(at + 32 + row * D + e + 2, value[2], value[3]);
        if (e == 0) put_state(at + 2 * row, most, sum);
      }
    }
    part /= JOIN;
    parts = (parts + JOIN - 1) / JOIN;
    apart *= JOIN;
  }
}

typedef void (*put_fn)(const Args);
typedef void (*get_fn)(const Args);
typedef void (*one_fn)(const OneArgs);
template <int D> static put_fn put_of(bool bf, bool pairs) {
  return bf ? (pairs ? ftcache_put<D, true, true> : ftcache_put<D, true, false>) : (pairs ? ftcache_put<D, false, true> : ftcache_put<D, false, false>);
}
template <int D, bool BF> static one_fn one_of(bool f32) { return f32 ? ftcache_one<D, BF, true> : ftcache_one<D, BF, false>; }

}  // namespace ftcache

using namespace ftcache;

struct ftcache_ctx {
  ftcache_config cfg;
  put_fn put = nullptr;
  get_fn get = nullptr;
  one_fn one = nullptr;
  int shift = 0, row_tiles = 1, chunks = 1, one_round = 1, most_parts = 1;
  void* scratch = nullptr;
  float* ws = nullptr;
  uint32_t* done = nullptr;
  int64_t done_level = 0;
  unsigned long long* refused = nullptr;
  std::string err;
};

static thread_local std::string g_cache_create_err;

static int cfail(ftcache_ctx* c, int code, const char* msg) {
  try {
    (c ? c->err : g_cache_create_err) = msg;
  } catch (...) {
  }
  return code;
}
static int cfail_hip(ftcache_ctx* c, const char* what, hipError_t e) {
  try {
    (c ? c->err : g_cache_create_err) = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return e == hipErrorOutOfMemory ? FTCACHE_ENOMEM : FTCACHE_EHIP;
}

namespace {
// the context's device for the time of a call
struct OnDevice {
  int before = 0, device;
  hipError_t status;
  explicit OnDevice(int d) : device(d) {
    status = hipGetDevice(&before);
    if (status == hipSuccess && before != device) status = hipSetDevice(device);
  }
  ~OnDevice() { if (before != device) (void)hipSetDevice(before); }
};

// nullptr, or what is wrong with a tensor of rows
const char* rows_of(const ftcache_rows* r, int size, bool none, Rows& out) {
  if (!r) return "null argument";
  if ((!r->data && !none) || ((uintptr_t)r->data & 15)) return "tensors must be 16-byte aligned device pointers";
  if (((uintptr_t)r->token_stride | (uintptr_t)r->head_stride) % (16 / size)) return "strides must be whole 16-byte words";
  if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride > (1ll << 40) || r->head_stride > (1ll << 40)) return "strides must lie in 0 to 2^40 elements";
  out = Rows{static_cast<char*>(r->data), r->token_stride * size, r->head_stride * size};
  return nullptr;
}
const char* places_of(const ftcache_places* p, Places& out) {
  if (!p || !p->cu_seqlens || !p->starts || !p->page_table) return "null argument";
  if (p->batch < 1 || p->tokens < 0) return "batch must be >= 1 and tokens >= 0";
  if (p->table_width < 1 || p->table_stride < p->table_width) return "table_width must be >= 1 and at most table_stride";
  out = Places{p->cu_seqlens, p->starts, p->page_table, p->table_stride, p->batch, p->tokens, p->table_width};
  return nullptr;
}
// blocks of 8 places that new tokens can touch: workgroups of append and read
int64_t blocks_of(const Places& p) { return (int64_t)p.tokens / 8 + 2ll * p.batch; }
const char* const TOO_MANY = "more tokens and sequences than a launch has workgroups for";
}  // namespace

extern "C" int ftcache_create(const ftcache_config* cfg, ftcache_ctx** out) {
  if (!cfg || !out) return cfail(nullptr, FTCACHE_EINVAL, "null argument");
  *out = nullptr;
  if (cfg->struct_size != sizeof(ftcache_config)) return cfail(nullptr, FTCACHE_EINVAL, "struct_size mismatch");
  if (cfg->heads < 1 || cfg->kv_heads < 1 || cfg->heads % cfg->kv_heads) return cfail(nullptr, FTCACHE_EINVAL, "heads must be a positive multiple of kv_heads");
  if (cfg->heads > 4096) return cfail(nullptr, FTCACHE_EUNSUPPORTED, "more than 4096 heads");
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return cfail(nullptr, FTCACHE_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (cfg->pages < 1) return cfail(nullptr, FTCACHE_EINVAL, "pages must be >= 1");
  if (cfg->page_size < 16 || cfg->page_size > 1024 || (cfg->page_size & (cfg->page_size - 1))) return cfail(nullptr, FTCACHE_EUNSUPPORTED, "page_size must be a power of two, 16 to 1024");
  if (cfg->in_dtype != FTCACHE_F16 && cfg->in_dtype != FTCACHE_BF16) return cfail(nullptr, FTCACHE_EINVAL, "in_dtype must be F16 or BF16");
  if (cfg->out_dtype != FTCACHE_F32 && cfg->out_dtype != cfg->in_dtype) return cfail(nullptr, FTCACHE_EINVAL, "out_dtype must be F32 or the input type");
  if (cfg->rotary_dim < 0 || cfg->rotary_dim > cfg->head_dim || cfg->rotary_dim % 16) return cfail(nullptr, FTCACHE_EUNSUPPORTED, "rotary_dim must be a multiple of 16 up to head_dim");
  if (cfg->interleaved != 0 && cfg->interleaved != 1) return cfail(nullptr, FTCACHE_EINVAL, "interleaved must be 0 or 1");
  if (!(std::fabs(cfg->softmax_scale) <= 3.0e38f) || cfg->softmax_scale * LOG2E > 3.4e38f) return cfail(nullptr, FTCACHE_EINVAL, "softmax_scale is not finite, or too large");
  if (cfg->max_batch < 1 || cfg->max_batch > 65536) return cfail(nullptr, FTCACHE_EINVAL, "max_batch must be 1 to 65536");
  ftcache_ctx* c = new (std::nothrow) ftcache_ctx();
  if (!c) return cfail(nullptr, FTCACHE_ENOMEM, "out of host memory");
  c->cfg = *cfg;
  ftcache_config& e = c->cfg;
  if (!(e.softmax_scale > 0.f)) e.softmax_scale = 1.0f / std::sqrt((float)e.head_dim);
  if (e.rotary_dim == 0) e.rotary_dim = e.head_dim;
  while ((1 << c->shift) < e.page_size) ++c->shift;
  c->row_tiles = (e.heads / e.kv_heads + 15) / 16;
  const bool bf = e.in_dtype == FTCACHE_BF16, f32 = e.out_dtype == FTCACHE_F32;
  if (e.head_dim == 128) {
    c->put = put_of<128>(bf, e.interleaved != 0);
    c->get = bf ? ftcache_get<128, true> : ftcache_get<128, false>;
    c->one = bf ? one_of<128, true>(f32) : one_of<128, false>(f32);
  } else {
    c->put = put_of<64>(bf, e.interleaved != 0);
    c->get = bf ? ftcache_get<64, true> : ftcache_get<64, false>;
    c->one = bf ? one_of<64, true>(f32) : one_of<64, false>(f32);
  }
  const int64_t heads = (int64_t)e.kv_heads * c->row_tiles;
  c->chunks = (int)(ONE_GROUPS / heads < 1 ? 1 : ONE_GROUPS / heads);
  c->one_round = (int)(ROUND / heads < 1 ? 1 : ROUND / heads);
  c->most_parts = (int)(MOST_PARTS / heads < 1 ? 1 : MOST_PARTS / heads);
  // divided sequences are longer than a piece: together they have fewer than twice `chunks` pieces
  const size_t states = (size_t)2 * c->chunks * heads, ws = states * (32 + 16 * e.head_dim) * sizeof(float), done = (LEVELS + 1) * states * sizeof(uint32_t);
  c->done_level = (int64_t)states;
  OnDevice here(e.device);
  hipError_t he = here.status;
  if (he == hipSuccess) he = hipMalloc(&c->scratch, 256 + ((done + 255) & ~(size_t)255) + ws);
  if (he == hipSuccess) he = hipMemset(c->scratch, 0, 256 + done);
  if (he == hipSuccess) he = hipDeviceSynchronize();
  if (he != hipSuccess) {
    const int rc = cfail_hip(nullptr, "device memory", he);
    if (c->scratch) (void)hipFree(c->scratch);
    delete c;
    return rc;
  }
  c->refused = static_cast<unsigned long long*>(c->scratch);
  c->done = reinterpret_cast<uint32_t*>(static_cast<char*>(c->scratch) + 256);
  c->ws = reinterpret_cast<float*>(static_cast<char*>(c->scratch) + 256 + ((done + 255) & ~(size_t)255));
  *out = c;
  return FTCACHE_OK;
}

extern "C" int ftcache_get_config(const ftcache_ctx* ctx, ftcache_config* effective) {
  if (!ctx || !effective) return FTCACHE_EINVAL;
  *effective = ctx->cfg;
  return FTCACHE_OK;
}

extern "C" int64_t ftcache_page_bytes(const ftcache_ctx* c) {
  return c ? (int64_t)c->cfg.kv_heads * c->cfg.page_size * (c->cfg.head_dim + 8) : FTCACHE_EINVAL;
}

static Pool pool_of(const ftcache_ctx* c, const void* pool) {
  return Pool{static_cast<char*>(const_cast<void*>(pool)), c->cfg.pages, c->cfg.kv_heads, c->shift, c->cfg.page_size * (c->cfg.head_dim + 8)};
}

extern "C" int ftcache_append(ftcache_ctx* c, void* pool, const ftcache_places* places, const float* rotation, int32_t positions,
                              const ftcache_rows* q, const ftcache_rows* k, const ftcache_rows* v, const ftcache_rows* q_out,
                              const ftcache_rows* k_out, void* hip_stream) {
  if (!c) return FTCACHE_EINVAL;
  if (!pool || ((uintptr_t)pool & 15)) return cfail(c, FTCACHE_EINVAL, "pool must be a 16-byte aligned device pointer");
  if (!rotation || ((uintptr_t)rotation & 15) || positions < 1) return cfail(c, FTCACHE_EINVAL, "rotation must be a 16-byte aligned device pointer to at least one position");
  const ftcache_config& e = c->cfg;
  Args a;
  const char* wrong = places_of(places, a.at);
  if (wrong) return cfail(c, FTCACHE_EINVAL, wrong);
  const bool none = a.at.tokens == 0;
  if ((wrong = rows_of(q, 2, true, a.q)) || (wrong = rows_of(k, 2, none, a.k)) || (wrong = rows_of(v, 2, none, a.v)) ||
      (wrong = rows_of(q_out, 2, true, a.q_out)) || (wrong = rows_of(k_out, 2, true, a.k_out)))
    return cfail(c, FTCACHE_EINVAL, wrong);
  if (!a.q.data != !a.q_out.data) return cfail(c, FTCACHE_EINVAL, "q and q_out go together");
  if (none) return FTCACHE_OK;
  a.pool = pool_of(c, pool);
  a.rotation = rotation;
  a.positions = positions;
  a.heads = e.heads;
  a.rotary = e.rotary_dim;
  a.refused = c->refused;
  if (blocks_of(a.at) > MOST_GROUPS) return cfail(c, FTCACHE_EUNSUPPORTED, TOO_MANY);
  const int blocks = (int)blocks_of(a.at), items = (a.q.data ? e.heads : 0) + e.kv_heads;
  // few blocks: their heads are dealt to more workgroups
  int split = (SPLIT_TO + blocks - 1) / blocks;
  split = split < 1 ? 1 : split > (items + 3) / 4 ? (items + 3) / 4 : split;
  OnDevice here(e.device);
  if (here.status != hipSuccess) return cfail_hip(c, "device", here.status);
  hipLaunchKernelGGL(c->put, dim3(blocks, split), dim3(256), 0, (hipStream_t)hip_stream, a);
  const hipError_t he = hipGetLastError();
  return he == hipSuccess ? FTCACHE_OK : cfail_hip(c, "launch", he);
}

extern "C" int ftcache_read(ftcache_ctx* c, const void* pool, const ftcache_places* places, const ftcache_rows* k, const ftcache_rows* v,
                            void* hip_stream) {
  if (!c) return FTCACHE_EINVAL;
  if (!pool || ((uintptr_t)pool & 15)) return cfail(c, FTCACHE_EINVAL, "pool must be a 16-byte aligned device pointer");
  const ftcache_config& e = c->cfg;
  Args a{};
  const char* wrong = places_of(places, a.at);
  if (wrong) return cfail(c, FTCACHE_EINVAL, wrong);
  const bool none = a.at.tokens == 0;
  if ((wrong = rows_of(k, 2, none, a.k)) || (wrong = rows_of(v, 2, none, a.v))) return cfail(c, FTCACHE_EINVAL, wrong);
  if (none) return FTCACHE_OK;
  a.pool = pool_of(c, pool);
  a.refused = c->refused;
  if (blocks_of(a.at) > MOST_GROUPS) return cfail(c, FTCACHE_EUNSUPPORTED, TOO_MANY);
  const int blocks = (int)blocks_of(a.at), items = 2 * e.kv_heads;
  int split = (SPLIT_TO + blocks - 1) / blocks;
  split = split < 1 ? 1 : split > (items + 3) / 4 ? (items + 3) / 4 : split;
  OnDevice here(e.device);
  if (here.status != hipSuccess) return cfail_hip(c, "device", here.status);
  hipLaunchKernelGGL(c->get, dim3(blocks, split), dim3(256), 0, (hipStream_t)hip_stream, a);
  const hipError_t he = hipGetLastError();
  return he == hipSuccess ? FTCACHE_OK : cfail_hip(c, "launch", he);
}

extern "C" int ftcache_attend(ftcache_ctx* c, const void* pool, int32_t batch, const int32_t* lengths, const int32_t* page_table,
                              int32_t table_width, int64_t table_stride, const ftcache_rows* q, const ftcache_rows* o, void* hip_stream) {
  if (!c) return FTCACHE_EINVAL;
  if (!pool || ((uintptr_t)pool & 15)) return cfail(c, FTCACHE_EINVAL, "pool must be a 16-byte aligned device pointer");
  const ftcache_config& e = c->cfg;
  if (batch < 1 || batch > e.max_batch) return cfail(c, FTCACHE_EINVAL, "batch must be 1 to max_batch");
  if (!lengths || !page_table) return cfail(c, FTCACHE_EINVAL, "null argument");
  if (table_width < 1 || table_stride < table_width) return cfail(c, FTCACHE_EINVAL, "table_width must be >= 1 and at most table_stride");
  OneArgs a;
  const char* wrong = rows_of(q, 2, false, a.q);
  if (!wrong) wrong = rows_of(o, e.out_dtype == FTCACHE_F32 ? 4 : 2, false, a.o);
  if (wrong) return cfail(c, FTCACHE_EINVAL, wrong);
  a.pool = pool_of(c, pool);
  a.lengths = lengths;
  a.table = page_table;
  a.table_stride = table_stride;
  a.batch = batch;
  const int64_t most = (int64_t)table_width << c->shift;
  a.most = (int32_t)(most > 0x7FFF0000 ? 0x7FFF0000 : most);      // (places a few steps behind the end still fit 32 bits)
  // pieces at most: what lengths that the table has room for can give
  const int64_t units = ((int64_t)a.most + ONE_UNIT - 1) / ONE_UNIT, room = units <= SHORT ? batch : units * batch;
  if (units * batch > 0x7FFFFFFFll) return cfail(c, FTCACHE_EUNSUPPORTED, "the page table has room for too many tokens");
  const int64_t pieces = room < (int64_t)c->chunks + batch ? room : (int64_t)c->chunks + batch;
  if (pieces * e.kv_heads * c->row_tiles > MOST_GROUPS) return cfail(c, FTCACHE_EUNSUPPORTED, TOO_MANY);
  a.group = e.heads / e.kv_heads;
  a.row_tiles = c->row_tiles;
  a.chunks = c->chunks;
  a.one_round = c->one_round;
  a.most_parts = c->most_parts;
  a.scale_log2 = e.softmax_scale * LOG2E;
  a.ws = c->ws;
  a.done = c->done;
  a.done_level = c->done_level;
  a.refused = c->refused;
  OnDevice here(e.device);
  if (here.status != hipSuccess) return cfail_hip(c, "device", here.status);
  hipLaunchKernelGGL(c->one, dim3((uint32_t)(pieces * e.kv_heads * c->row_tiles)), dim3(ONE_WAVES * 64), 0, (hipStream_t)hip_stream, a);
  const hipError_t he = hipGetLastError();
  return he == hipSuccess ? FTCACHE_OK : cfail_hip(c, "launch", he);
}

extern "C" int ftcache_report(ftcache_ctx* c, ftcache_report_view* out) {
  if (!c) return FTCACHE_EINVAL;
  if (!out) return cfail(c, FTCACHE_EINVAL, "null argument");
  OnDevice here(c->cfg.device);
  hipError_t he = here.status;
  unsigned long long n[2] = {0, 0};
  if (he == hipSuccess) he = hipDeviceSynchronize();
  if (he == hipSuccess) he = hipMemcpy(n, c->refused, sizeof n, hipMemcpyDeviceToHost);
  if (he == hipSuccess) he = hipMemset(c->refused, 0, sizeof n);
  if (he == hipSuccess) he = hipDeviceSynchronize();
  if (he != hipSuccess) return cfail_hip(c, "report", he);
  out->refused_tokens = (int64_t)n[0];
  out->refused_sequences = (int64_t)n[1];
  return FTCACHE_OK;
}

extern "C" int ftcache_destroy(ftcache_ctx* c) {
  if (!c) return FTCACHE_OK;
  {
    OnDevice here(c->cfg.device);
    (void)hipFree(c->scratch);
  }
  delete c;
  return FTCACHE_OK;
}

extern "C" const char* ftcache_last_error(const ftcache_ctx* c) { return c ? c->err.c_str() : g_cache_create_err.c_str(); }
