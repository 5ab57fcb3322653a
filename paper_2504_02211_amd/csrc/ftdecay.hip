// Linear attention with a decay for each head: the kernels and the C ABI of ../include/ftdecay.h.
#include "ftdecay.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>

namespace ftdecay {
using namespace ftserve;

struct Rows { char* data; int64_t token, head; };      // strides in bytes

struct Args {
  Rows q, k, v, o;
  const float* log_decay;
  float* states;
  const int32_t *slots, *cu, *starts;      // cu NULL: one token of every sequence
  int32_t n_slots, batch, total, heads, group;
  float scale;
  int32_t per;             // tokens of a segment, whole chunks
  float* between;          // states between segments, and behind these (STATES of them) the first states of divided sequences
};

template <bool BF> __device__ __forceinline__ float element(const char* row, int i) {
  if constexpr (BF) return as_f((uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
  else return (float)reinterpret_cast<const _Float16*>(row)[i];
}

// The decay in two words: rounded to one, it is off by up to 2^-25 in the same direction at every token, and a state that remembers thousands of tokens by 2^-13.
struct Decay {
  float high, low;
  // Of the i-th in a row: `high`, and every eighth time what `high` alone has left out of eight.
  __device__ __forceinline__ float of(int i) const { return (i & 7) == 7 ? __builtin_fmaf(8.f, low, high) : high; }
};
__device__ __forceinline__ Decay decay_of(const Args& a, int h) {
  const double d = exp((double)__builtin_fminf(a.log_decay[h], 0.f));
  const float high = (float)d;
  return Decay{high, (float)(d - (double)high)};
}

// Where sequence b has its state; NULL: nowhere.
template <int D> __device__ __forceinline__ float* state_of(const Args& a, int b, int h) {
  const int slot = __builtin_amdgcn_readfirstlane(a.slots ? a.slots[b] : b);
  return a.states && slot >= 0 && slot < a.n_slots ? a.states + ((int64_t)slot * a.heads + h) * (D * D) : nullptr;
}

// One token: the recurrence as it stands, a (sequence, head) a workgroup.  Thread (g, e) has column e of the state, rows of its g-th part, which are summed up over LDS.
// Bound by memory, each state read and written once: 96 sequences of 32 heads of 128, 403 MB, take 82 us (4.9 TB/s, what a copy reaches).
template <int D, bool BF> __global__ __launch_bounds__(256) void ftdecay_token(const Args a) {
  constexpr int PARTS = 256 / D, R = D / PARTS;
  __shared__ float qs[D], ks[D], part[PARTS][D];
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads, hk = h / a.group, e = threadIdx.x % D, g = threadIdx.x / D;
  float* const state = state_of<D>(a, b, h);
  const Decay decay = decay_of(a, h);
  float s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = state ? state[(g * R + i) * D + e] : 0.f;
  const float v = element<BF>(a.v.data + b * a.v.token + hk * a.v.head, e);
  if (g == 0) {
    qs[e] = element<BF>(a.q.data + b * a.q.token + h * a.q.head, e);
    ks[e] = element<BF>(a.k.data + b * a.k.token + hk * a.k.head, e);
  }
  __syncthreads();
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    s[i] = __builtin_fmaf(ks[g * R + i], v, __builtin_fmaf(s[i], decay.high, s[i] * decay.low));
    sum = __builtin_fmaf(qs[g * R + i], s[i], sum);
  }
  part[g][e] = sum;
  if (state)
#pragma unroll
    for (int i = 0; i < R; ++i) state[(g * R + i) * D + e] = s[i];
  __syncthreads();
  if (g == 0) {
    float all = 0.f;
    for (int i = 0; i < PARTS; ++i) all += part[i][e];
    all *= a.scale;
    reinterpret_cast<uint16_t*>(a.o.data + b * a.o.token + h * a.o.head)[e] = (uint16_t)pack2<BF>(all, all);
  }
}

// ---- Prompts, in chunks of 64 tokens.  With S the state before a chunk (D x D) and i, j places in it,
//
//     O[i] = scale (decay^(i+1) q_i S + sum over j <= i of decay^(i-j) (q_i . k_j) v_j),      S' = decay^n S + sum over j of decay^(n-1-j) k_j v_j^T
//
// (n tokens), all of them matrix products.  A wave owns 32 columns of values: its slab of S stays in registers (accumulators of k^T v, which are the left operand
// of O^T = S^T q^T as they lie) and so does its part of O; the weights q . k of a chunk are computed once, a 32 x 32 tile a wave, and shared through LDS.
//
// What is rounded to 16 bits before a product is held in more than one word.  bf16: weights and S in two words (2^-16 relative), decayed values in three (S is a state of
// 32 bits).  fp16: S under one power of two for its slab, and the decayed values, in two words, the lower one times 2^11 (22 bits; what the products of lower words add is kept apart until it is
// scaled back); weights, which have no bound, in two words of bf16 with the values as two words of bf16, which hold fp16 exactly.  As fp16 ends at 2^-24, values are lifted by a power of two, up
// to 2^15, as far as the slab's largest allows, and the state is held times as much until the next chunk: a decayed value is off by 2^-24 of itself, or by 2^-51 of a slab's values below 2 where
// that is more (2^-36 without it, which left values of 2^-24 with 12 bits; 16,384 tokens of 32 heads on 8, fp16, take 127 us with it and 121 without at head_dim 64, 201 and 200 at 128).
//
// Sequences are divided into segments of `per` tokens, so that there are workgroups for all CUs: ftdecay_gather forms what each segment alone adds to the state, ftdecay_join adds these up,
// ftdecay_chunks has the state before its segment and does the rest.  (Gathering is a second pass over keys and values, so that no workgroup waits for another.)
// The last segment of a sequence stores its state to the pool, which the first one, a workgroup of the same launch, therefore never reads: ftdecay_join keeps
// the state that a divided sequence begins with.
//
// Bound by vector instructions and the reads of operands from LDS that stand between the products (a product of 32 x 32 x 16 takes as long as eight vector instructions, and the
// words of S, of the weights and of the values are formed by several for each): 16,384 tokens of 32 heads of 128 on 8, bf16, take 194 us.  What goes in and out takes 69 at a
// copy's rate, with the second pass over keys and values and the states between segments, written twice and read twice, 109.  Without the vector work between the products, one after the
// other, 250 us; a token at a time 21.5 ms.  24 prompts of up to 1531 tokens, 12 heads of 64, fp16: 38 us, 890 a token at a time.
constexpr int C = 64;
// Segments: at most STATES states between them (67 MB at head_dim 128, 17 MB at 64; and as much room for first states), and no fewer than LEAST tokens in one: 24 prompts of up to 1531 tokens of 12 heads of 64, fp16, take
// 39.2 us in segments of 128, 39.0 of 192, 43.5 of 256, 67.6 of 512; 4096 tokens of 8 heads of 128, bf16, 36.6, 35.4, 38.4 and 55 us.
constexpr int STATES = 1024, LEAST = 192;

template <int D> constexpr int tile_bytes() { return C * D * 2; }
constexpr int P_BYTES = C * C * 2;      // a word of the weights
template <int D> constexpr int lds_bytes() { return 4 * tile_bytes<D>() + 2 * P_BYTES; }
template <int D> constexpr int gather_lds_bytes() { return 4 * tile_bytes<D>() + P_BYTES / 2; }

template <bool BF> __device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c) {
  if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

// N times 16 bytes per lane from (uniform base + per-lane byte offsets) straight into LDS, 1 KB apart from the uniform LDS address on.  (Opaque to the compiler, which
// would wait for the tile in flight before it reads another.  The first wait covers a base that a vector instruction has moved to its scalar registers just before: five states.)
__device__ __forceinline__ void load_lds16(const void* base, uint32_t off, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds_addr) : "memory", "m0");
}
__device__ __forceinline__ void everything_landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void lds_written() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Row r of a tile has its 16-byte chunk c at place c ^ place_of(r): sixteen lanes that read a chunk of as many rows meet all banks once, and so do
// 32 that read 32 bytes of four rows, twice.
template <int D> __device__ __forceinline__ int place_of(int r) { return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3); }

// Loads of a tile: rows t0 .. t0 + 63 of one head, those behind the last one are the last one again.
template <int D, int NW> struct Loader {
  static constexpr int CH = D / 8, RPL = 64 / CH, LOADS = tile_bytes<D>() / 1024 / NW;      // chunks of a row; rows of a load; loads of a wave
  const char* base;
  int64_t token;
  int wave, lane;
  __device__ __forceinline__ Loader(const Rows& r, int64_t row0, int head, int wave, int lane)
      : base(r.data + row0 * r.token + (int64_t)head * r.head), token(r.token), wave(wave), lane(lane) {}
  __device__ __forceinline__ void issue(int chunk, int tokens, uint32_t to) const {
    const char* const p = base + (int64_t)(chunk * C) * token;
    const int left = tokens - chunk * C, first = wave * LOADS * RPL;
    to += (uint32_t)(wave * LOADS) * 1024;
    int l = lane;
    asm volatile("" : "+v"(l));      // (nothing of this is worth a register outside of here)
    const int r = l / CH;
    if (left >= C) {
      const uint32_t row = (uint32_t)r * (uint32_t)token, place = (uint32_t)((l % CH) ^ place_of<D>(first + r)) * 16;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_lds16(p + (int64_t)(first + i * RPL) * token, row + (place ^ (uint32_t)(place_of<D>(i * RPL) * 16)), to + (uint32_t)i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int x = first + i * RPL + r, rc = x < left ? x : left - 1;
        load_lds16(p, (uint32_t)rc * (uint32_t)token + (uint32_t)((l % CH) ^ place_of<D>(x)) * 16, to + (uint32_t)i * 1024);
      }
    }
  }
};

// A segment: tokens of one sequence and head that one workgroup takes, `per` or fewer.
struct Segment {
  int b, h, number, tokens, first;      // number in its sequence; tokens of it; its first row
  bool last;
  int64_t before;                       // number of the sequence's first state between segments
};
__device__ __forceinline__ bool segment_of(const Args& a, int64_t id, Segment& s) {
  // The heads of a group, which share keys and values, run one after the other on one XCD; groups go round the XCDs, so that all have as many of them.
  // (Neighbouring groups on one XCD leave another without: 16,384 tokens of 32 heads on 8 took 316 us.)
  const int xcd = (int)(id & 7), place = (int)(id >> 3), group = __builtin_amdgcn_readfirstlane((place / a.group) * 8 + xcd), kv_heads = a.heads / a.group;
  // (divisions leave the scalar unit; everything here is the same in all lanes)
  const int unit = __builtin_amdgcn_readfirstlane(group / kv_heads);
  s.h = __builtin_amdgcn_readfirstlane(group % kv_heads * a.group + place % a.group);
  if (unit >= a.total / a.per + a.batch) return false;
  // sequence b owns the numbers from cu[b] / per + b on: at least as many as it has segments, whatever the others have
  auto begin = [&](int b) { return (int64_t)(clamped(a.cu[b], a.total) / a.per + b); };
  s.b = sequence_of(a.batch, unit, begin);
  const int t0 = clamped(a.cu[s.b], a.total), t1 = clamped(a.cu[s.b + 1], a.total), n = t1 > t0 ? t1 - t0 : 0;
  s.number = __builtin_amdgcn_readfirstlane(unit - (int)begin(s.b));
  const int segments = __builtin_amdgcn_readfirstlane(n > a.per ? (n + a.per - 1) / a.per : 1);
  if (s.number < 0 || s.number >= segments) return false;
  s.last = s.number == segments - 1;
  s.first = t0 + s.number * a.per;
  s.tokens = s.last ? n - s.number * a.per : a.per;
  s.before = __builtin_amdgcn_readfirstlane(t0 / a.per);
  return true;
}

__device__ __forceinline__ float in_scalar(float x) { return as_f((uint32_t)__builtin_amdgcn_readfirstlane((int)as_u(x))); }      // (the same in all lanes)

// log2 of the decay in two words: its multiples are exact to 32 bits
struct Powers {
  float high, low;
  double log;
  __device__ __forceinline__ Powers(const Args& a, int h) {
    log = (double)__builtin_fmaxf(__builtin_fminf(a.log_decay[h], 0.f), -1e30f);
    const double x = log * 1.4426950408889634074;
    high = in_scalar((float)x);
    low = in_scalar((float)(x - (double)(float)x));
  }
  __device__ __forceinline__ float to(int n) const { return ex2(__builtin_fmaf((float)n, high, (float)n * low)); }
  __device__ __forceinline__ Decay whole(int n) const {
    const double d = exp((double)n * log);
    const float f = (float)d;
    return Decay{in_scalar(f), in_scalar((float)(d - (double)f))};
  }
};

// Row m of an accumulator tile of the state stands for row swapped(m) of its 32: register 4g + r of lane (h, n) for 16 (g / 2) + 8h + 4 (g % 2) + r, eight in a row for each
// pair of g, as operands have them.
__device__ __forceinline__ int row_of(int v, int h) { return 16 * (v >> 3) + 8 * h + (v & 7); }

template <int D, bool BF> struct Chunk {
  static constexpr int NW = D / 32, NB = D / 32, KS = C / 16;      // waves; blocks of 32 rows of the state; steps of 16 tokens
  int lane, wave, h, n;
  uint32_t rows_at, columns_at[2];      // places of this lane's reads in a tile: of rows (block of 16 elements 0), transposed (the state's rows; values)
  // This wave's factors, in a place that the weights leave free: 16-byte words of queries 4 wave .. 4 wave + 3 for keys from 32 on, which these do not see.
  uint32_t falls_at;
  __device__ __forceinline__ uint32_t fall_word(int x) const {
    const int r = 4 * wave + (x >> 2);
    return falls_at + (uint32_t)(r * (2 * C) + (((4 + (x & 3)) ^ (r >> 1 & 7)) * 16));
  }
  __device__ __forceinline__ explicit Chunk(uint32_t weights) : lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), h(lane >> 5), n(lane & 31) {
    // (what the place of a row's chunk depends on is the same for rows 32 apart, and for tokens 16 apart)
    rows_at = (uint32_t)(n * (2 * D) + ((h ^ place_of<D>(n)) * 16));
    const int rr = lane >> 2 & 3, r = 8 * h + rr;
#pragma unroll
    for (int swap = 0; swap < 2; ++swap) {
      const int u = swap ? (lane & 1) << 1 | (lane >> 1 & 1) : lane & 3;
      columns_at[swap] = (uint32_t)(r * (2 * D) + (((2 * (lane >> 4 & 1) + (u >> 1)) ^ place_of<D>(r)) * 16) + (u & 1) * 8);
    }
    falls_at = weights;
  }

  // New values, as far as the compiler knows: what is computed from them in a loop stays there, where it would fill the registers in front of it.
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(rows_at), "+v"(columns_at[0]), "+v"(columns_at[1]), "+s"(falls_at)); }

  // The transposed operand of tokens 16s + 8h .. + 7 (two a register): column 32f + m in lane (h, n), m = n (values), or n with bits 2 and 3 exchanged.
  // Sixteen lanes read four rows of 16 columns, 8 bytes a lane, and get a column of four rows each.  Rows 4 further on have their chunks at places that differ in one bit.
  template <bool SWAP> __device__ __forceinline__ uint4v transposed(uint32_t tile, int s, int f) const {
    const uint32_t at = tile + (columns_at[SWAP] ^ (uint32_t)(f << 6));
    const uint2v x = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)(at + s * 32 * D)));
    const uint32_t further = tile + (columns_at[SWAP] ^ (uint32_t)(f << 6 | 16));
    const uint2v y = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)(uintptr_t)(further + s * 32 * D + 8 * D)));
    return uint4v{x[0], x[1], y[0], y[1]};
  }
  // Elements 16x + 8h .. + 7 of row 32t + n; `at`: rows_at, or that of another row.
  __device__ __forceinline__ uint4v row(uint32_t tile, uint32_t at, int t, int x) const {
    return *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)(tile + (at ^ (uint32_t)(x << 5)) + t * 64 * D);
  }

  // The decays from every token of a chunk of `tokens` to its end, to where this wave reads them.
  __device__ __forceinline__ void set_falls(const Powers& p, int tokens) const {
    const int left = tokens - 1 - lane;
    *(__attribute__((address_space(3))) float*)(uintptr_t)(fall_word(lane >> 2) + 4 * (lane & 3)) = left < 0 ? 0.f : p.to(left);
  }

  // The largest magnitudes of this lane's values, a pair's, as their 16 bits, which are ordered as the numbers are.
  static constexpr uint32_t INF = BF ? 0x7F80u : 0x7C00u;
  static __device__ __forceinline__ uint32_t largest(const uint4v (&vr)[KS]) {
    uint32_t most = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, most), __builtin_bit_cast(ushort2v, vr[s][x] & 0x7FFF7FFFu)));
    return most;
  }
  static __device__ __forceinline__ bool unbounded(uint32_t most) { return __any((most & 0xFFFFu) >= INF || most >> 16 >= INF); }
  // fp16, whose least number lies 2^-24 below 1: the power of two, up to 2^15, by which the slab's values may be lifted, and the state with them, so that what is left
  // of a word and of decayed values has room below.  (Exact: the largest stays a number.)
  static __device__ __forceinline__ int room(uint32_t most) {
    most = (most & 0xFFFFu) > most >> 16 ? most & 0xFFFFu : most >> 16;
    int t = 15;
#pragma unroll
    for (int b = 8; b; b >>= 1) t += __any(most >= (uint32_t)(t + b) << 10) ? b : 0;
    return 30 - t;
  }
  static __device__ __forceinline__ uint32_t lift_of(int e) { return (uint32_t)(15 + e) * 0x04000400u; }
  static __device__ __forceinline__ float power(int e) { return as_f((uint32_t)(127 + e) << 23); }

  // The values of tokens 16s + 8h .. + 7, lifted (fp16) and decayed to the end of the chunk, in words: in parts, so that matrix instructions can stand between them.
  static constexpr int WORDS = BF ? 3 : 2, PARTS = 4 * WORDS;
  struct Decayed {
    float4v f[2];
    float x, y;
    uint4v w[WORDS];
  };
  __device__ __forceinline__ void begin(Decayed& d, int s) const {
    // (words 4s + 2h and the next one: the same row, places 2h and 1 from each other)
    const uint32_t first = fall_word(4 * s) ^ (uint32_t)(h << 5);
    d.f[0] = *(const __attribute__((address_space(3))) float4v*)(uintptr_t)first;
    d.f[1] = *(const __attribute__((address_space(3))) float4v*)(uintptr_t)(first ^ 16u);
  }
  __device__ __forceinline__ void part(Decayed& d, const uint4v& v, uint32_t lift, int x) const {
    const int i = x / WORDS;
    if (x % WORDS == 0) {
      const uint32_t raw = v[i], y = BF ? raw : __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, raw) * __builtin_bit_cast(half2v, lift));
      d.x = low_of<BF>(y) * d.f[i >> 1][2 * (i & 1)];
      d.y = high_of<BF>(y) * d.f[i >> 1][2 * (i & 1) + 1];
      d.w[0][i] = pack2<BF>(d.x, d.y);
    } else if (x % WORDS == 1) {
      d.x -= low_of<BF>(d.w[0][i]);
      d.y -= high_of<BF>(d.w[0][i]);
      d.w[1][i] = BF ? pack2<BF>(d.x, d.y) : pack2<BF>(d.x * 2048.f, d.y * 2048.f);
    } else {
      d.w[WORDS - 1][i] = pack2<BF>(d.x - low_of<BF>(d.w[1][i]), d.y - high_of<BF>(d.w[1][i]));
    }
  }
  static __device__ __forceinline__ void here() { __builtin_amdgcn_sched_barrier(0); }

  // A sixteenth of the slab, decayed by a chunk.
  __device__ __forceinline__ void fade(float16v (&S)[NB], float by, int x) const {
#pragma unroll
    for (int v = x * NB; v < (x + 1) * NB; ++v) S[v >> 4][v & 15] *= by;
  }

  // The slab, decayed and lifted already, moves on by a chunk.  vr: its values, raw; d: those of the first step, ready.  `beside(i)`: what else is done, in 8 parts.
  template <class F> __device__ __forceinline__ void update(float16v (&S)[NB], const uint4v (&vr)[KS], uint32_t lift, Decayed& d, uint32_t ktile, F beside) const {
    uint4v k[2][NB];
    float16v low[BF ? 1 : NB];
    if constexpr (!BF)
#pragma unroll
      for (int b = 0; b < NB; ++b) low[b] = (float16v)0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) k[0][b] = transposed<true>(ktile, 0, b);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      uint4v w[WORDS];
#pragma unroll
      for (int x = 0; x < WORDS; ++x) w[x] = d.w[x];
      if (s + 1 < KS) begin(d, s + 1);
      here();
#pragma unroll
      for (int i = 0; i < WORDS * NB; ++i) {
        const int x = WORDS - 1 - i / NB, b = i % NB;
        if (!BF && x) low[BF ? 0 : b] = mfma32<BF>(k[s & 1][b], w[x], low[BF ? 0 : b]);
        else S[b] = mfma32<BF>(k[s & 1][b], w[x], S[b]);
        if (s + 1 < KS) {
          if (i < NB) k[(s + 1) & 1][i] = transposed<true>(ktile, s + 1, i);
#pragma unroll
          for (int y = PARTS * i / (WORDS * NB); y < PARTS * (i + 1) / (WORDS * NB); ++y) part(d, vr[s + 1 < KS ? s + 1 : 0], lift, y);
        }
        if (s == 0)
#pragma unroll
          for (int y = 8 * i / (WORDS * NB); y < 8 * (i + 1) / (WORDS * NB); ++y) beside(y);
        here();
      }
    }
    if constexpr (!BF)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) S[b][v] = __builtin_fmaf(low[b][v], 0x1p-11f, S[b][v]);
  }

  // The slab from and to memory: [row][column] of 32 bits.
  __device__ __forceinline__ void fetch(float16v (&S)[NB], const float* from) const {
    if (from) {
      const float* const at = from + 8 * h * D + 32 * wave + n;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) S[b][v] = at[(32 * b + row_of(v, 0)) * D];
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b) S[b] = (float16v)0.f;
    }
  }
  __device__ __forceinline__ void put(const float16v (&S)[NB], float* to, float by) const {      // (times `by` in fp16)
    float* const at = to + 8 * h * D + 32 * wave + n;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) at[(32 * b + row_of(v, 0)) * D] = BF ? S[b][v] : S[b][v] * by;
  }
};

typedef __attribute__((address_space(3))) char lds_char;

// What a segment alone adds to the state, for all but the last of a sequence: to the states between segments.
template <int D, bool BF> __global__ __launch_bounds__(2 * D, 2) void ftdecay_gather(const Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  Segment g;
  if (!segment_of(a, blockIdx.x, g) || g.last) return;
  constexpr uint32_t TILE = tile_bytes<D>();
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
  Chunk<D, BF> c(lds0 + 4 * TILE);
  const int hk = __builtin_amdgcn_readfirstlane(g.h / a.group), chunks = (g.tokens + C - 1) / C;
  const Powers powers(a, g.h);
  const Loader<D, D / 32> lk(a.k, g.first, hk, c.wave, c.lane), lv(a.v, g.first, hk, c.wave, c.lane);
  lk.issue(0, g.tokens, lds0);
  lv.issue(0, g.tokens, lds0 + TILE);
  c.set_falls(powers, C);
  const Decay whole = powers.whole(C);
  float16v S[D / 32];
  c.fetch(S, nullptr);
  int lifted = 0;      // the slab is 2^lifted times the state
  for (int i = 0; i < chunks; ++i) {
    const uint32_t tile = lds0 + (i & 1) * 2 * TILE;
    c.renew();
    everything_landed();
    if (i + 1 < chunks) {
      const uint32_t next = lds0 + (~i & 1) * 2 * TILE;
      lk.issue(i + 1, g.tokens, next);
      lv.issue(i + 1, g.tokens, next + TILE);
    }
    uint4v vr[C / 16];
#pragma unroll
    for (int s = 0; s < C / 16; ++s) vr[s] = c.template transposed<false>(tile + TILE, s, c.wave);
    float fading = whole.of(i);
    uint32_t lift = 0;
    typename Chunk<D, BF>::Decayed d;
    c.begin(d, 0);
    if constexpr (!BF) {
      uint32_t most = c.largest(vr);
      if (__builtin_expect(c.unbounded(most), 0)) {      // (what is not finite counts in its own column alone)
        uint4v finite[C / 16];
#pragma unroll
        for (int s = 0; s < C / 16; ++s)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            finite[s][x] = vr[s][x] & ((vr[s][x] & c.INF) == c.INF ? 0u : 0xFFFFu) | vr[s][x] & ((vr[s][x] >> 16 & c.INF) == c.INF ? 0u : 0xFFFF0000u);
        most = c.largest(finite);
      }
      const int e = c.room(most);
      fading *= c.power(e - lifted);
      lift = c.lift_of(e);
      lifted = e;
    }
    fading = in_scalar(fading);
#pragma unroll
    for (int x = 0; x < c.PARTS; ++x) c.part(d, vr[0], lift, x);
#pragma unroll
    for (int x = 0; x < 16; ++x) c.fade(S, fading, x);
    c.update(S, vr, lift, d, tile, [](int) {});
  }
  c.put(S, a.between + ((g.before + g.number) * a.heads + g.h) * (D * D), c.power(-lifted));
}

// The states between segments: each the sum of what the segments before it add, decayed, and of the sequence's first state.
template <int D> __global__ __launch_bounds__(256) void ftdecay_join(const Args a) {
  constexpr int BLOCKS = D * D / 1024;
  const int unit = blockIdx.x / BLOCKS, b = unit / a.heads, h = unit % a.heads, e = (blockIdx.x % BLOCKS * 256 + threadIdx.x) * 4;
  const int t0 = clamped(a.cu[b], a.total), t1 = clamped(a.cu[b + 1], a.total), n = t1 > t0 ? t1 - t0 : 0;
  const int segments = n > a.per ? (n + a.per - 1) / a.per : 1;
  if (segments < 2) return;
  const float* const first = a.starts && a.starts[b] > 0 ? state_of<D>(a, b, h) : nullptr;
  float4v x = first ? *reinterpret_cast<const float4v*>(first + e) : (float4v)0.f;
  const Decay whole = Powers(a, h).whole(a.per);
  const int64_t place = (int64_t)(t0 / a.per) * a.heads + h;      // (divided sequences are longer than `per`: no two begin in the same one)
  float4v* const at = reinterpret_cast<float4v*>(a.between + place * (D * D) + e);
  if (first) *reinterpret_cast<float4v*>(a.between + (STATES + place) * (D * D) + e) = x;
  const int64_t apart = (int64_t)a.heads * (D * D / 4);
  for (int s = 0; s + 1 < segments; s += 8) {      // (eight loads under way at a time)
    float4v y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s + i + 1 < segments) y[i] = at[(s + i) * apart];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s + i + 1 < segments) {
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = __builtin_fmaf(x[c], whole.high, __builtin_fmaf(x[c], whole.low, y[i][c]));
        at[(s + i) * apart] = x;
      }
  }
}

template <int D, bool BF> __global__ __launch_bounds__(2 * D, 2) void ftdecay_chunks(const Args a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int NW = D / 32, NB = D / 32, KS = C / 16;
  constexpr uint32_t TILE = tile_bytes<D>();
  Segment g;
  if (!segment_of(a, blockIdx.x, g)) return;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem, qt = lds0, vt = lds0 + TILE, keys = lds0 + 2 * TILE, pt = lds0 + 4 * TILE;
  Chunk<D, BF> c(pt);
  const int wave = c.wave;
  const int hk = __builtin_amdgcn_readfirstlane(g.h / a.group), chunks = (g.tokens + C - 1) / C;
  float* const state = state_of<D>(a, g.b, g.h);
  const float* from = nullptr;
  if (g.number > 0) from = a.between + ((g.before + g.number - 1) * a.heads + g.h) * (D * D);
  else if (state && a.starts && a.starts[g.b] > 0) from = g.last ? state : a.between + (STATES + g.before * a.heads + g.h) * (D * D);
  const Loader<D, NW> lq(a.q, g.first, g.h, wave, c.lane), lk(a.k, g.first, hk, wave, c.lane), lv(a.v, g.first, hk, wave, c.lane);
  if (chunks > 0) {
    lq.issue(0, g.tokens, qt);
    lk.issue(0, g.tokens, keys);
    lv.issue(0, g.tokens, vt);
  }
  float16v S[NB];
  c.fetch(S, from);
  const Powers powers(a, g.h);
  // Weights are computed in tiles of 32 keys x 32 queries: (0, 0), (0, 1) and (1, 1); no query of the other sees its keys.  Waves 0, 1 and 2 take one each, and
  // wave 3 does as wave 2 does (a branch would cost all of them more); of two waves the first takes both on the diagonal.  Lane (h, n) has query n and keys row_of(v, h).
  const int jt0 = wave >= 2, it0 = wave > 0;
  const int h0 = c.lane >> 5, n0 = c.lane & 31;
  float factor[16];
  c.set_falls(powers, C);
  const Decay whole = powers.whole(C);
  const float rest = powers.to(g.tokens - (chunks - 1) * C);      // of the last chunk
  const float rise = a.scale * powers.to(n0 + 1), rise32 = in_scalar(powers.to(32));
#pragma unroll
  for (int v = 0; v < 16; ++v) factor[v] = a.scale * powers.to(32 * (it0 - jt0) + n0 - row_of(v, h0));      // (those of keys behind the query are not used)
  const int m = (n0 & 0x13) | (n0 & 4) << 1 | (n0 & 8) >> 1;      // (row n of the left operand is key m)
  uint32_t key_at = (uint32_t)(m * (2 * D) + ((h0 ^ place_of<D>(m)) * 16));
  uint32_t weight_at = (uint32_t)(n0 * (2 * C) + ((h0 ^ (n0 >> 1 & 7)) * 16));      // (the same for queries 32 apart)
  char* const o0 = a.o.data + (int64_t)g.first * a.o.token + (int64_t)g.h * a.o.head + 64 * wave;

  int lifted = 0;      // the slab is 2^lifted times the state

  for (int i = 0; i < chunks; ++i) {
    const int left = g.tokens - i * C, tokens = left < C ? left : C;
    c.renew();
    asm volatile("" : "+v"(key_at), "+v"(weight_at));
    int h = h0, n = n0;
    if constexpr (!BF) {      // (two registers less)
      int lane = c.lane;
      asm volatile("" : "+v"(lane));
      h = lane >> 5;
      n = lane & 31;
    }
    const uint32_t kt = keys + (i & 1) * TILE;
    everything_landed();
    if (i + 1 < chunks) lk.issue(i + 1, g.tokens, keys + (~i & 1) * TILE);
    if (tokens < C) c.set_falls(powers, tokens);
    // Every matrix instruction is followed by what fits beside it: vector instructions in the shadow of the wave's own matrix instructions are nearly free.
    uint2v words[2];
    auto weight = [&](const float16v& w, int limit, int v) __attribute__((always_inline)) {      // weights v and v + 1
      const float p0 = row_of(v, 0) > limit ? 0.f : w[v] * factor[v], p1 = row_of(v + 1, 0) > limit ? 0.f : w[v + 1] * factor[v + 1];
      const uint32_t high = pack2<true>(p0, p1);
      words[0][v >> 1 & 1] = high;
      words[1][v >> 1 & 1] = pack2<true>(p0 - low_of<true>(high), p1 - high_of<true>(high));
    };
    auto share = [&](int jt, int it, int y) __attribute__((always_inline)) {      // four keys' words to LDS
#pragma unroll
      for (int x = 0; x < 2; ++x)
        *(__attribute__((address_space(3))) uint2v*)(uintptr_t)(pt + it * (64 * C) + x * P_BYTES + (weight_at ^ (uint32_t)((4 * jt + (y & 2)) << 4)) + 8 * (y & 1)) = words[x];
    };
    auto scores = [&](int jt, int it, auto beside) __attribute__((always_inline)) {
      float16v w = (float16v)0.f;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        w = mfma32<BF>(c.row(kt + jt * 64 * D, key_at, 0, x), c.row(qt + it * 64 * D, c.rows_at, 0, x), w);
        beside(x);
      }
      return w;
    };
    // the slab of the state in words of 16 bits: `high` and `low` of elements 16x + 8h ..  (fp16: times `up`, its largest just below 2^14)
    float up = 1.f, down = 1.f;
    bool huge = false;      // (a state that has no room to be lifted)
    if constexpr (!BF) {
      float most = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) most = __builtin_fmaxf(most, __builtin_fabsf(S[b][v]));
#pragma unroll
      for (int d = 32; d; d >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d));
      if (__builtin_expect(most > 3.4028235e38f, 0)) {      // (what is infinite is not counted: other columns stay what they are)
        most = 0.f;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) most = __builtin_fabsf(S[b][v]) <= 3.4028235e38f ? __builtin_fmaxf(most, __builtin_fabsf(S[b][v])) : most;
#pragma unroll
        for (int d = 32; d; d >>= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d));
      }
      int e = most > 0.f ? 140 - (int)(as_u(most) >> 23) : 0;
      e = __builtin_amdgcn_readfirstlane(e > 100 ? 100 : e);
      up = c.power(e);
      down = c.power(-e - lifted);
      huge = e < -90;
    }
    struct Words { uint4v high, low; };
    auto split = [&](Words& w, int x, int v) __attribute__((always_inline)) {
      float y = S[x >> 1][8 * (x & 1) + 2 * v], z = S[x >> 1][8 * (x & 1) + 2 * v + 1];
      if constexpr (!BF) {
        y *= up;
        z *= up;
      }
      w.high[v] = pack2<BF>(y, z);
      y -= low_of<BF>(w.high[v]);
      z -= high_of<BF>(w.high[v]);
      w.low[v] = BF ? pack2<BF>(y, z) : pack2<BF>(y * 2048.f, z * 2048.f);
    };
    Words sw[2];
    uint4v q[2][2];
    const float16v w0 = scores(jt0, it0, [&](int x) __attribute__((always_inline)) {
      if (x < 4) split(sw[0], 0, x);
    });
#pragma unroll
    for (int t = 0; t < 2; ++t) q[0][t] = c.row(qt, c.rows_at, t, 0);
    int limit = it0 == jt0 ? n - 8 * h : C;      // the last key of a row that the query sees, counted from 8h on
    asm volatile("" : "+v"(limit));
    c.here();
    // What the state has of earlier tokens.
    float16v O[2], Olow[2];
    O[0] = O[1] = Olow[0] = Olow[1] = (float16v)0.f;
    constexpr bool AHEAD = BF || D == 64;      // (queries are read a step ahead where there are registers for them)
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      if (!AHEAD && x)
#pragma unroll
        for (int t = 0; t < 2; ++t) q[x & 1][t] = c.row(qt, c.rows_at, t, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = i & 1;
        if (i < 2) (BF ? O : Olow)[t] = mfma32<BF>(sw[x & 1].low, q[x & 1][t], (BF ? O : Olow)[t]);
        else O[t] = mfma32<BF>(sw[x & 1].high, q[x & 1][t], O[t]);
        if (x + 1 < D / 16) {
          if (i < 2 && AHEAD) q[(x + 1) & 1][t] = c.row(qt, c.rows_at, t, x + 1);
          split(sw[(x + 1) & 1], x + 1 < D / 16 ? x + 1 : 0, i);
        }
        // 8 pairs of weights beside the instructions from the second step on
        constexpr int STEP = (4 * (D / 16) - 4) / 8;
        const int at = 4 * x + i - 4;
        if (at >= 0 && at % STEP == 0 && at / STEP < 8) {
          const int y = at / STEP;
          weight(w0, limit, 2 * y);
          if (y & 1) share(jt0, it0, y >> 1);
        }
        c.here();
      }
    }
    if (NW == 2 && wave == 0) {
      const float16v w1 = scores(1, 1, [](int) {});
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        weight(w1, limit, 2 * y);
        if (y & 1) share(1, 1, y >> 1);
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float up_to = t ? rise * rise32 : rise;
      if constexpr (BF) O[t] *= up_to;
      else {
        const float f = up_to * down;
#pragma unroll
        for (int v = 0; v < 16; ++v) O[t][v] = __builtin_fmaf(Olow[t][v], 0x1p-11f, O[t][v]) * f;
      }
    }
    uint4v vr[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) vr[s] = c.template transposed<false>(vt, s, wave);
    typename Chunk<D, BF>::Decayed d;
    c.begin(d, 0);
    lds_written();                         // the weights are there, and nobody reads this chunk's queries and values any more
    if (i + 1 < chunks) {
      lq.issue(i + 1, g.tokens, qt);
      lv.issue(i + 1, g.tokens, vt);
    }
    // Values that are not finite are left out of the products, which would bring them to tokens before theirs (0 times infinity); the tokens from theirs on, and the
    // state, get NaN in their column.
    uint32_t most = c.largest(vr);
    if (__builtin_expect(c.unbounded(most), 0)) {
      int first = C, from = 4 * h;
      asm volatile("" : "+v"(from));
#pragma unroll
      for (int s = KS - 1; s >= 0; --s)
#pragma unroll
        for (int x = 7; x >= 0; --x) {
          const uint32_t mask = c.INF << 16 * (x & 1);
          if ((vr[s][x >> 1] & mask) == mask) {
            first = 16 * s + x;
            vr[s][x >> 1] &= x & 1 ? 0xFFFFu : 0xFFFF0000u;
          }
        }
      first = first < C ? first + 8 * h : C;
      const int other = __shfl_xor(first, 32);
      first = other < first ? other : first;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int token = __shfl(first, from + 8 * (v >> 2) + (v & 3));
#pragma unroll
        for (int t = 0; t < 2; ++t) O[t][v] = 32 * t + n >= token ? __builtin_nanf("") : O[t][v];
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) S[b][v] = first < C ? __builtin_nanf("") : S[b][v];
      if constexpr (!BF) most = c.largest(vr);
    }
    float fading = tokens < C ? rest : whole.of(i);
    uint32_t lift = 0;
    if constexpr (!BF) {
      const int e = huge ? 0 : c.room(most);
      fading *= c.power(e - lifted);
      lift = c.lift_of(e);
      lifted = e;
    }
    fading = in_scalar(fading);
    c.here();
    // The chunk's own tokens: for each step of 16 keys the query blocks that see some of them, the lower words first.  Beside them the state fades.
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      uint4v v0 = vr[s], v1;
      if constexpr (!BF) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float y = low_of<false>(vr[s][x]), z = high_of<false>(vr[s][x]);
          v0[x] = pack2<true>(y, z);
          v1[x] = pack2<true>(y - low_of<true>(v0[x]), z - high_of<true>(v0[x]));
        }
      }
      uint4v p[2][2];
#pragma unroll
      for (int t = s / 2; t < 2; ++t) {
        const uint32_t at = pt + t * (64 * C) + (weight_at ^ (uint32_t)(s << 5));
#pragma unroll
        for (int x = 0; x < 2; ++x) p[t][x] = *(const __attribute__((address_space(3))) uint4v*)(uintptr_t)(at + x * P_BYTES);
      }
#pragma unroll
      for (int x = BF ? 1 : 2; x >= 0; --x)
#pragma unroll
        for (int t = s / 2; t < 2; ++t) {
          O[t] = mfma32<true>(x == 2 ? v1 : v0, p[t][x == 1], O[t]);
          const int done = x == 0 ? t : -1;
          if (s < 2 || t == 1) {
            // 16 parts of the fading, those of the first decayed values, over the last products of each step
            if (done >= 0) {
              constexpr int PLACES = 6;
              const int at = s < 2 ? 2 * s + t : 2 + s;
#pragma unroll
              for (int y = 16 * at / PLACES; y < 16 * (at + 1) / PLACES; ++y) c.fade(S, fading, y);
#pragma unroll
              for (int y = c.PARTS * at / PLACES; y < c.PARTS * (at + 1) / PLACES; ++y) c.part(d, vr[0], lift, y);
            }
          }
          c.here();
        }
    }
    // Lane (h, n): token n of a block, columns 8z + 4h + r of the slab.  (Rows behind the last token: an offset that the buffer does not have.)
    const auto out = __builtin_amdgcn_make_buffer_rsrc(o0 + (int64_t)(i * C) * a.o.token, 0, 0x7FFFFFFF, 0x00027000);
    uint32_t o_at[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) o_at[t] = 32 * t + n < tokens ? (uint32_t)n * (uint32_t)a.o.token + 8 * h : 0x80000000u;
    auto store = [&](int y) __attribute__((always_inline)) {
      const int t = y >> 2, z = y & 3;
      __builtin_amdgcn_raw_buffer_store_b64(uint2v{pack2<BF>(O[t][4 * z], O[t][4 * z + 1]), pack2<BF>(O[t][4 * z + 2], O[t][4 * z + 3])}, out, (int)(o_at[t] + 16 * z),
                                            t * 32 * (int)a.o.token, 0);
    };
    if constexpr (!BF)      // (the registers of these results are needed)
#pragma unroll
      for (int y = 0; y < 8; ++y) store(y);
    c.update(S, vr, lift, d, kt, [&](int y) __attribute__((always_inline)) {
      if constexpr (BF) store(y);
    });
  }
  if (g.last && state) c.put(S, state, c.power(-lifted));
}

typedef void (*kernel_fn)(const Args);

}  // namespace ftdecay

using namespace ftdecay;

struct ftdecay_ctx {
  ftdecay_config cfg;
  kernel_fn token = nullptr, gather = nullptr, join = nullptr, chunks = nullptr;
  int lds = 0, gather_lds = 0;
  float* between = nullptr;
  std::string err;
};

static thread_local std::string g_decay_create_err;

static int dfail(ftdecay_ctx* c, int code, const char* msg) {
  try {
    (c ? c->err : g_decay_create_err) = msg;
  } catch (...) {
  }
  return code;
}
static int dfail_hip(ftdecay_ctx* c, const char* what, hipError_t e) {
  try {
    (c ? c->err : g_decay_create_err) = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return e == hipErrorOutOfMemory ? FTDECAY_ENOMEM : FTDECAY_EHIP;
}

template <int D, bool BF> static void choose_kernels(ftdecay_ctx* c) {
  c->token = ftdecay_token<D, BF>;
  c->gather = ftdecay_gather<D, BF>;
  c->join = ftdecay_join<D>;
  c->chunks = ftdecay_chunks<D, BF>;
  c->lds = lds_bytes<D>();
  c->gather_lds = gather_lds_bytes<D>();
}

extern "C" int ftdecay_create(const ftdecay_config* cfg, ftdecay_ctx** out) {
  if (!cfg || !out) return dfail(nullptr, FTDECAY_EINVAL, "null argument");
  *out = nullptr;
  if (cfg->struct_size != sizeof(ftdecay_config)) return dfail(nullptr, FTDECAY_EINVAL, "struct_size mismatch");
  if (cfg->heads < 1 || cfg->kv_heads < 1 || cfg->heads % cfg->kv_heads) return dfail(nullptr, FTDECAY_EINVAL, "heads must be a positive multiple of kv_heads");
  if (cfg->heads > 65536) return dfail(nullptr, FTDECAY_EUNSUPPORTED, "more than 65536 heads");
  if (cfg->head_dim != 64 && cfg->head_dim != 128) return dfail(nullptr, FTDECAY_EUNSUPPORTED, "head_dim must be 64 or 128");
  if (cfg->in_dtype != FTDECAY_F16 && cfg->in_dtype != FTDECAY_BF16) return dfail(nullptr, FTDECAY_EINVAL, "in_dtype must be F16 or BF16");
  if (!(std::fabs(cfg->scale) <= 3.0e38f)) return dfail(nullptr, FTDECAY_EINVAL, "scale is not finite");
  ftdecay_ctx* c = new (std::nothrow) ftdecay_ctx();
  if (!c) return dfail(nullptr, FTDECAY_ENOMEM, "out of host memory");
  c->cfg = *cfg;
  if (!(c->cfg.scale > 0.f)) c->cfg.scale = 1.0f / std::sqrt((float)cfg->head_dim);
  if (cfg->head_dim == 128) {
    if (cfg->in_dtype == FTDECAY_BF16) choose_kernels<128, true>(c);
    else choose_kernels<128, false>(c);
  } else {
    if (cfg->in_dtype == FTDECAY_BF16) choose_kernels<64, true>(c);
    else choose_kernels<64, false>(c);
  }
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) {
    he = hipFuncSetAttribute((const void*)c->chunks, hipFuncAttributeMaxDynamicSharedMemorySize, c->lds);
    if (he == hipSuccess) he = hipFuncSetAttribute((const void*)c->gather, hipFuncAttributeMaxDynamicSharedMemorySize, c->gather_lds);
    if (he == hipSuccess) he = hipMalloc((void**)&c->between, (size_t)2 * STATES * cfg->head_dim * cfg->head_dim * sizeof(float));
    (void)hipSetDevice(before);
  }
  if (he != hipSuccess) {
    const int rc = dfail_hip(nullptr, "device", he);
    delete c;
    return rc;
  }
  *out = c;
  return FTDECAY_OK;
}

extern "C" int ftdecay_get_config(const ftdecay_ctx* ctx, ftdecay_config* effective) {
  if (!ctx || !effective) return FTDECAY_EINVAL;
  *effective = ctx->cfg;
  return FTDECAY_OK;
}

// What both calls check; fills in their tensors.  nullptr: nothing is wrong.
static const char* wrong_rows(const ftdecay_rows* const (&all)[4], bool none, Rows (&r)[4], int& code) {
  code = FTDECAY_EINVAL;
  for (int i = 0; i < 4; ++i) {
    if (!all[i]) return "null argument";
    if ((!all[i]->data && !none) || ((uintptr_t)all[i]->data & 15)) return "tensors must be 16-byte aligned device pointers";
    if (((uintptr_t)all[i]->token_stride | (uintptr_t)all[i]->head_stride) % 8) return "strides must be whole 16-byte words";
    if (all[i]->token_stride < 0 || all[i]->head_stride < 0 || all[i]->token_stride > (1 << 24) || all[i]->head_stride > (1ll << 40)) {
      code = FTDECAY_EUNSUPPORTED;
      return "strides must be >= 0, and those of tokens at most 2^24 elements";
    }
    r[i] = Rows{static_cast<char*>(all[i]->data), all[i]->token_stride * 2, all[i]->head_stride * 2};
  }
  return nullptr;
}
static const char* wrong_states(const float* log_decay, const float* states, int32_t n_slots, const int32_t* slots, int32_t batch) {
  if (!log_decay) return "null argument";
  if ((uintptr_t)states & 15) return "states must be 16-byte aligned";
  if (((uintptr_t)log_decay | (uintptr_t)slots) & 3) return "arrays must be aligned to their elements";
  if (states && (n_slots < 0 || (!slots && batch > n_slots))) return "n_slots must be >= 0, and at least batch without slots";
  return nullptr;
}

// Groups of heads of an XCD, over all segments.
static uint32_t groups_of(const Args& a) { return (uint32_t)(((int64_t)(a.total / a.per + a.batch) * (a.heads / a.group) + 7) / 8); }

// One pass over the sequences: prompts in segments, single tokens (no cu) a workgroup each.
static int launch(ftdecay_ctx* c, const Args& a, hipStream_t st) {
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess && before != c->cfg.device) he = hipSetDevice(c->cfg.device);
  if (he != hipSuccess) return dfail_hip(c, "device", he);
  const int threads = 2 * c->cfg.head_dim;
  if (!a.cu) {
    hipLaunchKernelGGL(c->token, dim3((uint32_t)(a.batch * a.heads)), dim3(256), 0, st, a);
  } else {
    const dim3 grid(groups_of(a) * 8u * (uint32_t)a.group);
    if (a.total > a.per) {
      hipLaunchKernelGGL(c->gather, grid, dim3(threads), c->gather_lds, st, a);
      hipLaunchKernelGGL(c->join, dim3((uint32_t)(a.batch * a.heads * (c->cfg.head_dim * c->cfg.head_dim / 1024))), dim3(256), 0, st, a);
    }
    hipLaunchKernelGGL(c->chunks, grid, dim3(threads), c->lds, st, a);
  }
  he = hipGetLastError();
  if (before != c->cfg.device) (void)hipSetDevice(before);
  return he == hipSuccess ? FTDECAY_OK : dfail_hip(c, "launch", he);
}

extern "C" int ftdecay_forward(ftdecay_ctx* c, const ftdecay_rows* q, const ftdecay_rows* k, const ftdecay_rows* v, const ftdecay_rows* o, const float* log_decay, float* states,
                               int32_t n_slots, const int32_t* slots, const int32_t* cu, const int32_t* starts, int32_t batch, int32_t total, void* hip_stream) {
  if (!c) return FTDECAY_EINVAL;
  if (!cu) return dfail(c, FTDECAY_EINVAL, "null argument");
  if (batch < 1 || total < 0) return dfail(c, FTDECAY_EINVAL, "batch must be >= 1 and total >= 0");
  if (((uintptr_t)cu | (uintptr_t)starts) & 3) return dfail(c, FTDECAY_EINVAL, "arrays must be aligned to their elements");
  Rows r[4];
  int code;
  const char* bad = wrong_rows({q, k, v, o}, total == 0, r, code);
  if (bad) return dfail(c, code, bad);
  bad = wrong_states(log_decay, states, n_slots, slots, batch);
  if (bad) return dfail(c, FTDECAY_EINVAL, bad);
  const ftdecay_config& e = c->cfg;
  // Two workgroups a CU: 16,384 tokens of 32 heads of 128 take 194 us in 512 segments, 209 in 1024, which have twice as many states between them.
  int64_t per = ((int64_t)total * e.heads + 511) / 512;
  per = per < LEAST ? LEAST : per;
  const int64_t least = ((int64_t)total * e.heads + STATES - 1) / STATES;      // total / per * heads states between segments, at most STATES
  per = ((per > least ? per : least) + C - 1) / C * C;
  // workgroups of the launches: segments, blocks of joined states
  const int64_t segments = (total / per + batch) * e.heads, blocks = total > per ? (int64_t)batch * e.heads * (e.head_dim * e.head_dim / 1024) : 0;
  if (segments + 8 * (e.heads / e.kv_heads) > MOST_GROUPS || blocks > MOST_GROUPS) return dfail(c, FTDECAY_EUNSUPPORTED, "too many sequences");
  return launch(c, Args{r[0], r[1], r[2], r[3], log_decay, states, slots, cu, starts, n_slots, batch, total, e.heads, e.heads / e.kv_heads, e.scale, (int32_t)per, c->between},
                (hipStream_t)hip_stream);
}

extern "C" int ftdecay_step(ftdecay_ctx* c, const ftdecay_rows* q, const ftdecay_rows* k, const ftdecay_rows* v, const ftdecay_rows* o, const float* log_decay, float* states,
                            int32_t n_slots, const int32_t* slots, int32_t batch, void* hip_stream) {
  if (!c) return FTDECAY_EINVAL;
  if (batch < 0) return dfail(c, FTDECAY_EINVAL, "batch must be >= 0");
  if (batch == 0) return FTDECAY_OK;
  if (!states) return dfail(c, FTDECAY_EINVAL, "null argument");
  Rows r[4];
  int code;
  const char* bad = wrong_rows({q, k, v, o}, false, r, code);
  if (bad) return dfail(c, code, bad);
  bad = wrong_states(log_decay, states, n_slots, slots, batch);
  if (bad) return dfail(c, FTDECAY_EINVAL, bad);
  const ftdecay_config& e = c->cfg;
  if ((int64_t)batch * e.heads > MOST_GROUPS) return dfail(c, FTDECAY_EUNSUPPORTED, "too many sequences");
  return launch(c, Args{r[0], r[1], r[2], r[3], log_decay, states, slots, nullptr, nullptr, n_slots, batch, batch, e.heads, e.heads / e.kv_heads, e.scale, C, nullptr}, (hipStream_t)hip_stream);
}

extern "C" int ftdecay_destroy(ftdecay_ctx* c) {
  if (!c) return FTDECAY_OK;
  int before = 0;
  const bool moved = hipGetDevice(&before) == hipSuccess && before != c->cfg.device && hipSetDevice(c->cfg.device) == hipSuccess;
  (void)hipFree(c->between);
  if (moved) (void)hipSetDevice(before);
  delete c;
  return FTDECAY_OK;
}

extern "C" const char* ftdecay_last_error(const ftdecay_ctx* c) { return c ? c->err.c_str() : g_decay_create_err.c_str(); }
