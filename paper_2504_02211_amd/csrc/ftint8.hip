// Linear layer on 8-bit integers: the kernels and the C ABI of ../include/ftint8.h.
#include "ftint8.h"
#include "ftserve_device.h"

#include <new>
#include <string>
#include <type_traits>
#include <utility>

namespace ftint8 {
using namespace ftserve;

typedef int int4v __attribute__((ext_vector_type(4)));

constexpr int KEXTRA = 128;            // rows of codes are a multiple of this
constexpr int MOST_K = 130944;         // 128 * 128 products of as many codes stay below 2^31

template <int DT> __device__ __forceinline__ float element(const void* row, int64_t i) {
  if constexpr (DT == FTINT8_BF16) return as_f((uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
  else return (float)reinterpret_cast<const _Float16*>(row)[i];
}

struct EncodeArgs {
  const char* x;
  int64_t stride;      // bytes
  int32_t k, k_padded, rows;
  int8_t* codes;
  float* scales;
};

// How the rows of one call are encoded, from the largest magnitude (as its bits) on: infinity and NaN are above all numbers.  Rows below 2^-100 are taken times
// 2^100, where the reciprocal stays finite.
struct Coding {
  float up, inverse;
  bool fine;
  __device__ __forceinline__ explicit Coding(uint32_t most) {
    fine = most < 0x7F800000u;
    up = as_f(most) < 0x1p-100f ? 0x1p100f : 1.f;
    inverse = most == 0 || !fine ? 0.f : 127.f * (1.f / (as_f(most) * up));
  }
  // The code in the lowest byte.  (The sum with 1.5 * 2^23 rounds to a whole number, ties to even; the product is rounded before it: no fused instruction.)
  __device__ __forceinline__ uint32_t code(float x) const {
    float y = x * up * inverse;
    asm("" : "+v"(y));
    return as_u(y + 12582912.f);
  }
  // Eight codes of eight elements in 16 bits.
  template <bool BF> __device__ __forceinline__ uint2v codes(const uint4v& v) const {
    uint2v out;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint32_t lo = v[2 * w], hi = v[2 * w + 1];
      const uint32_t c0 = code(low_of<BF>(lo)), c1 = code(high_of<BF>(lo)), c2 = code(low_of<BF>(hi)), c3 = code(high_of<BF>(hi));
      out[w] = fine ? __builtin_amdgcn_perm(c1, c0, 0x0C0C0400u) | __builtin_amdgcn_perm(c3, c2, 0x04000C0Cu) : 0u;
    }
    return out;
  }
};
__device__ __forceinline__ void put_scale(const EncodeArgs& a, int row, uint32_t most, bool fine) { a.scales[row] = fine ? as_f(most) / 127.f : __builtin_nanf(""); }

__device__ __forceinline__ uint32_t largest_of_wave(uint32_t x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const uint32_t y = __shfl_xor(x, d);
    x = y > x ? y : x;
  }
  return x;
}

// Rows that begin anywhere, or are longer than the registers of a workgroup: a row a workgroup, element after element, read twice.  4096 rows of 4001 elements take
// 25 us (of 4000, as below, 8.7), of 28,672 196 us (of 16,384 31).
template <int DT> __global__ __launch_bounds__(256) void ftint8_encode_any(const EncodeArgs a) {
  __shared__ uint32_t most_of[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  const char* const x = a.x + (int64_t)row * a.stride;
  uint32_t most = 0;
  for (int i = tid; i < a.k; i += 256) {
    const uint32_t u = as_u(element<DT>(x, i)) & 0x7FFFFFFFu;
    most = u > most ? u : most;
  }
  most = largest_of_wave(most);
  if ((tid & 63) == 0) most_of[tid >> 6] = most;
  __syncthreads();
  for (int w = 0; w < 4; ++w) most = most_of[w] > most ? most_of[w] : most;
  const Coding c(most);
  if (tid == 0) put_scale(a, row, most, c.fine);
  int8_t* const codes = a.codes + (int64_t)row * a.k_padded;
  for (int i = tid; i < a.k_padded; i += 256) codes[i] = i < a.k && c.fine ? (int8_t)c.code(element<DT>(x, i)) : (int8_t)0;
}

// Rows that begin at multiples of 16 bytes: WAVES waves hold a row in their registers, 8 elements in each of VECS words of a lane, from the one read to the write.
// Bound: memory.
template <int DT, int WAVES, int VECS> __global__ __launch_bounds__(256) void ftint8_encode_rows(const EncodeArgs a) {
  __shared__ uint32_t most_of[4];
  const int wave = threadIdx.x >> 6, t = threadIdx.x % (64 * WAVES), row = blockIdx.x * (4 / WAVES) + wave / WAVES;
  const bool on = row < a.rows;
  const char* const x = a.x + (int64_t)(on ? row : a.rows - 1) * a.stride;
  uint4v v[VECS];
  uint32_t most16 = 0;      // (of the magnitudes' 16 bits, which are ordered as the numbers are)
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int at = 8 * (t + 64 * WAVES * i);
    v[i] = (uint4v)0u;
    if (at + 8 <= a.k) v[i] = *reinterpret_cast<const uint4v*>(x + 2 * at);
    else if (at < a.k)
      for (int e = 0; e < a.k - at; ++e) v[i][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(x)[at + e] << 16 * (e & 1);
  }
#pragma unroll
  for (int i = 0; i < VECS; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w)
      most16 = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, most16), __builtin_bit_cast(ushort2v, v[i][w] & 0x7FFF7FFFu)));
  most16 = (most16 & 0xFFFFu) > most16 >> 16 ? most16 & 0xFFFFu : most16 >> 16;
  most16 = largest_of_wave(most16);
  if constexpr (WAVES == 4) {
    if ((threadIdx.x & 63) == 0) most_of[wave] = most16;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) most16 = most_of[w] > most16 ? most_of[w] : most16;
  }
  if (!on) return;
  const uint32_t most = as_u(low_of<DT == FTINT8_BF16>(most16));
  const Coding c(most);
  if (t == 0) put_scale(a, row, most, c.fine);
  int8_t* const codes = a.codes + (int64_t)row * a.k_padded;
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int at = 8 * (t + 64 * WAVES * i);
    if (at < a.k_padded) *reinterpret_cast<uint2v*>(codes + at) = c.codes<DT == FTINT8_BF16>(v[i]);
  }
}

struct ProductArgs {
  const int8_t *x, *w;
  const float *sx, *sw;
  char* y;
  int64_t y_stride;      // bytes
  int32_t m, n, k_padded;
  int32_t parts;         // > 1: the columns are divided among as many workgroups a tile (blockIdx.y), whose sums go to `sums`
  int4v* sums;           // [part][tile][wave][block of features][block of tokens][lane]
};

template <int N> __device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
}
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");      // (nor does anything behind it move before it)
  __builtin_amdgcn_sched_barrier(0);
}
// 16 bytes per lane from (uniform base + per-lane byte offset) straight into LDS at (uniform LDS address + 16 * lane).  (Opaque to the compiler, which would wait
// for the stage in flight before it reads another.  The wait covers a base that a vector instruction has moved to its scalar registers just before: five states.  It does not say
// that it writes memory, so that reads of LDS may be scheduled around it: what is loaded is read behind a counted wait and a barrier, what it overwrites was read before
// one, and these let nothing pass.  Were it to say so, 16,384 tokens on 16,384 x 4096 would take 1008 us, not 1000.)
__device__ __forceinline__ void load_lds16(const void* base, uint32_t off, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds_addr) : "m0");
}
// f(0), f(1), ... f(N - 1) with the index as a compile-time constant
template <class F, int... I> __device__ __forceinline__ void for_each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F> __device__ __forceinline__ void for_each(F&& f) { for_each_of(f, std::make_integer_sequence<int, N>{}); }

// A wide store to an address that is aligned to an element only.  (The device's vector stores take any.  Rows of 4001 results, stored an element at a time, take the product of
// 4000 tokens on 4001 x 4096 from 54 us to 72.)
template <int ES, class V> __device__ __forceinline__ void put_anywhere(char* to, V v) {
  struct __attribute__((packed, aligned(ES))) Loose { V v; };
  reinterpret_cast<Loose*>(to)->v = v;
}
// A result: the sum rounded to 32 bits, times the product of the scales.
__device__ __forceinline__ float scaled(int sum, float sx, float sw) {
  float y = (float)sum * (sx * sw);
  asm("" : "+v"(y));      // (rounded to 32 bits: the compiler would make one instruction of this product and its rounding to 16)
  return y;
}

// Tile shape: BM tokens x BF features, a wave takes WT x WF blocks of 16 x 16, a ring of NST stages of 128 columns, PER_CU workgroups to a CU.
template <int BM_, int BF_, int WT_, int WF_, int NST_, int PER_CU_ = 1> struct Tile {
  static constexpr int BM = BM_, BF = BF_, WT = WT_, WF = WF_, NST = NST_, PER_CU = PER_CU_;
  static constexpr int NWT = BM / (16 * WT), NWF = BF / (16 * WF), NW = NWT * NWF;      // waves along the tokens and along the features
  static constexpr int BK = 128, STAGE = (BM + BF) * BK, LDS = NST * STAGE;
  static constexpr int XP = BM / 8, WP = BF / 8;                                         // pieces of 8 rows, 1 KB
  static_assert(XP % NW == 0 && WP % NW == 0 && (NW == 4 || NW == 8), "pieces split evenly");
  static constexpr int XW = XP / NW, WW = WP / NW, NLOAD = XW + WW;                      // ... of a wave
  static constexpr int PITCH = 16 * WF * 4 + 16;                                         // of a row of results on its way through LDS
  static_assert(NW * 16 * PITCH <= LDS && PER_CU * LDS <= 160 * 1024 && (NST - 1) * NLOAD <= 63, "LDS; counted waits");
};

// Which tile a workgroup has.  Workgroups go round the 8 XCDs; each XCD gets neighbouring tiles, numbered in groups of 8 token tiles x all feature tiles, so that
// what it runs at a time shares rows of weights and of tokens in its L2.
template <class T> __device__ __forceinline__ void tile_of(const ProductArgs& a, int id, int& tm, int& tn) {
  constexpr int GM = 8;
  const int tiles_m = (a.m + T::BM - 1) / T::BM, tiles_n = (a.n + T::BF - 1) / T::BF;
  const int total = tiles_m * tiles_n, xcd = id & 7, slot = id >> 3, per = total >> 3, more = total & 7;
  const int t = xcd * per + (xcd < more ? xcd : more) + slot;
  const int group = t / (GM * tiles_n), first = group * GM, rows = tiles_m - first < GM ? tiles_m - first : GM, in = t - group * GM * tiles_n;
  tm = __builtin_amdgcn_readfirstlane(first + in % rows);
  tn = __builtin_amdgcn_readfirstlane(in / rows);
}

// Y^T = W X^T on 16x16x64 products: rows of weights are the left operand, tokens the right one, so that a lane holds one token per block of tokens and four features that lie
// side by side per block of features.  The steps of 128 columns go through a ring of LDS stages that direct loads fill; a row's 16-byte chunk c lies at place c ^ (row / 2 % 8), which keeps
// the reads of operands free of bank conflicts.  Operands are read ahead of their products, also across the border of two stages: the barrier of a stage sits AHEAD rows of
// products before its end, where its last operands are in registers, so that no wave waits for LDS behind it.
// Bound by power (the clock falls to some 1.8 GHz, the matrix pipe is 60 % busy): 16,384 tokens on 16,384 x 4096 (features x columns) 908 us, 2420 TOPS, one behind another (the first ones of a cold card 967 to 1050); the library's
// plain product of the codes, without scales, 974 us.
template <class T, int DT> __global__ __launch_bounds__(T::NW * 64, T::PER_CU * T::NW / 4) void ftint8_tile(const ProductArgs a) {
  constexpr int WT = T::WT, WF = T::WF, NST = T::NST, BK = T::BK, STAGE = T::STAGE, NLOAD = T::NLOAD, NKS = 2, AHEAD = 3;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wt = wave / T::NWF, wf = wave % T::NWF;
  int tm, tn;
  tile_of<T>(a, blockIdx.x, tm, tn);
  const int m0 = tm * T::BM, n0 = tn * T::BF;
  const int begin = a.k_padded / BK * (int)blockIdx.y / a.parts, steps = a.k_padded / BK * ((int)blockIdx.y + 1) / a.parts - begin;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

  // Piece p of an operand is its rows 8p .. 8p + 7; wave w takes pieces w, w + NW, ...  Rows behind the last one are the last one again (their results are not used).
  auto swizzle = [](int row) __attribute__((always_inline)) { return row >> 1 & 7; };
  const int chunk = (lane & 7) ^ swizzle(8 * wave + (lane >> 3));
  uint32_t off[NLOAD];
#pragma unroll
  for (int i = 0; i < NLOAD; ++i) {
    const int left = i < T::XW ? a.m - m0 : a.n - n0;
    int r = 8 * (wave + T::NW * (i < T::XW ? i : i - T::XW)) + (lane >> 3);
    r = r < left ? r : left - 1;
    off[i] = (uint32_t)r * (uint32_t)a.k_padded + 16u * chunk;
  }
  const int8_t *xb = a.x + (int64_t)m0 * a.k_padded + begin * BK, *wb = a.w + (int64_t)n0 * a.k_padded + begin * BK;
  const uint32_t wave_at = base + (uint32_t)wave * 1024u;
  auto issue = [&](int i, uint32_t stage) __attribute__((always_inline)) {
    load_lds16(i < T::XW ? xb : wb, off[i], wave_at + stage + (uint32_t)((i < T::XW ? T::NW * i : T::XP + T::NW * (i - T::XW)) * 1024));
  };
  auto next_step = [&]() __attribute__((always_inline)) { xb += BK; wb += BK; };

  int4v acc[WF][WT];
#pragma unroll
  for (int f = 0; f < WF; ++f)
#pragma unroll
    for (int t = 0; t < WT; ++t) acc[f][t] = (int4v)0;

  const uint32_t lane_at = base + (uint32_t)(lq * BK + ((lg ^ swizzle(lq)) << 4));
  const uint32_t xrow = lane_at + (uint32_t)(16 * WT * wt * BK), wrow = lane_at + (uint32_t)((T::BM + 16 * WF * wf) * BK);
  auto read = [](uint32_t at) __attribute__((always_inline)) { return *(const __attribute__((address_space(3))) int4v*)(uintptr_t)at; };
  // Operands in registers: tokens of two half-steps of 64 columns (one in use, one on its way), a ring of four blocks of weights.
  int4v xr[2][WT], wr[4];
  static_assert(WF >= AHEAD + 1 && (NKS * WF) % 4 == 0, "operand rings");
  auto read_x = [&](int ks, int t, uint32_t stage) __attribute__((always_inline)) { xr[ks & 1][t] = read(((xrow + stage) ^ (uint32_t)(ks << 6)) + t * 16 * BK); };
  auto read_w = [&](int p, uint32_t stage) __attribute__((always_inline)) { wr[p & 3] = read(((wrow + stage) ^ (uint32_t)(p / WF << 6)) + p % WF * 16 * BK); };
  // keeps `n` LDS reads behind the product they were written after
  auto pin = [](int n) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (n == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    else if (n == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    else if (n == 3) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
  };
#pragma unroll
  for (int st = 0; st < NST; ++st)
    if (st < steps) {
#pragma unroll
      for (int i = 0; i < NLOAD; ++i) issue(i, (uint32_t)(st * STAGE));
      next_step();
    }
  if (steps < NST) wait_loads<0>();
  else wait_loads<(NST - 1) * NLOAD>();
  barrier();
  uint32_t stage = 0;
  auto row_step = [&](auto row_tag, uint32_t stage, uint32_t next, auto load_tag) __attribute__((always_inline)) {
    constexpr bool LOAD = decltype(load_tag)::value;
    constexpr int ks = decltype(row_tag)::value / WF, y = decltype(row_tag)::value % WF;
    constexpr bool last = ks == NKS - 1, tail = last && y >= WF - AHEAD;
    constexpr int rows = last ? AHEAD : WF, r = last ? y - (WF - AHEAD) : y;
    constexpr int x0 = last && !tail ? 0 : WT * r / rows, x1 = last && !tail ? 0 : WT * (r + 1) / rows;      // operands of the next half-step that are read here
    int reads[WT];
#pragma unroll
    for (int m = 0; m < WT; ++m) {
      acc[y][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[(ks * WF + y) & 3], xr[ks & 1][m], acc[y][m], 0, 0, 0);
      int n = 0;
      constexpr int p = ks * WF + y + AHEAD;
      if (m == 0) { read_w(p % (NKS * WF), p < NKS * WF ? stage : next); ++n; }
      if (WT == 1) { if (x0 < x1) { read_x((ks + 1) % NKS, 0, last ? next : stage); ++n; } }
      else if (m >= 1 && x0 + m - 1 < x1) { read_x((ks + 1) % NKS, x0 + m - 1, last ? next : stage); ++n; }
      reads[m] = n;
      if (LOAD && tail) {
        constexpr int TAIL = AHEAD * WT;
        const int q = (y - (WF - AHEAD)) * WT + m;
#pragma unroll
        for (int i = NLOAD * q / TAIL; i < NLOAD * (q + 1) / TAIL; ++i) issue(i, stage);
      }
    }
#pragma unroll
    for (int m = 0; m < WT; ++m) pin(reads[m]);
  };
  auto stage_step = [&](int kb, auto load_tag) __attribute__((always_inline)) {
    constexpr bool LOAD = decltype(load_tag)::value;
    const uint32_t next = stage == (uint32_t)((NST - 1) * STAGE) ? 0u : stage + (uint32_t)STAGE;
    for_each<NKS * WF - AHEAD>([&](auto row) __attribute__((always_inline)) { row_step(row, stage, next, load_tag); });
    wait_lds();                            // the operands of the last rows are in registers: this wave is done with the stage
    if (LOAD || kb + NST - 1 < steps) wait_loads<(NST - 2) * NLOAD>();      // the next stage has landed; younger ones may be in flight
    else wait_loads<0>();
    barrier();                             // ... everyone's pieces of it, and everyone is done with this one
    for_each<AHEAD>([&](auto row) __attribute__((always_inline)) {
      row_step(std::integral_constant<int, NKS * WF - AHEAD + decltype(row)::value>{}, stage, next, load_tag);
    });
    if (LOAD) next_step();
    stage = next;
  };
#pragma unroll
  for (int t = 0; t < WT; ++t) read_x(0, t, 0u);
#pragma unroll
  for (int p = 0; p < AHEAD; ++p) read_w(p, 0u);
  int kb = 0;
  for (; kb + NST < steps; ++kb) stage_step(kb, std::true_type{});
  for (; kb < steps; ++kb) stage_step(kb, std::false_type{});
  if (a.parts > 1) {
    int4v* const to = a.sums + (((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * T::NW + wave) * (WF * WT * 64) + lane;
#pragma unroll
    for (int f = 0; f < WF; ++f)
#pragma unroll
      for (int t = 0; t < WT; ++t) to[(f * WT + t) * 64] = acc[f][t];
    return;
  }
  wait_lds();
  barrier();                               // the ring is free

  // Results go through LDS, a block of 16 tokens at a time, so that a wave stores whole rows.
  constexpr int ES = DT == FTINT8_F32 ? 4 : 2, PER = 16 / ES, LPR = 16 * WF / PER, RPI = 64 / LPR > 16 ? 16 : 64 / LPR;      // elements of a store; lanes of a row; rows of a store
  char* const out = smem + wave * 16 * T::PITCH;
  const int nf0 = n0 + 16 * WF * wf, mt0 = m0 + 16 * WT * wt;
  float sw[WF][4];
#pragma unroll
  for (int f = 0; f < WF; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int col = nf0 + 16 * f + 4 * lg + r;
      sw[f][r] = a.sw[col < a.n ? col : a.n - 1];
    }
#pragma unroll
  for (int t = 0; t < WT; ++t) {
    const int mine = mt0 + 16 * t + lq;
    const float sx = a.sx[mine < a.m ? mine : a.m - 1];
#pragma unroll
    for (int f = 0; f < WF; ++f) {
      float y[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = scaled(acc[f][t][r], sx, sw[f][r]);
      char* const at = out + lq * T::PITCH + (16 * f + 4 * lg) * ES;
      if constexpr (ES == 4) *reinterpret_cast<float4v*>(at) = float4v{y[0], y[1], y[2], y[3]};
      else *reinterpret_cast<uint2v*>(at) = uint2v{pack2<DT == FTINT8_BF16>(y[0], y[1]), pack2<DT == FTINT8_BF16>(y[2], y[3])};
    }
    const int r0 = mt0 + 16 * t;
    const int col = nf0 + lane % LPR * PER;
#pragma unroll
    for (int i = 0; i < 16 / RPI; ++i) {
      const int r = i * RPI + lane / LPR;
      const uint4v v = *reinterpret_cast<const uint4v*>(out + (r & 15) * T::PITCH + lane % LPR * 16);
      if (lane / LPR >= RPI || r0 + r >= a.m || col >= a.n) continue;
      char* const to = a.y + (int64_t)(r0 + r) * a.y_stride + col * ES;
      if (col + PER <= a.n) put_anywhere<ES>(to, v);
      else
        for (int e = 0; e < a.n - col; ++e) {
          if constexpr (ES == 4) reinterpret_cast<uint32_t*>(to)[e] = v[e];
          else reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(v[e >> 1] >> 16 * (e & 1));
        }
    }
    __builtin_amdgcn_sched_barrier(0);      // (one block's results at a time out of the accumulators)
  }
}

// Four features of one token out: the lane has them side by side.
template <int DT> __device__ __forceinline__ void put_four(const ProductArgs& a, int row, int col, int4v sum, float sx) {
  float y[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = scaled(sum[r], sx, a.sw[col + r < a.n ? col + r : a.n - 1]);
  constexpr int ES = DT == FTINT8_F32 ? 4 : 2;
  char* const to = a.y + (int64_t)row * a.y_stride + (int64_t)col * ES;
  if (col + 4 <= a.n) {
    if constexpr (ES == 4) put_anywhere<ES>(to, float4v{y[0], y[1], y[2], y[3]});
    else put_anywhere<ES>(to, uint2v{pack2<DT == FTINT8_BF16>(y[0], y[1]), pack2<DT == FTINT8_BF16>(y[2], y[3])});
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (col + r < a.n) {
        if constexpr (ES == 4) reinterpret_cast<float*>(to)[r] = y[r];
        else reinterpret_cast<uint16_t*>(to)[r] = (uint16_t)pack2<DT == FTINT8_BF16>(y[r], y[r]);
      }
  }
}

// The shares of divided columns, added up: a wave a block of 16 x 16.
template <class T, int DT> __global__ __launch_bounds__(256) void ftint8_finish(const ProductArgs a, int tiles) {
  constexpr int BLOCKS = T::NW * T::WF * T::WT;
  const int lane = threadIdx.x & 63, unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), id = unit / BLOCKS, block = unit % BLOCKS;
  if (id >= tiles) return;
  int tm, tn;
  tile_of<T>(a, id, tm, tn);
  const int wave = block / (T::WF * T::WT), f = block / T::WT % T::WF, t = block % T::WT, wt = wave / T::NWF, wf = wave % T::NWF;
  const int row = tm * T::BM + 16 * (T::WT * wt + t) + (lane & 15), col = tn * T::BF + 16 * (T::WF * wf + f) + 4 * (lane >> 4);
  if (row >= a.m || col >= a.n) return;
  const int4v* const from = a.sums + ((int64_t)id * BLOCKS + block) * 64 + lane;
  const int64_t apart = (int64_t)tiles * BLOCKS * 64;
  int4v sum = from[0];
  for (int p = 1; p < a.parts; ++p) sum += from[p * apart];
  put_four<DT>(a, row, col, sum, a.sx[row]);
}

// Few tokens: 16 features and all tokens (up to 16 TB) a workgroup, the columns divided among its eight waves, operands from memory straight into registers: every
// byte of the weights is wanted by one wave alone.  Stages of 256 columns, two of them under way; a token on 4096 columns has all it needs under way at once, and all
// workgroups of 16,384 features are on the chip together.  WORDS > 0 (up to TOKENS tokens of up to 4096 WORDS columns): they come in 16 bits, every workgroup encodes them for
// itself while its first weights are under way, and the second launch is saved.  Bound by memory: 67 MB of weights, one token on 16,384 features of 4096 columns,
// take 12.7 us with the encoding (5.3 TB/s; 15.0 in two launches).
constexpr int FEW_WAVES = 8, FUSED_K = 16384, FUSED_TOKENS = 4;
struct FewArgs {
  ProductArgs p;
  const char* raw;         // tokens in 16 bits, at multiples of 16 bytes
  int64_t raw_stride;      // bytes
  int32_t k;
};
template <int TB, int DT, int IN, int TOKENS, int WORDS> __global__ __launch_bounds__(FEW_WAVES * 64, WORDS == 1 ? TOKENS == 1 ? 8 : 6 : 2) void ftint8_few(const FewArgs b) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ uint32_t most_of[TOKENS][FEW_WAVES];
  constexpr bool FUSED = WORDS > 0;
  constexpr int U = 4;
  const ProductArgs& a = b.p;
  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 15, lg = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16, steps = a.k_padded / 64, stages = (steps + U - 1) / U;
  const int8_t* const wp = a.w + (int64_t)(n0 + lq < a.n ? n0 + lq : a.n - 1) * a.k_padded + 16 * lg;
  const int8_t* xp[TB];
#pragma unroll
  for (int t = 0; t < TB; ++t) xp[t] = a.x + (int64_t)(16 * t + lq < a.m ? 16 * t + lq : a.m - 1) * a.k_padded + 16 * lg;
  const int pitch = a.k_padded + 64;      // (four rows' words lie in different banks)
  const uint32_t row_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem + 16u * lg + (TOKENS > 1 ? (uint32_t)((lq < a.m ? lq : a.m - 1) * pitch) : 0u);

  // the tokens first: what is asked for last is waited for last
  uint4v raw[TOKENS][FUSED ? WORDS : 1];
  if constexpr (FUSED) {
#pragma unroll
    for (int t = 0; t < TOKENS; ++t)
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const int at = 8 * (tid + 512 * i);
        const char* const from = b.raw + t * b.raw_stride;
        raw[t][i] = (uint4v)0u;
        if (t > 0 && t >= a.m) continue;
        if (at + 8 <= b.k) raw[t][i] = *reinterpret_cast<const uint4v*>(from + 2 * at);
        else if (at < b.k)
          for (int e = 0; e < b.k - at; ++e) raw[t][i][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(from)[at + e] << 16 * (e & 1);
      }
  }
  int4v acc[TB], wr[2][U], xr[2][FUSED ? 1 : TB][U];
#pragma unroll
  for (int t = 0; t < TB; ++t) acc[t] = (int4v)0;
  auto fetch = [&](int to, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = stage * U + u < steps ? stage * U + u : steps - 1;      // (what is fetched twice is not multiplied twice)
      wr[to][u] = *reinterpret_cast<const int4v*>(wp + 64 * s);
      if constexpr (!FUSED)
#pragma unroll
        for (int t = 0; t < TB; ++t) xr[to][t][u] = *reinterpret_cast<const int4v*>(xp[t] + 64 * s);
    }
  };
  int stage = wave;
  if (stage < stages) fetch(0, stage);
  if (stage + FEW_WAVES < stages) fetch(1, stage + FEW_WAVES);
  float sx = 0.f;
  if constexpr (FUSED) {
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < WORDS; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w)
          most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, most), __builtin_bit_cast(ushort2v, raw[t][i][w] & 0x7FFF7FFFu)));
      most = (most & 0xFFFFu) > most >> 16 ? most & 0xFFFFu : most >> 16;
      most = largest_of_wave(most);
      if (lane == 0) most_of[t][wave] = most;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      if (t > 0 && t >= a.m) break;
      uint32_t most = 0;
#pragma unroll
      for (int w = 0; w < FEW_WAVES; ++w) most = most_of[t][w] > most ? most_of[t][w] : most;
      most = as_u(low_of<IN == FTINT8_BF16>(most));
      const Coding c(most);
      if (TOKENS == 1 || lq == t) sx = c.fine ? as_f(most) / 127.f : __builtin_nanf("");
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        const int at = 8 * (tid + 512 * i);
        if (at < a.k_padded) *reinterpret_cast<uint2v*>(smem + t * pitch + at) = c.codes<IN == FTINT8_BF16>(raw[t][i]);
      }
    }
    __syncthreads();
  } else if (tid < 64 * TB) {
    const int r = 16 * (tid >> 6) + lq;
    sx = a.sx[r < a.m ? r : a.m - 1];
  }
  auto multiply = [&](int from, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (stage * U + u < steps)
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          int4v x;
          if constexpr (FUSED) x = *(const __attribute__((address_space(3))) int4v*)(uintptr_t)(row_at + 64u * (stage * U + u));
          else x = xr[from][t][u];
          acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wr[from][u], x, acc[t], 0, 0, 0);
        }
  };
  while (stage < stages) {
    multiply(0, stage);
    if (stage + 2 * FEW_WAVES < stages) fetch(0, stage + 2 * FEW_WAVES);
    stage += FEW_WAVES;
    if (stage >= stages) break;
    multiply(1, stage);
    if (stage + 2 * FEW_WAVES < stages) fetch(1, stage + 2 * FEW_WAVES);
    stage += FEW_WAVES;
  }
  // the waves' sums, added up by the first TB of them
  if constexpr (FUSED) __syncthreads();
  int4v* const parts = reinterpret_cast<int4v*>(smem);
#pragma unroll
  for (int t = 0; t < TB; ++t) parts[(wave * TB + t) * 64 + lane] = acc[t];
  __syncthreads();
  if (wave >= TB) return;
  int4v sum = parts[wave * 64 + lane];
#pragma unroll
  for (int w = 1; w < FEW_WAVES; ++w) sum += parts[(w * TB + wave) * 64 + lane];
  const int row = 16 * wave + lq, col = n0 + 4 * lg;
  if (row >= a.m) return;
  if (col < a.n) put_four<DT>(a, row, col, sum, sx);
}

typedef void (*encode_fn)(const EncodeArgs);
typedef void (*product_fn)(const ProductArgs);
typedef void (*few_fn)(const FewArgs);
template <int DT> few_fn few_of(bool two) { return two ? ftint8_few<2, DT, 0, 1, 0> : ftint8_few<1, DT, 0, 1, 0>; }
template <int DT, int IN> few_fn fused_of(bool several, bool wide) {
  return several ? ftint8_few<1, DT, IN, FUSED_TOKENS, 1> : wide ? ftint8_few<1, DT, IN, 1, 4> : ftint8_few<1, DT, IN, 1, 1>;
}
template <int DT> few_fn fused_of(bool bf, bool several, bool wide) { return bf ? fused_of<DT, FTINT8_BF16>(several, wide) : fused_of<DT, FTINT8_F16>(several, wide); }
constexpr int few_lds(int blocks) { return FEW_WAVES * blocks * 64 * 16; }

// The kernel for rows of k_padded codes; per: rows of a workgroup.  Rows of up to 2048 elements take a wave each, of up to 16384 a workgroup.
template <int DT> encode_fn encode_of(int k_padded, bool whole, int& per) {
  if (!whole || k_padded > 16384) return ftint8_encode_any<DT>;
  if (k_padded <= 2048) {
    per = 4;
    return k_padded <= 512 ? ftint8_encode_rows<DT, 1, 1> : k_padded <= 1024 ? ftint8_encode_rows<DT, 1, 2> : ftint8_encode_rows<DT, 1, 4>;
  }
  return k_padded <= 4096 ? ftint8_encode_rows<DT, 4, 2> : k_padded <= 8192 ? ftint8_encode_rows<DT, 4, 4> : ftint8_encode_rows<DT, 4, 8>;
}

enum { WIDE, HALF, QUARTER, SMALL, N_TILES };
using TileWide = Tile<256, 256, 4, 8, 2>;
using TileHalf = Tile<128, 256, 4, 4, 3>;
using TileQuarter = Tile<64, 256, 2, 4, 3>;
using TileSmall = Tile<64, 128, 2, 4, 3, 2>;
struct TileInfo { int bm, bf, threads, lds; };
template <class T> constexpr TileInfo info_of() { return {T::BM, T::BF, T::NW * 64, T::LDS}; }
constexpr TileInfo TILES[N_TILES] = {info_of<TileWide>(), info_of<TileHalf>(), info_of<TileQuarter>(), info_of<TileSmall>()};
typedef void (*finish_fn)(const ProductArgs, int);
template <int DT> product_fn tile_kernel(int tile) {
  return tile == WIDE ? ftint8_tile<TileWide, DT> : tile == HALF ? ftint8_tile<TileHalf, DT> : tile == QUARTER ? ftint8_tile<TileQuarter, DT> : ftint8_tile<TileSmall, DT>;
}
// Shares of divided columns (stages of TileSmall::BK): at most as many at a time, tiles times parts.
constexpr int most_shares(int stages) { return stages < 64 ? 4 * stages : 256; }
// Their room in a context: none where there are too few columns to divide, or tiles enough for any number of tokens.
constexpr size_t sums_bytes(int n, int stages) {
  return stages < 16 || 2 * ((n + TileSmall::BF - 1) / TileSmall::BF) > most_shares(stages) ? 0 : (size_t)most_shares(stages) * TileSmall::BM * TileSmall::BF * 4;
}

}  // namespace ftint8

using namespace ftint8;

struct ftint8_ctx {
  ftint8_config cfg;
  int k_padded = 0;
  product_fn product[N_TILES] = {};
  finish_fn finish = nullptr;
  int4v* sums = nullptr;
  few_fn few[2] = {}, fused[2] = {};
  int8_t* codes = nullptr;       // of the tokens of a forward, and their scales behind them
  float* scales = nullptr;
  std::string err;
};

static thread_local std::string g_int8_create_err;

static int ifail(ftint8_ctx* c, int code, const char* msg) {
  try {
    (c ? c->err : g_int8_create_err) = msg;
  } catch (...) {
  }
  return code;
}
static int ifail_hip(ftint8_ctx* c, const char* what, hipError_t e) {
  try {
    (c ? c->err : g_int8_create_err) = std::string(what) + ": " + hipGetErrorString(e);
  } catch (...) {
  }
  return e == hipErrorOutOfMemory ? FTINT8_ENOMEM : FTINT8_EHIP;
}

extern "C" int ftint8_create(const ftint8_config* cfg, ftint8_ctx** out) {
  if (!cfg || !out) return ifail(nullptr, FTINT8_EINVAL, "null argument");
  *out = nullptr;
  if (cfg->struct_size != sizeof(ftint8_config)) return ifail(nullptr, FTINT8_EINVAL, "struct_size mismatch");
  if (cfg->n < 1 || cfg->k < 1) return ifail(nullptr, FTINT8_EINVAL, "n and k must be >= 1");
  if (cfg->k > MOST_K) return ifail(nullptr, FTINT8_EUNSUPPORTED, "k above 130944: sums could leave 32 bits");
  if (cfg->n > 1 << 24) return ifail(nullptr, FTINT8_EUNSUPPORTED, "n above 2^24");
  if (cfg->in_dtype != FTINT8_F16 && cfg->in_dtype != FTINT8_BF16) return ifail(nullptr, FTINT8_EINVAL, "in_dtype must be F16 or BF16");
  if (cfg->out_dtype != FTINT8_F32 && cfg->out_dtype != cfg->in_dtype) return ifail(nullptr, FTINT8_EINVAL, "out_dtype must be F32 or the input type");
  if (cfg->max_tokens < 1 || cfg->max_tokens > 1 << 22) return ifail(nullptr, FTINT8_EINVAL, "max_tokens must be 1 .. 2^22");
  ftint8_ctx* c = new (std::nothrow) ftint8_ctx();
  if (!c) return ifail(nullptr, FTINT8_ENOMEM, "out of host memory");
  c->cfg = *cfg;
  c->k_padded = (cfg->k + KEXTRA - 1) / KEXTRA * KEXTRA;
  for (int t = 0; t < N_TILES; ++t)
    c->product[t] = cfg->out_dtype == FTINT8_F32 ? tile_kernel<FTINT8_F32>(t) : cfg->out_dtype == FTINT8_BF16 ? tile_kernel<FTINT8_BF16>(t) : tile_kernel<FTINT8_F16>(t);
  c->finish = cfg->out_dtype == FTINT8_F32 ? ftint8_finish<TileSmall, FTINT8_F32> : cfg->out_dtype == FTINT8_BF16 ? ftint8_finish<TileSmall, FTINT8_BF16> : ftint8_finish<TileSmall, FTINT8_F16>;
  const bool bf = cfg->in_dtype == FTINT8_BF16, wide = c->k_padded > 4096;
  for (int i = 0; i < 2; ++i)
    c->few[i] = cfg->out_dtype == FTINT8_F32 ? few_of<FTINT8_F32>(i) : cfg->out_dtype == FTINT8_BF16 ? few_of<FTINT8_BF16>(i) : few_of<FTINT8_F16>(i);
  for (int i = 0; i < 2; ++i)
    c->fused[i] = cfg->out_dtype == FTINT8_F32 ? fused_of<FTINT8_F32>(bf, i, wide) : cfg->out_dtype == FTINT8_BF16 ? fused_of<FTINT8_BF16>(bf, i, wide) : fused_of<FTINT8_F16>(bf, i, wide);
  const size_t bytes = (size_t)cfg->max_tokens * c->k_padded, sums = sums_bytes(cfg->n, c->k_padded / TileSmall::BK);
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) {
    for (int t = 0; t < N_TILES && he == hipSuccess; ++t) he = hipFuncSetAttribute((const void*)c->product[t], hipFuncAttributeMaxDynamicSharedMemorySize, TILES[t].lds);
    if (he == hipSuccess) he = hipMalloc((void**)&c->codes, sums + bytes + (size_t)cfg->max_tokens * sizeof(float));
    (void)hipSetDevice(before);
  }
  if (he != hipSuccess) {
    const int rc = ifail_hip(nullptr, "device", he);
    delete c;
    return rc;
  }
  c->sums = reinterpret_cast<int4v*>(c->codes);
  c->codes += sums;
  c->scales = reinterpret_cast<float*>(c->codes + bytes);
  *out = c;
  return FTINT8_OK;
}

extern "C" int ftint8_get_config(const ftint8_ctx* ctx, ftint8_config* effective) {
  if (!ctx || !effective) return FTINT8_EINVAL;
  *effective = ctx->cfg;
  return FTINT8_OK;
}

extern "C" int ftint8_k_padded(const ftint8_ctx* ctx) { return ctx ? ctx->k_padded : FTINT8_EINVAL; }

// What both halves check of a call; nullptr: nothing is wrong.
static const char* wrong_matrix(const ftint8_matrix* a, int size, int64_t length) {
  if (!a || !a->data) return "null argument";
  if ((uintptr_t)a->data % size) return "matrices must be aligned to their elements";
  if (a->stride < length || a->stride > (1ll << 40)) return "strides of rows must be at least their length, and at most 2^40 elements";
  return nullptr;
}
static const char* wrong_codes(const void* codes, const void* scales) {
  if (!codes || !scales) return "null argument";
  if ((uintptr_t)codes % 16 || (uintptr_t)scales % 4) return "codes must be 16-byte aligned, scales 4-byte aligned";
  return nullptr;
}

namespace {
struct OnDevice {      // the context's device for the length of a call
  int before = 0, device;
  hipError_t error;
  explicit OnDevice(int d) : device(d) {
    error = hipGetDevice(&before);
    if (error == hipSuccess && before != device) error = hipSetDevice(device);
  }
  ~OnDevice() {
    if (error == hipSuccess && before != device) (void)hipSetDevice(before);
  }
};
}  // namespace

static hipError_t launch_encode(ftint8_ctx* c, const ftint8_matrix* x, int32_t rows, int8_t* codes, float* scales, hipStream_t st) {
  const EncodeArgs a{static_cast<const char*>(x->data), x->stride * 2, c->cfg.k, c->k_padded, rows, codes, scales};
  const bool bf = c->cfg.in_dtype == FTINT8_BF16, whole = ((uintptr_t)x->data | (uintptr_t)(x->stride * 2)) % 16 == 0;
  int per = 1;
  const encode_fn fn = bf ? encode_of<FTINT8_BF16>(c->k_padded, whole, per) : encode_of<FTINT8_F16>(c->k_padded, whole, per);
  hipLaunchKernelGGL(fn, dim3((uint32_t)((rows + per - 1) / per)), dim3(256), 0, st, a);
  return hipGetLastError();
}
static ProductArgs product_args(ftint8_ctx* c, const int8_t* x, const float* sx, int32_t m, const int8_t* w, const float* sw, const ftint8_matrix* y) {
  const int size = c->cfg.out_dtype == FTINT8_F32 ? 4 : 2;
  return ProductArgs{x, w, sx, sw, static_cast<char*>(y->data), y->stride * size, m, c->cfg.n, c->k_padded, 1, nullptr};
}
// Tokens of which a launch cannot have all tiles (it has fewer than 2^32 threads).
static bool too_many(const ftint8_ctx* c, int32_t m) {
  const TileInfo& t = TILES[WIDE];
  return (int64_t)((m + t.bm - 1) / t.bm) * ((c->cfg.n + t.bf - 1) / t.bf) * t.threads >= 1ll << 32;
}
static hipError_t launch_product(ftint8_ctx* c, const int8_t* x, const float* sx, int32_t m, const int8_t* w, const float* sw, const ftint8_matrix* y, hipStream_t st) {
  ProductArgs a = product_args(c, x, sx, m, w, sw, y);
  auto tiles = [&](int t) { return (int64_t)((m + TILES[t].bm - 1) / TILES[t].bm) * ((c->cfg.n + TILES[t].bf - 1) / TILES[t].bf); };
  // Up to 16 tokens: 9 on 4096 x 16,384 (features x columns) 15.2 us, on tiles 16.8; 16 on 1000 x 500 2.5, 4.1; but 16 on 32,000 x 4096 30.9, 20.8, as each workgroup
  // reads as many codes of tokens as of weights.  Up to 32, where it reads twice as many, where the weights fit a round of workgroups: 32 on 4096 x 4096 7.7 us, 9.1; on 1000 x 1000 3.4, 5.3;
  // but on 4096 x 8192 13.1, 12.6, on 16,384 x 4096 23.7, 13.2, on 500 x 10,000 15.2, 9.4.
  if (m <= 16 || (m <= 32 && c->k_padded <= 4096 && c->cfg.n <= 4096)) {
    const FewArgs f{a, nullptr, 0, 0};
    const int two = m > 16;
    hipLaunchKernelGGL(c->few[two], dim3((uint32_t)((c->cfg.n + 15) / 16)), dim3(FEW_WAVES * 64), few_lds(1 + two), st, f);
    return hipGetLastError();
  }
  // The largest tile that gives every CU one.  256 x 256, 128 x 256, 64 x 256, 64 x 128, in us: 4096 tokens on 4096 x 4096 (256 tiles of the first) 55, 64, 87, 88;
  // 2000 tokens (256 of the second) 49, 36, 47, 50; 1000 (256 of the third) 47, 28, 24, 26; 512 (256 of the last) 46, 27, 21, 16.
  int tile = WIDE;
  while (tile + 1 < N_TILES && tiles(tile) < 256) ++tile;
  const int64_t count = tiles(tile), stages = c->k_padded / TileSmall::BK;
  // Too few of the smallest: the columns are divided, in shares of at least eight stages, the fewer in all the less there is to divide, as shares are written and read
  // once more.  96 tokens on 4096 x 16,384 (64 tiles) 24 us in four, 55 in one; 1000 on 500 x 10,000 15, 27; 64 on 4096 x 4096 (32 tiles, 32 stages) 10.7
  // in four, 13.9 in one; 256 tokens there (128 tiles) 15.0 in two, 12.5 in one.
  if (tile == SMALL) {
    const int64_t shares = most_shares((int)stages) / count;
    a.parts = (int)(shares < stages / 8 ? shares : stages / 8);
    if (a.parts < 2) a.parts = 1;
  }
  a.sums = c->sums;
  hipLaunchKernelGGL(c->product[tile], dim3((uint32_t)count, (uint32_t)a.parts), dim3(TILES[tile].threads), TILES[tile].lds, st, a);
  const hipError_t he = hipGetLastError();
  if (he != hipSuccess || a.parts == 1) return he;
  constexpr int BLOCKS = TileSmall::BM * TileSmall::BF / 256;
  hipLaunchKernelGGL(c->finish, dim3((uint32_t)(count * BLOCKS / 4)), dim3(256), 0, st, a, (int)count);
  return hipGetLastError();
}
extern "C" int ftint8_encode(ftint8_ctx* c, const ftint8_matrix* x, int32_t rows, int8_t* codes, float* scales, void* hip_stream) {
  if (!c) return FTINT8_EINVAL;
  if (rows < 0) return ifail(c, FTINT8_EINVAL, "rows must be >= 0");
  if (rows == 0) return FTINT8_OK;
  if (rows > MOST_GROUPS) return ifail(c, FTINT8_EUNSUPPORTED, "too many rows");
  const char* bad = wrong_matrix(x, 2, c->cfg.k);
  if (!bad) bad = wrong_codes(codes, scales);
  if (bad) return ifail(c, FTINT8_EINVAL, bad);
  OnDevice on(c->cfg.device);
  if (on.error != hipSuccess) return ifail_hip(c, "device", on.error);
  const hipError_t he = launch_encode(c, x, rows, codes, scales, (hipStream_t)hip_stream);
  return he == hipSuccess ? FTINT8_OK : ifail_hip(c, "launch", he);
}

extern "C" int ftint8_product(ftint8_ctx* c, const int8_t* codes_x, const float* scales_x, int32_t m, const int8_t* codes_w, const float* scales_w, const ftint8_matrix* y,
                              void* hip_stream) {
  if (!c) return FTINT8_EINVAL;
  if (m < 0) return ifail(c, FTINT8_EINVAL, "m must be >= 0");
  if (m == 0) return FTINT8_OK;
  if (m > 1 << 22) return ifail(c, FTINT8_EUNSUPPORTED, "more than 2^22 tokens");
  if (too_many(c, m)) return ifail(c, FTINT8_EUNSUPPORTED, "too many tokens for as many features");
  const char* bad = wrong_matrix(y, c->cfg.out_dtype == FTINT8_F32 ? 4 : 2, c->cfg.n);
  if (!bad) bad = wrong_codes(codes_x, scales_x);
  if (!bad) bad = wrong_codes(codes_w, scales_w);
  if (bad) return ifail(c, FTINT8_EINVAL, bad);
  OnDevice on(c->cfg.device);
  if (on.error != hipSuccess) return ifail_hip(c, "device", on.error);
  const hipError_t he = launch_product(c, codes_x, scales_x, m, codes_w, scales_w, y, (hipStream_t)hip_stream);
  return he == hipSuccess ? FTINT8_OK : ifail_hip(c, "launch", he);
}

extern "C" int ftint8_forward(ftint8_ctx* c, const ftint8_matrix* x, int32_t m, const int8_t* codes_w, const float* scales_w, const ftint8_matrix* y, void* hip_stream) {
  if (!c) return FTINT8_EINVAL;
  if (m < 0 || m > c->cfg.max_tokens) return ifail(c, FTINT8_EINVAL, "m must be 0 .. max_tokens");
  if (m == 0) return FTINT8_OK;
  if (too_many(c, m)) return ifail(c, FTINT8_EUNSUPPORTED, "too many tokens for as many features");
  const char* bad = wrong_matrix(x, 2, c->cfg.k);
  if (!bad) bad = wrong_matrix(y, c->cfg.out_dtype == FTINT8_F32 ? 4 : 2, c->cfg.n);
  if (!bad) bad = wrong_codes(codes_w, scales_w);
  if (bad) return ifail(c, FTINT8_EINVAL, bad);
  OnDevice on(c->cfg.device);
  if (on.error != hipSuccess) return ifail_hip(c, "device", on.error);
  hipError_t he;
  // One token; up to four on small layers, where an eager call's second launch weighs most (4 on 1024 x 1024 take
  // 5.9 us in an eager call, 5 of them 8.4 in two launches; in a graph 4 on 4096 x 4096 8.0, in two launches 8.5; on 16,384 x 4096 17.9 and 17.1).
  const bool several = m > 1;
  if (several ? m <= FUSED_TOKENS && c->k_padded <= 4096 && c->cfg.n <= 4096 && ((uintptr_t)x->data | (uintptr_t)(x->stride * 2)) % 16 == 0
              : c->k_padded <= FUSED_K && (uintptr_t)x->data % 16 == 0) {
    const FewArgs f{product_args(c, nullptr, nullptr, m, codes_w, scales_w, y), static_cast<const char*>(x->data), x->stride * 2, c->cfg.k};
    const int codes = m * (c->k_padded + 64);
    hipLaunchKernelGGL(c->fused[several], dim3((uint32_t)((c->cfg.n + 15) / 16)), dim3(FEW_WAVES * 64), codes > few_lds(1) ? codes : few_lds(1), (hipStream_t)hip_stream, f);
    he = hipGetLastError();
    return he == hipSuccess ? FTINT8_OK : ifail_hip(c, "launch", he);
  }
  he = launch_encode(c, x, m, c->codes, c->scales, (hipStream_t)hip_stream);
  if (he == hipSuccess) he = launch_product(c, c->codes, c->scales, m, codes_w, scales_w, y, (hipStream_t)hip_stream);
  return he == hipSuccess ? FTINT8_OK : ifail_hip(c, "launch", he);
}

extern "C" int ftint8_destroy(ftint8_ctx* c) {
  if (!c) return FTINT8_OK;
  int before = 0;
  const bool moved = hipGetDevice(&before) == hipSuccess && before != c->cfg.device && hipSetDevice(c->cfg.device) == hipSuccess;
  (void)hipFree(c->sums);
  if (moved) (void)hipSetDevice(before);
  delete c;
  return FTINT8_OK;
}

extern "C" const char* ftint8_last_error(const ftint8_ctx* c) { return c ? c->err.c_str() : g_int8_create_err.c_str(); }
