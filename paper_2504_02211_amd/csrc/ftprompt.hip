// Attention over packed prompts with grouped heads: the kernel and the C ABI of include/ftprompt.h.
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
#include "ftprompt.h"
#include "ftserve_device.h"

#include <cmath>
#include <new>
#include <string>
#include <type_traits>

namespace ftprompt {
using namespace ftserve;

constexpr int BN = 64, SUB = 64, NW = 4, STAGES = 2;      // keys of a tile, of a step; waves; tiles in LDS
constexpr int64_t WIDE_FROM = 2 * 256 * 256;
constexpr int bm_of(int rb) { return NW * 32 * rb; }      // rows of a workgroup whose waves have rb blocks of 32

struct Rows { char* data; int64_t token, head; };         // strides in bytes

struct Args {
  Rows q, k, v, o;
  const int32_t *cu_q, *cu_k;
  int32_t batch, total_q, total_k, kv_heads, group, slots;
  float scale_log2;
};

template <int D> constexpr int tile_bytes() { return BN * D * 2; }
template <int D> constexpr int lds_bytes() { return STAGES * 2 * tile_bytes<D>(); }

// 16 bytes per lane from (uniform base + per-lane byte offset) straight into LDS at (uniform LDS address + 16 * lane).
// (Opaque to the compiler, which would wait for the tile in flight before it reads another; ordering against barriers and counted waits is kept
// because all of them are side-effecting instructions.)
__device__ __forceinline__ void load_lds16(const void* base, uint32_t byte_off, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(byte_off), "s"(base), "s"(lds_addr) : "memory");
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

typedef __attribute__((address_space(3))) char lds_char;

template <int D, bool BF, bool F32OUT, int RB>
__global__ __launch_bounds__(NW * 64, 2) void ftprompt_main(const Args a) {
  extern __shared__ uint4v lds[];
  constexpr int BM = bm_of(RB), NF = D / 32, TILE = tile_bytes<D>();
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int hk = blockIdx.x % a.kv_heads, slot = a.slots - 1 - blockIdx.x / a.kv_heads;
  const int G = a.group;
  // sequence b owns the row tiles from cu_q[b] * G / BM + b on: at least as many as it has rows for
  auto tiles_before = [&](int b) { return (int64_t)clamped(a.cu_q[b], a.total_q) * G / BM + b; };
  const int b = sequence_of(a.batch, slot, tiles_before);
  const int tile = slot - (int)tiles_before(b);
  const int q0 = clamped(a.cu_q[b], a.total_q), q1 = clamped(a.cu_q[b + 1], a.total_q);
  const int k0 = clamped(a.cu_k[b], a.total_k), k1 = clamped(a.cu_k[b + 1], a.total_k);
  const int nq = q1 - q0, nk = k1 - k0;
  if (tile < 0 || nq <= 0 || (int64_t)tile * BM >= (int64_t)nq * G) return;
  const int rows = nq * G, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, n = lane & 31;

  // keys that row r of the sequence sees (may be <= 0); rows behind the last count as it
  auto seen_by = [&](int r) { return nk - nq + (r < rows ? r : rows - 1) / G + 1; };
  const int row0 = tile * BM + wave * (32 * RB);
  const int all_seen = seen_by(row0), any_seen = seen_by(row0 + 32 * RB - 1), keys = seen_by(tile * BM + BM - 1);
  const int tiles = keys > 0 ? (keys + BN - 1) / BN : 0;
  const int steps = any_seen > 0 ? (any_seen + SUB - 1) / SUB : 0, full = all_seen > 0 ? all_seen / SUB : 0;      // steps of this wave; that every row sees whole

  int seen[RB];
  uint4v qf[RB][D / 16];
  auto row_of = [&](int rb, int& query, int& head) {
    const int r = row0 + 32 * rb + n, rc = r < rows ? r : rows - 1;
    query = rc / G;
    head = hk * G + rc - query * G;
    return r < rows;
  };
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    int query, head;
    row_of(rb, query, head);
    seen[rb] = nk - nq + query + 1;
    const char* qp = a.q.data + (int64_t)(q0 + query) * a.q.token + (int64_t)head * a.q.head + 16 * h;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) qf[rb][i] = *reinterpret_cast<const uint4v*>(qp + 32 * i);
  }

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
    if ((t + 1) * BN <= nk) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_lds16(p, off[i], to + i * 1024);
    } else {           // rows behind the last key: the last one again (no row sees them)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int r = (wave * LOADS + i) * RPL + lane / CH, rc = r < nk - 1 - t * BN ? r : nk - 1 - t * BN;
        load_lds16(p, (uint32_t)rc * (uint32_t)stride + chunk(r), to + i * 1024);
      }
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

  float16v o[RB][NF];
  float4v sums[RB];
  float ref[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    ref[rb] = -3.4028234e38f;
    sums[rb] = (float4v)0.f;
#pragma unroll
    for (int f = 0; f < NF; ++f) o[rb][f] = (float16v)0.f;
  }

  // scores of a tile, transposed
  auto scores = [&](uint32_t k_at, float16v (&to)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      to[t] = (float16v)0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) to[t] = mfma32<BF>(key(k_at + t * (64 * D), i), qf[0][i], to[t]);
    }
  };
  auto mask = [&](int t, float16v (&x)[2]) __attribute__((always_inline)) {
    const int limit = seen[0] - t * BN - 4 * h;
#pragma unroll
    for (int v = 0; v < 32; ++v)
      if (limit <= 8 * (v >> 2) + (v & 3)) x[v >> 4][v & 15] = -__builtin_inff();
  };
  // fp16 weights reach 2^14 rather than 2^8, so that those far below the largest keep their bits
  constexpr float ROOM = 8.f, UP = BF ? 0.f : 6.f;
  auto largest = [&](const float16v (&x)[2]) __attribute__((always_inline)) {
    float m = __builtin_fmaxf(x[0][0], x[1][0]);
#pragma unroll
    for (int v = 1; v < 16; ++v) m = __builtin_fmaxf(__builtin_fmaxf(m, x[0][v]), x[1][v]);
    return max32(m) * a.scale_log2;
  };
  // a row's reference moves when a score exceeds it by more than there is room for: rarely after the first step
  auto renew = [&](const float (&m)[RB]) __attribute__((always_inline)) {
    bool any = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) any |= m[rb] > ref[rb] + (ROOM + UP);
    if (__any(any)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float next = __builtin_fmaxf(m[rb] - UP, ref[rb]), f = ex2(ref[rb] - next);
        ref[rb] = next;
        sums[rb] *= f;
#pragma unroll
        for (int x = 0; x < NF; ++x) o[rb][x] *= f;
      }
    }
  };
  auto weight_pair = [&](const float16v (&x)[2], int v, uint4v (&p)[4]) __attribute__((always_inline)) {
    p[v >> 3][(v & 7) >> 1] = pack2<BF>(ex2(__builtin_fmaf(x[v >> 4][v & 15], a.scale_log2, -ref[0])), ex2(__builtin_fmaf(x[v >> 4][(v & 15) + 1], a.scale_log2, -ref[0])));
  };
  auto add_up = [&](const uint4v (&p)[4], int i) __attribute__((always_inline)) {        // the i-th four weights
    sums[0] = add4<BF>(i & 1 ? uint2v{p[i >> 1][2], p[i >> 1][3]} : uint2v{p[i >> 1][0], p[i >> 1][1]}, sums[0]);
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
        o[0][f] = mfma32<BF>(av, p[i], o[0][f]);
      }
  };

  // A value that a row does not see must not reach it, and 0 times infinity would: in steps that some row does not see whole, values that are not finite are
  // left out of the products, and added behind the loop to the rows that see them.
  // Stage t & 1 holds what iteration t reads: the values of tile t and the keys of tile t + 1.  An iteration computes the scores of the next tile beside the
  // exponentials of its own (vector instructions in the shadow of the wave's own matrix instructions are nearly free), then its products beside the maxima of the next.
  auto arrive = [&](int t) __attribute__((always_inline)) {
    // what iteration t reads is there, and nobody reads what t - 1 did any more: it makes room for t + 1
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const uint32_t next = lds0 + ((t + 1) & 1) * (2 * TILE);
    if (t + 1 < tiles) issue_v(t + 1, next + TILE);
    if (t + 2 < tiles) issue_k(t + 2, next);
    return (uint32_t)(t & 1) * (2 * TILE);      // (from the beginning of LDS)
  };
  float16v s[2];
  if (tiles > 0) {
    issue_k(0, lds0 + 2 * TILE);
    issue_v(0, lds0 + TILE);
    if (tiles > 1) issue_k(1, lds0);
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    scores(2 * TILE, s);
    if (full < 1) mask(0, s);
    const float m[RB] = {largest(s)};
    renew(m);
  }
  int t = 0;
  for (; t + 1 < full; ++t) {              // this tile and the next one are seen whole by every row of the wave
    const uint32_t at = arrive(t);
    // Written out in the order that it runs in: every matrix instruction with the operand that was requested AHEAD instructions before, the request of
    // another, and the vector instructions that fit beside it.
    constexpr int NK = D / 8, NV = 4 * NF, N = NK + NV, AHEAD = 4, PER = 32 / NK, MAXIMA = 16 / NV;
    auto operand = [&](int x) __attribute__((always_inline)) { return x < NK ? key(at + (x & 1) * (64 * D), x >> 1) : value(at + TILE, (x - NK) / NF, (x - NK) % NF); };
    uint4v ring[AHEAD], p[4];
    float16v then[2];
    float m[RB];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) ring[x] = operand(x);
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const uint4v mine = ring[x % AHEAD];
      if (x < NK) then[x & 1] = mfma32<BF>(mine, qf[0][x >> 1], x < 2 ? (float16v)0.f : then[x & 1]);
      else o[0][(x - NK) % NF] = mfma32<BF>(mine, p[(x - NK) / NF], o[0][(x - NK) % NF]);
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
        for (int v = y * MAXIMA; v < (y + 1) * MAXIMA; ++v) m[0] = v == 0 ? __builtin_fmaxf(then[0][0], then[1][0]) : __builtin_fmaxf(__builtin_fmaxf(m[0], then[0][v]), then[1][v]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    m[0] = max32(m[0]) * a.scale_log2;
    s[0] = then[0];
    s[1] = then[1];
    renew(m);
  }
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
      const float m[RB] = {largest(s)};
      renew(m);
    }
  }
  if (__any(__builtin_bit_cast(uint32_t, finite) != 0xFFFFFFFFu)) {
    for (int j = full > 1 ? (full - 1) * BN : 0; j < any_seen; ++j)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(vbase + (int64_t)j * a.v.token + 2 * (32 * f + 8 * (r >> 2) + 4 * h + (r & 3)));
            const float lo = low_of<BF>(w), hi = high_of<BF>(w);
            if (j < seen[rb] && !(__builtin_fabsf(lo) <= 3.4e38f)) o[rb][f][r] += lo;
            if (j < seen[rb] && !(__builtin_fabsf(hi) <= 3.4e38f)) o[rb][f][r + 1] += hi;
          }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    int query, head;
    const bool real = row_of(rb, query, head);
    const float l = sum32(sums[rb][0]), inv = l == 0.f ? 0.f : 1.f / l;
    if (!real) continue;
    char* op = a.o.data + (int64_t)(q0 + query) * a.o.token + (int64_t)head * a.o.head;
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float x0 = o[rb][f][4 * g] * inv, x1 = o[rb][f][4 * g + 1] * inv, x2 = o[rb][f][4 * g + 2] * inv, x3 = o[rb][f][4 * g + 3] * inv;
        const int e = 32 * f + 8 * g + 4 * h;
        if constexpr (F32OUT) *reinterpret_cast<float4v*>(op + 4 * e) = float4v{x0, x1, x2, x3};
        else *reinterpret_cast<uint2v*>(op + 2 * e) = uint2v{pack2<BF>(x0, x1), pack2<BF>(x2, x3)};
      }
  }
}

typedef void (*kernel_fn)(const Args);
template <int D, bool BF, int RB> static kernel_fn kernel_of(bool f32) { return f32 ? ftprompt_main<D, BF, true, RB> : ftprompt_main<D, BF, false, RB>; }
template <int RB> static kernel_fn kernel_for(const ftprompt_config& e) {
  const bool bf = e.in_dtype == FTPROMPT_BF16, f32 = e.out_dtype == FTPROMPT_F32;
  return e.head_dim == 128 ? (bf ? kernel_of<128, true, RB>(f32) : kernel_of<128, false, RB>(f32)) : (bf ? kernel_of<64, true, RB>(f32) : kernel_of<64, false, RB>(f32));
}

}  // namespace ftprompt

using namespace ftprompt;

struct ftprompt_ctx {
  ftprompt_config cfg;
  kernel_fn fn[2] = {nullptr, nullptr};       // one block of rows to a wave, two
  int lds = 0;
  std::string err;
};

// Whether waves take two blocks of 32 rows.
static int ftprompt_wide(int64_t total_q, int heads) { return total_q * heads >= WIDE_FROM; }

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
  if (!(std::fabs(cfg->softmax_scale) <= 3.0e38f)) return pfail(nullptr, FTPROMPT_EINVAL, "softmax_scale is not finite");
  ftprompt_ctx* c = new (std::nothrow) ftprompt_ctx();
  if (!c) return pfail(nullptr, FTPROMPT_ENOMEM, "out of host memory");
  c->cfg = *cfg;
  if (!(c->cfg.softmax_scale > 0.f)) c->cfg.softmax_scale = 1.0f / std::sqrt((float)cfg->head_dim);
  c->fn[0] = kernel_for<1>(*cfg);
  c->fn[1] = kernel_for<1>(*cfg);
  c->lds = cfg->head_dim == 128 ? lds_bytes<128>() : lds_bytes<64>();
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) {
    for (int i = 0; i < 2 && he == hipSuccess; ++i) he = hipFuncSetAttribute((const void*)c->fn[i], hipFuncAttributeMaxDynamicSharedMemorySize, c->lds);
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
  const int wide = 0;
  const int64_t slots = (int64_t)total_q * group / bm_of(wide + 1) + batch;
  if ((int64_t)total_q * group > 0x7FFFFF00ll || slots * e.kv_heads > 0x7FFFFFFFll) return pfail(c, FTPROMPT_EUNSUPPORTED, "too many rows");
  Args a{r[0], r[1], r[2], r[3], cu_q, cu_k, batch, total_q, total_k, e.kv_heads, group, (int32_t)slots, e.softmax_scale * LOG2E};
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess && before != e.device) he = hipSetDevice(e.device);
  if (he != hipSuccess) return pfail_hip(c, "device", he);
  hipLaunchKernelGGL(c->fn[wide], dim3((uint32_t)(slots * e.kv_heads)), dim3(NW * 64), c->lds, (hipStream_t)hip_stream, a);
  he = hipGetLastError();
  if (before != e.device) (void)hipSetDevice(before);
  return he == hipSuccess ? FTPROMPT_OK : pfail_hip(c, "launch", he);
}

extern "C" int ftprompt_destroy(ftprompt_ctx* c) {
  delete c;
  return FTPROMPT_OK;
}

extern "C" const char* ftprompt_last_error(const ftprompt_ctx* c) { return c ? c->err.c_str() : g_prompt_create_err.c_str(); }
