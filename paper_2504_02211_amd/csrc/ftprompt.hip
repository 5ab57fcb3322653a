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

namespace ftprompt {
using namespace ftserve;

constexpr int BM = 128, BN = 64, NW = 4;

struct Rows { char* data; int64_t token, head; };       // strides in bytes

struct Args {
  Rows q, k, v, o;
  const int32_t *cu_q, *cu_k;
  int32_t batch, total_q, total_k, kv_heads, group, slots;
  float scale_log2;
};

template <int D> constexpr int tile_bytes() { return BN * D * 2; }
template <int D> constexpr int lds_bytes() { return 2 * tile_bytes<D>(); }

// Place of 16-byte chunk c of row r in a tile.  Key tiles are read 16 bytes a lane from 32 rows, value tiles 4 rows of 32 bytes for every 16 lanes: ...
template <int D> __device__ __forceinline__ int k_place(int r, int c) {
  return D == 128 ? r * 16 + (c ^ (r & 15)) : r * 8 + (c ^ ((r >> 1) & 7));
}
template <int D> __device__ __forceinline__ int v_place(int r, int c) {
  return D == 128 ? r * 16 + (c ^ ((r & 3) << 2)) : r * 8 + (c ^ ((r >> 1 & 1) << 2));
}

template <bool BF> __device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c) {
  if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

__device__ __forceinline__ float max32(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
  return __builtin_fmaxf(as_f(r[0]), as_f(r[1]));
}
__device__ __forceinline__ float sum32(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(as_u(x), as_u(x), false, false);
  return as_f(r[0]) + as_f(r[1]);
}

template <int D, bool BF, bool F32OUT>
__global__ __launch_bounds__(NW * 64, 2) void ftprompt_main(const Args a) {
  extern __shared__ uint4v lds[];
  uint4v* const kt = lds;
  uint4v* const vt = lds + tile_bytes<D>() / 16;
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
  const int rows = nq * G, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5, n = lane & 31;

  const int row = tile * BM + wave * 32 + n, rowc = row < rows ? row : rows - 1;
  const int qi = rowc / G, head = hk * G + rowc % G;
  const int seen = nk - nq + qi + 1;                       // keys that the row sees: may be <= 0
  const int last_of = [&](int r) { return nk - nq + (r < rows ? r : rows - 1) / G + 1; }(tile * BM + BM - 1);
  const int keys = last_of < 0 ? 0 : last_of;              // of the longest row of the workgroup
  const int wave_row = tile * BM + wave * 32;
  const int all_seen = nk - nq + (wave_row < rows ? wave_row : rows - 1) / G + 1;      // keys that every row of the wave sees
  const int any_seen = nk - nq + (wave_row + 31 < rows ? wave_row + 31 : rows - 1) / G + 1;

  uint4v qf[D / 16];
  const char* qp = a.q.data + (int64_t)(q0 + qi) * a.q.token + (int64_t)head * a.q.head + 16 * h;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const uint4v*>(qp + 32 * i);

  float16v o[D / 32];
#pragma unroll
  for (int f = 0; f < D / 32; ++f) o[f] = (float16v)0.f;
  float ref = -3.4028234e38f, l = 0.f;
  const char* kbase = a.k.data + (int64_t)k0 * a.k.token + (int64_t)hk * a.k.head;
  const char* vbase = a.v.data + (int64_t)k0 * a.v.token + (int64_t)hk * a.v.head;
  constexpr int CH = D / 8, PER = BN * CH / (NW * 64);      // chunks per row, per thread

  for (int j0 = 0; j0 < keys; j0 += BN) {
    uint4v ks[PER], vs[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = tid + i * NW * 64, r = x / CH, c = x % CH;
      const int64_t t = j0 + r < nk ? j0 + r : nk - 1;
      ks[i] = *reinterpret_cast<const uint4v*>(kbase + t * a.k.token + 16 * c);
      vs[i] = *reinterpret_cast<const uint4v*>(vbase + t * a.v.token + 16 * c);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = tid + i * NW * 64, r = x / CH, c = x % CH;
      kt[k_place<D>(r, c)] = ks[i];
      vt[v_place<D>(r, c)] = vs[i];
    }
    __syncthreads();
    if (j0 >= any_seen) continue;

    float16v s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = (float16v)0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) s[t] = mfma32<BF>(kt[k_place<D>(32 * t + n, 2 * i + h)], qf[i], s[t]);
    }
    const bool masked = j0 + BN > all_seen;
    if (masked) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (j0 + 32 * t + 8 * (v >> 2) + 4 * h + (v & 3) >= seen) s[t][v] = -__builtin_inff();
    }
    float m = s[0][0];
#pragma unroll
    for (int v = 0; v < 16; ++v) m = __builtin_fmaxf(m, __builtin_fmaxf(s[0][v], s[1][v]));
    m = max32(m) * a.scale_log2;
    if (__any(m > ref + 8.f)) {
      const float next = __builtin_fmaxf(m, ref), f = ex2(ref - next);
      ref = next;
      l *= f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) o[x] *= f;
    }
    uint4v p[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const float x = ex2(__builtin_fmaf(s[t][v], a.scale_log2, -ref)), y = ex2(__builtin_fmaf(s[t][v + 1], a.scale_log2, -ref));
        l += x;
        l += y;
        p[2 * t + (v >> 3)][(v & 7) >> 1] = pack2<BF>(x, y);
      }
    // a value that a row does not see must not reach it, and 0 times infinity would: in tiles that some row does not see whole,
    // such values are taken out of the product and given to the rows that see them
    auto value = [&](int i, int f, int s4) {      // V^T: elements 32f + lane % 32, keys 16i + 8 s4 + 4h + 0..3
      const int r = 16 * i + 8 * s4 + 4 * h + ((lane & 15) >> 2), e = 32 * f + (lane & 16) + 4 * (lane & 3);
      const uint32_t at = (uint32_t)(tile_bytes<D>() + v_place<D>(r, e >> 3) * 16 + (e & 4) * 2);
      return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)((__attribute__((address_space(3))) char*)lds + at));
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int f = 0; f < D / 32; ++f) {
        const uint2v x = __builtin_bit_cast(uint2v, value(i, f, 0)), y = __builtin_bit_cast(uint2v, value(i, f, 1));
        uint4v av = {x[0], x[1], y[0], y[1]};
        if (masked) {
          uint32_t bad = 0;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t e = largest_finite_plus_one<BF>();
            const bool lo = (av[w] & e) == e, hi = (av[w] & (e << 16)) == (e << 16);
            bad |= (lo ? 1u : 0u) << (2 * w) | (hi ? 1u : 0u) << (2 * w + 1);
          }
          if (__any(bad != 0)) {
            // keys (h', slot) with such a value in any element of this block, one after the other
            for (int key = 0; key < 16; ++key) {
              const int hh = key >> 3, sl = key & 7;
              const uint64_t who = __ballot(h == hh && (bad >> sl & 1));
              if (!who) continue;
              const int j = j0 + 16 * i + 8 * (sl >> 2) + 4 * hh + (sl & 3);
              const uint32_t pw = p[i][sl >> 1];
              const float own = sl & 1 ? high_of<BF>(pw) : low_of<BF>(pw), w = __shfl(own, 32 * hh + n);
              const uint32_t vw = av[sl >> 1];
              const float val = sl & 1 ? high_of<BF>(vw) : low_of<BF>(vw);
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int e = 8 * (r >> 2) + 4 * h + (r & 3);
                const float ve = __shfl(val, 32 * hh + e);
                const bool is_bad = who >> (32 * hh + e) & 1;
                if (is_bad && j < seen) o[f][r] += w * ve;
              }
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) av[w] &= (bad >> (2 * w) & 1 ? 0u : 0xFFFFu) | (bad >> (2 * w + 1) & 1 ? 0u : 0xFFFF0000u);
          }
        }
        o[f] = mfma32<BF>(av, p[i], o[f]);
      }
  }
  l = sum32(l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (row >= rows) return;
  char* op = a.o.data + (int64_t)(q0 + qi) * a.o.token + (int64_t)head * a.o.head;
#pragma unroll
  for (int f = 0; f < D / 32; ++f)
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

}  // namespace ftprompt

using namespace ftprompt;

struct ftprompt_ctx {
  ftprompt_config cfg;
  kernel_fn fn = nullptr;
  int lds = 0;
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
  if (!(std::fabs(cfg->softmax_scale) <= 3.0e38f)) return pfail(nullptr, FTPROMPT_EINVAL, "softmax_scale is not finite");
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
  const int64_t slots = (int64_t)total_q * group / BM + batch;
  if ((int64_t)total_q * group > 0x7FFFFF00ll || slots * e.kv_heads > 0x7FFFFFFFll) return pfail(c, FTPROMPT_EUNSUPPORTED, "too many rows");
  Args a{r[0], r[1], r[2], r[3], cu_q, cu_k, batch, total_q, total_k, e.kv_heads, group, (int32_t)slots, e.softmax_scale * LOG2E};
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess && before != e.device) he = hipSetDevice(e.device);
  if (he != hipSuccess) return pfail_hip(c, "device", he);
  hipLaunchKernelGGL(c->fn, dim3((uint32_t)(slots * e.kv_heads)), dim3(NW * 64), c->lds, (hipStream_t)hip_stream, a);
  he = hipGetLastError();
  if (before != e.device) (void)hipSetDevice(before);
  return he == hipSuccess ? FTPROMPT_OK : pfail_hip(c, "launch", he);
}

extern "C" int ftprompt_destroy(ftprompt_ctx* c) {
  delete c;
  return FTPROMPT_OK;
}

extern "C" const char* ftprompt_last_error(const ftprompt_ctx* c) { return c ? c->err.c_str() : g_prompt_create_err.c_str(); }
