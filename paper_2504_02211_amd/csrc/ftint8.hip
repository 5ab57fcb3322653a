// Linear layer on 8-bit integers: the kernels and the C ABI of ../include/ftint8.h.
#include "ftint8.h"
#include "ftserve_device.h"

#include <new>
#include <string>

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
  int32_t k, k_padded;
  int8_t* codes;
  float* scales;
};

// A row a workgroup: its largest magnitude, then its codes.
template <int DT> __global__ __launch_bounds__(256) void ftint8_encode_rows(const EncodeArgs a) {
  __shared__ uint32_t most_of[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  const char* const x = a.x + (int64_t)row * a.stride;
  uint32_t most = 0;
  for (int i = tid; i < a.k; i += 256) {
    const uint32_t u = as_u(element<DT>(x, i)) & 0x7FFFFFFFu;
    most = u > most ? u : most;
  }
  for (int d = 32; d; d >>= 1) {
    const uint32_t y = __shfl_xor(most, d);
    most = y > most ? y : most;
  }
  if ((tid & 63) == 0) most_of[tid >> 6] = most;
  __syncthreads();
  for (int w = 0; w < 4; ++w) most = most_of[w] > most ? most_of[w] : most;
  // infinities and NaN are above all numbers.  Rows below 2^-100 are taken times 2^100, where the quotient stays finite.
  const bool fine = most < 0x7F800000u;
  const float up = as_f(most) < 0x1p-100f ? 0x1p100f : 1.f, inverse = most == 0 || !fine ? 0.f : 127.f * (1.f / (as_f(most) * up));
  if (tid == 0) a.scales[row] = fine ? as_f(most) / 127.f : __builtin_nanf("");
  int8_t* const codes = a.codes + (int64_t)row * a.k_padded;
  for (int i = tid; i < a.k_padded; i += 256) {
    const float y = i < a.k && fine ? element<DT>(x, i) * up * inverse : 0.f;
    codes[i] = (int8_t)(int)__builtin_rintf(y);
  }
}

struct ProductArgs {
  const int8_t *x, *w;
  const float *sx, *sw;
  char* y;
  int64_t y_stride;      // bytes
  int32_t m, n, k_padded;
};

// Y^T = W X^T: a wave takes 16 features and 64 tokens of a tile of 64 x 64.
template <int DT> __global__ __launch_bounds__(256) void ftint8_tile(const ProductArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lq = lane & 15, lg = lane >> 4;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64 + wave * 16;
  if (n0 >= a.n) return;
  int4v acc[4];
  const int8_t *wp, *xp[4];
  wp = a.w + (int64_t)(n0 + lq < a.n ? n0 + lq : a.n - 1) * a.k_padded + 16 * lg;
  for (int t = 0; t < 4; ++t) {
    const int r = m0 + 16 * t + lq;
    xp[t] = a.x + (int64_t)(r < a.m ? r : a.m - 1) * a.k_padded + 16 * lg;
    acc[t] = (int4v)0;
  }
  for (int k = 0; k < a.k_padded; k += 64) {
    const int4v w = *reinterpret_cast<const int4v*>(wp + k);
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, *reinterpret_cast<const int4v*>(xp[t] + k), acc[t], 0, 0, 0);
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int row = m0 + 16 * t + lq;
    if (row >= a.m) continue;
    const float sx = a.sx[row];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int col = n0 + 4 * lg + r;
      if (col >= a.n) continue;
      float y = (float)acc[t][r] * (sx * a.sw[col]);
      asm("" : "+v"(y));      // (rounded to 32 bits: the compiler would make one instruction of this product and its rounding to 16)
      char* const to = a.y + (int64_t)row * a.y_stride;
      if constexpr (DT == FTINT8_F32) reinterpret_cast<float*>(to)[col] = y;
      else reinterpret_cast<uint16_t*>(to)[col] = (uint16_t)pack2<DT == FTINT8_BF16>(y, y);
    }
  }
}

typedef void (*encode_fn)(const EncodeArgs);
typedef void (*product_fn)(const ProductArgs);

}  // namespace ftint8

using namespace ftint8;

struct ftint8_ctx {
  ftint8_config cfg;
  int k_padded = 0;
  encode_fn encode = nullptr;
  product_fn product = nullptr;
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
  c->encode = cfg->in_dtype == FTINT8_BF16 ? ftint8_encode_rows<FTINT8_BF16> : ftint8_encode_rows<FTINT8_F16>;
  c->product = cfg->out_dtype == FTINT8_F32 ? ftint8_tile<FTINT8_F32> : cfg->out_dtype == FTINT8_BF16 ? ftint8_tile<FTINT8_BF16> : ftint8_tile<FTINT8_F16>;
  const size_t bytes = (size_t)cfg->max_tokens * c->k_padded;
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) {
    he = hipMalloc((void**)&c->codes, bytes + (size_t)cfg->max_tokens * sizeof(float));
    (void)hipSetDevice(before);
  }
  if (he != hipSuccess) {
    const int rc = ifail_hip(nullptr, "device", he);
    delete c;
    return rc;
  }
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
  const EncodeArgs a{static_cast<const char*>(x->data), x->stride * 2, c->cfg.k, c->k_padded, codes, scales};
  hipLaunchKernelGGL(c->encode, dim3((uint32_t)rows), dim3(256), 0, st, a);
  return hipGetLastError();
}
static hipError_t launch_product(ftint8_ctx* c, const int8_t* x, const float* sx, int32_t m, const int8_t* w, const float* sw, const ftint8_matrix* y, hipStream_t st) {
  const int size = c->cfg.out_dtype == FTINT8_F32 ? 4 : 2;
  const ProductArgs a{x, w, sx, sw, static_cast<char*>(y->data), y->stride * size, m, c->cfg.n, c->k_padded};
  hipLaunchKernelGGL(c->product, dim3((uint32_t)((c->cfg.n + 63) / 64), (uint32_t)((m + 63) / 64)), dim3(256), 0, st, a);
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
  const char* bad = wrong_matrix(x, 2, c->cfg.k);
  if (!bad) bad = wrong_matrix(y, c->cfg.out_dtype == FTINT8_F32 ? 4 : 2, c->cfg.n);
  if (!bad) bad = wrong_codes(codes_w, scales_w);
  if (bad) return ifail(c, FTINT8_EINVAL, bad);
  OnDevice on(c->cfg.device);
  if (on.error != hipSuccess) return ifail_hip(c, "device", on.error);
  hipError_t he = launch_encode(c, x, m, c->codes, c->scales, (hipStream_t)hip_stream);
  if (he == hipSuccess) he = launch_product(c, c->codes, c->scales, m, codes_w, scales_w, y, (hipStream_t)hip_stream);
  return he == hipSuccess ? FTINT8_OK : ifail_hip(c, "launch", he);
}

extern "C" int ftint8_destroy(ftint8_ctx* c) {
  if (!c) return FTINT8_OK;
  int before = 0;
  const bool moved = hipGetDevice(&before) == hipSuccess && before != c->cfg.device && hipSetDevice(c->cfg.device) == hipSuccess;
  (void)hipFree(c->codes);
  if (moved) (void)hipSetDevice(before);
  delete c;
  return FTINT8_OK;
}

extern "C" const char* ftint8_last_error(const ftint8_ctx* c) { return c ? c->err.c_str() : g_int8_create_err.c_str(); }
