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
};

template <bool BF> __device__ __forceinline__ float element(const char* row, int i) {
  if constexpr (BF) return as_f((uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << 16);
  else return (float)reinterpret_cast<const _Float16*>(row)[i];
}

// The decay in two words: rounded to one, it is off by up to 2^-25 in the same direction at every token, and a state that remembers thousands of tokens by 2^-13.
struct Decay { float high, low; };
__device__ __forceinline__ Decay decay_of(const Args& a, int h) {
  const double d = exp((double)__builtin_fminf(a.log_decay[h], 0.f));
  const float high = (float)d;
  return Decay{high, (float)(d - (double)high)};
}

// Where sequence b has its state; NULL: nowhere.
template <int D> __device__ __forceinline__ float* state_of(const Args& a, int b, int h) {
  const int slot = a.slots ? a.slots[b] : b;
  return a.states && slot >= 0 && slot < a.n_slots ? a.states + ((int64_t)slot * a.heads + h) * (D * D) : nullptr;
}

// The recurrence, a (sequence, head) a workgroup: thread (g, e) has column e of the state, rows of its g-th part.
template <int D, bool BF> __global__ __launch_bounds__(256) void ftdecay_recurrent(const Args a) {
  constexpr int PARTS = 256 / D, R = D / PARTS;
  __shared__ float qs[D], ks[D], part[PARTS][D];
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads, hk = h / a.group, e = threadIdx.x % D, g = threadIdx.x / D;
  const int t0 = a.cu ? clamped(a.cu[b], a.total) : b, t1 = a.cu ? clamped(a.cu[b + 1], a.total) : b + 1;
  const bool fresh = a.cu && (!a.starts || a.starts[b] <= 0);
  float* const state = state_of<D>(a, b, h);
  const Decay decay = decay_of(a, h);
  float s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = state && !fresh ? state[(g * R + i) * D + e] : 0.f;
  for (int t = t0; t < t1; ++t) {
    const float v = element<BF>(a.v.data + t * a.v.token + hk * a.v.head, e);
    __syncthreads();
    if (g == 0) {
      qs[e] = element<BF>(a.q.data + t * a.q.token + h * a.q.head, e);
      ks[e] = element<BF>(a.k.data + t * a.k.token + hk * a.k.head, e);
    }
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      s[i] = __builtin_fmaf(ks[g * R + i], v, __builtin_fmaf(s[i], decay.high, s[i] * decay.low));
      sum = __builtin_fmaf(qs[g * R + i], s[i], sum);
    }
    part[g][e] = sum;
    __syncthreads();
    if (g == 0) {
      float all = 0.f;
      for (int i = 0; i < PARTS; ++i) all += part[i][e];
      all *= a.scale;
      reinterpret_cast<uint16_t*>(a.o.data + t * a.o.token + h * a.o.head)[e] = (uint16_t)pack2<BF>(all, all);
    }
  }
  if (state)
#pragma unroll
    for (int i = 0; i < R; ++i) state[(g * R + i) * D + e] = s[i];
}

typedef void (*kernel_fn)(const Args);

}  // namespace ftdecay

using namespace ftdecay;

struct ftdecay_ctx {
  ftdecay_config cfg;
  kernel_fn recurrent = nullptr;
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
  const bool bf = cfg->in_dtype == FTDECAY_BF16;
  c->recurrent = cfg->head_dim == 128 ? (bf ? ftdecay_recurrent<128, true> : ftdecay_recurrent<128, false>) : (bf ? ftdecay_recurrent<64, true> : ftdecay_recurrent<64, false>);
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess) he = hipSetDevice(cfg->device);
  if (he == hipSuccess) (void)hipSetDevice(before);
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

static int launch(ftdecay_ctx* c, const Args& a, hipStream_t st) {
  int before = 0;
  hipError_t he = hipGetDevice(&before);
  if (he == hipSuccess && before != c->cfg.device) he = hipSetDevice(c->cfg.device);
  if (he != hipSuccess) return dfail_hip(c, "device", he);
  hipLaunchKernelGGL(c->recurrent, dim3((uint32_t)(a.batch * a.heads)), dim3(256), 0, st, a);
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
  if ((int64_t)batch * e.heads > MOST_GROUPS) return dfail(c, FTDECAY_EUNSUPPORTED, "too many sequences");
  return launch(c, Args{r[0], r[1], r[2], r[3], log_decay, states, slots, cu, starts, n_slots, batch, total, e.heads, e.heads / e.kv_heads, e.scale}, (hipStream_t)hip_stream);
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
  return launch(c, Args{r[0], r[1], r[2], r[3], log_decay, states, slots, nullptr, nullptr, n_slots, batch, batch, e.heads, e.heads / e.kv_heads, e.scale}, (hipStream_t)hip_stream);
}

extern "C" int ftdecay_destroy(ftdecay_ctx* c) {
  delete c;
  return FTDECAY_OK;
}

extern "C" const char* ftdecay_last_error(const ftdecay_ctx* c) { return c ? c->err.c_str() : g_decay_create_err.c_str(); }
