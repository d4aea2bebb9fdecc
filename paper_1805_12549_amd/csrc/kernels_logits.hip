// What is done with the logits behind the classifier: log probabilities of given classes with the entropy and the top alternatives
// (cg_logprobs), and the distillation loss from a teacher's top logits with its gradient (cg_distill_forward, cg_distill_backward).
//
// One workgroup takes a row at a time.  With m = max z and c = 1 / temperature every quantity is formed from the differences (z - m) * c,
// which are exact before the product, so neither a large offset of a row nor logits at the type's lowest value cost precision or overflow.
// All sums are held in 32 bits.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "cg_device.h"
#include "cg_internal.h"

namespace cg {
int set_error(int code, const char* fmt, ...);   // defined with the host API
}

namespace {

using cg::bf16_to_float;
using cg::float_to_bf16;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2E = 1.44269504088896340736f;

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(uint16_t v) { return bf16_to_float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = float_to_bf16(v); }

// a class by its rank in a row: greater logits first, equal ones by index (-0 equals 0); never 0 for a class, so 0 is "none"
__device__ __forceinline__ uint64_t rank_key(float z, uint32_t index) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  const uint32_t up = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return ((uint64_t)up << 32) | (uint32_t)~index;
}

struct Sum {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct MaxKey {
  __device__ uint64_t operator()(uint64_t a, uint64_t b) const { return a > b ? a : b; }
};

// over the workgroup, in an order that does not change; `part` (kWaves values) may be used again after the next barrier
template <class V, class Op>
__device__ __forceinline__ V over_workgroup(V v, V* part, Op op) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) v = op(v, (V)__shfl_xor(v, s, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) v = op(v, part[w]);
  return v;
}

struct LogprobArgs {
  const void* logits;
  long long rows, stride;
  int classes, given, top;
  float scale;             // 1 / temperature
  const int64_t* labels;
  float *logprob, *entropy;
  int64_t* top_ids;
  float* top_logprobs;
};

template <class T>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobArgs a) {
  __shared__ float part[kWaves];
  __shared__ uint64_t part_key[kWaves];
  const int tid = (int)threadIdx.x;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* z = (const T*)a.logits + row * a.stride;
    float m = -INFINITY;
    for (long long v = tid; v < a.classes; v += kThreads) m = fmaxf(m, as_float(z[v]));
    m = over_workgroup(m, part, Max());
    const float from = m == -INFINITY ? 0.0f : m;      // (a row without a class: exponentials of -inf, no NaN)
    float sum = 0.0f, moment = 0.0f;                    // of e, and of e times its exponent
    for (long long v = tid; v < a.classes; v += kThreads) {
      const float y = (as_float(z[v]) - from) * a.scale, e = exp2f(y * kLog2E);
      sum += e;
      moment += e > 0.0f ? e * y : e;                   // (NaN stays)
    }
    sum = over_workgroup(sum, part, Sum());
    moment = over_workgroup(moment, part, Sum());
    const bool none = sum == 0.0f, bad = sum != sum;
    const float log_sum = logf(sum);
    const auto logprob = [&](float x) { return none ? -INFINITY : bad ? NAN : (x - m) * a.scale - log_sum; };
    for (int g = tid; g < a.given; g += kThreads) {
      const int64_t id = a.labels[row * a.given + g];
      a.logprob[row * a.given + g] = id < 0 ? 0.0f : id >= a.classes ? NAN : logprob(as_float(z[id]));
    }
    if (a.entropy && tid == 0) a.entropy[row] = none ? 0.0f : log_sum - moment / sum;
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
      uint64_t best = 0;
      for (long long v = tid; v < a.classes && !bad; v += kThreads) {
        const uint64_t key = rank_key(as_float(z[v]), (uint32_t)v);
        if (key < last && key > best) best = key;
      }
      last = over_workgroup(best, part_key, MaxKey());
      if (tid == 0) {
        const uint32_t id = ~(uint32_t)last;
        a.top_ids[row * a.top + k] = bad ? -1 : (int64_t)id;
        a.top_logprobs[row * a.top + k] = bad ? NAN : logprob(as_float(z[id]));
      }
    }
  }
}

struct DistillArgs {
  const void* logits;
  long long rows, stride, grad_stride;
  int classes, top;
  float scale;             // 1 / temperature
  float w_teacher, w_label;
  const int64_t* top_ids;
  const float* top_logits;
  const int64_t* labels;
  const float* grad_loss;
  const float* given_stats;
  float *loss, *stats;
  void* grad;
};

template <class T>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  __shared__ float part[kWaves];
  __shared__ float mass_of[CG_TOP_MAX];
  __shared__ int64_t id_of[CG_TOP_MAX];
  const int tid = (int)threadIdx.x;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* z = (const T*)a.logits + row * a.stride;
    T* g = a.grad ? (T*)a.grad + row * a.grad_stride : nullptr;
    // the teacher's distribution: one entry a thread
    const int64_t id = tid < a.top ? a.top_ids[row * a.top + tid] : -1;
    const float t = id >= 0 ? a.top_logits[row * a.top + tid] : -INFINITY;
    const float tm = over_workgroup(t, part, Max());
    const float ty = (t - (tm == -INFINITY ? 0.0f : tm)) * a.scale;
    float q = exp2f(ty * kLog2E);
    const float mass = over_workgroup(q, part, Sum());
    const float beyond = over_workgroup(id >= a.classes ? 1.0f : 0.0f, part, Max());
    const bool taught = a.w_teacher != 0.0f && (mass != 0.0f || beyond != 0.0f);
    const int64_t label = a.labels ? a.labels[row] : -1;
    const bool labelled = a.w_label != 0.0f && label >= 0;
    const float wt = !taught ? 0.0f : beyond != 0.0f || mass != mass ? NAN : a.w_teacher;
    const float wl = !labelled ? 0.0f : label >= a.classes ? NAN : a.w_label;
    if (mass != 0.0f) q /= mass;
    // the student's sums
    float m = -INFINITY, s1 = 0.0f, st = 0.0f;
    if (a.given_stats) {
      m = a.given_stats[row * 3];
      s1 = a.given_stats[row * 3 + 1];
      st = a.given_stats[row * 3 + 2];
    } else {
      for (long long v = tid; v < a.classes; v += kThreads) m = fmaxf(m, as_float(z[v]));
      m = over_workgroup(m, part, Max());
      const float from = m == -INFINITY ? 0.0f : m;
      for (long long v = tid; v < a.classes; v += kThreads) {
        const float y = as_float(z[v]) - from;
        s1 += exp2f(y * kLog2E);
        st += exp2f(y * a.scale * kLog2E);
      }
      s1 = over_workgroup(s1, part, Sum());
      st = over_workgroup(st, part, Sum());
      if (a.stats && tid == 0) {
        a.stats[row * 3] = m;
        a.stats[row * 3 + 1] = a.w_label != 0.0f ? s1 : NAN;
        a.stats[row * 3 + 2] = a.w_teacher != 0.0f ? st : NAN;
      }
    }
    const bool none = (a.w_label != 0.0f ? s1 : st) == 0.0f || (!taught && !labelled);     // nothing to learn from this row
    const float zi = id >= 0 && id < a.classes ? as_float(z[id]) : 0.0f;
    if (a.loss) {
      float l = taught && q != 0.0f ? wt * q * ((ty - logf(mass)) - ((zi - m) * a.scale - logf(st))) : 0.0f;
      if (tid == 0 && labelled) l += wl == wl ? wl * (logf(s1) - (as_float(z[label]) - m)) : NAN;
      l = over_workgroup(l, part, Sum());
      if (tid == 0) a.loss[row] = none ? 0.0f : beyond != 0.0f && taught ? NAN : l;
    }
    if (g) {
      const float up = a.grad_loss ? a.grad_loss[row] : 1.0f;
      const float ct = up * wt * a.scale, cl = up * wl;
      __syncthreads();
      if (tid < a.top) {
        id_of[tid] = id;
        mass_of[tid] = q;
      }
      __syncthreads();
      // the classes of the teacher's entries and the label: what one thread for each entry puts there after the others
      float mine = 0.0f;
      const int64_t at = tid < a.top ? id : tid == a.top ? label : -1;
      if (at >= 0 && at < a.classes && !none) {
        const float y = as_float(z[at]) - m;
        mine = (taught ? exp2f(y * a.scale * kLog2E) * (ct / st) : 0.0f) + (labelled ? exp2f(y * kLog2E) * (cl / s1) : 0.0f);
        float minus = 0.0f;
        if (taught)
          for (int k = 0; k < a.top; ++k) minus += id_of[k] == at ? mass_of[k] : 0.0f;
        mine -= ct * minus + (labelled && at == label ? cl : 0.0f);
      }
      __syncthreads();
      for (long long v = tid; v < a.classes; v += kThreads) {
        const float y = as_float(z[v]) - m;
        const float x = (taught ? exp2f(y * a.scale * kLog2E) * (ct / st) : 0.0f) + (labelled ? exp2f(y * kLog2E) * (cl / s1) : 0.0f);
        put(g + v, none ? 0.0f : x);
      }
      __syncthreads();
      if (at >= 0 && at < a.classes && !none) put(g + at, mine);
    }
  }
}

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int element_bytes(int dtype) { return dtype == CG_F32 ? 4 : 2; }

// what both operators ask of the logits
int check_logits(const char* who, const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t row_stride, float temperature) {
  if (rows < 0 || classes <= 0) return cg::set_error(CG_EINVAL, "%s: bad size", who);
  if (dtype != CG_F32 && dtype != CG_BF16) return cg::set_error(CG_EUNSUPPORTED, "%s: logits are CG_F32 or CG_BF16", who);
  if (row_stride < 0) return cg::set_error(CG_EINVAL, "%s: row_stride must not be negative", who);
  if (!(temperature > 0.0f) || !std::isfinite(temperature) || !std::isfinite(1.0f / temperature))
    return cg::set_error(CG_EINVAL, "%s: temperature must be positive and finite, and its inverse too", who);
  if (rows > 0 && row_stride > (int64_t)((1ull << 62) / (uint64_t)rows)) return cg::set_error(CG_EINVAL, "%s: bad size", who);
  if (rows > 0 && !logits) return cg::set_error(CG_EINVAL, "%s: logits must not be NULL", who);
  if (!aligned(logits, element_bytes(dtype))) return cg::set_error(CG_EINVAL, "%s: logits must be aligned to their elements", who);
  return CG_OK;
}

// workgroups of a launch that walks rows: a launch holds less than 2^32 threads
unsigned row_groups(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : (1 << 20)); }

int check_teacher(const char* who, int64_t rows, int32_t top, const int64_t* top_ids, const float* top_logits, const int64_t* labels, float w_teacher,
                  float w_label) {
  if (top < 0) return cg::set_error(CG_EINVAL, "%s: bad size", who);
  if (top > CG_TOP_MAX) return cg::set_error(CG_EUNSUPPORTED, "%s: at most %d teacher classes", who, CG_TOP_MAX);
  if (!std::isfinite(w_teacher) || !std::isfinite(w_label)) return cg::set_error(CG_EINVAL, "%s: weights must be finite", who);
  if (rows > 0 && top > 0 && (!top_ids || !top_logits)) return cg::set_error(CG_EINVAL, "%s: top_ids and top_logits must not be NULL", who);
  if (w_teacher != 0.0f && top == 0) return cg::set_error(CG_EINVAL, "%s: teacher_weight needs a teacher's classes", who);
  if (w_label != 0.0f && rows > 0 && !labels) return cg::set_error(CG_EINVAL, "%s: label_weight needs labels", who);
  if (!aligned(top_ids, 8) || !aligned(labels, 8) || !aligned(top_logits, 4))
    return cg::set_error(CG_EINVAL, "%s: top_ids, labels and top_logits must be aligned to their elements", who);
  return CG_OK;
}

int check_grad(const char* who, const void* grad, int32_t dtype, int64_t rows, int32_t classes, int64_t grad_stride, const void* logits, int64_t row_stride) {
  if (!aligned(grad, element_bytes(dtype))) return cg::set_error(CG_EINVAL, "%s: grad must be aligned to its elements", who);
  if (rows > 1 && grad_stride < classes) return cg::set_error(CG_EINVAL, "%s: the rows of grad overlap", who);
  if (rows > 0 && grad_stride > (int64_t)((1ull << 62) / (uint64_t)rows)) return cg::set_error(CG_EINVAL, "%s: bad size", who);
  if (rows > 1 && grad == logits && grad_stride != row_stride) return cg::set_error(CG_EINVAL, "%s: grad in place of logits needs their strides", who);
  return CG_OK;
}

int launch_distill(const char* who, const DistillArgs& a, int32_t dtype, hipStream_t s) {
  if (dtype == CG_F32)
    hipLaunchKernelGGL(distill_kernel<float>, dim3(row_groups(a.rows)), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(distill_kernel<uint16_t>, dim3(row_groups(a.rows)), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cg::set_error(CG_EHIP, "%s: %s", who, hipGetErrorString(e));
  return CG_OK;
}

}  // namespace

extern "C" {

size_t cg_logprobs_workspace_bytes(int64_t rows, int32_t classes, int32_t top) {
  (void)rows, (void)classes, (void)top;
  return 0;
}

int cg_logprobs(const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t row_stride, float temperature, const int64_t* labels,
                int32_t given, int32_t top, float* logprob, float* entropy, int64_t* top_ids, float* top_logprobs, void* workspace,
                size_t workspace_bytes, void* hip_stream) {
  const char* const who = "cg_logprobs";
  if (const int rc = check_logits(who, logits, dtype, rows, classes, row_stride, temperature)) return rc;
  if (given < 0 || top < 0 || top > classes) return cg::set_error(CG_EINVAL, "%s: given must not be negative, top lies in [0, classes]", who);
  if (top > CG_TOP_MAX) return cg::set_error(CG_EUNSUPPORTED, "%s: at most %d alternatives", who, CG_TOP_MAX);
  if (rows > 0 && given > 0 && (!labels || !logprob)) return cg::set_error(CG_EINVAL, "%s: labels and logprob must not be NULL", who);
  if (rows > 0 && top > 0 && (!top_ids || !top_logprobs)) return cg::set_error(CG_EINVAL, "%s: top_ids and top_logprobs must not be NULL", who);
  if (!aligned(labels, 8) || !aligned(top_ids, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(top_logprobs, 4))
    return cg::set_error(CG_EINVAL, "%s: labels and outputs must be aligned to their elements", who);
  if (rows == 0) return CG_OK;
  const size_t need = cg_logprobs_workspace_bytes(rows, classes, top);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256)))
    return cg::set_error(CG_EINVAL, "%s: needs %zu bytes of workspace, 256-byte aligned", who, need);
  const LogprobArgs a{logits, rows, row_stride, classes, given, top, 1.0f / temperature, labels, logprob, entropy, top_ids, top_logprobs};
  if (dtype == CG_F32)
    hipLaunchKernelGGL(logprobs_kernel<float>, dim3(row_groups(rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
  else
    hipLaunchKernelGGL(logprobs_kernel<uint16_t>, dim3(row_groups(rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cg::set_error(CG_EHIP, "%s: %s", who, hipGetErrorString(e));
  return CG_OK;
}

size_t cg_distill_workspace_bytes(int64_t rows, int32_t classes) {
  (void)rows, (void)classes;
  return 0;
}

int cg_distill_forward(const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t row_stride, float temperature, const int64_t* top_ids,
                       const float* top_logits, int32_t top, const int64_t* labels, float teacher_weight, float label_weight, float* loss, float* stats,
                       const float* grad_loss, void* grad, int64_t grad_stride, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* const who = "cg_distill_forward";
  if (const int rc = check_logits(who, logits, dtype, rows, classes, row_stride, temperature)) return rc;
  if (const int rc = check_teacher(who, rows, top, top_ids, top_logits, labels, teacher_weight, label_weight)) return rc;
  if (rows > 0 && !loss) return cg::set_error(CG_EINVAL, "%s: loss must not be NULL", who);
  if (!aligned(loss, 4) || !aligned(stats, 4) || !aligned(grad_loss, 4))
    return cg::set_error(CG_EINVAL, "%s: loss, stats and grad_loss must be aligned to their elements", who);
  if (grad)
    if (const int rc = check_grad(who, grad, dtype, rows, classes, grad_stride, logits, row_stride)) return rc;
  if (rows == 0) return CG_OK;
  const size_t need = cg_distill_workspace_bytes(rows, classes);
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256)))
    return cg::set_error(CG_EINVAL, "%s: needs %zu bytes of workspace, 256-byte aligned", who, need);
  const DistillArgs a{logits, rows, row_stride, grad_stride, classes, top, 1.0f / temperature, teacher_weight, label_weight, top_ids, top_logits,
                      labels, grad_loss, nullptr, loss, stats, grad};
  return launch_distill(who, a, dtype, (hipStream_t)hip_stream);
}

int cg_distill_backward(const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t row_stride, float temperature, const int64_t* top_ids,
                        const float* top_logits, int32_t top, const int64_t* labels, float teacher_weight, float label_weight, const float* stats,
                        const float* grad_loss, void* grad, int64_t grad_stride, void* hip_stream) {
  const char* const who = "cg_distill_backward";
  if (const int rc = check_logits(who, logits, dtype, rows, classes, row_stride, temperature)) return rc;
  if (const int rc = check_teacher(who, rows, top, top_ids, top_logits, labels, teacher_weight, label_weight)) return rc;
  if (rows > 0 && (!stats || !grad)) return cg::set_error(CG_EINVAL, "%s: stats and grad must not be NULL", who);
  if (!aligned(stats, 4) || !aligned(grad_loss, 4)) return cg::set_error(CG_EINVAL, "%s: stats and grad_loss must be aligned to their elements", who);
  if (const int rc = check_grad(who, grad, dtype, rows, classes, grad_stride, logits, row_stride)) return rc;
  if (rows == 0) return CG_OK;
  const DistillArgs a{logits, rows, row_stride, grad_stride, classes, top, 1.0f / temperature, teacher_weight, label_weight, top_ids, top_logits,
                      labels, grad_loss, stats, nullptr, nullptr, grad};
  return launch_distill(who, a, dtype, (hipStream_t)hip_stream);
}

}  // extern "C"
