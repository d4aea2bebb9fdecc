// The launches of the operators behind the classifier without a GPU: this program defines the HIP runtime calls that the library makes, which the loader finds
// before the runtime's own, and notes what would be launched.  For sizes over the whole range: the parts of shared rows fit the workspace that the size query
// asks for, launches stay below 2^32 threads, and a workspace that is too small is refused before any launch.  Run by tests/test_logits_launches_cpu.py.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <vector>

#include "cg_conv.h"

struct Launch { unsigned long long blocks, threads; };
static std::vector<Launch> launches;
static Launch config;
static long long checked = 0, shared = 0;
static int failures = 0;
#define EXPECT(c) do { ++checked; if (!(c)) { if (++failures < 20) std::printf("FAILED line %d: %s  [%s]\n", __LINE__, #c, cg_last_error()); } } while (0)

extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  config = Launch{(unsigned long long)grid.x * grid.y * grid.z, block.x};
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) {
  *grid = *block = dim3(1);
  *lds = 0;
  *s = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) {
  launches.push_back(config);
  return hipSuccess;
}
}

static char* const at = (char*)0x7f0000000000ull;      // addresses that nothing reads
static void* ws() { return at + (1ull << 40); }

static void check(long long rows, int classes, int dtype, int top) {
  const long long size = dtype == CG_F32 ? 4 : 2;
  const int t = top < classes ? top : classes;
  {
    const size_t need = cg_logprobs_workspace_bytes(rows, classes, t);
    launches.clear();
    EXPECT(cg_logprobs(at, dtype, rows, classes, classes, 0.7f, (const int64_t*)at, 1, t, (float*)at, (float*)at, (int64_t*)at, (float*)at, ws(), need, nullptr) == CG_OK);
    EXPECT(launches.size() == 1 || launches.size() == 2);
    if (launches.size() == 2) {
      ++shared;
      EXPECT(launches[0].blocks % rows == 0 && launches[0].blocks * (12 + 8 * (size_t)t) <= need && launches[1].blocks == (unsigned long long)rows);
    }
    for (const Launch& l : launches) EXPECT(l.blocks > 0 && l.blocks * l.threads < 1ull << 32);
    launches.clear();
    if (need) EXPECT(cg_logprobs(at, dtype, rows, classes, classes, 0.7f, (const int64_t*)at, 1, t, (float*)at, (float*)at, (int64_t*)at, (float*)at, ws(), need - 1, nullptr) == CG_EINVAL && launches.empty());
  }
  // the loss alone, with its gradient beside the logits, at another alignment, and in their place
  char* const grads[] = {nullptr, at + (1ull << 42), at + (1ull << 42) + size, at};
  for (char* grad : grads) {
    const size_t need = cg_distill_workspace_bytes(rows, classes);
    launches.clear();
    EXPECT(cg_distill_forward(at, dtype, rows, classes, classes, 2.0f, (const int64_t*)at, (const float*)at, t, (const int64_t*)at, 0.5f, 0.5f, (float*)at, (float*)at,
                              (const float*)at, grad, classes, ws(), need, nullptr) == CG_OK);
    EXPECT(launches.size() >= 1 && launches.size() <= 3);
    if (launches.size() > 1) {
      ++shared;
      EXPECT(launches[0].blocks % rows == 0 && launches[0].blocks * 12 <= need);
      EXPECT((launches.size() == 3) == (grad == at) && launches.back().blocks == (grad ? launches[0].blocks : (unsigned long long)rows));
    }
    for (const Launch& l : launches) EXPECT(l.blocks > 0 && l.blocks * l.threads < 1ull << 32);
    launches.clear();
    if (need) EXPECT(cg_distill_forward(at, dtype, rows, classes, classes, 2.0f, (const int64_t*)at, (const float*)at, t, (const int64_t*)at, 0.5f, 0.5f, (float*)at,
                                        (float*)at, (const float*)at, grad, classes, nullptr, need, nullptr) == CG_EINVAL && launches.empty());
    if (!grad) continue;
    launches.clear();
    EXPECT(cg_distill_backward(at, dtype, rows, classes, classes, 2.0f, (const int64_t*)at, (const float*)at, t, (const int64_t*)at, 0.5f, 0.5f, (const float*)at,
                               (const float*)at, grad, classes, nullptr) == CG_OK);
    EXPECT(launches.size() == 1 && launches[0].blocks > 0 && launches[0].blocks * launches[0].threads < 1ull << 32);
  }
}

int main() {
  const int classes[] = {1, 2, 7, 64, 1000, 4097, 8191, 16384, 16385, 32768, 40001, 65536, 131072, 200003, 1 << 20, 1 << 26, 2147483647};
  for (int c : classes)
    for (long long rows : {1ll, 2ll, 3ll, 7ll, 48ll, 63ll, 64ll, 65ll, 85ll, 127ll, 128ll, 129ll, 255ll, 256ll, 257ll, 511ll, 512ll, 513ll, 1024ll, 4097ll, 100000ll, 5000000ll})
      for (int dtype : {CG_F32, CG_BF16})
        for (int top : {1, 20, 128})
          if ((double)rows * c < 4.0e18) check(rows, c, dtype, top);
  std::printf("%lld checks, %lld calls with shared rows\n", checked, shared);
  if (!failures && shared > 100) std::printf("logits launches: ok\n");
  return failures != 0;
}
