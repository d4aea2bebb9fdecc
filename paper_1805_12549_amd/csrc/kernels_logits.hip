// What is done with the logits behind the classifier: log probabilities of given classes with the entropy and the top alternatives
// (cg_logprobs), and the distillation loss from a teacher's top logits with its gradient (cg_distill_forward, cg_distill_backward).
//
// With m = max z and c = 1 / temperature every quantity is formed from the differences, as (z - m) / 2 * 2 c: neither a large offset of a row nor logits at
// the type's ends cost precision or overflow.  Probabilities are e / sum, not exponentials of a difference from a rounded logarithm.  All sums are held in 32
// bits; only a gradient is rounded to the logits' type, once.  An element costs an exponential and some ten other instructions, so that memory bounds
// calls of a few hundred long rows (2048 of 50003 classes in bf16: 4.8 TB/s read), but for the loss alone at two temperatures (2048 of 32000 in fp32: 3.5 TB/s).  Rows
// of a few KB are bound by their latencies (the loss of 4096 rows of 1000 in fp32: 2.1 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
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
constexpr int kUnroll = 4;           // chunks that a lane takes at once
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

// exp2 by the hardware (one ulp; results below 2^-126 are 0)
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// (x - from) / 2, of which the factors below take twice the reciprocal temperature: the difference of two logits may pass the range of 32 bits where that over
// the temperature does not.  One fma, rounded as the difference is.
__device__ __forceinline__ float half_apart(float x, float from) { return fmaf(x, 0.5f, -0.5f * from); }

// A row as the lanes of a workgroup walk it: elements in front of the first 16-byte boundary, whole 16-byte chunks, elements behind the last one; or
// part `seg` of `segs` of its chunks, the elements beside them with the first part.
template <class T>
struct RowSpan {
  static constexpr int kPer = 16 / (int)sizeof(T);      // elements of a chunk
  const T* z;
  const uint4* body;
  int from, chunks;        // the element at which the part's chunks begin, their number
  int head, tail_from, end;
  __device__ RowSpan(const T* row, int n, int seg, int segs) : z(row), end(n) {
    const int lead = (int)((0 - (uintptr_t)row) & 15) / (int)sizeof(T);
    head = lead < n ? lead : n;
    const int all = (n - head) / kPer, each = segs == 1 ? all : (all + segs - 1) / segs, first = seg * each;
    tail_from = head + all * kPer;
    chunks = first >= all ? 0 : all - first < each ? all - first : each;
    from = head + first * kPer;
    body = (const uint4*)(row + from);
    if (seg) head = 0, tail_from = end;
  }
  // the element beside the chunks that lane `tid` takes (fewer than 16 in all), or -1
  __device__ int beside(int tid) const {
    const int v = tid < head ? tid : tail_from + tid - head;
    return v < (tid < head ? head : end) ? v : -1;
  }
  __device__ bool holds(int64_t v) const { return v < head || (v >= from && v < from + (int64_t)chunks * kPer) || (v >= tail_from && v < end); }
};

__device__ __forceinline__ void unpack(const uint4& c, float* x, const float*) {
  x[0] = __uint_as_float(c.x), x[1] = __uint_as_float(c.y), x[2] = __uint_as_float(c.z), x[3] = __uint_as_float(c.w);
}
__device__ __forceinline__ void unpack(const uint4& c, float* x, const uint16_t*) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
template <class T>
__device__ __forceinline__ uint4 all_minus_inf() {
  const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  return make_uint4(w, w, w, w);
}

constexpr float kLeast = -1.0e4f;     // in the place of exponents from there down to -inf, whose power is 0, where they are factors of it

// Over a wavefront whose lanes are all active: across the lanes of a row of 16 by moves between neighbours, then the four rows' results, which are
// the same bits in every lane.  (A shuffle through LDS takes some hundred clocks, a move a few.)
template <int kMove>
__device__ __forceinline__ float moved(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), kMove, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float x, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); }
template <class Op>
__device__ __forceinline__ float over_lanes(float x, Op op) {
  x = op(x, moved<0xB1>(x));       // the other of a pair
  x = op(x, moved<0x4E>(x));       // the other pair of four
  x = op(x, moved<0x141>(x));      // mirrored in eight
  x = op(x, moved<0x140>(x));      // mirrored in sixteen
  return op(op(lane_of(x, 0), lane_of(x, 16)), op(lane_of(x, 32), lane_of(x, 48)));
}
__device__ __forceinline__ float max_over_lanes(float x) {
  return over_lanes(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_over_lanes(float x) {
  return over_lanes(x, [](float a, float b) { return a + b; });
}

// `count` chunks, at most 2^27, as a buffer: what lies behind them is neither read nor written, and no access needs a branch or registers for an address
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_buffer(const void* at, int count) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)at, (short)0, count * 16, 0x00027000);
}

// the next OF * kOf chunks of a part from chunk `first` on; -inf where it has none
template <int OF, class T, int kOf>
__device__ __forceinline__ void load_chunks(const RowSpan<T>& z, int first, uint4 (&raw)[kOf]) {
  const int left = z.chunks - first, tid = (int)threadIdx.x;
  const __amdgpu_buffer_rsrc_t from = chunk_buffer(z.body + first, left < OF * kOf ? left : OF * kOf);
#pragma unroll
  for (int u = 0; u < kOf; ++u) raw[u] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, (tid + u * OF) * 16, 0, 0));
  if (left < OF * kOf) {
#pragma unroll
    for (int u = 0; u < kOf; ++u)
      if (tid + u * OF >= left) raw[u] = all_minus_inf<T>();
  }
}

// A softmax in one pass: with m the greatest logit so far, the sum of e = 2^y and the sum of e y, y = (z - m) / 2 * c, c = 2 log2(e) / temperature.
// A new maximum scales both.  NaN and +inf make the sum NaN; without any class m is -inf and the sum 0.
struct Online {
  float m, sum, moment;
  // to the maximum `to` >= m
  __device__ void raise(float to, float c) {
    const float d = fmaxf(half_apart(m, to) * c, kLeast), f = pow2(d);
    moment = f * (moment + d * sum);
    sum *= f;
    m = to;
  }
  template <int N>
  __device__ void take(const float* x, float most, float c) {
    if (most > m) raise(most, c);
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = half_apart(x[i], from) * c, e = pow2(y);
      sum += e;
      moment = fmaf(e, fmaxf(y, kLeast), moment);
    }
  }
  __device__ void add(const Online& b) {
    sum += b.sum;
    moment += b.moment;
  }
  __device__ void over_lanes() {
    sum = sum_over_lanes(sum);
    moment = sum_over_lanes(moment);
  }
};

template <class S>
__device__ __forceinline__ void join(S& o, S b, float c) {
  const float to = fmaxf(o.m, b.m);
  o.raise(to, c);
  b.raise(to, c);
  o.add(b);
}
template <class S>
__device__ __forceinline__ S over_wavefront(S o, float c) {
  o.raise(max_over_lanes(o.m), c);
  o.over_lanes();
  return o;
}
// Every thread gets the result.  `part`: one value for each wavefront, not those of the row before.
template <int kOf = kThreads / 64, class S>
__device__ __forceinline__ S over_workgroup(S o, S* part, float c) {
  o = over_wavefront(o, c);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = o;
  __syncthreads();
  if (kOf > 4) {
    const int lane = (int)threadIdx.x & 63;
    o = part[lane < kOf ? lane : 0];
    if (lane >= kOf) o = S{-INFINITY, 0.0f, 0.0f};
    return over_wavefront(o, c);
  }
  o = part[0];
#pragma unroll
  for (int w = 1; w < kOf; ++w) join(o, part[w], c);
  return o;
}
// parts[0, n), joined by each wavefront by itself
template <class S>
__device__ __forceinline__ S join_parts(const S* parts, int n, S o, float c) {
  for (int k = (int)threadIdx.x & 63; k < n; k += 64) join(o, parts[k], c);
  return over_wavefront(o, c);
}

// What a workgroup of OF threads needs to find the alternatives.
template <int OF>
struct TopLds {
  static constexpr int kMarks = OF == 64 ? 4 : 4096 / OF;         // stretches of a lane whose greatest logits are kept
  static constexpr int kCandidates = OF == 64 ? 256 : 1024;       // at most so many are compared with each other
  float mark[kMarks][OF];
  uint16_t stretch[kMarks * OF];     // those that are looked through
  uint32_t lane[2][OF];              // upper halves of the lanes' greatest keys (0: none), for rows in turn
  int count[2], stretches[2];
  alignas(16) uint64_t found[kCandidates];
};

// how many of keys[0, n), all different, are greater than `key`
__device__ __forceinline__ int rank_among(const uint64_t* keys, int n, uint64_t key) {
  int r = 0, j = 0;
#pragma unroll 4
  for (; j + 2 <= n; j += 2) {
    const ulonglong2 k = *(const ulonglong2*)(keys + j);
    r += (k.x > key) + (k.y > key);
  }
  return j < n ? r + (keys[j] > key) : r;
}

// The greatest number that at least `top` of a wavefront's lanes * W keys reach, its highest kBits of kOf bits: bit by bit.
template <int kBits, int kOf, class K, int W>
__device__ __forceinline__ K reached_by(const K (&k)[W], int top) {
  K cut = 0;
#pragma unroll(kBits == 16 ? 16 : 1)
  for (int bit = kOf - 1; bit >= kOf - kBits; --bit) {
    const K next = cut | (K)1 << bit;
    int n = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) n += __popcll(__ballot(k[w] >= next));
    if (n >= top) cut = next;
  }
  return cut;
}

// What a lane leaves for find_top, before a barrier.
template <int OF>
__device__ __forceinline__ void offer_lane(TopLds<OF>& l, int turn, uint32_t upper) {
  l.lane[turn][threadIdx.x] = upper;
  if (threadIdx.x == 0) l.count[turn] = l.stretches[turn] = 0;
}

template <int OF>
__device__ __forceinline__ void add_found(TopLds<OF>& l, int turn, uint64_t key) {
  const int at = atomicAdd(&l.count[turn], 1);
  if (at < TopLds<OF>::kCandidates) l.found[at] = key;
}

// The top-th of the lanes' greatest among found[0, n), more than OF keys: at least `top` of them reach it, and those of OF - top lanes do not.
template <int OF>
__device__ __forceinline__ uint64_t raised_bound(const TopLds<OF>& l, int n, int top) {
  uint32_t upper[OF / 64], lower[OF / 64];
#pragma unroll
  for (int w = 0; w < OF / 64; ++w) {
    uint64_t most = 0;
    for (int i = w * 64 + ((int)threadIdx.x & 63); i < n; i += OF) most = l.found[i] > most ? l.found[i] : most;
    upper[w] = (uint32_t)(most >> 32);
    lower[w] = (uint32_t)most;
  }
  const uint32_t u = reached_by<32, 32>(upper, top);
#pragma unroll
  for (int w = 0; w < OF / 64; ++w) lower[w] = upper[w] > u ? ~0u : upper[w] == u ? lower[w] : 0;
  return (uint64_t)u << 32 | reached_by<32, 32>(lower, top);
}

// The `top` < OF greatest keys of a workgroup's lanes, which are all different: found[0, n) holds them, and few others, at most OF in all.  scan(bound) calls
// add_found for every key from `bound` up, or for more than kCandidates of them.  least_key: one that `top` keys reach in any case, for rows in which fewer
// than `top` lanes have a greater logit than -inf: whatever else there is, classes of -inf among the first 2 * top fill the rest.  The top-th of the lanes'
// greatest keys, cut to 16 bits, is a bound that at least `top` keys reach; as a rule few more do.  Where more do than can be compared with each other (equal
// logits, or a lane that has many of the greatest), the same is done with those that `found` took, whichever these are, until they are few: the bound rises
// each time.  (256 rows of 1000 equal logits, 20 alternatives: 13 us; with a thousand keys compared with each other 64.)  Dear are rows with fewer chunks than
// alternatives, which have no bound at first (256 rows of 300 in fp32, 128 alternatives, 13.6 us, of 1000 in bf16 16.0; with 64 alternatives 7.5 and 7.7), and
// rising rows whose logits share their upper 16 bits, whose bound rises by some thousand keys a scan (129 rows of 65536 in fp32, 20 alternatives, 241 us, equal
// ones 36, others 16; of 2^20 1356, 211 and 116).
template <int OF, class Scan>
__device__ int find_top(TopLds<OF>& l, int turn, int top, uint64_t least_key, Scan scan) {
  constexpr int kFull = TopLds<OF>::kCandidates;
  const int tid = (int)threadIdx.x, lane = tid & 63;
  uint64_t bound;
  {
    uint32_t k[OF / 64];
#pragma unroll
    for (int w = 0; w < OF / 64; ++w) k[w] = l.lane[turn][w * 64 + lane];
    bound = (uint64_t)reached_by<16, 32>(k, top) << 32;
  }
  if (bound && (bound >> 32) < 0x00800000u) bound = least_key;
  for (;;) {
    scan(bound);
    __syncthreads();
    int n = l.count[turn];
    if (n <= OF) return n;
    const bool all = n <= kFull;
    bound = raised_bound(l, all ? n : kFull, top);
    uint64_t mine[kFull / OF];
#pragma unroll
    for (int q = 0; q < kFull / OF; ++q) mine[q] = all && tid + q * OF < n ? l.found[tid + q * OF] : 0;
    __syncthreads();
    if (tid == 0) l.count[turn] = l.stretches[turn] = 0;
    __syncthreads();
    if (!all) continue;
    while (true) {       // those that reach the raised bound, until they are few
#pragma unroll
      for (int q = 0; q < kFull / OF; ++q)
        if (mine[q] >= bound) add_found(l, turn, mine[q]);
      __syncthreads();
      n = l.count[turn];
      if (n <= OF) return n;
      bound = raised_bound(l, n, top);
      __syncthreads();
      if (tid == 0) l.count[turn] = 0;
      __syncthreads();
    }
  }
}
// the logit of a key
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t up = (uint32_t)(key >> 32);
  return __uint_as_float(up & 0x80000000u ? up ^ 0x80000000u : ~up);
}

// A bound as logits and indices meet it: greater logits than `least`, and equal ones up to the class `last`.
struct Bound {
  uint64_t key;
  float least;
  uint32_t last;
  __device__ explicit Bound(uint64_t k) : key(k), least((k >> 32) < 0x00800000u ? -INFINITY : logit_of(k)), last(~(uint32_t)k) {}
  // whether a logit of a class not before `first` may reach it
  __device__ bool met(float x, uint32_t first) const { return x > least || (x == least && first <= last); }
};

struct LogprobArgs {
  const void* logits;
  long long rows, stride;
  int classes, given, top, segs;
  float scale;             // 1 / temperature
  const int64_t* labels;
  float *logprob, *entropy;
  int64_t* top_ids;
  float* top_logprobs;
  Online* parts;           // [rows][segs] and their greatest keys [rows][top][segs] (0: fewer than that), where rows are shared out
  uint64_t* keys;
};

// A row's log probabilities.  The logits of given classes are on their way while the row is read.
template <class T, int OF>
struct RowAnswer {
  const LogprobArgs& a;
  const T* z;
  long long row;
  int64_t id0;
  float z0;
  float m, log_sum;
  bool none, bad;
  __device__ RowAnswer(const LogprobArgs& args, long long r) : a(args), z((const T*)args.logits + r * args.stride), row(r) {
    if ((int)threadIdx.x < a.given) take((int)threadIdx.x);
  }
  __device__ void take(int g) {
    id0 = a.labels[row * a.given + g];
    z0 = id0 >= 0 && id0 < a.classes ? as_float(z[id0]) : 0.0f;
  }
  __device__ void put(const Online& o) {
    m = o.m, log_sum = logf(o.sum), none = o.sum == 0.0f, bad = o.sum != o.sum;
    const int tid = (int)threadIdx.x;
    for (int g = tid; g < a.given; g += OF) {
      if (g != tid) take(g);
      a.logprob[row * a.given + g] = id0 < 0 ? 0.0f : id0 >= a.classes ? NAN : of(z0);
    }
    if (a.entropy && tid == 0) a.entropy[row] = none ? 0.0f : log_sum - o.moment / (o.sum * kLog2E);
    for (int k = tid; bad && k < a.top; k += OF) put_top(k, -1, NAN);
  }
  __device__ float of(float x) const { return none ? -INFINITY : bad ? NAN : half_apart(x, m) * (2.0f * a.scale) - log_sum; }
  __device__ void put_top(int at, int64_t id, float logprob) const {
    a.top_ids[row * a.top + at] = id;
    a.top_logprobs[row * a.top + at] = logprob;
  }
  __device__ void put_top(const uint64_t* found, int n) const {
    for (int k = (int)threadIdx.x; k < n; k += OF) {
      const int r = rank_among(found, n, found[k]);
      if (r < a.top) put_top(r, ~(uint32_t)found[k], of(logit_of(found[k])));
    }
  }
};

// One pass over the row (V elements are read once): every lane keeps its own running maximum and sums.  The alternatives come from what the pass leaves behind:
// the lanes' maxima give a bound that is reached by little more than `top` classes, the maxima of each lane's stretches say where those lie, and only such
// stretches are read again, all at once.  PART: a workgroup takes one of `segs` parts of a row, and leaves its sums and keys to logprobs_join_kernel.  4096
// rows of 131072 classes in bf16 with 64 alternatives 201 us (5.3 TB/s; without alternatives 192, 5.6), in fp32 401 us (without 364, 5.9 TB/s), 2048 rows of
// 50003 in bf16 43 us: bound by memory.  One row of 1000 classes 4.5 us (3.0 without alternatives): bound by its latencies, launch, loads, two barriers and the
// comparisons.
template <class T, bool PART, int OF>
__global__ __launch_bounds__(OF) void logprobs_kernel(LogprobArgs a) {
  __shared__ Online part[2][OF / 64];
  __shared__ TopLds<OF> top;
  constexpr int N = RowSpan<T>::kPer, kMarks = TopLds<OF>::kMarks;
  const int tid = (int)threadIdx.x, segs = PART ? a.segs : 1;
  const float c = 2.0f * a.scale * kLog2E;
  int turn = 0;
  for (long long i = blockIdx.x; i < a.rows * segs; i += gridDim.x, turn ^= 1) {
    const long long row = PART ? i / segs : i;
    const int seg = PART ? (int)(i - row * segs) : 0;
    RowAnswer<T, OF> answer(a, row);
    const RowSpan<T> z(answer.z, a.classes, seg, segs);
    const int groups = (z.chunks + OF * kUnroll - 1) / (OF * kUnroll);
    const int per_mark = (groups + kMarks - 1) / kMarks;       // groups of a stretch
    const int extra = z.beside(tid);
    Online o{-INFINITY, 0.0f, 0.0f};
    const float x0 = extra >= 0 ? as_float(z.z[extra]) : -INFINITY;
    float stretch = -INFINITY;
    uint4 raw[kUnroll], first;
    load_chunks<OF>(z, 0, raw);
    first = raw[0];
    for (int g = 0, in = 0, mark = 0; g < groups; ++g) {
      float x[kUnroll * N], most = -INFINITY;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) unpack(raw[u], x + u * N, (const T*)nullptr);
      if (g + 1 < groups) load_chunks<OF>(z, (g + 1) * OF * kUnroll, raw);      // on their way meanwhile
#pragma unroll
      for (int e = 0; e < kUnroll * N; ++e) most = fmaxf(most, x[e]);
      o.template take<kUnroll * N>(x, most, c);
      stretch = fmaxf(stretch, most);
      if (++in == per_mark || g + 1 == groups) {
        if (a.top) top.mark[mark][tid] = stretch;
        stretch = -INFINITY;
        in = 0;
        ++mark;
      }
    }
    o.template take<1>(&x0, x0, c);
    if (a.top) offer_lane(top, turn, tid < z.chunks || extra >= 0 ? (uint32_t)(rank_key(o.m, 0) >> 32) : 0);
    o = over_workgroup<OF / 64>(o, part[turn], c);
    const bool bad = o.sum != o.sum;
    // the classes of a chunk that reach the bound
    const auto look = [&](const Bound& b, const uint4& chunk, int ch) {
      float x[N];
      unpack(chunk, x, (const T*)nullptr);
      const int v = z.from + ch * N;
      uint32_t reach = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) reach |= (b.met(x[e], v) ? 1u : 0u) << e;
      for (; reach; reach &= reach - 1) {
        const int e = __builtin_ctz(reach);
        float y = x[0];
#pragma unroll
        for (int f = 1; f < N; ++f) y = e == f ? x[f] : y;
        const uint64_t key = rank_key(y, (uint32_t)(v + e));
        if (key >= b.key) add_found(top, turn, key);
      }
    };
    const auto scan = [&](uint64_t bound) {
      const Bound b(bound);
      if (extra >= 0 && rank_key(x0, (uint32_t)extra) >= bound) add_found(top, turn, rank_key(x0, (uint32_t)extra));
      if (z.chunks <= OF) {      // one a lane, still at hand
        if (tid < z.chunks) look(b, first, tid);
        return;
      }
      for (int mark = 0; mark * per_mark < groups; ++mark)
        if (b.met(top.mark[mark][tid], (uint32_t)z.from + (uint32_t)(mark * per_mark * OF * kUnroll + tid) * N))
          top.stretch[atomicAdd(&top.stretches[turn], 1)] = (uint16_t)(mark * OF + tid);
      __syncthreads();
      const int each = per_mark * kUnroll, all = top.stretches[turn] * each;
      for (int j = tid; j < all; j += OF) {
        const int s = each == kUnroll ? j / kUnroll : j / each, at = top.stretch[s];
        const int ch = at / OF * each * OF + at % OF + (j - s * each) * OF;
        if (ch < z.chunks) look(b, z.body[ch], ch);
        if (*(volatile int*)&top.count[turn] > TopLds<OF>::kCandidates) break;
      }
    };
    if (PART) {
      if (tid == 0) a.parts[i] = o;
      if (!a.top) continue;
      const int n = bad ? 0 : find_top(top, turn, a.top, rank_key(-INFINITY, (uint32_t)((seg ? z.from : 0) + 2 * a.top - 1)), scan);
      uint64_t* const keys = a.keys + row * segs * a.top + seg;
      for (int k = tid; k < n; k += OF) {
        const int r = rank_among(top.found, n, top.found[k]);
        if (r < a.top) keys[r * segs] = top.found[k];
      }
      for (int k = n + tid; k < a.top; k += OF) keys[k * segs] = 0;
    } else {
      answer.put(o);
      if (a.top && !bad) answer.put_top(top.found, find_top(top, turn, a.top, rank_key(-INFINITY, (uint32_t)(2 * a.top - 1)), scan));
    }
  }
}

// The parts of rows joined.  Keys lie by rank, so that a lane's first one is among the greatest of its part.
template <class T>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(LogprobArgs a) {
  __shared__ TopLds<kThreads> top;
  const int tid = (int)threadIdx.x, n_keys = a.segs * a.top;
  int turn = 0;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    RowAnswer<T, kThreads> answer(a, row);
    const uint64_t* const keys = a.keys + row * n_keys;
    uint64_t mine = 0;
    for (int k = tid; k < n_keys; k += kThreads) mine = keys[k] > mine ? keys[k] : mine;
    if (a.top) offer_lane(top, turn, (uint32_t)(mine >> 32));
    answer.put(join_parts(a.parts + row * a.segs, a.segs, Online{-INFINITY, 0.0f, 0.0f}, 2.0f * a.scale * kLog2E));
    if (!a.top) continue;
    __syncthreads();
    if (answer.bad) continue;
    const auto scan = [&](uint64_t bound) {
      for (int k = tid; k < n_keys && mine >= bound; k += kThreads)
        if (keys[k] && keys[k] >= bound) add_found(top, turn, keys[k]);
    };
    answer.put_top(top.found, find_top(top, turn, a.top, 1, scan));
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
  int segs, n_parts;       // parts of a row that this launch works on, and that the launch before it did (0: none)
  float* parts;            // [rows][parts][3]
};

// The teacher's side of a row and the logits that its terms ask for, taken by the first wavefront while the others start on the row.
struct TeacherLds {
  alignas(16) int id[CG_TOP_MAX];        // -1: absent, or no class
  alignas(16) float q[CG_TOP_MAX];
  float log_q[CG_TOP_MAX], z[CG_TOP_MAX];
  float mass, z_label;
  int beyond;                    // an id names no class
};

template <class T>
__device__ __forceinline__ void take_teacher(TeacherLds& l, const DistillArgs& a, long long row, const T* z, int64_t label) {
  const int lane = (int)threadIdx.x;
  constexpr int kEach = CG_TOP_MAX / 64;
  int64_t id[kEach];
  float t[kEach], most = -INFINITY, mass = 0.0f;
  bool beyond = false;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int at = lane + 64 * k;
    id[k] = at < a.top ? a.top_ids[row * a.top + at] : -1;
    t[k] = id[k] >= 0 ? a.top_logits[row * a.top + at] : -INFINITY;
    most = fmaxf(most, t[k]);
    beyond |= id[k] >= a.classes;
  }
  if (lane == 0) l.z_label = label >= 0 && label < a.classes ? as_float(z[label]) : 0.0f;
  most = max_over_lanes(most);
  if (most == -INFINITY) most = 0.0f;
  float e[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    t[k] = half_apart(t[k], most) * (2.0f * a.scale);
    e[k] = pow2(t[k] * kLog2E);
    mass += e[k];
  }
  mass = sum_over_lanes(mass);
  const float log_mass = logf(mass);
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int at = lane + 64 * k;
    const bool named = id[k] >= 0 && id[k] < a.classes;
    l.id[at] = named ? (int)id[k] : -1;
    l.q[at] = mass != 0.0f ? e[k] / mass : 0.0f;
    l.log_q[at] = t[k] - log_mass;
    l.z[at] = named ? as_float(z[id[k]]) : 0.0f;
  }
  if (lane == 0) l.mass = mass;
  beyond = __any(beyond);
  if (lane == 0) l.beyond = beyond;
}

// A row's sums for the one or two temperatures of a call: m the greatest logit, `sum` of 2^((z - m) / 2 * c), `sum1` (TWO) of 2^((z - m) log2 e).
template <bool TWO>
struct Sums {
  float m, sum, sum1;
  __device__ void raise(float to, float c) {
    const float d = half_apart(m, to);
    sum *= pow2(fmaxf(d * c, kLeast));
    if (TWO) sum1 *= pow2(fmaxf(d * (2.0f * kLog2E), kLeast));
    m = to;
  }
  template <int N>
  __device__ void take(const float* x, float most, float c) {
    if (most > m) raise(most, c);
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = half_apart(x[i], from);
      sum += pow2(d * c);
      if (TWO) sum1 += pow2(d * (2.0f * kLog2E));
    }
  }
  __device__ void add(const Sums& b) {
    sum += b.sum;
    if (TWO) sum1 += b.sum1;
  }
  __device__ void over_lanes() {
    sum = sum_over_lanes(sum);
    if (TWO) sum1 = sum_over_lanes(sum1);
  }
};

__device__ __forceinline__ uint4 pack(const float* g, const float*) {
  return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
}
__device__ __forceinline__ uint4 pack(const float* g, const uint16_t*) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)float_to_bf16(g[2 * i]) | (uint32_t)float_to_bf16(g[2 * i + 1]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The exponentials' factor of the first sum (the only one, or the teacher's).
__device__ __forceinline__ float first_factor(const DistillArgs& a) { return 2.0f * kLog2E * (a.w_teacher != 0.0f ? a.scale : 1.0f); }

template <class T, int kOf, bool TWO>
__device__ __forceinline__ void take_chunks(Sums<TWO>& o, const uint4* raw, float c) {
  constexpr int N = RowSpan<T>::kPer;
  float x[kOf * N], most = -INFINITY;
#pragma unroll
  for (int u = 0; u < kOf; ++u) unpack(raw[u], x + u * N, (const T*)nullptr);
#pragma unroll
  for (int i = 0; i < kOf * N; ++i) most = fmaxf(most, x[i]);
  o.template take<kOf * N>(x, most, c);
}

template <class T, int OF, bool TWO>
__device__ __forceinline__ Sums<TWO> sums_of(const RowSpan<T>& z, int extra, float c, Sums<TWO>* part) {
  Sums<TWO> o{-INFINITY, 0.0f, 0.0f};
  const float x0 = extra >= 0 ? as_float(z.z[extra]) : -INFINITY;
  for (int first = 0; first < z.chunks; first += OF * kUnroll) {
    uint4 raw[kUnroll];
    load_chunks<OF>(z, first, raw);
    take_chunks<T, kUnroll>(o, raw, c);
  }
  o.template take<1>(&x0, x0, c);
  return over_workgroup<OF / 64>(o, part, c);
}

template <bool TWO>
__device__ __forceinline__ void put_stats(const DistillArgs& a, long long row, const Sums<TWO>& o) {
  a.stats[row * 3] = o.m;
  a.stats[row * 3 + 1] = a.w_label == 0.0f ? NAN : TWO ? o.sum1 : o.sum;
  a.stats[row * 3 + 2] = a.w_teacher == 0.0f ? NAN : o.sum;
}

// What a row's terms are, once its teacher and its sums are known.
template <bool TWO>
struct Terms {
  bool taught, labelled, none;
  float wt, wl;            // weights; NaN where a label or an entry is no number or names no class
  float ct, cl;            // and with the gradient from above and 1 / temperature
  float kt, k1;            // the exponentials' factors in the gradient
  float m, c;
  __device__ Terms(const DistillArgs& a, long long row, const TeacherLds& l, const Sums<TWO>& o, int64_t label, float up) {
    taught = a.w_teacher != 0.0f && (l.mass != 0.0f || l.beyond);
    labelled = label >= 0;
    none = o.sum == 0.0f || (!taught && !labelled);
    wt = !taught ? 0.0f : l.beyond || l.mass != l.mass ? NAN : a.w_teacher;
    wl = !labelled ? 0.0f : label >= a.classes ? NAN : a.w_label;
    ct = up * wt * a.scale, cl = up * wl;
    k1 = TWO && labelled ? cl / o.sum1 : 0.0f;
    kt = (taught ? ct / o.sum : 0.0f) + (!TWO && labelled ? cl / o.sum : 0.0f);
    m = o.m, c = first_factor(a);
  }
  // the probabilities' part of a class's gradient
  __device__ float slope(float x) const {
    const float y = half_apart(x, m), p = kt * pow2(y * c);
    return none ? 0.0f : TWO ? fmaf(k1, pow2(y * (2.0f * kLog2E)), p) : p;
  }
};

// The loss of a row, by its first wavefront.
template <bool TWO>
__device__ __forceinline__ void put_loss(const DistillArgs& a, long long row, const TeacherLds& l, const Sums<TWO>& o, const Terms<TWO>& t) {
  const float log_sum = logf(o.sum);
  float loss = 0.0f;
  for (int k = (int)threadIdx.x; k < a.top && t.taught; k += 64)
    if (l.q[k] != 0.0f) loss += l.q[k] * (l.log_q[k] - (half_apart(l.z[k], o.m) * (2.0f * a.scale) - log_sum));
  loss = sum_over_lanes(loss);
  loss = t.taught ? loss * t.wt : 0.0f;
  if (t.labelled) loss += t.wl * ((TWO ? logf(o.sum1) : log_sum) - (l.z_label - o.m));
  if (threadIdx.x == 0) a.loss[row] = t.none ? 0.0f : loss;
}

// The class of the teacher's entry or of the label (entry a.top) that a thread writes again at the end, and the gradient there, in full and rounded once.
template <class T, bool TWO>
struct Named {
  int at;                  // -1: none
  float value;
  template <class Here>
  __device__ Named(const DistillArgs& a, const TeacherLds& l, const Terms<TWO>& t, int64_t label, int entry, Here here) {
    const int64_t id = entry < a.top ? l.id[entry] : entry == a.top ? label : -1;
    at = id >= 0 && !t.none && here(id) ? (int)id : -1;
    if (at < 0) return;
    float minus = 0.0f;
    if (t.taught) {
#pragma unroll 2
      for (int k = 0; k < a.top; k += 4) {       // (entries behind the last one are absent)
        const int4 ids = *(const int4*)(l.id + k);
        const float4 q = *(const float4*)(l.q + k);
        minus += (ids.x == at ? q.x : 0.0f) + (ids.y == at ? q.y : 0.0f) + (ids.z == at ? q.z : 0.0f) + (ids.w == at ? q.w : 0.0f);
      }
    }
    value = t.slope(entry < a.top ? l.z[entry] : l.z_label) - t.ct * minus - (t.labelled && at == label ? t.cl : 0.0f);
  }
  __device__ void put_into(T* g) const {
    if (at >= 0) put(g + at, value);
  }
};

template <class T, bool TWO>
__device__ __forceinline__ uint4 slopes_of(const Terms<TWO>& t, const uint4& raw) {
  constexpr int N = RowSpan<T>::kPer;
  float x[N];
  unpack(raw, x, (const T*)nullptr);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = t.slope(x[i]);
  return pack(x, (const T*)nullptr);
}

// the sums of parts of rows, where rows are shared out
template <class T, bool TWO>
__global__ __launch_bounds__(kThreads) void distill_part_kernel(DistillArgs a) {
  __shared__ Sums<TWO> part[2][kThreads / 64];
  int turn = 0;
  for (long long i = blockIdx.x; i < a.rows * a.segs; i += gridDim.x, turn ^= 1) {
    const long long row = i / a.segs;
    const RowSpan<T> z((const T*)a.logits + row * a.stride, a.classes, (int)(i - row * a.segs), a.segs);
    const Sums<TWO> o = sums_of<T, kThreads>(z, z.beside((int)threadIdx.x), first_factor(a), part[turn]);
    if (threadIdx.x == 0) ((Sums<TWO>*)a.parts)[i] = o;
  }
}

// Loss and gradient of a row, or of one of `segs` parts of it.  One pass for the sums (none where the call brings them, or where a launch before
// has formed those of parts), one that writes the gradient: for every class the probabilities' part; then the classes that the label or the teacher
// names are written again.  TWO: both terms are there at different temperatures, that is two sums and two exponentials an element.  Bound by memory: the loss of
// 4096 rows of 131072 classes in bf16 192 us (5.6 TB/s), the gradient from given sums 396 us (5.4 TB/s read and written).
template <class T, bool TWO, int OF>
__global__ __launch_bounds__(OF) void distill_kernel(DistillArgs a) {
  __shared__ Sums<TWO> part[OF / 64];
  __shared__ TeacherLds teacher;
  constexpr int N = RowSpan<T>::kPer;
  const int tid = (int)threadIdx.x;
  const float c = first_factor(a);
  for (long long i = blockIdx.x; i < a.rows * a.segs; i += gridDim.x) {
    const long long row = i / a.segs;
    const int seg = (int)(i - row * a.segs);
    const RowSpan<T> z((const T*)a.logits + row * a.stride, a.classes, seg, a.segs);
    const int64_t label = a.labels && a.w_label != 0.0f ? a.labels[row] : -1;
    const float up = a.grad && a.grad_loss ? a.grad_loss[row] : 1.0f;
    const int extra = z.beside(tid);
    if (tid < 64) take_teacher(teacher, a, row, z.z, label);
    Sums<TWO> o{-INFINITY, 0.0f, 0.0f};
    uint4 raw[kUnroll];
    float x0 = 0.0f;
    const auto load = [&](int at) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (at + u * OF < z.chunks) raw[u] = z.body[at + u * OF];
    };
    const bool known = a.given_stats || a.n_parts;
    if (!known) o = sums_of<T, OF>(z, extra, c, part);
    if (a.grad) {          // on their way while the sums are joined and the teacher is waited for
      load(tid);
      if (extra >= 0) x0 = as_float(z.z[extra]);
    }
    if (a.given_stats) {
      const float* const st = a.given_stats + row * 3;
      o = Sums<TWO>{st[0], a.w_teacher != 0.0f ? st[2] : st[1], st[1]};
    } else if (a.n_parts) {
      o = join_parts((const Sums<TWO>*)a.parts + row * a.n_parts, a.n_parts, o, c);
    }
    if (known) __syncthreads();
    if (a.stats && seg == 0 && tid == 0) put_stats(a, row, o);
    const Terms<TWO> terms(a, row, teacher, o, label, up);
    if (a.loss && seg == 0 && tid < 64) put_loss(a, row, teacher, o, terms);
    if (a.grad) {
      T* const g = (T*)a.grad + row * a.grad_stride;
      const auto here = [&](int64_t v) { return z.holds(v); };
      const Named<T, TWO> named(a, teacher, terms, label, tid, here);
      const bool same_phase = (((uintptr_t)g ^ (uintptr_t)z.z) & 15) == 0;
      if (extra >= 0) put(g + extra, terms.slope(x0));
      for (int at = tid; at < z.chunks; at += OF * kUnroll) {
        if (at != tid) load(at);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int ch = at + u * OF;
          if (ch >= z.chunks) continue;
          const uint4 v = slopes_of<T, TWO>(terms, raw[u]);
          T* const out = g + z.from + ch * N;
          if (same_phase) {
            *(uint4*)out = v;
          } else {
#pragma unroll
            for (int e = 0; e < N; ++e) out[e] = ((const T*)&v)[e];
          }
        }
      }
      __syncthreads();
      named.put_into(g);
      for (int entry = OF + tid; entry <= a.top; entry += OF) Named<T, TWO>(a, teacher, terms, label, entry, here).put_into(g);     // (64 threads)
    }
    __syncthreads();       // (the next row's teacher takes the place of this one's)
  }
}

// Loss and gradient in one pass: kHeld chunks a lane stay in the registers of the row's workgroup between the sums and the gradient (256 KB by 1024 threads,
// half of a compute unit's registers), and as the gradient leaves, the next row's chunks take their place, so that loads and stores are on their way together.
// A workgroup walks rows.  What a longer row has beside (1024 threads only) is read twice.  Rows of logits and gradient have the same alignment to 16 bytes.
// Bound by memory: 4096 rows of 131072 classes in bf16 461 us, 4.66 TB/s of one read and one write an element, where a plain copy reaches 4.83 and the gradient
// from given sums, which moves as much, 5.4; read twice by distill_kernel they took 647 us.  Rows of 50003 in bf16 192 us, by distill_kernel 243 (where a
// gradient given by the caller has another alignment than the logits).  2048 rows of 131072 in fp32 (twice what is held) 494 and 648 us, of 200003 839 and 1103
// us.
constexpr int kHeld = 16, kMore = 2;       // kMore: chunks a lane takes at once of what is beside
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class T, bool TWO, int OF>
__global__ __launch_bounds__(OF, 4) void distill_held_kernel(DistillArgs a) {
  __shared__ Sums<TWO> part[2][OF / 64];
  __shared__ TeacherLds teachers[2];
  constexpr int kTake = sizeof(T) == 2 ? 2 : 4;       // chunks between two looks at the maximum
  const int tid = (int)threadIdx.x;
  const float c = first_factor(a);
  uint4 raw[kHeld];
  float x0 = 0.0f;
  int turn = 0;
  const auto row_at = [&](long long row) { return RowSpan<T>((const T*)a.logits + row * a.stride, a.classes, 0, 1); };
  const auto held = [](const RowSpan<T>& z) { return z.chunks < kHeld * OF ? z.chunks : kHeld * OF; };
  const auto load = [&](__amdgpu_buffer_rsrc_t from, int u) {
    raw[u] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, (tid + u * OF) * 16, 0, 0));
  };
  const auto load_extra = [&](const RowSpan<T>& z) {
    const int extra = z.beside(tid);
    x0 = extra >= 0 ? as_float(z.z[extra]) : -INFINITY;
  };
  long long row = blockIdx.x;
  {
    const RowSpan<T> z = row_at(row);
    const __amdgpu_buffer_rsrc_t from = chunk_buffer(z.body, held(z));
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
      if (u * OF < z.chunks) load(from, u);
    load_extra(z);
  }
  for (;; turn ^= 1) {
    TeacherLds& teacher = teachers[turn];
    const RowSpan<T> z = row_at(row);
    const int64_t label = a.labels && a.w_label != 0.0f ? a.labels[row] : -1;
    const float up = a.grad_loss ? a.grad_loss[row] : 1.0f;
    if (tid < 64) take_teacher(teacher, a, row, z.z, label);
    Sums<TWO> o{-INFINITY, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < kHeld; u += kTake) {
      if (u * OF >= z.chunks) break;
      if ((u + kTake) * OF > z.chunks) {
#pragma unroll
        for (int v = u; v < u + kTake; ++v)
          if (tid + v * OF >= z.chunks) raw[v] = all_minus_inf<T>();
      }
      take_chunks<T, kTake>(o, raw + u, c);
    }
    if (OF == 1024) {        // what a longer row has beside, a second time below
#pragma unroll 1
      for (int first = kHeld * OF; first < z.chunks; first += OF * kMore) {
        uint4 some[kMore];
        load_chunks<OF>(z, first, some);
        take_chunks<T, kMore>(o, some, c);
      }
    }
    o.template take<1>(&x0, x0, c);
    o = over_workgroup<OF / 64>(o, part[turn], c);
    if (a.stats && tid == 0) put_stats(a, row, o);
    const Terms<TWO> terms(a, row, teacher, o, label, up);
    if (tid < 64) put_loss(a, row, teacher, o, terms);
    T* const g = (T*)a.grad + row * a.grad_stride;
    const auto here = [&](int64_t v) { return v < a.classes; };
    const Named<T, TWO> named(a, teacher, terms, label, tid, here);
    if (const int extra = z.beside(tid); extra >= 0) put(g + extra, terms.slope(x0));
    if (OF == 1024) {
#pragma unroll 1
      for (int first = kHeld * OF; first < z.chunks; first += OF * kMore) {
        uint4 some[kMore];
        load_chunks<OF>(z, first, some);
        const __amdgpu_buffer_rsrc_t to = chunk_buffer(g + z.from + (long long)first * RowSpan<T>::kPer, z.chunks - first < OF * kMore ? z.chunks - first : OF * kMore);
#pragma unroll
        for (int u = 0; u < kMore; ++u)
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, slopes_of<T, TWO>(terms, some[u])), to, (tid + u * OF) * 16, 0, 0);
      }
    }
    const long long next = row + gridDim.x;
    const bool more = next < a.rows;
    const RowSpan<T> zn = row_at(more ? next : row);
    const __amdgpu_buffer_rsrc_t to = chunk_buffer(g + z.from, held(z)), from = chunk_buffer(zn.body, more ? held(zn) : 0);
#pragma unroll
    for (int u = 0; u < kHeld; ++u) {
      if (u * OF < z.chunks) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, slopes_of<T, TWO>(terms, raw[u])), to, (tid + u * OF) * 16, 0, 0);
      if (u * OF < zn.chunks) load(from, u);
    }
    if (more) load_extra(zn);
    __syncthreads();
    named.put_into(g);
    for (int entry = OF + tid; entry <= a.top; entry += OF) Named<T, TWO>(a, teacher, terms, label, entry, here).put_into(g);     // (64 threads)
    if (!more) return;
    row = next;
  }
}

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int element_bytes(int dtype) { return dtype == CG_F32 ? 4 : 2; }

// what both operators ask of the logits
int check_logits(const char* who, const void* logits, int32_t dtype, int64_t rows, int32_t classes, int64_t row_stride, float temperature) {
  if (rows < 0 || classes <= 0) return cg::set_error(CG_EINVAL, "%s: bad size", who);
  if (dtype != CG_F32 && dtype != CG_BF16) return cg::set_error(CG_EUNSUPPORTED, "%s: logits are CG_F32 or CG_BF16", who);
  if (row_stride < 0) return cg::set_error(CG_EINVAL, "%s: row_stride must not be negative", who);
  if (!(temperature > 0.0f) || !std::isfinite(temperature) || !std::isnormal(1.0f / temperature) || !std::isfinite(2.0f / temperature * kLog2E))
    return cg::set_error(CG_EINVAL, "%s: temperature must be positive and lie between 2^-126 and 2^126", who);
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

// How rows are given to workgroups.  `chunks` are 16 bytes; 256 threads take kPart of them at once.
constexpr int64_t kPart = kThreads * kUnroll;
int64_t chunks_in(int64_t classes, int bytes) { return classes * bytes / 16; }

// Parts of rows that are shared out, in a first launch for their sums and a second one that joins them: a few long rows, in parts of 16 KB and as many as
// make `enough` workgroups, `fewest` at least.  One row of 131072 classes in bf16 with 20 alternatives 19.1 us whole, 10.8 us in 16 parts; 64 rows 20.4 and
// 14.7 (8 parts), 128 rows 20.6 and 17.6 (4), 256 rows 21.2 and 23.3 (2); rows of 64 KB are never faster in parts (one row 8.7 and 11.1).  The loss alone, 32
// teacher classes: 16 rows 11.0 and 7.8 us, 64 rows 12.2 and 11.1 (8 parts), 128 rows 12.8 and 14.0 (4).  Loss and gradient: one row 17.5 and 8.5,
// 64 rows 21.3 and 16.7, 128 rows 24.0 and 23.3 (8 parts), 192 rows 27.3 and 34.3.
constexpr int kEnough = 512;
int parts_of(int64_t rows, int64_t chunks, int enough, int fewest) {
  if (rows <= 0 || enough / rows < fewest || chunks <= 4 * kPart) return 1;
  return (int)std::min<int64_t>(enough / rows, (chunks + kPart - 1) / kPart);
}
int logprob_parts(int64_t rows, int64_t chunks) { return parts_of(rows, chunks, kEnough, 4); }
int distill_parts(int64_t rows, int64_t chunks, bool grad) { return parts_of(rows, chunks, grad ? 2 * kEnough : kEnough, 8); }

// Many short rows: a wavefront each, while 256 threads had too little to do between their barriers.  Alternatives: 4096 rows of 2048 classes in bf16 11.3 us, by
// workgroups of 256 threads 25.5 us; 1024 rows of 4096 8.1 and 9.0, of 8192 10.7 and 10.2; 256 rows of 2048 6.7 and 6.4.  The loss alone: 4096 rows of 1000 7.7 and
// 16.8 us, of 8192 17.3 and 21.6; 512 rows of 4096 5.3 and 5.4, of 8192 6.4 and 5.4.
bool wavefront_each(int64_t rows, int64_t chunks) { return rows >= 512 && chunks <= std::min<int64_t>(rows / 2, 1024); }

template <class T>
void launch_logprobs(const LogprobArgs& a, hipStream_t s) {
  if (a.segs > 1) {
    hipLaunchKernelGGL((logprobs_kernel<T, true, 256>), dim3((unsigned)(a.rows * a.segs)), dim3(256), 0, s, a);
    hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a);
  } else if (wavefront_each(a.rows, chunks_in(a.classes, sizeof(T))) && a.top <= 32) {       // (a bound from 64 lanes)
    hipLaunchKernelGGL((logprobs_kernel<T, false, 64>), dim3(row_groups(a.rows)), dim3(64), 0, s, a);
  } else {
    hipLaunchKernelGGL((logprobs_kernel<T, false, 256>), dim3(row_groups(a.rows)), dim3(256), 0, s, a);
  }
}

// Threads of distill_held_kernel for a row: as few as hold it, and more as long as all of them find room at once (1024 threads on each of 256 compute units)
// and each has four chunks.  32768 classes in bf16: 64 rows 9.6 us on 256 threads, 8.1 on 512, 8.0 on 1024, 512 rows 18.9, 18.0 and 19.3, 1024 rows 32.8, 33.5
// and 38.5; rows of 1000 in fp32 on 64 and on 256 threads: 4096 rows 12.4 and 22.5 us, 1024 6.3 and 7.1, 512 5.8 and 5.8, 128 5.4 and 5.2, one 5.0 and 4.8.
constexpr int64_t kRoom = 256 * 1024;
int held_threads(int64_t rows, int64_t chunks) {
  int of = 64;
  while (of < 1024) {
    const int more = of == 64 ? 256 : of * 2;
    if (chunks <= kHeld * of && (rows * more > kRoom || chunks < 4 * more)) break;
    of = more;
  }
  return of;
}

template <class T, bool TWO>
void launch_held(const DistillArgs& a, int64_t chunks, hipStream_t s) {
  const int of = held_threads(a.rows, chunks);
  const dim3 grid((unsigned)std::min<int64_t>(a.rows, kRoom / of));
  if (of == 64)
    hipLaunchKernelGGL((distill_held_kernel<T, TWO, 64>), grid, dim3(64), 0, s, a);
  else if (of == 256)
    hipLaunchKernelGGL((distill_held_kernel<T, TWO, 256>), grid, dim3(256), 0, s, a);
  else if (of == 512)
    hipLaunchKernelGGL((distill_held_kernel<T, TWO, 512>), grid, dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((distill_held_kernel<T, TWO, 1024>), grid, dim3(1024), 0, s, a);
}

// a.segs parts a row by workgroups of 256 threads; whole rows also by wavefronts, and long ones by 512 threads up to two rows a compute unit.  On 512 and on
// 256 threads, bf16: the loss alone, 256 rows of 131072 classes 14.4 and 19.2 us; of 32768 128 rows 5.8 and 8.0, 256 7.3 and 8.5, 384 9.4 and 10.0, 512 10.7
// and 10.8, 640 14.2 and 12.1; of 16384 128 rows 4.9 and 5.4, 512 7.8 and 8.0; at two temperatures 384 rows of 32768 10.9 and 11.7, 640 15.9 and 14.6.  Loss
// and gradient at another alignment: 256 rows of 16384 8.5 and 10.2, 384 of 50003 23.4 and 25.9, 512 28.6 and 29.6, 640 43.2 and 40.7.  The gradient alone
// comes here whole with 512 rows of 16384 to 32767 only: 16384 11.2 and 10.8, 24000 12.7 and 12.9.
template <class T, bool TWO>
void launch_rows_of(const DistillArgs& a, int64_t chunks, hipStream_t s) {
  const dim3 grid(row_groups(a.rows * a.segs));
  if (a.segs == 1 && wavefront_each(a.rows, chunks))
    hipLaunchKernelGGL((distill_kernel<T, TWO, 64>), grid, dim3(64), 0, s, a);
  else if (a.segs == 1 && !a.n_parts && a.rows <= 512 && chunks >= 2 * kPart)
    hipLaunchKernelGGL((distill_kernel<T, TWO, 512>), grid, dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((distill_kernel<T, TWO, 256>), grid, dim3(256), 0, s, a);
}

template <class T, bool TWO>
void launch_distill_as(DistillArgs a, hipStream_t s) {
  const int64_t chunks = chunks_in(a.classes, sizeof(T));
  if (a.given_stats) {
    // The gradient alone, in parts of 32 KB (16 KB where those are few): 1024 rows of 131072 classes in bf16 105.5 us, by whole rows 117.9; 64 rows 10.7 and 22.9.
    const int64_t parts = std::max<int64_t>(1, chunks / (2 * kPart));
    a.segs = (int)(a.rows * parts < kEnough ? std::max<int64_t>(1, chunks / kPart) : parts);
    launch_rows_of<T, TWO>(a, chunks, s);
    return;
  }
  const bool same_phase = (((uintptr_t)a.grad ^ (uintptr_t)a.logits) & 15) == 0 && (a.rows == 1 || (a.grad_stride - a.stride) * (int)sizeof(T) % 16 == 0);
  const int segs = distill_parts(a.rows, chunks, a.grad != nullptr);
  if (segs > 1) {
    a.segs = segs;
    hipLaunchKernelGGL((distill_part_kernel<T, TWO>), dim3((unsigned)(a.rows * segs)), dim3(kThreads), 0, s, a);
    a.n_parts = segs;
    if (!a.grad) {
      a.segs = 1;
    } else if (a.grad == a.logits) {      // the loss asks for logits that another part's workgroup replaces by their gradient: it goes first
      DistillArgs first = a;
      first.grad = nullptr;
      first.segs = 1;
      launch_rows_of<T, TWO>(first, chunks, s);
      a.loss = nullptr;
    }
    launch_rows_of<T, TWO>(a, chunks, s);
  } else if (a.grad && same_phase) {
    launch_held<T, TWO>(a, chunks, s);
  } else {
    launch_rows_of<T, TWO>(a, chunks, s);
  }
}

template <class T>
void launch_distill_of(const DistillArgs& a, hipStream_t s) {
  if (a.scale != 1.0f && a.w_teacher != 0.0f && a.w_label != 0.0f)
    launch_distill_as<T, true>(a, s);
  else
    launch_distill_as<T, false>(a, s);
}

int launch_distill(const char* who, const DistillArgs& a, int32_t dtype, hipStream_t s) {
  if (dtype == CG_F32)
    launch_distill_of<float>(a, s);
  else
    launch_distill_of<uint16_t>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cg::set_error(CG_EHIP, "%s: %s", who, hipGetErrorString(e));
  return CG_OK;
}

}  // namespace

extern "C" {

size_t cg_logprobs_workspace_bytes(int64_t rows, int32_t classes, int32_t top) {
  if (rows <= 0 || classes <= 0 || top < 0 || top > CG_TOP_MAX) return 0;
  const int segs = logprob_parts(rows, chunks_in(classes, 4));      // (the larger of the two types' needs)
  return segs == 1 ? 0 : (size_t)rows * segs * (sizeof(Online) + 8 * (size_t)top);
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
  LogprobArgs a{logits, rows, row_stride, classes, given, top, 1, 1.0f / temperature, labels, logprob, entropy, top_ids, top_logprobs, nullptr, nullptr};
  a.segs = logprob_parts(rows, chunks_in(classes, element_bytes(dtype)));
  if (a.segs > 1) {
    a.keys = (uint64_t*)workspace;
    a.parts = (Online*)(a.keys + rows * a.segs * top);
  }
  if (dtype == CG_F32)
    launch_logprobs<float>(a, (hipStream_t)hip_stream);
  else
    launch_logprobs<uint16_t>(a, (hipStream_t)hip_stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cg::set_error(CG_EHIP, "%s: %s", who, hipGetErrorString(e));
  return CG_OK;
}

size_t cg_distill_workspace_bytes(int64_t rows, int32_t classes) {
  if (rows <= 0 || classes <= 0) return 0;
  const int segs = std::max(distill_parts(rows, chunks_in(classes, 4), false), distill_parts(rows, chunks_in(classes, 4), true));      // (fp32: the larger need)
  return segs == 1 ? 0 : (size_t)rows * segs * 3 * sizeof(float);
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
                      labels, grad_loss, nullptr, loss, stats, grad, 1, 0, (float*)workspace};
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
                      labels, grad_loss, stats, nullptr, nullptr, grad, 1, 0, nullptr};
  return launch_distill(who, a, dtype, (hipStream_t)hip_stream);
}

}  // extern "C"
