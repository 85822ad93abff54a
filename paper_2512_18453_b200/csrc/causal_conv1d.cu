// Short causal convolution per channel (nova_causal_conv1d).
//
// What bounds it: x read and y written once, 2 e bytes an element, and next to that the two special-function instructions of each
// SiLU.  A thread slides a window of W inputs over a run of rows, 16 bytes each, with the next seven or eight in flight.
// 2 x 4096 x 4096, 4 taps, bf16: 29.2 us (71 % of the copy rate), without SiLU 23.3 (89 %); 4096 x 4096 float without it 20.7
// (100 %), with it 22.5.  Where rows are on no such boundary, two channels a thread by themselves: 6000 packed rows of 777 halves
// 12.3 us (24 %), bound by instructions; with 64 registers, for eight CTAs an SM, most of these spill 4 to 52 bytes.
#include <type_traits>

#include "sm100.cuh"
#include "tma_host.h"
#include "token_mixer.cuh"

namespace nova {
namespace {
using namespace mix;

constexpr int kThreads = 128;
// CTAs of an SM: 128 registers for whole vectors, 64 for pairs
constexpr int resident(bool whole) { return whole ? 4 : 8; }

struct ConvArgs {
  Seqs q;
  Rows x, y;
  const void *weight, *bias;
  void* state;
  int channels, silu;
  int run;                         // rows of a run, at least those in flight
  unsigned items, runs;            // runs of rows: in all, and of a dense sequence or of all packed rows
  unsigned runs_mul, runs_shift;   // n / runs = (mulhi(n, mul) + n) >> shift for n < 2^31
};

// VEC neighbouring channels of one row in one access where rows are aligned to VEC elements; else two channels that are as far
// apart as the accesses of a warp are wide, so that each of them is contiguous.  `second`: how far, 0 where that one is behind the
// last channel.
template <typename T, int VEC, bool WHOLE>
struct Vec {
  static constexpr int BYTES = VEC * sizeof(T), H = VEC / 2;
  using Word = std::conditional_t<BYTES == 16, uint4, uint2>;
  static_assert(WHOLE ? BYTES == sizeof(Word) : VEC == 2);
  alignas(WHOLE ? sizeof(Word) : sizeof(T) * 2) T v[VEC];
  __device__ __forceinline__ static Vec load(const T* p, int second) {
    Vec r;
    if constexpr (WHOLE) {
      const Word w = *reinterpret_cast<const Word*>(p);
      memcpy(r.v, &w, BYTES);
    } else {
      r.v[0] = p[0];
      r.v[1] = p[second];
    }
    return r;
  }
  __device__ __forceinline__ void store(T* p, int second) const {
    if constexpr (WHOLE) {
      Word w;
      memcpy(&w, v, BYTES);
      *reinterpret_cast<Word*>(p) = w;
    } else {
      p[0] = v[0];
      if (second) p[second] = v[1];
    }
  }
  __device__ __forceinline__ void floats(float2 (&f)[H]) const {
#pragma unroll
    for (int h = 0; h < H; ++h) f[h] = load_pair(v + 2 * h);
  }
  __device__ __forceinline__ static Vec of(const float2 (&f)[H]) {
    Vec r;
#pragma unroll
    for (int h = 0; h < H; ++h) store_pair(r.v + 2 * h, f[h]);
    return r;
  }
  __device__ __forceinline__ static Vec zero() {
    Vec r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) r.v[i] = from_float<T>(0.f);
    return r;
  }
};

// A run is a.run rows.  The first of them of a sequence are its head: their run begins with the state, and the same thread
// leaves the final one, so that no other reads a slot that it writes.  Of packed sequences there is a run for every head and one
// for as many rows of all, which takes those behind the head of the sequence that its first row belongs to (rows of the next
// one are its head's).
template <typename T, int W, int VEC, bool WHOLE, int AHEAD>
__global__ void __launch_bounds__(kThreads, resident(WHOLE)) conv_kernel(const __grid_constant__ ConvArgs a) {
  static_assert(AHEAD >= W - 1, "a run behind a head needs no state");
  const int run = a.run;
  sm100::pdl_wait();
  sm100::pdl_launch_dependents();
  const unsigned item = blockIdx.x * blockDim.y + threadIdx.y;
  const unsigned column = blockIdx.y * blockDim.x + threadIdx.x, apart = min(32u, blockDim.x);
  const int d = WHOLE ? column * VEC : column / apart * (2 * apart) + column % apart;
  Seq s;
  int t, end;
  if (!a.q.cu) {
    if (item >= a.items) return;
    const unsigned i = (__umulhi(item, a.runs_mul) + item) >> a.runs_shift;      // a division takes the unit of the exponentials
    s = find_seq(a.q, (int)i, a.state != nullptr);
    t = (int)(item - i * a.runs) * run;
    end = t + run;
  } else {
    // the sequence of a run's first row: as many as end at or before it come before
    const long long first = ((long long)item - threadIdx.y - a.q.count) * run;          // of the CTA's first run; heads are below 0
    int before = 0;
    if (first + (long long)blockDim.y * run > 0)
      for (int i0 = 0; i0 < a.q.count; i0 += kThreads) {
        const int i = i0 + (int)(threadIdx.y * blockDim.x + threadIdx.x);
        long long ends = INT64_MAX;
        if (i < a.q.count) {
          const Seq c = find_seq(a.q, i, false);
          ends = c.at + c.len;
        }
        for (int j = 0; j < (int)blockDim.y; ++j) {
          const int n = __syncthreads_count(ends <= first + (long long)j * run);
          if (j == (int)threadIdx.y) before += n;
        }
      }
    if (item >= a.items) return;
    if (item < (unsigned)a.q.count) {
      s = find_seq(a.q, (int)item, a.state != nullptr);
      t = 0;
      end = run;
    } else {
      if (before >= a.q.count) return;
      s = find_seq(a.q, before, a.state != nullptr);
      const long long row = (long long)(item - a.q.count) * run;
      t = (int)max(row - s.at, (long long)run);
      end = (int)min(row + run - s.at, (long long)s.len);
    }
  }
  if (s.skip || d >= a.channels) return;
  end = min(end, s.len);
  if (t >= end) return;
  using V = Vec<T, VEC, WHOLE>;
  constexpr int H = V::H;
  const int second = d + (int)apart < a.channels ? (int)apart : 0;
  T* state = a.state ? (T*)a.state + (size_t)s.slot * (W - 1) * a.channels + d : nullptr;
  const bool head = t == 0;
  const T* x = row_ptr<const T>(a.x, s, t) + d;
  V in[W - 1], next[AHEAD];
#pragma unroll
  for (int k = 0; k < W - 1; ++k)
    in[k] = !head ? V::load(x + (k - (W - 1)) * a.x.row, second) : s.resume ? V::load(state + (size_t)k * a.channels, second) : V::zero();
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (t + i < end) next[i] = V::load(x + i * a.x.row, second);
  if (head && state) {
    if (s.len >= W - 1) {
#pragma unroll
      for (int k = 0; k < W - 1; ++k)
        V::load(row_ptr<const T>(a.x, s, s.len - (W - 1) + k) + d, second).store(state + (size_t)k * a.channels, second);
    } else {
#pragma unroll
      for (int len = 1; len < W - 1; ++len)
        if (s.len == len)
#pragma unroll
          for (int k = 0; k < W - 1; ++k) (k + len < W - 1 ? in[k + len] : next[k + len - (W - 1)]).store(state + (size_t)k * a.channels, second);
    }
  }
  // weights and bias as float, with SiLU scaled by 1/256 as silu_of_256th wants the sum (exactly but for floats below 2^-118)
  float2 w[W][H], b[H], win[W - 1][H];
  const float scale = a.silu ? 1.f / 256 : 1.f;
  {
    V taps[W];                                                  // VEC rows of W weights, one behind the other
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if constexpr (WHOLE) taps[k] = V::load((const T*)a.weight + (size_t)d * W + k * VEC, 0);
      else
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int at = k * VEC + e;                             // of both channels' weights, one behind the other
          taps[k].v[e] = ((const T*)a.weight)[(size_t)(at < W ? d : d + second) * W + at % W];
        }
    }
    (a.bias ? V::load((const T*)a.bias + d, second) : V::zero()).floats(b);
#pragma unroll
    for (int h = 0; h < H; ++h) b[h] = make_float2(b[h].x * scale, b[h].y * scale);
#pragma unroll
    for (int c = 0; c < VEC; ++c)
#pragma unroll
      for (int k = 0; k < W; ++k)
        (c & 1 ? w[k][c / 2].y : w[k][c / 2].x) = to_float(taps[(c * W + k) / VEC].v[(c * W + k) % VEC]) * scale;
  }
#pragma unroll
  for (int k = 0; k < W - 1; ++k) in[k].floats(win[k]);
  T* y = row_ptr<T>(a.y, s, t) + d;
  for (; t < end; t += AHEAD) {
    x += AHEAD * a.x.row;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      float2 row[H], v[H];
      next[i].floats(row);
      if (t + AHEAD + i < end) next[i] = V::load(x + i * a.x.row, second);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        v[h] = b[h];
#pragma unroll
        for (int k = 0; k < W - 1; ++k) v[h] = __ffma2_rn(w[k][h], win[k][h], v[h]);
        v[h] = __ffma2_rn(w[W - 1][h], row[h], v[h]);
#pragma unroll
        for (int k = 0; k < W - 2; ++k) win[k][h] = win[k + 1][h];
        win[W - 2][h] = row[h];
        if (a.silu) v[h] = silu_of_256th(v[h]);
      }
      if (t + i < end) V::of(v).store(y, second);
      y += a.y.row;
    }
  }
}

template <typename T, int W, int VEC, bool WHOLE, int AHEAD>
int start(ConvArgs a, cudaStream_t s) {
  const int columns = (a.channels + VEC - 1) / VEC;
  // threads across a row: as many as fill up with columns, at most a tenth more than the narrowest blocks would take
  int across = kThreads;
  while (across > 32 && (columns + across - 1) / across * across > (columns + 31) / 32 * 32 * 11 / 10) across /= 2;
  while (across / 2 >= columns) across /= 2;
  const int down = kThreads / across;
  const int column_blocks = (columns + across - 1) / across;           // 65535 at most: kThreads across and two channels each
  // one wave of CTAs where there are rows enough, so that each streams until the end
  const long long rows = a.q.cu ? a.q.tokens : a.q.tokens * a.q.count, wave = 148ll * resident(WHOLE) * down / column_blocks;
  long long run = (rows + wave) / (wave + 1);
  run = (run + AHEAD - 1) / AHEAD * AHEAD;
  a.run = (int)(run < AHEAD ? AHEAD : run > 4096 ? 4096 : run);
  const long long runs = (a.q.tokens + a.run - 1) / a.run, items = a.q.cu ? a.q.count + runs : a.q.count * runs;
  if (items >= INT32_MAX) return (int)cudaErrorInvalidConfiguration;
  a.items = (unsigned)items;
  a.runs = (unsigned)runs;
  a.runs_shift = 0;
  while ((1ll << a.runs_shift) < runs) ++a.runs_shift;
  a.runs_mul = (unsigned)(((1ull << 32) * ((1ull << a.runs_shift) - runs)) / runs + 1);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((items + down - 1) / down), column_blocks);
  cfg.blockDim = dim3(across, down);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return (int)cudaLaunchKernelEx(&cfg, conv_kernel<T, W, VEC, WHOLE, AHEAD>, a);
}
template <typename T, int W>
int start(const ConvArgs& a, cudaStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  const size_t e = sizeof(T);
  const bool vec = a.channels % VEC == 0 && rows_aligned(a.x, e, VEC * e) && rows_aligned(a.y, e, VEC * e) && aligned(a.state, VEC * e) && aligned(a.weight, VEC * e) && aligned(a.bias, VEC * e);
  // Rows in flight: eight, seven of two bytes with four taps, where eight do not fit the registers in half (bf16 / half, 2 x 4096 x
  // 4096: 8 rows 28.7 / 37.2 us, 7 rows 29.2 / 29.3; of seven, half spills one register).
  constexpr int AHEAD = sizeof(T) == 2 && W == 4 ? 7 : 8;
  // Short sequences: narrower, so that a token has more threads (channels a thread 8 / 4: one token of 1 x 1024 bf16 4.0 / 2.85 us, of
  // 256 x 4096 12.1 / 11.8; four tokens of 64 x 4096 5.0 / 4.4; 64 tokens of it 23.2 / 25.9)
  if (vec && !a.q.cu && a.q.tokens <= 4) return start<T, W, 4, true, 4>(a, s);
  return vec ? start<T, W, VEC, true, AHEAD>(a, s) : start<T, W, 2, false, 8>(a, s);
}
template <typename T>
int start(const ConvArgs& a, int width, cudaStream_t s) {
  return width == 2 ? start<T, 2>(a, s) : width == 3 ? start<T, 3>(a, s) : start<T, 4>(a, s);
}

}  // namespace
}  // namespace nova

extern "C" int nova_causal_conv1d(const nova_sequences* q, int type, const nova_rows* x, const void* weight, const void* bias,
                                  int channels, int width, void* state, const nova_rows* y, int flags, nova_stream stream) {
  using namespace nova;
  using namespace nova::mix;
  if (!type_ok(type) || !seqs_ok(q, state != nullptr) || !x || !y || channels <= 0 || channels > NOVA_CONV1D_MAX_CHANNELS || width < 2 || width > 4 || (flags & ~NOVA_SILU))
    return NOVA_ERR_INVALID_ARG;
  if (q->sequences == 0 || q->tokens == 0) return NOVA_OK;
  const size_t e = type_bytes(type);
  if (!rows_ok(*x, type) || !rows_ok(*y, type) || x->data_dev == y->data_dev || !weight || !aligned(weight, e) || !aligned(bias, e) ||
      !aligned(state, e))
    return NOVA_ERR_INVALID_ARG;
  // as many CTAs as the smallest variant takes
  if ((long long)((channels + kThreads - 1) / kThreads) * q->sequences > INT32_MAX) return NOVA_ERR_INVALID_ARG;
  const ConvArgs a = {make_seqs(q), make_rows(*x), make_rows(*y), weight, bias, state, channels, flags & NOVA_SILU};
  cudaStream_t s = (cudaStream_t)stream;
  return launch_status(type == NOVA_F32 ? start<float>(a, width, s)
                       : type == NOVA_F16 ? start<__half>(a, width, s) : start<__nv_bfloat16>(a, width, s));
}
