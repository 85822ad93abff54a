// Selective scan (nova_selective_scan).
//
// h_t = a_t h_{t-1} + b_t for every channel and state, a_t = exp(dt A), b_t = dt u B; y_t = sum_n C h.  A sequence is cut
// into pieces of TC tokens, and the warps of a CTA take them in turn.  Within a piece a warp starts from zeros and keeps, for
// every token, y as it comes out of that and w_t = C_t a_1 .. a_t, what a unit of the state before the piece would add to it:
//   y_t = yloc_t + sum_n w_t,n h_in,n        h_out = hloc + (a_1 .. a_TC) h_in
// so that each exponential is computed once and all that passes from piece to piece is h.  Eight lanes share two channels, the
// operands of the packed float instructions, and have NS states each.
//
// What bounds it: instructions.  1 x 4096 x 4096 with 16 states takes 193 us; the special-function unit, 16 a cycle and SM, would take
// 72 (58 for the exponentials of the decays, 14 for softplus and gate) and the bytes 21.  The schedulers issue in 65 % of the cycles,
// 30 instructions of a warp for each pair of exponentials: nine are the recurrence and what the state before the piece adds, the
// others make B and C float for each pair of channels, sum over lanes, and do step sizes, gates and copies.  512 CTAs, of which 296
// are resident at a time, end unevenly.
#include "sm100.cuh"
#include "tma_host.h"
#include "token_mixer.cuh"

namespace nova {
namespace {
using namespace mix;

constexpr int kCh = 8;           // channels of a CTA
constexpr int kMaxWarps = 8;     // of a CTA; named barrier i is the hand-over to warp i

struct ScanArgs {
  Seqs q;
  Rows u, delta, B, C, z, y;
  long long B_group, C_group;
  const float *A, *D, *bias;
  float* state;
  int channels, states, per_group, blocks_per_group, softplus;
  int vec_x, vec_bc, pair_y;     // copies of 16 bytes allowed for u, delta, z and for B, C; pairs of y stored at once
};

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// An infinite A (or A log2(e)) counts as float's number of that sign with the largest magnitude: the decay is 0 for any step from
// 2^-120 on, and for a step of 0, which tokens behind the end have too, it is 1 and no NaN.
__device__ __forceinline__ float finite(float A) {
  asm("min.NaN.f32 %0, %0, 0f7F7FFFFF;" : "+f"(A));
  asm("max.NaN.f32 %0, %0, 0fFF7FFFFF;" : "+f"(A));
  return A;
}

// Four neighbouring values in one access
__device__ __forceinline__ void load_quad(const float* p, float2 (&v)[2]) {
  const float4 w = *reinterpret_cast<const float4*>(p);
  v[0] = make_float2(w.x, w.y);
  v[1] = make_float2(w.z, w.w);
}
template <typename T>
__device__ __forceinline__ void load_quad(const T* p, float2 (&v)[2]) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  v[0] = load_pair(reinterpret_cast<const T*>(&w.x));
  v[1] = load_pair(reinterpret_cast<const T*>(&w.y));
}

// NS neighbouring values from pairs: whole words of shared memory
template <typename T, int NS>
__device__ __forceinline__ void load_states(const T* p, float (&v)[NS]) {
  if constexpr (NS == 2) {
    const float2 w = load_pair(p);
    v[0] = w.x;
    v[1] = w.y;
  } else {
#pragma unroll
    for (int j = 0; j < NS; j += 4) {
      float2 w[2];
      load_quad(p + j, w);
      v[j] = w[0].x; v[j + 1] = w[0].y; v[j + 2] = w[1].x; v[j + 3] = w[1].y;
    }
  }
}

// A behind the last state: not 0, so that its product with an infinite step is no NaN that a C of 0 would pass on to y
constexpr float kNoState = -1.17549435e-38f;

constexpr int TC = 8;            // tokens of a piece: one for each of the eight lanes that share two channels
// What a warp keeps in shared memory.  NS states a lane, 8 NS >= states.
template <typename T, int NS>
struct Piece {
  static constexpr int NP = 8 * NS;
  struct Stage { T u[TC][kCh], delta[TC][kCh], z[TC][kCh], B[TC][NP], C[TC][NP]; } stage[2];
  float4 step[TC][kCh / 2];               // dt of two channels, dt u of two channels
  float2 carry[NS][32];                   // h before this warp's piece, from the warp before
};

// COLS columns of TC rows, zeros behind the sequence's end and the tensor's columns: by copies of 16 bytes, or of 4 where an element
// has as many
template <typename T, int COLS>
__device__ __forceinline__ void fetch(T (*dst)[COLS], const char* src, long long row_bytes, int tokens, int cols, bool vec, int lane) {
  if (vec) {
    constexpr int PER = COLS * (int)sizeof(T) / 16;
#pragma unroll
    for (int i = lane; i < TC * PER; i += 32) {
      const int r = i / PER, c = i % PER * (16 / (int)sizeof(T));
      const bool there = r < tokens && c < cols;
      copy16(sm100::smem_u32(&dst[r][c]), there ? src + r * row_bytes + c * sizeof(T) : src, there);
    }
  } else if (sizeof(T) == 4) {
#pragma unroll 4
    for (int i = lane; i < TC * COLS; i += 32) {
      const int r = i / COLS, c = i % COLS;
      const bool there = r < tokens && c < cols;
      copy4(sm100::smem_u32(&dst[r][c]), there ? src + r * row_bytes + c * sizeof(T) : src, there);
    }
  }
}
// The same for elements of two bytes anywhere, through registers: all loads of a piece first, then the stores (store)
template <typename T, int COLS>
struct Elements {
  static constexpr int COUNT = TC * COLS / 32;
  T v[COUNT];
  __device__ __forceinline__ void load(const char* src, long long row_bytes, int tokens, int cols, int lane) {
#pragma unroll
    for (int k = 0; k < COUNT; ++k) {
      const int r = (32 * k + lane) / COLS, c = (32 * k + lane) % COLS;
      v[k] = r < tokens && c < cols ? reinterpret_cast<const T*>(src + r * row_bytes)[c] : from_float<T>(0.f);
    }
  }
  __device__ __forceinline__ void store(T (*dst)[COLS], int lane) const {
#pragma unroll
    for (int k = 0; k < COUNT; ++k) (&dst[0][0])[32 * k + lane] = v[k];
  }
};

// EXACT: 8 NS states, none to mask.  QUICK: those, of two bytes, and everything on boundaries of 16 bytes; a kernel of its own because
// the other copies cost this one registers (1 x 4096 x 4096: 193 us, 217 with both in one).
template <typename T, int NS, bool EXACT, bool QUICK, int RESIDENT>
__global__ void __launch_bounds__(32 * kMaxWarps, RESIDENT) scan_kernel(const __grid_constant__ ScanArgs a) {
  using P = Piece<T, NS>;
  constexpr int NP = P::NP;
  extern __shared__ __align__(16) unsigned char smem[];
  sm100::pdl_wait();
  sm100::pdl_launch_dependents();
  const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int q = lane & 7, pair = lane >> 3;
  const int per_seq = a.blocks_per_group * (a.channels / a.per_group);
  const int blk = blockIdx.x % per_seq, group = blk / a.blocks_per_group, in_group = (blk % a.blocks_per_group) * kCh;
  const Seq s = find_seq(a.q, blockIdx.x / per_seq, a.state != nullptr);
  if (s.skip) return;
  const int pieces = (s.len + TC - 1) / TC;
  if (warp >= pieces) return;
  P* mine = reinterpret_cast<P*>(smem) + warp;
  P* next = reinterpret_cast<P*>(smem) + (warp + 1 == warps ? 0 : warp + 1);
  const int d0 = group * a.per_group + in_group, cols = min(kCh, a.per_group - in_group), N = a.states;

  // QUICK: of u, delta and z a copy is a token, eight lanes each; the lower half of the warp copies B and the upper C.  What is added
  // per piece is a row count times a stride.
  static_assert(!QUICK || (EXACT && sizeof(T) == 2));
  const int c_of = lane >> 3;
  constexpr int PER_ROW = NS, PER_ROUND = 16 / PER_ROW;           // copies of a row of B or C, rows of a round
  auto lane_ptr = [&](const Rows& r, int token, long long col) { return reinterpret_cast<const char*>(row_ptr<const T>(r, s, token) + col); };
  const char *from_x = nullptr, *from_b = nullptr;
  if constexpr (QUICK) {
    from_x = c_of == 1 ? lane_ptr(a.delta, q, d0) : c_of == 2 && a.z.p ? lane_ptr(a.z, q, d0) : lane_ptr(a.u, q, d0);
    from_b = lane < 16 ? lane_ptr(a.B, lane / PER_ROW, group * a.B_group + lane % PER_ROW * 8)
                       : lane_ptr(a.C, (lane - 16) / PER_ROW, group * a.C_group + lane % PER_ROW * 8);
  }
  auto prefetch = [&](int piece, int slot) {
    const int t = piece * TC, tokens = s.len - t;
    typename P::Stage& st = mine->stage[slot];
    if constexpr (QUICK) {
      const uint32_t at = sm100::smem_u32(&st.u[0][0]);
      const long long rows = t * (long long)sizeof(T);
      if (c_of < (a.z.p ? 3 : 2)) {
        const bool in = q < tokens;
        copy16(at + 16 * lane, in ? from_x + rows * (c_of == 0 ? a.u.row : c_of == 1 ? a.delta.row : a.z.row) : from_x, in);
      }
      const uint32_t to = at + 3 * TC * kCh * 2 + (lane < 16 ? 0 : TC * NP * 2) + 16 * (lane & 15);
      const long long row = lane < 16 ? a.B.row : a.C.row;
#pragma unroll
      for (int r = 0; r < TC / PER_ROUND; ++r) {
        const bool in = (lane & 15) / PER_ROW + r * PER_ROUND < tokens;
        copy16(to + 256 * r, in ? from_b + (rows + r * PER_ROUND * 2) * row : from_b, in);
      }
      copy_commit();
    } else {
      auto from = [&](const Rows& r, long long col) { return reinterpret_cast<const char*>(row_ptr<const T>(r, s, t) + col); };
      const char *u = from(a.u, d0), *delta = from(a.delta, d0), *z = a.z.p ? from(a.z, d0) : nullptr;
      const char *B = from(a.B, group * a.B_group), *C = from(a.C, group * a.C_group);
      constexpr long long E = sizeof(T);
      if (E == 4 || a.vec_x) {
        fetch<T, kCh>(st.u, u, a.u.row * E, tokens, cols, a.vec_x, lane);
        fetch<T, kCh>(st.delta, delta, a.delta.row * E, tokens, cols, a.vec_x, lane);
        if (z) fetch<T, kCh>(st.z, z, a.z.row * E, tokens, cols, a.vec_x, lane);
      }
      if (E == 4 || a.vec_bc) {
        fetch<T, NP>(st.B, B, a.B.row * E, tokens, N, a.vec_bc, lane);
        fetch<T, NP>(st.C, C, a.C.row * E, tokens, N, a.vec_bc, lane);
      }
      if constexpr (E == 2) {
        Elements<T, kCh> x[3];
        Elements<T, NP> bc[2];
        if (!a.vec_x) {
          x[0].load(u, a.u.row * E, tokens, cols, lane);
          x[1].load(delta, a.delta.row * E, tokens, cols, lane);
          if (z) x[2].load(z, a.z.row * E, tokens, cols, lane);
        }
        if (!a.vec_bc) {
          bc[0].load(B, a.B.row * E, tokens, N, lane);
          bc[1].load(C, a.C.row * E, tokens, N, lane);
        }
        if (!a.vec_x) {
          x[0].store(st.u, lane);
          x[1].store(st.delta, lane);
          if (z) x[2].store(st.z, lane);
        }
        if (!a.vec_bc) {
          bc[0].store(st.B, lane);
          bc[1].store(st.C, lane);
        }
      }
      copy_commit();
    }
  };
  prefetch(warp, 0);

  const int ch = 2 * pair;                              // this lane's channels of the block: ch, ch + 1
  const bool has0 = ch < cols, has1 = ch + 1 < cols;
  float2 A[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int n = q * NS + j;
    A[j].x = has0 && n < N ? finite(a.A[(size_t)(d0 + ch) * N + n] * kLog2e) : kNoState;
    A[j].y = has1 && n < N ? finite(a.A[(size_t)(d0 + ch + 1) * N + n] * kLog2e) : kNoState;
  }
  const float2 bias = make_float2(a.bias && has0 ? a.bias[d0 + ch] : 0.f, a.bias && has1 ? a.bias[d0 + ch + 1] : 0.f);
  const float2 skip = make_float2(a.D && has0 ? a.D[d0 + ch] : 0.f, a.D && has1 ? a.D[d0 + ch + 1] : 0.f);
  float* state = a.state ? a.state + ((size_t)s.slot * a.channels + d0 + ch) * N + q * NS : nullptr;

  int slot = 0;
  for (int piece = warp; piece < pieces; piece += warps, slot ^= 1) {
    const int tokens = s.len - piece * TC;
    if (piece + warps < pieces) {
      prefetch(piece + warps, slot ^ 1);
      copy_wait<1>();
    } else {
      copy_wait<0>();
    }
    __syncwarp();
    typename P::Stage& st = mine->stage[slot];
    // the step sizes, a token of its pair of channels each lane
    {
      const float2 u = load_pair(&st.u[q][ch]), dl = load_pair(&st.delta[q][ch]);
      float2 dt = make_float2(dl.x + bias.x, dl.y + bias.y);
      if (a.softplus) dt = softplus(dt);
      if (q >= tokens) dt = make_float2(0.f, 0.f);
      mine->step[q][pair] = make_float4(dt.x, dt.y, dt.x * u.x, dt.y * u.y);
    }
    __syncwarp();
    float2 h[NS], decay[NS], y[TC], w[TC][NS];
#pragma unroll
    for (int t = 0; t < TC; ++t) {
      const float4 step = mine->step[t][pair];
      const float2 dt = make_float2(step.x, step.y), du = make_float2(step.z, step.w);
      // B and C as they came, made float here: what comes back from shared memory, 128 bytes a cycle, would bound this loop
      float B[NS], C[NS];
      load_states(&st.B[t][q * NS], B);
      load_states(&st.C[t][q * NS], C);
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        const float2 arg = mul2(dt, A[j]), e = make_float2(ex2(arg.x), ex2(arg.y));
        float2 b = mul2(du, both(B[j]));
        if (!EXACT && q * NS + j >= N) b = both(0.f);          // an infinite dt u times a zero behind the last state
        h[j] = t ? fma2(e, h[j], b) : b;
        y[t] = j ? fma2(both(C[j]), h[j], y[t]) : mul2(both(C[j]), h[j]);
        decay[j] = t ? mul2(decay[j], e) : e;
        w[t][j] = mul2(both(C[j]), decay[j]);
      }
    }
    // the state before this piece
    float2 in[NS];
    if (piece == 0) {
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        const bool there = s.resume && q * NS + j < N;
        in[j] = make_float2(there && has0 ? state[j] : 0.f, there && has1 ? state[N + j] : 0.f);
      }
    } else {
      __syncwarp();
      asm volatile("bar.sync %0, 64;" ::"r"(warp) : "memory");
#pragma unroll
      for (int j = 0; j < NS; ++j) in[j] = mine->carry[j][lane];
    }
    // nothing to add to a start from zeros, and nothing times a product of decays that has left the range
    const bool from_state = piece > 0 || s.resume;
    if (from_state) {
#pragma unroll
      for (int j = 0; j < NS; ++j) h[j] = fma2(decay[j], in[j], h[j]);
    }
    if (piece + 1 < pieces) {
#pragma unroll
      for (int j = 0; j < NS; ++j) next->carry[j][lane] = h[j];
      __threadfence_block();
      __syncwarp();
      asm volatile("bar.arrive %0, 64;" ::"r"(warp + 1 == warps ? 0 : warp + 1) : "memory");
    } else if (state) {
#pragma unroll
      for (int j = 0; j < NS; ++j)
        if (q * NS + j < N) {
          if (has0) state[j] = h[j].x;
          if (has1) state[N + j] = h[j].y;
        }
    }
    if (from_state) {
#pragma unroll
      for (int t = 0; t < TC; ++t)
#pragma unroll
        for (int j = 0; j < NS; ++j) y[t] = fma2(w[t][j], in[j], y[t]);
    }
    // sums over the eight lanes of a channel pair: each exchange halves the tokens of a lane, and token q stays
    auto exchange = [&](float2 keep, float2 give, int m) {
      return __fadd2_rn(keep, make_float2(__shfl_xor_sync(0xffffffffu, give.x, m), __shfl_xor_sync(0xffffffffu, give.y, m)));
    };
#pragma unroll
    for (int m = 4; m; m >>= 1)
#pragma unroll
      for (int t = 0; t < m; ++t) y[t] = exchange(q & m ? y[t + m] : y[t], q & m ? y[t] : y[t + m], m);
    if (q < tokens && has0) {
      float2 v = y[0];
      if (a.D) v = fma2(skip, load_pair(&st.u[q][ch]), v);
      if (a.z.p) v = mul2(v, silu(load_pair(&st.z[q][ch])));
      T* out = row_ptr<T>(a.y, s, piece * TC + q) + d0 + ch;
      if (a.pair_y && has1) store_pair(out, v);
      else {
        out[0] = from_float<T>(v.x);
        if (has1) out[1] = from_float<T>(v.y);
      }
    }
    __syncwarp();                                       // the stage is overwritten by the copies of the next turn
  }
}

template <typename T, int NS, bool EXACT, bool QUICK, int RESIDENT>
int start_pieces(const ScanArgs& a, cudaStream_t s) {
  constexpr int kMost = sizeof(Piece<T, NS>) * kMaxWarps;
  auto kernel = scan_kernel<T, NS, EXACT, QUICK, RESIDENT>;
  if (int e = (int)allow_dynamic_smem<kMost>(kernel)) return e;
  // as many warps as an average sequence has pieces, two at least: a piece is handed to another warp.  The lengths of packed sequences
  // are on the device; a long one among many short ones has as few warps as they have.
  const long long longest = a.q.cu ? (a.q.tokens + a.q.count - 1) / a.q.count : a.q.tokens, pieces = (longest + TC - 1) / TC;
  const int warps = pieces > kMaxWarps ? kMaxWarps : pieces < 2 ? 2 : (int)pieces;
  const int per_seq = a.blocks_per_group * (a.channels / a.per_group);
  return (int)launch_overlapped(kernel, per_seq * a.q.count, 32 * warps, sizeof(Piece<T, NS>) * warps, s, a);
}
template <typename T, int NS, bool EXACT, bool QUICK>
int start_pieces(const ScanArgs& a, cudaStream_t s) {
  // Up to 16 states: two CTAs on an SM with 128 registers a thread, or one with all of them where there are no more CTAs than SMs
  // (one / two: 3 x 701 x 354 float, 138 CTAs, 16.2 / 17.6 us; 1 x 1000 x 1024 bf16, 128 CTAs, 17.7 / 19.5; 192 CTAs
  // 33.5 / 28.6, 512 238 / 206).
  if constexpr (NS == 2)
    if ((long long)a.blocks_per_group * (a.channels / a.per_group) * a.q.count > 148) return start_pieces<T, NS, EXACT, QUICK, 2>(a, s);
  return start_pieces<T, NS, EXACT, QUICK, 1>(a, s);
}
template <typename T, int NS>
int start_pieces(const ScanArgs& a, cudaStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (a.states == 8 * NS && a.vec_x && a.vec_bc) return start_pieces<T, NS, true, true>(a, s);
  } else {
    if (a.states == 8 * NS) return start_pieces<T, NS, true, false>(a, s);
  }
  return start_pieces<T, NS, false, false>(a, s);
}

// One token for each sequence: the state is read and written once, 8 N bytes a channel, and that is what bounds it (128 sequences x
// 4096 channels x 16 states 18.8 us, 3.8 TB/s; four sequences of one channel a thread instead 30.5; one of one 37.8).  Four lanes
// share a channel, four states each at a time (16 bytes).  A thread has R channels of one sequence, a CTA's width apart, so that
// R loads of states are under way and B and C are read and made float once for them; with R = 4 each lane of the four makes the step
// size and the output of one of the four channels, and hands the former to the others.  64 registers, so that four CTAs are resident,
// cost R = 4 some 24 to 48 bytes of spills.
// R = 4 from kManySteps sequences x channels on: 4 x 4096 of 16 states 2.65 us with R = 1 and 2.97 with R = 4, 8 x 4096 3.6 and 3.05,
// 16 x 2048 of 64 states 6.7 and 7.9, 32 x 2048 11.5 and 10.8.
constexpr long long kManySteps = 1 << 15;
constexpr int kStepThreads = 256, kStepWidth = kStepThreads / 4;
template <typename T, int R, bool WHOLE>
__global__ void __launch_bounds__(kStepThreads, 4) step_kernel(const __grid_constant__ ScanArgs a) {
  static_assert(R == 1 || R == 4, "a lane for each channel, or one channel");
  sm100::pdl_wait();
  sm100::pdl_launch_dependents();
  const int q = threadIdx.x & 3, d0 = blockIdx.y * (kStepWidth * R) + threadIdx.x / 4, N = a.states;
  const Seq s = find_seq(a.q, blockIdx.x, a.state != nullptr);
  if (s.skip) return;                                         // the whole CTA
  const int d = d0 + (R == 4 ? q * kStepWidth : 0);           // this lane's own channel of the R
  const bool there = d < a.channels;
  float u = 0.f, dt = 0.f, z = 0.f;
  if (there) {
    u = to_float(row_ptr<const T>(a.u, s, 0)[d]);
    dt = to_float(row_ptr<const T>(a.delta, s, 0)[d]) + (a.bias ? a.bias[d] : 0.f);
    if (a.z.p) z = to_float(row_ptr<const T>(a.z, s, 0)[d]);
  }
  float* state = a.state ? a.state + ((size_t)s.slot * a.channels + d0) * N + 4 * q : nullptr;
  const float* A = a.A + (size_t)d0 * N + 4 * q;
  const size_t apart = (size_t)kStepWidth * N;                // between the states of a thread's channels
  const long long group = R == 1 ? min(d0, a.channels - 1) / a.per_group : 0;
  const T* Bp = row_ptr<const T>(a.B, s, 0) + group * a.B_group + 4 * q;
  const T* Cp = row_ptr<const T>(a.C, s, 0) + group * a.C_group + 4 * q;
  float y[R];
#pragma unroll
  for (int r = 0; r < R; ++r) y[r] = 0.f;
  for (int n0 = 0; n0 < N; n0 += 16, Bp += 16, Cp += 16, A += 16) {
    const int here = min(max(N - n0 - 4 * q, 0), 4);
    auto take = [&](float (&v)[4], const float* p, bool in) {
      if (WHOLE) {
        const float4 w = in && here == 4 ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = in && j < here ? p[j] : 0.f;
      }
    };
    float h[R][4], Ar[R][4], B[4], C[4];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool in = d0 + r * kStepWidth < a.channels;
      take(h[r], state + r * apart + n0, in && state && s.resume);
      take(Ar[r], A + r * apart, in);
    }
    if (a.vec_bc && here == 4) {
      const float2 b0 = load_pair(Bp), b1 = load_pair(Bp + 2), c0 = load_pair(Cp), c1 = load_pair(Cp + 2);
      B[0] = b0.x; B[1] = b0.y; B[2] = b1.x; B[3] = b1.y;
      C[0] = c0.x; C[1] = c0.y; C[2] = c1.x; C[3] = c1.y;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        B[j] = j < here ? to_float(Bp[j]) : 0.f;
        C[j] = j < here ? to_float(Cp[j]) : 0.f;
      }
    }
    if (n0 == 0 && a.softplus) dt = softplus(make_float2(dt, dt)).x;             // while the states are under way
    const float du = dt * u;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float dtr = (R == 4 ? __shfl_sync(0xffffffffu, dt, (threadIdx.x & 28) | r) : dt) * kLog2e;
      const float dur = R == 4 ? __shfl_sync(0xffffffffu, du, (threadIdx.x & 28) | r) : du;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!WHOLE && j >= here) continue;                     // an infinite dt u times a zero behind the last state
        h[r][j] = fmaf(ex2(dtr * finite(Ar[r][j])), h[r][j], dur * B[j]);
        if (WHOLE && here == 0) continue;
        y[r] = fmaf(C[j], h[r][j], y[r]);
      }
      if (!state || d0 + r * kStepWidth >= a.channels || here == 0) continue;
      float* to = state + r * apart + n0;
      if (WHOLE) *reinterpret_cast<float4*>(to) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
      else
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < here) to[j] = h[r][j];
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    y[r] += __shfl_xor_sync(0xffffffffu, y[r], 1);
    y[r] += __shfl_xor_sync(0xffffffffu, y[r], 2);
  }
  if (!there || (R == 1 && q != 0)) return;
  float v = y[0];
#pragma unroll
  for (int r = 1; r < R; ++r)
    if (q == r) v = y[r];
  if (a.D) v = fmaf(a.D[d], u, v);
  if (a.z.p) v *= silu(make_float2(z, z)).x;
  row_ptr<T>(a.y, s, 0)[d] = from_float<T>(v);
}

template <typename T, int R, bool WHOLE>
int start_step(const ScanArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.q.count, (a.channels + kStepWidth * R - 1) / (kStepWidth * R));
  cfg.blockDim = dim3(kStepThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return (int)cudaLaunchKernelEx(&cfg, step_kernel<T, R, WHOLE>, a);
}
template <typename T>
int start_step(const ScanArgs& a, cudaStream_t s) {
  const bool whole = a.states % 4 == 0 && aligned(a.A, 16) && aligned(a.state, 16);
  // four channels a thread where there are many, and where B and C are the same for all of them (in two groups 128 x 4096 take
  // 37.7 us with one)
  const bool many = a.per_group == a.channels && (long long)a.q.count * a.channels >= kManySteps;
  if (whole) return many ? start_step<T, 4, true>(a, s) : start_step<T, 1, true>(a, s);
  return many ? start_step<T, 4, false>(a, s) : start_step<T, 1, false>(a, s);
}

template <typename T>
int start(const ScanArgs& a, cudaStream_t s) {
  // the blocks of channels are the step kernel's second grid dimension
  if (!a.q.cu && a.q.tokens == 1 && a.channels <= 65535 * kStepWidth) return start_step<T>(a, s);
  return a.states <= 16 ? start_pieces<T, 2>(a, s) : a.states <= 32 ? start_pieces<T, 4>(a, s) : start_pieces<T, 8>(a, s);
}

}  // namespace
}  // namespace nova

extern "C" int nova_selective_scan(const nova_sequences* q, int type, const nova_scan* c, nova_stream stream) {
  using namespace nova;
  using namespace nova::mix;
  if (!c || !type_ok(type) || !seqs_ok(q, c->state_dev != nullptr) || c->channels <= 0 || c->states < 1 || c->states > 64 ||
      c->groups < 1 || c->channels % c->groups || c->B_group < 0 || c->C_group < 0 || (c->flags & ~NOVA_SOFTPLUS))
    return NOVA_ERR_INVALID_ARG;
  if (q->sequences == 0 || q->tokens == 0) return NOVA_OK;
  for (const nova_rows* r : {&c->u, &c->delta, &c->B, &c->C, &c->y})
    if (!rows_ok(*r, type)) return NOVA_ERR_INVALID_ARG;
  if (c->z.data_dev && !rows_ok(c->z, type)) return NOVA_ERR_INVALID_ARG;
  for (const nova_rows* r : {&c->u, &c->delta, &c->B, &c->C, &c->z})
    if (r->data_dev == c->y.data_dev) return NOVA_ERR_INVALID_ARG;
  if (!c->A_dev || !aligned(c->A_dev, 4) || !aligned(c->D_dev, 4) || !aligned(c->delta_bias_dev, 4) || !aligned(c->state_dev, 4))
    return NOVA_ERR_INVALID_ARG;
  const int per_group = c->channels / c->groups, blocks = (per_group + kCh - 1) / kCh;
  if ((long long)blocks * c->groups * q->sequences > INT32_MAX) return NOVA_ERR_INVALID_ARG;
  ScanArgs a = {make_seqs(q), make_rows(c->u), make_rows(c->delta), make_rows(c->B), make_rows(c->C), make_rows(c->z),
                make_rows(c->y), (long long)c->B_group, (long long)c->C_group, c->A_dev, c->D_dev, c->delta_bias_dev,
                c->state_dev, c->channels, c->states, per_group, blocks, c->flags & NOVA_SOFTPLUS, 0, 0, 0};
  const size_t e = type_bytes(type);
  a.vec_x = per_group * e % 16 == 0 && rows_aligned(a.u, e, 16) && rows_aligned(a.delta, e, 16) && rows_aligned(a.z, e, 16);
  a.vec_bc = c->states * e % 16 == 0 && rows_aligned(a.B, e, 16) && rows_aligned(a.C, e, 16) && a.B_group * e % 16 == 0 && a.C_group * e % 16 == 0;
  a.pair_y = per_group % 2 == 0 && rows_aligned(a.y, e, 2 * e);
  cudaStream_t s = (cudaStream_t)stream;
  return launch_status(type == NOVA_F32 ? start<float>(a, s) : type == NOVA_F16 ? start<__half>(a, s) : start<__nv_bfloat16>(a, s));
}
