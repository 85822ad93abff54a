// A few rows times a matrix of 4-bit weights with group scales (nova_linear_int4).
//
// What has to move: the codes, N K / 2 bytes read once.  The products run on the tensor cores, by mma.sync m16n8k16, whose operand
// comes out of registers, where the codes become numbers: 16 outputs are its rows, eight rows of x its columns.  The sum over a
// group is multiplied by the group's scale in float, so that no weight is rounded.  The order of k is free in such a sum: the four
// lanes of a row take neighbouring words, eight codes each, and the elements of x that go with them.
//
// What bounds it: not the bytes but the way from codes to products (five to seven integer instructions for eight codes, at half the
// issue rate, and four to take off the zero), x from shared memory, and what a CTA does before its first product.  1 x 4096 x 4096
// half 6.4 us (floor 1.4), 1 x 14336 x 8192 half 20.9 (9.5), 16 x 14336 x 8192 bf16 in groups of 64 35.5 us (10): 2.9 and 1.8 TB/s.
#include <cooperative_groups.h>

#include <type_traits>

#include "sm100.cuh"
#include "tma_host.h"
#include "token_mixer.cuh"

namespace nova {
namespace {
using namespace mix;

constexpr int kMaxWarps = 8;
// CTAs at once: two on an SM, less what clusters of eight leave over.  One wave of them, each with as many tiles as it takes: several
// waves of one tile each took 60 us where this took 41.  With many rows of a long k a CTA's shared memory passes half of an SM's (16 rows
// of k = 11008 in groups of 32, 14336 outputs: 122 KB): one CTA an SM, and two waves.
constexpr int kCtas = 264;

struct Int4Args {
  const void *x, *scales, *bias;
  const unsigned char *codes, *zeros;
  void* y;
  long long x_row, y_row;
  int M, N, K, x_vec, k_range, k_part, wk, tiles, table_vec;
};

// c = a b + (first ? 0 : c)
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool first) {
  const float z0 = first ? 0.f : c[0], z1 = first ? 0.f : c[1], z2 = first ? 0.f : c[2], z3 = first ? 0.f : c[3];
  if constexpr (std::is_same_v<T, __half>)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(z0), "f"(z1), "f"(z2), "f"(z3));
}

// The eight codes of a word, less their zero, as numbers of the type; pair p holds codes p and p + 4.  All exact, so that a code
// equal to its zero adds nothing.
// half: the bits of a code, as they are, are a subnormal number, q 2^-24, and those of its neighbour, four bits up, 16 q 2^-24,
// which a multiply-add takes to the first's unit.  bfloat16, whose subnormals are beyond float's range once multiplied: the bits are
// the lowest of the mantissa of 128, 128 + q, and 128 + zero is taken off.
template <typename T> struct Codes;
template <> struct Codes<__half> {
  static constexpr uint32_t BASE = 0;
  static constexpr float UNIT = 16777216.f;                     // codes in units of the numbers
  using Pair = __half2;
  __device__ __forceinline__ static Pair pair(uint32_t bits) { return *reinterpret_cast<const Pair*>(&bits); }
  __device__ __forceinline__ static void numbers(uint32_t w, uint32_t, Pair zero, Pair (&out)[4]) {
    const Pair sixteenth = __float2half2_rn(1.f / 16), less = __hneg2(zero);
    out[0] = __hsub2(pair(w & 0x000f000fu), zero);
    out[1] = __hfma2(pair(w & 0x00f000f0u), sixteenth, less);
    out[2] = __hsub2(pair((w >> 8) & 0x000f000fu), zero);
    out[3] = __hfma2(pair((w >> 8) & 0x00f000f0u), sixteenth, less);
  }
};
template <> struct Codes<__nv_bfloat16> {
  static constexpr uint32_t BASE = 0x43004300u;
  static constexpr float UNIT = 1.f;
  using Pair = __nv_bfloat162;
  __device__ __forceinline__ static Pair pair(uint32_t bits) { return *reinterpret_cast<const Pair*>(&bits); }
  __device__ __forceinline__ static void numbers(uint32_t w, uint32_t base, Pair zero, Pair (&out)[4]) {
#pragma unroll
    for (int p = 0; p < 4; ++p) out[p] = __hsub2(pair(((w >> 4 * p) & 0x000f000fu) | base), zero);
  }
};

constexpr int kChunk = 128;                       // k of a warp's step: four words of eight codes a lane and row
constexpr int kMaxSplit = 8;                      // CTAs of a cluster, which share k
constexpr int kMostSmem = 227 * 1024;

// Shared memory: x of the CTA's k as the operand wants it, rows 64 bytes apart modulo the 128 of the banks; for each warp scale and
// zero of its 16 outputs and groups, rows two banks apart; the sums of the products.
struct Layout {
  int x_row, table, table_row, part, bytes;             // in bytes
  __host__ __device__ Layout(int warps, int M, int k_range, int k_part, int part_floats, int log_group) {
    x_row = (2 * k_range + 127) / 128 * 128 + 64;
    table = M * x_row;
    table_row = (((k_part >> log_group) + 15) / 16 * 16 + 1) * 8;
    part = table + warps * 16 * table_row;
    bytes = part + part_floats * 4;
  }
};

// The sums run over the four lanes of a row, so that every group has to be spread over all four.  Of a group of 128 a lane's share is
// 16 bytes, of one of 64 it is 8.  Of one of 32 it would be 4: there a lane loads 16 bytes too, a whole group, and the four lanes
// transpose their words (1 x 14336 x 8192 when the zero was taken off after the sum: 30.7 us, 36.8 with loads of 4; the same for groups
// of 64, 16 rows, 41.8 against 40.6).
__device__ __forceinline__ void transpose(uint32_t (&w)[4], int q) {
  auto swap = [](bool upper, uint32_t& low, uint32_t& high, int m) {           // the lower lane's high with the upper lane's low
    const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? low : high, m);
    low = upper ? got : low;
    high = upper ? high : got;
  };
  swap((q & 1) != 0, w[0], w[1], 1);
  swap((q & 1) != 0, w[2], w[3], 1);
  swap((q & 2) != 0, w[0], w[2], 2);
  swap((q & 2) != 0, w[1], w[3], 2);
}

// The CTAs of a cluster share k and have the same outputs, `tiles` of 16.  x of a CTA's k is laid out once; then its warps go
// through (tile, part of k) by themselves: codes from memory to registers DEPTH steps ahead, across the ends of tiles.  The sums of
// all parts are added up at the end, through each other's shared memory.
template <typename T, int TILES, int LOG_GROUP>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) linear_kernel(const __grid_constant__ Int4Args a) {
  constexpr int WORDS = 1 << (LOG_GROUP - 5), HELD = kChunk >> LOG_GROUP, DEPTH = 4;      // words of a lane in a group, groups of a step
  extern __shared__ __align__(128) unsigned char smem[];
  const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane >> 2, q = lane & 3;
  const int in_k = warp % a.wk, stride = warps / a.wk;                // this warp's part of k; tiles between its items
  const int k_first = blockIdx.x * a.k_range, k_count = min(a.k_range, a.K - k_first);
  const int t_first = blockIdx.y * a.tiles, t_count = min(a.tiles, (a.N + 15) / 16 - t_first), width = 16 * a.tiles;
  const int my_k = in_k * a.k_part, my_count = max(min(a.k_part, k_count - my_k), 0), steps = (my_count + kChunk - 1) / kChunk;
  const Layout at(warps, a.M, a.k_range, a.k_part, a.wk * a.M * width, LOG_GROUP);
  sm100::pdl_wait();
  sm100::pdl_launch_dependents();

  // What is fetched next: a tile and a step of it.  Rows behind the last output are read as the last one: what comes of them is not
  // stored.
  const unsigned char* from[2];
  int next_tile = warp / a.wk, next_step = 0;
  auto aim = [&] {
#pragma unroll
    for (int r = 0; r < 2; ++r)
      from[r] = a.codes + (size_t)min((t_first + next_tile) * 16 + g + 8 * r, a.N - 1) * (a.K / 2) + (k_first + my_k) / 2 + (WORDS == 2 ? 8 : 16) * q;
  };
  // Behind the last k zeros, which x is there too.
  auto fetch = [&](uint32_t (&w)[2][4]) {
    if (next_tile >= t_count) return;
    const int left = my_count - next_step * kChunk;                             // k from here on
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if constexpr (WORDS == 2) {
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
          const uint2 v = h << LOG_GROUP < left ? __ldg(reinterpret_cast<const uint2*>(from[r] + (h << LOG_GROUP) / 2)) : make_uint2(0, 0);
          w[r][2 * h] = v.x; w[r][2 * h + 1] = v.y;
        }
      } else {
        const uint4 v = 32 * q < left ? __ldcs(reinterpret_cast<const uint4*>(from[r])) : make_uint4(0, 0, 0, 0);
        w[r][0] = v.x; w[r][1] = v.y; w[r][2] = v.z; w[r][3] = v.w;
      }
    }
    from[0] += kChunk / 2;
    from[1] += kChunk / 2;
    if (++next_step == steps) {
      next_step = 0;
      next_tile += stride;
      aim();
    }
  };
  // BASE, but not as a constant: an instruction takes one, and the mask of the codes is one already (M > 0; 1 x 14336 x 8192 bfloat16
  // 21.9 us, 25.9 with two)
  const uint32_t base = Codes<T>::BASE | (uint32_t)(a.M >> 31);
  uint32_t held[DEPTH][2][4];
  if (steps > 0) {
    aim();
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(held[d]);
  }

  // x as pairs (0, 4), (1, 5), (2, 6), (3, 7) of eight elements, in the order of the products: pairs 0 and 2, then 1 and 3.  Piece
  // WORDS q + i of a group goes with word i of lane q and stands where the four lanes of word i find theirs side by side.
  constexpr int PIECES = 1 << (LOG_GROUP - 3), BATCH = 4;
  const int per_row = (k_count + kChunk - 1) / kChunk * (kChunk / 8);          // a multiple of 16: no group is cut
  for (int i0 = warp * 32; i0 < a.M * per_row; i0 += BATCH * blockDim.x) {
    uint32_t v[BATCH][4];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int i = i0 + j * blockDim.x + lane, m = i / per_row, k = 8 * (i - m * per_row);
      v[j][0] = v[j][1] = v[j][2] = v[j][3] = 0;
      if (m < a.M && k < k_count) {
        const T* src = (const T*)a.x + m * a.x_row + k_first + k;
        if (a.x_vec) {
          const uint4 w = *reinterpret_cast<const uint4*>(src);
          v[j][0] = w.x; v[j][1] = w.y; v[j][2] = w.z; v[j][3] = w.w;
        } else {
          const unsigned short* s = reinterpret_cast<const unsigned short*>(src);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[j][e] = s[2 * e] | (uint32_t)s[2 * e + 1] << 16;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      if (i0 + j * (int)blockDim.x >= a.M * per_row) break;
      const int i = i0 + j * blockDim.x + lane, m = i / per_row, piece = i - m * per_row;
      if (m >= a.M) continue;
      const int in_group = piece % PIECES, place = piece - in_group + in_group % WORDS * 4 + in_group / WORDS;
      *reinterpret_cast<uint4*>(smem + m * at.x_row + 16 * place) =
          make_uint4(__byte_perm(v[j][0], v[j][2], 0x5410), __byte_perm(v[j][1], v[j][3], 0x5410), __byte_perm(v[j][0], v[j][2], 0x7632),
                     __byte_perm(v[j][1], v[j][3], 0x7632));
    }
  }
  __syncthreads();

  float2* table = reinterpret_cast<float2*>(smem + at.table + warp * 16 * at.table_row);
  float* part = reinterpret_cast<float*>(smem + at.part) + in_k * a.M * width;               // [m][output of the cluster]
  const int table_row = at.table_row / 8, groups = my_count >> LOG_GROUP, all_groups = a.K >> LOG_GROUP;
  const T* scales = (const T*)a.scales + ((k_first + my_k) >> LOG_GROUP);
  const unsigned char* zeros = a.zeros + ((k_first + my_k) >> LOG_GROUP);
  auto entry = [](float scale, uint32_t zero) { return make_float2(scale * Codes<T>::UNIT, __uint_as_float(Codes<T>::BASE | zero * 0x10001u)); };
  const unsigned char* x_of_lane[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t)              // rows of x behind the last are read as that one: what comes of them is not stored
    x_of_lane[t] = smem + min(8 * t + g, a.M - 1) * at.x_row + 2 * my_k + 16 * q;
  for (int tile = warp / a.wk; tile < t_count; tile += stride) {
    // the scale as float, what the sums are multiplied by, and the zero as it is taken off a pair of codes
    __syncwarp();
    if (a.table_vec) {                                        // eight groups at once
      const int per_row = groups >> 3;
#pragma unroll 2
      for (int i = lane; i < 16 * per_row; i += 32) {
        const int r = i / per_row, h = 8 * (i - r * per_row);
        const size_t n = (size_t)min((t_first + tile) * 16 + r, a.N - 1) * all_groups + h;
        float2* dst = table + r * table_row + h;
        const uint4 s = *reinterpret_cast<const uint4*>(scales + n);
        const uint2 z = a.zeros ? *reinterpret_cast<const uint2*>(zeros + n) : make_uint2(0x08080808u, 0x08080808u);
        const uint32_t sw[4] = {s.x, s.y, s.z, s.w}, zw[2] = {z.x, z.y};
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float2 f = load_pair(reinterpret_cast<const T*>(&sw[e / 2]));
          dst[e] = entry(f.x, zw[e / 4] >> 8 * (e & 3) & 15);
          dst[e + 1] = entry(f.y, zw[e / 4] >> 8 * (e & 3) + 8 & 15);
        }
      }
    } else {
#pragma unroll 4
      for (int i = lane; i < 16 * groups; i += 32) {
        const int r = i / groups, h = i - r * groups;
        const size_t n = (size_t)min((t_first + tile) * 16 + r, a.N - 1) * all_groups + h;
        table[r * table_row + h] = entry(to_float(scales[n]), a.zeros ? zeros[n] & 15u : 8u);
      }
    }
    __syncwarp();
    float sum[TILES][4];
#pragma unroll
    for (int i = 0; i < TILES * 4; ++i) (&sum[0][0])[i] = 0.f;
    const float2* my_table = table + g * table_row;
    const unsigned char* xs[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) xs[t] = x_of_lane[t];
    auto bits = [](const auto& pair) { return *reinterpret_cast<const uint32_t*>(&pair); };
    auto products = [&](const uint32_t (&held)[2][4], int step) {
      uint32_t words[2][4];
#pragma unroll
      for (int r = 0; r < 8; ++r) words[r / 4][r % 4] = held[r / 4][r % 4];
      if constexpr (WORDS == 1) {
        transpose(words[0], q);
        transpose(words[1], q);
      }
      const int left = (my_count - step * kChunk) >> LOG_GROUP;        // groups from here on
#pragma unroll
      for (int h = 0; h < HELD; ++h) {
        if (h >= left) break;
        const float2 entry0 = my_table[h], entry1 = my_table[8 * table_row + h];
        const auto zero0 = Codes<T>::pair(__float_as_uint(entry0.y)), zero1 = Codes<T>::pair(__float_as_uint(entry1.y));
        float c[TILES][4];
#pragma unroll
        for (int u = 0; u < WORDS; ++u) {
          typename Codes<T>::Pair r0[4], r1[4];
          Codes<T>::numbers(words[0][h * WORDS + u], base, zero0, r0);
          Codes<T>::numbers(words[1][h * WORDS + u], base, zero1, r1);
          const uint32_t f0[4] = {bits(r0[0]), bits(r1[0]), bits(r0[2]), bits(r1[2])}, f1[4] = {bits(r0[1]), bits(r1[1]), bits(r0[3]), bits(r1[3])};
#pragma unroll
          for (int t = 0; t < TILES; ++t) {
            const uint4 x = *reinterpret_cast<const uint4*>(xs[t] + 64 * (h * WORDS + u));
            mma<T>(c[t], f0, x.x, x.y, u == 0);
            mma<T>(c[t], f1, x.z, x.w, false);
          }
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[t][e] = fmaf(e < 2 ? entry0.x : entry1.x, c[t][e], sum[t][e]);
      }
#pragma unroll
      for (int t = 0; t < TILES; ++t) xs[t] += 2 * kChunk;
      my_table += HELD;
    };
    // DEPTH steps at a time; the steps of a tile are a multiple of that but for its last turn, after which what is held moves up
    for (int step = 0; step < steps; step += DEPTH) {
      if (step + DEPTH <= steps) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
          products(held[d], step + d);
          fetch(held[d]);
        }
      } else {
        const int over = steps - step;
#pragma unroll
        for (int d = 0; d < DEPTH - 1; ++d)
          if (d < over) products(held[d], step + d);
        for (int d = 0; d < over; ++d) {
#pragma unroll
          for (int e = 0; e < DEPTH - 1; ++e)
#pragma unroll
            for (int r = 0; r < 8; ++r) (&held[e][0][0])[r] = (&held[e + 1][0][0])[r];
          fetch(held[DEPTH - 1]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = 8 * t + 2 * q + (e & 1);
        if (m < a.M) part[m * width + tile * 16 + g + 8 * (e >> 1)] = sum[t][e];
      }
  }
  cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
  const int ranks = gridDim.x, rank = blockIdx.x, in_use = 16 * t_count;             // a cluster is a row of the grid
  if (ranks > 1) cluster.sync();
  else __syncthreads();
  float* all = reinterpret_cast<float*>(smem + at.part);
  for (int v = threadIdx.x + rank * blockDim.x; v < in_use * a.M; v += blockDim.x * ranks) {
    const int m = v / in_use, col = v - m * in_use, n = t_first * 16 + col;
    if (n >= a.N) continue;
    float s = 0.f;
    for (int r = 0; r < ranks; ++r) {
      const float* p = (ranks > 1 ? cluster.map_shared_rank(all, r) : all) + m * width + col;
      for (int w = 0; w < a.wk; ++w) s += p[w * a.M * width];
    }
    if (a.bias) s += to_float(((const T*)a.bias)[n]);
    ((T*)a.y)[m * a.y_row + n] = from_float<T>(s);
  }
  if (ranks > 1) cluster.sync();                             // no CTA leaves while another reads its sums
}

template <typename T, int LOG_GROUP>
int start(const Int4Args& a, cudaStream_t s);
template <typename T, int TILES, int LOG_GROUP>
int start(Int4Args a, cudaStream_t s) {
  const int tiles = (a.N + 15) / 16, chunks = (a.K + kChunk - 1) / kChunk;
  int split = 1;
  auto range = [&] { return (chunks + split - 1) / split * kChunk; };
  // shares of k: until x of one is at most 40 KB, and until there are CTAs enough of a tile each
  while (split < kMaxSplit && chunks > split && (a.M * range() * 2 > 40 * 1024 || tiles * split < 148)) split *= 2;
  a.k_range = range();
  while (split > 1 && (split - 1) * a.k_range >= a.K) split /= 2, a.k_range = range();      // rounded up, the last shares may be empty
  int rows = kCtas / split;
  a.tiles = (tiles + rows - 1) / rows;
  // parts of k: as many as keep the warps even, at least eight steps each where the tiles are many
  const int steps = a.k_range / kChunk;
  a.wk = kMaxWarps;
  while (a.wk > 1 && (a.wk > steps || (a.tiles * a.wk >= 4 * kMaxWarps && steps < 8 * a.wk))) a.wk /= 2;
  while (a.tiles > 1 && a.wk * a.M * a.tiles > 768) a.tiles = (a.tiles + 1) / 2;        // sums of the products: 48 KB
  int warps = kMaxWarps;
  while (warps > a.wk && warps / 2 >= a.tiles * a.wk) warps /= 2;
  a.k_part = (steps + a.wk - 1) / a.wk * kChunk;
  // every CTA's and every warp's first group, and so every row's piece of the scales, on a boundary of eight
  a.table_vec = (a.K >> LOG_GROUP) % 8 == 0 && (split == 1 || (a.k_range >> LOG_GROUP) % 8 == 0) && (a.wk == 1 || (a.k_part >> LOG_GROUP) % 8 == 0) &&
                 aligned(a.scales, 16) && aligned(a.zeros, 8);
  const Layout at(warps, a.M, a.k_range, a.k_part, a.wk * a.M * 16 * a.tiles, LOG_GROUP);
  if (at.bytes > kMostSmem) {                    // many rows of a long k: half of the rows at a time
    if (a.M == 1) return (int)cudaErrorInvalidValue;
    Int4Args b = a;
    a.M /= 2;
    b.M -= a.M;
    b.x = (const T*)b.x + a.M * b.x_row;
    b.y = (T*)b.y + a.M * b.y_row;
    if (int e = start<T, LOG_GROUP>(a, s)) return e;
    return start<T, LOG_GROUP>(b, s);
  }
  const int row_blocks = (tiles + a.tiles - 1) / a.tiles;
  if (row_blocks > 65535) {                      // as many as a grid may have in this direction: half of the outputs at a time
    Int4Args b = a;
    a.N = tiles / 2 * 16;
    b.N -= a.N;
    b.codes += (size_t)a.N * (a.K / 2);
    b.scales = (const T*)b.scales + (size_t)a.N * (a.K >> LOG_GROUP);
    if (b.zeros) b.zeros += (size_t)a.N * (a.K >> LOG_GROUP);
    if (b.bias) b.bias = (const T*)b.bias + a.N;
    b.y = (T*)b.y + a.N;
    if (int e = start<T, LOG_GROUP>(a, s)) return e;
    return start<T, LOG_GROUP>(b, s);
  }
  auto kernel = linear_kernel<T, TILES, LOG_GROUP>;
  if (int e = (int)allow_dynamic_smem<kMostSmem>(kernel)) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(split, row_blocks);
  cfg.blockDim = dim3(32 * warps);
  cfg.dynamicSmemBytes = at.bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 2 : 1;
  return (int)cudaLaunchKernelEx(&cfg, kernel, a);
}
template <typename T, int LOG_GROUP>
int start(const Int4Args& a, cudaStream_t s) {
  return a.M <= 8 ? start<T, 1, LOG_GROUP>(a, s) : start<T, 2, LOG_GROUP>(a, s);
}
template <typename T>
int start(const Int4Args& a, int group, cudaStream_t s) {
  return group == 32 ? start<T, 5>(a, s) : group == 64 ? start<T, 6>(a, s) : start<T, 7>(a, s);
}

}  // namespace
}  // namespace nova

extern "C" int nova_linear_int4(int type, const void* x, int64_t x_row, int M, int K, const void* codes, const void* scales,
                                const void* zeros, int group, const void* bias, int N, void* y, int64_t y_row, nova_stream stream) {
  using namespace nova;
  using namespace nova::mix;
  if (type == NOVA_F32) return NOVA_ERR_UNSUPPORTED;
  if (!type_ok(type) || !x || !codes || !scales || !y || x == y || M < 1 || M > NOVA_INT4_MAX_ROWS || N < 1 || N > NOVA_INT4_MAX_N || K < 1 || K > NOVA_INT4_MAX_K ||
      (group != 32 && group != 64 && group != 128) || K % group || x_row < 0 || y_row < 0)
    return NOVA_ERR_INVALID_ARG;
  if (!aligned(x, 2) || !aligned(scales, 2) || !aligned(bias, 2) || !aligned(y, 2) || !aligned(codes, 16)) return NOVA_ERR_INVALID_ARG;
  const Int4Args a = {x, scales, bias, (const unsigned char*)codes, (const unsigned char*)zeros, y, (long long)x_row, (long long)y_row, M, N, K,
                      aligned(x, 16) && x_row % 8 == 0, 1};
  cudaStream_t s = (cudaStream_t)stream;
  return launch_status(type == NOVA_F16 ? start<__half>(a, group, s) : start<__nv_bfloat16>(a, group, s));
}
