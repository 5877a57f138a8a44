// Weight gradient from 8-bit rows:  dw[m, n] = sum over tokens t of dy[t, m] x[t, n], x the e4m3 rows that the product read (and
// the program kept), dy bf16 or e4m3 rows, fp32 sums.
//
// The contraction runs over tokens, along which every block has a scale of its own: the scaled matrix instruction, one byte for 32
// of k, cannot take them.  So the operands are brought back to bf16 on their way into LDS (v_cvt_scalef32_pk_bf16_fp8, exact: 4
// bits of significand and a power of two) and multiplied by v_mfma_f32_32x32x16_bf16.  They pass through registers for it: 16 bytes of
// a row per load, one scale byte each, two 16-byte LDS writes.  The rest is the bf16 weight gradient's way: rows as they are
// in LDS, operands by transposing reads, 64 kMB x 256 tiles by 8 waves, steps of 64 tokens in two stages, the tokens split over
// workgroups where the tiles are few, partial tiles added in a fixed order.  26963 x 768 x 6144 takes 225 us in three splits, 12 of them
// the adding.  (Where it took 235, in seven, it took 195 without the steps' loads and LDS writes and 231 without conversions.)
#include "fp8_util.h"

namespace mb {
namespace {

constexpr int kRows = 64;         // tokens per step
constexpr int kMaxSplits = 128;

struct Wgrad {
  const void* dy;                 // bf16 [T, n_out] of row stride dy_stride, or e4m3 with scales dys
  const uint8_t* dys;
  int64_t dy_stride;
  const uint8_t *x, *xs;
  int n_out, n_in, n_tiles, tiles, splits, T_cap;
  const int32_t* meta;
  float* out;                     // of the first split; split s is n_out n_in floats further on, s times
};

// Piece x (8 bf16 columns) of row r sits at position x ^ 4 (r % 4) ^ (x / 8 + x / 16) % 2.  The four rows a transposing read touches
// lie in different banks (of 64), and so do the pieces that 8 lanes of a row write at a time, every second one of 8 or 16 and
// of another 8, in the 32 banks that a write sees.
__device__ __forceinline__ int place_of(int x, int r) { return x ^ (4 * (r & 3)) ^ ((x >> 3 ^ x >> 4) & 1); }

// The rows of one operand on their way into LDS: kCols columns of 64 tokens, 512 threads.  In 8 bits a thread takes 16 bytes of one
// row, or 16 and those 64 further on, which have one scale (a load of its own for each 16 bytes took a tenth of the whole time).
template <bool kEight, int kCols>
struct Stager {
  static constexpr int kPieces = kCols / (kEight ? 16 : 8);   // 16-byte pieces of a row in memory
  static constexpr int kN = kRows * kPieces / 512;            // per thread
  static constexpr int kLanes = kEight ? 8 : kPieces;         // threads per row
  u32x4 data[kN];
  uint32_t byte;
  int row, piece;           // of the first; the n-th lies 4 pieces on (8 bits), or 512 / kLanes rows
  uint32_t off, soff;       // byte offsets in a step's rows
  int there;                // bytes from here to the row's end
  const uint8_t *base, *sbase;
  int64_t pitch;            // bytes from row to row
  int blocks, T;
  __device__ __forceinline__ Stager(const void* p, const uint8_t* s, int64_t stride, int first_col, int cols, int T_, int tid) {
    constexpr int kEs = kEight ? 1 : 2;
    row = tid / kLanes;
    piece = tid % kLanes + (kEight && kN == 2 ? tid & 4 : 0);   // (4 lanes request 64 bytes in one go)
    pitch = stride * kEs;
    blocks = fp8_blocks(cols);
    T = T_;
    const int col = first_col + piece * (16 / kEs);
    there = (cols - col) * kEs;   // (columns are a multiple of 16)
    base = static_cast<const uint8_t*>(p) + (int64_t)first_col * kEs;
    sbase = s;
    off = (uint32_t)row * (uint32_t)pitch + piece * 16;
    soff = there > 0 ? (uint32_t)row * (uint32_t)blocks + col / kFp8Block : 0x80000000u;
  }
  // The rows of 64 tokens from `first` on are what is requested next (rows at or beyond T, and what is no column: zeros).
  __amdgpu_buffer_rsrc_t rsrc, srsrc;
  __device__ __forceinline__ void aim(int first) {
    const int rows = max(min(T - first, kRows), 0);
    const int at = rows > 0 ? first : 0;
    rsrc = uniform_rsrc(base + (int64_t)at * pitch, (uint32_t)rows * (uint32_t)pitch);
    if (kEight) srsrc = uniform_rsrc(sbase + (int64_t)at * blocks, (uint32_t)rows * (uint32_t)blocks);
  }
  __device__ __forceinline__ void request(int i) {
    data[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, there > (kEight ? 64 * i : 0) ? off : 0x80000000u,
                                                    kEight ? 64 * i : (uint32_t)(i * (512 / kLanes)) * (uint32_t)pitch, 0);
  }
  __device__ __forceinline__ void request_scale() {
    if (kEight) byte = __builtin_amdgcn_raw_buffer_load_b8(srsrc, soff, 0, 0);
  }
  // After the i-th put: requests what it was the last to need.
  __device__ __forceinline__ void request_behind(int i) {
    if ((i + 1) % kParts == 0) request(i / kParts);
    if (i + 1 == kPuts) request_scale();
  }
  // brings the i-th 16 bytes of bf16 of what was requested to LDS
  static constexpr int kParts = kEight ? 2 : 1, kPuts = kN * kParts;
  __device__ __forceinline__ void put(uint16_t* to, int i) const {
    if (kEight) {
      *reinterpret_cast<bf16x8*>(to + row * kCols + place_of(2 * (piece + 4 * (i / 2)) + i % 2, row) * 8) =
          to_bf16x8(data[i / 2][i % 2 * 2], data[i / 2][i % 2 * 2 + 1], scale_bits(byte));
    } else {
      const int r = row + i * (512 / kLanes);
      *reinterpret_cast<u32x4*>(to + r * kCols + place_of(piece, r) * 8) = data[i];
    }
  }
};

template <bool kEight, int kMB>
__global__ __launch_bounds__(512, 2) void fp8_wgrad_kernel(Wgrad pr) {
  constexpr int kM = 64 * kMB, kStage = kRows * (kM + 256), kMfma = 2 * kMB, kFrags = kMB + 2;
  __shared__ __attribute__((aligned(1024))) uint16_t smem[2 * kStage];
  const int T = __builtin_amdgcn_readfirstlane(pr.meta ? min(pr.meta[0], pr.T_cap) : pr.T_cap);
  // workgroup -> split and tile, every XCD a contiguous run: its compute units stream the same token rows
  const int total = pr.tiles * pr.splits, run = total >> 3;
  int lin = blockIdx.x;
  if (lin < (run << 3)) lin = (lin & 7) * run + (lin >> 3);
  const int split = __builtin_amdgcn_readfirstlane(lin / pr.tiles);
  const int tile = __builtin_amdgcn_readfirstlane(lin - split * pr.tiles);
  const int tile_m = __builtin_amdgcn_readfirstlane(tile / pr.n_tiles);
  const int m0 = tile_m * kM, n0 = (tile - tile_m * pr.n_tiles) * 256;
  const int steps_total = (T + kRows - 1) / kRows;
  const int per = __builtin_amdgcn_readfirstlane((steps_total + pr.splits - 1) / pr.splits);
  const int begin = split * per;
  const int nsteps = max(min(steps_total - begin, per), 0);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, g = lane >> 5;
  const int wm = wave >> 2, wn = wave & 3;
  const int end = min(T, (begin + nsteps) * kRows);   // (of the split's own tokens)
  Stager<kEight, kM> ps(pr.dy, pr.dys, pr.dy_stride, m0, pr.n_out, end, tid);
  Stager<true, 256> qs(pr.x, pr.xs, pr.n_in, n0, pr.n_in, end, tid);

  // Fragment reads: lane -> row tr_row (+ 8) and 4 columns of a 16 x 32 patch; P columns 32 (kMB wm + mb), Q columns
  // 64 wn + 32 nb.
  const int tr_i = lane & 15, tr_q = lane >> 4;
  const int tr_row = (tr_i >> 2) + 4 * (tr_q >> 1);
  const int tr_piece = 2 * (tr_q & 1) + ((tr_i & 3) >> 1), tr_sub = 4 * (tr_i & 1);
  uint32_t foff[kFrags];
#pragma unroll
  for (int i = 0; i < kFrags; ++i) {
    const int x = (i < kMB ? 4 * (kMB * wm + i) : 8 * wn + 4 * (i - kMB)) + tr_piece;
    foff[i] = (i < kMB ? 0 : kRows * kM) + tr_row * (i < kMB ? kM : 256) + place_of(x, tr_i >> 2) * 8 + tr_sub;
  }
  bf16x8 pf[2][kMB], qf[2][2];
  auto read_frag = [&](int stage, int kk, int i) {
    const int cols = i < kMB ? kM : 256;
    const uint16_t* p = smem + stage * kStage + foff[i] + kk * (16 * cols);
    const bf16x8 f = join_tr(lds_read_tr4(p), lds_read_tr4(p + 8 * cols));
    if (i < kMB) pf[kk & 1][i] = f;
    else qf[kk & 1][i - kMB] = f;
  };
  constexpr auto nth_needed = [](int n) { return n == 0 ? kMB : n == 1 ? 0 : n == 2 ? kMB + 1 : n - 2; };   // (read in this order)
  constexpr int kPuts = Stager<kEight, kM>::kPuts + Stager<true, 256>::kPuts;
  auto put = [&](int stage, int i) {
    if (i < qs.kPuts) qs.put(smem + stage * kStage + kRows * kM, i);
    else ps.put(smem + stage * kStage, i - qs.kPuts);
  };
  auto aim = [&](int step) {
    qs.aim((begin + step) * kRows);
    ps.aim((begin + step) * kRows);
  };
  auto request_behind = [&](int i) {
    if (i < qs.kPuts) qs.request_behind(i);
    else ps.request_behind(i - qs.kPuts);
  };
  f32x16 acc[kMB][2];   // [m block][n block]
#pragma unroll
  for (int x = 0; x < kMB; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.f;

  aim(0);
#pragma unroll
  for (int i = 0; i < kPuts; ++i) request_behind(i);
  aim(1);
#pragma unroll
  for (int i = 0; i < kPuts; ++i) {
    put(0, i);
    request_behind(i);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kFrags; ++i) read_frag(0, 0, i);
  // A step is four quarters of 16 tokens; during a quarter the next one's fragments are read.  In the first three the step
  // after this one goes to the other stage, piece by piece, and behind each piece the same one of the step after that is
  // requested, a whole step before it is needed.  Behind the last quarter's first product stands the barrier behind which the
  // other stage is whole and this one is read no more.  (Steps past the last read zeros that nobody uses.)
#pragma unroll 1
  for (int st = 0; st < nsteps; ++st) {
    const int stage = st & 1, next = stage ^ 1;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      if (kk == 0) aim(st + 2);
#pragma unroll
      for (int x = 0; x < kMfma; ++x) {
        acc[x >> 1][x & 1] = mfma32(pf[kk & 1][x >> 1], qf[kk & 1][x & 1], acc[x >> 1][x & 1]);
        __builtin_amdgcn_sched_barrier(0);
        if (kk == 3 && x == 0) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");   // (under the first products)
#pragma unroll
        for (int i = x; i < kFrags; i += kMfma) read_frag(kk == 3 ? next : stage, (kk + 1) & 3, nth_needed(i));
#pragma unroll
        for (int i = 0; i < kPuts; ++i) {
          if (i * (3 * kMfma) / kPuts == kk * kMfma + x) {   // (spread evenly over the first three quarters)
            put(next, i);
            request_behind(i);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // fp32 tile: register v of block (x, y) is row 8 (v / 4) + 4 g + v % 4, lane c is the column
  const int row0 = m0 + wm * (32 * kMB);
  float* const dst = pr.out + (int64_t)split * pr.n_out * pr.n_in + (int64_t)min(row0, pr.n_out) * pr.n_in;
  const __amdgpu_buffer_rsrc_t ors = uniform_rsrc(dst, (uint32_t)max(min(pr.n_out - row0, 32 * kMB), 0) * (uint32_t)pr.n_in * 4u);
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int col = n0 + wn * 64 + y * 32 + c;
    const uint32_t at = col < pr.n_in ? ((uint32_t)(4 * g) * (uint32_t)pr.n_in + col) * 4u : 0x80000000u;
#pragma unroll
    for (int x = 0; x < kMB; ++x)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(acc[x][y][v]), ors, at,
                                              (uint32_t)(x * 32 + 8 * (v >> 2) + (v & 3)) * (uint32_t)pr.n_in * 4u, 0);
  }
}

// Few tokens: 64 x 64 tiles by 8 waves that share the tokens, wave w the chunks w, w + 8, ... of 32.  A wave stages its chunk in
// LDS of its own, so nothing waits for a barrier, requests the next one while it multiplies, and the waves' sums meet in LDS
// once, w + 4 to w first and then in order.
constexpr int kChunk = 32;
template <bool kEight>
__global__ __launch_bounds__(512, 4) void fp8_wgrad_slice_kernel(Wgrad pr) {
  constexpr int kArea = 2 * kChunk * 64;   // bf16 elements of a wave: 32 rows of 64 columns of dy, then of x
  __shared__ __attribute__((aligned(1024))) uint16_t smem[8 * kArea];
  static_assert(sizeof(smem) == 4 * 64 * 64 * sizeof(float), "the sums of four waves take its place");
  const int T = __builtin_amdgcn_readfirstlane(pr.meta ? min(pr.meta[0], pr.T_cap) : pr.T_cap);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = blockIdx.x, tile_m = tile / pr.n_tiles;
  const int m0 = tile_m * 64, n0 = (tile - tile_m * pr.n_tiles) * 64;
  uint16_t* const area = smem + wave * kArea;
  // Piece x (8 columns) of row r at position x ^ r % 2 ^ 4 (r / 2 % 2): four rows' reads in different banks of 64, and the writes of
  // 8 lanes, every second piece of two rows, in different ones of 32.
  auto place = [](int x, int r) { return r * 64 + ((x ^ (r & 1) ^ (4 * (r >> 1 & 1))) * 8); };
  constexpr int kPer = kEight ? 4 : 8, kP = kChunk * kPer / 64, kQ = kChunk * 4 / 64;   // lanes per row of dy, loads of dy and x
  const int64_t ppitch = pr.dy_stride * (kEight ? 1 : 2);
  const int blocks_p = fp8_blocks(pr.n_out), blocks_q = fp8_blocks(pr.n_in);
  const int prow = lane / kPer, pcol = lane % kPer * (kEight ? 16 : 8), qrow = lane >> 2, qcol = (lane & 3) * 16;
  const bool pthere = m0 + pcol < pr.n_out, qthere = n0 + qcol < pr.n_in;
  const uint32_t poff = pthere ? (uint32_t)prow * (uint32_t)ppitch + pcol * (kEight ? 1 : 2) : 0x80000000u;
  const uint32_t qoff = qthere ? (uint32_t)qrow * (uint32_t)pr.n_in + qcol : 0x80000000u;
  const uint32_t psoff = pthere ? (uint32_t)prow * (uint32_t)blocks_p + (m0 + pcol) / kFp8Block : 0x80000000u;
  const uint32_t qsoff = qthere ? (uint32_t)qrow * (uint32_t)blocks_q + (n0 + qcol) / kFp8Block : 0x80000000u;
  u32x4 pd[kP], qd[kQ];
  uint32_t pb[kP] = {}, qb[kQ];
  auto request = [&](int chunk) {   // (rows at or beyond T: zeros)
    const int first = min(chunk * kChunk, T), rows = min(T - first, kChunk);
    const __amdgpu_buffer_rsrc_t p = uniform_rsrc(static_cast<const uint8_t*>(pr.dy) + first * ppitch + (int64_t)m0 * (kEight ? 1 : 2),
                                                  (uint32_t)rows * (uint32_t)ppitch);
    const __amdgpu_buffer_rsrc_t q = uniform_rsrc(pr.x + (int64_t)first * pr.n_in + n0, (uint32_t)rows * (uint32_t)pr.n_in);
    const __amdgpu_buffer_rsrc_t qs = uniform_rsrc(pr.xs + (int64_t)first * blocks_q, (uint32_t)rows * (uint32_t)blocks_q);
#pragma unroll
    for (int i = 0; i < kQ; ++i) qd[i] = __builtin_amdgcn_raw_buffer_load_b128(q, qoff, (uint32_t)(16 * i) * (uint32_t)pr.n_in, 0);
#pragma unroll
    for (int i = 0; i < kP; ++i)
      pd[i] = __builtin_amdgcn_raw_buffer_load_b128(p, poff, (uint32_t)(64 / kPer * i) * (uint32_t)ppitch, 0);
#pragma unroll
    for (int i = 0; i < kQ; ++i) qb[i] = __builtin_amdgcn_raw_buffer_load_b8(qs, qsoff, (uint32_t)(16 * i) * (uint32_t)blocks_q, 0);
    if (kEight) {
      const __amdgpu_buffer_rsrc_t ps = uniform_rsrc(pr.dys + (int64_t)first * blocks_p, (uint32_t)rows * (uint32_t)blocks_p);
#pragma unroll
      for (int i = 0; i < kP; ++i) pb[i] = __builtin_amdgcn_raw_buffer_load_b8(ps, psoff, (uint32_t)(16 * i) * (uint32_t)blocks_p, 0);
    }
  };
  auto put8 = [&](uint16_t* to, u32x4 d, uint32_t byte, int row, int col) {
    *reinterpret_cast<bf16x8*>(to + place(col / 8, row)) = to_bf16x8(d[0], d[1], scale_bits(byte));
    *reinterpret_cast<bf16x8*>(to + place(col / 8 + 1, row)) = to_bf16x8(d[2], d[3], scale_bits(byte));
  };
  // Fragment reads: lane -> row tr_row (+ 8) of 16 and 4 columns of a block of 32
  const int tr_i = lane & 15, tr_q = lane >> 4;
  const int tr_row = (tr_i >> 2) + 4 * (tr_q >> 1), tr_piece = 2 * (tr_q & 1) + ((tr_i & 3) >> 1), tr_sub = 4 * (tr_i & 1);
  f32x16 acc[2][2] = {};
  const int chunks = (T + kChunk - 1) / kChunk;
  if (wave < chunks) request(wave);
  for (int chunk = wave; chunk < chunks; chunk += 8) {
#pragma unroll
    for (int i = 0; i < kQ; ++i) put8(area + kChunk * 64, qd[i], qb[i], 16 * i + qrow, qcol);
#pragma unroll
    for (int i = 0; i < kP; ++i) {
      if (kEight) put8(area, pd[i], pb[i], 16 * i + prow, pcol);
      else *reinterpret_cast<u32x4*>(area + place(pcol / 8, 8 * i + prow)) = pd[i];
    }
    if (chunk + 8 < chunks) request(chunk + 8);
    // (a wave's LDS operations complete in order)
#pragma unroll
    for (int kk = 0; kk < kChunk / 16; ++kk) {
      bf16x8 f[2][2];
#pragma unroll
      for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint16_t* from = area + o * (kChunk * 64);
          const int r = 16 * kk + tr_row, x = 4 * b + tr_piece;
          f[o][b] = join_tr(lds_read_tr4(from + place(x, r) + tr_sub), lds_read_tr4(from + place(x, r + 8) + tr_sub));
        }
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) acc[a][b] = mfma32(f[0][a], f[1][b], acc[a][b]);
    }
  }
  float* const sums = reinterpret_cast<float*>(smem);
  const int l = lane_again(), c = l & 31, g = l >> 5;
  auto at = [&](int w, int a, int b, int v) { return (w * 64 + a * 32 + 8 * (v >> 2) + 4 * g + (v & 3)) * 64 + b * 32 + c; };
#pragma unroll
  for (int round = 0; round < 2; ++round) {   // waves 4 .. 7 hand theirs over, then waves 0 .. 3 the sums of two
    __syncthreads();
    if (wave >> 2 == 1 - round) {
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            float& s = sums[at(wave & 3, a, b, v)];
            s = round == 0 ? acc[a][b][v] : acc[a][b][v] + s;
          }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = wave * 64 + l + 512 * i, m = m0 + (p >> 4), n = n0 + (p & 15) * 4;
    if (m >= pr.n_out || n >= pr.n_in) continue;
    float4 s = *reinterpret_cast<const float4*>(&sums[p * 4]);
#pragma unroll
    for (int w = 1; w < 4; ++w) {
      const float4 b = *reinterpret_cast<const float4*>(&sums[w * 4096 + p * 4]);
      s.x += b.x; s.y += b.y; s.z += b.z; s.w += b.w;
    }
    *reinterpret_cast<float4*>(pr.out + (int64_t)m * pr.n_in + n) = s;
  }
}

// out[i] = sum over splits of partial[s][i], four at a time: kGroups groups of threads take an equal share of the splits each,
// in order, and then their sums are added in order.  (With many splits there are few results: one thread for all of a result's
// would add up one round trip after the other.)
template <int kGroups>
__global__ __launch_bounds__(256) void fp8_wgrad_add_kernel(const float* __restrict__ partial, int splits, int64_t count4,
                                                            float* __restrict__ out) {
  constexpr int kItems = 256 / kGroups;
  __shared__ float4 sums[kGroups > 1 ? 256 : 1];
  const float4* src = reinterpret_cast<const float4*>(partial);
  const int item = threadIdx.x % kItems, group = threadIdx.x / kItems;
  const int64_t i = (int64_t)blockIdx.x * kItems + item;
  const int share = (splits + kGroups - 1) / kGroups, from = group * share, to = min(from + share, splits);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (i < count4) {
#pragma unroll 4
    for (int s = from; s < to; ++s) {
      const float4 b = src[(int64_t)s * count4 + i];
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
  }
  if (kGroups > 1) {
    sums[threadIdx.x] = a;
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int g = 1; g < kGroups; ++g) {
      const float4 b = sums[g * kItems + item];
      a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
    }
  }
  if (i < count4) reinterpret_cast<float4*>(out)[i] = a;
}

// Splits of the tokens and the tile's height (0: slices) with the least estimated time.  (Fitted to 16 shapes, which it meets
// within a fifth.  One piece in slices, tiles of 256 and 128 rows: 64 x 768 x 768 4.9 / 8.5 / 6.3 us, 945 x 768 x 768 8.2 / 26 / 18,
// 945 x 768 x 2304 13.9 / 27 / 18.7, 945 x 768 x 6144 28 / 29 / 21, 2500 x 768 x 768 14.9 / 57 / 39 (in 5 splits 26 / 20.7), 26963 x
// 768 x 768 94 / 530 / 359 (24 and 14 splits 47 / 44), 26963 x 768 x 6144 638 / 541 / 380 (3 and 5 splits 226 / 277;
// in 7 of 256 rows 230).)
struct Choice {
  int splits, height;
};
Choice choose(int T_cap, int n_in, int n_out) {
  const int steps = (T_cap + kRows - 1) / kRows;
  const double bytes = 4.0 * n_in * n_out;
  const double slices = (double)((n_out + 63) / 64) * ((n_in + 63) / 64) / kComputeUnits;
  Choice best{1, 0};
  double least = 2.2 + (slices > 1.0 ? slices : 1.0) * (1.7 + 0.85 * ((T_cap + 8 * kChunk - 1) / (8 * kChunk)));
  for (int mb = 4; mb >= 2; mb -= 2) {
    const int64_t tiles = (int64_t)((n_out + 64 * mb - 1) / (64 * mb)) * ((n_in + 255) / 256);
    for (int s = 1; s <= kMaxSplits && s <= (steps > 0 ? steps : 1); ++s) {
      const double full = tiles * s < kComputeUnits ? (double)(tiles * s) / kComputeUnits : 1.0;
      const double power = full * full * full;   // (a step takes longer as the card fills up and its clock falls)
      const double step = mb == 4 ? 1.25 + 0.35 * power : 0.85 + 0.2 * power;
      const double cost = 3.0 + (double)((tiles * s + kComputeUnits - 1) / kComputeUnits) * (step * ((steps + s - 1) / s) + 2.5) +
                          (s > 1 ? 2.5 + (s + 1) * bytes / 7e6 : 0.0);
      if (cost < least) {
        least = cost;
        best = Choice{s, mb};
      }
    }
  }
  return best;
}

template <bool kEight>
void launch_wgrad(const Wgrad& pr, int height, hipStream_t stream) {
  const dim3 grid((unsigned)(pr.tiles * pr.splits));
  if (height == 4) fp8_wgrad_kernel<kEight, 4><<<grid, dim3(512), 0, stream>>>(pr);
  else fp8_wgrad_kernel<kEight, 2><<<grid, dim3(512), 0, stream>>>(pr);
}

}  // namespace

size_t linear_fp8_wgrad_workspace_bytes(int T_cap, int n_in, int n_out) {
  const Choice ch = choose(T_cap, n_in, n_out);
  return ch.splits > 1 ? (size_t)ch.splits * n_in * n_out * sizeof(float) : 0;
}

mb_status launch_linear_fp8_wgrad(const void* dy, const uint8_t* dys, int64_t dy_row_stride, const uint8_t* xq,
                                  const uint8_t* xs, int T_cap, const int32_t* meta, int n_in, int n_out, float* dw,
                                  void* workspace, hipStream_t stream) {
  const Choice ch = choose(T_cap, n_in, n_out);
  if (ch.height == 0) {
    const int n_tiles = (n_in + 63) / 64, tiles = (n_out + 63) / 64 * n_tiles;
    const Wgrad pr{dy, dys, dy_row_stride, xq, xs, n_out, n_in, n_tiles, tiles, 1, T_cap, meta, dw};
    if (dys) fp8_wgrad_slice_kernel<true><<<dim3(tiles), dim3(512), 0, stream>>>(pr);
    else fp8_wgrad_slice_kernel<false><<<dim3(tiles), dim3(512), 0, stream>>>(pr);
    return check_launch("fp8_wgrad_slice_kernel");
  }
  const int n_tiles = (n_in + 255) / 256, tiles = (n_out + 64 * ch.height - 1) / (64 * ch.height) * n_tiles;
  const bool whole = ch.splits == 1;
  const Wgrad pr{dy, dys, dy_row_stride, xq, xs, n_out, n_in, n_tiles, tiles, ch.splits, T_cap, meta,
                 whole ? dw : static_cast<float*>(workspace)};
  if (dys) launch_wgrad<true>(pr, ch.height, stream);
  else launch_wgrad<false>(pr, ch.height, stream);
  if (!whole) {
    const int64_t count4 = (int64_t)n_in * n_out / 4;
    const float* partial = static_cast<const float*>(workspace);
    if (ch.splits >= 8)
      fp8_wgrad_add_kernel<8><<<dim3((unsigned)((count4 + 31) / 32)), dim3(256), 0, stream>>>(partial, ch.splits, count4, dw);
    else
      fp8_wgrad_add_kernel<1><<<dim3((unsigned)((count4 + 255) / 256)), dim3(256), 0, stream>>>(partial, ch.splits, count4, dw);
  }
  return check_launch("fp8_wgrad_kernel");
}

}  // namespace mb
