// Storing rows and weights in 8 bits, bringing them back, and the backward of the GeGLU gate on stored rows.  All bound by memory.
#include "fp8_util.h"

namespace mb {
namespace {

// 16 consecutive values of a row as floats.
__device__ __forceinline__ void load16(const float* p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(p + 4 * i);
    x[4 * i] = v.x;
    x[4 * i + 1] = v.y;
    x[4 * i + 2] = v.z;
    x[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void load16(const uint16_t* p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p + 8 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[8 * i + 2 * j] = __uint_as_float(v[j] << 16);
      x[8 * i + 2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void store16(float* p, const float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(p + 4 * i) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}
__device__ __forceinline__ void store16(uint16_t* p, const float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack_bf16(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
    *reinterpret_cast<u32x4*>(p + 8 * i) = v;
  }
}
__device__ __forceinline__ u32x4 pack16(const float (&x)[16], int byte) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack_e4m3(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], scale_bits(byte));
  return r;
}

// The k-th of the items from `first` (the same in all lanes) on, k < 256, rows of `per` items: its row and place in it.  (Below
// 512 items a row k crosses several rows: c m / 2^20 with m the next integer over 2^20 / per is c / per exactly for c < 768.  The
// division of 64-bit numbers that stood here was a fifth of the gate backward's instructions.)
__device__ __forceinline__ void locate(uint32_t first, uint32_t per, uint32_t k, int64_t& row, int& at) {
  const uint32_t row0 = __builtin_amdgcn_readfirstlane(first / per);
  const uint32_t c = first - row0 * per + k;
  const uint32_t m = __builtin_amdgcn_readfirstlane((1u << 20) / per + 1);
  const uint32_t rows = per > 512 ? (c >= per ? 1u : 0u) : (c * m) >> 20;
  row = (int64_t)row0 + rows;
  at = (int)(c - rows * per);
}

// Rows -> 8 bits: eight lanes per block of 128, 16 values each, a thread per 16 values and nothing in it but one trip to memory.
// (26963 x 3072 bf16: 43.4 us, 5.7 TB/s.)
template <typename T>
__global__ __launch_bounds__(256) void fp8_quant_kernel(const T* __restrict__ x, int64_t stride, int T_cap,
                                                        const int32_t* __restrict__ meta, int W, int blocks,
                                                        uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int rows = meta ? min(meta[0], T_cap) : T_cap;
  const int piece = threadIdx.x & 7;
  int64_t row;
  int block;
  locate(blockIdx.x * 32, blocks, threadIdx.x >> 3, row, block);
  if (row >= rows) return;
  const int col = block * kFp8Block + piece * 16;
  float v[16];
  if (col < W) {
    load16(x + row * stride + col, v);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
  }
  const int byte = scale_byte(max_of_8_lanes(largest_of_16(v)));
  if (col < W) *reinterpret_cast<u32x4*>(q + row * W + col) = pack16(v, byte);
  if (piece == 0) s[row * blocks + block] = (uint8_t)byte;
}

// 8-bit rows -> rows: 16 values per lane.  (26963 x 768 to bf16: 11.6 us, 5.4 TB/s.)
template <typename T>
__global__ __launch_bounds__(256) void fp8_dequant_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                          int T_cap, const int32_t* __restrict__ meta, int W, int blocks,
                                                          T* __restrict__ x, int64_t stride) {
  const int rows = meta ? min(meta[0], T_cap) : T_cap;
  int64_t row;
  int piece;
  locate(blockIdx.x * 256, W >> 4, threadIdx.x, row, piece);
  if (row >= rows) return;
  const int col = piece * 16;
  const u32x4 w = *reinterpret_cast<const u32x4*>(q + row * W + col);
  const float scale = scale_bits(s[row * blocks + (col >> 7)]);
  float v[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f[4];
    unpack_e4m3(w[i], scale, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 * i + j] = f[j];
  }
  store16(x + row * stride + col, v);
}

// One 128 x 128 block of a weight per workgroup: thread t holds rows 4 (t / 8) .. + 3, columns 16 (t % 8) .. + 15.  The
// transposed copy goes through LDS, four rows' bytes of a column in one word.  (6144 x 768 fp32, both copies: 7.6 us a
// call, 28 MB.)
constexpr int kTransPitch = 33;   // words of a column's 128 rows, and one so that columns start in different banks
template <typename T>
__global__ __launch_bounds__(256) void fp8_quant_weight_kernel(const T* __restrict__ w, int n_out, int n_in,
                                                               uint8_t* __restrict__ q, uint8_t* __restrict__ s,
                                                               uint8_t* __restrict__ qt, uint8_t* __restrict__ st) {
  __shared__ float top[4];
  __shared__ uint32_t words[128 * kTransPitch];
  const int r0 = blockIdx.y * 128, c0 = blockIdx.x * 128, tid = threadIdx.x;
  const int row = r0 + 4 * (tid >> 3), col = c0 + 16 * (tid & 7);
  float v[4][16], a = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (row + i < n_out && col < n_in) {
      load16(w + (int64_t)(row + i) * n_in + col, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[i][j] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) a = fmaxf(a, largest_of_16(v[i]));
#pragma unroll
  for (int k = 1; k < 64; k *= 2) a = fmaxf(a, __shfl_xor(a, k));
  if ((tid & 63) == 0) top[tid >> 6] = a;
  __syncthreads();
  const int byte = scale_byte(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
  u32x4 r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = pack16(v[i], byte);
    if (row + i < n_out && col < n_in) *reinterpret_cast<u32x4*>(q + (int64_t)(row + i) * n_in + col) = r[i];
  }
  if (tid == 0) {
    s[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = (uint8_t)byte;
    if (st) st[(int64_t)blockIdx.x * gridDim.y + blockIdx.y] = (uint8_t)byte;
  }
  if (!qt) return;
#pragma unroll
  for (int j = 0; j < 16; ++j) {   // column j of the thread's patch: a byte of each of its four rows
    const int k = j >> 2, b = 8 * (j & 3);
    words[(16 * (tid & 7) + j) * kTransPitch + (tid >> 3)] = (r[0][k] >> b & 0xffu) | (r[1][k] >> b & 0xffu) << 8 |
                                                             (r[2][k] >> b & 0xffu) << 16 | (r[3][k] >> b & 0xffu) << 24;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {   // columns become rows: 8 lanes write 128 bytes of one
    const int c = 32 * i + (tid >> 3), p = tid & 7;
    if (c0 + c < n_in && r0 + 16 * p < n_out) {
      const uint32_t* from = &words[c * kTransPitch + 4 * p];
      const u32x4 out = {from[0], from[1], from[2], from[3]};
      *reinterpret_cast<u32x4*>(qt + (int64_t)(c0 + c) * n_out + r0 + 16 * p) = out;
    }
  }
}

__device__ __forceinline__ double bf16_value(uint16_t b) { return (double)__uint_as_float((uint32_t)b << 16); }

// Backward of the gate act = GeLU(h) (*) g from dA and h | g (bf16, or 8 bits with scales): dh | dg in 8 bits.  Eight lanes
// per 128 columns, 16 values of dA, h and g each; both results' blocks are those lanes' own.  (26963 x 3072, h | g in 8 bits: 98 us,
// 5.1 TB/s; two transcendentals and some 30 other instructions a value stay just under the memory's time.)
constexpr uint32_t kReach = 1024;   // 7e-5 of a value; gelu_tail_and_grad leaves 5.9e-5 beside the derivative's zero and 9e-6 elsewhere
template <bool kEight>
__global__ __launch_bounds__(256) void fp8_gate_bwd_kernel(const uint16_t* __restrict__ da, const void* __restrict__ hg,
                                                           const uint8_t* __restrict__ hgs, int T_cap,
                                                           const int32_t* __restrict__ meta, int inter,
                                                           uint8_t* __restrict__ q, uint8_t* __restrict__ s) {
  const int rows = meta ? min(meta[0], T_cap) : T_cap;
  const int blocks = inter / kFp8Block;
  const int piece = threadIdx.x & 7;
  int64_t row;
  int block;
  locate(blockIdx.x * 32, blocks, threadIdx.x >> 3, row, block);
  if (row >= rows) return;
  const int col = block * kFp8Block + piece * 16;
  float a[16], h[16], g[16];
  load16(da + row * inter + col, a);
  const int64_t place = row * (2 * inter) + col;
  if (kEight) {
    const uint8_t* p = static_cast<const uint8_t*>(hg) + place;
    const u32x4 hw = *reinterpret_cast<const u32x4*>(p), gw = *reinterpret_cast<const u32x4*>(p + inter);
    const uint8_t* sc = hgs + row * (2 * blocks) + block;
    const float hs = scale_bits(sc[0]), gs = scale_bits(sc[blocks]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f[4], e[4];
      unpack_e4m3(hw[i], hs, f);
      unpack_e4m3(gw[i], gs, e);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[4 * i + j] = f[j];
        g[4 * i + j] = e[j];
      }
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(hg) + place;
    load16(p, h);
    load16(p + inter, g);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float val, grad;
    gelu_tail_and_grad(h[i], val, grad);
    h[i] = a[i] * (g[i] * grad);   // (a g may be beyond the largest float where the derivative is next to nothing)
    g[i] = a[i] * val;
    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (four values at a time: 98 us, with all 16 interleaved 107)
  }
  float htop = max_of_8_lanes(largest_of_16(h)), gtop = max_of_8_lanes(largest_of_16(g));
  if (__builtin_expect(__ballot(near_border(htop, kReach) || near_border(gtop, kReach)) != 0, 0)) {
    // a block in some thousand: the values that decide once more, in 64 bits, each lane one of its own after the other
    const float hfrom = near_border(htop, kReach) ? border_from(htop, kReach) : __builtin_inff();
    const float gfrom = near_border(gtop, kReach) ? border_from(gtop, kReach) : __builtin_inff();
    uint32_t left = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      left |= finite_abs(h[i]) >= hfrom ? 1u << i : 0u;
      left |= finite_abs(g[i]) >= gfrom ? 0x10000u << i : 0u;
    }
    float h64 = 0.f, g64 = 0.f;
#pragma unroll 1
    for (; __ballot(left != 0); left &= left - 1) {
      const int bit = left ? __builtin_ctz(left) : 0, i = bit & 15;
      const double x = bf16_value(da[row * inter + col + i]);
      double hv, gv, slope;
      if (kEight) {
        const uint8_t* p = static_cast<const uint8_t*>(hg) + place + i;
        const uint8_t* sc = hgs + row * (2 * blocks) + block;
        hv = (double)__builtin_amdgcn_cvt_f32_fp8(p[0], 0) * scale_value(sc[0]);
        gv = (double)__builtin_amdgcn_cvt_f32_fp8(p[inter], 0) * scale_value(sc[blocks]);
      } else {
        const uint16_t* p = static_cast<const uint16_t*>(hg) + place + i;
        hv = bf16_value(p[0]);
        gv = bf16_value(p[inter]);
      }
      const double value = gelu64(hv, &slope);
      const float top = finite_abs(round_beside_border(x * (bit < 16 ? gv * slope : value)));
      if (left && bit < 16) h64 = fmaxf(h64, top);
      if (left && bit >= 16) g64 = fmaxf(g64, top);
    }
    h64 = max_of_8_lanes(h64);
    g64 = max_of_8_lanes(g64);
    if (near_border(htop, kReach)) htop = h64;
    if (near_border(gtop, kReach)) gtop = g64;
  }
  const int hb = scale_byte(htop), gb = scale_byte(gtop);
  *reinterpret_cast<u32x4*>(q + place) = pack16(h, hb);
  *reinterpret_cast<u32x4*>(q + place + inter) = pack16(g, gb);
  if (piece == 0) {
    s[row * (2 * blocks) + block] = (uint8_t)hb;
    s[row * (2 * blocks) + blocks + block] = (uint8_t)gb;
  }
}

unsigned grid_for(int64_t threads) { return (unsigned)((threads + 255) / 256); }

}  // namespace

mb_status launch_fp8_quant(mb_dtype dt, const void* x, int64_t stride, int T_cap, const int32_t* meta, int W, uint8_t* q,
                           uint8_t* s, hipStream_t stream) {
  const int blocks = fp8_blocks(W);
  const dim3 grid(grid_for((int64_t)T_cap * blocks * 8));
  if (dt == MB_F32)
    fp8_quant_kernel<<<grid, dim3(256), 0, stream>>>(static_cast<const float*>(x), stride, T_cap, meta, W, blocks, q, s);
  else
    fp8_quant_kernel<<<grid, dim3(256), 0, stream>>>(static_cast<const uint16_t*>(x), stride, T_cap, meta, W, blocks, q, s);
  return check_launch("fp8_quant_kernel");
}

mb_status launch_fp8_dequant(mb_dtype dt, const uint8_t* q, const uint8_t* s, int T_cap, const int32_t* meta, int W, void* x,
                             int64_t stride, hipStream_t stream) {
  const int blocks = fp8_blocks(W);
  const dim3 grid(grid_for((int64_t)T_cap * (W / 16)));
  if (dt == MB_F32)
    fp8_dequant_kernel<<<grid, dim3(256), 0, stream>>>(q, s, T_cap, meta, W, blocks, static_cast<float*>(x), stride);
  else
    fp8_dequant_kernel<<<grid, dim3(256), 0, stream>>>(q, s, T_cap, meta, W, blocks, static_cast<uint16_t*>(x), stride);
  return check_launch("fp8_dequant_kernel");
}

mb_status launch_fp8_quant_weight(mb_dtype dt, const void* w, int n_out, int n_in, uint8_t* q, uint8_t* s, uint8_t* qt,
                                  uint8_t* st, hipStream_t stream) {
  const dim3 grid(fp8_blocks(n_in), fp8_blocks(n_out));
  if (dt == MB_F32)
    fp8_quant_weight_kernel<<<grid, dim3(256), 0, stream>>>(static_cast<const float*>(w), n_out, n_in, q, s, qt, st);
  else
    fp8_quant_weight_kernel<<<grid, dim3(256), 0, stream>>>(static_cast<const uint16_t*>(w), n_out, n_in, q, s, qt, st);
  return check_launch("fp8_quant_weight_kernel");
}

mb_status launch_gelu_gate_fp8_bwd(const void* da, const void* hg, const uint8_t* hgs, int T_cap, const int32_t* meta,
                                   int inter, uint8_t* q, uint8_t* s, hipStream_t stream) {
  const dim3 grid(grid_for((int64_t)T_cap * (inter / 16)));
  if (hgs)
    fp8_gate_bwd_kernel<true><<<grid, dim3(256), 0, stream>>>(static_cast<const uint16_t*>(da), hg, hgs, T_cap, meta, inter, q, s);
  else
    fp8_gate_bwd_kernel<false><<<grid, dim3(256), 0, stream>>>(static_cast<const uint16_t*>(da), hg, hgs, T_cap, meta, inter, q, s);
  return check_launch("fp8_gate_bwd_kernel");
}

}  // namespace mb
