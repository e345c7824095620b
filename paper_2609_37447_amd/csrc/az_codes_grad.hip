// The weight's and bias's gradients of a dense layer whose input was saved as
// codes: dw[n][k] = sum_m dy[m][n] x[m][k], db[n] = sum_m dy[m][n].
//
// A saved value is a bf16 number exactly, and dy is bf16, so the product runs on the
// bf16 matrix instruction with exact terms and fp32 sums.  The summed dimension runs
// down the rows of both operands: tiles stay in LDS as they lie in memory, and the
// transposing LDS read gives a lane four rows of its column.
//
// Four waves own T = 64 W rows of dw and as many columns, a wave a quarter of them (W x W
// blocks of 32 x 32), and step through 64 rows of dy and x at a time, two steps' tiles in
// turn in LDS.  dy is copied straight into LDS (through registers if its rows are not 16-byte
// aligned); the codes become bf16 on their way through registers, once for the whole workgroup.
// A wave reads the fragments of half a step while the matrix unit works on the half before.
//
// LDS rows hold T bf16 in 16-byte chunks, exchanged by the row (chunk ^ 4 (row % 4)): the four
// rows that a transposing read takes at a time then lie in different banks.
#include "az_codes_common.h"

namespace {

constexpr int NT = 256;
constexpr int MS = 64;  // rows of a step

typedef __attribute__((address_space(3))) uint8_t lds_bytes;
typedef __attribute__((ext_vector_type(4))) __bf16 cm_bf16x4;

template <bool F32>
__device__ __forceinline__ void put(void* p, int64_t at, float v, bool add) {
  if constexpr (F32) {
    float* o = (float*)p + at;
    *o = add ? *o + v : v;
  } else {
    uint16_t* o = (uint16_t*)p + at;
    *o = bf16_of(add ? f32_of_bf16(*o) + v : v);
  }
}

// Four neighbouring results, `left` of them (or more) before the row's end.
template <bool F32>
__device__ __forceinline__ void put4(void* p, int64_t at, cm_f32x4 v, int left, bool add) {
  if (left >= 4) {
    if constexpr (F32) {
      float* o = (float*)p + at;
      if (add) {
        cm_f32x4 old;
        __builtin_memcpy(&old, o, 16);
        v += old;
      }
      __builtin_memcpy(o, &v, 16);
    } else {
      uint16_t* o = (uint16_t*)p + at;
      uint16_t w[4] = {};
      if (add) __builtin_memcpy(w, o, 8);
#pragma unroll
      for (int e = 0; e < 4; e++) w[e] = bf16_of(f32_of_bf16(w[e]) + v[e]);
      __builtin_memcpy(o, w, 8);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 3; e++)
      if (e < left) put<F32>(p, at + e, v[e], add);
  }
}

// Eight bf16 of a row of n from column c on, zeros past its end, at any alignment: where the row
// ends before they do, the row's last eight are read and moved down.  Rows of fewer than
// eight are read one by one (in kernels that are instantiated for them).
struct Chunk8 {
  int at, down;
  __device__ __forceinline__ Chunk8(int c, int n) : at(min(c, n - 8)), down(min(c - min(c, n - 8), 8) * 16) {}
  __device__ __forceinline__ cm_i32x4 load(const uint16_t* row) const {
    cm_i32x4 v;
    __builtin_memcpy(&v, row + at, 16);
    return v;
  }
  __device__ __forceinline__ cm_i32x4 place(const cm_i32x4& v) const {
    typedef __attribute__((ext_vector_type(2))) uint64_t u64x2;
    const u64x2 w = __builtin_bit_cast(u64x2, v);
    u64x2 o;
    o[0] = down < 64 ? (w[0] >> down) | ((w[1] << 1) << (63 - down)) : w[1] >> (down & 63);
    o[1] = down < 64 ? w[1] >> down : 0;
    if (down >= 128) o[0] = 0;
    return __builtin_bit_cast(cm_i32x4, o);
  }
};

__device__ __forceinline__ cm_i32x4 short_row(const uint16_t* row, int c, int n) {
  cm_i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; i++)
    if (c + i < n) v[i >> 1] |= (int)((uint32_t)row[c + i] << (16 * (i & 1)));
  return v;
}

// 64 columns of dy summed over `m` rows by one workgroup: 32 groups of rows, joined in order.
__device__ void bias_columns(const uint16_t* __restrict__ dy, int64_t ldy, int n, int m, int n0, float* db, bool add, float* sums) {
  const int c = (threadIdx.x & 7) * 8, q = threadIdx.x >> 3;
  float s[8] = {};
  auto more = [&](const cm_i32x4& v) {
#pragma unroll
    for (int e = 0; e < 8; e++) s[e] += f32_of_bf16(((uint32_t)v[e >> 1] >> (16 * (e & 1))) & 0xffffu);
  };
  if (n >= 8) {
    const Chunk8 k(n0 + c, n);
    int i = q;
    constexpr int AHEAD = 16;  // loads on their way: a workgroup alone on its compute unit has latency to hide
    for (; i + (AHEAD - 1) * 32 < m; i += AHEAD * 32) {
      cm_i32x4 v[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; u++) v[u] = k.load(dy + (i + u * 32) * ldy);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < AHEAD; u++) more(k.place(v[u]));
    }
    for (; i < m; i += 32) more(k.place(k.load(dy + i * ldy)));
  } else {
    for (int i = q; i < m; i += 32) more(short_row(dy + i * ldy, n0 + c, n));
  }
#pragma unroll
  for (int e = 0; e < 8; e++) sums[q * 64 + c + e] = s[e];
  __syncthreads();
  const int t = threadIdx.x;
  if (t < 64 && n0 + t < n) {
    float v = 0.0f;
    for (int i = 0; i < 32; i++) v += sums[i * 64 + t];
    db[n0 + t] = add ? db[n0 + t] + v : v;
  }
}

// How a workgroup gets dy's tiles into LDS: copied (16-byte aligned rows), through registers at
// any alignment, or element by element (rows of fewer than eight).
enum { COPY = 0, MOVE = 1, SHORT = 2 };

template <int W>
struct Grad {
  static constexpr int T = 64 * W;
  static constexpr int ROW = 2 * T;            // LDS bytes of a row
  static constexpr int TILE = MS * ROW;        // of one operand's step
  static constexpr int STAGE = 2 * TILE;       // of both
  static constexpr int YROWS = 1024 / ROW;     // rows that one copy instruction of a wave fills
  static constexpr int YCOPIES = MS / (4 * YROWS);
  static constexpr int XCHUNKS = MS * T / 16 / NT;  // 16-code chunks of a thread

  struct Frag {
    cm_bf16x8 y[2][W], x[2][W];  // two sums of 16 rows
  };

  // A thread's chunks of a step of dy, straight into LDS; `rows` bytes lie between their rows.
  static __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t tile, lds_bytes* to, uint32_t off, int rows) {
#pragma unroll
    for (int j = 0; j < YCOPIES; j++) __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, to + j * 4 * YROWS * ROW, 16, off, j * rows, 0, 0);
  }
  static __device__ __forceinline__ cm_bf16x8 transposed(const uint8_t* p) {
    typedef __attribute__((address_space(3))) cm_bf16x4 lds4;
    const cm_bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)p);
    const cm_bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds4*)(p + 4 * ROW));
    return cm_bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  }
  // Fragments of half a step; yo, xo: the lane's places of the W blocks in the half's first rows.
  static __device__ __forceinline__ void read(Frag& f, const uint8_t* smem, const uint32_t (&yo)[W], const uint32_t (&xo)[W], uint32_t at) {
#pragma unroll
    for (int q = 0; q < 2; q++)
#pragma unroll
      for (int i = 0; i < W; i++) {
        f.y[q][i] = transposed(smem + (yo[i] + at) + q * 16 * ROW);
        f.x[q][i] = transposed(smem + (xo[i] + at) + q * 16 * ROW + TILE);
      }
  }
  static __device__ __forceinline__ void multiply(cm_f32x16 (&acc)[W][W], const Frag& f) {
#pragma unroll
    for (int q = 0; q < 2; q++)
#pragma unroll
      for (int i = 0; i < W; i++)
#pragma unroll
        for (int j = 0; j < W; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.x[q][j], f.y[q][i], acc[i][j], 0, 0, 0);
  }
  // Spreads half a step's LDS reads, loads and writes over its matrix instructions, reads first.
  template <int READS>
  static __device__ __forceinline__ void interleave() {
#pragma unroll
    for (int i = 0; i < 2 * W * W; i++) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < 8 * W / READS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
      else {
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 2, 0);
      }
    }
  }
};

// Blocks 0..bias-1 sum dy's columns; the others own a tile of dw each.  Both take the rows
// part * part_rows on, part = blockIdx.y; sums over one of several parts go to a workspace, dw's at
// part * part_stride and db's at part * n.  16384 x 4096 x 4096: 465-490 us warm (1,120-1,180 TFLOP/s, power);
// 1024 x 1880 x 10240: 59 us, of which 77 MB of results take 17 at a copy's rate.
template <int W, bool F32, int FEED>
__global__ __launch_bounds__(NT, W == 4 ? 1 : 2) void az_weight_grad(const uint16_t* __restrict__ dy, int64_t ldy, int n, CodeView x,
                                                                     void* __restrict__ dw, int64_t ldw, float* __restrict__ db,
                                                                     int bias, int add, int part_rows, int64_t part_stride) {
  using G = Grad<W>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  if ((int)blockIdx.x < bias) {
    const int from = (int)blockIdx.y * part_rows;
    bias_columns(dy + from * ldy, ldy, n, min(part_rows, x.rows - from), (int)blockIdx.x * 64, db + (int64_t)blockIdx.y * n, add,
                 reinterpret_cast<float*>(smem));
    return;
  }
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const uint32_t kt = (uint32_t)(x.cols + G::T - 1) / G::T, id = blockIdx.x - bias;
  const int n0 = (int)(id / kt) * G::T, k0 = (int)(id % kt) * G::T;
  // Rows are unsigned: a part's last steps begin past 2^31 where there are nearly as many.  (Counted from the part's
  // first row instead, with the pointers moved there, unaligned rows took 4% more.)
  const uint32_t mb = blockIdx.y * (uint32_t)part_rows, me = mb + (uint32_t)min(part_rows, x.rows - (int)mb);

  // dy, copied: a wave fills YROWS rows at a time, a lane one chunk.
  const int yr = G::YROWS * wave + lane / (G::T / 8), yp = lane % (G::T / 8), yc = yp ^ ((yr & 3) << 2);
  const uint32_t yoff = (uint32_t)yr * (uint32_t)ldy * 2u + (uint32_t)yc * 16u;
  lds_bytes* const ylds = (lds_bytes*)smem + G::YROWS * wave * G::ROW;
  auto copy_y = [&](uint32_t m, int stage) {
    // (past the last row: nothing is in range, and zeros are read.  The range is checked by whole words, of
    // which the row's last holds one element where n is odd: the range ends behind that word, which lies in
    // the row's last aligned 16 bytes.)
    const int rows = min((int)(me - m), MS);
    const uint32_t first = min(m, me - 1);
    const uint32_t bytes = (((uint32_t)max(rows, 1) - 1u) * (uint32_t)ldy + (((uint32_t)(n - n0) + 1u) & ~1u)) * 2u;
    const __amdgpu_buffer_rsrc_t buf =
        __builtin_amdgcn_make_buffer_rsrc((void*)(dy + first * ldy + n0), 0, (int)(bytes & (uint32_t)-(int)(rows > 0)), 0x00027000);
    G::copy(buf, ylds + stage, yoff, 4 * G::YROWS * (int)ldy * 2);
  };
  const Chunk8 yk(n0 + 8 * yc, n);
  cm_i32x4 yv[FEED == COPY ? 1 : G::YCOPIES];
  auto load_y = [&](uint32_t m) {
#pragma unroll
    for (int j = 0; j < G::YCOPIES; j++) {
      const uint16_t* row = dy + min(m + (uint32_t)(yr + j * 4 * G::YROWS), me - 1) * ldy;
      yv[FEED == COPY ? 0 : j] = FEED == SHORT ? short_row(row, n0 + 8 * yc, n) : yk.load(row);
    }
  };
  auto store_y = [&](uint32_t m, int stage) {
#pragma unroll
    for (int j = 0; j < G::YCOPIES; j++) {
      cm_i32x4 v = yv[FEED == COPY ? 0 : j];
      if constexpr (FEED == MOVE) v = yk.place(v);
      if (m + yr + j * 4 * G::YROWS >= me) v = cm_i32x4{0, 0, 0, 0};
      *reinterpret_cast<cm_i32x4*>(smem + stage + (yr + j * 4 * G::YROWS) * G::ROW + yp * 16) = v;
    }
  };

  // x: a thread's chunks of 16 codes, one of each NT * 16 / T rows.
  constexpr int XR = NT * 16 / G::T;
  const int xr = t / (G::T / 16), xk = k0 + 16 * (t % (G::T / 16)), xb = min(xk / CB, x.nb - 1);
  const uint32_t xoff = (uint32_t)xr * (uint32_t)x.ld + (xk < x.cols ? xk : 0);  // (other columns: of no output)
  const uint32_t soff = (uint32_t)xr * (uint32_t)x.nb + xb;
  uint8_t* const xlds = smem + G::TILE + xr * G::ROW + (((t % (G::T / 16)) * 2) ^ ((xr & 3) << 2)) * 16;
  cm_i32x4 xv[G::XCHUNKS];
  uint32_t xs[G::XCHUNKS];
  auto load_x = [&](uint32_t m) {
    const int rows = min((int)(me - m), MS), some = -(int)(rows > 0);
    const uint32_t first = min(m, me - 1);
    const uint32_t bytes = ((uint32_t)max(rows, 1) - 1u) * (uint32_t)x.ld + (((uint32_t)x.cols + 15u) & ~15u);
    const __amdgpu_buffer_rsrc_t codes =
        __builtin_amdgcn_make_buffer_rsrc(x.codes + first * x.ld, 0, (int)(bytes & (uint32_t)some), 0x00027000);
    const __amdgpu_buffer_rsrc_t scales =
        __builtin_amdgcn_make_buffer_rsrc(x.scales + (int64_t)first * x.nb, 0, (max(rows, 0) * x.nb) & some, 0x00027000);
#pragma unroll
    for (int j = 0; j < G::XCHUNKS; j++) {
      xv[j] = __builtin_bit_cast(cm_i32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, xoff, j * XR * (int)x.ld, 0));
      xs[j] = __builtin_amdgcn_raw_buffer_load_b8(scales, soff, j * XR * x.nb, 0);
    }
  };
  auto store_x = [&](int stage) {
#pragma unroll
    for (int j = 0; j < G::XCHUNKS; j++) {
      const float s = scale_value(xs[j]);
      cm_i32x4 w[2];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        w[i >> 1][2 * (i & 1)] = (int)code_pair_bf16<false>((uint32_t)xv[j][i], s);
        w[i >> 1][2 * (i & 1) + 1] = (int)code_pair_bf16<true>((uint32_t)xv[j][i], s);
      }
      cm_i32x4* to = reinterpret_cast<cm_i32x4*>(xlds + stage + j * XR * G::ROW);
      to[0] = w[0];
      to[1] = w[1];
    }
  };

  // Reading: lane l of 16 takes row l / 4 of four, columns 4 (l % 4) on, and gets its own column.
  const int wn = (wave & 1) * 32 * W, wk = (wave >> 1) * 32 * W;
  const int i16 = lane & 15, g = lane >> 4, rr = 8 * (g >> 1) + (i16 >> 2);
  uint32_t yo[W], xo[W];
#pragma unroll
  for (int i = 0; i < W; i++) {
    const uint32_t in = rr * G::ROW + (2 * (g & 1) + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
    yo[i] = in + (((wn / 32 + i) ^ (i16 >> 2)) * 64);
    xo[i] = in + (((wk / 32 + i) ^ (i16 >> 2)) * 64);
  }
  cm_f32x16 acc[W][W];
#pragma unroll
  for (int i = 0; i < W; i++)
#pragma unroll
    for (int j = 0; j < W; j++) acc[i][j] = cm_f32x16{};

  typename G::Frag f0, f1;
  load_x(mb);
  if constexpr (FEED == COPY) {
    copy_y(mb, 0);
  } else {
    load_y(mb);
    store_y(mb, 0);
    load_y(mb + MS);
  }
  store_x(0);
  load_x(mb + MS);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if constexpr (FEED == COPY) {
    copy_y(mb + MS, G::STAGE);
  } else {
    store_y(mb + MS, G::STAGE);
    load_y(mb + 2 * MS);
  }
  store_x(G::STAGE);
  load_x(mb + 2 * MS);
  G::read(f0, smem, yo, xo, 0);
  uint32_t stage = 0;
  for (uint32_t m = mb; m < me; m += MS, stage ^= G::STAGE) {
    G::read(f1, smem, yo, xo, stage + 32 * G::ROW);
    G::multiply(acc, f0);
    G::template interleave<2>();
    __builtin_amdgcn_sched_barrier(0);
    // This wave's reads of the step are done and its part of the next step's tiles is in LDS; after
    // the barrier that holds for every wave.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    G::read(f0, smem, yo, xo, stage ^ G::STAGE);
    if constexpr (FEED == COPY) copy_y(m + 2 * MS, (int)stage);
    else store_y(m + 2 * MS, (int)stage);
    store_x((int)stage);
    if constexpr (FEED != COPY) load_y(m + 3 * MS);
    load_x(m + 3 * MS);
    G::multiply(acc, f1);
    G::template interleave<2>();
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy into LDS is under way when the workgroup ends

  // D's rows are k and its columns n: a lane holds four neighbouring k of one n.  They leave through LDS
  // (half of each wave's rows at a time where all do not fit), so that whole rows of the tile are written;
  // chunks are exchanged by the row against bank conflicts.  100 x 4096 x 4096: 25.3 us by single values
  // straight from the registers, 19.0 so; rows of 8393 gradients, not 16 bytes apart: 183 and 142 us.
  constexpr int PASSES = 2 * G::STAGE >= G::T * G::T * 4 ? 1 : 2, PF = W / PASSES, PROWS = G::T / PASSES;
  constexpr int OROW = G::T * 4, RC = G::T / 4;  // bytes and chunks of a row
  static_assert(PROWS * OROW <= 2 * G::STAGE && W % PASSES == 0, "a pass fits the stages");
  const int r = lane & 31, h = lane >> 5;
  const int64_t out = (int64_t)blockIdx.y * part_stride;
#pragma unroll
  for (int p = 0; p < PASSES; p++) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PF; i++)
#pragma unroll
      for (int j = 0; j < W; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const cm_f32x16& d = acc[PF * p + i][j];
          const int row = (wave & 1) * 32 * PF + 32 * i + r, k4 = (wk + 32 * j + 8 * q + 4 * h) >> 2;
          *reinterpret_cast<cm_f32x4*>(smem + row * OROW + ((k4 ^ r) * 16)) = cm_f32x4{d[4 * q], d[4 * q + 1], d[4 * q + 2], d[4 * q + 3]};
        }
    __syncthreads();
#pragma unroll 4
    for (int c = t; c < PROWS * RC; c += NT) {
      const int row = c / RC, k4 = c % RC, k = k0 + 4 * k4;
      const cm_f32x4 v = *reinterpret_cast<const cm_f32x4*>(smem + row * OROW + ((k4 ^ (row & 31)) * 16));
      // rows of the waves lie W blocks apart
      const int nn = n0 + row / (32 * PF) * (32 * W) + p * 32 * PF + row % (32 * PF);
      if (nn < n) put4<F32>(dw, out + nn * ldw + k, v, x.cols - k, add);
    }
  }
}

// dw and db from the sums over parts, in the order of the parts (db's lie behind dw's).
template <bool F32>
__global__ __launch_bounds__(NT) void az_join_parts(const float* __restrict__ parts, int count, int n, int cols,
                                                    void* __restrict__ dw, int64_t ldw, float* __restrict__ db, int add) {
  const int64_t total = (int64_t)n * cols, all = total + (db ? n : 0);
  for (int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x; i < all; i += (int64_t)gridDim.x * NT) {
    const bool weight = i < total;
    const float* from = weight ? parts + i : parts + count * total + (i - total);
    const int64_t step = weight ? total : n;
    float v = 0.0f;
    for (int p = 0; p < count; p++) v += from[p * step];
    if (weight) {
      const int64_t r = i / cols;
      put<F32>(dw, r * ldw + (i - r * cols), v, add);
    } else {
      put<true>(db, i - total, v, add);
    }
  }
}

// How a gradient is cut: tiles of 64 W, and `parts` parts of the rows.
struct Cut {
  int w, parts, part_rows;
};

// The cut with the least estimated time, in microseconds.  A 64-row step takes a workgroup 0.72 (W = 2)
// or 1.48 (W = 4) alone on a compute unit, bound by the step's own chain, 1.0 with two workgroups there
// (W = 2) and 1.86 with every compute unit busy (W = 4), as measured.  Parts cost their way through
// memory and a second launch.  Measured, chosen against others: 16384 x 512 x 512 in 16 parts of small
// tiles 27 (32 parts 32, large tiles 44); 16384 x 4096 x 4096 in one part of large tiles 475; 16384 x
// 1024 x 1024 in 8 parts of small tiles 56 (16 of large ones 57).
Cut choose_cut(int64_t rows, int64_t n, int64_t cols) {
  const int64_t steps = rows > 0 ? (rows + MS - 1) / MS : 1;
  const double write = 1.0 / 4.5e6, outputs = (double)n * (double)cols;  // microseconds a byte
  Cut best = {2, 1, (int)(steps * MS)};
  double least = 0;
  for (int w = n < 8 ? 2 : 4; w >= 2; w -= 2) {  // (rows of fewer than eight are read by the small tile alone)
    const int64_t t = 64 * w, tiles = ((n + t - 1) / t) * ((cols + t - 1) / t);
    for (int64_t parts = 1; parts <= 64 && (parts == 1 || 2 * parts <= steps); parts *= 2) {
      const int64_t per = (steps + parts - 1) / parts, groups = tiles * parts, slots = w == 4 ? 256 : 512;
      if (per * MS > 1 << 30) continue;  // (a part's own rows are counted in an int, with some to spare)
      const double step = w == 4 ? (groups <= 128 ? 1.48 : 1.86) : (groups <= 256 ? 0.72 : 1.0);
      double cost = (double)((groups + slots - 1) / slots) * ((double)per * step + 3.0) + outputs * 4 * write;
      if (parts > 1) cost += 3.5 + (double)parts * outputs * 8 * write;
      if (least == 0 || cost < least) {
        least = cost;
        best = {w, (int)((steps + per - 1) / per), (int)(per * MS)};
      }
    }
  }
  return best;
}

template <int W, bool F32, int FEED>
int launch(const uint16_t* dy, int64_t ldy, int n, const CodeView& x, void* dw, int64_t ldw, float* db, int add, const Cut& cut,
           int64_t part_stride, hipStream_t s) {
  using G = Grad<W>;
  constexpr int LDS = 2 * G::STAGE;
  const int bias = db ? (int)(((int64_t)n + 63) / 64) : 0;
  const int64_t groups = bias + ((int64_t)n + G::T - 1) / G::T * ((x.cols + G::T - 1) / G::T);
  if (!grid_fits(groups, NT)) return AZ_ERR_UNSUPPORTED;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(az_weight_grad<W, F32, FEED>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (e != hipSuccess) return AZ_ERR_DEVICE;
  hipLaunchKernelGGL((az_weight_grad<W, F32, FEED>), dim3((unsigned)groups, (unsigned)cut.parts), dim3(NT), LDS, s, dy, ldy, n, x,
                     dw, ldw, db, bias, add, cut.part_rows, part_stride);
  return AZ_OK;
}

template <int W, bool F32>
int launch_feed(int feed, const uint16_t* dy, int64_t ldy, int n, const CodeView& x, void* dw, int64_t ldw, float* db, int add,
                const Cut& cut, int64_t part_stride, hipStream_t s) {
  if (feed == COPY) return launch<W, F32, COPY>(dy, ldy, n, x, dw, ldw, db, add, cut, part_stride, s);
  if constexpr (W == 2) {
    if (feed == SHORT) return launch<W, F32, SHORT>(dy, ldy, n, x, dw, ldw, db, add, cut, part_stride, s);
  }
  return launch<W, F32, MOVE>(dy, ldy, n, x, dw, ldw, db, add, cut, part_stride, s);
}

}  // namespace

extern "C" size_t az_codes_weight_grad_workspace(int64_t rows, int32_t n, int64_t cols) {
  if (rows <= 0 || n <= 0 || cols <= 0 || !code_sizes(rows, cols)) return 0;
  const Cut cut = choose_cut(rows, n, cols);
  return cut.parts > 1 ? (size_t)cut.parts * (size_t)n * ((size_t)cols + 1) * sizeof(float) : 0;
}

extern "C" int az_codes_weight_grad(const void* dy, int64_t ld_dy, int32_t n, const az_code_matrix* x, void* dw,
                                    int32_t dtype, int64_t ld_dw, float* db, int32_t accumulate, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  static const char who[] = "az_codes_weight_grad";
  int st = code_check(x, who);
  if (st != AZ_OK) return st;
  if (x->scale_rows != 1) return code_fail(AZ_ERR_INVALID_ARG, who, "x needs scale_rows 1");
  if (x->ld >= (1 << 25)) return code_fail(AZ_ERR_UNSUPPORTED, who, "rows of x of 2^25 bytes or more");  // 64 rows in 32-bit offsets
  if (n < 0) return code_fail(AZ_ERR_INVALID_ARG, who, "n < 0");
  if (n == 0) return AZ_OK;
  if ((st = dense_check(dw, dtype, ld_dw, x->cols, who)) != AZ_OK) return st;
  if (x->rows > 0 && (st = dense_check(dy, AZ_BF16, ld_dy, n, who)) != AZ_OK) return st;
  if ((uintptr_t)db & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "db must be 4-byte aligned");
  const size_t need = az_codes_weight_grad_workspace(x->rows, n, x->cols);
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if ((uintptr_t)workspace & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const CodeView v = code_view(*x);
  const Cut cut = choose_cut(x->rows, n, x->cols);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint16_t* y = static_cast<const uint16_t*>(dy);
  // straight into LDS: whole 16-byte chunks, and a step's offsets below 2^31 (no rows: nothing is read)
  const int feed = x->rows == 0 || (rows_aligned16(dy, ld_dy, 2) && ld_dy < (1 << 23)) ? COPY : n >= 8 ? MOVE : SHORT;
  const int add = accumulate != 0;
  (void)hipGetLastError();
  const bool direct = cut.parts == 1;
  void* to = direct ? dw : workspace;
  const int64_t ld = direct ? ld_dw : x->cols, stride = direct ? 0 : (int64_t)n * x->cols;
  const int add_here = direct ? add : 0;
  float* bias = !db || direct ? db : static_cast<float*>(workspace) + (int64_t)cut.parts * n * x->cols;
  if (dtype == AZ_F32 || !direct)
    st = cut.w == 4 ? launch_feed<4, true>(feed, y, ld_dy, n, v, to, ld, bias, add_here, cut, stride, s)
                    : launch_feed<2, true>(feed, y, ld_dy, n, v, to, ld, bias, add_here, cut, stride, s);
  else
    st = cut.w == 4 ? launch_feed<4, false>(feed, y, ld_dy, n, v, to, ld, bias, add_here, cut, stride, s)
                    : launch_feed<2, false>(feed, y, ld_dy, n, v, to, ld, bias, add_here, cut, stride, s);
  if ((st = launched(who, st)) != AZ_OK) return st;
  if (!direct) {
    const int64_t groups = ((int64_t)n * x->cols + NT - 1) / NT;
    const dim3 g((unsigned)(groups < 8192 ? groups : 8192));
    if (dtype == AZ_F32)
      hipLaunchKernelGGL((az_join_parts<true>), g, dim3(NT), 0, s, static_cast<const float*>(workspace), cut.parts, n, (int)x->cols, dw, ld_dw, db, add);
    else
      hipLaunchKernelGGL((az_join_parts<false>), g, dim3(NT), 0, s, static_cast<const float*>(workspace), cut.parts, n, (int)x->cols, dw, ld_dw, db, add);
  }
  return launch_status(who);
}
