// Rows in 4 bits with a power of two for each 32 values (OCP MXFP4), their values, and the product of two such matrices.
//
// A group's scale byte is the exponent of its largest magnitude less 2 (e2m1's largest power of two is 4), plus 127; its codes
// are the values over that power, to nearest even, at most 6. Every step but that rounding is exact.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lce_gemm16.hpp"
#include "ops_row.hpp"

namespace lce {

constexpr int kMxGroup = 32;

struct MxRowsArgs {
  const void* x;  // rows (quantise)
  void* y;        // rows (dequantise)
  uint8_t *codes, *scales;
  int64_t ld, N;  // the rows' pitch in elements; codes and scales are contiguous
  int H;
};

// TPR threads a row, 8 values each, so that four neighbours share a group. Bound by HBM: 8192 x 4096 in bf16 16.1 us (85 MB, 5.3 TB/s).
template <typename T, int TPR>
__global__ __launch_bounds__(256) void mxfp4_quantize_kernel(const MxRowsArgs a) {
  constexpr int kRows = 256 / TPR, kAhead = 2;
  const int t = threadIdx.x % TPR;
  for (int64_t i = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; i < a.N; i += (int64_t)gridDim.x * kRows) {
    const T* p = (const T*)a.x + i * a.ld;
    for (int c0 = t * kNormVec; c0 < a.H; c0 += kAhead * TPR * kNormVec) {
      RawRow<T> raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        raw[u].clear();
        load_raw<WHOLE>(p + c0 + u * TPR * kNormVec, a.H - c0 - u * TPR * kNormVec, raw[u]);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int c = c0 + u * TPR * kNormVec;
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) top = max(top, __builtin_bit_cast(uint32_t, raw[u].at(e)) & 0x7fffffffu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        const uint32_t e8 = top >> 23;  // 255: an infinity or a NaN
        const uint32_t byte = e8 == 255 ? 255u : e8 > 2 ? e8 - 2 : 0u;
        const float inv = __builtin_bit_cast(float, (254u - (e8 == 255 ? 127u : byte)) << 23);  // 2^(127 - byte), exact
        uint32_t q = 0;
        if (e8 != 255) {
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, raw[u].at(0) * inv, raw[u].at(1) * inv, 1.f, 0);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, raw[u].at(2) * inv, raw[u].at(3) * inv, 1.f, 1);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, raw[u].at(4) * inv, raw[u].at(5) * inv, 1.f, 2);
          q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, raw[u].at(6) * inv, raw[u].at(7) * inv, 1.f, 3);
        }
        if (c < a.H) {
          *(uint32_t*)(a.codes + i * (a.H / 2) + c / 2) = q;
          if (t % 4 == 0) a.scales[i * (a.H / kMxGroup) + c / kMxGroup] = (uint8_t)byte;
        }
      }
    }
  }
}

// 8192 x 4096 in bf16: 19.4 us (85 MB, 4.4 TB/s).
template <typename T, int TPR>
__global__ __launch_bounds__(256) void mxfp4_dequantize_kernel(const MxRowsArgs a) {
  constexpr int kRows = 256 / TPR, kAhead = 2;
  const int t = threadIdx.x % TPR;
  for (int64_t i = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; i < a.N; i += (int64_t)gridDim.x * kRows) {
    for (int c0 = t * kNormVec; c0 < a.H; c0 += kAhead * TPR * kNormVec) {
      uint32_t q[kAhead], byte[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int c = min(c0 + u * TPR * kNormVec, a.H - kNormVec);
        q[u] = *(const uint32_t*)(a.codes + i * (a.H / 2) + c / 2);
        byte[u] = a.scales[i * (a.H / kMxGroup) + c / kMxGroup];
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int c = c0 + u * TPR * kNormVec;
        float y[kNormVec];
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) {
          const uint32_t m = (q[u] >> (4 * e)) & 7u;
          // Twice the magnitude: 0, 1, 2, 3, 4, 6, 8, 12 (a byte each).
          const float v = (float)((0x0c08060403020100ull >> (8 * m)) & 0xffu);
          const float s = __builtin_amdgcn_ldexpf((q[u] >> (4 * e)) & 8u ? -v : v, (int)byte[u] - 128);
          y[e] = byte[u] == 255 ? __builtin_nanf("") : s;
        }
        if (c < a.H) store_row<WHOLE>((T*)a.y + i * a.ld + c, kNormVec, y);
      }
    }
  }
}

// ---- the product ----
//
// out[m][v] = sum_k x[m][k] w[v][k] with v_mfma_scale_f32_16x16x128_f8f6f4: a lane gives 32 values (16 bytes, one group, with
// one scale byte) of row lane % 16. Any order of the groups serves as long as both operands have the same: of 256
// values, lane quarter q takes groups 2q and 2q + 1 in turn, so that what it reads of a row is together.
// W is the first operand: a lane then holds four consecutive v of one m.

struct MxMatmulArgs {
  const uint8_t *x, *x_scales, *w, *w_scales;
  void* out;
  int64_t out_ld;
  int64_t M, V;
  int K;
  int tiles_m, tiles_v;
};

typedef int i32x8 __attribute__((ext_vector_type(8)));

template <int J>
__device__ __forceinline__ f32x4 mx_mfma(const u32x4& w, uint32_t ws, const u32x4& x, uint32_t xs, f32x4 c) {
  const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3]}, b = {(int)x[0], (int)x[1], (int)x[2], (int)x[3]};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, J, (int)ws, J, (int)xs);
}

constexpr int kMxStep = 256, kMxStepBytes = kMxStep / 2, kMxStepGroups = kMxStep / kMxGroup;

// Rows of a matrix from a tile's first one on: what lies past the last row reads as zeros.
struct MxRows {
  __amdgpu_buffer_rsrc_t codes, scales;
};
__device__ __forceinline__ MxRows mx_rows(const uint8_t* codes, const uint8_t* scales, int64_t first, int rows, uint32_t pitch, uint32_t groups) {
  return {make_rsrc((const void*)uniform64((uint64_t)(codes + first * pitch)), __builtin_amdgcn_readfirstlane((uint32_t)rows * pitch)),
          make_rsrc((const void*)uniform64((uint64_t)(scales + first * groups)), __builtin_amdgcn_readfirstlane((uint32_t)rows * groups))};
}

// The scales of a run of steps go through LDS: a wave that loads the 8 bytes of 16 rows that a step needs waits for as many cache
// lines as for the codes (4096 x 128256, one row of x: 64 us, 46 without scales; 64 rows 114 and 79).
constexpr int kMxRunSteps = 32, kMxRunBytes = kMxRunSteps * kMxStepGroups, kMxRunPitch = kMxRunBytes + 16;

// ROWS rows' scales of groups first .. first + bytes - 1 (of `groups` in a row).
template <int ROWS>
struct MxScaleRun {
  static constexpr int kPieces = ROWS * (kMxRunBytes / 8) / 256;  // a thread's, at most
  u32x2 piece[kPieces];
  // Whole steps (bytes % 8 == 0): requested together, stored later. lanes, a power of two, have a row's.
  __device__ __forceinline__ void load(const MxRows& r, uint32_t groups, int first, int bytes, int lanes) {
    const int rows = 256 / lanes, c = (int)threadIdx.x % lanes * 8;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      if (k * rows >= ROWS) break;
      const int row = k * rows + (int)threadIdx.x / lanes;
      const uint32_t at = row < ROWS && c < bytes ? (uint32_t)row * groups + (uint32_t)(first + c) : kOOB;
      piece[k] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r.scales, at, 0, 0));
    }
  }
  __device__ __forceinline__ void store(char* lds, int lanes) {
    const int rows = 256 / lanes, c = (int)threadIdx.x % lanes * 8;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int row = k * rows + (int)threadIdx.x / lanes;
      if (k * rows < ROWS && row < ROWS) *(u32x2*)(lds + row * kMxRunPitch + c) = piece[k];
    }
  }
  // Any number of bytes, 4 at a time and the rest one by one, each within the row: what follows it may be no memory, or
  // a NaN's scale.
  static __device__ __forceinline__ void copy(const MxRows& r, uint32_t groups, int first, int bytes, char* lds) {
    int lanes = 2;  // (a step's eight bytes at least, the last ones zeros)
    while (lanes * 4 < bytes) lanes *= 2;
#pragma unroll 4
    for (int k = threadIdx.x; k < ROWS * lanes; k += 256) {
      const int row = k / lanes, c = k % lanes * 4, left = bytes - c;
      const uint32_t at = (uint32_t)row * groups + (uint32_t)(first + c);
      uint32_t v = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r.scales, left >= 4 ? at : kOOB, 0, 0);
      if (bytes % 4 != 0) {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          v |= (uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r.scales, left > e && left < 4 ? at + e : kOOB, 0, 0) << (8 * e);
      }
      *(uint32_t*)(lds + row * kMxRunPitch + c) = v;
    }
  }
};

// Few rows of x (up to 16 MT): W is read once, straight into registers, and nothing else takes long. A workgroup has 16 NV rows
// of W; its four waves take the steps of K in turn, the next one requested before the current one's products, and add up at
// the end. x comes from L2: 16 NV rows of W for each read of it. Lane quarter q takes groups q and 4 + q of a step's eight.
// Bound by HBM for one row (4096 x 128256: 47 us, 279 MB, 5.9 TB/s), for more by x's way from L2 as well (48 rows 77 us; 48 rows of
// 12288 x 32768 56 us: 3.9 TB/s of W, and 171 MB of L2 hits, mostly x: the waves take different steps, so a workgroup shares nothing of it).
template <typename T, int MT, int NV>
__global__ __launch_bounds__(256, 2) void mxfp4_few_kernel(const MxMatmulArgs a) {
  constexpr int kRowsW = 16 * NV, kRowsX = 16 * MT, kPitch = kRowsW + 4, kWaves = 4, kTiles = NV > MT ? NV : MT;
  constexpr int kScales = (kRowsW + kRowsX) * kMxRunPitch, kSums = kWaves * kRowsX * kPitch * 4;
  __shared__ __attribute__((aligned(16))) char smem[kScales > kSums ? kScales : kSums];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
  const int64_t v0 = (int64_t)blockIdx.x * kRowsW;
  const uint32_t pitch = (uint32_t)a.K / 2, groups = (uint32_t)a.K / kMxGroup;
  const MxRows rw = mx_rows(a.w, a.w_scales, v0, (int)min(a.V - v0, (int64_t)kRowsW), pitch, groups);
  const MxRows rx = mx_rows(a.x, a.x_scales, 0, (int)a.M, pitch, groups);
  uint32_t at[kTiles];  // of both: rows 16 i + lane % 16
#pragma unroll
  for (int i = 0; i < kTiles; ++i) at[i] = (uint32_t)(16 * i + row) * pitch + 16 * quarter;
  f32x4 acc[NV][MT] = {};
  struct Step {
    u32x4 w[NV][2], x[MT][2];
  };
  auto request = [&](int step, Step& b) {
    const uint32_t k = (uint32_t)step * kMxStepBytes;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) b.w[i][h] = load16(rw.codes, at[i] + 64 * h, k);
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) b.x[j][h] = load16(rx.codes, at[j] + 64 * h, k);
    __builtin_amdgcn_sched_barrier(0);  // (the compiler would move the requests down to their use)
  };
  const char* scales_w = smem + row * kMxRunPitch;
  const char* scales_x = scales_w + kRowsW * kMxRunPitch;
  auto multiply = [&](const Step& b, int step) {  // step: of the run
    u32x2 sw[NV], sx[MT];
#pragma unroll
    for (int i = 0; i < NV; ++i) sw[i] = *(const u32x2*)(scales_w + 16 * i * kMxRunPitch + step * kMxStepGroups) >> (uint32_t)(8 * quarter);
#pragma unroll
    for (int j = 0; j < MT; ++j) sx[j] = *(const u32x2*)(scales_x + 16 * j * kMxRunPitch + step * kMxStepGroups) >> (uint32_t)(8 * quarter);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = mx_mfma<0>(b.w[i][h], sw[i][h], b.x[j][h], sx[j][h], acc[i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  const int steps = a.K / kMxStep;  // whole ones
  for (int s0 = 0; s0 * kMxStep < a.K; s0 += kMxRunSteps) {
    const int end = min(steps, s0 + kMxRunSteps), bytes = min(kMxRunBytes, (int)groups - s0 * kMxStepGroups);
    int lanes = 1;
    while (lanes * 8 < bytes) lanes *= 2;
    MxScaleRun<kRowsW> run_w;
    MxScaleRun<kRowsX> run_x;
    const bool pieces = bytes % 8 == 0;
    if (pieces) {
      run_w.load(rw, groups, s0 * kMxStepGroups, bytes, lanes);
      run_x.load(rx, groups, s0 * kMxStepGroups, bytes, lanes);
    }
    int s = s0 + wave;
    Step b0, b1;
    if (s < end) request(s, b0);
    if (s0 > 0) __syncthreads();
    if (pieces) {
      run_w.store(smem, lanes);
      run_x.store(smem + kRowsW * kMxRunPitch, lanes);
    } else {
      MxScaleRun<kRowsW>::copy(rw, groups, s0 * kMxStepGroups, bytes, smem);
      MxScaleRun<kRowsX>::copy(rx, groups, s0 * kMxStepGroups, bytes, smem + kRowsW * kMxRunPitch);
    }
    __syncthreads();
    if (s < end) {
      // (requests past the last step read it again: behind a branch the compiler would wait for all of them)
      for (;;) {
        request(min(s + kWaves, end - 1), b1);
        multiply(b0, s - s0);
        if ((s += kWaves) >= end) break;
        request(min(s + kWaves, end - 1), b0);
        multiply(b1, s - s0);
        if ((s += kWaves) >= end) break;
      }
    }
    // The last, shorter step: groups past the row's end are zeros.
    if (end == steps && steps - s0 < kMxRunSteps && a.K % kMxStep != 0 && wave == steps % kWaves) {
      const int left = a.K % kMxStep / kMxGroup;
      const uint32_t k = (uint32_t)steps * kMxStepBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = quarter + 4 * h < left;
#pragma unroll
        for (int i = 0; i < NV; ++i) b0.w[i][h] = load16(rw.codes, in ? at[i] + 64 * h + k : kOOB);
#pragma unroll
        for (int j = 0; j < MT; ++j) b0.x[j][h] = load16(rx.codes, in ? at[j] + 64 * h + k : kOOB);
      }
      multiply(b0, steps - s0);
    }
  }
  __syncthreads();
  float* sums = (float*)smem;  // [wave][row of x][row of W]
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) *(f32x4*)&sums[(wave * kRowsX + 16 * j + row) * kPitch + 16 * i + 4 * quarter] = acc[i][j];
  __syncthreads();
  constexpr int kRowLanes = kRowsW / 4, kRows = 256 / kRowLanes;  // threads that share a row of the result
#pragma unroll
  for (int k = 0; k < 16 * MT; k += kRows) {
    const int m = k + (int)threadIdx.x / kRowLanes, c = threadIdx.x % kRowLanes * 4;
    if (m >= 16 * MT || m >= a.M) break;
    f32x4 y = *(f32x4*)&sums[m * kPitch + c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) y += *(f32x4*)&sums[(w * kRowsX + m) * kPitch + c];
    T* p = (T*)a.out + m * a.out_ld + v0 + c;
    T q[4] = {from_f32<T>(y[0]), from_f32<T>(y[1]), from_f32<T>(y[2]), from_f32<T>(y[3])};
    if (v0 + c + 4 <= a.V) {
      __builtin_memcpy(p, q, sizeof(q));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v0 + c + e < a.V) p[e] = q[e];
    }
  }
}

// Many rows: a tile of 256 rows of W by BN of x for WAVES waves in two columns, each with 16 x 16 blocks of its part (BN 256: eight
// waves, 64 x 128; four of 128 x 128 read less from LDS but have nothing to run under their waits, 924 us against 733 for
// 2048 x 3584 x 152064; BN 128: four waves, 128 x 64, 89 us against 91 with eight for 128 x 4096 x 128256). A step is 256
// values of K, 128 bytes of a row: whole cache lines, LDS-DMA loads of 8 rows each into one of two slots. The 16-byte
// pieces of LDS row r are permuted by r % 8: a fragment's rows r and r + 8 still share their banks, all others differ (half of a read's 8
// cycles). The scales go through registers, since their rows may begin at any byte. 2048 x 3584 x 152064: 3.0 PFLOP/s, 4096 x 8192 x 32000:
// 3.5. Bound by waiting: the MFMAs are busy 33% of the time and LDS 29% (counters, first shape); a step's loads are one step ahead and
// all waited for, its fragments are all read behind that barrier, and a tile's first loads and its result have nothing beside them.
template <typename T, int BN, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mxfp4_many_kernel(const MxMatmulArgs a) {
  constexpr int kBM = 256, kWaves = WAVES, kWavesV = WAVES / 2, kI = kBM / kWavesV / 16, kJ = BN / 32, kThreads = 64 * WAVES;
  constexpr int kW = kBM * kMxStepBytes, kX = BN * kMxStepBytes, kSw = kBM * kMxStepGroups, kSx = BN * kMxStepGroups;
  constexpr int kSlot = kW + kX + kSw + kSx;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)smem;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
  int tm, tv;
  tile_coords(blockIdx.x, gridDim.x, a.tiles_m, a.tiles_m, tm, tv);
  const int64_t m0 = (int64_t)tm * BN, v0 = (int64_t)tv * kBM;
  const uint32_t pitch = (uint32_t)a.K / 2, groups = (uint32_t)a.K / kMxGroup;
  const int rows_w = (int)min(a.V - v0, (int64_t)kBM), rows_x = (int)min(a.M - m0, (int64_t)BN);
  // Rows past the last are zeros by the descriptors' ranges.
  const auto rsrc_w = make_rsrc((const void*)uniform64((uint64_t)(a.w + v0 * pitch)), __builtin_amdgcn_readfirstlane((uint32_t)rows_w * pitch));
  const auto rsrc_x = make_rsrc((const void*)uniform64((uint64_t)(a.x + m0 * pitch)), __builtin_amdgcn_readfirstlane((uint32_t)rows_x * pitch));
  const int steps = (a.K + kMxStep - 1) / kMxStep;
  const uint32_t piece = (uint32_t)((lane & 7) ^ (lane >> 3)) * 16u, row_off = (uint32_t)(lane >> 3) * pitch;
  auto dma = [&](int step, int slot) {
    const uint32_t k = (uint32_t)step * kMxStepBytes;
    // Pieces past the rows' end are zeros too.
    const bool in = k + piece < pitch;
    char* to = smem + slot * kSlot;
#pragma unroll
    for (int n = 0; n < kBM / 8 / kWaves; ++n) {
      const int b = wave * (kBM / 8 / kWaves) + n;
      dma16(rsrc_w, to + b * 1024, in ? row_off + piece + k + (uint32_t)(8 * b) * pitch : kOOB);
    }
#pragma unroll
    for (int n = 0; n < BN / 8 / kWaves; ++n) {
      const int b = wave * (BN / 8 / kWaves) + n;
      dma16(rsrc_x, to + kW + b * 1024, in ? row_off + piece + k + (uint32_t)(8 * b) * pitch : kOOB);
    }
  };
  // A thread has the scales of one row or two: of W's rows, then of x's.
  constexpr int kScaleRows = (kBM + BN + kThreads - 1) / kThreads;
  const uint8_t* ps[kScaleRows];
#pragma unroll
  for (int k = 0; k < kScaleRows; ++k) {
    const int r = k * kThreads + (int)threadIdx.x;
    ps[k] = r < kBM ? a.w_scales + (v0 + min(r, rows_w - 1)) * groups : a.x_scales + (m0 + min(r - kBM, rows_x - 1)) * groups;
  }
  auto has_scales = [&](int k) { return (k + 1) * kThreads <= kBM + BN || k * kThreads + (int)threadIdx.x < kBM + BN; };
  auto load_scales = [&](int step, uint64_t (&s)[kScaleRows]) {
    const uint32_t g = (uint32_t)step * kMxStepGroups;
#pragma unroll
    for (int k = 0; k < kScaleRows; ++k) {
      s[k] = 0x7f7f7f7f7f7f7f7full;
      if (!has_scales(k) || step >= steps) continue;
      if (g + kMxStepGroups <= groups) {
        __builtin_memcpy(&s[k], ps[k] + g, 8);
      } else {
        for (uint32_t j = g; j < groups; ++j) s[k] = (s[k] & ~(0xffull << (8 * (j - g)))) | (uint64_t)ps[k][j] << (8 * (j - g));
      }
    }
  };
  auto put_scales = [&](int slot, const uint64_t (&s)[kScaleRows]) {
#pragma unroll
    for (int k = 0; k < kScaleRows; ++k)
      if (has_scales(k)) *(uint64_t*)(smem + slot * kSlot + kW + kX + (k * kThreads + threadIdx.x) * 8) = s[k];
  };
  f32x4 acc[kI][kJ] = {};
  constexpr int kRowsV = kBM / kWavesV;  // of a wave
  const int wv = wave % kWavesV, wm = wave / kWavesV;
  // Fragment of block b (16 rows), group pair half j: piece 2 quarter + j of row 16 b + row.
  const uint32_t frag0 = (uint32_t)(row * kMxStepBytes) + (uint32_t)(((2 * quarter) ^ (row & 7)) * 16);
  const uint32_t addr_w = base + (uint32_t)(wv * kRowsV * kMxStepBytes) + frag0;
  const uint32_t addr_x = base + kW + (uint32_t)(wm * (BN / 2) * kMxStepBytes) + frag0;
  const uint32_t addr_sw = base + kW + kX + (uint32_t)((wv * kRowsV + row) * kMxStepGroups + 2 * quarter);
  const uint32_t addr_sx = base + kW + kX + kSw + (uint32_t)((wm * (BN / 2) + row) * kMxStepGroups + 2 * quarter);
  uint64_t next[kScaleRows];
  dma(0, 0);
  load_scales(0, next);
  put_scales(0, next);
  load_scales(1, next);
  for (int t = 0; t < steps; ++t) {
    const uint32_t slot = (uint32_t)(t & 1) * kSlot;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + 1 < steps) {
      dma(t + 1, (t + 1) & 1);
      put_scales((t + 1) & 1, next);
      load_scales(t + 2, next);
    }
    uint32_t sw[kI], sx[kJ];
#pragma unroll
    for (int i = 0; i < kI; ++i) sw[i] = *lds_at<uint16_t>(addr_sw + slot + i * 16 * kMxStepGroups);
#pragma unroll
    for (int j = 0; j < kJ; ++j) sx[j] = *lds_at<uint16_t>(addr_sx + slot + j * 16 * kMxStepGroups);
    u32x4 w[2][kI], x[2][kJ];
    // (the pieces' permutation flips bits 4 to 6; group 2 quarter + 1 is group 2 quarter's bit 4 flipped)
    auto fragments = [&](auto h) {
      constexpr int kH = decltype(h)::value;
#pragma unroll
      for (int i = 0; i < kI; ++i) w[kH][i] = *lds_at<u32x4>(((addr_w + slot) ^ (16u * kH)) + i * 16 * kMxStepBytes);
#pragma unroll
      for (int j = 0; j < kJ; ++j) x[kH][j] = *lds_at<u32x4>(((addr_x + slot) ^ (16u * kH)) + j * 16 * kMxStepBytes);
    };
    auto multiply = [&](auto h) {
      constexpr int kH = decltype(h)::value;
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int i = 0; i < kI; ++i) acc[i][j] = mx_mfma<kH>(w[kH][i], sw[i], x[kH][j], sx[j], acc[i][j]);
    };
    using std::integral_constant;
    fragments(integral_constant<int, 0>{});
    fragments(integral_constant<int, 1>{});
    __builtin_amdgcn_sched_barrier(0);
    multiply(integral_constant<int, 0>{});
    multiply(integral_constant<int, 1>{});
  }
  // Element r of block (i, j): v = 16 i + 4 quarter + r, m = 16 j + row of the wave's part.
#pragma unroll
  for (int j = 0; j < kJ; ++j) {
    const int64_t m = m0 + wm * (BN / 2) + 16 * j + row;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < kI; i += 2) {
        const int64_t v = v0 + wv * kRowsV + 16 * i + 8 * quarter;
        const u32x4 y = regroup16<T>(acc[i][j], acc[i + 1][j]);
        T* p = (T*)a.out + m * a.out_ld + v;
        if (m >= a.M) continue;
        if (v + 8 <= a.V) {
          __builtin_memcpy(p, &y, 16);
        } else {
          T q[8];
          __builtin_memcpy(q, &y, 16);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (v + e < a.V) p[e] = q[e];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        const int64_t v = v0 + wv * kRowsV + 16 * i + 4 * quarter;
        T* p = (T*)a.out + m * a.out_ld + v;
        if (m >= a.M) continue;
        if (v + 4 <= a.V) {
          __builtin_memcpy(p, &acc[i][j], 16);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v + e < a.V) p[e] = acc[i][j][e];
        }
      }
    }
  }
}
template <int BN>
constexpr int mx_many_smem() { return 2 * (256 + BN) * (kMxStepBytes + kMxStepGroups); }

}  // namespace lce
