// The 1x1 projection of rows in 8 bits (e4m3): y[n, o] = x_scale[n] w_scale[o] sum_c x8[n, c] w8[o, c].
//
// What 8 bits save here is memory; the products run on the fp16 matrix instructions, at the rate that 16x16x32 has for e4m3 as well.  The e4m3
// form was measured first: its sums keep some 14 bits of their terms' magnitudes (a million sums of 32 normal products: errors up to 2^-13.5 of
// sum |x w|, where fp16 operands, which hold every e4m3 value, leave exact products and fp32 sums, 2^-24.4).  A lane's 16 bytes of a row make two operands, the low and the
// high eight contraction slots, so both sides are read 16 bytes a lane in memory order.
#include "msla_device.h"
#include "msla_sequence_kernels.h"

namespace msla {
namespace {

constexpr int kTileK = 128;         // bytes of the contraction a stage

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// sixteen e4m3 values as two operands of fp16 (which has every e4m3 value)
struct Pair { f16x8 v[2]; };
__device__ __forceinline__ Pair widen(u32x4 b) {
    Pair p;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b[j], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b[j], 1.0f, true);
        p.v[j / 2][4 * (j % 2)] = lo[0];
        p.v[j / 2][4 * (j % 2) + 1] = lo[1];
        p.v[j / 2][4 * (j % 2) + 2] = hi[0];
        p.v[j / 2][4 * (j % 2) + 3] = hi[1];
    }
    return p;
}

__device__ __forceinline__ f32x4 mma8(f32x4 c, const Pair& a, const Pair& b) {
    c = Traits<_Float16>::mma_vec(c, a.v[0], b.v[0]);
    return Traits<_Float16>::mma_vec(c, a.v[1], b.v[1]);
}

template <class T>
__device__ __forceinline__ void store8(T* p, const f32x4& a, const f32x4& b) {
    if constexpr (sizeof(T) == 2) {
        typename Traits<T>::Vec v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] = Traits<T>::from_f32(a[r]);
            v[4 + r] = Traits<T>::from_f32(b[r]);
        }
        *(typename Traits<T>::Vec*)p = v;
    } else {
        *(f32x4*)p = a;
        *(f32x4*)(p + 4) = b;
    }
}

// A workgroup has 128 rows x 128 outputs, a wave 64 x 64.  Tiles lie in LDS as rows of 128 bytes whose 16-byte pieces are XORed with the
// row's number modulo 8, which gives the eight rows that a read serves together all banks.  Outputs are the rows of the matrix
// instructions, dealt to pairs of blocks so that a lane ends up with eight neighbours of a row of y.
// 4096 rows, 4096 -> 8192: 250 us (after some 80 launches in a row; 300 for the first ones behind an idle GPU), 1.1 PFLOP/s of the 1.4 that a large
// bf16 product reaches: bound by issue, the conversions of eight operands for sixteen products of two instructions.  256 x 256 tiles: 8% less here, more where the grid is small.
template <class T>
__global__ void __launch_bounds__(256, 2) linear_quantized_kernel(const unsigned char* x8, const float* x_scale, const unsigned char* w8,
                                                                  const float* w_scale, T* y, int64_t rows, int c_in, int c_out, int tiles_o) {
    constexpr int kM = 128, kN = 128, kPieces = (kM + kN) * kTileK / 16 / 256;
    __shared__ __align__(16) char lds[2][(kM + kN) * kTileK];
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_o) * kM;
    const int o0 = blockIdx.x % tiles_o * kN;
    const int wave = threadIdx.x >> 6, lane = lane_id(), x = lane & 15, q = lane >> 4;
    const int wn = wave / 2 * 64, wo = wave % 2 * 64;
    u32x4 hold[kPieces];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = threadIdx.x + i * 256, row = p / 8, c = k0 + p % 8 * 16;
            hold[i] = u32x4{0, 0, 0, 0};
            if (row < kM) {
                if (n0 + row < rows && c < c_in) hold[i] = *(const u32x4*)(x8 + (n0 + row) * c_in + c);
            } else {
                if (o0 + row - kM < c_out && c < c_in) hold[i] = *(const u32x4*)(w8 + (int64_t)(o0 + row - kM) * c_in + c);
            }
        }
    };
    auto park = [&](char* at) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = threadIdx.x + i * 256, row = p / 8;
            *(u32x4*)(at + row * kTileK + ((p % 8) ^ (row & 7)) * 16) = hold[i];
        }
    };
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    const int stages = (c_in + kTileK - 1) / kTileK;
    load(0);
    for (int s = 0; s < stages; ++s) {
        char* at = lds[s & 1];
        park(at);
        __syncthreads();
        if (s + 1 < stages) load((s + 1) * kTileK);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Pair a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ro = kM + wo + 32 * (i / 2) + 8 * (x >> 2) + 4 * (i & 1) + (x & 3), rn = wn + 16 * i + x;
                a[i] = widen(*(const u32x4*)(at + ro * kTileK + ((4 * h + q) ^ (ro & 7)) * 16));
                b[i] = widen(*(const u32x4*)(at + rn * kTileK + ((4 * h + q) ^ (rn & 7)) * 16));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mma8(acc[i][j], a[i], b[j]);
        }
        // (one barrier a stage: the buffer that the next stage fills was last read before this stage's barrier)
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + wn + 16 * j + x;
        if (n >= rows) continue;
        const float sx = x_scale[n];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int o = o0 + wo + 32 * p + 8 * q;
            if (o >= c_out) continue;
            f32x4 lo = acc[2 * p][j], hi = acc[2 * p + 1][j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                lo[r] *= sx * w_scale[o + r];
                hi[r] *= sx * w_scale[o + 4 + r];
            }
            store8<T>(y + n * c_out + o, lo, hi);
        }
    }
}

// Which of the two: by rounds of their workgroups over the 256 compute units.  By measurement at 512 .. 128000 outputs a round takes, a channel of the
// contraction, 1.0, 1.45, 1.95 or 2.7 ns here (up to 16, 32, 48, 64 rows, 16 outputs) and 9.8 ns there (128 rows, 128 outputs, one workgroup to a
// unit).  us here against there, 4096 channels: into 4096 outputs 64 rows 13 against 43, 192 rows 34 against 43, 256 rows 44 against 43; into 16000
// 48 rows 32 against 43; into 32000 16 rows 33 against 42, 17 rows 36 against 42 (taken for 45), 32 rows 45 against 43, 48 rows 60 against 44; into
// 128000 16 rows 124 against 135, 48 rows 248 against 140.
bool rows_kernel_wins(int64_t rows, int c_out) {
    const int64_t here = ((rows + 63) / 64 * (c_out / 16) + 255) / 256, there = ((rows + 127) / 128 * ((c_out + 127) / 128) + 255) / 256;
    return here * (rows <= 16 ? 100 : (rows <= 32 ? 145 : (rows <= 48 ? 195 : 270))) < there * 980;
}

// Few rows: the weights are read once and that is what there is to do, so a workgroup has 16 outputs, its eight waves take 128 bytes of the
// contraction each in turn, and their sums meet in LDS.  Up to 64 rows a workgroup (BLOCKS of 16), which come out of L2.
// 48 rows, 4096 -> 4096: 10 us, 17 MB at 1.7 TB/s: the rows come out of L2 to each of 256 workgroups, which is three times the weights' bytes.
template <class T, int BLOCKS>
__global__ void __launch_bounds__(512) linear_quantized_rows_kernel(const unsigned char* x8, const float* x_scale, const unsigned char* w8,
                                                                    const float* w_scale, T* y, int64_t rows, int c_in, int c_out) {
    constexpr int kWaves = 8;
    __shared__ float sums[kWaves][BLOCKS][16][17];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), x = lane & 15, q = lane >> 4;
    const int tiles_o = c_out / 16, o0 = blockIdx.x % tiles_o * 16;
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_o) * (16 * BLOCKS);
    const unsigned char* wp = w8 + (int64_t)(o0 + x) * c_in + 16 * q;
    const unsigned char* xp[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) xp[b] = x8 + min(n0 + 16 * b + x, rows - 1) * c_in + 16 * q;     // (rows behind the last: not stored)
    f32x4 acc[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) acc[b] = f32x4{0, 0, 0, 0};
    struct Stage { u32x4 w[2], x[BLOCKS][2]; };
    auto load = [&](Stage& s, int k0) {
        if (k0 + kTileK <= c_in) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s.w[h] = *(const u32x4*)(wp + k0 + 64 * h);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) s.x[b][h] = *(const u32x4*)(xp[b] + k0 + 64 * h);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = k0 + 64 * h + 16 * q < c_in;
                s.w[h] = u32x4{0, 0, 0, 0};
                if (in) s.w[h] = *(const u32x4*)(wp + k0 + 64 * h);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    s.x[b][h] = u32x4{0, 0, 0, 0};
                    if (in) s.x[b][h] = *(const u32x4*)(xp[b] + k0 + 64 * h);
                }
            }
        }
    };
    auto multiply = [&](const Stage& s) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Pair w = widen(s.w[h]);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) acc[b] = mma8(acc[b], w, widen(s.x[b][h]));
        }
    };
    constexpr int kStride = kWaves * kTileK;
    Stage s0, s1;
    int k = wave * kTileK;
    if (k < c_in) load(s0, k);
    for (; k < c_in; k += 2 * kStride) {
        if (k + kStride < c_in) load(s1, k + kStride);
        multiply(s0);
        if (k + 2 * kStride < c_in) load(s0, k + 2 * kStride);
        if (k + kStride < c_in) multiply(s1);
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) sums[wave][b][x][4 * q + r] = acc[b][r];
    __syncthreads();
    for (int e = threadIdx.x; e < BLOCKS * 256; e += 512) {
        const int n = e / 16, o = e % 16;
        if (n0 + n >= rows) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sums[w][n / 16][n % 16][o];
        y[(n0 + n) * c_out + o0 + o] = Traits<T>::from_f32(v * (x_scale[n0 + n] * w_scale[o0 + o]));
    }
}

template <class T>
hipError_t linear_of(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in, int c_out,
                     hipStream_t stream) {
    // (a launch has fewer than 2^32 threads: more rows than these, 128 at the most channels, go in several)
    const int64_t most = (((int64_t)1 << 26) / (c_out / 16) + 1) / 128 * 128 + 128;
    const unsigned char* wp = (const unsigned char*)w8;
    for (int64_t from = 0; from < rows; from += most) {
        const int64_t n = rows - from < most ? rows - from : most;
        const unsigned char* xp = (const unsigned char*)x8 + from * c_in;
        T* yp = (T*)y + from * c_out;
        const float* xs = x_scale + from;
        if (rows_kernel_wins(n, c_out)) {
            const dim3 grid((unsigned)((n + 63) / 64 * (c_out / 16))), threads(512);
            if (n <= 16) hipLaunchKernelGGL((linear_quantized_rows_kernel<T, 1>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
            else if (n <= 32) hipLaunchKernelGGL((linear_quantized_rows_kernel<T, 2>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
            else if (n <= 48) hipLaunchKernelGGL((linear_quantized_rows_kernel<T, 3>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
            else hipLaunchKernelGGL((linear_quantized_rows_kernel<T, 4>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
        } else {
            const int tiles_o = (c_out + 127) / 128;
            hipLaunchKernelGGL((linear_quantized_kernel<T>), dim3((unsigned)((n + 127) / 128 * tiles_o)), dim3(256), 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out, tiles_o);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_linear_quantized(int dt, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows,
                                   int c_in, int c_out, hipStream_t stream) {
    switch (dt) {
        case 0: return linear_of<float>(x8, x_scale, w8, w_scale, y, rows, c_in, c_out, stream);
        case 1: return linear_of<_Float16>(x8, x_scale, w8, w_scale, y, rows, c_in, c_out, stream);
        case 2: return linear_of<__bf16>(x8, x_scale, w8, w_scale, y, rows, c_in, c_out, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace msla
