// The 1x1 projection of rows in 8-bit integers: y[n, o] = x_scale[n] w_scale[o] sum_c x8[n, c] w8[o, c], on the 8-bit integer matrix instructions, whose
// sums are exact in 32 bits (131056 products of -128 and -128 stay below 2^31).
#include "msla_device.h"
#include "msla_layer_kernels.h"

namespace msla {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kTileK = 128;         // bytes of the contraction a stage

__device__ __forceinline__ i32x4 mma(i32x4 c, i32x4 a, i32x4 b) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// A workgroup has 128 rows x 128 outputs, a wave 64 x 64.  Tiles lie in LDS as rows of 128 bytes whose 16-byte pieces are XORed with the
// row's number modulo 8, which gives the eight rows that a read serves together all banks.  Outputs are the rows of the matrix
// instructions, dealt to pairs of blocks so that a lane ends up with eight neighbours of a row of y.
template <class T>
__global__ void __launch_bounds__(256, 2) linear_integer_kernel(const char* x8, const float* x_scale, const char* w8, const float* w_scale, T* y,
                                                                int64_t rows, int c_in, int c_out, int tiles_o) {
    constexpr int kM = 128, kN = 128, kPieces = (kM + kN) * kTileK / 16 / 256;
    __shared__ __align__(16) char lds[2][(kM + kN) * kTileK];
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_o) * kM;
    const int o0 = blockIdx.x % tiles_o * kN;
    const int wave = threadIdx.x >> 6, lane = lane_id(), x = lane & 15, q = lane >> 4;
    const int wn = wave / 2 * 64, wo = wave % 2 * 64;
    i32x4 hold[kPieces];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = threadIdx.x + i * 256, row = p / 8, c = k0 + p % 8 * 16;
            hold[i] = i32x4{0, 0, 0, 0};
            if (row < kM) {
                if (n0 + row < rows && c < c_in) hold[i] = *(const i32x4*)(x8 + (n0 + row) * c_in + c);
            } else {
                if (o0 + row - kM < c_out && c < c_in) hold[i] = *(const i32x4*)(w8 + (int64_t)(o0 + row - kM) * c_in + c);
            }
        }
    };
    auto park = [&](char* at) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int p = threadIdx.x + i * 256, row = p / 8;
            *(i32x4*)(at + row * kTileK + ((p % 8) ^ (row & 7)) * 16) = hold[i];
        }
    };
    i32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    const int stages = (c_in + kTileK - 1) / kTileK;
    load(0);
    for (int s = 0; s < stages; ++s) {
        char* at = lds[s & 1];
        park(at);
        __syncthreads();
        if (s + 1 < stages) load((s + 1) * kTileK);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int ro = kM + wo + 32 * (i / 2) + 8 * (x >> 2) + 4 * (i & 1) + (x & 3), rn = wn + 16 * i + x;
                a[i] = *(const i32x4*)(at + ro * kTileK + ((4 * h + q) ^ (ro & 7)) * 16);
                b[i] = *(const i32x4*)(at + rn * kTileK + ((4 * h + q) ^ (rn & 7)) * 16);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mma(acc[i][j], a[i], b[j]);
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
            T out[8];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                out[r] = Traits<T>::from_f32((float)acc[2 * p][j][r] * (sx * w_scale[o + r]));
                out[4 + r] = Traits<T>::from_f32((float)acc[2 * p + 1][j][r] * (sx * w_scale[o + 4 + r]));
            }
            __builtin_memcpy(__builtin_assume_aligned(y + n * c_out + o, 16), out, 8 * sizeof(T));
        }
    }
}

// Few rows: the weights are read once and that is what there is to do, so a workgroup has 16 outputs, its eight waves take 128 bytes of the
// contraction each in turn, and their sums meet in LDS.  Up to 64 rows a workgroup (BLOCKS of 16), which come out of L2.
template <class T, int BLOCKS>
__global__ void __launch_bounds__(512) linear_integer_rows_kernel(const char* x8, const float* x_scale, const char* w8, const float* w_scale, T* y,
                                                                  int64_t rows, int c_in, int c_out) {
    constexpr int kWaves = 8;
    __shared__ int sums[kWaves][BLOCKS][16][17];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), x = lane & 15, q = lane >> 4;
    const int tiles_o = c_out / 16, o0 = blockIdx.x % tiles_o * 16;
    const int64_t n0 = (int64_t)(blockIdx.x / tiles_o) * (16 * BLOCKS);
    const char* wp = w8 + (int64_t)(o0 + x) * c_in + 16 * q;
    const char* xp[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) xp[b] = x8 + min(n0 + 16 * b + x, rows - 1) * c_in + 16 * q;     // (rows behind the last: not stored)
    i32x4 acc[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) acc[b] = i32x4{0, 0, 0, 0};
    struct Stage { i32x4 w[2], x[BLOCKS][2]; };
    auto load = [&](Stage& s, int k0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool in = k0 + 64 * h + 16 * q < c_in;
            s.w[h] = i32x4{0, 0, 0, 0};
            if (in) s.w[h] = *(const i32x4*)(wp + k0 + 64 * h);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                s.x[b][h] = i32x4{0, 0, 0, 0};
                if (in) s.x[b][h] = *(const i32x4*)(xp[b] + k0 + 64 * h);
            }
        }
    };
    auto multiply = [&](const Stage& s) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) acc[b] = mma(acc[b], s.w[h], s.x[b][h]);
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
        int v = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sums[w][n / 16][n % 16][o];
        y[(n0 + n) * c_out + o0 + o] = Traits<T>::from_f32((float)v * (x_scale[n0 + n] * w_scale[o0 + o]));
    }
}

template <class T>
hipError_t linear_of(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in, int c_out,
                     hipStream_t stream) {
    // (a launch has fewer than 2^32 threads: more rows than these, 128 at the most channels, go in several)
    const int64_t most = (((int64_t)1 << 26) / (c_out / 16) + 1) / 128 * 128 + 128;
    const char* wp = (const char*)w8;
    for (int64_t from = 0; from < rows; from += most) {
        const int64_t n = rows - from < most ? rows - from : most;
        const char* xp = (const char*)x8 + from * c_in;
        T* yp = (T*)y + from * c_out;
        const float* xs = x_scale + from;
        if (n <= 64) {
            const dim3 grid((unsigned)((n + 63) / 64 * (c_out / 16))), threads(512);
            if (n <= 16) hipLaunchKernelGGL((linear_integer_rows_kernel<T, 1>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
            else if (n <= 32) hipLaunchKernelGGL((linear_integer_rows_kernel<T, 2>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
            else if (n <= 48) hipLaunchKernelGGL((linear_integer_rows_kernel<T, 3>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
            else hipLaunchKernelGGL((linear_integer_rows_kernel<T, 4>), grid, threads, 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
        } else {
            const int tiles_o = (c_out + 127) / 128;
            hipLaunchKernelGGL((linear_integer_kernel<T>), dim3((unsigned)((n + 127) / 128 * tiles_o)), dim3(256), 0, stream, xp, xs, wp, w_scale, yp, n, c_in, c_out, tiles_o);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_linear_integer(int dt, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in,
                                 int c_out, hipStream_t stream) {
    switch (dt) {
        case 0: return linear_of<float>(x8, x_scale, w8, w_scale, y, rows, c_in, c_out, stream);
        case 1: return linear_of<_Float16>(x8, x_scale, w8, w_scale, y, rows, c_in, c_out, stream);
        case 2: return linear_of<__bf16>(x8, x_scale, w8, w_scale, y, rows, c_in, c_out, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace msla
