// The 1x1 projection of rows in 8-bit integers: y[n, o] = x_scale[n] w_scale[o] sum_c x8[n, c] w8[o, c], on the 8-bit integer matrix instructions, whose
// sums are exact in 32 bits (131056 products of -128 and -128 stay below 2^31).  4096 rows, 4096 -> 8192: 195 us, 1.4 POP/s of the 2.1 that a large library
// product reaches here (159 with the instruction of 64 slots, below); 48 rows, 4096 -> 4096: 11 us, the rows out of L2 to each of 256 workgroups beside 17 MB of weights.
#include "msla_device.h"
#include "msla_layer_kernels.h"

namespace msla {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
// A lane's 16 bytes of a row are the operands of two instructions, the low and the high eight contraction slots (the one of 64 slots, which has twice the rate, is
// not among those whose wait states the built library is checked for).
template <int HALF>
__device__ __forceinline__ i32x4 mma(i32x4 c, i32x4 a, i32x4 b) {
    typedef long i64x2 __attribute__((ext_vector_type(2)));
    const i64x2 p = __builtin_bit_cast(i64x2, a), q = __builtin_bit_cast(i64x2, b);
    const long row = p[HALF], column = q[HALF];
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(row, column, c, 0, 0, 0);
}

// A workgroup of four waves, two by two, has 32 NB rows x 32 OB outputs, a wave half of each: NB OB products of 16 x 16 for NB + OB operands out of LDS, whose
// bandwidth is what large tiles are for.  A stage is 64 bytes of the contraction.  Tiles lie in LDS as rows of 64 bytes whose 16-byte pieces are XORed
// with what the row's number has by 4 and by 16, which gives the sixteen rows that a read serves together all banks: rows of x follow each other, outputs, the rows of the
// matrix instructions, come in fours, dealt to pairs of blocks so that a lane ends up with eight neighbours of a row of y.
template <class T, int NB, int OB>
__global__ void __launch_bounds__(256, 2) linear_integer_kernel(const char* x8, const float* x_scale, const char* w8, const float* w_scale, T* y,
                                                                int64_t rows, int c_in, int c_out, int tiles_n, int tiles_o) {
    constexpr int kM = 32 * NB, kN = 32 * OB, kStage = 64, kPieces = (kM + kN) * kStage / 16 / 256;
    __shared__ __align__(16) char lds[2][(kM + kN) * kStage];
    // neighbours on an XCD take tiles of kGroup rows of tiles in turn, so that what they read stays in its L2
    constexpr int kGroup = 8;
    const int id = (int)xcd_remap(blockIdx.x, gridDim.x), per_group = kGroup * tiles_o, first_n = id / per_group * kGroup;
    const int in_group = min(kGroup, tiles_n - first_n), at = id % per_group;
    const int64_t n0 = (int64_t)(first_n + at % in_group) * kM;
    const int o0 = at / in_group * kN;
    const int wave = threadIdx.x >> 6, lane = lane_id(), x = lane & 15, q = lane >> 4;
    const int wn = wave / 2 * (kM / 2), wo = wave % 2 * (kN / 2);
    auto swizzle = [](int row) { return (row / 4 + row / 16) % 4 * 16; };
    // a thread's pieces of a stage: rows behind the last one are read from the last one (and not stored), pieces behind the contraction as zeros
    const char* from[kPieces];
    int park_at[kPieces];
    const int piece = threadIdx.x % 4 * 16;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int row = threadIdx.x / 4 + i * 64;
        from[i] = (row < kM ? x8 + min(n0 + row, rows - 1) * c_in : w8 + (int64_t)min(o0 + row - kM, c_out - 1) * c_in) + piece;
        park_at[i] = row * kStage + (piece ^ swizzle(row));
    }
    i32x4 hold[kPieces];
    auto load = [&](int k0) {
        const bool in = k0 + piece < c_in;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            hold[i] = i32x4{0, 0, 0, 0};
            if (in) hold[i] = *(const i32x4*)(from[i] + k0);
        }
    };
    i32x4 acc[OB][NB];
#pragma unroll
    for (int i = 0; i < OB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    int a_at[OB], b_at[NB];
#pragma unroll
    for (int i = 0; i < OB; ++i) {
        const int row = kM + wo + 32 * (i / 2) + 8 * (x >> 2) + 4 * (i & 1) + (x & 3);
        a_at[i] = row * kStage + (16 * q ^ swizzle(row));
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int row = wn + 16 * j + x;
        b_at[j] = row * kStage + (16 * q ^ swizzle(row));
    }
    const int stages = (c_in + kStage - 1) / kStage;
    load(0);
    for (int s = 0; s < stages; ++s) {
        char* tile = lds[s & 1];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) *(i32x4*)(tile + park_at[i]) = hold[i];
        __syncthreads();
        if (s + 1 < stages) load((s + 1) * kStage);
        i32x4 a[OB], b[NB];
#pragma unroll
        for (int i = 0; i < OB; ++i) a[i] = *(const i32x4*)(tile + a_at[i]);
#pragma unroll
        for (int j = 0; j < NB; ++j) b[j] = *(const i32x4*)(tile + b_at[j]);
        __builtin_amdgcn_s_setprio(1);
        // (all low halves first: a sum's two products would wait for each other)
        static_for<0, 2>([&](auto half) {
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < OB; ++i) acc[i][j] = mma<decltype(half)::value>(acc[i][j], a[i], b[j]);
        });
        __builtin_amdgcn_s_setprio(0);
        // (one barrier a stage: the buffer that the next stage fills was last read before this stage's barrier)
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int64_t n = n0 + wn + 16 * j + x;
        if (n >= rows) continue;
        const float sx = x_scale[n];
#pragma unroll
        for (int p = 0; p < OB / 2; ++p) {
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
    constexpr int kWaves = 8, kTileK = 128;
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
            for (int b = 0; b < BLOCKS; ++b) acc[b] = mma<1>(mma<0>(acc[b], s.w[h], s.x[b][h]), s.w[h], s.x[b][h]);
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

// Which kernel: by rounds of its workgroups over the 256 compute units, each of which takes so many ns a channel of the contraction, and no call less than
// `least`.  Measured at 4096 channels, us with `rows` of 16 / 32 / 48 / 64, and with tiles of 64 x 64, 64 x 128, 128 x 128 (256 x 128 gains nowhere: 216 where these take
// 210): 16 rows into 4096 outputs 6.3 / 6.8 / 7.4 / 7.9, 21, 29, 38; 96 rows 24 / 18.8 / 17.4 / 18.6, 21, 29, 40; 128 rows 31 / 24 / 23 / 21, 21.6, 30, 40; 512 rows
// 114 / 87 / 79 / 74, 26.8, 33, 42; 1024 rows 226 / 171 / 154 / 144, 44, 42, 44; 2048 rows -, 94, 73, 64; 4096 rows into 8192 -, 338, 265, 210; 64 rows into 16000
// 60 / 46 / 50 / 40, 28.6, 35, 42.
struct Kind { int rows, outputs; float round, least; };
constexpr int kKindCount = 7;
constexpr Kind kKinds[kKindCount] = {{16, 16, 0.95f, 1.54f}, {32, 16, 1.44f, 1.66f}, {48, 16, 1.86f, 2.1f}, {64, 16, 2.44f, 2.6f},
                                     {64, 64, 2.7f, 5.2f}, {64, 128, 4.4f, 7.1f}, {128, 128, 6.4f, 9.7f}};
int kind_of(int64_t rows, int c_out) {
    int best = 0;
    float least = 0.0f;
    for (int k = 0; k < kKindCount; ++k) {
        const Kind& kind = kKinds[k];
        const int64_t groups = (rows + kind.rows - 1) / kind.rows * ((c_out + kind.outputs - 1) / kind.outputs), rounds = (groups + 255) / 256;
        const float all = (float)rounds * kind.round, cost = all > kind.least ? all : kind.least;
        if (k == 0 || cost < least) best = k, least = cost;
    }
    return best;
}

template <class T>
hipError_t linear_of(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in, int c_out,
                     hipStream_t stream) {
    // (a launch has fewer than 2^32 threads: more rows than these, 256 at the most channels, go in several)
    const int64_t most = (((int64_t)1 << 26) / (c_out / 16) + 1) / 256 * 256 + 256;
    const char* wp = (const char*)w8;
    for (int64_t from = 0; from < rows; from += most) {
        const int64_t n = rows - from < most ? rows - from : most;
        const char* xp = (const char*)x8 + from * c_in;
        T* yp = (T*)y + from * c_out;
        const float* xs = x_scale + from;
        auto by_rows = [&](auto blocks) {
            constexpr int kBlocks = decltype(blocks)::value;
            hipLaunchKernelGGL((linear_integer_rows_kernel<T, kBlocks>), dim3((unsigned)((n + 16 * kBlocks - 1) / (16 * kBlocks) * (c_out / 16))), dim3(512), 0,
                               stream, xp, xs, wp, w_scale, yp, n, c_in, c_out);
        };
        auto by_tiles = [&](auto nb, auto ob) {
            constexpr int kM = 32 * decltype(nb)::value, kN = 32 * decltype(ob)::value;
            const int tiles_n = (int)((n + kM - 1) / kM), tiles_o = (c_out + kN - 1) / kN;
            hipLaunchKernelGGL((linear_integer_kernel<T, decltype(nb)::value, decltype(ob)::value>), dim3((unsigned)tiles_n * (unsigned)tiles_o), dim3(256), 0,
                               stream, xp, xs, wp, w_scale, yp, n, c_in, c_out, tiles_n, tiles_o);
        };
        using std::integral_constant;
        switch (kind_of(n, c_out)) {
            case 0: by_rows(integral_constant<int, 1>{}); break;
            case 1: by_rows(integral_constant<int, 2>{}); break;
            case 2: by_rows(integral_constant<int, 3>{}); break;
            case 3: by_rows(integral_constant<int, 4>{}); break;
            case 4: by_tiles(integral_constant<int, 2>{}, integral_constant<int, 2>{}); break;
            case 5: by_tiles(integral_constant<int, 2>{}, integral_constant<int, 4>{}); break;
            default: by_tiles(integral_constant<int, 4>{}, integral_constant<int, 4>{});
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
