// Root-mean-square norm of rows with the residual's addition, its gradient, and rows into 8 bits (e4m3 with a scale a row).
//
// Bound by memory: a row is read once, stays in registers as fp32 through the sum of its squares (and, into 8 bits, its largest
// magnitude), and is written once.  16 bytes a lane and access, whatever the row's alignment; where the row's length is no multiple of that, the
// last piece starts early, at the row's end less 16 bytes: what it has in common with the piece before counts once in sums and is stored twice
// with the same values.  LPR lanes share a row: few for short rows, so that a wave holds several, a whole workgroup for long ones.
// 16384 rows of 4096 with a residual in bf16: 95 us (537 MB, 5.6 TB/s); 48 rows of 4096 into 8 bits 5 us; the gradient of 8192 rows of 2051
// 32 us and 4 for d_weight's parts (134 MB, 3.7 TB/s).
#include "msla_device.h"
#include "msla_sequence_kernels.h"
#include "norm_rows.h"

namespace msla {
namespace {

constexpr float kTop8 = 448.0f;     // the largest e4m3 value

template <int VEC>
__device__ __forceinline__ void store_row8(unsigned char* p, int at, int channels, const float (&f)[VEC]) {
    unsigned w[VEC / 4];
#pragma unroll
    for (int e = 0; e < VEC / 4; ++e) {
        int v = 0;
        v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * e], f[4 * e + 1], v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * e + 2], f[4 * e + 3], v, true);
        w[e] = (unsigned)v;
    }
    if (channels >= VEC) {
        __builtin_memcpy(__builtin_assume_aligned(p + at, 1), w, VEC);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < channels) p[e] = (unsigned char)(w[e / 4] >> (8 * (e % 4)));
    }
}

template <class T, int LPR, int PER, bool EIGHT, bool PLAIN>
__global__ void __launch_bounds__(LPR > 256 ? LPR : 256) norm_kernel(const T* x, const T* residual, const T* weight, void* y, float* scale, T* sum,
                                                                     int64_t rows, int channels, float eps) {
    constexpr int kVec = Traits<T>::kVec, kThreads = LPR > 256 ? LPR : 256, kRows = kThreads / LPR;
    __shared__ float room[kThreads / 64];
    const int lane = threadIdx.x % LPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR;
    const bool live = row < rows;
    const int64_t base = (live ? row : 0) * channels;
    float r[PER][kVec];
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const Piece<kVec> pc(lane + i * LPR, channels);
        if (live && pc.live) {
            load_row<T>(x + base, pc.at, channels, r[i]);
            if (residual != nullptr) {
                float f[kVec];
                load_row<T>(residual + base, pc.at, channels, f);
#pragma unroll
                for (int e = 0; e < kVec; ++e) r[i][e] += f[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) r[i][e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) squares += e < pc.skip ? 0.0f : r[i][e] * r[i][e];
    }
    if constexpr (!PLAIN) {
        squares = over_row<LPR>(squares, room, [](float a, float b) { return a + b; });
        // (only now that the whole row has been read: sum may lie on x or residual, and the last piece shares channels with another lane's)
        if (sum != nullptr) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const Piece<kVec> pc(lane + i * LPR, channels);
                if (live && pc.live) store_row<T>(sum + base, pc.at, channels, r[i]);
            }
        }
        const float rstd = 1.0f / sqrtf(squares / (float)channels + eps);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            if (!pc.live) continue;
            float w[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) w[e] = 1.0f;
            if (weight != nullptr) load_row<T>(weight, pc.at, channels, w);
#pragma unroll
            for (int e = 0; e < kVec; ++e) r[i][e] *= rstd * w[e];
        }
    }
    if constexpr (EIGHT) {
        float top = 0.0f;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                top = fmaxf(top, fabsf(r[i][e]));
                odd |= r[i][e] != r[i][e];
            }
        if (odd) top = __builtin_nanf("");
        // (a NaN anywhere makes the row's scale one: fmaxf would drop it)
        top = over_row<LPR>(top, room, [](float a, float b) { return a != a || b != b ? __builtin_nanf("") : fmaxf(a, b); });
        // (rows so small that 448 / top has no fp32 value are lifted first; a row of zeros stays one)
        const float s = top / kTop8, lift = top < 1e-30f ? 0x1p64f : 1.0f, by = top == 0.0f ? 0.0f : kTop8 / (top * lift);
        if (live && lane == 0) scale[row] = s;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            if (!live || !pc.live) continue;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float v = r[i][e] * lift * by;
                r[i][e] = v > kTop8 ? kTop8 : (v < -kTop8 ? -kTop8 : v);
            }
            store_row8<kVec>((unsigned char*)y + base, pc.at, channels, r[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            if (live && pc.live) store_row<T>((T*)y + base, pc.at, channels, r[i]);
        }
    }
}

// A workgroup walks over rows; a lane has the same channels of each, so it sums their part of d_weight in registers.  The next row is on its way
// while this one is reduced.
template <class T, int LPR, int PER>
__global__ void __launch_bounds__(LPR > 256 ? LPR : 256) norm_backward_kernel(const T* sum, const T* weight, const T* d_y, const T* d_sum, T* d_r,
                                                                              float* partials, int64_t rows, int channels, float eps) {
    constexpr int kVec = Traits<T>::kVec, kThreads = LPR > 256 ? LPR : 256, kRows = kThreads / LPR;
    typedef typename Traits<T>::Vec Vec;
    __shared__ f32x2 room[2][kThreads / 64];
    __shared__ float groups[kRows > 1 ? kThreads * PER * kVec : 1];
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    const Vec zero = {};
    // Rows of up to two pieces a lane stay in registers, and the next one is asked for before this one is reduced; longer ones, and the weight,
    // are read again (out of L2) for the second pass.
    constexpr bool kHold = LPR < 1024 ? PER <= 2 : PER == 1;
    float dw[PER][kVec];
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) dw[i][e] = 0.0f;
    auto weight_of = [&](int i) {
        const Piece<kVec> pc(lane + i * LPR, channels);
        Vec v;
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = Traits<T>::from_f32(1.0f);
        if (weight != nullptr && pc.live) v = load_raw<T>(weight, pc.at, channels);
        return v;
    };
    Vec kept[kHold ? PER : 1];
    if constexpr (kHold) {
#pragma unroll
        for (int i = 0; i < PER; ++i) kept[i] = weight_of(i);
    }
    struct Row { Vec r[kHold ? PER : 1], g[kHold ? PER : 1], past[kHold ? PER : 1]; };
    auto read = [&](int64_t row, int i, Vec& r, Vec& g, Vec& past) {
        const Piece<kVec> pc(lane + i * LPR, channels);
        r = g = past = zero;
        if (row < rows && pc.live) {
            r = load_raw<T>(sum + row * channels, pc.at, channels);
            g = load_raw<T>(d_y + row * channels, pc.at, channels);
            if (d_sum != nullptr) past = load_raw<T>(d_sum + row * channels, pc.at, channels);
        }
    };
    auto fetch = [&](Row& to, int64_t row) {
        if constexpr (kHold) {
#pragma unroll
            for (int i = 0; i < PER; ++i) read(row, i, to.r[i], to.g[i], to.past[i]);
        }
    };
    auto step = [&](const Row& now, int64_t row, int turn) {
        float squares = 0.0f, along = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            Vec r, g, past, w;
            if constexpr (kHold) r = now.r[i], g = now.g[i], w = kept[i];
            else read(row, i, r, g, past), w = weight_of(i);
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float one = e < pc.skip ? 0.0f : Traits<T>::to_f32(r[e]);
                squares = fmaf(one, one, squares);
                along = fmaf(one * Traits<T>::to_f32(w[e]), Traits<T>::to_f32(g[e]), along);
            }
        }
        sum_row<LPR>(squares, along, room[turn]);
        const float rstd = 1.0f / sqrtf(squares / (float)channels + eps);
        const float back = along * rstd * rstd / (float)channels;       // of r, in units of rstd
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            Vec r, g, past, w;
            if constexpr (kHold) r = now.r[i], g = now.g[i], past = now.past[i], w = kept[i];
            else read(row, i, r, g, past), w = weight_of(i);
            if (row >= rows || !pc.live) continue;
            float d[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float rf = Traits<T>::to_f32(r[e]), gf = Traits<T>::to_f32(g[e]);
                dw[i][e] = fmaf(gf, rf * rstd, dw[i][e]);
                d[e] = fmaf(rstd, Traits<T>::to_f32(w[e]) * gf - rf * back, Traits<T>::to_f32(past[e]));
            }
            if (kHold || pc.skip == 0) {
                store_row<T>(d_r + row * channels, pc.at, channels, d);
            } else {
                // (d_r may be d_y, and what the lane before has stored there was read again here: its own channels alone)
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (e >= pc.skip) d_r[row * channels + pc.at + e] = Traits<T>::from_f32(d[e]);
            }
        }
    };
    int64_t row = (int64_t)blockIdx.x * kRows + group;
    const int64_t last = rows + group, stride = (int64_t)gridDim.x * kRows;     // (all of a workgroup's rows pass `last` in the same step)
    Row here, there;
    fetch(here, row);
    for (; row < last; row += 2 * stride) {
        fetch(there, row + stride);
        step(here, row, 0);
        if (row + stride >= last) break;
        fetch(here, row + 2 * stride);
        step(there, row + stride, 1);
    }
    if (partials == nullptr) return;
    float* out = partials + (int64_t)blockIdx.x * channels;
    if constexpr (kRows > 1) {
        // (by channel: a piece that starts early leaves out what the one before has)
        constexpr int kWidth = LPR * PER * kVec;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (pc.live && e >= pc.skip) groups[group * kWidth + pc.at + e] = dw[i][e];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < channels; c += kThreads) {
            float s = 0.0f;
#pragma unroll 4
            for (int k = 0; k < kRows; ++k) s += groups[k * kWidth + c];
            out[c] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (pc.live && e >= pc.skip) out[pc.at + e] = dw[i][e];
        }
    }
}

// d_weight = the sum of the workgroups' parts, in an order of its own: 32 channels a workgroup, 32 runs of parts, then those.
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* partials, float* d_weight, int blocks, int channels) {
    __shared__ float room[32][33];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, run = threadIdx.x / 32;
    float s = 0.0f;
    if (c < channels) {
#pragma unroll 8
        for (int b = run; b < blocks; b += 32) s += partials[(int64_t)b * channels + c];
    }
    room[run][threadIdx.x % 32] = s;
    __syncthreads();
    if (run == 0 && c < channels) {
#pragma unroll
        for (int k = 1; k < 32; ++k) s += room[k][threadIdx.x];
        d_weight[c] = s;
    }
}

template <class T>
hipError_t norm_of(const NormCall& c, hipStream_t stream) {
    return with_lanes<sizeof(T)>(lanes_for(c.channels, sizeof(T)), [&](auto lpr, auto per) {
        constexpr int kLpr = decltype(lpr)::value, kPer = decltype(per)::value, kThreads = kLpr > 256 ? kLpr : 256, kRows = kThreads / kLpr;
        // (a launch has fewer than 2^32 threads: more rows than these go in several)
        constexpr int64_t kMost = ((int64_t)1 << 31) / kThreads * kRows;
        for (int64_t from = 0; from < c.rows; from += kMost) {
            const int64_t rows = c.rows - from < kMost ? c.rows - from : kMost, at = from * c.channels;
            const dim3 grid((unsigned)((rows + kRows - 1) / kRows)), threads(kThreads);
            const T *x = (const T*)c.x + at, *res = c.residual ? (const T*)c.residual + at : nullptr, *w = (const T*)c.weight;
            T* sum = c.sum ? (T*)c.sum + at : nullptr;
            float* scale = c.scale ? c.scale + from : nullptr;
            void* y = (char*)c.y + at * (int64_t)(c.scale ? 1 : sizeof(T));
            if (c.plain) hipLaunchKernelGGL((norm_kernel<T, kLpr, kPer, true, true>), grid, threads, 0, stream, x, res, w, y, scale, sum, rows, c.channels, c.eps);
            else if (c.scale) hipLaunchKernelGGL((norm_kernel<T, kLpr, kPer, true, false>), grid, threads, 0, stream, x, res, w, y, scale, sum, rows, c.channels, c.eps);
            else hipLaunchKernelGGL((norm_kernel<T, kLpr, kPer, false, false>), grid, threads, 0, stream, x, res, w, y, scale, sum, rows, c.channels, c.eps);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

template <class T>
hipError_t norm_backward_of(const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight, float* partials,
                            int64_t rows, int channels, float eps, hipStream_t stream) {
    const int blocks = norm_backward_blocks(rows, channels, sizeof(T));
    // (no rows: nothing but a d_weight of zeros)
    hipError_t e = blocks == 0 ? hipSuccess : with_lanes<sizeof(T)>(lanes_for(channels, sizeof(T)), [&](auto lpr, auto per) {
        constexpr int kLpr = decltype(lpr)::value, kPer = decltype(per)::value, kThreads = kLpr > 256 ? kLpr : 256;
        hipLaunchKernelGGL((norm_backward_kernel<T, kLpr, kPer>), dim3(blocks), dim3(kThreads), 0, stream, (const T*)sum, (const T*)weight,
                           (const T*)d_y, (const T*)d_sum, (T*)d_r, d_weight ? partials : nullptr, rows, channels, eps);
        return hipGetLastError();
    });
    if (e != hipSuccess || d_weight == nullptr) return e;
    hipLaunchKernelGGL(norm_weight_kernel, dim3((channels + 31) / 32), dim3(1024), 0, stream, partials, d_weight, blocks, channels);
    return hipGetLastError();
}

}  // namespace

// Workgroups of the backward pass: what the compute units work on at once, so that their parts of d_weight are few, and those no more than one
// for four rows while there is one a unit.  bf16, us with 256 / 512 (768, 1024) of them: 8192 x 2051 50 / 36 (42, 40), 2048 x 2051 18.7 /
// 17.2, 1024 x 4096 15.6 / 18.2, 512 x 2048 9.4 / 11.1; of 1024 threads 2048 x 8192 31 / 39 (46, 52), 4096 x 16384 116 / 126.
int norm_backward_blocks(int64_t rows, int channels, int elem) {
    const Lanes l = lanes_for(channels, elem);
    const int per_block = (l.lpr > 256 ? l.lpr : 256) / l.lpr;
    const int64_t all = (rows + per_block - 1) / per_block;
    const int64_t most = l.lpr > 256 || rows / 4 < 256 ? 256 : (rows / 4 < 512 ? rows / 4 : 512);
    return (int)(all < most ? all : most);
}

hipError_t launch_norm(int dt, const NormCall& c, hipStream_t stream) {
    switch (dt) {
        case 0: return norm_of<float>(c, stream);
        case 1: return norm_of<_Float16>(c, stream);
        case 2: return norm_of<__bf16>(c, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_norm_backward(int dt, const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight,
                                float* partials, int64_t rows, int channels, float eps, hipStream_t stream) {
    switch (dt) {
        case 0: return norm_backward_of<float>(sum, weight, d_y, d_sum, d_r, d_weight, partials, rows, channels, eps, stream);
        case 1: return norm_backward_of<_Float16>(sum, weight, d_y, d_sum, d_r, d_weight, partials, rows, channels, eps, stream);
        case 2: return norm_backward_of<__bf16>(sum, weight, d_y, d_sum, d_r, d_weight, partials, rows, channels, eps, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace msla
