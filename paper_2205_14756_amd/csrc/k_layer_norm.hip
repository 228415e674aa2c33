// Layer norm of rows with the residual's addition, its gradient, and rows into 8-bit integers with a scale a row.
//
// Bound by memory, like the root-mean-square norm, whose pieces and lanes it has: a row is read once, stays in registers as fp32 through its mean and
// then the squares of what is left, and is written once.  (Two reductions a row: the squares less the mean's would lose what a mean that is
// large beside the deviations costs.)  16384 rows of 4096 with a residual in bf16: 96 us (537 MB, 5.6 TB/s); the gradient of 8192 rows of 1024 in fp32 30 us (4.5
// TB/s), of 4096 in bf16 61 (4.4), of 2051 in fp16, whose 257th piece makes two of each lane's, 44 and 5 for the parts (3.1).
#include "msla_device.h"
#include "msla_layer_kernels.h"
#include "msla_sequence_kernels.h"
#include "norm_rows.h"

namespace msla {
namespace {

constexpr float kTop = 127.0f;

// whether channel e of a lane's piece counts: within the row, and not in the piece before as well
template <int VEC>
__device__ __forceinline__ bool counts(const Piece<VEC>& pc, int e, int channels) { return pc.live && e >= pc.skip && pc.at + e < channels; }

template <class T, int LPR, int PER>
__global__ void __launch_bounds__(LPR > 256 ? LPR : 256) layer_norm_kernel(const T* x, const T* residual, const T* weight, const T* bias, T* y, T* sum,
                                                                           int64_t rows, int channels, float eps) {
    constexpr int kVec = Traits<T>::kVec, kThreads = LPR > 256 ? LPR : 256, kRows = kThreads / LPR;
    __shared__ float room[kThreads / 64];
    const int lane = threadIdx.x % LPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR;
    const bool live = row < rows;
    const int64_t base = (live ? row : 0) * channels;
    auto add = [](float a, float b) { return a + b; };
    float r[PER][kVec];
    float total = 0.0f;
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
        for (int e = 0; e < kVec; ++e) total += e < pc.skip ? 0.0f : r[i][e];
    }
    const float mean = over_row<LPR>(total, room, add) / (float)channels;
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const Piece<kVec> pc(lane + i * LPR, channels);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float d = r[i][e] - mean;
            squares += counts(pc, e, channels) ? d * d : 0.0f;
        }
    }
    squares = over_row<LPR>(squares, room, add);
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
        if (!live || !pc.live) continue;
        float w[kVec], b[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) w[e] = 1.0f, b[e] = 0.0f;
        if (weight != nullptr) load_row<T>(weight, pc.at, channels, w);
        if (bias != nullptr) load_row<T>(bias, pc.at, channels, b);
#pragma unroll
        for (int e = 0; e < kVec; ++e) r[i][e] = fmaf((r[i][e] - mean) * rstd, w[e], b[e]);
        store_row<T>(y + base, pc.at, channels, r[i]);
    }
}

// A workgroup walks over rows; a lane has the same channels of each, so it sums their parts of d_weight and d_bias in registers.  The next row is on
// its way while this one is reduced.
// Lanes of a row in the gradient, in whole waves: one piece each up to 256, two up to 512 lanes (which then take two waves a SIMD).
constexpr int threads_of(int lpr) { return lpr < 192 ? 256 : lpr; }
template <int ELEM, class F>
hipError_t with_lanes_back(int channels, F&& f) {
    using std::integral_constant;
    const int pieces = (channels * ELEM + 15) / 16;
    integral_constant<int, 1> one;
    integral_constant<int, 2> two;
    if (pieces <= 4) return f(integral_constant<int, 4>{}, one);
    if (pieces <= 16) return f(integral_constant<int, 16>{}, one);
    if (pieces <= 64) return f(integral_constant<int, 64>{}, one);
    if (pieces <= 128) return f(integral_constant<int, 128>{}, one);
    if (pieces <= 192) return f(integral_constant<int, 192>{}, one);
    if (pieces <= 256) return f(integral_constant<int, 256>{}, one);
    if (pieces <= 512) return f(integral_constant<int, 256>{}, two);
    if (pieces <= 1024) return f(integral_constant<int, 512>{}, two);
    if (pieces <= 2048) return f(integral_constant<int, 1024>{}, two);
    if constexpr (ELEM == 4)
        if (pieces > 4096) return f(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

template <class T, int LPR, int PER>
__global__ void __launch_bounds__(threads_of(LPR)) layer_norm_backward_kernel(const T* sum, const T* weight, const T* d_y, const T* d_sum, T* d_r,
                                                                                    float* parts, int64_t rows, int channels, float eps) {
    constexpr int kVec = Traits<T>::kVec, kThreads = threads_of(LPR), kRows = kThreads / LPR;
    typedef typename Traits<T>::Vec Vec;
    __shared__ f32x4 room[2][kThreads / 64];
    __shared__ float groups[kRows > 1 ? kThreads * PER * kVec : 1];
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    const Vec zero = {};
    constexpr int kIn = LPR < 64 ? LPR : 64;
    auto add = [](float x, float y) { return x + y; };
    // Rows of up to 1024 pieces (4096 channels of fp32, 8192 of 16 bits) stay in registers, and the next one is asked for before this one is reduced; longer
    // ones, and the weight, are read again (out of L2) for each pass, as 1024 lanes have 128 registers.  What they keep for d_weight and d_bias spills even so: 81 to 391 registers
    // of fp32 rows, 103 to 310 of 16 bits.
    constexpr bool kHold = LPR < 1024;
    float dw[PER][kVec], db[PER][kVec];
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) dw[i][e] = db[i][e] = 0.0f;
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
    // how many channels each wave has of a row, and one over that
    __shared__ f32x2 sizes[kThreads / 64];
    float per_wave;
    {
        float own = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
#pragma unroll
            for (int e = 0; e < kVec; ++e) own += counts(pc, e, channels) ? 1.0f : 0.0f;
        }
        own = over_lanes<kIn>(own, add);
        per_wave = own > 0.0f ? 1.0f / own : 0.0f;
        if constexpr (LPR > 64) {
            if ((threadIdx.x & 63) == 0) sizes[threadIdx.x >> 6] = f32x2{per_wave, own};
            __syncthreads();
        }
    }
    auto step = [&](const Row& now, int64_t row, int turn) {
        auto piece = [&](int i, Vec& r, Vec& g, Vec& past, Vec& w) {
            if constexpr (kHold) r = now.r[i], g = now.g[i], past = now.past[i], w = kept[i];
            else read(row, i, r, g, past), w = weight_of(i);
        };
        // Sums of r and of w dy, then of the squares of r's deviations and of their products with w dy: about the mean of what a wave has of the row, so
        // that one exchange between the waves does.  About the row's mean they are more by the waves' means' own deviations.
        float total = 0.0f, pull = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            Vec r, g, past, w;
            piece(i, r, g, past, w);
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                total += e < pc.skip ? 0.0f : Traits<T>::to_f32(r[e]);
                pull += e < pc.skip ? 0.0f : Traits<T>::to_f32(w[e]) * Traits<T>::to_f32(g[e]);
            }
        }
        total = over_lanes<kIn>(total, add);
        pull = over_lanes<kIn>(pull, add);
        float mean = total * per_wave;
        float squares = 0.0f, along = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            Vec r, g, past, w;
            piece(i, r, g, past, w);
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float d = counts(pc, e, channels) ? Traits<T>::to_f32(r[e]) - mean : 0.0f;
                squares = fmaf(d, d, squares);
                along = fmaf(d * Traits<T>::to_f32(w[e]), Traits<T>::to_f32(g[e]), along);
            }
        }
        squares = over_lanes<kIn>(squares, add);
        along = over_lanes<kIn>(along, add);
        if constexpr (LPR > 64) {
            constexpr int kWaves = LPR / 64;
            if ((threadIdx.x & 63) == 0) room[turn][threadIdx.x >> 6] = f32x4{total, pull, squares, along};
            __syncthreads();
            total = pull = squares = along = 0.0f;
            const int first = group * kWaves;       // of the row's waves
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                total += room[turn][first + w][0];
                pull += room[turn][first + w][1];
            }
            mean = total / (float)channels;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const f32x4 v = room[turn][first + w];
                const float off = sizes[w][0] * v[0] - mean;
                squares += fmaf(sizes[w][1] * off, off, v[2]);
                along += fmaf(off, v[1], v[3]);
            }
        }
        pull = pull / (float)channels;
        const float rstd = 1.0f / sqrtf(squares / (float)channels + eps);
        const float back = along * rstd * rstd / (float)channels;       // of the deviation, in units of rstd
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Piece<kVec> pc(lane + i * LPR, channels);
            Vec r, g, past, w;
            piece(i, r, g, past, w);
            if (row >= rows || !pc.live) continue;
            float d[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float df = Traits<T>::to_f32(r[e]) - mean, gf = Traits<T>::to_f32(g[e]);
                dw[i][e] = fmaf(gf, df * rstd, dw[i][e]);
                db[i][e] += gf;
                d[e] = fmaf(rstd, fmaf(Traits<T>::to_f32(w[e]), gf, -pull) - df * back, Traits<T>::to_f32(past[e]));
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
    if (parts == nullptr) return;
    auto leave = [&](float* out, const float (&d)[PER][kVec]) {
        if constexpr (kRows > 1) {
            // (by channel: a piece that starts early leaves out what the one before has)
            constexpr int kWidth = LPR * PER * kVec;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const Piece<kVec> pc(lane + i * LPR, channels);
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (pc.live && e >= pc.skip) groups[group * kWidth + pc.at + e] = d[i][e];
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
                    if (pc.live && e >= pc.skip && pc.at + e < channels) out[pc.at + e] = d[i][e];
            }
        }
    };
    leave(parts + (int64_t)blockIdx.x * 2 * channels, dw);
    leave(parts + (int64_t)blockIdx.x * 2 * channels + channels, db);
}

// Rows into 8-bit integers: scale = max |x| times fp32's 1 / 127, x8 = x / scale to the nearest whole number, ties to even; product and quotient are rounded
// as IEEE says, so that the same x gives the same integers everywhere.  A row with a NaN has a NaN for its scale, one with an infinity an infinity, and zeros.
// 16384 rows of 4096 in bf16: 52 us (201 MB, 3.9 TB/s).
template <class T, int LPR, int PER>
__global__ void __launch_bounds__(LPR > 256 ? LPR : 256) quantize_integer_kernel(const T* x, signed char* x8, float* scale, int64_t rows, int channels) {
    constexpr int kVec = Traits<T>::kVec, kThreads = LPR > 256 ? LPR : 256, kRows = kThreads / LPR;
    __shared__ float room[kThreads / 64];
    const int lane = threadIdx.x % LPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR;
    const bool live = row < rows;
    const int64_t base = (live ? row : 0) * channels;
    float r[PER][kVec], top = 0.0f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const Piece<kVec> pc(lane + i * LPR, channels);
        if (live && pc.live) {
            load_row<T>(x + base, pc.at, channels, r[i]);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) r[i][e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            top = fmaxf(top, fabsf(r[i][e]));
            odd |= r[i][e] != r[i][e];
        }
    }
    if (odd) top = __builtin_nanf("");
    // (a NaN anywhere makes the row's scale one: fmaxf would drop it)
    top = over_row<LPR>(top, room, [](float a, float b) { return a != a || b != b ? __builtin_nanf("") : fmaxf(a, b); });
    const float s = top * (1.0f / kTop);
    const bool fine = s > 0.0f && s <= 3.4e38f;
    if (live && lane == 0) scale[row] = s;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const Piece<kVec> pc(lane + i * LPR, channels);
        if (!live || !pc.live) continue;
        unsigned w[kVec / 4];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float q = fine ? fminf(fmaxf(rintf(r[i][e] / s), -kTop), kTop) : 0.0f;
            const unsigned b = (unsigned)(int)q & 255u;
            w[e / 4] = e % 4 == 0 ? b : w[e / 4] | b << (8 * (e % 4));
        }
        signed char* p = x8 + base;
        if (channels >= kVec) {
            __builtin_memcpy(__builtin_assume_aligned(p + pc.at, 1), w, kVec);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (e < channels) p[e] = (signed char)(w[e / 4] >> (8 * (e % 4)));
        }
    }
}

// (a launch has fewer than 2^32 threads: more rows than these go in several)
template <int LPR, class F>
hipError_t in_launches(int64_t rows, F&& f) {
    constexpr int kThreads = LPR > 256 ? LPR : 256, kRows = kThreads / LPR;
    constexpr int64_t kMost = ((int64_t)1 << 31) / kThreads * kRows;
    for (int64_t from = 0; from < rows; from += kMost) {
        const int64_t n = rows - from < kMost ? rows - from : kMost;
        f(from, n, dim3((unsigned)((n + kRows - 1) / kRows)), dim3(kThreads));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class F>
hipError_t with_type(int dt, F&& f) {
    switch (dt) {
        case 0: return f(float{});
        case 1: return f(_Float16{});
        case 2: return f(__bf16{});
    }
    return hipErrorInvalidValue;
}

}  // namespace

// Workgroups of the gradient: what the compute units work on at once, twelve waves of lanes with one piece and eight of those with two, so that their
// parts of d_weight and d_bias are few.  us with 4 / 8 / 12 / 16 waves: 16384 x 1024 in bf16 44 / 35 / 32 / 32, 8192 x 1024 in fp32 49 / 34 / 30 / 30, 2048 x 768
// 18 / 17 / 20 / 17; of two pieces, 8192 x 2051 in fp16, 66 / 50 / 57 / 58.
int layer_norm_blocks(int64_t rows, int channels, int elem) {
    int threads = 256, per_block = 1, waves = 12;
    auto take = [&](auto lpr, auto per) {
        threads = threads_of(decltype(lpr)::value);
        per_block = threads / decltype(lpr)::value;
        waves = decltype(per)::value > 1 ? 8 : 12;
        return hipSuccess;
    };
    (void)(elem == 4 ? with_lanes_back<4>(channels, take) : with_lanes_back<2>(channels, take));
    const int64_t all = (rows + per_block - 1) / per_block, most = 256 * (waves * 64 > threads ? waves * 64 / threads : 1);
    return (int)(all < most ? all : most);
}

hipError_t launch_layer_norm(int dt, const LayerNormCall& c, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        return with_lanes<sizeof(T)>(lanes_for(c.channels, sizeof(T)), [&](auto lpr, auto per) {
            constexpr int kLpr = decltype(lpr)::value, kPer = decltype(per)::value;
            return in_launches<kLpr>(c.rows, [&](int64_t from, int64_t rows, dim3 grid, dim3 threads) {
                const int64_t at = from * c.channels;
                hipLaunchKernelGGL((layer_norm_kernel<T, kLpr, kPer>), grid, threads, 0, stream, (const T*)c.x + at, c.residual ? (const T*)c.residual + at : nullptr,
                                   (const T*)c.weight, (const T*)c.bias, (T*)c.y + at, c.sum ? (T*)c.sum + at : nullptr, rows, c.channels, c.eps);
            });
        });
    });
}

hipError_t launch_layer_norm_backward(int dt, const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight,
                                      float* d_bias, float* parts, int64_t rows, int channels, float eps, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        const int blocks = layer_norm_blocks(rows, channels, sizeof(T));
        const bool sums = d_weight != nullptr || d_bias != nullptr;
        // (no rows: nothing but sums of zeros)
        const hipError_t e = blocks == 0 ? hipSuccess : with_lanes_back<sizeof(T)>(channels, [&](auto lpr, auto per) {
            constexpr int kLpr = decltype(lpr)::value, kPer = decltype(per)::value;
            hipLaunchKernelGGL((layer_norm_backward_kernel<T, kLpr, kPer>), dim3(blocks), dim3(threads_of(kLpr)), 0, stream, (const T*)sum, (const T*)weight,
                               (const T*)d_y, (const T*)d_sum, (T*)d_r, sums ? parts : nullptr, rows, channels, eps);
            return hipGetLastError();
        });
        if (e != hipSuccess || !sums) return e;
        return launch_sum_parts(parts, blocks, 2 * (int64_t)channels, PartSums{{d_weight, d_bias, nullptr}, {channels, channels, 0}}, stream);
    });
}

hipError_t launch_quantize_integer(int dt, const void* x, void* x8, float* scale, int64_t rows, int channels, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        return with_lanes<sizeof(T)>(lanes_for(channels, sizeof(T)), [&](auto lpr, auto per) {
            constexpr int kLpr = decltype(lpr)::value, kPer = decltype(per)::value;
            return in_launches<kLpr>(rows, [&](int64_t from, int64_t n, dim3 grid, dim3 threads) {
                hipLaunchKernelGGL((quantize_integer_kernel<T, kLpr, kPer>), grid, threads, 0, stream, (const T*)x + from * channels,
                                   (signed char*)x8 + from * channels, scale + from, n, channels);
            });
        });
    });
}

}  // namespace msla
