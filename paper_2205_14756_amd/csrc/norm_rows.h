// Rows of channels in pieces of 16 bytes, some to a lane, and sums over a row's lanes: shared by the norms and what else goes over rows.
#pragma once
#include "msla_device.h"

namespace msla {
namespace {

// A lane's i-th piece of a row: its first channel, and how many of its channels the piece before has.
template <int VEC>
struct Piece {
    int at, skip;
    bool live;
    __device__ __forceinline__ Piece(int i, int channels) {
        const int first = i * VEC;
        live = first < channels;
        at = max(0, min(first, channels - VEC));
        skip = first - at;
    }
};

// (rows shorter than a piece go by elements)
template <class T>
__device__ __forceinline__ typename Traits<T>::Vec load_raw(const T* p, int at, int channels) {
    constexpr int kVec = Traits<T>::kVec;
    typename Traits<T>::Vec v;
    if (channels >= kVec) {
        __builtin_memcpy(&v, __builtin_assume_aligned(p + at, sizeof(T)), 16);
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = e < channels ? p[e] : Traits<T>::from_f32(0.0f);
    }
    return v;
}

template <class T>
__device__ __forceinline__ void load_row(const T* p, int at, int channels, float (&f)[Traits<T>::kVec]) {
    const typename Traits<T>::Vec v = load_raw<T>(p, at, channels);
#pragma unroll
    for (int e = 0; e < Traits<T>::kVec; ++e) f[e] = Traits<T>::to_f32(v[e]);
}

template <class T>
__device__ __forceinline__ void store_row(T* p, int at, int channels, const float (&f)[Traits<T>::kVec]) {
    constexpr int kVec = Traits<T>::kVec;
    typename Traits<T>::Vec v;
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = Traits<T>::from_f32(f[e]);
    if (channels >= kVec) {
        __builtin_memcpy(__builtin_assume_aligned(p + at, sizeof(T)), &v, 16);
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (e < channels) p[e] = v[e];
    }
}

// The join of v over the LANES neighbours (a power of two, 64 at most) that it belongs to, to all of them: pairs, fours, eights, ... by data-parallel
// moves, a tenth of the latency of a permutation through LDS.
template <int CTRL>
__device__ __forceinline__ float moved_by(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LANES, class F>
__device__ __forceinline__ float over_lanes(float v, F&& join) {
    if constexpr (LANES >= 2) v = join(v, moved_by<0xB1>(v));                       // lane ^ 1
    if constexpr (LANES >= 4) v = join(v, moved_by<0x4E>(v));                       // lane ^ 2
    if constexpr (LANES >= 8) v = join(v, moved_by<0x141>(v));                      // 7 - lane: the other four, which are alike
    if constexpr (LANES >= 16) v = join(v, moved_by<0x128>(v));                     // lane ^ 8
    if constexpr (LANES >= 32) {
        const unsigned bits = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
        const unsigned first = r[0], second = r[1];
        v = join(__builtin_bit_cast(float, first), __builtin_bit_cast(float, second));
    }
    if constexpr (LANES >= 64) {
        const unsigned bits = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
        const unsigned first = r[0], second = r[1];
        v = join(__builtin_bit_cast(float, first), __builtin_bit_cast(float, second));
    }
    return v;
}

// two sums over the LPR lanes of a row; `room`: two pairs a wave, which take turns, so that one barrier does
template <int LPR>
__device__ __forceinline__ void sum_row(float& a, float& b, f32x2* room) {
    constexpr int kIn = LPR < 64 ? LPR : 64;
    auto add = [](float x, float y) { return x + y; };
    a = over_lanes<kIn>(a, add);
    b = over_lanes<kIn>(b, add);
    if constexpr (LPR > 64) {
        constexpr int kWaves = LPR / 64;
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = f32x2{a, b};
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const f32x2 v = room[w];
            a += v[0];
            b += v[1];
        }
    }
}

// over the LPR lanes of a row; `room`: a float a wave
template <int LPR, class F>
__device__ __forceinline__ float over_row(float v, float* room, F&& join) {
    v = over_lanes<LPR < 64 ? LPR : 64>(v, join);
    if constexpr (LPR > 64) {
        constexpr int kWaves = LPR / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();                // (the room's last readers are through)
        if ((threadIdx.x & 63) == 0) room[wave] = v;
        __syncthreads();
        v = room[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = join(v, room[w]);
    }
    return v;
}

// Lanes of a row: the fewest that leave each at most two 16-byte pieces, so that short rows share a wave and long ones have a
// workgroup; 1024 lanes with up to eight pieces take the longest (32768 fp32 channels).
struct Lanes { int lpr, per; };
inline Lanes lanes_for(int channels, int elem) {
    const int pieces = (channels * elem + 15) / 16;
    for (int lpr : {4, 16, 64, 256})
        if (pieces <= lpr) return {lpr, 1};
        else if (pieces <= 2 * lpr) return {lpr, 2};
    return {1024, pieces <= 1024 ? 1 : (pieces <= 2048 ? 2 : (pieces <= 4096 ? 4 : 8))};
}

// (ELEM: bytes of an element; 32768 channels of 2 are half of the longest row)
template <int ELEM, class F>
hipError_t with_lanes(Lanes l, F&& f) {
    using std::integral_constant;
    auto per2 = [&](auto lpr) { return l.per == 1 ? f(lpr, integral_constant<int, 1>{}) : f(lpr, integral_constant<int, 2>{}); };
    switch (l.lpr) {
        case 4: return per2(integral_constant<int, 4>{});
        case 16: return per2(integral_constant<int, 16>{});
        case 64: return per2(integral_constant<int, 64>{});
        case 256: return per2(integral_constant<int, 256>{});
    }
    if (l.per == 1) return f(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    if (l.per == 2) return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    if constexpr (ELEM == 4)
        if (l.per == 8) return f(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

}  // namespace
}  // namespace msla
