// A lane's eight values of a head vector, as the appends load, widen, round and
// store them: two quads, apart (the halves of a rotary pair) or neighbours.
#pragma once

#include "cl_device.h"

namespace cl {
namespace {

struct Raw {                   // four 16-bit values as they stand
    uint32_t a, b;
};

struct Quad {
    float v[4];
};

// A lane's two quads at `lo` and `hi`: neighbours (hi = lo + 4, 16-byte aligned)
// in one access.
template <bool VEC>
__device__ __forceinline__ void load8(const uint16_t* p, int lo, int hi, bool apart, Raw& x, Raw& y) {
    if constexpr (VEC) {
        if (apart) {
            const u32x2 u = *reinterpret_cast<const u32x2*>(p + lo), v = *reinterpret_cast<const u32x2*>(p + hi);
            x = Raw{u[0], u[1]};
            y = Raw{v[0], v[1]};
        } else {
            const u32x4 u = *reinterpret_cast<const u32x4*>(p + lo);
            x = Raw{u[0], u[1]};
            y = Raw{u[2], u[3]};
        }
    } else {
        const auto two = [](const uint16_t* q) { return q[0] | static_cast<uint32_t>(q[1]) << 16; };
        x = Raw{two(p + lo), two(p + lo + 2)};
        y = Raw{two(p + hi), two(p + hi + 2)};
    }
}

// STREAM: a prompt's results (four heads a group, see choose) are stored past the
// L2 caches (8593 tokens 56.5 -> 47.3 us when it was changed).
// Attention behind the call is no slower for it: 1500 tokens, both, 56.2 us
// against 57.2 with ordinary stores, 3000 103.5 / 104.8, 8593 627 / 626.
template <bool STREAM, class T>
__device__ __forceinline__ void put(uint16_t* p, T v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<T*>(p));
    else *reinterpret_cast<T*>(p) = v;
}

template <bool VEC, bool STREAM>
__device__ __forceinline__ void store8(uint16_t* p, int lo, int hi, bool apart, Raw x, Raw y) {
    if constexpr (VEC) {
        if (apart) {
            put<STREAM>(p + lo, u32x2{x.a, x.b});
            put<STREAM>(p + hi, u32x2{y.a, y.b});
        } else {
            put<STREAM>(p + lo, u32x4{x.a, x.b, y.a, y.b});
        }
    } else {
        const auto two = [](uint16_t* q, uint32_t v) {
            q[0] = static_cast<uint16_t>(v);
            q[1] = static_cast<uint16_t>(v >> 16);
        };
        two(p + lo, x.a), two(p + lo + 2, x.b);
        two(p + hi, y.a), two(p + hi + 2, y.b);
    }
}

__device__ __forceinline__ Quad widen(Raw r, int dt) {
    return Quad{{act_to_f32(static_cast<uint16_t>(r.a & 0xffff), dt), act_to_f32(static_cast<uint16_t>(r.a >> 16), dt),
                 act_to_f32(static_cast<uint16_t>(r.b & 0xffff), dt), act_to_f32(static_cast<uint16_t>(r.b >> 16), dt)}};
}

__device__ __forceinline__ Raw narrow(const Quad& q, int dt) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = dt == DT_FP16 ? f32_to_f16_bits(q.v[i]) : f32_to_bf16_bits(q.v[i]);
    return Raw{b[0] | b[1] << 16, b[2] | b[3] << 16};
}

}  // namespace
}  // namespace cl
