// Pieces of rows between memory and registers, and the tokens that name rows.
#pragma once

#include "gsr_device.h"

namespace gsr {

// ---- pieces of a row ------------------------------------------------------------------------------------
// Rows move in pieces of 16 bytes of the plane's type (V = 4 floats or 8 16-bit values).  The last piece of a row whose width
// is no multiple of V starts V elements before the row's end and overlaps the one before it: both lanes load, sum and store the
// same numbers, so nothing is predicated.  Rows narrower than a piece are taken element by element (V = 1).  Pieces are aligned
// to their elements only.
template <typename T, int V>
struct Piece {                       // V elements as they lie in memory
    static constexpr int NW = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[NW];
    // STREAM: read once, not to be kept in the caches
    template <bool STREAM = false>
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
            else w[0] = (uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16;
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < NW; i += 4) {
                const u32x4a* q = reinterpret_cast<const u32x4a*>(p + i);
                const u32x4a t = STREAM ? __builtin_nontemporal_load(q) : *q;
                w[i] = t[0]; w[i + 1] = t[1]; w[i + 2] = t[2]; w[i + 3] = t[3];
            }
        } else if constexpr (NW == 2) {
            const u32x2h t = *reinterpret_cast<const u32x2h*>(p);
            w[0] = t[0]; w[1] = t[1];
        } else {
            const u32x4h* q = reinterpret_cast<const u32x4h*>(p);
            const u32x4h t = STREAM ? __builtin_nontemporal_load(q) : *q;
            w[0] = t[0]; w[1] = t[1]; w[2] = t[2]; w[3] = t[3];
        }
    }
    __device__ __forceinline__ float at(int i) const {
        if constexpr (V == 1 || sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? (w[i >> 1] & 0xFFFF0000u) : (w[i >> 1] << 16));
    }
};

template <int V, bool STREAM = false, typename T>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[V]) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (V == 1) {
            *p = v[0];
        } else {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                u32x4a t;
                t[0] = __float_as_uint(v[i]); t[1] = __float_as_uint(v[i + 1]);
                t[2] = __float_as_uint(v[i + 2]); t[3] = __float_as_uint(v[i + 3]);
                if constexpr (STREAM) __builtin_nontemporal_store(t, reinterpret_cast<u32x4a*>(p + i));
                else *reinterpret_cast<u32x4a*>(p + i) = t;
            }
        }
    } else {
        if constexpr (V == 1) {
            p->bits = (uint16_t)bf16_bits(v[0]);
        } else {
            static_assert(V == 8, "16-bit pieces hold eight values");
            u32x4h t;
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
            if constexpr (STREAM) __builtin_nontemporal_store(t, reinterpret_cast<u32x4h*>(p));
            else *reinterpret_cast<u32x4h*>(p) = t;
        }
    }
}

// a token's row of the table, or `vocab` where it has none
template <typename I>
__device__ __forceinline__ int32_t token_row(I id, int32_t vocab) { return id >= 0 && id < (I)vocab ? (int32_t)id : vocab; }

}  // namespace gsr
