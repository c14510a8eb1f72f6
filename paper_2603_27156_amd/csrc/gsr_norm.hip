// Group norm with an activation over a batch of graphs, channels last, its gradient, and activation checkpoints in 8 bits.
//
// Rows of a plane belong to graphs, one behind the other; the d columns are cut into `groups` groups of cg.  Over the rows of a graph and
// the columns of a group
//   m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps),  xh = (x - m) r,  y = act(gamma xh + beta)
//   dz = dy act'(gamma xh + beta),  h = gamma dz,  dx = r (h - mean h - xh mean(h xh)),  dgamma = sum dz xh,  dbeta = sum dz.
// A checkpoint holds a row's columns in blocks of up to 64: with A = max |x| (at least 127 * 2^-126) the codes are 127 x / A rounded to the
// nearest whole number, ties to even, and the block's scale is A / 127.
//
// Both directions are two passes over the rows (a small graph's in one launch), sums first: a wave takes `rows` consecutive rows of one slab of columns, keeps the sums of
// its columns in registers, and leaves one pair of sums for every (graph, group) that it met.  Those pairs ("pieces") are joined by a launch
// between the passes, in an order that the sizes and the graphs alone fix.
#include "gsr_internal.h"
#include "gsr_pieces.h"

#include <algorithm>
#include <cmath>

namespace gsr {

constexpr int kBlock = 64;                      // columns that share the scale of a checkpoint
constexpr float kSmallestTop = 127.0f * 0x1p-126f;
constexpr float kLargestScale = 0x1.020406p+121f;       // the largest float of which 127 times is one

// First rows of the graphs, ascending, int32 or int64; NULL: one graph of all rows.  What lies outside the plane counts as its border, so that
// no offsets lead out of it.
struct GraphRows {
    const void* ptr;
    int32_t i64;
    int64_t graphs, n;
    __device__ __forceinline__ int64_t at(int64_t s) const {
        if (!ptr) return s ? n : 0;
        const int64_t v = i64 ? static_cast<const int64_t*>(ptr)[s] : static_cast<const int32_t*>(ptr)[s];
        return v < 0 ? 0 : v > n ? n : v;
    }
};

// How rows and columns are dealt out.  Columns go to lanes in pieces of V; 2^lanes_log2 lanes hold a slab of a row and the wave 64 >> lanes_log2
// rows at a time.  A slab never crosses the border of a plane of a GROUP_PLANAR tensor.  Where V divides a plane's columns and a group's, every lane's columns lie
// in one group.  Else (TAIL) the last piece of a row begins before its own columns, in those of the lane before, which count there alone, and a lane's
// columns lie in two groups at most, no group being narrower than V.
struct NormShape {
    int64_t n, chunks;              // chunks of `rows` rows, one per wave
    int32_t d, dg, cg, groups;
    int32_t lanes_log2, group_slabs, slabs;     // slabs of one plane, and of all
    int32_t rows;
    __host__ __device__ int64_t stride() const { return slabs + groups; }       // pieces of one graph in one chunk
};
struct RowPlane {
    int64_t ld, gs;                 // elements between rows, between planes
};

// What a lane holds of its slab.
struct LaneColumns {
    int sub, subs;                  // its row of the wave's, and how many there are
    int plane, col;                 // plane and first column of it that is loaded
    int column;                     // the same in the whole row of d
    int own;                        // first column of its own: col + skip
    int skip;                       // TAIL: columns that are the lane's before
    int group;                      // the group of its first own column; -1 for a lane without columns
    int begin, split;               // TAIL: loaded columns before `begin` lie in the group before, those from `split` on in the next one (0, V: none do)
    bool on, head, last;            // head: the first lane of its group in the slab; last: the last one with columns
    uint32_t joins;                 // bit k: the lane 2^k further holds columns of the same group (begins with one)
};
template <int V>
__device__ __forceinline__ LaneColumns lane_columns(const NormShape& s, int slab) {
    LaneColumns c;
    const int lanes = 1 << s.lanes_log2, lane = lane_id(), li = lane & (lanes - 1);
    c.sub = lane >> s.lanes_log2;
    c.subs = 64 >> s.lanes_log2;
    c.plane = slab / s.group_slabs;
    const int first = (slab - c.plane * s.group_slabs) * lanes * V;
    auto group = [&](int l) {
        const int col = first + l * V;
        return l >= 0 && l < lanes && col < s.dg ? (c.plane * s.dg + col) / s.cg : -1;
    };
    c.own = first + li * V;
    c.on = c.own < s.dg;
    if (!c.on) c.own = 0;
    c.col = c.own + V <= s.dg ? c.own : s.dg - V;
    c.skip = c.own - c.col;
    c.column = c.plane * s.dg + c.col;
    c.group = group(li);
    c.head = c.on && group(li - 1) != c.group;
    c.last = c.on && group(li + 1) < 0;
    const int from = c.group * s.cg - c.column, to = from + s.cg;
    c.begin = c.on && from > 0 ? from : 0;
    c.split = c.on && to < V ? to : V;
    c.joins = 0;
    for (int k = 0; k < s.lanes_log2; ++k) c.joins |= (uint32_t)(c.on && group(li + (1 << k)) == c.group) << k;
    return c;
}

// The first graph that ends behind `row` (g.graphs if none does): the wave's lanes probe 64 borders at a time.
__device__ __forceinline__ int64_t graph_of(const GraphRows& g, int64_t row) {
    int64_t lo = 0, len = g.graphs;             // it is one of [lo, lo + len], and lo + len if none of [lo, lo + len) does
    while (len > 0) {
        const int64_t step = (len + 63) >> 6, begin = lane_id() * step, end = begin + step < len ? begin + step : len;
        const uint64_t behind = ballot(begin < len && g.at(lo + (begin < len ? end : len)) > row);      // by the last of each lane's graphs
        if (!behind) break;
        const int64_t skip = __builtin_ctzll(behind) * step;
        lo += skip;
        len = (step < len - skip ? step : len - skip) - 1;
    }
    return lo + len;
}

// body(graph, a, b) for the rows [a, b) of every graph that has some in chunk w.  Of graphs without rows, of which a batch of fixed size may have any number at one
// offset, the first is met and the others passed over.
__device__ __forceinline__ int64_t uniform(int64_t v) {                // the same in every lane: kept in scalar registers
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32);
}
template <typename Body>
__device__ __forceinline__ void over_graphs(const NormShape& s, const GraphRows& g, int64_t w, Body body) {
    const int64_t r0 = uniform(w) * s.rows, r1 = r0 + s.rows < s.n ? r0 + s.rows : s.n;
    int64_t i = g.ptr ? graph_of(g, r0) : 0;
    if (i >= g.graphs) return;
    for (int64_t first = uniform(g.at(i)); first < r1;) {
        const int64_t last = uniform(g.at(i + 1)), a = first > r0 ? first : r0, b = last < r1 ? last : r1;
        if (a < b) body(i, a, b);
        const bool empty = a >= b;
        const int64_t next = empty ? graph_of(g, a) : 0;
        i = next > i ? next : i + 1;                    // (goes on whatever the offsets)
        if (i >= g.graphs) break;
        first = empty ? uniform(g.at(i)) : last;
    }
}

// The sums over a group's columns in the slab and over the wave's rows, in the group's first lane.
__device__ __forceinline__ void join_lanes(const NormShape& s, const LaneColumns& c, double& u, double& v) {
    for (int o = 1 << s.lanes_log2; o < 64; o <<= 1) {
        u += __shfl_xor(u, o);
        v += __shfl_xor(v, o);
    }
    for (int k = 0; k < s.lanes_log2; ++k) {
        const double a = __shfl_down(u, 1 << k), b = __shfl_down(v, 1 << k);
        if (c.joins >> k & 1) {
            u += a;
            v += b;
        }
    }
}
// TAIL: u2, v2 are sums of columns in the group after; they go to the next lane, which begins in it, or are a piece of their own in the slab's last
template <bool TAIL>
__device__ __forceinline__ void hand_on(const NormShape& s, const LaneColumns& c, double& u, double& v, double& u2, double& v2) {
    if constexpr (TAIL) {
        const bool first = (lane_id() & ((1 << s.lanes_log2) - 1)) == 0;
        const double a = __shfl_up(u2, 1), b = __shfl_up(v2, 1);
        if (!first && c.on) {
            u += a;
            v += b;
        }
        for (int o = 1 << s.lanes_log2; o < 64; o <<= 1) {
            u2 += __shfl_xor(u2, o);
            v2 += __shfl_xor(v2, o);
        }
    }
}
template <bool TAIL, int V>
__device__ __forceinline__ void leave_piece(const NormShape& s, const LaneColumns& c, int slab, int64_t w, int64_t graph, double u, double v, double u2, double v2,
                                            double2* __restrict__ pieces) {
    hand_on<TAIL>(s, c, u, v, u2, v2);
    if (TAIL && c.last && c.split < V && c.sub == 0) pieces[(w + graph) * s.stride() + slab + c.group + 1] = make_double2(u2, v2);
    join_lanes(s, c, u, v);
    // chunks and graphs both go up along the rows, slabs and groups along the columns: the sums of two indices name a piece
    if (c.head && c.sub == 0) pieces[(w + graph) * s.stride() + slab + c.group] = make_double2(u, v);
}

// The pieces of (graph, group): chunks from w0 on, `count` slabs from s0 on of each, `all` together.
struct PieceRange {
    int64_t graph, w0, all, rows;
    int group, s0, count;
    __device__ __forceinline__ PieceRange(const NormShape& s, const GraphRows& g, int V, int64_t graph_, int group_) : graph(graph_), group(group_) {
        const int64_t first = g.at(graph), last = g.at(graph + 1);
        rows = last > first ? last - first : 0;
        const int width = V << s.lanes_log2;
        auto slab_of = [&](int column) { return column / s.dg * s.group_slabs + column % s.dg / width; };
        s0 = slab_of(group * s.cg);
        count = slab_of(group * s.cg + s.cg - 1) - s0 + 1;
        w0 = first / s.rows;
        all = rows ? ((last - 1) / s.rows - w0 + 1) * count : 0;
    }
};
// .. added up by `threads` threads, of which this is `thread`
__device__ __forceinline__ void add_pieces(const NormShape& s, const PieceRange& r, int thread, int threads, const double2* __restrict__ pieces, double& u, double& v) {
    u = v = 0.0;
    constexpr int U = 4;
    for (int64_t i = thread; i < r.all; i += U * threads) {
        double2 p[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t j = i + (int64_t)k * threads < r.all ? i + (int64_t)k * threads : i;
            p[k] = pieces[(r.w0 + j / r.count + r.graph) * s.stride() + r.s0 + j % r.count + r.group];
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const bool in = i + (int64_t)k * threads < r.all;
            u += in ? p[k].x : 0.0;
            v += in ? p[k].y : 0.0;
        }
    }
}
template <int LANES>
__device__ __forceinline__ double lanes_total(double v) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
// (graph, group) of these THREADS neighbouring threads (16, a wave, a workgroup of 1,024) and the sums of its pieces, in all of them or the first wave; false: no
// task, or not the wave that has the sums.  Sixteen threads leave what has more than 128 pieces to their whole wave.
template <int THREADS>
__device__ __forceinline__ bool joined(const NormShape& s, const GraphRows& g, int V, int64_t block, const double2* __restrict__ pieces,
                                       int64_t& task, double& u, double& v, int64_t& rows) {
    constexpr bool WIDE = THREADS == 1024;
    const int64_t tasks = g.graphs * s.groups;
    task = block * (1024 / THREADS) + threadIdx.x / THREADS;
    const bool on = task < tasks;
    if (THREADS >= 64 && !on) return false;             // (the whole wave, the whole workgroup)
    const PieceRange mine(s, g, V, on ? task / s.groups : 0, on ? (int)(task % s.groups) : 0);
    rows = mine.rows;
    u = v = 0.0;
    const bool large = THREADS == 16 && mine.all > 128;
    if (!large) add_pieces(s, mine, threadIdx.x % THREADS, THREADS, pieces, u, v);
    u = lanes_total<THREADS < 64 ? THREADS : 64>(u);
    v = lanes_total<THREADS < 64 ? THREADS : 64>(v);
    if constexpr (THREADS == 16) {
        for (uint64_t left = ballot(large && on); left;) {
            const int lane = __builtin_ctzll(left), part = lane / 16;
            const int64_t other = block * 64 + (threadIdx.x >> 6) * 4 + part;
            double a, b;
            add_pieces(s, PieceRange(s, g, V, other / s.groups, (int)(other % s.groups)), lane_id(), 64, pieces, a, b);
            a = lanes_total<64>(a);
            b = lanes_total<64>(b);
            if (lane_id() / 16 == part) {
                u = a;
                v = b;
            }
            left &= ~((uint64_t)0xFFFF << 16 * part);
        }
        return on;
    }
    if constexpr (WIDE) {
        __shared__ double s_sum[16][2];
        __syncthreads();                        // the task before has read its sums
        if (lane_id() == 0) {
            s_sum[threadIdx.x >> 6][0] = u;
            s_sum[threadIdx.x >> 6][1] = v;
        }
        __syncthreads();
        if (threadIdx.x >= 64) return false;
        u = v = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            u += s_sum[i][0];
            v += s_sum[i][1];
        }
    }
    return true;
}

// ---- 8 bits ----------------------------------------------------------------------------------------------
// The largest over the 2^k >= 4 neighbouring lanes that share a block.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
    return v > o ? v : o;
}
__device__ __forceinline__ uint32_t lanes_umax(uint32_t v, int lanes) {
    v = dpp_umax<0xB1>(v);          // quad_perm [1,0,3,2]
    v = dpp_umax<0x4E>(v);          // quad_perm [2,3,0,1]
    if (lanes > 4) v = dpp_umax<0x141>(v);              // row_half_mirror
    if (lanes > 8) v = dpp_umax<0x140>(v);              // row_mirror
    if (lanes > 16) {
        const uint32_t o = __shfl_xor(v, 16);
        v = v > o ? v : o;
    }
    if (lanes > 32) {
        const uint32_t o = __shfl_xor(v, 32);
        v = v > o ? v : o;
    }
    return v;
}
// 127 x / top to the nearest whole number, ties to even, exactly: x * (127 / top) in 32 bits, three roundings and a reciprocal good to one unit, is off by
// less than 127 * 5 * 2^-24 < 2^-14, and where it lies that near to a border the exact products decide (16-bit values are half of the largest, a tie,
// all the time).
__device__ __forceinline__ int code_of(float x, float top, float inv) {
    const float t = x * inv;
    float q = __builtin_rintf(t);
    const float f = t - q;
    if (fabsf(f) >= 0.5f - 0x1p-14f) {
        const float side = copysignf(1.0f, f);
        const double over = (double)side * fma(127.0, (double)x, -(double)(q + 0.5f * side) * (double)top);      // (the second product is exact)
        if (over > 0.0 || (over == 0.0 && ((int)q & 1))) q += side;
    }
    return (int)q;
}
// top / 127, correctly rounded: a quotient within one unit, corrected by its exact remainder times the rounded 1 / 127 (Markstein)
__device__ __forceinline__ float by_127(float top) {
    const float q = top * (1.0f / 127.0f);
    return fmaf(fmaf(-127.0f, q, top), 1.0f / 127.0f, q);
}
typedef uint32_t u32_b __attribute__((aligned(1)));
typedef uint16_t u16_b __attribute__((aligned(1)));
// V codes, or with a tail the last V - skip of them
template <int V, bool TAIL>
__device__ __forceinline__ void store_codes(int8_t* p, const int (&q)[V], int skip) {
    if constexpr (V == 1) {
        *p = (int8_t)q[0];
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(V / 4), aligned(TAIL ? 1 : 4)));
        words t;
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            t[i] = (q[4 * i] & 0xFF) | (q[4 * i + 1] & 0xFF) << 8 | (q[4 * i + 2] & 0xFF) << 16 | (uint32_t)q[4 * i + 3] << 24;
        if (TAIL && skip) {
            uint64_t w = t[0];
            if constexpr (V == 8) w |= (uint64_t)t[1] << 32;
            w >>= 8 * skip;
            p += skip;
            const int own = V - skip;
            if (own & 4) {
                *reinterpret_cast<u32_b*>(p) = (uint32_t)w;
                w >>= 32;
                p += 4;
            }
            if (own & 2) {
                *reinterpret_cast<u16_b*>(p) = (uint16_t)w;
                w >>= 16;
                p += 2;
            }
            if (own & 1) *p = (int8_t)w;
        } else {
            __builtin_nontemporal_store(t, reinterpret_cast<words*>(p));
        }
    }
}
struct Checkpoint {
    int8_t* codes;                  // [planes][n][dg]
    float* scales;                  // [planes][n][blocks]
    int32_t blocks;                 // of a row of a plane
    __device__ __forceinline__ int8_t* codes_at(const NormShape& s, const LaneColumns& c, int64_t row) const { return codes + (c.plane * s.n + row) * s.dg + c.col; }
    __device__ __forceinline__ float* scales_at(const NormShape& s, const LaneColumns& c, int64_t row) const { return scales + (c.plane * s.n + row) * blocks; }
};
// The codes of a lane's V values; every lane of the wave takes part.
template <int V, bool TAIL>
__device__ __forceinline__ void save_piece(const Checkpoint& k, const NormShape& s, const LaneColumns& c, int64_t row, bool in, const float (&x)[V]) {
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;         // an infinity is above every number, NaN above that
        bits = bits > b || (TAIL && j < c.skip) ? bits : b;
    }
    if (!c.on) bits = 0;
    const int lanes = 1 << s.lanes_log2;
    bits = lanes_umax(bits, lanes < kBlock / V ? lanes : kBlock / V);
    const bool finite = bits < 0x7F800000u;
    const float top = fmaxf(__uint_as_float(finite ? bits : 0u), kSmallestTop), inv = __builtin_amdgcn_rcpf(fmaxf(top * (1.0f / 127.0f), 0x1p-126f));
    if (!in || !c.on) return;
    int q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) q[j] = finite ? code_of(x[j], top, inv) : 0;
    store_codes<V, TAIL>(k.codes_at(s, c, row), q, c.skip);
    if (c.own % kBlock == 0)
        k.scales_at(s, c, row)[c.own / kBlock] = finite ? fminf(by_127(top), kLargestScale) : __builtin_nanf("");
}

// Where the values of a plane come from: the plane, or its checkpoint.
template <typename T, int V, bool STREAM>
struct PlaneSource {
    const T* x;
    RowPlane p;
    Piece<T, V> w;
    __device__ __forceinline__ void load(const NormShape&, const LaneColumns& c, int64_t row) {
        w.template load<STREAM>(x + c.plane * p.gs + row * p.ld + c.col);
    }
    __device__ __forceinline__ float at(int j) const { return w.at(j); }
};
template <int V, bool TAIL>
struct CodeSource {
    Checkpoint k;
    uint32_t w[V == 1 ? 1 : V / 4];
    float scale, scale_before;      // scale_before: of the columns before a block's border, in a tail
    int before;
    __device__ __forceinline__ void load(const NormShape& s, const LaneColumns& c, int64_t row) {
        const int8_t* p = k.codes_at(s, c, row);
        if constexpr (V == 1) {
            w[0] = (uint8_t)*p;
        } else {
            typedef uint32_t words __attribute__((ext_vector_type(V / 4), aligned(TAIL ? 1 : 4)));
            const words t = *reinterpret_cast<const words*>(p);
#pragma unroll
            for (int i = 0; i < V / 4; ++i) w[i] = t[i];
        }
        const float* scales = k.scales_at(s, c, row);
        scale = scales[(c.col + V - 1) / kBlock];
        if constexpr (TAIL) {
            scale_before = scales[c.col / kBlock];
            before = (c.col + V - 1) / kBlock * kBlock - c.col;
        }
    }
    __device__ __forceinline__ float at(int j) const {
        return (float)(int8_t)(w[j >> 2] >> 8 * (j & 3)) * (TAIL && j < before ? scale_before : scale);
    }
};

// ---- forward ---------------------------------------------------------------------------------------------
// Sums of x - k and (x - k)^2 in 64 bits, with the first value of a graph's group as k: squares are all but exact there, and k, being one of `count` values, lies at
// most sqrt(count) standard deviations from the mean, so that mean (x - k)^2 - (mean (x - k))^2 loses some count 2^-53 of the variance to cancellation.  k of another
// graph would have no such bound.
// 1M x 256 floats 178 us, 5.8 TB/s; 500k x 256 16-bit values 57 us, 4.5 TB/s, where the 64-bit sums take as long as the reads.  4,096 waves: with 2,048 or 16,384
// the forward of the floats takes 498 or 495 us instead of 484, and its gradient from a checkpoint some 50 more.
template <typename T>
__device__ __forceinline__ float group_shift(const NormShape& s, const T* x, const RowPlane& p, int64_t first, int group) {
    const int column = group * s.cg, plane = column / s.dg;
    const float v = to_float(x[plane * p.gs + first * p.ld + (column - plane * s.dg)]);
    return fabsf(v) < INFINITY ? v : 0.0f;
}
template <typename T, int V, bool TAIL>
__global__ __launch_bounds__(256) void k_norm_sums(NormShape s, GraphRows g, const T* __restrict__ x, RowPlane p, double2* __restrict__ pieces,
                                                   float* __restrict__ shifts) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= s.chunks) return;
    const int slab = blockIdx.y;
    const LaneColumns c = lane_columns<V>(s, slab);
    over_graphs(s, g, w, [&](int64_t graph, int64_t a, int64_t b) {
        const int64_t first = g.at(graph);
        const float k1 = group_shift(s, x, p, first, c.on ? c.group : 0), k2 = TAIL && c.split < V ? group_shift(s, x, p, first, c.group + 1) : k1;
        // by the lane in whose own columns the group begins, of the wave that has the graph's first row
        if (a == first && c.on && c.sub == 0) {
            if (c.plane * s.dg + c.own == c.group * s.cg) shifts[graph * s.groups + c.group] = k1;
            if (TAIL && c.split < V) shifts[graph * s.groups + c.group + 1] = k2;
        }
        const double shift = k1, shift2 = k2;
        constexpr int U = 4;
        constexpr int A = TAIL ? V : 1;             // sums of every column, or of all
        double u[A], v[A];
#pragma unroll
        for (int j = 0; j < A; ++j) u[j] = v[j] = 0.0;
        for (int64_t r = a; r < b; r += U * c.subs) {
            PlaneSource<T, V, false> q[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t row = r + k * c.subs + c.sub;
                q[k].x = x;
                q[k].p = p;
                q[k].load(s, c, row < b ? row : a);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const bool in = r + k * c.subs + c.sub < b;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const double from = TAIL && j >= c.split ? shift2 : shift, t = (double)(in ? q[k].at(j) : (float)from) - from;
                    u[TAIL ? j : 0] += t;
                    v[TAIL ? j : 0] = fma(t, t, v[TAIL ? j : 0]);
                }
            }
        }
        double u1 = 0.0, v1 = 0.0, u2 = 0.0, v2 = 0.0;
#pragma unroll
        for (int j = 0; j < A; ++j) {
            const bool next = TAIL && j >= c.split, none = TAIL && j < c.skip;
            u1 += next || none ? 0.0 : u[j];
            v1 += next || none ? 0.0 : v[j];
            u2 += next ? u[j] : 0.0;
            v2 += next ? v[j] : 0.0;
        }
        leave_piece<TAIL, V>(s, c, slab, w, graph, u1, v1, u2, v2, pieces);
    });
}
__device__ __forceinline__ void statistics(double u, double v, double count, double shift, double eps, float& mean, float& rstd) {
    const double m = count ? u / count : 0.0, var = count ? v / count - m * m : 0.0;
    mean = count ? (float)(m + shift) : 0.0f;
    rstd = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps));          // (NaN stays NaN)
}
template <int THREADS>
__global__ __launch_bounds__(1024) void k_norm_join(NormShape s, GraphRows g, int V, const double2* __restrict__ pieces,
                                                    const float* __restrict__ shifts, int64_t task_blocks, double eps,
                                                    float* __restrict__ mean, float* __restrict__ rstd) {
    for (int64_t block = blockIdx.x; block < task_blocks; block += gridDim.x) {
        int64_t task, rows;
        double u, v;
        if (!joined<THREADS>(s, g, V, block, pieces, task, u, v, rows) || threadIdx.x % THREADS) continue;
        float m, r;
        statistics(u, v, (double)rows * s.cg, rows ? (double)shifts[task] : 0.0, eps, m, r);
        mean[task] = m;
        rstd[task] = r;
    }
}

__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
template <int ACT>
__device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == GSR_ACT_RELU) return z < 0.0f ? 0.0f : z;
    else if constexpr (ACT == GSR_ACT_SILU) return z * logistic(z);
    else return z;
}
template <int V>
__device__ __forceinline__ void load_affine(const float* __restrict__ p, const LaneColumns& c, float other, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = p ? p[c.column + j] : other;
}
struct Affine {
    const float *gamma, *beta, *mean, *rstd;
};
// What a lane's columns have by their group: one value, or with TAIL each column one of three (those that are the lane's before it are written again).
__device__ __forceinline__ float pick(bool which, float a, float b) { return which ? a : b; }         // of values: a conditional on members may become one on addresses
template <int V, bool TAIL>
struct ByGroup {
    float before, one, after;
    int begin, split;
    __device__ __forceinline__ ByGroup(const LaneColumns& c, const float* p, int64_t at, int step = 1) : one(p[at * step]), begin(c.begin), split(c.split) {
        before = TAIL && begin > 0 ? p[(at - 1) * step] : one;
        after = TAIL && split < V ? p[(at + 1) * step] : one;
    }
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (TAIL) return pick(j < begin, before, pick(j >= split, after, one));
        else return one;
    }
};

// Bound by its reads and writes: 1M x 256 floats 299 us, 6.8 TB/s, with a checkpoint 390, 6.0; 500k x 256 16-bit values 78 us, 6.5 TB/s.
template <typename T, int V, bool TAIL, int ACT, bool SAVE>
__global__ __launch_bounds__(256) void k_norm_apply(NormShape s, GraphRows g, const T* x, RowPlane p, Affine f, T* y, RowPlane py, Checkpoint ck) {
    const int64_t w = s.chunks - 1 - ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6));        // rows backwards: of one slab what was read last may still be cached (several go in the order that they were read in)
    if (w < 0) return;
    const LaneColumns c = lane_columns<V>(s, blockIdx.y);
    float gamma[V], beta[V];
    load_affine<V>(f.gamma, c, 1.0f, gamma);
    load_affine<V>(f.beta, c, 0.0f, beta);
    over_graphs(s, g, w, [&](int64_t graph, int64_t a, int64_t b) {
        constexpr int U = 4;
        const int64_t at = graph * s.groups + (c.on ? c.group : 0);
        const ByGroup<V, TAIL> m(c, f.mean, at), rs(c, f.rstd, at);
        for (int64_t r = a; r < b; r += U * c.subs) {
            PlaneSource<T, V, true> q[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t row = r + k * c.subs + c.sub;
                q[k].x = x;
                q[k].p = p;
                q[k].load(s, c, row < b ? row : a);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t row = r + k * c.subs + c.sub;
                float v[V];
                if constexpr (SAVE) {
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] = q[k].at(j);
                    save_piece<V, TAIL>(ck, s, c, row, row < b, v);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = activation<ACT>((q[k].at(j) - m[j]) * rs[j] * gamma[j] + beta[j]);
                if (row < b && c.on) store_piece<V, true>(y + c.plane * py.gs + row * py.ld + c.col, v);
            }
        }
    });
}

// One launch for a single graph whose slabs are small and hold whole groups: every workgroup takes the sums of all rows of its slab by itself, and then
// writes its share of the rows.
__device__ __forceinline__ double2 small_total(const NormShape& s, const LaneColumns& c, double u, double v) {          // over the lane's group
    __shared__ double2 s_sum[16][64];
    join_lanes(s, c, u, v);
    const int first = __builtin_amdgcn_readfirstlane(c.group), mine = c.on ? c.group - first : 0;
    if (c.head && c.sub == 0) s_sum[threadIdx.x >> 6][mine] = make_double2(u, v);
    __syncthreads();
    double2 t = make_double2(0.0, 0.0);
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        t.x += s_sum[w][mine].x;
        t.y += s_sum[w][mine].y;
    }
    return t;
}
template <typename T, int V, int ACT, bool SAVE>
__global__ __launch_bounds__(1024) void k_norm_small(NormShape s, GraphRows g, const T* x, RowPlane p, const float* __restrict__ gamma_in,
                                                     const float* __restrict__ beta_in, double eps, float* __restrict__ mean, float* __restrict__ rstd,
                                                     T* y, RowPlane py, Checkpoint ck) {
    const LaneColumns c = lane_columns<V>(s, blockIdx.y);
    const int wave = threadIdx.x >> 6;
    const int64_t a = g.at(0), b = g.at(1) > a ? g.at(1) : a;
    constexpr int U = 4;
    const double shift = a < b ? (double)group_shift(s, x, p, a, c.on ? c.group : 0) : 0.0;
    double u = 0.0, v = 0.0;
    for (int64_t r = a + (int64_t)wave * U * c.subs; r < b; r += 16 * U * c.subs) {
        PlaneSource<T, V, false> q[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t row = r + k * c.subs + c.sub;
            q[k].x = x;
            q[k].p = p;
            q[k].load(s, c, row < b ? row : a);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const bool in = r + k * c.subs + c.sub < b;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const double t = in ? (double)q[k].at(j) - shift : 0.0;
                u += t;
                v = fma(t, t, v);
            }
        }
    }
    float gamma[V], beta[V], m, rs;
    load_affine<V>(gamma_in, c, 1.0f, gamma);
    load_affine<V>(beta_in, c, 0.0f, beta);
    const double2 t = small_total(s, c, u, v);
    statistics(t.x, t.y, (double)(b - a) * s.cg, shift, eps, m, rs);
    if (blockIdx.x == 0 && wave == 0 && c.head && c.sub == 0) {
        mean[c.group] = m;
        rstd[c.group] = rs;
    }
    for (int64_t r = a + ((int64_t)blockIdx.x * 16 + wave) * c.subs; r < b; r += (int64_t)gridDim.x * 16 * c.subs) {
        const int64_t row = r + c.sub, have = row < b ? row : a;
        PlaneSource<T, V, false> q;
        q.x = x;
        q.p = p;
        q.load(s, c, have);
        float z[V];
        if constexpr (SAVE) {
#pragma unroll
            for (int j = 0; j < V; ++j) z[j] = q.at(j);
            save_piece<V, false>(ck, s, c, row, row < b, z);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] = activation<ACT>((q.at(j) - m) * rs * gamma[j] + beta[j]);
        if (row < b && c.on) store_piece<V>(y + c.plane * py.gs + row * py.ld + c.col, z);
    }
}

// ---- backward --------------------------------------------------------------------------------------------
// dz = dy act'(z) for a lane's columns in a graph.  Which side of zero z = a x + b lies on is decided as in 64 bits (in 32 one value in ten million falls on the other
// one): with x' = sign(a) x it is above where x' > -b / |a|, and so where x' is above the largest float that is not above -b / |a|, one comparison.
// 500k x 256 16-bit values, sums and gradient: 110 and 133 us with it, 117 and 146 with z in 64 bits, 92 and 127 without an activation (before the sums had four
// waves a SIMD).
__device__ __forceinline__ float float_below(double v) {               // the largest that is not above
    const float f = (float)v;
    if (!((double)f > v)) return f;
    const uint32_t u = __float_as_uint(f);
    return __uint_as_float(f > 0.0f ? u - 1 : f < 0.0f ? u + 1 : 0x80000001u);
}
template <int V, int ACT>
struct BeforeActivation {
    float edge[ACT == GSR_ACT_RELU ? V : 1];
    uint32_t sign[ACT == GSR_ACT_RELU ? V : 1];
    template <typename S>
    __device__ __forceinline__ BeforeActivation(const S& m, const S& rs, const float (&gamma)[V], const float (&beta)[V]) {
        if constexpr (ACT == GSR_ACT_RELU) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const double a = (double)rs[j] * (double)gamma[j], b = fma(-(double)m[j], a, (double)beta[j]);
                sign[j] = a < 0.0 ? 0x80000000u : 0u;
                edge[j] = a == 0.0 ? (b > 0.0 ? -INFINITY : INFINITY) : float_below(-b / fabs(a));
            }
        }
    }
    // (a NaN comes to 0 here and is one again when it meets xh)
    __device__ __forceinline__ float operator()(int j, float dy, float x, float xh, const float (&gamma)[V], const float (&beta)[V]) const {
        if constexpr (ACT == GSR_ACT_RELU) {
            return __uint_as_float(__float_as_uint(x) ^ sign[j]) > edge[j] ? dy : 0.0f;
        } else if constexpr (ACT == GSR_ACT_SILU) {
            const float z = xh * gamma[j] + beta[j], l = logistic(z);
            return dy * (l * (1.0f + z * (1.0f - l)));
        } else {
            return dy;
        }
    }
};

// Sums of a chunk in 32 bits (`rows` of a column at most), joined in 64.  columns: [workgroups][2][d], sums of dz xh and of dz.
// 1M x 256 floats from a checkpoint, silu, 258 us, 5.0 TB/s; 500k x 256 16-bit values, relu, 98 us, 5.3 TB/s (110 with the columns' sums in registers, which left
// room for three waves a SIMD; fewer selects or more rows in flight change nothing).
template <typename T, int V, bool TAIL, int ACT, typename Source>
__global__ __launch_bounds__(256) void k_norm_grad_sums(NormShape s, GraphRows g, const T* __restrict__ dy, RowPlane pd, Source source, Affine f,
                                                        double2* __restrict__ pieces, float* __restrict__ columns) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int slab = blockIdx.y;
    const LaneColumns c = lane_columns<V>(s, slab);
    __shared__ float s_col[4][2][V][64];            // every lane's sums of its columns over the graphs: in registers they would leave room for fewer waves
    const int lane = lane_id();
    float (&all)[2][V][64] = s_col[threadIdx.x >> 6];
#pragma unroll
    for (int j = 0; j < V; ++j) all[0][j][lane] = all[1][j][lane] = 0.0f;
    if (w < s.chunks) {
        float gamma[V], beta[V];
        load_affine<V>(f.gamma, c, 1.0f, gamma);
        load_affine<V>(f.beta, c, 0.0f, beta);
        over_graphs(s, g, w, [&](int64_t graph, int64_t a, int64_t b) {
            constexpr int U = 2;
            const int64_t at = graph * s.groups + (c.on ? c.group : 0);
            const ByGroup<V, TAIL> m(c, f.mean, at), rs(c, f.rstd, at);
            const BeforeActivation<V, ACT> before(m, rs, gamma, beta);
            float sum_x[V], sum_z[V];
#pragma unroll
            for (int j = 0; j < V; ++j) sum_x[j] = sum_z[j] = 0.0f;
            for (int64_t r = a; r < b; r += U * c.subs) {
                PlaneSource<T, V, false> e[U];
                Source q[U];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int64_t row = r + k * c.subs + c.sub, have = row < b ? row : a;
                    e[k].x = dy;
                    e[k].p = pd;
                    e[k].load(s, c, have);
                    q[k] = source;
                    q[k].load(s, c, have);
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const bool in = r + k * c.subs + c.sub < b;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float x = q[k].at(j), xh = (x - m[j]) * rs[j];
                        const float dz = before(j, e[k].at(j), x, xh, gamma, beta);
                        const bool counts = in && !(TAIL && j < c.skip);
                        sum_z[j] += counts ? dz : 0.0f;
                        sum_x[j] += counts ? dz * xh : 0.0f;
                    }
                }
            }
            double u = 0.0, v = 0.0, u2 = 0.0, v2 = 0.0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool next = TAIL && j >= c.split;
                const double z = (double)gamma[j] * (double)sum_z[j], x = (double)gamma[j] * (double)sum_x[j];
                u += next ? 0.0 : z;
                v += next ? 0.0 : x;
                u2 += next ? z : 0.0;
                v2 += next ? x : 0.0;
                all[0][j][lane] += sum_x[j];
                all[1][j][lane] += sum_z[j];
            }
            leave_piece<TAIL, V>(s, c, slab, w, graph, u, v, u2, v2, pieces);
        });
    }
    __syncthreads();
    const int lanes = 1 << s.lanes_log2, first = (slab % s.group_slabs) * lanes * V, plane = slab / s.group_slabs;
    for (int i = threadIdx.x; i < 2 * lanes * V; i += 256) {
        const int li = i & (lanes - 1), which = (i >> s.lanes_log2) / V, own = (i >> s.lanes_log2) % V, col = first + li * V + own;
        if (col >= s.dg) continue;
        const int begin = first + li * V, j = own + (TAIL && begin + V > s.dg ? begin + V - s.dg : 0);       // (the columns before a tail's own come first)
        double sum = 0.0;
        for (int l = li; l < 64; l += lanes)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum += (double)s_col[k][which][j][l];
        columns[((int64_t)blockIdx.x * 2 + which) * s.d + plane * s.dg + col] = (float)sum;
    }
}

// The first `task_wgs` workgroups join the pieces: means of h and of h xh of every (graph, group).  The others add up 16 columns of
// dgamma and dbeta each, with 64 threads a column.
template <int THREADS>
__global__ __launch_bounds__(1024) void k_norm_grad_join(NormShape s, GraphRows g, int V, const double2* __restrict__ pieces, int64_t task_blocks,
                                                        int64_t task_wgs, float2* __restrict__ means, const float* __restrict__ columns, int64_t parts,
                                                        float* __restrict__ dgamma, float* __restrict__ dbeta) {
    if ((int64_t)blockIdx.x < task_wgs) {
        for (int64_t block = blockIdx.x; block < task_blocks; block += task_wgs) {
            int64_t task, rows;
            double u, v;
            if (!joined<THREADS>(s, g, V, block, pieces, task, u, v, rows) || threadIdx.x % THREADS) continue;
            const double count = (double)rows * s.cg;
            means[task] = rows ? make_float2((float)(u / count), (float)(v / count)) : make_float2(0.0f, 0.0f);
        }
        return;
    }
    __shared__ double s_part[64][16];
    const int64_t block = blockIdx.x - task_wgs;
    const int col = (int)(block * 16 + (threadIdx.x & 15)), k = threadIdx.x >> 4;       // of 2 d: dgamma's columns, then dbeta's
    double sum = 0.0;
    if (col < 2 * s.d) {
        constexpr int U = 8;
        const float* from = columns + col;
        const int64_t stride = 2 * (int64_t)s.d;
        for (int64_t i = k; i < parts; i += 64 * U) {
            float t[U];
#pragma unroll
            for (int q = 0; q < U; ++q) t[q] = from[(i + 64 * q < parts ? i + 64 * q : i) * stride];
#pragma unroll
            for (int q = 0; q < U; ++q) sum += i + 64 * q < parts ? (double)t[q] : 0.0;
        }
    }
    s_part[k][threadIdx.x & 15] = sum;
    __syncthreads();
    if (threadIdx.x >= 16 || col >= 2 * s.d) return;
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < 64; ++i) sum += s_part[i][threadIdx.x];
    float* out = col < s.d ? dgamma : dbeta;
    if (out) out[col < s.d ? col : col - s.d] = (float)sum;
}

// Bound by its reads and writes: 1M x 256 floats from a checkpoint 371 us, 6.3 TB/s; 500k x 256 16-bit values 135 us, 5.7 TB/s.
template <typename T, int V, bool TAIL, int ACT, typename Source>
__global__ __launch_bounds__(256) void k_norm_grad_apply(NormShape s, GraphRows g, const T* dy, RowPlane pd, Source source, Affine f,
                                                         const float* __restrict__ means, T* dx, RowPlane px) {
    const int64_t w = s.chunks - 1 - ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6));        // backwards, as k_norm_apply
    if (w < 0) return;
    const LaneColumns c = lane_columns<V>(s, blockIdx.y);
    float gamma[V], beta[V];
    load_affine<V>(f.gamma, c, 1.0f, gamma);
    load_affine<V>(f.beta, c, 0.0f, beta);
    over_graphs(s, g, w, [&](int64_t graph, int64_t a, int64_t b) {
        constexpr int U = 2;
        const int64_t at = graph * s.groups + (c.on ? c.group : 0);
        const ByGroup<V, TAIL> m(c, f.mean, at), rs(c, f.rstd, at);
        const ByGroup<V, TAIL> m1(c, means, at, 2), m2(c, means + 1, at, 2);
        const BeforeActivation<V, ACT> before(m, rs, gamma, beta);
        for (int64_t r = a; r < b; r += U * c.subs) {
            PlaneSource<T, V, true> e[U];
            Source q[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t row = r + k * c.subs + c.sub, have = row < b ? row : a;
                e[k].x = dy;
                e[k].p = pd;
                e[k].load(s, c, have);
                q[k] = source;
                q[k].load(s, c, have);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int64_t row = r + k * c.subs + c.sub;
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float x = q[k].at(j), xh = (x - m[j]) * rs[j];
                    const float dz = before(j, e[k].at(j), x, xh, gamma, beta);
                    v[j] = rs[j] * (gamma[j] * dz - m1[j] - xh * m2[j]);
                }
                if (row < b && c.on) store_piece<V, true>(dx + c.plane * px.gs + row * px.ld + c.col, v);
            }
        }
    });
}

// k_norm_small's counterpart.  One workgroup of a slab also writes the gradients of gamma and beta.
template <typename T, int V, int ACT, typename Source>
__global__ __launch_bounds__(1024) void k_norm_grad_small(NormShape s, GraphRows g, const T* dy, RowPlane pd, Source source, Affine f, T* dx, RowPlane px,
                                                          float* __restrict__ dgamma, float* __restrict__ dbeta) {
    const int slab = blockIdx.y, wave = threadIdx.x >> 6;
    const LaneColumns c = lane_columns<V>(s, slab);
    const int64_t a = g.at(0), b = g.at(1) > a ? g.at(1) : a;
    float gamma[V], beta[V];
    load_affine<V>(f.gamma, c, 1.0f, gamma);
    load_affine<V>(f.beta, c, 0.0f, beta);
    const int group = c.on ? c.group : 0;
    const ByGroup<V, false> m(c, f.mean, group), rs(c, f.rstd, group);
    const BeforeActivation<V, ACT> before(m, rs, gamma, beta);
    float sum_x[V], sum_z[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum_x[j] = sum_z[j] = 0.0f;
    constexpr int U = 2;
    for (int64_t r = a + (int64_t)wave * U * c.subs; r < b; r += 16 * U * c.subs) {
        PlaneSource<T, V, false> e[U];
        Source q[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t row = r + k * c.subs + c.sub, have = row < b ? row : a;
            e[k].x = dy;
            e[k].p = pd;
            e[k].load(s, c, have);
            q[k] = source;
            q[k].load(s, c, have);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const bool in = r + k * c.subs + c.sub < b;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float x = q[k].at(j), xh = (x - m[j]) * rs[j], dz = before(j, e[k].at(j), x, xh, gamma, beta);
                sum_z[j] += in ? dz : 0.0f;
                sum_x[j] += in ? dz * xh : 0.0f;
            }
        }
    }
    double u = 0.0, v = 0.0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        u = fma((double)gamma[j], (double)sum_z[j], u);
        v = fma((double)gamma[j], (double)sum_x[j], v);
    }
    __shared__ float s_col[16][2][64 * V];
    const int lanes = 1 << s.lanes_log2, li = lane_id() & (lanes - 1);
    if (blockIdx.x == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            for (int o = lanes; o < 64; o <<= 1) {
                sum_x[j] += __shfl_xor(sum_x[j], o);
                sum_z[j] += __shfl_xor(sum_z[j], o);
            }
            if (c.sub == 0) {
                s_col[wave][0][li * V + j] = sum_x[j];
                s_col[wave][1][li * V + j] = sum_z[j];
            }
        }
    }
    const double2 t = small_total(s, c, u, v);              // (meets the other waves)
    if (blockIdx.x == 0) {
        const int first = (slab % s.group_slabs) * lanes * V, plane = slab / s.group_slabs;
        for (int i = threadIdx.x; i < 2 * lanes * V; i += 1024) {
            const int which = i >= lanes * V, k = which ? i - lanes * V : i;
            float* out = which ? dbeta : dgamma;
            if (first + k >= s.dg || !out) continue;
            double sum = 0.0;
            for (int w = 0; w < 16; ++w) sum += (double)s_col[w][which][k];
            out[plane * s.dg + first + k] = (float)sum;
        }
    }
    const double count = (double)(b - a) * s.cg;
    const float m1 = (float)(t.x / count), m2 = (float)(t.y / count);           // (an empty graph has no rows to use them)
    for (int64_t r = a + ((int64_t)blockIdx.x * 16 + wave) * c.subs; r < b; r += (int64_t)gridDim.x * 16 * c.subs) {
        const int64_t row = r + c.sub, have = row < b ? row : a;
        PlaneSource<T, V, false> e;
        e.x = dy;
        e.p = pd;
        e.load(s, c, have);
        Source q = source;
        q.load(s, c, have);
        float w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float x = q.at(j), xh = (x - m[j]) * rs[j], dz = before(j, e.at(j), x, xh, gamma, beta);
            w[j] = rs[j] * (gamma[j] * dz - m1 - xh * m2);
        }
        if (row < b && c.on) store_piece<V>(dx + c.plane * px.gs + row * px.ld + c.col, w);
    }
}

// ---- checkpoints by themselves -----------------------------------------------------------------------------
// 1M x 256 floats: 214 us to save, 220 to load, 6.1 and 5.9 TB/s.  250k x 385 16-bit values 86 and 66, 3.5 and 4.6 TB/s: rows of odd width share lines.
template <typename T, int V, bool TAIL>
__global__ __launch_bounds__(256) void k_checkpoint_save(NormShape s, const T* __restrict__ x, RowPlane p, Checkpoint ck) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= s.chunks) return;
    const LaneColumns c = lane_columns<V>(s, blockIdx.y);
    const int64_t a = w * s.rows, b = a + s.rows < s.n ? a + s.rows : s.n;
    constexpr int U = 4;
    for (int64_t r = a; r < b; r += U * c.subs) {
        PlaneSource<T, V, true> q[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t row = r + k * c.subs + c.sub;
            q[k].x = x;
            q[k].p = p;
            q[k].load(s, c, row < b ? row : a);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t row = r + k * c.subs + c.sub;
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = q[k].at(j);
            save_piece<V, TAIL>(ck, s, c, row, row < b, v);
        }
    }
}
template <typename T, int V, bool TAIL>
__global__ __launch_bounds__(256) void k_checkpoint_load(NormShape s, Checkpoint ck, T* __restrict__ x, RowPlane p) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= s.chunks) return;
    const LaneColumns c = lane_columns<V>(s, blockIdx.y);
    const int64_t a = w * s.rows, b = a + s.rows < s.n ? a + s.rows : s.n;
    constexpr int U = 4;
    for (int64_t r = a; r < b; r += U * c.subs) {
        CodeSource<V, TAIL> q[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t row = r + k * c.subs + c.sub;
            q[k].k = ck;
            q[k].load(s, c, row < b ? row : a);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t row = r + k * c.subs + c.sub;
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = q[k].at(j);
            if (row < b && c.on) store_piece<V, true>(x + c.plane * p.gs + row * p.ld + c.col, v);
        }
    }
}

// ---- host side ---------------------------------------------------------------------------------------------
namespace {

constexpr int kMaxWidth = 131072;
constexpr int64_t kMaxPieces = (int64_t)1 << 31;

bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// Rows of a wave: as many as make kChunks waves of all slabs together; at most kMaxRows, and eight pieces of every lane at least, two where a wave would meet many
// graphs, which take their turns.
constexpr int64_t kChunks = 4096, kMaxRows = 1024;
int64_t least_rows(const NormShape& s, int64_t graphs) { return (graphs > 1 ? 2 : 8) * (64 >> s.lanes_log2); }

// Pieces of 16 bytes of the plane's type, but for groups or planes narrower than that; with a tail, single columns in place, where the last piece of a row overlaps
// the one before it, whose lane may have stored already.  480k x 136 16-bit values in eight groups of 17, relu, in pieces and in single
// columns: forward 48 and 98 us, sums of the gradient 79 and 300, gradient 118 and 207.
struct PieceRule {
    int v;
    bool tail;
};
PieceRule piece_of(int32_t dg, int32_t cg, int32_t dtype, bool in_place) {
    const int v = dtype == GSR_BF16 ? 8 : 4;
    if (dg % v == 0 && cg % v == 0) return {v, false};
    if (dg > v && cg >= v && !in_place) return {v, true};
    return {1, false};
}
NormShape norm_shape(int64_t n, int64_t graphs, int32_t d, int32_t planes, int32_t groups, int32_t dtype, int V) {
    NormShape s{};
    s.n = n;
    s.d = d;
    s.dg = d / planes;
    s.groups = groups;
    s.cg = d / groups;
    const int pieces = (s.dg + V - 1) / V;
    // as few idle lanes as can be, or up to a quarter more for longer rows, twice as many where slabs would share lines of memory; a block of a checkpoint
    // in one slab.  480k x 136 16-bit values in one slab of 32 lanes against three of 8: forward 43 and 145 us.
    auto lanes_for = [&](int k) { return (((pieces - 1) >> k) + 1) << k; };
    auto fits = [&](int k) { return (V << k) % kBlock == 0 || (V << k) >= s.dg; };
    int least = 1 << 30;
    for (int k = 2; k <= 6; ++k) if (fits(k)) least = std::min(least, lanes_for(k));
    const int most = s.dg * (int)dtype_size(dtype) % 128 ? 2 * least : least + least / 4;
    for (int k = 2; k <= 6; ++k) if (fits(k) && lanes_for(k) <= most) s.lanes_log2 = k;
    s.group_slabs = lanes_for(s.lanes_log2) >> s.lanes_log2;
    s.slabs = s.group_slabs * planes;
    s.rows = (int32_t)std::min(kMaxRows, std::max(least_rows(s, graphs), (n * s.slabs + kChunks - 1) / kChunks));
    s.chunks = (n + s.rows - 1) / s.rows;
    return s;
}
int planes_of(int32_t c, int32_t layout) { return layout == GSR_LAYOUT_GROUP_PLANAR ? c : 1; }

gsr_status_t plane_shape(int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype) {
    if (n < 0) return fail(GSR_ERR_INVALID_ARG, "negative n");
    if (n >= ((int64_t)1 << 31)) return fail(GSR_ERR_UNSUPPORTED, "n=%lld at or above 2^31", (long long)n);
    if (d < 1 || d > kMaxWidth) return fail(GSR_ERR_UNSUPPORTED, "d=%d outside [1, %d]", d, kMaxWidth);
    if (c < 1 || d % c) return fail(GSR_ERR_UNSUPPORTED, "c=%d does not divide d=%d", c, d);
    if (layout != GSR_LAYOUT_ROW_MAJOR && layout != GSR_LAYOUT_GROUP_PLANAR) return fail(GSR_ERR_INVALID_ARG, "layout %d", layout);
    if (dtype != GSR_F32 && dtype != GSR_BF16) return fail(GSR_ERR_UNSUPPORTED, "dtype %d", dtype);
    if (planes_of(c, layout) > 4096) return fail(GSR_ERR_UNSUPPORTED, "c=%d above 4096", c);
    return GSR_OK;
}
gsr_status_t row_plane(const char* name, const void* at, int64_t n, int32_t dg, int64_t ld, int32_t dtype, RowPlane* p) {
    if (ld < dg || ld >= ((int64_t)1 << 31)) return fail(GSR_ERR_INVALID_ARG, "row stride %lld of %s outside [%d, 2^31)", (long long)ld, name, dg);
    if (n > 0 && !at) return fail(GSR_ERR_INVALID_ARG, "%s is null", name);
    if (!aligned_to(at, dtype_size(dtype))) return fail(GSR_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    p->ld = ld;
    p->gs = n * ld;
    return GSR_OK;
}
gsr_status_t checkpoint_of(int64_t n, int32_t dg, const int8_t* codes, const float* scales, Checkpoint* k) {
    if (n > 0 && (!codes || !scales)) return fail(GSR_ERR_INVALID_ARG, "null codes or scales");
    if (!aligned_to(codes, 4) || !aligned_to(scales, 4)) return fail(GSR_ERR_INVALID_ARG, "codes or scales not aligned to 4 bytes");
    k->codes = const_cast<int8_t*>(codes);
    k->scales = const_cast<float*>(scales);
    k->blocks = (dg + kBlock - 1) / kBlock;
    return GSR_OK;
}
gsr_status_t graph_rows(const void* graph_ptr, int32_t ptr_i64, int64_t graphs, int64_t n, GraphRows* g) {
    if (graphs < 0) return fail(GSR_ERR_INVALID_ARG, "negative number of graphs");
    if (graphs >= ((int64_t)1 << 31)) return fail(GSR_ERR_UNSUPPORTED, "%lld graphs", (long long)graphs);
    if (!graph_ptr && graphs != 1) return fail(GSR_ERR_INVALID_ARG, "%lld graphs without their first rows", (long long)graphs);
    if (!aligned_to(graph_ptr, ptr_i64 ? 8 : 4)) return fail(GSR_ERR_INVALID_ARG, "graph_ptr is not aligned to its elements");
    *g = GraphRows{graph_ptr, ptr_i64, graphs, n};
    return GSR_OK;
}
gsr_status_t norm_args(int32_t d, int32_t groups, int32_t act, const float* gamma, const float* beta, const float* mean, const float* rstd,
                       int64_t graphs) {
    if (groups < 1 || groups > d || d % groups) return fail(GSR_ERR_UNSUPPORTED, "%d groups do not divide d=%d", groups, d);
    if (act != GSR_ACT_NONE && act != GSR_ACT_RELU && act != GSR_ACT_SILU) return fail(GSR_ERR_UNSUPPORTED, "activation %d", act);
    if (graphs > 0 && (!mean || !rstd)) return fail(GSR_ERR_INVALID_ARG, "null mean or rstd");
    if (!aligned_to(gamma, 4) || !aligned_to(beta, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return fail(GSR_ERR_INVALID_ARG, "gamma, beta, mean or rstd is not aligned to its elements");
    return GSR_OK;
}

// The workspace of both directions: pieces; what the sums of every (graph, group) are taken from, or in the gradient its means; the columns' partial sums.
struct NormWs {
    size_t pieces, means, columns, total;
    int threads;                    // for a (graph, group) in the join
    int64_t task_blocks, task_wgs;
};
NormWs carve_norm(const NormShape& s, int64_t graphs) {
    NormWs w{};
    w.pieces = 0;
    // at least as many chunks as any number of rows up to n has, so that a workspace serves them all
    const int64_t chunks = std::max((s.n + kMaxRows - 1) / kMaxRows, std::min((s.n + least_rows(s, graphs) - 1) / least_rows(s, graphs), kChunks / s.slabs + 1));
    w.means = align_up((size_t)(chunks + graphs) * s.stride() * sizeof(double2));
    w.columns = w.means + align_up((size_t)graphs * s.groups * sizeof(float2));
    w.total = w.columns + align_up((size_t)((chunks + 3) / 4) * 2 * s.d * 4);
    // (301 graphs of 32 groups, 500k x 256 16-bit values: the join 7.9 us with 16 threads, 13.7 with waves)
    w.threads = s.chunks > 64 * graphs ? 1024 : s.chunks > 32 * graphs ? 64 : 16;
    const int64_t tasks = graphs * s.groups;
    w.task_blocks = (tasks * w.threads + 1023) / 1024;
    w.task_wgs = std::min<int64_t>(w.task_blocks, 1 << 20);
    return w;
}
gsr_status_t workspace_of(const NormWs& w, const NormShape& s, int64_t graphs, void* workspace, size_t bytes) {
    if ((s.chunks + graphs) * s.stride() >= kMaxPieces || graphs * s.groups >= kMaxPieces)
        return fail(GSR_ERR_UNSUPPORTED, "%lld graphs of %d groups", (long long)graphs, s.groups);
    if (bytes < w.total) return fail(GSR_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", bytes, w.total);
    if ((w.total && !workspace) || !aligned_to(workspace, 16)) return fail(GSR_ERR_INVALID_ARG, "workspace null or not aligned to 16 bytes");
    return GSR_OK;
}

// A pass that leaves no sums takes eight pieces of every lane a wave, so that the waves at work lie close together in memory, and with offsets to
// look up 16.  1M x 256 floats with 2,048 waves of a plane / 8 / 16 pieces: forward with a checkpoint 517 / 391 / 403 us, gradient from it 527 / 399 / 419,
// save 336 / 297 / 313; 500k x 256 16-bit values in 301 graphs, gradient: 143 / 154 / 144.
// Fewer where that would make less than 2,048 waves (and fewer rows for the waves that leave sums): 524 rows of 381 floats, each its own graph, gradient
// 59 -> 24 us; 3,960 rows of 96 in 635 graphs, forward 57 -> 29.
NormShape apply_shape(NormShape s, const void* graph_ptr) {
    const int64_t subs = 64 >> s.lanes_log2, most = graph_ptr ? 16 : 8, least = graph_ptr ? 1 : 4, even = s.n * s.slabs / (2048 * subs);
    s.rows = (int32_t)(std::max(std::min(most, std::max(least, even)), (s.n >> 25) / subs + 1) * subs);            // (a grid holds fewer than 2^32 threads)
    s.chunks = (s.n + s.rows - 1) / s.rows;
    return s;
}
// Workgroups for a slab of a graph that takes one launch, or 0: a workgroup takes its slab's rows by rounds of 16 waves, 16 rounds at most and 32 of single columns.
// One launch against three, silu, in a captured graph.  Floats, 64 columns in two groups, 8 rounds (512 rows): 8.0 us / 11.6, gradient 10.3 / 13.3; 16: 10.1 / 11.6
// and 14.4 / 13.4; 32: 14.4 / 10.6 and 22.7 / 12.0.  One column, 16 rounds (4,096 rows): 9.3 / 9.6 and 11.4 / 10.4; 64: 22.8 / 11.2 and 33.0 / 12.3.  64 columns, each
// its own group, 32 rounds (512 rows): 10.3 / 12.7 and 12.2 / 12.8; 64: 14.9 / 12.1 and 19.6 / 12.8.  Called from Python, where launches wait for the host: 2,000 rows of
// 32 floats in two planes, 16 rounds, 12.2 / 16.4 and 13.7 / 18.2, 4,000 rows 12.8 / 16.4 and 20.2 / 18.2.
constexpr int kSmallShares = 32, kSmallRounds = 16, kSmallColumnRounds = 32;
unsigned small_shares(const NormShape& s, const PieceRule& rule, int64_t graphs, bool in_place) {
    const int width = rule.v << s.lanes_log2, rows = 16 * (64 >> s.lanes_log2);
    const bool whole = s.dg % s.cg == 0 && (s.group_slabs == 1 || width % s.cg == 0);
    if (graphs != 1 || rule.tail || !whole || s.n < 1 || s.n > (int64_t)rows * (rule.v == 1 ? kSmallColumnRounds : kSmallRounds)) return 0;
    if (in_place) return 1;                     // others would read what it has written
    return (unsigned)std::min<int64_t>(kSmallShares, (s.n + rows - 1) / rows);
}
dim3 rows_grid(const NormShape& s) { return dim3((unsigned)((s.chunks + 3) / 4), (unsigned)s.slabs); }

// call(T{}, integral_constant<V>, bool_constant<TAIL>) for the storage type and piece
template <typename T, int W, typename Call>
void by_tail(const PieceRule& r, Call call) {
    if (r.tail) call(T{}, std::integral_constant<int, W>{}, std::true_type{});
    else if (r.v == W) call(T{}, std::integral_constant<int, W>{}, std::false_type{});
    else call(T{}, std::integral_constant<int, 1>{}, std::false_type{});
}
template <typename Call>
void by_piece(int32_t dtype, const PieceRule& r, Call call) {
    if (dtype == GSR_F32) by_tail<float, 4>(r, call);
    else by_tail<bf16_t, 8>(r, call);
}
template <typename Call>
void by_threads(int threads, Call call) {
    if (threads == 1024) call(std::integral_constant<int, 1024>{});
    else if (threads == 64) call(std::integral_constant<int, 64>{});
    else call(std::integral_constant<int, 16>{});
}
template <typename Call>
void by_activation(int32_t act, Call call) {
    if (act == GSR_ACT_RELU) call(std::integral_constant<int, GSR_ACT_RELU>{});
    else if (act == GSR_ACT_SILU) call(std::integral_constant<int, GSR_ACT_SILU>{});
    else call(std::integral_constant<int, GSR_ACT_NONE>{});
}

}  // namespace
}  // namespace gsr

using namespace gsr;

extern "C" {

size_t gsr_group_norm_workspace(int64_t n, int64_t graphs, int32_t d, int32_t c, int32_t layout, int32_t dtype, int32_t groups) {
    if (plane_shape(n, d, c, layout, dtype) != GSR_OK || graphs < 0 || graphs >= ((int64_t)1 << 31) || groups < 1 || groups > d || d % groups) return 0;
    const int planes = planes_of(c, layout);
    // in place, single columns may take the place of pieces
    size_t bytes = 0;
    for (bool in_place : {false, true})
        bytes = std::max(bytes, carve_norm(norm_shape(n, graphs, d, planes, groups, dtype, piece_of(d / planes, d / groups, dtype, in_place).v), graphs).total);
    return bytes;
}

gsr_status_t gsr_group_norm(const void* x, int64_t ldx, int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype, const void* graph_ptr,
                            int32_t ptr_i64, int64_t graphs, int32_t groups, const float* gamma, const float* beta, float eps, int32_t act,
                            void* y_out, int64_t ldy, float* mean_out, float* rstd_out, int8_t* codes_out, float* scales_out, void* workspace,
                            size_t workspace_bytes, void* stream) {
    GSR_TRY(plane_shape(n, d, c, layout, dtype));
    const int planes = planes_of(c, layout), dg = d / planes;
    RowPlane px, py;
    GraphRows g;
    Checkpoint ck{};
    GSR_TRY(row_plane("x", x, n, dg, ldx, dtype, &px));
    GSR_TRY(row_plane("y_out", y_out, n, dg, ldy, dtype, &py));
    GSR_TRY(graph_rows(graph_ptr, ptr_i64, graphs, n, &g));
    GSR_TRY(norm_args(d, groups, act, gamma, beta, mean_out, rstd_out, graphs));
    if (!(eps > 0.0f) || std::isinf(eps)) return fail(GSR_ERR_INVALID_ARG, "eps=%g is not a positive number", (double)eps);
    if (x == y_out && ldx != ldy) return fail(GSR_ERR_INVALID_ARG, "in place, but with row strides of %lld and %lld", (long long)ldx, (long long)ldy);
    const bool save = codes_out || scales_out;
    if (save) GSR_TRY(checkpoint_of(n, dg, codes_out, scales_out, &ck));
    const PieceRule rule = piece_of(dg, d / groups, dtype, x == y_out);
    const int V = rule.v;
    const NormShape s = norm_shape(n, graphs, d, planes, groups, dtype, V);
    const NormWs ws = carve_norm(s, graphs);
    GSR_TRY(workspace_of(ws, s, graphs, workspace, workspace_bytes));
    if (graphs == 0) return GSR_OK;
    hipStream_t st = (hipStream_t)stream;
    double2* pieces = (double2*)((char*)workspace + ws.pieces);
    float* shifts = (float*)((char*)workspace + ws.means);
    by_piece(dtype, rule, [&](auto t, auto v, auto tail) {
        using T = decltype(t);
        constexpr int P = v.value;
        if (const unsigned shares = small_shares(s, rule, graphs, x == y_out)) {
            const dim3 grid(shares, (unsigned)s.slabs);
            by_activation(act, [&](auto a) {
                if (save)
                    hipLaunchKernelGGL((k_norm_small<T, P, a.value, true>), grid, dim3(1024), 0, st, s, g, (const T*)x, px, gamma, beta, (double)eps, mean_out,
                                       rstd_out, (T*)y_out, py, ck);
                else
                    hipLaunchKernelGGL((k_norm_small<T, P, a.value, false>), grid, dim3(1024), 0, st, s, g, (const T*)x, px, gamma, beta, (double)eps, mean_out,
                                       rstd_out, (T*)y_out, py, ck);
            });
            return;
        }
        if (n) hipLaunchKernelGGL((k_norm_sums<T, P, tail.value>), rows_grid(s), dim3(256), 0, st, s, g, (const T*)x, px, pieces, shifts);
        by_threads(ws.threads, [&](auto k) {
            hipLaunchKernelGGL((k_norm_join<k.value>), dim3((unsigned)ws.task_wgs), dim3(1024), 0, st, s, g, V, pieces, shifts, ws.task_blocks, (double)eps, mean_out, rstd_out);
        });
        if (!n) return;
        const Affine f{gamma, beta, mean_out, rstd_out};
        const NormShape q = apply_shape(s, graph_ptr);
        by_activation(act, [&](auto a) {
            if (save) hipLaunchKernelGGL((k_norm_apply<T, P, tail.value, a.value, true>), rows_grid(q), dim3(256), 0, st, q, g, (const T*)x, px, f, (T*)y_out, py, ck);
            else hipLaunchKernelGGL((k_norm_apply<T, P, tail.value, a.value, false>), rows_grid(q), dim3(256), 0, st, q, g, (const T*)x, px, f, (T*)y_out, py, ck);
        });
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

gsr_status_t gsr_group_norm_grad(const void* dy, int64_t lddy, const void* x, int64_t ldx, const int8_t* codes, const float* scales, int64_t n,
                                 int32_t d, int32_t c, int32_t layout, int32_t dtype, const void* graph_ptr, int32_t ptr_i64, int64_t graphs,
                                 int32_t groups, const float* mean, const float* rstd, const float* gamma, const float* beta, int32_t act,
                                 void* dx_out, int64_t lddx, float* dgamma_out, float* dbeta_out, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    GSR_TRY(plane_shape(n, d, c, layout, dtype));
    const int planes = planes_of(c, layout), dg = d / planes;
    RowPlane pd, px{}, po;
    GraphRows g;
    Checkpoint ck{};
    const bool coded = codes || scales;
    if (coded && x) return fail(GSR_ERR_INVALID_ARG, "x and its checkpoint");
    GSR_TRY(row_plane("dy", dy, n, dg, lddy, dtype, &pd));
    if (coded) GSR_TRY(checkpoint_of(n, dg, codes, scales, &ck));
    else GSR_TRY(row_plane("x", x, n, dg, ldx, dtype, &px));
    GSR_TRY(row_plane("dx_out", dx_out, n, dg, lddx, dtype, &po));
    GSR_TRY(graph_rows(graph_ptr, ptr_i64, graphs, n, &g));
    GSR_TRY(norm_args(d, groups, act, gamma, beta, mean, rstd, graphs));
    if (!aligned_to(dgamma_out, 4) || !aligned_to(dbeta_out, 4)) return fail(GSR_ERR_INVALID_ARG, "dgamma_out or dbeta_out is not aligned to its elements");
    if (x && x == dx_out) return fail(GSR_ERR_INVALID_ARG, "dx_out is x, whose rows are read again while it is written");
    if (dy == dx_out && lddy != lddx) return fail(GSR_ERR_INVALID_ARG, "in place, but with row strides of %lld and %lld", (long long)lddy, (long long)lddx);
    const PieceRule rule = piece_of(dg, d / groups, dtype, dy == dx_out);
    const int V = rule.v;
    const NormShape s = norm_shape(n, graphs, d, planes, groups, dtype, V);
    const NormWs ws = carve_norm(s, graphs);
    GSR_TRY(workspace_of(ws, s, graphs, workspace, workspace_bytes));
    hipStream_t st = (hipStream_t)stream;
    double2* pieces = (double2*)((char*)workspace + ws.pieces);
    float2* means = (float2*)((char*)workspace + ws.means);
    float* columns = (float*)((char*)workspace + ws.columns);
    const Affine f{gamma, beta, mean, rstd};
    const NormShape q = apply_shape(s, graph_ptr);
    auto both = [&](auto t, auto v, auto tail, auto a, auto source) {
        using T = decltype(t);
        using Source = decltype(source);
        constexpr int P = v.value, ACT = a.value;
        if (const unsigned shares = small_shares(s, rule, graphs, dy == dx_out)) {
            if constexpr (!tail.value)
                hipLaunchKernelGGL((k_norm_grad_small<T, P, ACT, Source>), dim3(shares, (unsigned)s.slabs), dim3(1024), 0, st, s, g, (const T*)dy, pd, source, f,
                                   (T*)dx_out, po, dgamma_out, dbeta_out);
            return;
        }
        if (n) hipLaunchKernelGGL((k_norm_grad_sums<T, P, tail.value, ACT, Source>), rows_grid(s), dim3(256), 0, st, s, g, (const T*)dy, pd, source, f, pieces, columns);
        const int64_t column_blocks = dgamma_out || dbeta_out ? (2 * (int64_t)d + 15) / 16 : 0;
        const dim3 grid((unsigned)(ws.task_wgs + column_blocks));
        const int64_t parts = (s.chunks + 3) / 4;
        if (grid.x)
            by_threads(ws.threads, [&](auto k) {
                hipLaunchKernelGGL((k_norm_grad_join<k.value>), grid, dim3(1024), 0, st, s, g, V, pieces, ws.task_blocks, ws.task_wgs, means, columns, parts, dgamma_out, dbeta_out);
            });
        if (n && graphs) hipLaunchKernelGGL((k_norm_grad_apply<T, P, tail.value, ACT, Source>), rows_grid(q), dim3(256), 0, st, q, g, (const T*)dy, pd, source, f, (const float*)means, (T*)dx_out, po);
    };
    by_piece(dtype, rule, [&](auto t, auto v, auto tail) {
        using T = decltype(t);
        constexpr int P = v.value;
        by_activation(act, [&](auto a) {
            if (coded) both(t, v, tail, a, CodeSource<P, tail.value>{ck});
            else both(t, v, tail, a, PlaneSource<T, P, false>{(const T*)x, px, {}});
        });
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

gsr_status_t gsr_checkpoint_save(const void* x, int64_t ldx, int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype, int8_t* codes_out,
                                 float* scales_out, void* stream) {
    GSR_TRY(plane_shape(n, d, c, layout, dtype));
    const int planes = planes_of(c, layout), dg = d / planes;
    RowPlane p;
    Checkpoint ck;
    GSR_TRY(row_plane("x", x, n, dg, ldx, dtype, &p));
    GSR_TRY(checkpoint_of(n, dg, codes_out, scales_out, &ck));
    if (n == 0) return GSR_OK;
    const PieceRule rule = piece_of(dg, dg, dtype, false);
    const NormShape s = apply_shape(norm_shape(n, 1, d, planes, 1, dtype, rule.v), nullptr);
    by_piece(dtype, rule, [&](auto t, auto v, auto tail) {
        using T = decltype(t);
        hipLaunchKernelGGL((k_checkpoint_save<T, v.value, tail.value>), rows_grid(s), dim3(256), 0, (hipStream_t)stream, s, (const T*)x, p, ck);
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

gsr_status_t gsr_checkpoint_load(const int8_t* codes, const float* scales, int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype,
                                 void* x_out, int64_t ldx, void* stream) {
    GSR_TRY(plane_shape(n, d, c, layout, dtype));
    const int planes = planes_of(c, layout), dg = d / planes;
    RowPlane p;
    Checkpoint ck;
    GSR_TRY(row_plane("x_out", x_out, n, dg, ldx, dtype, &p));
    GSR_TRY(checkpoint_of(n, dg, codes, scales, &ck));
    if (n == 0) return GSR_OK;
    const PieceRule rule = piece_of(dg, dg, dtype, false);
    const NormShape s = apply_shape(norm_shape(n, 1, d, planes, 1, dtype, rule.v), nullptr);
    by_piece(dtype, rule, [&](auto t, auto v, auto tail) {
        using T = decltype(t);
        hipLaunchKernelGGL((k_checkpoint_load<T, v.value, tail.value>), rows_grid(s), dim3(256), 0, (hipStream_t)stream, s, ck, (T*)x_out, p);
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

}  // extern "C"
