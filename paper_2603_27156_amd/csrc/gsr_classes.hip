// Softmax cross entropy of a linear head over many classes, without its logits, and its gradient.
//
//   z_ij = x_i . E_j + b_j        lse_i = log sum_j exp z_ij        loss = mean over the rows with a class of lse_i - z_i,t_i
//   dz_ij = (exp(z_ij - lse_i) - [j = t_i]) scale / rows with a class;    dx = dz E,   dE = dz^T x,   db_j = sum_i dz_ij
//
// The n x classes logits exist only as 32-row tiles in the registers of the matrix cores.  A workgroup keeps a block of rows of one side
// (x or E) in registers, the other side streams through LDS in tiles of 32 rows, and of every tile the wave takes the products Z^T with its own
// rows, then exp, and, in the backward, a second product that adds dz times the streamed tile to its rows' gradients.  The accumulators of the first
// product hold a lane's row and four neighbouring streamed rows, which is how the second one wants its operand (the K index is permuted
// alike on both sides), so dz never leaves the registers.  dx and dE are the same kernel with the sides exchanged; each computes the logits anew.
//
// Operands are laid out once per call as the matrix instructions take them: rows in blocks of 16, columns in steps of 32, and of every (block, step)
// 64 pieces of 16 bytes in lane order, zeros behind the last row and column.  So tiles are copied to LDS as they lie, from any layout, stride and
// width.  bf16 planes go in as they are.  Floats go in as two fp16 pieces h + l of 11 bits each: every row is first multiplied by the power of two that
// brings its largest value to 2^14 .. 2^15, which keeps both pieces in fp16's range (what is left out is below 2^-22 of a value, or 2^-39 of the
// largest; a power for 32 rows together would let one row, such as a padding one, take the others' bits), and a product of floats is hh + hl + lh
// (l l is below 2^-24 of it), added up in float32.  Exact products of three bf16 pieces, which need no powers of two, are six:
// 8,191 x 4,099 at D = 384, gradients 708 us instead of 362.
#include "gsr_internal.h"
#include "gsr_pieces.h"

#include <algorithm>
#include <cmath>

namespace gsr {

constexpr int kMaxClassWidth = 512;
constexpr int kTileRows = 32;                   // streamed rows of a tile
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNoMax = -1.0e38f;              // a running maximum that no logit has reached; times log2 e it is finite

// ---- operands ------------------------------------------------------------------------------------------
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short frag8 __attribute__((ext_vector_type(8)));        // a lane's eight values of a step: bf16, or a piece in fp16
template <int NP>
__device__ __forceinline__ f32x4 mfma_frag(frag8 a, frag8 b, f32x4 c) {
    if constexpr (NP == 1) return mfma_k32(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

struct RowSource {              // rows of a plane, or of a table
    const void* at;
    int64_t rows, ld, gs;
    int32_t d, dg;
};
struct ClassTokens {
    const void* ids;
    int32_t i64, classes;
    __device__ __forceinline__ int32_t at(int64_t i) const {        // -1: none
        const int64_t t = i64 ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
        return t >= 0 && t < classes ? (int32_t)t : -1;
    }
};
// What a launch lays out.  Blocks of 256 threads: x, then E, then 1,024 rows' classes and lse each, then 1,024 biases each.
struct ClassSetup {
    RowSource x, e;
    ClassTokens ids;
    uint4 *xf, *ef;                 // in pieces
    float *x_scale, *e_scale;       // floats: the power of two that a row's pieces have to be multiplied by
    const float *lse, *bias;        // lse: NULL in the forward
    float *lse_out, *bias_out;      // of all rows that the kernels read, padded ones too
    int32_t *target, *counts;       // class of every row; rows with a class of every block
    int64_t x_pad, e_pad;           // rows laid out
    int32_t ks;
    unsigned x_blocks, e_blocks, row_blocks, bias_blocks;
};
// Columns col .. col + 7 of a row, zeros where there are none.
template <typename T>
__device__ __forceinline__ void load_eight(const RowSource& s, int64_t row, bool in, int col, float (&v)[8]) {
    if (s.dg % 8 == 0) {
        if (in && col < s.d) {
            const int plane = col / s.dg;
            Piece<T, 8> p;
            p.load(static_cast<const T*>(s.at) + plane * s.gs + row * s.ld + (col - plane * s.dg));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p.at(j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = col + j, plane = c / s.dg;
            v[j] = in && c < s.d ? to_float(static_cast<const T*>(s.at)[plane * s.gs + row * s.ld + (c - plane * s.dg)]) : 0.0f;
        }
    }
}
__device__ __forceinline__ uint32_t f16_bits(float v) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v)); }
// a float in two pieces
__device__ __forceinline__ void two_pieces(float v, uint32_t& h, uint32_t& l) {
    const _Float16 top = static_cast<_Float16>(v);
    h = __builtin_bit_cast(uint16_t, top);
    l = f16_bits(v - static_cast<float>(top));
}
// 16-bit rows: 16 pieces by a workgroup
constexpr int kPieces = 16;
__device__ __forceinline__ void lay_out(const RowSource& s, uint4* __restrict__ out, float*, int64_t pad, int ks, int64_t block, const ClassTokens* known, bf16_t) {
    const int lane = lane_id();
    float v[kPieces / 4][8];
#pragma unroll
    for (int i = 0; i < kPieces / 4; ++i) {
        const int64_t piece = block * kPieces + i * 4 + (threadIdx.x >> 6), row = piece / ks * 16 + (lane & 15);
        load_eight<bf16_t>(s, row, row < s.rows && (!known || known->at(row) >= 0), (int)(piece % ks) * 32 + (lane >> 4) * 8, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kPieces / 4; ++i) {
        const int64_t piece = block * kPieces + i * 4 + (threadIdx.x >> 6);
        if (piece >= pad / 16 * ks) return;
        uint4 w;
        w.x = __builtin_amdgcn_perm(__float_as_uint(v[i][1]), __float_as_uint(v[i][0]), 0x07060302u);
        w.y = __builtin_amdgcn_perm(__float_as_uint(v[i][3]), __float_as_uint(v[i][2]), 0x07060302u);
        w.z = __builtin_amdgcn_perm(__float_as_uint(v[i][5]), __float_as_uint(v[i][4]), 0x07060302u);
        w.w = __builtin_amdgcn_perm(__float_as_uint(v[i][7]), __float_as_uint(v[i][6]), 0x07060302u);
        out[piece * 64 + lane] = w;
    }
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }         // of a normal one
// floats: 32 rows by a workgroup, all of them in its registers
__device__ __forceinline__ void lay_out(const RowSource& s, uint4* __restrict__ out, float* __restrict__ scales, int64_t pad, int ks, int64_t tile,
                                        const ClassTokens* known, float) {
    constexpr int MOST = kMaxClassWidth / 32 * 2 / 4;           // of a wave
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    bool in[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int64_t row = tile * kTileRows + b * 16 + (lane & 15);
        in[b] = row < s.rows && (!known || known->at(row) >= 0);
    }
    float v[MOST][8];
    uint32_t top[2] = {0, 0};           // of the lane's rows: bits of the largest finite value
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int piece = i * 4 + wave, b = piece >= ks, k = b ? piece - ks : piece;
        if (piece < 2 * ks) load_eight<float>(s, tile * kTileRows + b * 16 + (lane & 15), b ? in[1] : in[0], k * 32 + (lane >> 4) * 8, v[i]);
    }
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int piece = i * 4 + wave;
        if (piece >= 2 * ks) continue;
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t u = __float_as_uint(v[i][j]) & 0x7FFFFFFFu;
            if (u < 0x7F800000u) most = most > u ? most : u;
        }
        if (piece < ks) top[0] = top[0] > most ? top[0] : most;
        else top[1] = top[1] > most ? top[1] : most;
    }
    __shared__ uint32_t s_top[4][2][16];
    float up[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        for (int o = 16; o < 64; o <<= 1) {
            const uint32_t u = __shfl_xor(top[b], o);
            top[b] = top[b] > u ? top[b] : u;
        }
        if (lane < 16) s_top[wave][b][lane] = top[b];
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t u = s_top[w][b][lane & 15];
            top[b] = top[b] > u ? top[b] : u;
        }
        // rows of zeros, and rows below 2^-100, whose products are nothing beside the rounding of any logit
        int e = (int)(top[b] >> 23) - 127;
        if (top[b] == 0) e = 0;
        if (e < -100) e = -100;
        up[b] = power_of_two(14 - e);
        if (wave == 0 && lane < 16) scales[tile * kTileRows + b * 16 + lane] = power_of_two(e - 14);
    }
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int piece = i * 4 + wave;
        if (piece >= 2 * ks) continue;
        uint32_t h[8], l[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) two_pieces(v[i][j] * (piece < ks ? up[0] : up[1]), h[j], l[j]);
        uint4* to = out + (tile * 2 * ks + piece) * 128 + lane;
        to[0] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        to[64] = make_uint4(l[0] | l[1] << 16, l[2] | l[3] << 16, l[4] | l[5] << 16, l[6] | l[7] << 16);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void k_class_setup(ClassSetup s) {
    unsigned b = blockIdx.x;
    const int wave = threadIdx.x >> 6;
    if (b < s.x_blocks) {
        lay_out(s.x, s.xf, s.x_scale, s.x_pad, s.ks, b, s.lse ? &s.ids : nullptr, T{});
        return;
    }
    b -= s.x_blocks;
    if (b < s.e_blocks) {
        lay_out(s.e, s.ef, s.e_scale, s.e_pad, s.ks, b, nullptr, T{});
        return;
    }
    b -= s.e_blocks;
    if (b < s.row_blocks) {
        int count = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t i = (int64_t)b * 1024 + k * 256 + threadIdx.x;
            if (i >= s.x_pad) continue;
            const int32_t t = i < s.x.rows ? s.ids.at(i) : -1;
            s.target[i] = t;
            if (s.lse) s.lse_out[i] = t >= 0 ? s.lse[i] : INFINITY;         // exp(z - inf): no part in any gradient
            count += t >= 0;
        }
        __shared__ int s_count[4];
        for (int o = 32; o; o >>= 1) count += __shfl_xor(count, o);
        if (lane_id() == 0) s_count[wave] = count;
        __syncthreads();
        if (threadIdx.x == 0) s.counts[b] = s_count[0] + s_count[1] + s_count[2] + s_count[3];
        return;
    }
    b -= s.row_blocks;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t j = (int64_t)b * 1024 + k * 256 + threadIdx.x;
        if (j < s.e_pad) s.bias_out[j] = j < s.e.rows ? (s.bias ? s.bias[j] : 0.0f) : -INFINITY;          // exp(-inf): no class
    }
}

// A tile of N pieces of 1 KB into LDS; arrives once this wave has waited for its loads and all waves have met.
template <int N>
__device__ __forceinline__ void fetch_tile(const uint4* __restrict__ from, uint4* to, int wave, int lane) {
#pragma unroll 8
    for (int c = 0; c < (N + 3) / 4; ++c) {
        const int piece = c * 4 + wave;
        if (N % 4 == 0 || piece < N)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(from + piece * 64 + lane),
                                             (__attribute__((address_space(3))) uint32_t*)(to + piece * 64), 16, 0, 0);
    }
}
// 16-row blocks that a wave keeps, by the registers that they take (operands: 4 NP a step; sums: 8 a step), waves of a SIMD that these and LDS leave room
// for, and whether a workgroup has two tiles in LDS.
constexpr int tile_kilobytes(int ks, int np) { return 2 * ks * np; }
constexpr int loss_blocks(int ks, int np) { return ks * np * 16 <= 128 ? 4 : ks * np * 8 <= 128 ? 2 : 1; }
constexpr int loss_waves(int ks, int np) { return 2 * tile_kilobytes(ks, np) <= 160 ? 2 : 1; }
constexpr bool loss_two(int ks, int np) { return 2 * loss_waves(ks, np) * tile_kilobytes(ks, np) <= 160; }
constexpr int grad_registers(int ks, int np, int rb) { return rb * ks * (4 * np + 8); }
constexpr int grad_blocks(int ks, int np) { return grad_registers(ks, np, 4) <= 128 ? 4 : grad_registers(ks, np, 2) <= (np == 1 ? 192 : 128) ? 2 : 1; }
// (8,191 x 4,099 floats, dx: two waves of one block each against one of two, D = 192 / 256 / 384: 96 / 117 / 170 us against 128 / 160 / 268)
constexpr int grad_waves(int ks, int np) { return grad_registers(ks, np, grad_blocks(ks, np)) <= 192 && 2 * tile_kilobytes(ks, np) <= 160 ? 2 : 1; }
constexpr bool grad_two(int ks, int np) { return 2 * grad_waves(ks, np) * tile_kilobytes(ks, np) <= 160; }
__device__ __forceinline__ void tile_arrived() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}
__device__ __forceinline__ frag8 piece_of_lds(const uint4* p) { return __builtin_bit_cast(frag8, *p); }

// Product i of two values' pieces: 0 .. products<NP>() - 1, small ones first.  They are added to one accumulator, so products of others stand between them.
template <int NP>
constexpr int products() { return NP == 2 ? 3 : 1; }
template <int NP>
__device__ __forceinline__ f32x4 mfma_product(int i, const frag8 (&a)[NP], const frag8 (&b)[NP], f32x4 c) {
    if constexpr (NP == 2) return i == 0 ? mfma_frag<NP>(a[1], b[0], c) : i == 1 ? mfma_frag<NP>(a[0], b[1], c) : mfma_frag<NP>(a[0], b[0], c);
    else return mfma_frag<NP>(a[0], b[0], c);
}

// z[blk][r] += products of the streamed rows 16 blk + 4 (lane / 16) + reg with this wave's row 16 r + lane % 16
template <int KS, int NP, int RB>
__device__ __forceinline__ void tile_logits(const uint4* tile, const frag8 (&own)[RB][KS][NP], int lane, f32x4 (&z)[2][RB]) {
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        frag8 a[2][NP];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int p = 0; p < NP; ++p) a[blk][p] = piece_of_lds(tile + ((blk * KS + k) * NP + p) * 64 + lane);
#pragma unroll
        for (int i = 0; i < products<NP>(); ++i)
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int r = 0; r < RB; ++r) z[blk][r] = mfma_product<NP>(i, a[blk], own[r][k], z[blk][r]);
    }
}
template <int KS, int NP, int RB>
__device__ __forceinline__ void load_own(const uint4* __restrict__ from, int64_t block0, int lane, frag8 (&own)[RB][KS][NP]) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int p = 0; p < NP; ++p) own[r][k][p] = __builtin_bit_cast(frag8, from[(((block0 + r) * KS + k) * NP + p) * 64 + lane]);
}
__device__ __forceinline__ f32x4 four(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 all_four(float v) { return f32x4{v, v, v, v}; }

// ---- forward ---------------------------------------------------------------------------------------------
// A lane adds up exp(z - top) of its rows.  What a nearly learnt row's loss consists of, classes of 2^-24 and less of the largest's probability, is lost in a running
// sum of 32 bits, so only the eight of a tile are added in 32 bits and the tiles in 64.  top follows the largest logit where it is left behind by more than 1: a few
// times over any number of classes, each of which multiplies the sum by a rounded exponential; and a class 1 above the others is exactly 1 in the sum.
struct alignas(16) SoftmaxSum {
    double sum;
    float top;
};
struct ClassLossArgs {
    const uint4 *xf, *ef;
    const float *x_scale, *e_scale;         // floats only
    const float* bias;
    const int32_t* target;
    SoftmaxSum* part;               // [splits][x_pad]
    float* at_target;               // [x_pad]
    int64_t x_pad;
    int32_t tiles, splits;
};
// 32,749 x 50,021 of 256 16-bit values: 718 us, 1,170 TFLOP/s (a large library product reaches 1,444 on the same card); matrix cores busy 51 % of the cycles.  With sums of
// 32 bits and exp by one multiply-add 4 % less, 12 % at 70,000 x 2,000 of 32 columns.
template <int KS, int NP, int RB>
__global__ __launch_bounds__(256, loss_waves(KS, NP)) void k_class_loss(ClassLossArgs g) {
    constexpr int N = 2 * KS * NP;
    constexpr bool TWO = loss_two(KS, NP);
    __shared__ uint4 s_tile[TWO ? 2 : 1][N * 64];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4;
    const int64_t block0 = ((int64_t)blockIdx.x * 4 + wave) * RB;
    const int t0 = (int)((int64_t)g.tiles * blockIdx.y / g.splits), t1 = (int)((int64_t)g.tiles * (blockIdx.y + 1) / g.splits);
    fetch_tile<N>(g.ef + (int64_t)t0 * N * 64, s_tile[0], wave, lane);          // (no part is empty)
    frag8 own[RB][KS][NP];
    load_own<KS, NP, RB>(g.xf, block0, lane, own);
    int target[RB];
    float top[RB], own_scale[RB];
    double sum[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        target[r] = g.target[(block0 + r) * 16 + (lane & 15)];
        own_scale[r] = NP == 2 ? g.x_scale[(block0 + r) * 16 + (lane & 15)] : 0.0f;
        top[r] = kNoMax;
        sum[r] = 0.0;
    }
    tile_arrived();
    for (int t = t0; t < t1; ++t) {
        const uint4* tile = s_tile[TWO ? (t - t0) & 1 : 0];
        if (TWO && t + 1 < t1) fetch_tile<N>(g.ef + (int64_t)(t + 1) * N * 64, s_tile[TWO ? (t - t0 + 1) & 1 : 0], wave, lane);
        f32x4 z[2][RB], bias[2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            const int64_t i = (int64_t)t * kTileRows + blk * 16 + grp * 4;
            bias[blk] = four(g.bias + i);
#pragma unroll
            for (int r = 0; r < RB; ++r) z[blk][r] = NP == 2 ? all_four(0.0f) : bias[blk];
        }
        tile_logits<KS, NP, RB>(tile, own, lane, z);
        if constexpr (NP == 2) {
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const f32x4 scale = four(g.e_scale + (int64_t)t * kTileRows + blk * 16 + grp * 4);
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[blk][r][i] = fmaf(z[blk][r][i] * scale[i], own_scale[r], bias[blk][i]);
            }
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            if (ballot((unsigned)(target[r] - t * kTileRows) < (unsigned)kTileRows)) {
#pragma unroll
                for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (target[r] == t * kTileRows + blk * 16 + grp * 4 + i) g.at_target[(block0 + r) * 16 + (lane & 15)] = z[blk][r][i];
            }
            float m = top[r];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, z[blk][r][i]);
            m = m > top[r] + 1.0f ? m : top[r];
            const float before = __builtin_amdgcn_exp2f((top[r] - m) * kLog2e);
            top[r] = m;
            f32x4 e[2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int i = 0; i < 4; ++i) e[blk][i] = __builtin_amdgcn_exp2f((z[blk][r][i] - m) * kLog2e);
            const f32x4 pairs = e[0] + e[1];
            sum[r] = fma((double)before, sum[r], (double)((pairs[0] + pairs[1]) + (pairs[2] + pairs[3])));
        }
        if constexpr (!TWO) {
            __syncthreads();
            if (t + 1 < t1) fetch_tile<N>(g.ef + (int64_t)(t + 1) * N * 64, s_tile[0], wave, lane);
        }
        tile_arrived();
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        float m = fmaxf(top[r], __shfl_xor(top[r], 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        double s = sum[r] * (double)__builtin_amdgcn_exp2f((top[r] - m) * kLog2e);
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (grp == 0) g.part[blockIdx.y * g.x_pad + (block0 + r) * 16 + lane] = SoftmaxSum{s, m};
    }
}
// lse of rows and their part of the loss; a single workgroup writes the loss itself
struct LossPart {
    double sum;
    int64_t count;
};
__device__ __forceinline__ void add_up(double& sum, int64_t& count) {          // over 1,024 threads, in the first
    __shared__ double s_sum[16];
    __shared__ int64_t s_count[16];
    for (int o = 32; o; o >>= 1) {
        sum += __shfl_xor(sum, o);
        count += __shfl_xor(count, o);
    }
    if (lane_id() == 0) {
        s_sum[threadIdx.x >> 6] = sum;
        s_count[threadIdx.x >> 6] = count;
    }
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0.0;
    count = 0;
    for (int i = 0; i < 16; ++i) {
        sum += s_sum[i];
        count += s_count[i];
    }
}
// 2^q lanes take the splits of a row.  Sums in 64 bits; exponentials and logarithms of 32 bits, off by 3 u of themselves.  2,000 rows of two parts,
// one workgroup: 4.9 us; with each part read twice and 64-bit functions 9.4.
__global__ __launch_bounds__(1024) void k_class_lse(const SoftmaxSum* __restrict__ part, const float* __restrict__ at_target,
                                                    const int32_t* __restrict__ target, int64_t n, int64_t x_pad, int splits, int q,
                                                    float* __restrict__ lse_out, LossPart* __restrict__ parts, float* __restrict__ loss) {
    double sum = 0.0;
    int64_t count = 0;
    const int first = threadIdx.x & ((1 << q) - 1), step = 1 << q;
    for (int64_t r = (int64_t)blockIdx.x * (1024 >> q); r < n; r += (int64_t)gridDim.x * (1024 >> q)) {          // the same for a workgroup
        const int64_t row = r + (threadIdx.x >> q), i = row < n ? row : n - 1;
        const int32_t t = target[i];
        const float at = at_target[i];
        constexpr int U = 4;                    // parts of a lane that stay in its registers: as many as it has, but for long sides
        SoftmaxSum p[U];
#pragma unroll
        for (int k = 0; k < U; ++k) p[k] = first + k * step < splits ? part[(first + k * step) * x_pad + i] : SoftmaxSum{0.0, kNoMax};
        float m = kNoMax;
#pragma unroll
        for (int k = 0; k < U; ++k) m = fmaxf(m, p[k].top);
        for (int s = first + U * step; s < splits; s += step) m = fmaxf(m, part[s * x_pad + i].top);
        for (int o = step >> 1; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        auto to_top = [&](const SoftmaxSum& q) { return q.sum * (double)__builtin_amdgcn_exp2f((q.top - m) * kLog2e); };
        double l = 0.0;
#pragma unroll
        for (int k = 0; k < U; ++k) l += to_top(p[k]);
        for (int s = first + U * step; s < splits; s += step) l += to_top(part[s * x_pad + i]);
        for (int o = step >> 1; o; o >>= 1) l += __shfl_xor(l, o);
        if (first || row >= n) continue;
        const float above = l < 1.5 ? log1pf((float)(l - 1.0)) : logf((float)l);            // (l is 1 at least, or 0 if no class is left)
        lse_out[i] = (float)((double)m + (double)above);
        if (t >= 0) {
            sum += ((double)m - (double)at) + (double)above;
            ++count;
        }
    }
    add_up(sum, count);
    if (threadIdx.x) return;
    if (gridDim.x == 1) *loss = count ? (float)(sum / (double)count) : 0.0f;
    else parts[blockIdx.x] = LossPart{sum, count};
}
__global__ __launch_bounds__(1024) void k_class_loss_sum(const LossPart* __restrict__ parts, int blocks, float* __restrict__ loss) {
    double sum = 0.0;
    int64_t count = 0;
    for (int i = threadIdx.x; i < blocks; i += 1024) {
        sum += parts[i].sum;
        count += parts[i].count;
    }
    add_up(sum, count);
    if (threadIdx.x == 0) *loss = count ? (float)(sum / (double)count) : 0.0f;
}

// ---- backward --------------------------------------------------------------------------------------------
struct ClassGradArgs {
    const uint4 *own, *stream;      // in pieces: the rows that a workgroup keeps, and the tiles
    const float *own_scale, *stream_scale;      // floats only: of their rows
    const float *lse, *bias;
    const int32_t *target, *counts;
    void* out;                      // rows x d of T: a plane, or a table
    int64_t rows, ld, gs;
    float* part;                    // [splits][own_pad][KS * 32], where there are several; of rows and of classes each its own
    double* bias_part;              // BY_CLASS: [splits][own_pad], where there are several
    float* dbias;                   // BY_CLASS
    int64_t own_pad;
    int32_t d, dg, tiles, splits, count_blocks;
    uint32_t blocks;                // workgroups of a part; 0: this side is not asked for
    float scale;
};
__device__ __forceinline__ float gradient_scale(const int32_t* __restrict__ counts, int blocks, float scale) {
    int count = 0;
    for (int i = lane_id(); i < blocks; i += 64) count += counts[i];
    for (int o = 32; o; o >>= 1) count += __shfl_xor(count, o);
    return count ? scale / (float)count : 0.0f;
}
__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_as(bf16_t* p, float v) { p->bits = (uint16_t)bf16_bits(v); }

// Eight dz as the operand of the second product: rounded to bf16 (at most 2^-8 of each, as the gradients that they are summed to are), or in two pieces.  The first
// rounding shows beside the second where sums are short: the error of dx and dE in norm is 0.0020 instead of 0.0017 with two or three terms a sum, 0.0017 either way with
// 32,749 x 50,021.  It was left, since what takes it away costs every call more than it gives: fp16 operands with 11 bits of dz and a power of two for every row 3,270 us
// instead of 2,880 there (fewer cycles, but the clock falls by 13 % with fp16 products), 72 -> 88 at 100,000 x 300 of 128 columns, 131 -> 167 at 70,000 x 2,000 of 32; two
// bf16 pieces of dz 4,000, 83 and 174.
template <int NP>
__device__ __forceinline__ void operand_of(const f32x4& a, const f32x4& b, frag8 (&o)[NP]) {
    if constexpr (NP == 1) {
        bf16x8 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = static_cast<__bf16>(a[i]);
            w[4 + i] = static_cast<__bf16>(b[i]);
        }
        o[0] = __builtin_bit_cast(frag8, w);
    } else {
        f16x8 h, l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = i < 4 ? a[i & 3] : b[i & 3];
            h[i] = static_cast<_Float16>(v);
            l[i] = static_cast<_Float16>(v - static_cast<float>(h[i]));
        }
        o[0] = __builtin_bit_cast(frag8, h);
        o[1] = __builtin_bit_cast(frag8, l);
    }
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
// the streamed rows 4 (lane / 16) .. + 3 of block blk at column 16 cb + lane % 16: 16 lanes together read four rows of 16 columns
template <int KS, int NP>
__device__ __forceinline__ s16x4 column_of_lds(const uint4* tile, int blk, int cb, int p, int lane) {
    const int grp = lane >> 4, i = lane & 15;
    const char* at = reinterpret_cast<const char*>(tile + ((blk * KS + (cb >> 1)) * NP + p) * 64) +
                     (((cb & 1) * 2 + ((i & 3) >> 1)) * 16 + 4 * grp + (i >> 2)) * 16 + (i & 1) * 8;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
}

// Two pieces of fp16 hold dz only in its range, and gradients of rare classes and of rows that are nearly learnt are far below 1.  So every own row has a power of
// two k by which its dz (times the streamed row's power of two) and its sums are multiplied; k begins so high that products of a dz and a streamed
// value of 2^-88 and more keep all their bits, stays below 2^100 over the streamed rows' powers (so that a dz of 1 is finite), and whenever a value of the row would leave
// fp16's range it goes down so far that the row may grow eightfold before it does again.  A dz is held to 2^-22 of itself, or its product with the streamed row's
// largest value to 2^-36 of the largest so far.
constexpr float kLargestRow = 0x1p100f, kLargestPiece = 32768.0f;
// room: what k already had to go down by for the tile's sake
template <int KS, int RB>
__device__ __forceinline__ void fit_row(int r, float room, float largest, float& k, f32x4 (&z)[2][RB], f32x4 (&acc)[RB][2 * KS], int grp) {
    const bool over = largest >= kLargestPiece;         // (not for NaN)
    const float f = over ? power_of_two(14 - 3 + 127 - (int)(__float_as_uint(largest) >> 23)) : 1.0f;
    k = k * room * f;                                   // (room * f by itself may be below the smallest number)
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 4; ++i) z[blk][r][i] *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float row = __shfl(room * f, grp * 4 + i);        // sums lie by rows, values by columns
#pragma unroll
        for (int c = 0; c < 2 * KS; ++c) acc[r][c][i] *= row;
    }
}
// what brings k times `scale`, both powers of two, to kLargestRow at most
__device__ __forceinline__ float room_for(float k, float scale) {
    const int over = (int)(__float_as_uint(k) >> 23) + (int)(__float_as_uint(scale) >> 23) - 2 * 127 - 100;
    return over > 0 ? power_of_two(-over) : 1.0f;
}

// Workgroup `index` of those of one side: a block of its rows and a part of the tiles.
template <int KS, int NP, int RB, bool BY_CLASS, typename T>
__device__ __forceinline__ void grad_side(const ClassGradArgs& g, unsigned index, uint4 (*s_tile)[2 * KS * NP * 64]) {
    constexpr int N = 2 * KS * NP;
    constexpr bool TWO = grad_two(KS, NP);
    const unsigned part = index / g.blocks;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4;
    const int64_t block0 = ((int64_t)(index - part * g.blocks) * 4 + wave) * RB;
    const int t0 = (int)((int64_t)g.tiles * part / g.splits), t1 = (int)((int64_t)g.tiles * (part + 1) / g.splits);
    if (t0 < t1) fetch_tile<N>(g.stream + (int64_t)t0 * N * 64, s_tile[0], wave, lane);
    frag8 own[RB][KS][NP];
    load_own<KS, NP, RB>(g.own, block0, lane, own);
    // of this wave's rows: lse and class (BY_CLASS: bias and class number), and their powers of two; the same of streamed rows comes with the tile
    float own_f[RB], own_scale[RB], k[RB];
    int own_c[RB];
    f32x4 acc[RB][2 * KS];
    double bias_sum[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int64_t i = (block0 + r) * 16 + (lane & 15);
        own_f[r] = BY_CLASS ? g.bias[i] : g.lse[i];
        own_c[r] = BY_CLASS ? (int)i : g.target[i];
        own_scale[r] = NP == 2 ? g.own_scale[i] : 0.0f;
        k[r] = kLargestRow;
        bias_sum[r] = 0.0;
#pragma unroll
        for (int c = 0; c < 2 * KS; ++c) acc[r][c] = all_four(0.0f);
    }
    tile_arrived();
    for (int t = t0; t < t1; ++t) {
        const uint4* tile = s_tile[TWO ? (t - t0) & 1 : 0];
        if (TWO && t + 1 < t1) fetch_tile<N>(g.stream + (int64_t)(t + 1) * N * 64, s_tile[TWO ? (t - t0 + 1) & 1 : 0], wave, lane);
        f32x4 z[2][RB], row_f[2], row_scale[2];
        int row_c[2][4];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            const int64_t i = (int64_t)t * kTileRows + blk * 16 + grp * 4;
            row_f[blk] = four((BY_CLASS ? g.lse : g.bias) + i);
            if constexpr (NP == 2) row_scale[blk] = four(g.stream_scale + i);
            int4 c = make_int4((int)i, (int)i + 1, (int)i + 2, (int)i + 3);
            if constexpr (BY_CLASS) c = *reinterpret_cast<const int4*>(g.target + i);
            row_c[blk][0] = c.x; row_c[blk][1] = c.y; row_c[blk][2] = c.z; row_c[blk][3] = c.w;
#pragma unroll
            for (int r = 0; r < RB; ++r) z[blk][r] = NP == 2 ? all_four(0.0f) : BY_CLASS ? all_four(own_f[r]) : row_f[blk];
        }
        // A wave in its products goes before one that fetches or is at its exponentials: 16 bits at D = 256, 3,140 -> 3,100 us; no gain for floats or the loss.
        __builtin_amdgcn_s_setprio(1);
        tile_logits<KS, NP, RB>(tile, own, lane, z);
        __builtin_amdgcn_s_setprio(0);
        frag8 dz[RB][NP];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float b = BY_CLASS ? own_f[r] : row_f[blk][i], l = BY_CLASS ? row_f[blk][i] : own_f[r];
                    if constexpr (NP == 2) z[blk][r][i] = fmaf(z[blk][r][i] * row_scale[blk][i], own_scale[r], b);
                    const float p = __builtin_amdgcn_exp2f((z[blk][r][i] - l) * kLog2e);
                    z[blk][r][i] = row_c[blk][i] == own_c[r] ? p - 1.0f : p;
                }
            if constexpr (BY_CLASS) {
                const f32x4 s = z[0][r] + z[1][r];
                bias_sum[r] += (double)((s[0] + s[1]) + (s[2] + s[3]));
            }
            if constexpr (NP == 2) {
                float scale = 0.0f, largest = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) scale = fmaxf(scale, fmaxf(row_scale[0][i], row_scale[1][i]));
                const bool high = ballot(scale > 1.0f);                 // (rows of values above 2^14 may leave k too little room)
                const float room = high ? room_for(k[r], quarter_fmax(scale)) : 1.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int blk = 0; blk < 2; ++blk) z[blk][r][i] = z[blk][r][i] * (k[r] * room) * row_scale[blk][i];
                    largest = fmaxf(largest, fmaxf(fabsf(z[0][r][i]), fabsf(z[1][r][i])));
                }
                largest = quarter_fmax(largest);
                if (high || ballot(largest >= kLargestPiece)) fit_row<KS, RB>(r, room, largest, k[r], z, acc, grp);
            }
            operand_of<NP>(z[0][r], z[1][r], dz[r]);
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int c = 0; c < 2 * KS; c += 2) {
            frag8 b[2][NP];
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int p = 0; p < NP; ++p)
                    b[q][p] = __builtin_shufflevector(column_of_lds<KS, NP>(tile, 0, c + q, p, lane), column_of_lds<KS, NP>(tile, 1, c + q, p, lane), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int i = 0; i < products<NP>(); ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int r = 0; r < RB; ++r) acc[r][c + q] = mfma_product<NP>(i, dz[r], b[q], acc[r][c + q]);
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (!TWO) {
            __syncthreads();
            if (t + 1 < t1) fetch_tile<N>(g.stream + (int64_t)(t + 1) * N * 64, s_tile[0], wave, lane);
        }
        tile_arrived();
    }
    const float scale = gradient_scale(g.counts, g.count_blocks, g.scale);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int64_t row0 = (block0 + r) * 16 + grp * 4;
        if constexpr (BY_CLASS) {
            bias_sum[r] += __shfl_xor(bias_sum[r], 16);
            bias_sum[r] += __shfl_xor(bias_sum[r], 32);
            const int64_t j = (block0 + r) * 16 + lane;
            if (grp == 0 && g.splits > 1) g.bias_part[part * g.own_pad + j] = bias_sum[r];
            else if (grp == 0 && g.dbias && j < g.rows) g.dbias[j] = (float)(bias_sum[r] * (double)scale);
        }
        if (!g.out) continue;                   // only the bias is asked for
        if constexpr (NP == 2) {
            const float f = __uint_as_float(0x7F000000u - __float_as_uint(k[r]));           // 1 / k
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float row = __shfl(f, grp * 4 + i);
#pragma unroll
                for (int c = 0; c < 2 * KS; ++c) acc[r][c][i] *= row;
            }
        }
        if (g.splits > 1) {
            float* to = g.part + ((int64_t)part * g.own_pad + row0) * (KS * 32) + (lane & 15);
#pragma unroll
            for (int c = 0; c < 2 * KS; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i * (KS * 32) + c * 16] = acc[r][c][i];
            continue;
        }
        const int64_t left = g.rows - row0;             // of the lane's four rows
#pragma unroll
        for (int c = 0; c < 2 * KS; ++c) {
            const int col = c * 16 + (lane & 15), plane = col / g.dg;
            if (col >= g.d) continue;
            T* to = static_cast<T*>(g.out) + plane * g.gs + row0 * g.ld + (col - plane * g.dg);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) store_as(to + i * g.ld, acc[r][c][i] * scale);
        }
    }
}
// dx and dE, or one of them, in one launch: what is left of the one's last round is filled by the other, and few rows and classes wait for one launch less.
// 32,749 x 50,021 of 256 16-bit values: four products (each side has the logits anew) in 2.91 ms, 1,150 TFLOP/s; 8,191 x 4,099 floats at D = 384, 308 us, 1,000.
// Matrix cores busy 49 % of the cycles.  With a quarter fewer vector instructions (exponents in one multiply-add, classes looked for by tile) the cycles
// fall by 2 % and the time grows by 3 %, since the clock falls; four blocks a wave, one wave a SIMD: 4.5 ms.
template <int KS, int NP, int RB, typename T>
__global__ __launch_bounds__(256, grad_waves(KS, NP)) void k_class_grad(ClassGradArgs by_row, ClassGradArgs by_class, unsigned row_from, unsigned class_from) {
    __shared__ uint4 s_tile[grad_two(KS, NP) ? 2 : 1][2 * KS * NP * 64];
    const unsigned row = blockIdx.x - row_from;             // (wraps before row_from)
    if (row < by_row.blocks * by_row.splits) grad_side<KS, NP, RB, false, T>(by_row, row, s_tile);
    else grad_side<KS, NP, RB, true, T>(by_class, blockIdx.x - class_from, s_tile);
}
// The parts' sums joined, 2^q threads of a workgroup a value: every 2^q-th part each, then one after the other.
template <typename V, typename Part, typename Store>
__device__ __forceinline__ void join_parts(int64_t first, int64_t count, int splits, int q, V* s_sum, Part part, Store store) {
    const int each = 256 >> q, mine = threadIdx.x & (each - 1), lane = threadIdx.x >> (8 - q);
    const int64_t i = first + mine;
    V v{};
    if (i < count) {
        constexpr int U = 4;
        for (int s = lane; s < splits; s += U << q) {
            V t[U];
#pragma unroll
            for (int k = 0; k < U; ++k) t[k] = s + (k << q) < splits ? part(s + (k << q), i) : V{};
#pragma unroll
            for (int k = 0; k < U; ++k) v += t[k];
        }
    }
    if (q) {
        s_sum[threadIdx.x] = v;
        __syncthreads();
        if (lane) return;
        for (int k = 1; k < 1 << q; ++k) v += s_sum[(k << (8 - q)) + mine];
    }
    if (i < count) store(i, v);
}
__host__ __device__ constexpr unsigned join_quads(int d) { return (unsigned)(d + 3) / 4; }
__device__ __forceinline__ void store_four(float* p, f32x4 v) { *reinterpret_cast<u32x4a*>(p) = __builtin_bit_cast(u32x4a, v); }
__device__ __forceinline__ void store_four(bf16_t* p, f32x4 v) {
    u32x2h t;
    t[0] = bf16_bits(v[0]) | bf16_bits(v[1]) << 16;
    t[1] = bf16_bits(v[2]) | bf16_bits(v[3]) << 16;
    *reinterpret_cast<u32x2h*>(p) = t;
}
struct JoinShape {
    unsigned row_blocks, class_blocks, bias_blocks;         // workgroups of each; 0: nothing to join
    int row_q, class_q, width;
};
template <typename T>
__global__ __launch_bounds__(256) void k_class_grad_join(ClassGradArgs by_row, ClassGradArgs by_class, JoinShape j) {
    __shared__ f32x4 s_sum[256];
    unsigned b = blockIdx.x;
    const bool rows = b < j.row_blocks;
    if (!rows) b -= j.row_blocks;
    const ClassGradArgs& g = rows ? by_row : by_class;
    const int q = rows ? j.row_q : j.class_q;
    const float scale = gradient_scale(g.counts, g.count_blocks, g.scale);
    if (rows || b < j.class_blocks) {
        const unsigned quads = join_quads(g.d);         // four columns each; (there are fewer than 2^32 of them where a side is split)
        join_parts<f32x4>((int64_t)b * (256 >> q), g.rows * quads, g.splits, q, s_sum,
            [&](int s, int64_t i) { return four(g.part + ((int64_t)s * g.own_pad + (unsigned)i / quads) * j.width + (unsigned)i % quads * 4); },
            [&](int64_t i, f32x4 v) {
                const unsigned row = (unsigned)i / quads;
                const int col = (int)((unsigned)i % quads) * 4, plane = col / g.dg;
                T* to = static_cast<T*>(g.out) + plane * g.gs + row * g.ld + (col - plane * g.dg);
                v *= scale;
                if (g.dg % 4 == 0) return store_four(to, v);
                for (int k = 0; k < 4 && col + k < g.d; ++k) {
                    const int other = (col + k) / g.dg;
                    store_as(static_cast<T*>(g.out) + other * g.gs + row * g.ld + (col + k - other * g.dg), v[k]);
                }
            });
    } else {
        join_parts<double>((int64_t)(b - j.class_blocks) * (256 >> q), g.rows, g.splits, q, reinterpret_cast<double*>(s_sum),
            [&](int s, int64_t i) { return g.bias_part[(int64_t)s * g.own_pad + i]; }, [&](int64_t i, double v) { g.dbias[i] = (float)(v * (double)scale); });
    }
}

// ---- host side ---------------------------------------------------------------------------------------------
namespace {

constexpr int kPadRows = 256;                   // operands are laid out to a multiple of what a workgroup keeps at most
constexpr int64_t kMaxRows = (int64_t)1 << 28;  // of x and of E: a grid holds fewer than 2^32 threads
constexpr int kMaxSplits = 512;
constexpr int64_t kMaxPartRows = 1 << 17;       // rows of partial sums, of all parts together

bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

int steps_of(int d) {
    for (int ks : {1, 2, 4, 6, 8, 12}) if (d <= 32 * ks) return ks;
    return 16;
}
// Parts that the streamed side is cut into: of those that make whole rounds of 512 workgroups, and halves of the most, the shortest by this estimate.  A tile takes
// `tile_ns`, of which every part has one more (its own rows), and the partial sums, `row_bytes` a row, are written and read at 4 bytes a picosecond.
// 731 rows x 12,547 classes of 64 16-bit columns: 51 us with as many parts as fill the card, 34 with these.
int splits_of(int64_t blocks, int64_t tiles, int64_t pad, double tile_ns, double row_bytes) {
    constexpr int64_t places = 512;
    const int64_t most = std::max<int64_t>(1, std::min({(int64_t)kMaxSplits, tiles, blocks ? kMaxPartRows / pad : 1}));
    int64_t best = 1;
    double least = 1e300;
    auto look = [&](int64_t s) {
        s = std::min(most, std::max<int64_t>(1, s));
        const double rounds = (double)((blocks * s + places - 1) / places), length = (double)((tiles + s - 1) / s) + 1.0;
        const double time = rounds * length * tile_ns + (s > 1 ? (double)(s * pad) * row_bytes * 2.0 / 4000.0 : 0.0);
        if (time < 0.97 * least) {
            least = time;
            best = s;
        }
    };
    look(1);
    for (int64_t rounds = 1; rounds <= 8; ++rounds) look(places * rounds / std::max<int64_t>(1, blocks));
    for (int64_t s = most; s > 1; s /= 2) look(s);
    return (int)best;
}
// 16 cycles an instruction at 2 GHz, and what a tile takes besides
double tile_time(int ks, int np, int rb, int products) { return products * 2.0 * ks * rb * (np == 2 ? 3 : 1) * 8.0 + 300.0; }
// Rows of partial sums that a workspace has room for: what any split of as many rows or fewer can need, so that a workspace serves them all.
int64_t part_rows(int64_t tiles, int64_t pad) { return std::min(kMaxPartRows, std::min<int64_t>(kMaxSplits, tiles) * pad); }
struct ClassPlan {
    int ks, np, loss_rb, grad_rb;
    int64_t x_pad, e_pad;
    int loss_splits, x_splits, e_splits;
    size_t xf, ef, x_scale, e_scale, lse, bias, target, counts, loss_bytes;         // the first of these are shared
    size_t part, at_target, parts;                              // forward
    size_t x_part, e_part, bias_part, grad_bytes;               // backward
};
ClassPlan class_plan(int64_t n, int64_t classes, int32_t d, int32_t dtype) {
    ClassPlan p{};
    p.ks = steps_of(d);
    p.np = dtype == GSR_F32 ? 2 : 1;
    p.loss_rb = loss_blocks(p.ks, p.np);
    p.grad_rb = grad_blocks(p.ks, p.np);
    p.x_pad = (n + kPadRows - 1) / kPadRows * kPadRows;
    p.e_pad = (classes + kPadRows - 1) / kPadRows * kPadRows;
    const int64_t x_tiles = (n + kTileRows - 1) / kTileRows, e_tiles = (classes + kTileRows - 1) / kTileRows;
    auto blocks = [](int64_t rows, int rb) { return (rows + 64 * rb - 1) / (64 * rb); };
    p.loss_splits = splits_of(blocks(n, p.loss_rb), e_tiles, p.x_pad, tile_time(p.ks, p.np, p.loss_rb, 1), 8.0);
    p.x_splits = splits_of(blocks(n, p.grad_rb), e_tiles, p.x_pad, tile_time(p.ks, p.np, p.grad_rb, 2), p.ks * 128.0);
    p.e_splits = splits_of(blocks(classes, p.grad_rb), x_tiles, p.e_pad, tile_time(p.ks, p.np, p.grad_rb, 2), p.ks * 128.0);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    p.xf = take((size_t)p.x_pad * p.ks * 64 * p.np);
    p.ef = take((size_t)p.e_pad * p.ks * 64 * p.np);
    p.x_scale = take((size_t)p.x_pad * 4);
    p.e_scale = take((size_t)p.e_pad * 4);
    p.lse = take((size_t)p.x_pad * 4);
    p.bias = take((size_t)p.e_pad * 4);
    p.target = take((size_t)p.x_pad * 4);
    p.counts = take((size_t)((p.x_pad + 1023) / 1024) * 4);
    const size_t shared = at;
    const int64_t x_parts = part_rows(e_tiles, p.x_pad), e_parts = part_rows(x_tiles, p.e_pad);
    p.part = take((size_t)std::max(p.x_pad, x_parts) * sizeof(SoftmaxSum));
    p.at_target = take((size_t)p.x_pad * 4);
    p.parts = take((size_t)((n + 1023) / 1024 + 64) * sizeof(LossPart));       // (65,536 threads at most where a row has several)
    p.loss_bytes = at;
    at = shared;
    p.bias_part = take((size_t)std::max(p.e_pad, e_parts) * sizeof(double));
    p.x_part = take((size_t)x_parts * p.ks * 128);
    p.e_part = take((size_t)e_parts * p.ks * 128);
    p.grad_bytes = at;
    return p;
}

template <typename Call>
void by_steps(int ks, Call call) {
    switch (ks) {
        case 1: return call(std::integral_constant<int, 1>{});
        case 2: return call(std::integral_constant<int, 2>{});
        case 4: return call(std::integral_constant<int, 4>{});
        case 6: return call(std::integral_constant<int, 6>{});
        case 8: return call(std::integral_constant<int, 8>{});
        case 12: return call(std::integral_constant<int, 12>{});
        default: return call(std::integral_constant<int, 16>{});
    }
}

struct ClassShape {
    RowSource x, e;
    ClassTokens ids;
};
gsr_status_t class_shape(const void* x, int64_t ldx, int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype, const void* table, int64_t classes,
                         int64_t ldt, const float* bias, const void* ids, int32_t ids_i64, ClassShape* s) {
    if (n < 0) return fail(GSR_ERR_INVALID_ARG, "negative n");
    if (n >= kMaxRows) return fail(GSR_ERR_UNSUPPORTED, "n=%lld at or above 2^28", (long long)n);
    if (classes < 1) return fail(GSR_ERR_INVALID_ARG, "%lld classes", (long long)classes);
    if (classes >= kMaxRows) return fail(GSR_ERR_UNSUPPORTED, "%lld classes, 2^28 or more", (long long)classes);
    if (d < 1 || d > kMaxClassWidth) return fail(GSR_ERR_UNSUPPORTED, "d=%d outside [1, %d]", d, kMaxClassWidth);
    if (c < 1 || d % c) return fail(GSR_ERR_UNSUPPORTED, "c=%d does not divide d=%d", c, d);
    if (layout != GSR_LAYOUT_ROW_MAJOR && layout != GSR_LAYOUT_GROUP_PLANAR) return fail(GSR_ERR_INVALID_ARG, "layout %d", layout);
    if (dtype != GSR_F32 && dtype != GSR_BF16) return fail(GSR_ERR_UNSUPPORTED, "dtype %d", dtype);
    const int dg = layout == GSR_LAYOUT_GROUP_PLANAR ? d / c : d;
    if (ldx < dg || ldx >= ((int64_t)1 << 31)) return fail(GSR_ERR_INVALID_ARG, "row stride %lld outside [%d, 2^31)", (long long)ldx, dg);
    if (ldt < d || ldt >= ((int64_t)1 << 31)) return fail(GSR_ERR_INVALID_ARG, "row stride %lld of the table outside [%d, 2^31)", (long long)ldt, d);
    if (!table || (n > 0 && (!x || !ids))) return fail(GSR_ERR_INVALID_ARG, "null pointer");
    if (!aligned_to(x, dtype_size(dtype)) || !aligned_to(table, dtype_size(dtype)) || !aligned_to(bias, 4) || !aligned_to(ids, ids_i64 ? 8 : 4))
        return fail(GSR_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
    s->x = RowSource{x, n, ldx, n * ldx, d, dg};
    s->e = RowSource{table, classes, ldt, 0, d, d};
    s->ids = ClassTokens{ids, ids_i64, (int32_t)classes};
    return GSR_OK;
}
gsr_status_t class_workspace(size_t need, const void* workspace, size_t bytes) {
    if (bytes < need) return fail(GSR_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", bytes, need);
    if (!workspace || !aligned_to(workspace, 16)) return fail(GSR_ERR_INVALID_ARG, "workspace null or not aligned to 16 bytes");
    return GSR_OK;
}
ClassSetup launch_setup(const ClassShape& s, const ClassPlan& p, const float* bias, const float* lse, char* ws, int32_t dtype, hipStream_t st) {
    ClassSetup a{};
    a.x = s.x;
    a.e = s.e;
    a.ids = s.ids;
    a.xf = (uint4*)(ws + p.xf);
    a.ef = (uint4*)(ws + p.ef);
    a.x_scale = (float*)(ws + p.x_scale);
    a.e_scale = (float*)(ws + p.e_scale);
    a.lse = lse;
    a.bias = bias;
    a.lse_out = (float*)(ws + p.lse);
    a.bias_out = (float*)(ws + p.bias);
    a.target = (int32_t*)(ws + p.target);
    a.counts = (int32_t*)(ws + p.counts);
    a.x_pad = p.x_pad;
    a.e_pad = p.e_pad;
    a.ks = p.ks;
    auto share = [&](int64_t pad) { return (unsigned)(dtype == GSR_F32 ? pad / kTileRows : pad / 16 * p.ks / kPieces); };        // (rows are padded to 256)
    a.x_blocks = share(p.x_pad);
    a.e_blocks = share(p.e_pad);
    a.row_blocks = (unsigned)((p.x_pad + 1023) / 1024);
    a.bias_blocks = (unsigned)((p.e_pad + 1023) / 1024);
    const dim3 grid(a.x_blocks + a.e_blocks + a.row_blocks + a.bias_blocks);
    if (dtype == GSR_F32) hipLaunchKernelGGL((k_class_setup<float>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_class_setup<bf16_t>), grid, dim3(256), 0, st, a);
    return a;
}

// Threads for a value of a join: four parts each.
int join_lanes(int splits) {
    int q = 0;
    while (q < 4 && splits > 4 << q) ++q;
    return q;
}
template <int KS, typename T>
void launch_grad(ClassGradArgs by_row, ClassGradArgs by_class, hipStream_t st) {
    constexpr int NP = sizeof(T) == 4 ? 2 : 1, RB = grad_blocks(KS, NP);
    auto blocks = [](const ClassGradArgs& g) { return (unsigned)((g.rows + 64 * RB - 1) / (64 * RB)); };
    if (by_row.splits) by_row.blocks = blocks(by_row);
    if (by_class.splits) by_class.blocks = blocks(by_class);
    const unsigned row_wgs = by_row.blocks * by_row.splits, class_wgs = by_class.blocks * by_class.splits;
    if (!(row_wgs + class_wgs)) return;
    // The classes' side first where its workgroups are longer by a fifth, so that the rows fill what it leaves.  32,749 x 50,021 of 256 16-bit values (1.31 times
    // as long) 2,975 us, 3,080 with the rows first; 74,701 x 23 of 64 floats (9 times) 51 and 62; 8,191 x 4,099 of 384 floats (1.14 times) 336 and 332.
    const bool class_first = class_wgs && (!row_wgs || 5 * (int64_t)by_class.tiles * by_row.splits > 6 * (int64_t)by_row.tiles * by_class.splits);
    hipLaunchKernelGGL((k_class_grad<KS, NP, RB, T>), dim3(row_wgs + class_wgs), dim3(256), 0, st, by_row, by_class, class_first ? class_wgs : 0,
                       class_first ? 0 : row_wgs);
    JoinShape j{};
    j.width = KS * 32;
    auto values = [](int64_t count, int q) { return (unsigned)((count + (256 >> q) - 1) / (256 >> q)); };
    if (by_row.splits > 1) {
        j.row_q = join_lanes(by_row.splits);
        j.row_blocks = values(by_row.rows * join_quads(by_row.d), j.row_q);
    }
    if (by_class.splits > 1) {
        j.class_q = join_lanes(by_class.splits);
        if (by_class.out) j.class_blocks = values(by_class.rows * join_quads(by_class.d), j.class_q);
        if (by_class.dbias) j.bias_blocks = values(by_class.rows, j.class_q);
    }
    const unsigned joins = j.row_blocks + j.class_blocks + j.bias_blocks;
    if (joins) hipLaunchKernelGGL((k_class_grad_join<T>), dim3(joins), dim3(256), 0, st, by_row, by_class, j);
}

}  // namespace
}  // namespace gsr

using namespace gsr;

extern "C" {

size_t gsr_class_loss_workspace(int64_t n, int64_t classes, int32_t d, int32_t dtype) {
    if (n < 0 || n >= kMaxRows || classes < 1 || classes >= kMaxRows || d < 1 || d > kMaxClassWidth ||
        (dtype != GSR_F32 && dtype != GSR_BF16))
        return 0;
    return class_plan(n, classes, d, dtype).loss_bytes;
}
size_t gsr_class_grad_workspace(int64_t n, int64_t classes, int32_t d, int32_t dtype) {
    return gsr_class_loss_workspace(n, classes, d, dtype) ? class_plan(n, classes, d, dtype).grad_bytes : 0;
}

gsr_status_t gsr_class_loss(const void* x, int64_t ldx, int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype, const void* table,
                            int64_t classes, int64_t ldt, const float* bias, const void* ids, int32_t ids_i64, float* loss_out, float* lse_out,
                            void* workspace, size_t workspace_bytes, void* stream) {
    ClassShape s;
    GSR_TRY(class_shape(x, ldx, n, d, c, layout, dtype, table, classes, ldt, bias, ids, ids_i64, &s));
    if (!loss_out || (n > 0 && !lse_out)) return fail(GSR_ERR_INVALID_ARG, "null loss_out or lse_out");
    if (!aligned_to(loss_out, 4) || !aligned_to(lse_out, 4)) return fail(GSR_ERR_INVALID_ARG, "loss_out or lse_out is not aligned to its elements");
    const ClassPlan p = class_plan(n, classes, d, dtype);
    GSR_TRY(class_workspace(p.loss_bytes, workspace, workspace_bytes));
    hipStream_t st = (hipStream_t)stream;
    char* ws = (char*)workspace;
    int q = 0;                                  // lanes of a row in the join of the splits
    while (q < 6 && 4 << q < p.loss_splits && n << (q + 1) <= 65536) ++q;
    const int blocks = n << q <= 4096 ? (n ? 1 : 0) : (int)((n + (1024 >> q) - 1) / (1024 >> q));
    LossPart* parts = (LossPart*)(ws + p.parts);
    if (n) {
        const ClassSetup a = launch_setup(s, p, bias, nullptr, ws, dtype, st);
        const ClassLossArgs g{a.xf, a.ef, a.x_scale, a.e_scale, a.bias_out, a.target, (SoftmaxSum*)(ws + p.part), (float*)(ws + p.at_target), p.x_pad,
                              (int32_t)((classes + kTileRows - 1) / kTileRows), p.loss_splits};
        by_steps(p.ks, [&](auto k) {
            constexpr int KS = k.value, R1 = loss_blocks(KS, 1), R2 = loss_blocks(KS, 2);
            const dim3 grid((unsigned)((n + 64 * p.loss_rb - 1) / (64 * p.loss_rb)), (unsigned)p.loss_splits);
            if (dtype == GSR_F32) hipLaunchKernelGGL((k_class_loss<KS, 2, R2>), grid, dim3(256), 0, st, g);
            else hipLaunchKernelGGL((k_class_loss<KS, 1, R1>), grid, dim3(256), 0, st, g);
        });
        hipLaunchKernelGGL(k_class_lse, dim3(blocks), dim3(1024), 0, st, g.part, g.at_target, a.target, n, p.x_pad, p.loss_splits, q, lse_out, parts, loss_out);
    }
    if (blocks != 1) hipLaunchKernelGGL(k_class_loss_sum, dim3(1), dim3(1024), 0, st, parts, blocks, loss_out);
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

gsr_status_t gsr_class_grad(const void* x, int64_t ldx, int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype, const void* table,
                            int64_t classes, int64_t ldt, const float* bias, const void* ids, int32_t ids_i64, const float* lse, float scale,
                            void* dx_out, int64_t lddx, void* dtable_out, int64_t lddt, float* dbias_out, void* workspace, size_t workspace_bytes,
                            void* stream) {
    ClassShape s;
    GSR_TRY(class_shape(x, ldx, n, d, c, layout, dtype, table, classes, ldt, bias, ids, ids_i64, &s));
    if (n > 0 && !lse) return fail(GSR_ERR_INVALID_ARG, "null lse");
    if (!dx_out && !dtable_out && !dbias_out) return fail(GSR_ERR_INVALID_ARG, "no gradient asked for");
    if (dx_out && (lddx < s.x.dg || lddx >= ((int64_t)1 << 31))) return fail(GSR_ERR_INVALID_ARG, "row stride %lld of dx_out outside [%d, 2^31)", (long long)lddx, s.x.dg);
    if (dtable_out && (lddt < d || lddt >= ((int64_t)1 << 31))) return fail(GSR_ERR_INVALID_ARG, "row stride %lld of dtable_out outside [%d, 2^31)", (long long)lddt, d);
    if (!aligned_to(lse, 4) || !aligned_to(dbias_out, 4) || !aligned_to(dx_out, dtype_size(dtype)) || !aligned_to(dtable_out, dtype_size(dtype)))
        return fail(GSR_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
    const ClassPlan p = class_plan(n, classes, d, dtype);
    GSR_TRY(class_workspace(p.grad_bytes, workspace, workspace_bytes));
    hipStream_t st = (hipStream_t)stream;
    char* ws = (char*)workspace;
    ClassSetup a{};
    a = launch_setup(s, p, bias, lse, ws, dtype, st);
    ClassGradArgs g{}, h{};                     // by row, by class
    g.lse = a.lse_out;
    g.bias = a.bias_out;
    g.target = a.target;
    g.counts = a.counts;
    g.count_blocks = (int32_t)a.row_blocks;
    g.scale = scale;
    g.d = d;
    h = g;
    if (dx_out && n) {
        g.own = a.xf;
        g.stream = a.ef;
        g.own_scale = a.x_scale;
        g.stream_scale = a.e_scale;
        g.out = dx_out;
        g.rows = n;
        g.ld = lddx;
        g.gs = n * lddx;
        g.dg = s.x.dg;
        g.own_pad = p.x_pad;
        g.part = (float*)(ws + p.x_part);
        g.tiles = (int32_t)((classes + kTileRows - 1) / kTileRows);
        g.splits = p.x_splits;
    }
    if (dtable_out || dbias_out) {
        h.own = a.ef;
        h.stream = a.xf;
        h.own_scale = a.e_scale;
        h.stream_scale = a.x_scale;
        h.out = dtable_out;
        h.dbias = dbias_out;
        h.rows = classes;
        h.ld = lddt;
        h.dg = d;
        h.own_pad = p.e_pad;
        h.part = (float*)(ws + p.e_part);
        h.bias_part = (double*)(ws + p.bias_part);
        h.tiles = (int32_t)((n + kTileRows - 1) / kTileRows);
        h.splits = p.e_splits;
    }
    by_steps(p.ks, [&](auto k) {
        if (dtype == GSR_F32) launch_grad<k.value, float>(g, h, st);
        else launch_grad<k.value, bf16_t>(g, h, st);
    });
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

}  // extern "C"
