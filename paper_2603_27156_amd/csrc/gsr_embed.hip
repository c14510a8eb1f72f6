// Node embeddings: the plane a stack of layers starts from, looked up by token, and the gradient of the table.
//
//   gsr_embed_lookup   x[n, :] = scale * E[id_n, :]
//   gsr_embed_grad     dE[v, :] = scale * sum over the rows n with id_n = v of dx[n, :]
//
// A token outside [0, vocab) has no embedding: its row of x is zero, its row of dx has no part in the sums (where such rows stand next to others in
// the sorted list they are loaded with them, and dropped).  The product is rounded to float32, which a 16-bit plane rounds once more.
#include "gsr_internal.h"
#include "gsr_pieces.h"

#include <algorithm>

namespace gsr {

// ---- lookup ---------------------------------------------------------------------------------------------
// blockIdx.y: the group (planes) or 0 (rows); a workgroup writes whole rows of it, about 512 pieces, two a thread.  `magic` divides a piece's
// number by the pieces per row (ceil(2^32 / pg), 0 for one piece; exact below 2^16).  Bound by the writes (the table comes from the caches
// unless it is larger than the plane).  They are streamed past the caches: 1M rows of 256 floats 217 -> 181 us, and with two pieces a thread
// instead of four 143 us (7.2 TB/s; a fill by itself reaches 6.8).  gsr_step on the plane right after it, lookup included: 4,990 us cached,
// 4,908 and 4,899 streamed; planes of 4 to 128 MB are as fast or faster streamed too.  Rows that start anywhere (odd widths): 4.0 to 4.4 TB/s, 1M rows of
// 77 floats 73 us; cached 70, and going on at the next multiple of 16 bytes after a row's first piece 71.5.
constexpr int kLookupPieces = 2;                // of a thread
template <typename TT, typename T, typename I, int V>
__global__ __launch_bounds__(256) void k_embed_lookup(const TT* __restrict__ table, int64_t ldt, int32_t vocab,
                                                      const I* __restrict__ ids, int64_t n, int dg, int pg, uint32_t magic,
                                                      int rows_per_wg, float scale, T* __restrict__ x, int64_t ldx, int64_t gs) {
    const int group = blockIdx.y;
    const TT* tab = table + (int64_t)group * dg;
    T* plane = x + group * gs;
    for (int64_t row0 = (int64_t)blockIdx.x * rows_per_wg; row0 < n; row0 += (int64_t)gridDim.x * rows_per_wg) {
        const int rows = n - row0 < rows_per_wg ? (int)(n - row0) : rows_per_wg;
        const uint32_t count = (uint32_t)rows * (uint32_t)pg;
        for (uint32_t t0 = threadIdx.x; t0 < count; t0 += kLookupPieces * 256) {
            constexpr int U = kLookupPieces;
            uint32_t row[U], col[U];
            int32_t id[U];
            Piece<TT, V> p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t t = t0 + 256 * u < count ? t0 + 256 * u : count - 1;
                row[u] = magic ? __umulhi(t, magic) : t;
                const uint32_t q = (t - row[u] * (uint32_t)pg) * V;
                col[u] = q + V <= (uint32_t)dg ? q : (uint32_t)(dg - V);
                id[u] = token_row(ids[row0 + row[u]], vocab);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) p[u].load(tab + (id[u] < vocab ? id[u] : 0) * ldt + col[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (t0 + 256 * u >= count) break;
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = id[u] < vocab ? scale * p[u].at(i) : 0.0f;
                store_piece<V, true>(plane + (row0 + row[u]) * ldx + col[u], v);
            }
        }
    }
}

// ---- positions sorted by token ----------------------------------------------------------------------------
// A stable counting sort, so that the sums are taken in an order that the tokens alone fix.  A pass is three launches: every workgroup counts
// the digits of its stretch; a wave per digit turns the counts into places; every workgroup hands its elements out.  Within a workgroup each
// wave owns a stretch; lanes of equal digits find their order from one ballot per bit.  Bound by its launches and the round trips in them: 500k
// elements and digits of 8 bits take 5 + 5 + 8 us a pass, for 12 MB.
// Digits of up to 10 bits (vocabularies below 1,024: one pass, below 2^20: two).  Whole gradient of 32 columns, at most 8 / 9 / 10 / 11 bits: 1M rows,
// 900 tokens 78 / 78 / 69 / 70 us, 2,000 tokens 79 / 80 / 80 / 80; 4M rows, 300 tokens 185 / 155 / 155 / 163, 200k tokens 236 / 218 / 219 / 231.
constexpr int kDigitBits = 10;
constexpr int kSortWaves = 4;
constexpr int kSortBatch = 8;        // elements that a lane has in flight
constexpr int kSortStretch = 256 * kSortBatch;   // elements of a workgroup, or a multiple of them beyond kSortWgs workgroups
constexpr int kSortWgs = 1024;
// The second launch of a pass is left out where the third can add the counts up by itself: few workgroups and digits (20,000 rows of 64 floats, 40
// tokens 22.6 -> 19.3 us in a captured graph, 5,000 tokens 40 -> 34; with 2,048 digits 16,000 rows took 53 against 32).
constexpr int kFewWgs = 32, kFewDigits = 512;
constexpr int kSmallSort = 4096;     // elements that one workgroup sorts in LDS
constexpr int kSmallBits = 8;
static_assert(kSmallSort <= 16 * 64 * 4, "a wave of the small sort takes four elements a lane");

// What the sort moves: pairs of a row of the table (or vocab) and a position.  The first pass makes them of the tokens.
struct SortPair {
    int32_t key;
    uint32_t place;
};
template <typename I>
struct TokenSource {
    const I* ids;
    int32_t vocab;
    __device__ __forceinline__ SortPair get(int64_t i) const { return {token_row(ids[i], vocab), (uint32_t)i}; }
};
struct PairSource {
    const SortPair* pairs;
    __device__ __forceinline__ SortPair get(int64_t i) const { return pairs[i]; }
};

// inclusive sum over the wave
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    const int lane = lane_id();
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = __shfl_up(v, o);
        if (lane >= o) v += t;
    }
    return v;
}

// The table's gradient is cleared by workgroups behind those of the sort's launches, a share in each: the sort waits for its round trips and leaves
// the memory to them.  Sums are stored later, over the zeros.  Streamed past the caches, 8 KB a workgroup.  8,192 rows of 1,024 floats, 128k tokens
// (525 MB; a fill takes 77 us): 149 us with all of it in the first launch, cached, 103 so; 65,536 rows of 512: 119 and 103.
struct ClearSpan {
    float* out;
    int64_t ldt, rows;
    int d, wgs;                 // the last workgroups of the launch
};
constexpr int kClearFloats = 2048;              // of a workgroup at a time
__device__ __forceinline__ void clear_rows(const ClearSpan& s, int64_t wg) {
    if (s.ldt == s.d) {
        const int64_t total = s.rows * s.d;
        for (int64_t base = wg * kClearFloats; base < total; base += (int64_t)s.wgs * kClearFloats) {
#pragma unroll
            for (int u = 0; u < kClearFloats / 1024; ++u) {
                const int64_t i = base + 1024 * u + 4 * threadIdx.x;
                const u32x4a z = {0, 0, 0, 0};
                if (i + 4 <= total) __builtin_nontemporal_store(z, reinterpret_cast<u32x4a*>(s.out + i));
                else
                    for (int64_t j = i; j < total; ++j) s.out[j] = 0.0f;
            }
        }
    } else {                                    // a wave per row
        for (int64_t row = 4 * wg + (threadIdx.x >> 6); row < s.rows; row += 4 * (int64_t)s.wgs)
            for (int col = lane_id(); col < s.d; col += 64) s.out[row * s.ldt + col] = 0.0f;
    }
}

template <typename Src>
__global__ __launch_bounds__(256) void k_embed_count(Src src, int64_t n, int stretch, int wgs, int shift, int bits, uint32_t* __restrict__ hist,
                                                     ClearSpan clear) {
    __shared__ uint32_t s_count[1 << kDigitBits];
    if ((int)blockIdx.x >= wgs) return clear_rows(clear, (int)blockIdx.x - wgs);
    const int digits = 1 << bits;
    for (int i = threadIdx.x; i < digits; i += 256) s_count[i] = 0;
    __syncthreads();
    const int64_t a = (int64_t)blockIdx.x * stretch, b = a + stretch < n ? a + stretch : n;
    for (int64_t i = a + threadIdx.x; i < b; i += kSortBatch * 256) {
        int32_t key[kSortBatch];
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u) key[u] = src.get(i + u * 256 < b ? i + u * 256 : b - 1).key;
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u)
            if (i + u * 256 < b) atomicAdd(&s_count[((uint32_t)key[u] >> shift) & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < digits; i += 256) hist[(int64_t)i * wgs + blockIdx.x] = s_count[i];
}

// counts of a digit -> elements of that digit in the workgroups before; total[digit].  A wave per digit.
__global__ __launch_bounds__(256) void k_embed_places(uint32_t* __restrict__ hist, int wgs, int digits, uint32_t* __restrict__ total,
                                                      ClearSpan clear) {
    if ((int)blockIdx.x >= (digits + 3) / 4) return clear_rows(clear, (int)blockIdx.x - (digits + 3) / 4);
    const int digit = blockIdx.x * 4 + (threadIdx.x >> 6), lane = lane_id();
    if (digit >= digits) return;
    uint32_t* h = hist + (int64_t)digit * wgs;
    uint32_t before = 0;
    for (int i = 0; i < wgs; i += 64 * kSortBatch) {
        uint32_t c[kSortBatch];
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u) {
            const int at = i + 64 * u + lane;
            c[u] = h[at < wgs ? at : wgs - 1];
            if (at >= wgs) c[u] = 0;
        }
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u) {
            const uint32_t s = wave_scan(c[u]);
            if (i + 64 * u + lane < wgs) h[i + 64 * u + lane] = before + s - c[u];
            before += __shfl(s, 63);
        }
    }
    if (lane == 0) total[digit] = before;
}

// Up to 64 kSortBatch elements from i - lane on, below b: the batch that a lane holds of them.
struct SortBatch {
    SortPair e[kSortBatch];
    template <typename Src>
    __device__ __forceinline__ void load(const Src& src, int64_t i, int64_t b) {
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u) e[u] = src.get(i + 64 * u < b ? i + 64 * u : b - 1);
    }
    __device__ __forceinline__ void count(int64_t i, int64_t b, int shift, int bits, uint32_t* counts) const {
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u)
            if (i + 64 * u < b) atomicAdd(&counts[((uint32_t)e[u].key >> shift) & ((1u << bits) - 1)], 1u);
    }
    // start[digit]: the place of the wave's next element of that digit.  The lanes of equal digits are found for N elements of the batch side by
    // side (one ballot per bit and element), only the counters are a chain: with 500k elements and digits of 8 bits 10.0 -> 8.3 us a launch
    // against one element after the other.
    template <int N>
    __device__ __forceinline__ void hand_out(int64_t i, int64_t b, int shift, int bits, uint32_t* start, SortPair* to) const {
        const uint32_t mask = (1u << bits) - 1;
        uint32_t lo[N], hi[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const uint64_t m = ballot(i + 64 * u < b);
            lo[u] = (uint32_t)m;
            hi[u] = (uint32_t)(m >> 32);
        }
        for (int x = 0; x < bits; ++x)
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const bool one = ((uint32_t)e[u].key >> (shift + x)) & 1;
                const uint64_t o = ballot(one);
                const uint32_t flip = one ? 0u : ~0u;
                lo[u] &= (uint32_t)o ^ flip;
                hi[u] &= (uint32_t)(o >> 32) ^ flip;
            }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (i - lane_id() + 64 * u >= b) break;
            const bool valid = i + 64 * u < b;
            const uint32_t digit = ((uint32_t)e[u].key >> shift) & mask;
            const int rank = __builtin_amdgcn_mbcnt_hi(hi[u], __builtin_amdgcn_mbcnt_lo(lo[u], 0));
            const uint32_t place = start[digit] + rank;
            wave_sync();
            if (valid && rank == 0) start[digit] = place + (uint32_t)(__popc(lo[u]) + __popc(hi[u]));
            wave_sync();
            if (valid) to[place] = e[u];
        }
    }
};

// exclusive sums of v[0 .. count) for a workgroup of `waves` waves; s_wave: a word per wave
__device__ __forceinline__ void wg_scan(uint32_t* v, int count, uint32_t* s_wave, int waves) {
    const int per = (count + 64 * waves - 1) / (64 * waves), a = threadIdx.x * per;
    uint32_t sum = 0;
    for (int i = a; i < a + per && i < count; ++i) sum += v[i];
    const uint32_t s = wave_scan(sum);
    if (lane_id() == 63) s_wave[threadIdx.x >> 6] = s;
    __syncthreads();
    uint32_t at = s - sum;
    for (int w = 0; a < count && w < (int)(threadIdx.x >> 6); ++w) at += s_wave[w];
    for (int i = a; i < a + per && i < count; ++i) {
        const uint32_t c = v[i];
        v[i] = at;
        at += c;
    }
    __syncthreads();
}

// A workgroup sorts 2,048 elements at a time in LDS and writes them out in that order: elements of a digit lie side by side in both places.
template <typename Src>
__global__ __launch_bounds__(256) void k_embed_hand_out(Src src, int64_t n, int stretch, int wgs, int shift, int bits,
                                                        const uint32_t* __restrict__ hist, const uint32_t* __restrict__ total,
                                                        SortPair* __restrict__ out, ClearSpan clear) {
    if ((int)blockIdx.x >= wgs) return clear_rows(clear, (int)blockIdx.x - wgs);
    constexpr int PER = (1 << kDigitBits) / 256;             // digits of a thread
    __shared__ uint32_t s_start[kSortWaves << kDigitBits];
    __shared__ uint32_t s_first[1 << kDigitBits];            // places: of a digit in the workgroup, then from there to memory
    __shared__ uint32_t s_wave[kSortWaves];
    __shared__ SortPair s_pair[kSortStretch];
    const int digits = 1 << bits, w = threadIdx.x >> 6;
    const int64_t a0 = (int64_t)blockIdx.x * stretch, b0 = a0 + stretch < n ? a0 + stretch : n;
    // what comes from memory is asked for at once: the first batch, the digits' totals and places
    SortBatch batch;
    const int64_t mine = a0 + w * (kSortStretch / kSortWaves) + lane_id();
    if (a0 < b0) batch.load(src, mine, b0);
    uint32_t next[PER];                                      // where this workgroup's next element of the thread's digits goes
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = threadIdx.x + 256 * j;
        next[j] = 0;
        if (i >= digits) break;
        if (total) {
            next[j] = hist[(int64_t)i * wgs + blockIdx.x];
            s_first[i] = total[i];
        } else {                                             // counts, of a few workgroups
            uint32_t c[kFewWgs], sum = 0;
#pragma unroll
            for (int v = 0; v < kFewWgs; ++v) c[v] = hist[(int64_t)i * wgs + (v < wgs ? v : 0)];
#pragma unroll
            for (int v = 0; v < kFewWgs; ++v) {
                if (v == (int)blockIdx.x) next[j] = sum;
                sum += v < wgs ? c[v] : 0;
            }
            s_first[i] = sum;
        }
    }
    __syncthreads();
    wg_scan(s_first, digits, s_wave, kSortWaves);
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (threadIdx.x + 256 * j < digits) next[j] += s_first[threadIdx.x + 256 * j];
    uint32_t* start = s_start + w * digits;
    for (int64_t a = a0; a < b0; a += kSortStretch) {
        const int64_t i = mine + (a - a0), end = a + kSortStretch < b0 ? a + kSortStretch : b0;
        const int64_t b = i - lane_id() + kSortStretch / kSortWaves < end ? i - lane_id() + kSortStretch / kSortWaves : end;
        if (a > a0) batch.load(src, i, b0);
        for (int x = threadIdx.x; x < kSortWaves * digits; x += 256) s_start[x] = 0;
        __syncthreads();
        batch.count(i, b, shift, bits, start);
        __syncthreads();
        uint32_t c[PER][kSortWaves];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int x = threadIdx.x + 256 * j;
            if (x >= digits) break;
            uint32_t sum = 0;
#pragma unroll
            for (int v = 0; v < kSortWaves; ++v) sum += c[j][v] = s_start[v * digits + x];
            s_first[x] = sum;
        }
        __syncthreads();
        wg_scan(s_first, digits, s_wave, kSortWaves);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int x = threadIdx.x + 256 * j;
            if (x >= digits) break;
            const uint32_t first = s_first[x];
            uint32_t at = first;
#pragma unroll
            for (int v = 0; v < kSortWaves; ++v) {
                s_start[v * digits + x] = at;
                at += c[j][v];
            }
            s_first[x] = next[j] - first;                    // (added modulo 2^32)
            next[j] += at - first;
        }
        __syncthreads();
        batch.hand_out<kSortBatch>(i, b, shift, bits, start, s_pair);
        __syncthreads();
        const int count = (int)(end - a);
#pragma unroll
        for (int u = 0; u < kSortBatch; ++u) {
            const int x = threadIdx.x + 256 * u;
            if (x >= count) break;
            const SortPair p = s_pair[x];
            out[x + s_first[((uint32_t)p.key >> shift) & (digits - 1)]] = p;
        }
        __syncthreads();
    }
}

// ---- sums over the rows of a token ------------------------------------------------------------------------
// The sorted list is cut into chunks of equal length, one per sub-wave of as many lanes as a row has pieces (up to 64), so that a
// token of a million rows and a million tokens of one row cost the same.  A run of equal tokens that lies in one chunk is stored as it
// is; of a run that goes on beyond its chunk the sum is left in one of the chunk's two places of a list of partial rows (0: the run goes
// on from the chunk before, 1: it begins here), whose tokens are ascending again.  The same kernel shortens that list 16-fold at a time, and
// where few chunks are left, k_embed_join adds up each run that began in one of them.
//
// Bound by the reads of dx.  Those are streamed past the caches (1M rows of 256 floats, chunks of 64: 235 -> 212 us for the whole gradient), and
// chunks are long, so that about 4,096 waves read ascending rows each (16-bit rows, in pieces of eight: half as many): float32 with 64 / 128 / 256
// rows a chunk 212 / 200 / 190 us.  With 97 tokens the sums of those rows take 159 us (6.5 TB/s; a loop that only reads past the caches 7.1), with 50k
// tokens 200 (the table's 51 MB are written twice: cleared, then stored); 500k rows of 256 16-bit values with 50k tokens 66 us for 279 MB (1,956 waves).
struct EmbedSums {
    const void* src;            // FIRST: the plane dx; else partial rows of d floats
    int64_t ld, gs;             // row and group stride
    const SortPair* pairs;      // FIRST: rows of the table, ascending (vocab: nothing), and rows of dx
    const int32_t* keys;        // else: rows of the table, ascending (negative: nothing)
    int32_t entries, chunks;
    int chunk;                  // entries per chunk, a multiple of kSumBatch
    int d;                      // columns of a row of the table
    int lanes_log2;             // lanes per chunk
    int pieces, pg, dg;         // of a whole row; of a group; columns of a group
    int32_t vocab;
    float scale;
    float* out;
    int64_t ldt;
    float* part;                // [2 chunks][d]
    int32_t* part_keys;         // [2 chunks], negative: nothing
};
constexpr int kSumLanesMin = 3;                                        // (lanes per chunk as a logarithm)
// Partial rows in flight, of a chunk; rows of dx half as many.  Whole gradient with 4 / 8 / 16 rows of dx: 1M rows of 256 floats, 97 tokens 185.1 / 186.4 /
// 186.4 us, 50,021 tokens 269 / 255 / 244; 500k rows of 256 16-bit values 69.4 / 69.3 / 69.8 and 133 / 125 / 119; 20,000 rows of 64 floats, 40 tokens
// 20.1 / 19.3 / 19.7; 1M rows of 77 floats 95.8 / 97.1 / 96.5.
constexpr int kSumBatch = 16;
constexpr int kSumEntries = 2048;                                      // of a workgroup, at most
constexpr int kPartChunk = 32;                                         // partial rows per chunk (64: 12.6 us a level, 32: 5.7)
constexpr int kJoinChunks = 1024;                                      // chunks from which k_embed_join takes over

template <typename S, int V, bool FIRST>
__global__ __launch_bounds__(256) void k_embed_sums(EmbedSums a) {
    constexpr int U = FIRST ? kSumBatch / 2 : kSumBatch;       // partial rows: few waves, each with more in flight
    __shared__ int32_t s_key[kSumEntries + 4 * (256 >> kSumLanesMin)];
    __shared__ int32_t s_pos[kSumEntries + 4 * (256 >> kSumLanesMin)];
    const int subs = 256 >> a.lanes_log2, sub = threadIdx.x >> a.lanes_log2, stride = a.chunk + 4;
    const int64_t e0 = (int64_t)blockIdx.x * subs * a.chunk;
    for (int i = threadIdx.x; i < subs * a.chunk; i += 256) {
        const int64_t e = e0 + i;
        int32_t key = -1, pos = 0;
        if (e < a.entries) {
            if constexpr (FIRST) {
                const SortPair p = a.pairs[e];
                key = p.key < a.vocab ? p.key : -1;
                pos = (int32_t)p.place;
            } else {
                key = a.keys[e];
                pos = (int32_t)e;
            }
        }
        const int at = i / a.chunk * stride + i % a.chunk;
        s_key[at] = key;
        s_pos[at] = pos;
    }
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * subs + sub;
    if (c >= a.chunks) return;
    const int32_t* keys = s_key + sub * stride;
    const int32_t* rows = s_pos + sub * stride;
    const int piece = blockIdx.y * (1 << a.lanes_log2) + (threadIdx.x & ((1 << a.lanes_log2) - 1));
    const bool mine = piece < a.pieces;
    const int q = mine ? piece : a.pieces - 1, group = q / a.pg;
    const int in_group = (q - group * a.pg) * V, col = in_group + V <= a.dg ? in_group : a.dg - V;
    const S* src = static_cast<const S*>(a.src) + group * a.gs + col;
    const int column = group * a.dg + col;
    float* out = a.out + column;

    const int64_t s = c * a.chunk, e = s + a.chunk;
    const int32_t first = keys[0];
    bool left = false, right = false;           // whether the first run goes on from before, the last one beyond
    if (first >= 0 && s > 0) left = !FIRST || a.pairs[s - 1].key == first;
    if (e < a.entries) right = FIRST ? keys[a.chunk - 1] >= 0 && a.pairs[e].key == keys[a.chunk - 1] : a.keys[e] >= 0;

    float acc[V];
    int32_t cur = -1;
    bool open = left;                           // the present run is the one that goes on from before
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    auto store = [&](bool to_part, int64_t place) {
        if (!mine) return;
        float v[V];
        if (to_part) {
            store_piece<V>(a.part + place * a.d + column, acc);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = a.scale * acc[i];
            store_piece<V>(out + (int64_t)cur * a.ldt, v);
        }
    };
    for (int b = 0; b < a.chunk; b += U) {
        int32_t k[U];
        Piece<S, V> p[U];
        bool any = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            k[u] = keys[b + u];
            any |= k[u] >= 0;
        }
        if (!__any(any)) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) p[u].template load<FIRST>(src + rows[b + u] * a.ld);
        bool same = cur >= 0;
#pragma unroll
        for (int u = 0; u < U; ++u) same &= k[u] == cur;
        if (same) {                             // a batch within a run, added up by pairs: a sum of 256 rows is 35 additions deep
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = p[u].at(i);
#pragma unroll
                for (int w = U / 2; w; w /= 2)
#pragma unroll
                    for (int u = 0; u < w; ++u) v[u] += v[u + w];
                acc[i] += v[0];
            }
            continue;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (k[u] < 0) continue;
            if (k[u] != cur) {
                if (cur >= 0) store(open, 2 * c);
                open = open && cur < 0;
                cur = k[u];
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += p[u].at(i);
        }
    }
    if (cur >= 0) store(open || right, open ? 2 * c : 2 * c + 1);
    if (piece == 0) {
        a.part_keys[2 * c] = left ? first : -1;
        a.part_keys[2 * c + 1] = right && !open ? cur : -1;
    }
}

// Partial rows of `chunks` chunks: workgroup (i, j) adds up the run that began in chunk i, if one did, in columns 16 V j to 16 V (j + 1): the place
// where it begins and the first places of the chunks after it that carry on its token.  Sixteen lanes take a row, sixteen rows side by side, eight of
// each in flight: 4.7 us for 245 chunks of 1M rows, and two levels of k_embed_sums (20 us) less.
template <int V>
__global__ __launch_bounds__(256) void k_embed_join(const float* __restrict__ part, const int32_t* __restrict__ keys, int chunks, int d,
                                                    float scale, float* __restrict__ out, int64_t ldt) {
    constexpr int U = 8;
    __shared__ float s_sum[16][16 * V];
    const int i = blockIdx.x;
    const int32_t key = keys[2 * i + 1];
    if (key < 0) return;
    int more = 0, found;
    do {                                        // every thread looks at a chunk: those that carry on come first
        const int j = i + 1 + more + (int)threadIdx.x;
        found = __syncthreads_count(j < chunks && keys[2 * (j < chunks ? j : chunks - 1)] == key);
        more += found;
    } while (found == 256);
    const int sub = threadIdx.x >> 4, lane = threadIdx.x & 15, piece = blockIdx.y * 16 + lane;
    const int col = piece * V + V <= d ? piece * V : d - V;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.0f;
    for (int r = sub; r <= more; r += 16 * U) {
        Piece<float, V> p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = r + 16 * u <= more ? r + 16 * u : more;
            p[u].load(part + (int64_t)(row ? 2 * (i + row) : 2 * i + 1) * d + col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (r + 16 * u <= more) acc[e] += p[u].at(e);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) s_sum[sub][lane * V + e] = acc[e];
    __syncthreads();
    if (threadIdx.x >= 16 || piece * V >= d) return;
    const int rows = more + 1 < 16 ? more + 1 : 16;
    for (int s = 1; s < rows; ++s)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] += s_sum[s][lane * V + e];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] *= scale;
    store_piece<V>(out + (int64_t)key * ldt + col, acc);
}

// ---- few rows: one launch ----------------------------------------------------------------------------------
// Up to kSmallSort rows.  Every workgroup sorts all positions by itself in LDS (digits of up to 8 bits; the others do the same at the same
// time), then takes the runs that begin among its kSmallSpan sorted entries, in 64 columns (16 without pieces): 64 sub-waves cut those
// entries evenly, a run that goes on in the next sub-wave's part is joined through LDS.  Rows of the table without a token are cleared by the
// workgroups too, each its share, unless they are too many for that (`clear`).
constexpr int kSmallSpan = 512, kSmallSubs = 64;

template <typename S, int V, typename I>
__global__ __launch_bounds__(1024) void k_embed_small(TokenSource<I> ids, int n, int bits, int passes, EmbedSums a, int clear) {
    constexpr int W = 16, U = kSumBatch / 2, FLAGS = W << kSmallBits;
    __shared__ SortPair s_pair[2][kSmallSort];
    __shared__ uint32_t s_start[W << kSmallBits];
    __shared__ uint32_t s_first[1 << kSmallBits];
    __shared__ uint32_t s_wave[W];
    __shared__ float s_part[kSmallSubs][16 * V];             // sums of runs that go on from the sub-wave before
    __shared__ int32_t s_on[kSmallSubs + 8];                 // their tokens, or -1 (8 more: read ahead)
    __shared__ int s_bound[3];
    const int digits = 1 << bits, w = threadIdx.x >> 6, share = (n + 64 * W - 1) / (64 * W) * 64;
    const int wa = w * share < n ? w * share : n, wb = wa + share < n ? wa + share : n;
    for (int p = 0; p < passes; ++p) {
        uint32_t* start = s_start + w * digits;
        SortBatch batch;                                     // (at most 256 elements per wave)
        if (wa < wb) {
            if (p == 0) batch.load(ids, wa + lane_id(), wb);
            else batch.load(PairSource{s_pair[p & 1]}, wa + lane_id(), wb);
        }
        for (int i = threadIdx.x; i < W * digits; i += 1024) s_start[i] = 0;
        __syncthreads();
        if (wa < wb) batch.count(wa + lane_id(), wb, p * bits, bits, start);
        __syncthreads();
        if ((int)threadIdx.x < digits) {
            uint32_t c[W], sum = 0;
#pragma unroll
            for (int v = 0; v < W; ++v) c[v] = s_start[v * digits + threadIdx.x];
#pragma unroll
            for (int v = 0; v < W; ++v) {
                s_start[v * digits + threadIdx.x] = sum;
                sum += c[v];
            }
            s_first[threadIdx.x] = sum;
        }
        __syncthreads();
        wg_scan(s_first, digits, s_wave, W);
        for (int i = threadIdx.x; i < W * digits; i += 1024) s_start[i] += s_first[i & (digits - 1)];
        __syncthreads();
        if (wa < wb) {
            if (share <= 64) batch.hand_out<1>(wa + lane_id(), wb, p * bits, bits, start, s_pair[(p + 1) & 1]);
            else if (share <= 128) batch.hand_out<2>(wa + lane_id(), wb, p * bits, bits, start, s_pair[(p + 1) & 1]);
            else batch.hand_out<4>(wa + lane_id(), wb, p * bits, bits, start, s_pair[(p + 1) & 1]);
        }
        __syncthreads();
    }
    const SortPair* pairs = s_pair[passes & 1];
    // s_bound[i] = the entries of tokens up to `key`: the thread at the border writes it
    auto bound = [&](int i, int32_t key) {
        for (int at = threadIdx.x; at <= n; at += 1024)
            if ((at == 0 || pairs[at - 1].key <= key) && (at == n || pairs[at].key > key)) s_bound[i] = at;
    };
    bound(0, a.vocab - 1);
    __syncthreads();
    const int valid = s_bound[0], b = (int)blockIdx.x * kSmallSpan, e = b + kSmallSpan < valid ? b + kSmallSpan : valid;
    int from = 0, to = 0;                                    // the runs that begin in [b, e)
    if (b < e) {                                             // (uniform)
        if (b) bound(1, pairs[b - 1].key);
        bound(2, pairs[e - 1].key);
        __syncthreads();
        from = b ? s_bound[1] : 0;
        to = from < e ? s_bound[2] : from;
    }
    const int sub = threadIdx.x >> 4, lane = threadIdx.x & 15, piece = blockIdx.y * 16 + lane;
    const bool mine = piece < a.pieces;
    const int q = mine ? piece : a.pieces - 1, group = q / a.pg;
    const int in_group = (q - group * a.pg) * V, col = in_group + V <= a.dg ? in_group : a.dg - V;
    const S* src = static_cast<const S*>(a.src) + group * a.gs + col;
    float* out = a.out + group * a.dg + col;

    const int part = (to - from + kSmallSubs - 1) / kSmallSubs, s = from + sub * part, t = s + part < to ? s + part : to;
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
    int32_t cur = -1;
    bool open = false, right = false;
    auto store = [&]() {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = a.scale * acc[i];
        if (mine) store_piece<V>(out + (int64_t)cur * a.ldt, v);
    };
    auto leave = [&]() {
#pragma unroll
        for (int i = 0; i < V; ++i) s_part[sub][lane * V + i] = acc[i];
    };
    if (lane == 0) s_on[sub] = -1;
    if (threadIdx.x < 8) s_on[kSmallSubs + threadIdx.x] = -1;
    if (s < t) {
        open = s > from && pairs[s - 1].key == pairs[s].key;
        right = t < to && pairs[t].key == pairs[t - 1].key;
        if (open && lane == 0) s_on[sub] = pairs[s].key;
        for (int i0 = s; i0 < t; i0 += U) {
            int32_t k[U];
            Piece<S, V> p[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const SortPair e = pairs[i0 + u < t ? i0 + u : t - 1];
                k[u] = e.key;
                p[u].load(src + (int64_t)e.place * a.ld);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u >= t) break;
                if (k[u] != cur) {
                    if (cur >= 0) {
                        if (open) leave();
                        else store();
                        open = false;
                    }
                    cur = k[u];
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += p[u].at(i);
            }
        }
        if (open) leave();
    }
    __syncthreads();
    if (cur >= 0 && !open) {                                 // the last run began here: what follows of it is in the next places
        for (int j = sub + 1; right && j < kSmallSubs; j += 8) {
            float v[8][V];                                   // all asked for before the first is looked at
            int32_t on[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                on[x] = s_on[j + x];
#pragma unroll
                for (int i = 0; i < V; ++i) v[x][i] = s_part[j + x < kSmallSubs ? j + x : j][lane * V + i];
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                right = right && on[x] == cur;
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += right ? v[x][i] : 0.0f;
            }
        }
        store();
    }
    if (!clear) return;
    uint8_t* has = reinterpret_cast<uint8_t*>(s_start);      // whether a token occurs, FLAGS rows of the table at a time
    const int64_t each = ((int64_t)a.vocab + gridDim.x - 1) / gridDim.x, v0 = blockIdx.x * each;
    const int64_t v1 = v0 + each < a.vocab ? v0 + each : a.vocab;
    for (int64_t base = v0; base < v1; base += FLAGS) {
        const int count = v1 - base < FLAGS ? (int)(v1 - base) : FLAGS;
        for (int i = threadIdx.x; i < count; i += 1024) has[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < valid; i += 1024)
            if (pairs[i].key >= base && pairs[i].key < base + count) has[pairs[i].key - base] = 1;
        __syncthreads();
        const float zero[V] = {};
        for (int r = sub; r < count; r += kSmallSubs)
            if (!has[r] && mine) store_piece<V, true>(out + (base + r) * a.ldt, zero);
        __syncthreads();
    }
}
__global__ __launch_bounds__(256) void k_embed_clear(ClearSpan clear) { clear_rows(clear, blockIdx.x); }

// ---- host side ----------------------------------------------------------------------------------------------
namespace {

constexpr int kMaxWidth = 1 << 17;
// Elements of the table that k_embed_small clears beside its sums; a launch of its own costs a call but has the whole chip: 10 rows of 64 columns,
// tables of 0.3 / 4 / 15 MB 9.0 / 9.4 / 10.5 us beside the sums, 12.2 / 12.6 / 12.4 before them, 1,000 rows 12.1 / 12.9 / 14.3 and 12.7 / 13.3 / 15.1;
// 2,048 rows and 525 MB 114 and 106.
constexpr int64_t kSmallClear = 1 << 22;

struct EmbedShape {             // a plane as the kernels take it: one group, or one per plane
    int64_t n, ldx, gs;
    int dg, c;
};

gsr_status_t embed_shape(int64_t n, int32_t d, int32_t c, int32_t layout, int64_t ldx, int64_t vocab, int64_t ldt, EmbedShape* s) {
    if (n < 0) return fail(GSR_ERR_INVALID_ARG, "negative n");
    if (n >= ((int64_t)1 << 31)) return fail(GSR_ERR_UNSUPPORTED, "n=%lld at or above 2^31", (long long)n);
    if (d < 1 || d > kMaxWidth) return fail(GSR_ERR_UNSUPPORTED, "d=%d outside [1, %d]", d, kMaxWidth);
    if (c < 1 || d % c) return fail(GSR_ERR_UNSUPPORTED, "c=%d does not divide d=%d", c, d);
    if (layout != GSR_LAYOUT_ROW_MAJOR && layout != GSR_LAYOUT_GROUP_PLANAR) return fail(GSR_ERR_INVALID_ARG, "layout %d", layout);
    s->n = n;
    s->c = layout == GSR_LAYOUT_GROUP_PLANAR ? c : 1;       // the groups of a row-major plane are its columns in order
    s->dg = d / s->c;
    s->ldx = ldx;
    s->gs = n * ldx;
    if (s->c > 65535) return fail(GSR_ERR_UNSUPPORTED, "c=%d above 65535", c);
    if (ldx < s->dg || ldx >= ((int64_t)1 << 31)) return fail(GSR_ERR_INVALID_ARG, "row stride %lld outside [%d, 2^31)", (long long)ldx, s->dg);
    if (vocab < 1) return fail(GSR_ERR_INVALID_ARG, "vocab=%lld below 1", (long long)vocab);
    if (vocab >= ((int64_t)1 << 31) - 1) return fail(GSR_ERR_UNSUPPORTED, "vocab=%lld at or above 2^31 - 1", (long long)vocab);
    if (ldt < d || ldt >= ((int64_t)1 << 31)) return fail(GSR_ERR_INVALID_ARG, "row stride %lld of the table outside [%d, 2^31)", (long long)ldt, d);
    return GSR_OK;
}
gsr_status_t plane_dtype(int32_t dtype) {
    if (dtype != GSR_F32 && dtype != GSR_BF16) return fail(GSR_ERR_UNSUPPORTED, "dtype %d", dtype);
    return GSR_OK;
}
bool aligned_to(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

template <typename TT, typename T, typename I, int V>
void launch_lookup(const EmbedShape& s, const void* table, int64_t ldt, int32_t vocab, const void* ids, float scale, void* x, hipStream_t st) {
    const int pg = (s.dg + V - 1) / V, rows = std::max(1, 256 * kLookupPieces / pg);
    const unsigned wgs = (unsigned)std::min<int64_t>((s.n + rows - 1) / rows, 1 << 20);
    const uint32_t magic = pg == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + pg - 1) / pg);
    hipLaunchKernelGGL((k_embed_lookup<TT, T, I, V>), dim3(wgs, s.c), dim3(256), 0, st, (const TT*)table, ldt, vocab, (const I*)ids, s.n, s.dg,
                       pg, magic, rows, scale, (T*)x, s.ldx, s.gs);
}
template <typename TT, typename T, typename I>
void launch_lookup(const EmbedShape& s, const void* table, int64_t ldt, int32_t vocab, const void* ids, float scale, void* x, hipStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    if (s.dg >= V) launch_lookup<TT, T, I, V>(s, table, ldt, vocab, ids, scale, x, st);
    else launch_lookup<TT, T, I, 1>(s, table, ldt, vocab, ids, scale, x, st);
}
template <typename TT, typename T>
void launch_lookup(const EmbedShape& s, const void* table, int64_t ldt, int32_t vocab, const void* ids, bool i64, float scale, void* x, hipStream_t st) {
    if (i64) launch_lookup<TT, T, int64_t>(s, table, ldt, vocab, ids, scale, x, st);
    else launch_lookup<TT, T, int32_t>(s, table, ldt, vocab, ids, scale, x, st);
}

// How gsr_embed_grad sorts and cuts, and where its workspace holds what.  Depends on the sizes alone.
struct EmbedPlan {
    int bits, passes;               // bits of a digit
    bool small;
    int wgs, stretch;               // workgroups of a pass and elements of each
    int chunk;
    size_t pairs[2], hist, total;
    struct Level { int64_t entries, chunks; size_t part, part_keys; } level[8];
    int levels;
    size_t bytes;
};
EmbedPlan embed_plan(int64_t n, int64_t vocab, int d) {
    EmbedPlan p{};
    int bits = 1;
    while (((int64_t)1 << bits) <= vocab) ++bits;           // keys are 0 .. vocab
    // one launch against five or more, a call from Python: 4,096 rows of 64 floats, 40 tokens 14 us / 22, one token 23 / 22, of 256 floats,
    // 1,000 tokens 18 / 25 (2,000 rows of 64, 40 tokens: 11 us).  Every 64 columns of 512 rows sort again: with 1,000 tokens 4,096 x 4,096 43 / 47,
    // 4,096 x 8,192 84 / 70.
    p.small = n <= kSmallSort && n * d <= (int64_t)1 << 24;
    const int most = p.small ? kSmallBits : kDigitBits;
    p.passes = (bits + most - 1) / most;
    p.bits = (bits + p.passes - 1) / p.passes;
    const int64_t stretches = std::max<int64_t>(1, (n + kSortStretch - 1) / kSortStretch);
    p.stretch = kSortStretch * (int)((stretches + kSortWgs - 1) / kSortWgs);
    p.wgs = (int)std::max<int64_t>(1, (n + p.stretch - 1) / p.stretch);
    if (p.small) return p;                                  // the workspace is not used
    p.chunk = 16;
    // so few chunks that they are joined at once: 20,000 rows of 64 floats 26.0 -> 22.6 us; with chunks of 64 60,000 rows take longer, not less
    if (n > 16 * kJoinChunks && n <= 32 * kJoinChunks) p.chunk = 32;
    while (p.chunk < 256 && p.chunk < (n * d) >> 20 && p.chunk < d) p.chunk *= 2;       // about 4,096 waves of float32 rows, kSumEntries
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        p.pairs[i] = i < p.passes ? take(sizeof(SortPair) * (size_t)n) : p.pairs[0];
    }
    p.hist = take(((size_t)std::min<int64_t>(stretches, kSortWgs) << p.bits) * 4);      // (p.wgs at most, and not falling as n grows)
    p.total = take(((size_t)1 << p.bits) * 4);
    int64_t entries = n;
    int chunk = p.chunk;
    do {
        EmbedPlan::Level& l = p.level[p.levels++];
        l.entries = entries;
        l.chunks = (entries + chunk - 1) / chunk;           // several: more than 4,096 rows, or 129 and chunks of under n / 4; then more than 2,048 entries
        l.part_keys = take((size_t)l.chunks * 2 * 4);
        l.part = take((size_t)l.chunks * 2 * d * 4);
        entries = 2 * l.chunks;
        chunk = kPartChunk;
    } while (entries > 2 * kJoinChunks);
    p.bytes = at;
    return p;
}

// Workspace for n rows and for any fewer of them.  That of one size falls behind the last size of a chunk length, so those sizes count too.
size_t embed_workspace(int64_t n, int64_t vocab, int d) {
    size_t bytes = embed_plan(n, vocab, d).bytes;
    auto last_size = [&](int64_t m) {
        if (m < n) bytes = std::max(bytes, embed_plan(m, vocab, d).bytes);
    };
    last_size(16 * kJoinChunks);
    for (int64_t chunk = 16; chunk < 256; chunk *= 2) last_size((((chunk + 1) << 20) - 1) / d);
    return bytes;
}

// share k of n of the rows of a gradient
ClearSpan clear_share(float* out, int64_t ldt, int64_t vocab, int d, int k, int n) {
    const int64_t a = vocab * k / n, rows = vocab * (k + 1) / n - a;
    const int64_t wgs = ldt == d ? (rows * d + kClearFloats - 1) / kClearFloats : (rows + 3) / 4;
    return {out + a * ldt, ldt, rows, d, (int)std::min<int64_t>(wgs, 1 << 20)};
}

EmbedSums sums_of(const EmbedShape& s, const void* dx, int d, float scale, int64_t vocab, float* out, int64_t ldt) {
    EmbedSums a{};
    a.vocab = (int32_t)vocab;
    a.scale = scale;
    a.out = out;
    a.ldt = ldt;
    a.d = d;
    a.src = dx;
    a.ld = s.ldx;
    a.gs = s.gs;
    a.dg = s.dg;
    return a;
}

template <typename S, int V, typename I>
void launch_small(const EmbedPlan& p, const void* ids, int64_t n, EmbedSums a, hipStream_t st) {
    a.pg = (a.dg + V - 1) / V;
    a.pieces = a.pg * (a.d / a.dg);
    const int slabs = (a.pieces + 15) / 16;
    const bool clear = (int64_t)a.vocab * a.d <= kSmallClear;
    int64_t wgs = std::max<int64_t>(1, (n + kSmallSpan - 1) / kSmallSpan);
    if (clear) wgs = std::max(wgs, std::min<int64_t>(std::max(1, 256 / slabs), ((int64_t)a.vocab + 511) / 512));
    if (!clear) {
        const ClearSpan all = clear_share(a.out, a.ldt, a.vocab, a.d, 0, 1);
        hipLaunchKernelGGL(k_embed_clear, dim3(all.wgs), dim3(256), 0, st, all);
    }
    const TokenSource<I> src{(const I*)ids, a.vocab};
    hipLaunchKernelGGL((k_embed_small<S, V, I>), dim3((unsigned)wgs, slabs), dim3(1024), 0, st, src, (int)n, p.bits, p.passes, a, (int)clear);
}
template <typename I>
void launch_small(const EmbedPlan& p, const void* ids, int64_t n, int32_t dtype, const EmbedSums& a, hipStream_t st) {
    if (dtype == GSR_F32 && a.dg >= 4) launch_small<float, 4, I>(p, ids, n, a, st);
    else if (dtype == GSR_F32) launch_small<float, 1, I>(p, ids, n, a, st);
    else if (a.dg >= 4) launch_small<bf16_t, 4, I>(p, ids, n, a, st);
    else launch_small<bf16_t, 1, I>(p, ids, n, a, st);
}

template <typename S, int V, bool FIRST>
void launch_level(const EmbedPlan& p, int level, EmbedSums a, char* ws, hipStream_t st) {
    const EmbedPlan::Level& v = p.level[level];
    a.entries = (int32_t)v.entries;
    a.chunks = (int32_t)v.chunks;
    a.part = (float*)(ws + v.part);
    a.part_keys = (int32_t*)(ws + v.part_keys);
    a.chunk = FIRST ? p.chunk : kPartChunk;
    a.pg = (a.dg + V - 1) / V;
    a.pieces = a.pg * (a.d / a.dg);
    a.lanes_log2 = kSumLanesMin;
    while (a.lanes_log2 < 6 && (1 << a.lanes_log2) < a.pieces) ++a.lanes_log2;
    const int subs = 256 >> a.lanes_log2, lanes = 1 << a.lanes_log2;
    const dim3 grid((unsigned)((v.chunks + subs - 1) / subs), (unsigned)((a.pieces + lanes - 1) / lanes));
    hipLaunchKernelGGL((k_embed_sums<S, V, FIRST>), grid, dim3(256), 0, st, a);
}

void launch_sums(const EmbedPlan& p, EmbedSums a, int32_t dtype, int last, char* ws, hipStream_t st) {
    const int d = a.d;
    a.pairs = (const SortPair*)(ws + p.pairs[last]);
    if (dtype == GSR_F32 && a.dg >= 4) launch_level<float, 4, true>(p, 0, a, ws, st);
    else if (dtype == GSR_F32) launch_level<float, 1, true>(p, 0, a, ws, st);
    else if (a.dg >= 8) launch_level<bf16_t, 8, true>(p, 0, a, ws, st);
    else launch_level<bf16_t, 1, true>(p, 0, a, ws, st);
    a.ld = a.dg = d;
    a.gs = 0;
    for (int l = 1; l < p.levels; ++l) {
        a.src = ws + p.level[l - 1].part;
        a.keys = (const int32_t*)(ws + p.level[l - 1].part_keys);
        if (d >= 4) launch_level<float, 4, false>(p, l, a, ws, st);
        else launch_level<float, 1, false>(p, l, a, ws, st);
    }
    const EmbedPlan::Level& v = p.level[p.levels - 1];
    const float* part = (const float*)(ws + v.part);
    const int32_t* keys = (const int32_t*)(ws + v.part_keys);
    if (d >= 4)
        hipLaunchKernelGGL((k_embed_join<4>), dim3((unsigned)v.chunks, (d + 63) / 64), dim3(256), 0, st, part, keys, (int)v.chunks, d, a.scale, a.out, a.ldt);
    else
        hipLaunchKernelGGL((k_embed_join<1>), dim3((unsigned)v.chunks, 1), dim3(256), 0, st, part, keys, (int)v.chunks, d, a.scale, a.out, a.ldt);
}

template <typename I>
int launch_sort(const EmbedPlan& p, const void* ids, int64_t n, int64_t vocab, float* out, int64_t ldt, int d, char* ws, hipStream_t st) {
    const TokenSource<I> src{(const I*)ids, (int32_t)vocab};
    auto at = [&](size_t o) { return ws + o; };
    uint32_t *hist = (uint32_t*)at(p.hist), *total = (uint32_t*)at(p.total);
    const int digits = 1 << p.bits;
    if (p.wgs <= kFewWgs && digits <= kFewDigits) total = nullptr;
    const int launches = p.passes * (total ? 3 : 2);
    int launch = 0;
    auto share = [&] { return clear_share(out, ldt, vocab, d, launch++, launches); };
    for (int i = 0; i < p.passes; ++i) {
        const int to = i & 1;
        SortPair* out_pairs = (SortPair*)at(p.pairs[to]);
        const PairSource again{(const SortPair*)at(p.pairs[to ^ 1])};
        ClearSpan clear = share();
        if (i == 0)
            hipLaunchKernelGGL((k_embed_count<TokenSource<I>>), dim3(p.wgs + clear.wgs), dim3(256), 0, st, src, n, p.stretch, p.wgs, 0, p.bits, hist,
                               clear);
        else
            hipLaunchKernelGGL((k_embed_count<PairSource>), dim3(p.wgs + clear.wgs), dim3(256), 0, st, again, n, p.stretch, p.wgs, i * p.bits, p.bits,
                               hist, clear);
        if (total) {
            clear = share();
            hipLaunchKernelGGL(k_embed_places, dim3((digits + 3) / 4 + clear.wgs), dim3(256), 0, st, hist, p.wgs, digits, total, clear);
        }
        clear = share();
        if (i == 0)
            hipLaunchKernelGGL((k_embed_hand_out<TokenSource<I>>), dim3(p.wgs + clear.wgs), dim3(256), 0, st, src, n, p.stretch, p.wgs, 0, p.bits,
                               hist, total, out_pairs, clear);
        else
            hipLaunchKernelGGL((k_embed_hand_out<PairSource>), dim3(p.wgs + clear.wgs), dim3(256), 0, st, again, n, p.stretch, p.wgs, i * p.bits,
                               p.bits, hist, total, out_pairs, clear);
    }
    return (p.passes - 1) & 1;
}

}  // namespace
}  // namespace gsr

using namespace gsr;

extern "C" {

gsr_status_t gsr_embed_lookup(const void* table, int64_t vocab, int64_t ldt, int32_t table_dtype, const void* ids, int32_t ids_i64,
                              int64_t n, int32_t d, int32_t c, int32_t layout, int32_t dtype, float scale, void* x_out, int64_t ldx,
                              void* stream) {
    EmbedShape s;
    GSR_TRY(embed_shape(n, d, c, layout, ldx, vocab, ldt, &s));
    GSR_TRY(plane_dtype(table_dtype));
    GSR_TRY(plane_dtype(dtype));
    if (n == 0) return GSR_OK;
    if (!table || !ids || !x_out) return fail(GSR_ERR_INVALID_ARG, "null pointer");
    if (!aligned_to(table, dtype_size(table_dtype)) || !aligned_to(x_out, dtype_size(dtype)) || !aligned_to(ids, ids_i64 ? 8 : 4))
        return fail(GSR_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
    hipStream_t st = (hipStream_t)stream;
    const int32_t v = (int32_t)vocab;
    if (table_dtype == GSR_F32 && dtype == GSR_F32) launch_lookup<float, float>(s, table, ldt, v, ids, ids_i64, scale, x_out, st);
    else if (table_dtype == GSR_F32) launch_lookup<float, bf16_t>(s, table, ldt, v, ids, ids_i64, scale, x_out, st);
    else if (dtype == GSR_F32) launch_lookup<bf16_t, float>(s, table, ldt, v, ids, ids_i64, scale, x_out, st);
    else launch_lookup<bf16_t, bf16_t>(s, table, ldt, v, ids, ids_i64, scale, x_out, st);
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

size_t gsr_embed_grad_workspace(int64_t n, int64_t vocab, int32_t d) {
    if (n < 0 || n >= ((int64_t)1 << 31) || vocab < 1 || vocab >= ((int64_t)1 << 31) - 1 || d < 1 || d > kMaxWidth) return 0;
    return embed_workspace(n, vocab, d);
}

gsr_status_t gsr_embed_grad(const void* ids, int32_t ids_i64, int64_t n, const void* dx, int64_t ldx, int32_t d, int32_t c, int32_t layout,
                            int32_t dtype, float scale, int64_t vocab, float* dtable_out, int64_t ldt, void* workspace,
                            size_t workspace_bytes, void* stream) {
    EmbedShape s;
    GSR_TRY(embed_shape(n, d, c, layout, ldx, vocab, ldt, &s));
    GSR_TRY(plane_dtype(dtype));
    if (!dtable_out || (n > 0 && (!ids || !dx))) return fail(GSR_ERR_INVALID_ARG, "null pointer");
    const EmbedPlan p = embed_plan(n, vocab, d);
    if (workspace_bytes < p.bytes) return fail(GSR_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
    if (p.bytes && !workspace) return fail(GSR_ERR_INVALID_ARG, "null workspace");
    if (!aligned_to(dx, dtype_size(dtype)) || !aligned_to(dtable_out, 4) || !aligned_to(ids, ids_i64 ? 8 : 4) || !aligned_to(workspace, 16))
        return fail(GSR_ERR_INVALID_ARG, "a pointer is not aligned to its elements (the workspace: to 16 bytes)");
    hipStream_t st = (hipStream_t)stream;
    char* ws = (char*)workspace;
    const EmbedSums a = sums_of(s, dx, d, scale, vocab, dtable_out, ldt);
    if (p.small) {
        if (ids_i64) launch_small<int64_t>(p, ids, n, dtype, a, st);
        else launch_small<int32_t>(p, ids, n, dtype, a, st);
    } else {
        const int last = ids_i64 ? launch_sort<int64_t>(p, ids, n, vocab, dtable_out, ldt, d, ws, st)
                                 : launch_sort<int32_t>(p, ids, n, vocab, dtable_out, ldt, d, ws, st);
        launch_sums(p, a, dtype, last, ws, st);
    }
    GSR_HIP_CHECK(hipGetLastError());
    return GSR_OK;
}

}  // extern "C"
