// Multi-head attention with a learned bias by the bucket of the distance between key and query, forward and backward:
//   s_ij = scale q_i . k_j + table[h][bucket(j - i - start)],  p = softmax over the visible j,  y_i = sum_j p_ij v_j
//   delta_i = sum_j p_ij (dy_i . v_j) = dy_i . y_i,  ds_ij = p_ij (dy_i . v_j - delta_i),  dv_j = sum_i p_ij dy_i,  dq_i = scale sum_j ds_ij k_j,
//   dk_j = scale sum_i ds_ij q_i,  dtable[h][b] = sum of ds over the pairs of bucket b
// Scores are never stored: the forward pass walks the keys once with the running maximum and sum of each row's softmax, the backward pass
// makes p again from the two.  A block has 128 rows (queries; keys in the kernel that makes dk and dv), a wavefront 32 of them, or two or four wavefronts share 32 rows
// where blocks are few; tiles of the other side's rows go through LDS, the next one on its way while one is at work.  The products are formed
// transposed -- keys x queries = K Q' -- so that a lane holds scores of one query: a row's statistics need one lane exchange, and the
// probabilities already lie as the next product's operand (matrix.h), whose other operand is read from the same LDS tile by columns.
// A piece's products run in a fixed order with their LDS operands six ahead, and the softmax of a piece stands beside the product of the piece before, so
// that the matrix cores work while it does.
// Bias: the buckets' values by distance, -reach .. reach and a margin of repeated ends, lie in LDS, over the scale, and the sums q . k begin with them; pieces wholly
// beyond the reach begin with one number.  Its gradient: sums of ds along the diagonals of 32 x 32 tiles, which a wavefront carries from tile to tile, so
// that each distance is stored once per wavefront; two small kernels add up wavefronts, then the distances of a bucket.  No atomics: every sum has one order.
// What bounds it: with long sequences the matrix cores and what runs beside them on one card's power -- 16 heads on 4 of 8192 causal positions x 128 channels, bf16:
// forward 355 us (775 TFLOP/s), dq 470 (875), dk and dv 800 (690; 34 % of its CU cycles multiply, 56 % issue) -- with 512 positions the way into and out of a block: 96 heads x 64
// channels 19, 40 and 33 us, and 10 for the table; with one query a row the cache's bytes: 806 MB in 165 us, 4.9 TB/s.
#include "matrix.h"
#include "lds_dma.h"
#include "lpm_internal.h"
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <initializer_list>

using namespace lpm;

namespace lpm {

constexpr int RA_THREADS = 256, RA_WAVES = 4;
constexpr int RA_PAD = 96;                // margin of the bias by distance: a tile of up to 64 x 32 that is not wholly beyond the reach stays within it
constexpr int RA_MAX_REACH = 2048;
constexpr int RA_MAX_LD = 1 << 23;         // elements between positions: 128 of them are offsets of 32 bits
constexpr float RA_LOG2E = 1.4426950408889634f;
constexpr int RA_DIAG_PITCH = 36;         // floats of a line of a wavefront's diagonals

struct float2_ { float x, y; };

struct AttnArgs {
    int32_t m, H, G, pq, pk, d, causal, nb, reach, splits;
    int32_t fold;                         // forward: a block's rows are the queries of all heads that share keys (few queries)
    int64_t ldq, ldk, ldv, ldy;           // elements between positions
    float scale, scale2, inv_scale;       // scale2 = scale log2(e)
    const void *q, *k, *v, *dy;
    void *y, *dq, *dk, *dv;
    const int32_t *len, *start, *map;
    const float* table;
    float2_* stats;                       // per row (n, h, i): the softmax's reference in units of log2, and -log2 of the sum behind it (-inf: no visible key)
    float *part, *part_ml;                // splits: [split][row][d] and [split][row][2]
    float *delta, *diag;                  // backward: [row], [m H][lines][2 reach + 1]
};

// WK wavefronts share a block's 128 / WK rows, each with its 32 rows of every tile of the other side.  DMA: tiles go straight from memory to LDS (channels in
// whole 16-byte chunks, rows on whole dwords); else by way of registers, where a row's last chunk is put in order.
template <typename T, int DP, int WK_, bool DMA_, int OCC, bool SMALL = false> struct Ra {
    static constexpr int WK = WK_, BLOCKS = OCC;              // wavefronts that share rows, blocks of a CU
    static constexpr bool DMA = DMA_;
    static constexpr int EPC = Mm<T>::EPC, CHUNKS = DP / EPC, KS = DP / (2 * EPC), ES = (int)sizeof(T);
    static constexpr int BM = 128 / WK;
    static constexpr int BN = WK > 1 ? 32 * WK : ES == 2 && !(SMALL && 32 * CHUNKS % RA_THREADS == 0) ? 64 : 32;      // rows of a staged tile, whole chunks of every thread
    static constexpr int SUB = BN / (32 * WK);                // 32-row pieces of it that a wavefront takes
    static constexpr int ROW = DP * ES;                       // bytes
    static constexpr int TILE = BN * ROW;
    static constexpr int STAGE = 2 * TILE;                    // tiles of both operands
    // the tile at work, the next on its way, and the one before still in a product where that leaves OCC blocks their room in a CU
    static constexpr int STAGES = 3 * STAGE <= (OCC == 2 ? 72 : 148) * 1024 ? 3 : 2;
    static constexpr bool CARRY = STAGES == 3;
    static constexpr int LDS = STAGES * STAGE;
    // the wavefronts' diagonals: bfloat16 goes through them in a walk of its own, which needs two stages
    static constexpr int DIAGONALS = RA_WAVES * 63 * RA_DIAG_PITCH * 4;
    static constexpr int AREAS = ES == 2 ? 2 * STAGE : LDS, LDS_Q = AREAS + DIAGONALS > LDS ? AREAS + DIAGONALS : LDS;
    static constexpr int PER = BN * CHUNKS / RA_THREADS;      // chunks of a tile a thread brings
    static_assert(PER * RA_THREADS == BN * CHUNKS, "every chunk of a tile is brought by one thread");
    static constexpr int DT = DP / 32;                        // 32-channel pieces of a head
    static constexpr int AHEAD = DMA ? 6 : 2;                 // operands of a product on their way (8192 keys, dk and dv, 6 against 4: 847 -> 819 us)
    static constexpr int NU = 16 / EPC;                       // operands of a column of 32 probabilities
    // Chunk c of a row lies at position c ^ place(row).  A row-wise read takes one chunk of eight rows at a time, a column-wise one 64 bytes of four rows: of
    // the 256 bytes that the banks hold side by side, four consecutive rows have a quarter each, and eight rows a position each.
    static __device__ __forceinline__ int place(int row) {
        return ROW % 256 == 0 ? (row & 3) << 2 | (row >> 1 & 2) : ROW % 128 == 0 ? (row >> 1 & 1) << 2 | (row >> 1 & 2) : row >> 1 & 2;
    }
};

// Blocks of a CU that a kernel's registers leave room for, and its tiles.  Tiles of wide heads are of 32 rows in the forward pass and for dq, where 64 would leave room for one
// block only (the forward pass of 8192 keys of 128 channels: 535 us with one, 355 with two); dk and dv have one block either way, whose 64 rows halve the barriers.
template <typename T, int DP> constexpr int RA_OCC_Q = sizeof(T) == 2 || DP <= 32 ? 2 : 1;
template <typename T, int DP> constexpr int RA_OCC_KV = DP <= 32 || (sizeof(T) == 2 && DP <= 64) ? 2 : 1;
template <typename T, int DP, int WK, bool DMA> using RaFwd = Ra<T, DP, WK, DMA, DMA || sizeof(T) == 2 || DP <= 64 ? 2 : 1, (DP > 64)>;
template <typename T, int DP, int WK, bool DMA> using RaBwdQ = Ra<T, DP, WK, DMA, DMA || DP <= 64 ? RA_OCC_Q<T, DP> : 1, (DP > 64)>;
template <typename T, int DP, int WK, bool DMA> using RaBwdKv = Ra<T, DP, WK, DMA, RA_OCC_KV<T, DP>>;

// Sixteen bytes of a row of d channels from channel c on, through a buffer whose end is the last row's: rows beyond are zeros.  Where d is no whole
// number of chunks the last one is taken from the row's end (ra_shift puts it in its place).
template <typename T> __device__ __forceinline__ unsigned ra_offset(int64_t row, int64_t ld, int c, int d) {
    constexpr int EPC = Mm<T>::EPC;
    if (c >= d) return 0xffffffffu;
    return (unsigned)((row * ld + (c + EPC > d ? d - EPC : c)) * (int64_t)sizeof(T));
}
template <typename T> __device__ __forceinline__ unsigned ra_bytes(int64_t ld, int rows, int d) {
    return rows > 0 ? (unsigned)(((int64_t)(rows - 1) * ld + d) * (int64_t)sizeof(T)) : 0u;
}
template <typename T> __device__ __forceinline__ __amdgpu_buffer_rsrc_t ra_buffer(const T* base, int64_t ld, int rows, int d) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, ra_bytes<T>(ld, rows, d), 0x00020000);
}
typedef unsigned int ra_u4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ra_load(__amdgpu_buffer_rsrc_t r, unsigned off) {
    const ra_u4 v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
    return make_uint4(v.x, v.y, v.z, v.w);
}
template <typename T> __device__ __forceinline__ uint4 ra_shift(uint4 v, int c, int d) {
    constexpr int EPC = Mm<T>::EPC;
    const int s = c + EPC > d && c < d ? (c + EPC - d) * 8 * (int)sizeof(T) : 0;
    uint64_t lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
    lo = s >= 64 ? hi >> (s & 63) : s ? lo >> s | hi << (64 - s) : lo;
    hi = s >= 64 ? 0 : hi >> s;
    return make_uint4((unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32));
}

// A tile on its way from memory to LDS, straight or in registers meanwhile: load() into stage `s` of the operand's ring, done() before the barrier behind
// which the tile is read.  The stage that load() writes is one that no wavefront reads any more: its tile was the one before the last barrier's.
template <typename T, typename R> struct RaTile {
    uint4 v[R::DMA ? 1 : R::PER];
    unsigned off[R::PER];
    unsigned char* lds;
    __device__ __forceinline__ void place(unsigned char* ring, int64_t ld, int d) {
        lds = ring;
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            const int at = i * RA_THREADS + (int)threadIdx.x, r = at / R::CHUNKS;
            off[i] = ra_offset<T>(r, ld, ((at - r * R::CHUNKS) ^ R::place(r)) * R::EPC, d);
        }
    }
    // rows row0 .. of `rows`
    __device__ __forceinline__ void load(const T* base, int64_t ld, int row0, int rows, int d, int s) {
        const int n = min(rows - row0, R::BN);
        base += (int64_t)row0 * ld;
        if constexpr (R::DMA) {
            const u32x4_ buf = buffer_words(base, ra_bytes<T>(ld, n, d));
            unsigned char* to = lds + s * R::STAGE + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024;
#pragma unroll
            for (int i = 0; i < R::PER; ++i) load_to_lds16(buf, to + i * RA_THREADS * 16, off[i]);
        } else {
            const auto buf = ra_buffer(base, ld, n, d);
#pragma unroll
            for (int i = 0; i < R::PER; ++i) v[i] = ra_load(buf, off[i]);
        }
    }
    __device__ __forceinline__ void done(int d, int s) {
        if constexpr (!R::DMA) {
#pragma unroll
            for (int i = 0; i < R::PER; ++i) {
                const int at = i * RA_THREADS + (int)threadIdx.x, r = at / R::CHUNKS;
                const uint4 w = d % R::EPC ? ra_shift<T>(v[i], ((at - r * R::CHUNKS) ^ R::place(r)) * R::EPC, d) : v[i];
                *reinterpret_cast<uint4*>(lds + s * R::STAGE + at * 16) = w;
            }
        }
    }
};
template <typename R> __device__ __forceinline__ void ra_landed() {
    if constexpr (R::DMA) LPM_WAIT_VM(0);
}
// a wavefront's 32 rows as an operand: the lane's row (`first` elements into a buffer; not there: zeros), its half of every 2 * EPC channels
template <typename T, typename R> struct RaRows {
    uint4 v[R::KS];
    __device__ __forceinline__ void load(const T* base, unsigned bytes, int64_t first, bool there, int d, int g) {
        const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, bytes, 0x00020000);
        const unsigned at = (unsigned)(first * (int64_t)sizeof(T));
#pragma unroll
        for (int s = 0; s < R::KS; ++s) {
            const int c = (2 * s + g) * R::EPC;
            v[s] = ra_load(buf, there && c < d ? at + ra_offset<T>(0, 0, c, d) : 0xffffffffu);
        }
        if constexpr (!R::DMA) {
#pragma unroll
            for (int s = 0; s < R::KS; ++s) if (d % R::EPC) v[s] = ra_shift<T>(v[s], (2 * s + g) * R::EPC, d);
        }
    }
    // row l of `rows` that lie ld elements apart
    __device__ __forceinline__ void load(const T* base, int64_t ld, int l, int rows, int d, int g) { load(base, ra_bytes<T>(ld, rows, d), l * ld, l < rows, d, g); }
};
// Where a lane finds its operands in a tile, as byte offsets from its first row: row-wise (its row, a chunk of every step) and column-wise
template <typename T, typename R> struct RaOffsets {
    int row[R::KS], col[R::DT];
    __device__ __forceinline__ explicit RaOffsets(int lane) {
#pragma unroll
        for (int s = 0; s < R::KS; ++s) row[s] = (lane & 31) * R::ROW + (((2 * s + (lane >> 5)) ^ R::place(lane & 31)) * 16);
#pragma unroll
        for (int t = 0; t < R::DT; ++t) col[t] = Mm<T>::template column<R>(t, lane);
    }
};
// Pins a value to the place where it is made (the compiler would sink arithmetic that stands beside products to where its result is used)
__device__ __forceinline__ void ra_here(float& v) { asm volatile("" : "+v"(v)); }

// A run of N products: the LDS operands read(i) are asked for AHEAD of use(i, operand), and beside(i) is arithmetic that has nothing to do with them, which runs
// while the matrix cores multiply.  The order is the code's: left to itself the compiler reads an operand, waits for it and multiplies, 130 cycles of
// latency for 32 of work.  begin() asks for the first operands -- as what stands beside the last products of the run before.
template <int N, int MOST> struct RaStream {
    static constexpr int AHEAD = N < MOST ? N : MOST, SLOTS = AHEAD + 1;
    uint4 f[SLOTS];
    template <typename F> __device__ __forceinline__ void begin(int k, F&& read) { f[k] = read(k); }
    template <typename F, typename G, typename L> __device__ __forceinline__ void run(F&& read, G&& use, L&& beside) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i + AHEAD < N) f[(i + AHEAD) % SLOTS] = read(i + AHEAD);
            use(i, f[i % SLOTS]);
            beside(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};
// What stands beside the products of a run of N before the run `next` of operands read(k): its first reads, one beside each of the last products
template <int N, typename S, typename F> __device__ __forceinline__ auto ra_before(S& next, F& read) {
    return [&](int i) __attribute__((always_inline)) {
        const int k = i - (N - S::AHEAD);
        if (N >= S::AHEAD) { if (k >= 0) next.begin(k, read); }
        else if (i == 0) {
#pragma unroll
            for (int x = 0; x < S::AHEAD; ++x) next.begin(x, read);
        }
    };
}
template <int N> __device__ __forceinline__ void ra_zero(uint4 (&w)[N]) {
#pragma unroll
    for (int x = 0; x < N; ++x) w[x] = make_uint4(0, 0, 0, 0);
}
// a lane's 16 values as operands of the next product
template <typename T, typename R> __device__ __forceinline__ void ra_pack(const mm_f16& v, uint4* w) {
    float x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = v[e];
#pragma unroll
    for (int u = 0; u < R::NU; ++u) w[u] = Mm<T>::pack(x + u * R::EPC);
}
// Row-wise operand s of a tile (`tile` points at its first row); column-wise operand: rows 2 EPC u .., channels 32 t ..
template <typename T, typename R> __device__ __forceinline__ uint4 ra_row(const unsigned char* tile, const RaOffsets<T, R>& at, int s) {
    return *reinterpret_cast<const uint4*>(tile + at.row[s]);
}
template <typename T, typename R> __device__ __forceinline__ uint4 ra_column(const unsigned char* tile, const RaOffsets<T, R>& at, int u, int t) {
    return Mm<T>::template columns<R>(tile + 2 * R::EPC * u * R::ROW, at.col[t]);
}
// four consecutive channels of a row, n of them there (WHOLE: all)
template <bool WHOLE, typename T>
__device__ __forceinline__ void ra_store4(T* p, int n, const float (&v)[4]) {
    T e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = to_store<T>(v[k]);
    if (WHOLE || n >= 4) { __builtin_memcpy(p, e, 4 * sizeof(T)); return; }
#pragma unroll
    for (int k = 0; k < 4; ++k) if (k < n) p[k] = e[k];
}
// channel of register r of piece t
__device__ __forceinline__ int ra_channel(int t, int r, int g) { return 32 * t + 4 * g + 2 * r; }

// Sums over the WK wavefronts that share rows, by pieces of 32 channels: afterwards wavefront wk holds the sums of the pieces t with t % WK == wk.  `area`
// is no longer read by anybody; every wavefront calls.
template <typename R>
__device__ __forceinline__ void ra_gather(mm_f16 (&out)[R::DT], float* area, int wq, int wk, int lane) {
    constexpr int WK = R::WK;
    if (WK == 1) return;
    float* mine = area + (int64_t)(wq * WK) * R::DT * 1024;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < R::DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *reinterpret_cast<float4*>(mine + ((wk * R::DT + t) * 4 + r) * 256 + lane * 4) = make_float4(out[t][4 * r], out[t][4 * r + 1], out[t][4 * r + 2], out[t][4 * r + 3]);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < R::DT; ++t) {
        if (t % WK != wk) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(mine + ((w * R::DT + t) * 4 + r) * 256 + lane * 4);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
            out[t][4 * r] = s.x; out[t][4 * r + 1] = s.y; out[t][4 * r + 2] = s.z; out[t][4 * r + 3] = s.w;
        }
    }
}

__device__ __forceinline__ int ra_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ int ra_keys(const AttnArgs& a, int n) { return a.len ? __builtin_amdgcn_readfirstlane(ra_clamp(a.len[n], 0, a.pk)) : a.pk; }
__device__ __forceinline__ int ra_start(const AttnArgs& a, int n) { return a.start ? __builtin_amdgcn_readfirstlane(ra_clamp(a.start[n], -(1 << 29), 1 << 29)) : 0; }
__device__ __forceinline__ bool ra_any(bool v) {
#ifdef __HIP__
    return __builtin_amdgcn_ballot_w64(v) != 0;
#else
    int s = v;
    for (int o = 1; o < 64; o <<= 1) s |= __shfl_xor(s, o, 64);
    return s != 0;
#endif
}

// The bias of `heads` heads from h on by distance, lut[head][rel + reach + RA_PAD], over the scale: the sums q . k begin with it.  Finite values stay
// finite (a mask of the type's lowest value leaves a row of such values with equal probabilities, as the formula does); *huge: some are so large
// that the differences of scores have to be taken in the order of the formula.
constexpr float RA_BIG = 3.402823466e38f, RA_HUGE = 1e28f;
__host__ __device__ inline int ra_lut(int reach) { return 2 * reach + 1 + 2 * RA_PAD; }
struct RaBias {
    static constexpr int EARLY = 2;        // entries of a thread whose buckets are on their way from the kernel's beginning on
    int id[EARLY];
    __device__ __forceinline__ void begin(const AttnArgs& a) {
#pragma unroll
        for (int k = 0; k < EARLY; ++k) id[k] = a.table ? a.map[ra_clamp((int)threadIdx.x + k * RA_THREADS - RA_PAD, 0, 2 * a.reach)] : 0;
    }
    static __device__ __forceinline__ float put(const AttnArgs& a, float b, int* huge) {
        if (!(fabsf(b) <= RA_BIG)) return b;
        const float most = a.scale2 > 1.f ? RA_BIG / a.scale2 : RA_BIG;
        b = fminf(fmaxf(b * a.inv_scale, -most), most);
        if (fabsf(b) > RA_HUGE) *huge = 1;
        return b;
    }
    // (between two barriers: nobody reads lut or *huge before the second, and *huge is 0 before the first)
    __device__ __forceinline__ void store(const AttnArgs& a, int h, int heads, float* lut, int* huge) const {
        const int n = ra_lut(a.reach), first = (int)threadIdx.x;
        for (int hh = 0; hh < heads; ++hh) {
            const float* row = a.table ? a.table + (int64_t)(h + hh) * a.nb : nullptr;
            float b[EARLY];
#pragma unroll
            for (int k = 0; k < EARLY; ++k) b[k] = row ? row[ra_clamp(id[k], 0, a.nb - 1)] : 0.f;
#pragma unroll
            for (int k = 0; k < EARLY; ++k) if (first + k * RA_THREADS < n) lut[hh * n + first + k * RA_THREADS] = put(a, b[k], huge);
            for (int t = first + EARLY * RA_THREADS; t < n; t += RA_THREADS)
                lut[hh * n + t] = row ? put(a, row[ra_clamp(a.map[ra_clamp(t - RA_PAD, 0, 2 * a.reach)], 0, a.nb - 1)], huge) : 0.f;
        }
    }
};
// whether all distances relmin .. relmax have one bias
__device__ __forceinline__ bool ra_far(int reach, int relmin, int relmax) { return relmax <= -reach || relmin >= reach; }
// (a far piece's one value is at hand: its products wait for no read of the bias)
template <int DIR> __device__ __forceinline__ mm_f16 ra_bias_of(const float* at, bool far, float end) {
    mm_f16 v;
    if (far) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = end;
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = at[DIR * ((e & 3) + 8 * (e >> 2))];
    }
    return v;
}
// Where biases are huge: a score that stands for the distance from the reference `top`, the two subtracted after the score is rounded
__device__ __forceinline__ float ra_apart(float acc, float scale2, float top) {
#pragma clang fp contract(off)
    const float v = acc * scale2;
    return (v - top) * (1.f / scale2);
}

__host__ __device__ inline int64_t ra_distances(int reach) { return 2 * (int64_t)reach + 1; }

// Blocks of one head lie on one XCD, one after the other.  Causal: those with the most visible keys first, heads in turn (REVERSE: the last tiles have the
// most), over as many heads as an XCD has -- all of them, where they do not come in eights.
struct RaBlock { int n, h, tile, split; };
template <bool REVERSE> __device__ __forceinline__ RaBlock ra_block(int m, int heads, int tiles, int splits, bool causal) {
    const int pairs = m * heads;
    RaBlock r;
    int b = (int)blockIdx.x, pair;
    if (!causal) {
        b = xcd_remap(b, (int)gridDim.x);
        r.split = b % splits;
        b /= splits;
        pair = b / tiles;
        r.tile = b - pair * tiles;
    } else {
        r.split = b % splits;
        b /= splits;
        const int sets = pairs % 8 ? 1 : 8, per = pairs / sets, x = b % sets;
        b /= sets;
        const int t = b / per;
        pair = x * per + (b - t * per);
        r.tile = REVERSE ? tiles - 1 - t : t;
    }
    r.h = pair % heads;
    r.n = pair / heads;
    return r;
}

template <typename T, int DP, int WK, bool DMA>
__global__ void __launch_bounds__(RA_THREADS, (RaFwd<T, DP, WK, DMA>::BLOCKS)) relattn_fwd(AttnArgs a) {
    typedef RaFwd<T, DP, WK, DMA> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char ra_lds[];
    int* huge = reinterpret_cast<int*>(ra_lds + R::LDS);
    float* lut = reinterpret_cast<float*>(huge + 4);
    if (threadIdx.x == 0) *huge = 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = lane & 31, g = lane >> 5, wq = wave / WK, wk = wave % WK;
    RaBias bias;
    bias.begin(a);
    const int share = a.H / a.G, rows = a.fold ? share * a.pq : a.pq, tiles = (rows + R::BM - 1) / R::BM;
    const RaBlock b = ra_block<true>(a.m, a.fold ? a.G : a.H, tiles, a.splits, a.causal);
    const int n = b.n, hk = a.fold ? b.h : b.h / share, h0 = a.fold ? hk * share : b.h;
    const int r0 = b.tile * R::BM + wq * 32, r = min(r0 + l, rows - 1);
    const int hh = a.fold ? r / a.pq : 0, i = r - hh * a.pq, h = h0 + hh;
    const bool work = r0 < rows;
    const int start = ra_start(a, n), keys = ra_keys(a, n), qpos = i + start;
    const int qmin = (a.fold ? 0 : r0) + start, qmax = (a.fold ? a.pq - 1 : min(r0 + 31, a.pq - 1)) + start;
    const T* kb = (const T*)a.k + (int64_t)n * a.pk * a.ldk + (int64_t)hk * a.d;
    const T* vb = (const T*)a.v + (int64_t)n * a.pk * a.ldv + (int64_t)hk * a.d;
    int end = keys;
    if (a.causal) end = ra_clamp((a.fold ? a.pq : min(b.tile * R::BM + R::BM, a.pq)) + start, 0, keys);
    const int all = (end + R::BN - 1) / R::BN, per = (all + a.splits - 1) / a.splits, t0 = b.split * per, t1 = min(all, t0 + per);
    RaTile<T, R> kr, vr;
    kr.place(ra_lds, a.ldk, a.d);
    vr.place(ra_lds + R::TILE, a.ldv, a.d);
    auto load = [&](int t, int stage) __attribute__((always_inline)) {
        kr.load(kb, a.ldk, t * R::BN, end, a.d, stage);
        vr.load(vb, a.ldv, t * R::BN, end, a.d, stage);
    };
    if (t0 < t1) load(t0, 0);
    RaRows<T, R> qr;
    if (a.fold)
        qr.load((const T*)a.q + (int64_t)n * a.pq * a.ldq + (int64_t)h0 * a.d, ra_bytes<T>(a.ldq, a.pq, share * a.d), i * a.ldq + hh * a.d, work, a.d, g);
    else
        qr.load((const T*)a.q + ((int64_t)n * a.pq + r0) * a.ldq + (int64_t)h * a.d, a.ldq, l, min(32, a.pq - r0), a.d, g);
    const RaOffsets<T, R> at(lane);
    __syncthreads();
    bias.store(a, h0, a.fold ? share : 1, lut, huge);
    lut += hh * ra_lut(a.reach);
    mm_f16 o[R::DT] = {};
    float top = -INFINITY, sum = 0.f, before_end = 0.f, behind_end = 0.f;      // (the bias's ends are known behind the first barrier)
    bool some_huge = false;
    // A piece's p enters its product while the next piece's is made: `prev` are the values it belongs to, w its operands.  (Before the first piece w is zero, and
    // prev the first piece's own values.)
    const unsigned char* prev = nullptr;
    uint4 w[R::NU] = {};
    RaStream<R::NU * R::DT, R::AHEAD> mix;
    auto values_of = [&](int x) __attribute__((always_inline)) { return ra_column<T, R>(prev, at, x / R::DT, x % R::DT); };
    auto add = [&](int x, uint4 f) __attribute__((always_inline)) { o[x % R::DT] = Mm<T>::mul(f, w[x / R::DT], o[x % R::DT]); };
    int stage = 0;
    auto next_tile = [&](int t) __attribute__((always_inline)) {
        kr.done(a.d, stage);
        vr.done(a.d, stage);
        ra_landed<R>();
        __syncthreads();
        if (t + 1 < t1) load(t + 1, stage == R::STAGES - 1 ? 0 : stage + 1);
    };
    // the tiles that hold keys for this wavefront: the others of the block may have more
    const int mine_end = !work ? 0 : a.causal ? min(end, qmax + 1) : end, tw = ra_clamp((mine_end - wk * R::SUB * 32 + R::BN - 1) / R::BN, t0, max(t0, t1));
    int t = t0;
    for (; t < tw; ++t, stage = stage == R::STAGES - 1 ? 0 : stage + 1) {
        next_tile(t);
        if (t == t0) { before_end = lut[0]; behind_end = lut[2 * a.reach + RA_PAD]; some_huge = __builtin_amdgcn_readfirstlane(*huge); }
#pragma unroll 1
        for (int u = 0; u < R::SUB; ++u) {
            const int at_row = (wk * R::SUB + u) * 32, j0 = t * R::BN + at_row, last = j0 + 31;
            if (j0 >= mine_end) continue;
            const unsigned char* kt = ra_lds + stage * R::STAGE + at_row * R::ROW;
            const bool far = ra_far(a.reach, j0 - qmax, last - qmin), behind = j0 - qmax >= a.reach;
            const bool edge = last >= keys || (a.causal && last > qmin);
            if (!prev) prev = kt + R::TILE;
            constexpr int N = R::NU * R::DT;
            RaStream<R::KS, R::AHEAD> products;
            auto keys_of = [&](int x) __attribute__((always_inline)) { return ra_row<T, R>(kt, at, x); };
#pragma unroll
            for (int k = 0; k < products.AHEAD; ++k) products.begin(k, keys_of);
            mm_f16 s = ra_bias_of<1>(lut + j0 + 4 * g - qpos + a.reach + RA_PAD, far, behind ? behind_end : before_end);
            products.run(keys_of, [&](int x, uint4 f) __attribute__((always_inline)) { s = Mm<T>::mul(f, qr.v[x], s); }, ra_before<R::KS>(mix, values_of));
            if (edge) {
                const int least = (a.causal ? min(keys - 1, qpos) : keys - 1) - j0 - 4 * g;      // the last key that this query sees
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = (e & 3) + 8 * (e >> 2) > least ? -INFINITY : s[e];
            }
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
            mx *= a.scale2;
            // the reference moves only where a row's maximum has passed it by 2^8 (or it had none): until then p is up to 2^8, which float and
            // bfloat16 hold as exactly as 1
            const bool move = ra_any(mx > top + 8.f || (top == -INFINITY && mx > top));
            float to = top;
            if (move) {
                to = fmaxf(fmaxf(mx, __shfl_xor(mx, 32, 64)), top);
                const float shrink = exp2_fast(top - (to == -INFINITY ? 0.f : to));
                sum *= shrink;
#pragma unroll
                for (int c = 0; c < R::DT; ++c)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[c][e] *= shrink;
#pragma unroll
                for (int x = 0; x < R::NU; ++x) w[x] = Mm<T>::scale(w[x], shrink);
            }
            const float base = to == -INFINITY ? 0.f : to;
            float part = 0.f, shift = -base;
            if (some_huge) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = ra_apart(s[e], a.scale2, base);
                shift = 0.f;
            }
            mix.run(values_of, add, [&](int i) __attribute__((always_inline)) {
#pragma unroll
                for (int e = i * 16 / N; e < (i + 1) * 16 / N; ++e) {
                    float p = exp2_fast(fmaf(s[e], a.scale2, shift));
                    ra_here(p);
                    s[e] = p;
                    part += p;
                }
            });
            top = to;
            sum += part;
            // (p enters the product in the element type: for bfloat16 an error of 2^-9 of each term, below the rounding of y)
            ra_pack<T, R>(s, w);
            prev = kt + R::TILE;
        }
        if constexpr (!R::CARRY) {             // (the tile's place is wanted)
            if (prev) {
#pragma unroll
                for (int k = 0; k < mix.AHEAD; ++k) mix.begin(k, values_of);
                mix.run(values_of, add, [](int) {});
            }
            prev = nullptr;
            ra_zero(w);
        }
    }
    if (prev) {
#pragma unroll
        for (int k = 0; k < mix.AHEAD; ++k) mix.begin(k, values_of);
        mix.run(values_of, add, [](int) {});
    }
    for (; t < t1; ++t, stage = stage == R::STAGES - 1 ? 0 : stage + 1) next_tile(t);
    sum += __shfl_xor(sum, 32, 64);
    if (WK > 1) {                           // one reference for the wavefronts that share the rows
        float* red = reinterpret_cast<float*>(ra_lds);
        __syncthreads();
        if (g == 0) { red[(wave * 32 + l) * 2] = top; red[(wave * 32 + l) * 2 + 1] = sum; }
        __syncthreads();
        float to = -INFINITY, all_sum = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) to = fmaxf(to, red[((wq * WK + w) * 32 + l) * 2]);
        const float base = to == -INFINITY ? 0.f : to;
#pragma unroll
        for (int w = 0; w < WK; ++w) all_sum = fmaf(red[((wq * WK + w) * 32 + l) * 2 + 1], exp2_fast(red[((wq * WK + w) * 32 + l) * 2] - base), all_sum);
        const float shrink = exp2_fast(top - base);
#pragma unroll
        for (int c = 0; c < R::DT; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[c][e] *= shrink;
        top = to;
        sum = all_sum;
        ra_gather<R>(o, reinterpret_cast<float*>(ra_lds), wq, wk, lane);
    }
    if (r0 + l >= rows) return;
    const int64_t row = ((int64_t)n * a.H + h) * a.pq + i;
    if (a.splits > 1) {
        const int64_t at = b.split * ((int64_t)a.m * a.H * a.pq) + row;
        if (g == 0 && wk == 0) { a.part_ml[2 * at] = top; a.part_ml[2 * at + 1] = sum; }
#pragma unroll
        for (int c = 0; c < R::DT; ++c) {
            if (c % WK != wk) continue;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int ch = ra_channel(c, e, g);
                const float v[4] = {o[c][e], o[c][e + 1], o[c][e + 2], o[c][e + 3]};
                if (ch < a.d) ra_store4<R::DMA>(a.part + at * a.d + ch, a.d - ch, v);
            }
        }
        return;
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (a.stats && g == 0 && wk == 0) a.stats[row] = {top, sum == 0.f ? -INFINITY : -log2f(sum)};
    T* yr = (T*)a.y + ((int64_t)n * a.pq + i) * a.ldy + (int64_t)h * a.d;
#pragma unroll
    for (int c = 0; c < R::DT; ++c) {
        if (c % WK != wk) continue;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int ch = ra_channel(c, e, g);
            const float v[4] = {o[c][e] * inv, o[c][e + 1] * inv, o[c][e + 2] * inv, o[c][e + 3] * inv};
            if (ch < a.d) ra_store4<R::DMA>(yr + ch, a.d - ch, v);
        }
    }
}

// Joins the parts of a row: a wavefront per row; lane s knows part s's weight, then a lane has a channel
constexpr int RA_MAX_SPLITS = 32;
template <typename T>
__global__ void __launch_bounds__(RA_THREADS) relattn_join(AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.m * a.H * a.pq, row = (int64_t)blockIdx.x * RA_WAVES + (threadIdx.x >> 6);
    if (row >= rows) return;
    float top = -INFINITY, sum = 0.f;
    if (lane < a.splits) { top = a.part_ml[2 * (lane * rows + row)]; sum = a.part_ml[2 * (lane * rows + row) + 1]; }
    float to = top;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) to = fmaxf(to, __shfl_xor(to, o, 64));
    const float weight = exp2_fast(top - (to == -INFINITY ? 0.f : to));
    sum *= weight;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (a.stats && lane == 0) a.stats[row] = {to, sum == 0.f ? -INFINITY : -log2f(sum)};
    const int64_t nh = row / a.pq;
    const int i = (int)(row - nh * a.pq), h = (int)(nh % a.H), n = (int)(nh / a.H);
    T* yr = (T*)a.y + ((int64_t)n * a.pq + i) * a.ldy + (int64_t)h * a.d;
    float v[2] = {0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
        const float w = __shfl(weight, s, 64);
        const float* p = a.part + (s * rows + row) * a.d;
#pragma unroll
        for (int k = 0; k < 2; ++k) if (lane + 64 * k < a.d) v[k] = fmaf(p[lane + 64 * k], w, v[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) if (lane + 64 * k < a.d) st(yr, lane + 64 * k, v[k] * inv);
}

// Sums of ds along the diagonals of a wavefront's 32 x 32 tiles (its queries stay, its keys ascend): `held` is this lane's sum for distance rel0 + lane.
// What tiles that follow each other share is carried; every distance is stored once.
struct RaDiagonals {
    float lo = 0.f, hi = 0.f, held = 0.f;      // distances of -reach and below, reach and above; the carried one
    int rel0 = 0, from = 0, to = 0;            // distances from .. to - 1 are stored
    bool carrying = false, stored = false;
    float* line;
    int reach;

    __device__ __forceinline__ void emit(int lane, int count) {      // of lanes 0 .. count - 1
        const int rel = rel0 + lane;
        if (lane < count) {
            if (rel <= -reach) lo += held;
            else if (rel >= reach) hi += held;
            else line[rel + reach] = held;
        }
        const int a = max(rel0, 1 - reach), b = min(rel0 + count, reach);
        if (a < b) { from = stored ? from : a; to = b; stored = true; }
    }
    __device__ __forceinline__ void flush(int lane) {
        if (!carrying) return;
        emit(lane, 63);
        held = 0.f;
        carrying = false;
    }
    // a tile whose key 0 is relmin + 31 positions behind its query 0, not wholly beyond the reach
    __device__ __forceinline__ void add(const mm_f16& ds, int relmin, float* area, int lane) {
        const int l = lane & 31, g = lane >> 5;
        if (!carrying || rel0 != relmin) {
            flush(lane);
            if (stored) {                      // (distances that no tile of this wavefront meets)
                for (int rel = to + lane; rel < min(relmin, reach); rel += 64) line[rel + reach] = 0.f;
                to = max(to, min(relmin, reach));
            }
            rel0 = relmin;
            carrying = true;
        }
        // line D of the area: the pairs of distance relmin + D, by query; lines hold zeros where there is no such pair
#pragma unroll
        for (int r = 0; r < 16; ++r) area[((r & 3) + 8 * (r >> 2) + 4 * g + 31 - l) * RA_DIAG_PITCH + l] = ds[r];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float4 v = *reinterpret_cast<const float4*>(area + min(lane, 62) * RA_DIAG_PITCH + 4 * c);
            s += (v.x + v.y) + (v.z + v.w);
        }
        held += lane < 63 ? s : 0.f;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        emit(lane, 32);
        const float up = __shfl(held, lane + 32, 64);
        held = lane < 31 ? up : 0.f;
        rel0 += 32;
    }
    __device__ __forceinline__ void finish(int lane) {
        flush(lane);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { lo += __shfl_xor(lo, o, 64); hi += __shfl_xor(hi, o, 64); }
        for (int rel = 1 - reach + lane; rel < reach; rel += 64)
            if (!stored || rel < from || rel >= to) line[rel + reach] = 0.f;
        if (lane == 0) {
            line[0] = reach ? lo : lo + hi;
            if (reach) line[2 * reach] = hi;
        }
    }
};

// dq of a block's queries, their delta, and the wavefronts' sums of ds by distance.
// delta: dy . y has the rounding of a bfloat16 y in it.  dq and dk do not mind, but in the sums over buckets most of ds cancels, and that error does not.  So
// the sum of a row's ds, which is 0 but for delta's error, corrects it: the sums of tiles beyond the reach afterwards, with those of p beside them,
// while the tiles within the reach are gone through once more.  (Float: y is as exact as the rest, one walk does it all.)
template <typename T, int DP, int WK, bool DMA>
__global__ void __launch_bounds__(RA_THREADS, (RaBwdQ<T, DP, WK, DMA>::BLOCKS)) relattn_bwd_q(AttnArgs a) {
    typedef RaBwdQ<T, DP, WK, DMA> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char ra_lds[];
    float* areas = reinterpret_cast<float*>(ra_lds + R::AREAS);
    int* huge = reinterpret_cast<int*>(ra_lds + R::LDS_Q);
    float* lut = reinterpret_cast<float*>(huge + 4);
    if (threadIdx.x == 0) *huge = 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = lane & 31, g = lane >> 5, wq = wave / WK, wk = wave % WK;
    RaBias bias;
    bias.begin(a);
    float* area = areas + wave * 63 * RA_DIAG_PITCH;
    const int tiles = (a.pq + R::BM - 1) / R::BM;
    const RaBlock b = ra_block<true>(a.m, a.H, tiles, 1, a.causal);
    const int n = b.n, h = b.h, hk = h / (a.H / a.G);
    const int i0 = b.tile * R::BM + wq * 32, i = min(i0 + l, a.pq - 1);
    const bool work = i0 < a.pq, mine = i0 + l < a.pq;
    const int start = ra_start(a, n), keys = ra_keys(a, n), qmin = i0 + start, qmax = min(i0 + 31, a.pq - 1) + start, qpos = i + start;
    const T* kb = (const T*)a.k + (int64_t)n * a.pk * a.ldk + (int64_t)hk * a.d;
    const T* vb = (const T*)a.v + (int64_t)n * a.pk * a.ldv + (int64_t)hk * a.d;
    const int block_qmin = b.tile * R::BM + start, block_qmax = min(b.tile * R::BM + R::BM, a.pq) - 1 + start;
    int end = keys;
    if (a.causal) end = ra_clamp(block_qmax + 1, 0, keys);
    const int all = (end + R::BN - 1) / R::BN;
    RaTile<T, R> kr, vr;
    kr.place(ra_lds, a.ldk, a.d);
    vr.place(ra_lds + R::TILE, a.ldv, a.d);
    auto load = [&](int t, int stage) __attribute__((always_inline)) {
        kr.load(kb, a.ldk, t * R::BN, end, a.d, stage);
        vr.load(vb, a.ldv, t * R::BN, end, a.d, stage);
    };
    if (all > 0) load(0, 0);
    const int64_t row = ((int64_t)n * a.H + h) * a.pq + i, first = ((int64_t)n * a.pq + i0) * a.ldy + (int64_t)h * a.d;
    RaRows<T, R> qr, gr;
    qr.load((const T*)a.q + ((int64_t)n * a.pq + i0) * a.ldq + (int64_t)h * a.d, a.ldq, l, min(32, a.pq - i0), a.d, g);
    gr.load((const T*)a.dy + first, a.ldy, l, min(32, a.pq - i0), a.d, g);
    float delta = 0.f;
    {
        RaRows<T, R> yr;
        yr.load((const T*)a.y + first, a.ldy, l, min(32, a.pq - i0), a.d, g);
#pragma unroll
        for (int s = 0; s < R::KS; ++s) {
            T e[R::EPC], f[R::EPC];
            __builtin_memcpy(e, &gr.v[s], 16);
            __builtin_memcpy(f, &yr.v[s], 16);
#pragma unroll
            for (int k = 0; k < R::EPC; ++k) delta = fmaf(ld(e, k), ld(f, k), delta);
        }
    }
    delta += __shfl_xor(delta, 32, 64);
    const float2_ stat = mine ? a.stats[row] : float2_{0.f, -INFINITY};
    const bool some = stat.y != -INFINITY;                 // the query sees a key
    const float top = some ? stat.x : 0.f;
    float shift = stat.y - top;
    const int least = !some ? -1 : a.causal ? min(keys - 1, qpos) : keys - 1;
    const RaOffsets<T, R> at(lane);
    __syncthreads();
    bias.store(a, h, 1, lut, huge);
    auto clear = [&]() __attribute__((always_inline)) {
        for (int t = lane * 4; t < 63 * RA_DIAG_PITCH; t += 256) *reinterpret_cast<float4*>(area + t) = make_float4(0.f, 0.f, 0.f, 0.f);
    };
    if (R::ES == 4) clear();
    RaDiagonals dg;
    dg.reach = a.reach;
    dg.line = a.diag ? a.diag + (((int64_t)n * a.H + h) * tiles * RA_WAVES + b.tile * RA_WAVES + wave) * ra_distances(a.reach) : nullptr;
    mm_f16 dq[R::DT] = {};
    float rowsum = 0.f, lo = 0.f, hi = 0.f, far_lo = 0.f, far_hi = 0.f;      // sums of ds over the row, of ds and of p beyond the reach on either side
    float before_end = 0.f, behind_end = 0.f;              // (the bias's ends are known behind the first barrier)
    bool some_huge = false;
    // s and dp of the 32 keys from j0 on; beside(i) beside its products
    auto products = [&](const unsigned char* kt, int j0, bool far, mm_f16& s, mm_f16& dp, auto beside) __attribute__((always_inline)) {
        RaStream<2 * R::KS, R::AHEAD> run;
        auto rows_of = [&](int x) __attribute__((always_inline)) { return ra_row<T, R>(x & 1 ? kt + R::TILE : kt, at, x >> 1); };
#pragma unroll
        for (int x = 0; x < run.AHEAD; ++x) run.begin(x, rows_of);
        s = ra_bias_of<1>(lut + j0 + 4 * g - qpos + a.reach + RA_PAD, far, j0 - qmax >= a.reach ? behind_end : before_end);
        dp = mm_f16{};
        run.run(rows_of, [&](int x, uint4 f) __attribute__((always_inline)) {
            if (x & 1) dp = Mm<T>::mul(f, gr.v[x >> 1], dp);
            else s = Mm<T>::mul(f, qr.v[x >> 1], s);
        }, beside);
    };
    // what stands in the way of p = exp2(scale2 s + shift): pairs that are not visible, and huge biases
    auto prepare = [&](int j0, mm_f16& s) __attribute__((always_inline)) {
        if (j0 + 31 >= keys || i0 + 32 > a.pq || (a.causal && j0 + 31 > qmin)) {
            const int seen = least - j0 - 4 * g;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = (e & 3) + 8 * (e >> 2) <= seen ? s[e] : -INFINITY;
        }
        if (some_huge) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = ra_apart(s[e], a.scale2, top);
        }
    };
    // of one pair, p in the place of its score and p (dp - delta) in that of dp
    auto pair = [&](int e, mm_f16& s, mm_f16& dp) __attribute__((always_inline)) {
        float p = exp2_fast(fmaf(s[e], a.scale2, shift)), ds = p * (dp[e] - delta);
        ra_here(p);
        ra_here(ds);
        s[e] = p;
        dp[e] = ds;
    };
    // A piece's ds enters its product while the next piece's is made: `prev` are the keys it belongs to, w its operands.  (Before the first piece w is zero,
    // and prev the first piece's own keys.)
    const unsigned char* prev = nullptr;
    uint4 w[R::NU] = {};
    RaStream<R::NU * R::DT, R::AHEAD> mix;
    auto keys_of = [&](int x) __attribute__((always_inline)) { return ra_column<T, R>(prev, at, x / R::DT, x % R::DT); };
    auto add = [&](int x, uint4 f) __attribute__((always_inline)) { dq[x % R::DT] = Mm<T>::mul(f, w[x / R::DT], dq[x % R::DT]); };
    int stage = 0;
    auto next_tile = [&](int t) __attribute__((always_inline)) {
        kr.done(a.d, stage);
        vr.done(a.d, stage);
        ra_landed<R>();
        __syncthreads();
        if (t + 1 < all) load(t + 1, stage == R::STAGES - 1 ? 0 : stage + 1);
    };
    // the tiles that hold keys for this wavefront: the others of the block may have more
    const int mine_end = !work ? 0 : a.causal ? min(end, qmax + 1) : end, tw = ra_clamp((mine_end - wk * R::SUB * 32 + R::BN - 1) / R::BN, 0, all);
    int t = 0;
    for (; t < tw; ++t, stage = stage == R::STAGES - 1 ? 0 : stage + 1) {
        next_tile(t);
        if (t == 0) {
            before_end = lut[0];
            behind_end = lut[2 * a.reach + RA_PAD];
            some_huge = __builtin_amdgcn_readfirstlane(*huge);
            if (some_huge) shift = stat.y;
        }
#pragma unroll 1
        for (int u = 0; u < R::SUB; ++u) {
            const int at_row = (wk * R::SUB + u) * 32, j0 = t * R::BN + at_row;
            if (j0 >= mine_end) continue;
            const unsigned char* kt = ra_lds + stage * R::STAGE + at_row * R::ROW;
            const bool far = ra_far(a.reach, j0 - qmax, j0 + 31 - qmin);
            if (!prev) prev = kt;
            constexpr int N = R::NU * R::DT;
            mm_f16 s, dp;                      // scores and dy . v, then p and ds
            products(kt, j0, far, s, dp, ra_before<2 * R::KS>(mix, keys_of));
            prepare(j0, s);
            float total = 0.f, ps = 0.f;
            mix.run(keys_of, add, [&](int i) __attribute__((always_inline)) {
#pragma unroll
                for (int e = i * 16 / N; e < (i + 1) * 16 / N; ++e) {
                    pair(e, s, dp);
                    total += dp[e];
                    ps += s[e];
                }
            });
            rowsum += total;
            const float before = far && j0 - qmax < a.reach ? 1.f : 0.f, behind = far && j0 - qmax >= a.reach ? 1.f : 0.f;
            lo = fmaf(before, total, lo);
            hi = fmaf(behind, total, hi);
            far_lo = fmaf(before, ps, far_lo);
            far_hi = fmaf(behind, ps, far_hi);
            if (R::ES == 4 && dg.line && !far) dg.add(dp, j0 - qmin - 31, area, lane);
            ra_pack<T, R>(dp, w);
            prev = kt;
        }
        if constexpr (!R::CARRY) {             // (the tile's place is wanted)
            if (prev) {
#pragma unroll
                for (int k = 0; k < mix.AHEAD; ++k) mix.begin(k, keys_of);
                mix.run(keys_of, add, [](int) {});
            }
            prev = nullptr;
            ra_zero(w);
        }
    }
    if (prev) {
#pragma unroll
        for (int k = 0; k < mix.AHEAD; ++k) mix.begin(k, keys_of);
        mix.run(keys_of, add, [](int) {});
    }
    for (; t < all; ++t, stage = stage == R::STAGES - 1 ? 0 : stage + 1) next_tile(t);
    if (R::ES == 2 && dg.line) {
        rowsum += __shfl_xor(rowsum, 32, 64);
        __syncthreads();                    // (the tiles have been read)
        if (WK > 1) {                       // ... over the wavefronts that share the row
            float* red = reinterpret_cast<float*>(ra_lds);
            if (g == 0) red[wave * 32 + l] = rowsum;
            __syncthreads();
            rowsum = 0.f;
#pragma unroll
            for (int x = 0; x < WK; ++x) rowsum += red[(wq * WK + x) * 32 + l];
            __syncthreads();
        }
        delta += some ? rowsum : 0.f;
        lo = fmaf(-rowsum, far_lo, lo);
        hi = fmaf(-rowsum, far_hi, hi);
        clear();
        // the tiles with distances within the reach of some query of the block
        const int t0 = ra_clamp(block_qmin - a.reach, 0, end) / R::BN, t1 = min(all, ra_clamp(block_qmax + a.reach, 0, end) / R::BN + 1);
        if (t0 < t1) load(t0, 0);
        for (int t = t0; t < t1; ++t) {
            const int s2 = (t - t0) & 1;
            kr.done(a.d, s2);
            vr.done(a.d, s2);
            ra_landed<R>();
            __syncthreads();
            if (t + 1 < t1) load(t + 1, s2 ^ 1);
#pragma unroll 1
            for (int u = 0; u < R::SUB; ++u) {
                const int at_row = (wk * R::SUB + u) * 32, j0 = t * R::BN + at_row;
                if (!work || j0 >= end || (a.causal && j0 > qmax) || ra_far(a.reach, j0 - qmax, j0 + 31 - qmin)) continue;
                mm_f16 s, dp;
                products(ra_lds + s2 * R::STAGE + at_row * R::ROW, j0, false, s, dp, [](int) {});
                prepare(j0, s);
#pragma unroll
                for (int e = 0; e < 16; ++e) pair(e, s, dp);
                dg.add(dp, j0 - qmin - 31, area, lane);
            }
        }
    }
    dg.lo += lo;
    dg.hi += hi;
    if (mine && g == 0 && wk == 0) a.delta[row] = delta;
    if (dg.line) dg.finish(lane);
    ra_gather<R>(dq, reinterpret_cast<float*>(ra_lds), wq, wk, lane);
    if (!mine) return;
    T* out = (T*)a.dq + ((int64_t)n * a.pq + i) * a.ldq + (int64_t)h * a.d;
#pragma unroll
    for (int c = 0; c < R::DT; ++c) {
        if (c % WK != wk) continue;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int ch = ra_channel(c, e, g);
            const float v[4] = {dq[c][e] * a.scale, dq[c][e + 1] * a.scale, dq[c][e + 2] * a.scale, dq[c][e + 3] * a.scale};
            if (ch < a.d) ra_store4<R::DMA>(out + ch, a.d - ch, v);
        }
    }
}

// dk and dv of a block's keys: the queries of every head that shares them, one head after the other
template <typename T, int DP, int WK, bool DMA>
__global__ void __launch_bounds__(RA_THREADS, (RaBwdKv<T, DP, WK, DMA>::BLOCKS)) relattn_bwd_kv(AttnArgs a) {
    typedef RaBwdKv<T, DP, WK, DMA> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char ra_lds[];
    float* rowvs = reinterpret_cast<float*>(ra_lds + R::LDS);         // two of [4][BN]: -log2 sum less top, delta, top, -log2 sum
    int* huge = reinterpret_cast<int*>(rowvs + 8 * R::BN);
    float* lut = reinterpret_cast<float*>(huge + 4);
    if (threadIdx.x == 0) *huge = 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l = lane & 31, g = lane >> 5, wq = wave / WK, wk = wave % WK;
    RaBias bias;
    bias.begin(a);
    const int tiles = (a.pk + R::BM - 1) / R::BM;
    const RaBlock b = ra_block<false>(a.m, a.G, tiles, 1, a.causal);
    const int n = b.n, hk = b.h, share = a.H / a.G;
    const int j0 = b.tile * R::BM + wq * 32, j = min(j0 + l, a.pk - 1);
    const int start = ra_start(a, n), keys = ra_keys(a, n);
    const bool work = j0 < keys, mine = j0 + l < keys;
    RaRows<T, R> kr, vr;
    kr.load((const T*)a.k + ((int64_t)n * a.pk + j0) * a.ldk + (int64_t)hk * a.d, a.ldk, l, min(32, keys - j0), a.d, g);
    vr.load((const T*)a.v + ((int64_t)n * a.pk + j0) * a.ldv + (int64_t)hk * a.d, a.ldv, l, min(32, keys - j0), a.d, g);
    const RaOffsets<T, R> at(lane);
    mm_f16 dk[R::DT] = {}, dv[R::DT] = {};
    const int first = a.causal ? ra_clamp(b.tile * R::BM - start, 0, a.pq) : 0;       // no query before it sees one of the block's keys
    const int t0 = first / R::BN, t1 = b.tile * R::BM < keys ? (a.pq + R::BN - 1) / R::BN : 0;
    RaTile<T, R> qs, gs;
    qs.place(ra_lds, a.ldq, a.d);
    gs.place(ra_lds + R::TILE, a.ldy, a.d);
    float before_end = 0.f, behind_end = 0.f;              // (the bias's ends are known behind a head's first barrier)
    bool some_huge = false;
    // A piece's p and ds enter their products while the next piece's are made: `prev` are the queries they belong to, w the operands.  (Before the first piece w is
    // zero, and prev the first piece's own queries.)
    const unsigned char* prev;
    uint4 w[2 * R::NU];
    RaStream<2 * R::NU * R::DT, R::AHEAD> mix;
    auto columns_of = [&](int x) __attribute__((always_inline)) {
        return ra_column<T, R>(x < R::NU * R::DT ? prev + R::TILE : prev, at, x / R::DT % R::NU, x % R::DT);
    };
    auto add = [&](int x, uint4 f) __attribute__((always_inline)) {
        if (x < R::NU * R::DT) dv[x % R::DT] = Mm<T>::mul(f, w[x / R::DT], dv[x % R::DT]);
        else dk[x % R::DT] = Mm<T>::mul(f, w[x / R::DT], dk[x % R::DT]);
    };
    for (int hh = 0; hh < share; ++hh) {
        const int h = hk * share + hh;
        const T* qb = (const T*)a.q + (int64_t)n * a.pq * a.ldq + (int64_t)h * a.d;
        const T* gb = (const T*)a.dy + (int64_t)n * a.pq * a.ldy + (int64_t)h * a.d;
        const int64_t row0 = ((int64_t)n * a.H + h) * a.pq;
        float2_ st = {0.f, -INFINITY};
        float dl = 0.f;
        auto load = [&](int t, int stage) __attribute__((always_inline)) {
            qs.load(qb, a.ldq, t * R::BN, a.pq, a.d, stage);
            gs.load(gb, a.ldy, t * R::BN, a.pq, a.d, stage);
            const int i = min(t * R::BN + min((int)threadIdx.x, R::BN - 1), a.pq - 1);      // (rows beyond the last are masked)
            st = a.stats[row0 + i];
            dl = a.delta[row0 + i];
        };
        __syncthreads();                                   // (the tiles and the bias of the head before have been read)
        if (t0 < t1) load(t0, 0);
        bias.store(a, h, 1, lut, huge);
        prev = nullptr;
        ra_zero(w);
        int stage = 0;
        for (int t = t0; t < t1; ++t, stage = stage == R::STAGES - 1 ? 0 : stage + 1) {
            float* rowv = rowvs + (t & 1) * 4 * R::BN;
            qs.done(a.d, stage);
            gs.done(a.d, stage);
            if ((int)threadIdx.x < R::BN) {
                const float tp = st.y == -INFINITY ? 0.f : st.x;
                rowv[threadIdx.x] = st.y - tp;
                rowv[R::BN + threadIdx.x] = dl;
                rowv[2 * R::BN + threadIdx.x] = tp;
                rowv[3 * R::BN + threadIdx.x] = st.y;
            }
            ra_landed<R>();
            __syncthreads();
            if (t + 1 < t1) load(t + 1, stage == R::STAGES - 1 ? 0 : stage + 1);
            if (t == t0) { before_end = lut[0]; behind_end = lut[2 * a.reach + RA_PAD]; some_huge = __builtin_amdgcn_readfirstlane(*huge); }
#pragma unroll 1
            for (int u = 0; u < R::SUB; ++u) {
                const int at_row = (wk * R::SUB + u) * 32, i0 = t * R::BN + at_row, qmin = i0 + start, qmax = min(i0 + 31, a.pq - 1) + start;
                if (!work || i0 >= a.pq || (a.causal && j0 > qmax)) continue;      // (before the first piece, or behind the last)
                const unsigned char *qt = ra_lds + stage * R::STAGE + at_row * R::ROW, *gt = qt + R::TILE;
                const float* rv = rowv + at_row + 4 * g;
                const int relmin = j0 - i0 - start - 31;
                const bool far = ra_far(a.reach, relmin, j0 + 31 - qmin), behind = relmin >= a.reach;
                const bool edge = j0 + 32 > keys || i0 + 32 > a.pq || (a.causal && j0 + 31 > qmin);
                if (!prev) prev = qt;
                constexpr int N = 2 * R::NU * R::DT;
                RaStream<2 * R::KS, R::AHEAD> products;
                auto rows_of = [&](int x) __attribute__((always_inline)) { return ra_row<T, R>(x & 1 ? gt : qt, at, x >> 1); };
#pragma unroll
                for (int x = 0; x < products.AHEAD; ++x) products.begin(x, rows_of);
                mm_f16 s = ra_bias_of<-1>(lut + j0 + l - i0 - start - 4 * g + a.reach + RA_PAD, far, behind ? behind_end : before_end), dp = {};
                products.run(rows_of, [&](int x, uint4 f) __attribute__((always_inline)) {
                    if (x & 1) dp = Mm<T>::mul(f, vr.v[x >> 1], dp);
                    else s = Mm<T>::mul(f, kr.v[x >> 1], s);
                }, ra_before<2 * R::KS>(mix, columns_of));
                if (edge) {
                    // queries of the piece that see this key
                    const int from = (a.causal ? max(j0 + l - start, 0) : 0) - i0 - 4 * g, to = mine ? a.pq - i0 - 4 * g : 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int i = (e & 3) + 8 * (e >> 2);
                        s[e] = i < to && i >= from ? s[e] : -INFINITY;
                    }
                }
                const float* shift_at = rv;
                if (some_huge) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = ra_apart(s[e], a.scale2, rv[2 * R::BN + (e & 3) + 8 * (e >> 2)]);
                    shift_at = rv + 3 * R::BN;
                }
                float4 shifts[2], deltas[2];       // of four rows, and of the next four
                auto rows4 = [&](int c) __attribute__((always_inline)) {
                    shifts[c & 1] = *reinterpret_cast<const float4*>(shift_at + 8 * c);
                    deltas[c & 1] = *reinterpret_cast<const float4*>(rv + R::BN + 8 * c);
                };
                rows4(0);
                mix.run(columns_of, add, [&](int x) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = x * 16 / N; e < (x + 1) * 16 / N; ++e) {
                        const int c = e >> 2;
                        if (e % 4 == 0 && c < 3) rows4(c + 1);
                        const float4 sh = shifts[c & 1], de = deltas[c & 1];
                        const float delta = e % 4 == 0 ? de.x : e % 4 == 1 ? de.y : e % 4 == 2 ? de.z : de.w;
                        float p = exp2_fast(fmaf(s[e], a.scale2, e % 4 == 0 ? sh.x : e % 4 == 1 ? sh.y : e % 4 == 2 ? sh.z : sh.w)), ds = p * (dp[e] - delta);
                        ra_here(p);
                        ra_here(ds);
                        s[e] = p;
                        dp[e] = ds;
                    }
                });
                ra_pack<T, R>(s, w);
                ra_pack<T, R>(dp, w + R::NU);
                prev = qt;
            }
            if constexpr (!R::CARRY) {             // (the tile's place is wanted)
                if (prev) {
#pragma unroll
                    for (int k = 0; k < mix.AHEAD; ++k) mix.begin(k, columns_of);
                    mix.run(columns_of, add, [](int) {});
                }
                prev = nullptr;
                ra_zero(w);
            }
        }
        if (prev) {
#pragma unroll
            for (int k = 0; k < mix.AHEAD; ++k) mix.begin(k, columns_of);
            mix.run(columns_of, add, [](int) {});
        }
    }
    ra_gather<R>(dk, reinterpret_cast<float*>(ra_lds), wq, wk, lane);
    ra_gather<R>(dv, reinterpret_cast<float*>(ra_lds), wq, wk, lane);
    if (j0 + l >= a.pk) return;                            // (keys behind the last one of the sample have gradients of zero)
    T* ok = (T*)a.dk + ((int64_t)n * a.pk + j) * a.ldk + (int64_t)hk * a.d;
    T* ov = (T*)a.dv + ((int64_t)n * a.pk + j) * a.ldv + (int64_t)hk * a.d;
#pragma unroll
    for (int c = 0; c < R::DT; ++c) {
        if (c % WK != wk) continue;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const int ch = ra_channel(c, e, g);
            const float vk[4] = {dk[c][e] * a.scale, dk[c][e + 1] * a.scale, dk[c][e + 2] * a.scale, dk[c][e + 3] * a.scale};
            const float vv[4] = {dv[c][e], dv[c][e + 1], dv[c][e + 2], dv[c][e + 3]};
            if (ch < a.d) { ra_store4<R::DMA>(ok + ch, a.d - ch, vk); ra_store4<R::DMA>(ov + ch, a.d - ch, vv); }
        }
    }
}

// The wavefronts' sums by distance, `lines` of them a head and sample: block (64 distances, head, share of the samples' lines) -> shares[share][head][distance]
constexpr int RA_SHARES = 16;
__global__ void __launch_bounds__(RA_THREADS) relattn_diagonals(const float* __restrict__ diag, int m, int H, int lines, int nd, float* __restrict__ shares) {
    __shared__ float red[RA_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, h = blockIdx.y;
    const int64_t all = (int64_t)m * lines, per = (all + RA_SHARES - 1) / RA_SHARES, from = blockIdx.z * per, to = from + per < all ? from + per : all;
    float s = 0.f;
    if (c < nd)
        for (int64_t x = from + wave; x < to; x += RA_WAVES) {
            const int64_t n = x / lines;
            s += diag[((n * H + h) * lines + (x - n * lines)) * nd + c];
        }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < nd) shares[((int64_t)blockIdx.z * H + h) * nd + c] = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}
// dtable[h][bucket] (+)= the distances of the bucket
__global__ void __launch_bounds__(RA_THREADS) relattn_buckets(const float* __restrict__ shares, const int32_t* __restrict__ map, int H, int nb, int nd,
                                                              float* __restrict__ dtable, int accumulate) {
    extern __shared__ __attribute__((aligned(16))) float ra_sums[];
    int* ids = reinterpret_cast<int*>(ra_sums + nd);
    const int h = blockIdx.x;
    for (int c = threadIdx.x; c < nd; c += RA_THREADS) {
        float v[RA_SHARES], s = 0.f;
        ids[c] = ra_clamp(map[c], 0, nb - 1);
#pragma unroll
        for (int k = 0; k < RA_SHARES; ++k) v[k] = shares[((int64_t)k * H + h) * nd + c];
#pragma unroll
        for (int k = 0; k < RA_SHARES; ++k) s += v[k];
        ra_sums[c] = s;
    }
    __syncthreads();
    // eight lanes a bucket
    const int part = threadIdx.x & 7;
    for (int b0 = 0; b0 < nb; b0 += RA_THREADS / 8) {
        const int b = b0 + (int)(threadIdx.x >> 3);
        float s = 0.f;
        for (int c = part; c < nd; c += 8) s += ids[c] == b ? ra_sums[c] : 0.f;
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) s += __shfl_xor(s, o, 64);
        if (part == 0 && b < nb) dtable[(int64_t)h * nb + b] = accumulate ? dtable[(int64_t)h * nb + b] + s : s;
    }
}

static size_t ra_up(size_t b) { return (b + 255) & ~(size_t)255; }
// Wavefronts that share rows (and walk the other side's tiles together), at most as many as the tiles leave room for in LDS ...
template <typename T, int DP> constexpr int ra_most() { return sizeof(T) == 2 ? (DP <= 64 ? 4 : 2) : DP <= 32 ? 4 : DP <= 64 ? 2 : 1; }
static int ra_dp(int d, bool dma) { return d <= 32 && dma ? 32 : d <= 64 ? 64 : d <= 96 && dma ? 96 : 128; }
static int ra_most_of(int32_t dtype, int dp) { return dtype == LPM_BF16 ? (dp <= 64 ? 4 : 2) : dp <= 32 ? 4 : dp <= 64 ? 2 : 1; }
// ... and as many as there are blocks missing: the CUs are 256, and a block of shared rows takes 0.6 (two wavefronts) or 0.46 (four) of the time of one
// with rows for each.  (512 keys, dq: 32 float heads of 32 channels, 128 blocks of 128 rows, by wavefronts 1, 2, 4: 44, 28, 37 us; 16 heads: 43, 27, 20; 48 heads: 46,
// 52, 54.  bf16 heads of 128 channels, 1 and 2: 32 heads 39 and 28 us, 48 heads 41 and 52.)  Two of the small blocks of bf16 heads up to 64 channels run as fast side
// by side (dq, 48 heads of 64 channels, 1, 2, 4: 32, 27, 43 us; 80 heads: 42, 42, 69), three in the forward pass (96 heads, 1 and 2: 22 and 19 us; 128 heads: 24 and 26), and causal
// blocks, whose keys differ, even out when there are more.
static int ra_wk(int32_t dtype, int d, bool dma, bool causal, int64_t pairs, int rows, bool forward = false) {
    const int dp = ra_dp(d, dma), most = ra_most_of(dtype, dp), two = dtype == LPM_BF16 && dp <= 64 ? (forward ? 768 : 512) : causal ? 512 : 256;
    auto blocks = [&](int wk) { return pairs * ((rows + 128 / wk - 1) / (128 / wk)); };
    for (int wk = most; wk > 1; wk /= 2)
        if (blocks(wk) == blocks(1) || blocks(wk) <= (wk == 2 ? two : 256)) return wk;
    return 1;
}
static int ra_bm(const lpm_attn_geom& g, int32_t dtype, bool dma) { return 128 / ra_wk(dtype, g.d, dma, g.causal != 0, (int64_t)g.m * g.heads, g.pq); }
// lines of sums by distance that a head and sample's blocks of queries leave
static int ra_lines(const lpm_attn_geom& g, int32_t dtype, bool dma) {
    const int bm = ra_bm(g, dtype, dma);
    return (g.pq + bm - 1) / bm * RA_WAVES;
}
// The forward pass's blocks: rows folded over the heads that share keys where these fit two operands of 32 rows, and the keys over several blocks -- 1024 in all, of 512
// keys at least -- where the blocks do not fill the card.  (A query a row, a cache of 806 MB, four heads share keys: 361 us head by head, 168 folded, the join of 9 among them;
// over 512 blocks 170, over 2048 182.)
struct RaForward { bool fold; int rows, splits; int64_t pairs; };
static RaForward ra_plan(const lpm_attn_geom& g, int32_t dtype) {
    RaForward f{};
    const int share = g.heads / g.kv_heads;
    f.fold = share > 1 && g.pq <= 32 && share * g.pq <= 64 && share * ra_lut(g.reach) <= 8192;
    f.rows = f.fold ? share * g.pq : g.pq;
    f.pairs = (int64_t)g.m * (f.fold ? g.kv_heads : g.heads);
    const int bm = 128 / ra_wk(dtype, g.d, false, g.causal != 0, f.pairs, f.rows, true);      // (what a call's pointers decide is not known here)
    const int64_t blocks = std::max<int64_t>(1, f.pairs * ((f.rows + bm - 1) / bm));
    f.splits = blocks >= 512 ? 1 : (int)std::min<int64_t>({std::max(1, g.pk / 512), (1024 + blocks - 1) / blocks, RA_MAX_SPLITS});
    return f;
}
struct AttnLayout { size_t part_ml, fwd_all, diag, shares, bwd_all; };
static AttnLayout ra_layout(const lpm_attn_geom& g, int32_t dtype) {
    AttnLayout o;
    const RaForward f = ra_plan(g, dtype);
    const size_t rows = (size_t)g.m * g.heads * g.pq, nd = ra_distances(g.reach);
    const size_t lines = std::max(ra_lines(g, dtype, false), ra_lines(g, dtype, true));      // (what a call's pointers decide is not known here)
    o.part_ml = f.splits > 1 ? ra_up((size_t)f.splits * rows * g.d * 4) : 0;
    o.fwd_all = f.splits > 1 ? o.part_ml + ra_up((size_t)f.splits * rows * 8) : 0;
    o.diag = ra_up(rows * 4);
    o.shares = o.diag + (g.n_buckets ? ra_up((size_t)g.m * g.heads * lines * nd * 4) : 0);
    o.bwd_all = o.shares + (g.n_buckets ? ra_up((size_t)RA_SHARES * g.heads * nd * 4) : 0);
    return o;
}

template <typename K> static hipError_t ra_launch(K kernel, DeviceSet& done, int64_t blocks, size_t lds, const AttnArgs& a, hipStream_t st) {
    if (!blocks) return hipSuccess;
    const hipError_t e = allow_lds(kernel, 160 * 1024, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(RA_THREADS), lds, st, a);
    return hipGetLastError();
}
template <typename T, int DP, int WK, bool DMA> static hipError_t ra_forward(const AttnArgs& a, hipStream_t st) {
    typedef RaFwd<T, DP, WK, DMA> R;
    static DeviceSet done;
    static_assert(WK == 1 || 128 / WK / 32 * WK * R::DT * 4096 <= R::LDS, "the sums of wavefronts that share rows fit over the tiles");
    const int share = a.H / a.G, rows = a.fold ? share * a.pq : a.pq;
    return ra_launch(relattn_fwd<T, DP, WK, DMA>, done, (int64_t)a.m * (a.fold ? a.G : a.H) * ((rows + R::BM - 1) / R::BM) * a.splits,
                     R::LDS + 16 + (size_t)(a.fold ? share : 1) * ra_lut(a.reach) * 4, a, st);
}
template <typename T, int DP, int WK, bool DMA> static hipError_t ra_backward_q(const AttnArgs& a, hipStream_t st) {
    typedef RaBwdQ<T, DP, WK, DMA> R;
    static DeviceSet done;
    static_assert(R::LDS_Q + 16 + (2 * RA_MAX_REACH + 1 + 2 * RA_PAD) * 4 <= 160 * 1024, "the tiles, diagonals and bias fit");
    static_assert(WK == 1 || 128 / WK / 32 * WK * R::DT * 4096 <= R::LDS, "the sums of wavefronts that share rows fit over the tiles");
    return ra_launch(relattn_bwd_q<T, DP, WK, DMA>, done, (int64_t)a.m * a.H * ((a.pq + R::BM - 1) / R::BM),
                     R::LDS_Q + 16 + (size_t)ra_lut(a.reach) * 4, a, st);
}
template <typename T, int DP, int WK, bool DMA> static hipError_t ra_backward_kv(const AttnArgs& a, hipStream_t st) {
    typedef RaBwdKv<T, DP, WK, DMA> R;
    static DeviceSet done;
    static_assert(WK == 1 || 128 / WK / 32 * WK * R::DT * 4096 <= R::LDS, "the sums of wavefronts that share rows fit over the tiles");
    return ra_launch(relattn_bwd_kv<T, DP, WK, DMA>, done, (int64_t)a.m * a.G * ((a.pk + R::BM - 1) / R::BM), R::LDS + (8 * R::BN + 4 + (size_t)ra_lut(a.reach)) * 4, a, st);
}
// Tiles straight to LDS: channels in whole chunks, every row of both operands on a whole dword
static bool ra_dma(int32_t dtype, int d, const void* p, int64_t ldp, const void* q, int64_t ldq) {
    const int es = dtype == LPM_BF16 ? 2 : 4;
    return d % (16 / es) == 0 && ((uintptr_t)p | (uintptr_t)q | (uintptr_t)(ldp * es) | (uintptr_t)(ldq * es)) % 4 == 0;
}
// f<T, padded channels, wavefronts that share rows, DMA>
#define LPM_RA_WIDE(f_, T_, DP_, wk_, dma_)                                                                                                        \
    ((wk_) == 4 ? f_<T_, DP_, ra_most<T_, DP_>(), dma_>(a, st) : (wk_) == 2 ? f_<T_, DP_, (ra_most<T_, DP_>() > 1 ? 2 : 1), dma_>(a, st)            \
     : f_<T_, DP_, 1, dma_>(a, st))
#define LPM_RA_CHANNELS(f_, T_, wk_, dma_)                                                                                                     \
    (!(dma_) ? (a.d <= 64 ? LPM_RA_WIDE(f_, T_, 64, wk_, false) : LPM_RA_WIDE(f_, T_, 128, wk_, false))                                     \
     : a.d <= 32 ? LPM_RA_WIDE(f_, T_, 32, wk_, true) : a.d <= 64 ? LPM_RA_WIDE(f_, T_, 64, wk_, true)                                      \
     : a.d <= 96 ? LPM_RA_WIDE(f_, T_, 96, wk_, true) : LPM_RA_WIDE(f_, T_, 128, wk_, true))
#define LPM_RA(f_, dtype_, wk_, dma_) ((dtype_) == LPM_BF16 ? LPM_RA_CHANNELS(f_, bf16_t, wk_, dma_) : LPM_RA_CHANNELS(f_, float, wk_, dma_))

}  // namespace lpm

static int32_t ra_check(const lpm_attn_geom* g, int32_t dtype, lpm_attn_geom& o) {
    if (!g) return fail(LPM_EINVAL, "geometry is NULL");
    if (dtype != LPM_F32 && dtype != LPM_BF16) return fail(LPM_EINVAL, "dtype must be LPM_F32 or LPM_BF16");
    o = *g;
    if (o.m < 0 || o.pq < 0 || o.pk < 0 || o.pq > (1 << 28) || o.pk > (1 << 28) || o.heads <= 0 || o.heads > 65535 || o.kv_heads <= 0 || o.heads % o.kv_heads)
        return fail(LPM_ESHAPE, "attention of %d samples, %d queries, %d keys, %d heads on %d", o.m, o.pq, o.pk, o.heads, o.kv_heads);
    if (o.d < 8 || o.d > 128) return fail(LPM_ESHAPE, "heads of %d channels (8 to 128)", o.d);
    if (o.n_buckets < 0 || o.n_buckets > 65536 || o.reach < 0 || o.reach > RA_MAX_REACH)
        return fail(LPM_ESHAPE, "%d buckets (0 to 65536) of distances up to %d (0 to %d)", o.n_buckets, o.reach, RA_MAX_REACH);
    if (o.scale != 0.f && !(o.scale >= 1e-30f && o.scale <= 1e30f)) return fail(LPM_EINVAL, "scale must be 0 (for 1 / sqrt(d)) or 1e-30 to 1e30");
    const int64_t wq = (int64_t)o.heads * o.d, wk = (int64_t)o.kv_heads * o.d;
    if (wq > RA_MAX_LD) return fail(LPM_ESHAPE, "%d heads of %d channels", o.heads, o.d);
    if (!o.ldq) o.ldq = (int32_t)wq;
    if (!o.ldk) o.ldk = (int32_t)wk;
    if (!o.ldv) o.ldv = (int32_t)wk;
    if (!o.ldy) o.ldy = (int32_t)wq;
    if (o.ldq < wq || o.ldy < wq || o.ldk < wk || o.ldv < wk) return fail(LPM_ESHAPE, "positions closer than their heads are wide");
    if (std::max({o.ldq, o.ldk, o.ldv, o.ldy}) > RA_MAX_LD) return fail(LPM_ESHAPE, "positions more than %d elements apart", RA_MAX_LD);
    if (o.scale == 0.f) o.scale = 1.f / sqrtf((float)o.d);
    if (!o.n_buckets) o.reach = 0;
    const int64_t most = std::max<int64_t>(o.pq, o.pk) / 32 + 1;
    if ((int64_t)o.m * o.heads >= ((int64_t)1 << 31) / most / RA_MAX_SPLITS) return fail(LPM_ESHAPE, "more blocks than a launch takes");
    return LPM_OK;
}
static AttnArgs ra_args(const lpm_attn_geom& g, const void* q, const void* k, const void* v, const int32_t* len, const int32_t* start, const int32_t* map,
                        const float* table) {
    AttnArgs a{};
    a.m = g.m; a.H = g.heads; a.G = g.kv_heads; a.pq = g.pq; a.pk = g.pk; a.d = g.d; a.causal = g.causal != 0;
    a.nb = g.n_buckets; a.reach = g.reach; a.splits = 1;
    a.ldq = g.ldq; a.ldk = g.ldk; a.ldv = g.ldv; a.ldy = g.ldy;
    a.scale = g.scale; a.scale2 = g.scale * RA_LOG2E; a.inv_scale = 1.f / g.scale;
    a.q = q; a.k = k; a.v = v;
    a.len = len; a.start = start; a.map = map; a.table = table;
    return a;
}
static int32_t ra_operands(const lpm_attn_geom& g, int32_t dtype, const void* q, const void* k, const void* v, const int32_t* len, const int32_t* start,
                           const int32_t* map, const float* table, std::initializer_list<const void*> rows, std::initializer_list<const void*> buffers) {
    if (!g.n_buckets != !table || !table != !map) return fail(LPM_EINVAL, "the table and the map go with n_buckets > 0, none of them without");
    const uintptr_t es = dtype == LPM_BF16 ? 1 : 3;
    for (const void* p : {q, k, v}) if ((uintptr_t)p & es) return fail(LPM_EALIGN, "q, k and v must be aligned to their elements");
    for (const void* p : rows) if ((uintptr_t)p & es) return fail(LPM_EALIGN, "gradients must be aligned to their elements");
    for (const void* p : {(const void*)len, (const void*)start, (const void*)map, (const void*)table})
        if ((uintptr_t)p & 3u) return fail(LPM_EALIGN, "key_len, q_start, map and table must be 4-byte aligned");
    for (const void* p : buffers) if ((uintptr_t)p & 255u) return fail(LPM_EALIGN, "y, dy, dtable, stats and scratch must be 256-byte aligned");
    return LPM_OK;
}

extern "C" int32_t lpm_attn_ws_bytes(const lpm_attn_geom* geom, int32_t dtype, size_t* forward, size_t* backward) {
    lpm_attn_geom g;
    const int32_t rc = ra_check(geom, dtype, g);
    if (rc) return rc;
    const AttnLayout o = ra_layout(g, dtype);
    if (forward) *forward = o.fwd_all;
    if (backward) *backward = o.bwd_all;
    return LPM_OK;
}

extern "C" int32_t lpm_attn_stats_bytes(const lpm_attn_geom* geom, int32_t dtype, size_t* bytes) {
    if (!bytes) return fail(LPM_EINVAL, "bytes is NULL");
    lpm_attn_geom g;
    const int32_t rc = ra_check(geom, dtype, g);
    if (rc) return rc;
    *bytes = (size_t)g.m * g.heads * g.pq * sizeof(float2_);
    return LPM_OK;
}

extern "C" int32_t lpm_attn_forward(const lpm_attn_geom* geom, int32_t dtype, const void* q, const void* k, const void* v, const int32_t* key_len,
                                    const int32_t* q_start, const int32_t* map, const float* table, void* y, void* stats, void* ws, void* stream) {
    lpm_attn_geom g;
    int32_t rc = ra_check(geom, dtype, g);
    if (rc) return rc;
    if ((rc = ra_operands(g, dtype, q, k, v, key_len, q_start, map, table, {}, {y, stats, ws}))) return rc;
    if (g.m == 0 || g.pq == 0) return LPM_OK;
    if (!q || !y || (g.pk > 0 && (!k || !v))) return fail(LPM_EINVAL, "NULL argument");
    AttnArgs a = ra_args(g, q, k, v, key_len, q_start, map, table);
    const RaForward plan = ra_plan(g, dtype);
    a.splits = plan.splits;
    a.fold = plan.fold;
    if (a.splits > 1 && !ws) return fail(LPM_EINVAL, "scratch required");
    a.y = y;
    a.stats = (float2_*)stats;
    a.part = (float*)ws;
    a.part_ml = (float*)((char*)ws + ra_layout(g, dtype).part_ml);
    hipStream_t st = (hipStream_t)stream;
    const bool dma = ra_dma(dtype, g.d, k, g.ldk, v, g.ldv);
    LPM_HIP(LPM_RA(ra_forward, dtype, ra_wk(dtype, g.d, dma, a.causal, plan.pairs, plan.rows, true), dma));
    if (a.splits > 1) {
        const dim3 grid((unsigned)(((int64_t)g.m * g.heads * g.pq + RA_WAVES - 1) / RA_WAVES));
        if (dtype == LPM_BF16) hipLaunchKernelGGL(relattn_join<bf16_t>, grid, dim3(RA_THREADS), 0, st, a);
        else hipLaunchKernelGGL(relattn_join<float>, grid, dim3(RA_THREADS), 0, st, a);
        LPM_HIP(hipGetLastError());
    }
    return LPM_OK;
}

extern "C" int32_t lpm_attn_backward(const lpm_attn_geom* geom, int32_t dtype, const void* q, const void* k, const void* v, const void* y, const void* stats,
                                     const void* dy, const int32_t* key_len, const int32_t* q_start, const int32_t* map, const float* table, void* dq, void* dk,
                                     void* dv, float* dtable, int32_t accumulate, void* ws, void* stream) {
    lpm_attn_geom g;
    int32_t rc = ra_check(geom, dtype, g);
    if (rc) return rc;
    if ((rc = ra_operands(g, dtype, q, k, v, key_len, q_start, map, table, {dq, dk, dv}, {y, stats, dy, dtable, ws}))) return rc;
    if (dtable && !table) return fail(LPM_EINVAL, "a gradient of a table that is not there");
    const bool queries = g.m > 0 && g.pq > 0, keys = g.m > 0 && g.pk > 0;
    if ((queries && (!q || !y || !stats || !dy || !dq)) || (keys && (!k || !v || !dk || !dv))) return fail(LPM_EINVAL, "NULL argument");
    if ((queries || dtable) && !ws) return fail(LPM_EINVAL, "scratch required");
    const AttnLayout o = ra_layout(g, dtype);
    AttnArgs a = ra_args(g, q, k, v, key_len, q_start, map, table);
    a.y = const_cast<void*>(y);
    a.dy = dy;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.stats = (float2_*)const_cast<void*>(stats);
    a.delta = (float*)ws;
    a.diag = dtable ? (float*)((char*)ws + o.diag) : nullptr;
    hipStream_t st = (hipStream_t)stream;
    const bool dma_k = ra_dma(dtype, g.d, k, g.ldk, v, g.ldv), dma_q = ra_dma(dtype, g.d, q, g.ldq, dy, g.ldy);
    if (queries) LPM_HIP(LPM_RA(ra_backward_q, dtype, ra_wk(dtype, g.d, dma_k, a.causal, (int64_t)g.m * g.heads, g.pq), dma_k));
    if (keys) LPM_HIP(LPM_RA(ra_backward_kv, dtype, ra_wk(dtype, g.d, dma_q, a.causal, (int64_t)g.m * g.kv_heads, g.pk), dma_q));
    if (dtable) {
        const int nd = 2 * g.reach + 1;
        float* shares = (float*)((char*)ws + o.shares);
        hipLaunchKernelGGL(relattn_diagonals, dim3((unsigned)((nd + 63) / 64), (unsigned)g.heads, RA_SHARES), dim3(RA_THREADS), 0, st, (const float*)a.diag, g.m,
                           g.heads, ra_lines(g, dtype, dma_k), nd, shares);
        hipLaunchKernelGGL(relattn_buckets, dim3((unsigned)g.heads), dim3(RA_THREADS), (size_t)nd * 8, st, (const float*)shares, map, g.heads, g.n_buckets, nd, dtable,
                           accumulate);
        LPM_HIP(hipGetLastError());
    }
    return LPM_OK;
}

extern "C" int32_t lpm_relbias_buckets(int32_t n_buckets, int32_t reach, int32_t both_sides, int32_t* map) {
    if (!map) return fail(LPM_EINVAL, "map is NULL");
    if (n_buckets < (both_sides ? 2 : 1) || (both_sides && n_buckets % 2) || reach < 0 || reach > RA_MAX_REACH)
        return fail(LPM_EINVAL, "%d buckets for distances up to %d", n_buckets, reach);
    const int n = both_sides ? n_buckets / 2 : n_buckets, exact = std::max(1, n / 2);
    for (int rel = -reach; rel <= reach; ++rel) {
        int r = both_sides ? std::abs(rel) : std::max(0, -rel);
        if (r >= exact) r = std::min(n - 1, exact + (int)(std::log((double)r / exact) / std::log((double)std::max(reach, exact + 1) / exact) * (n - exact)));
        map[rel + reach] = (both_sides && rel > 0 ? n : 0) + r;
    }
    return LPM_OK;
}
