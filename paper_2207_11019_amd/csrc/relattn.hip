// Multi-head attention with a learned bias by the bucket of the distance between key and query, forward and backward:
//   s_ij = scale q_i . k_j + table[h][bucket(j - i - start)],  p = softmax over the visible j,  y_i = sum_j p_ij v_j
//   delta_i = dy_i . y_i,  ds_ij = p_ij (dy_i . v_j - delta_i),  dv_j = sum_i p_ij dy_i,  dq_i = scale sum_j ds_ij k_j,
//   dk_j = scale sum_i ds_ij q_i,  dtable[h][b] = sum of ds over the pairs of bucket b
// Scores are never stored: the forward pass walks the keys once with the running maximum and sum of each row's softmax, the backward pass
// makes p again from the two.  A block has 128 queries (keys, in the kernel that makes dk and dv), a wavefront 32 of them, and tiles of the other
// side's rows go through LDS.  The products are formed transposed -- keys x queries = K Q' -- so that a lane holds scores of one query:
// the row statistics need one lane exchange, and the probabilities already lie as the next product's operand (matrix.h), whose other
// operand is read from the same LDS tile by columns.
// Bias: the buckets' values by distance, -reach .. reach and a margin of repeated ends, lie in LDS in units of log2; tiles wholly beyond the
// reach add one number.  Its gradient: sums of ds along the diagonals of 32 x 32 tiles, which a wavefront carries from tile to tile, so that each
// distance is stored once per wavefront; two small kernels add up wavefronts, then the distances of a bucket.  No atomics: every sum has one order.
#include "matrix.h"
#include "lpm_internal.h"
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <initializer_list>

using namespace lpm;

namespace lpm {

constexpr int RA_THREADS = 256, RA_WAVES = 4, RA_BM = 128;
constexpr int RA_PAD = 96;                // margin of the bias by distance: a tile that is not wholly beyond the reach stays within it (63 + 31)
constexpr int RA_MAX_REACH = 2048;
constexpr float RA_LOG2E = 1.4426950408889634f;
constexpr int RA_DIAG_PITCH = 36;         // floats of a line of a wavefront's diagonals

struct float2_ { float x, y; };

struct AttnArgs {
    int32_t m, H, G, pq, pk, d, causal, nb, reach, splits;
    int64_t ldq, ldk, ldv, ldy;           // elements between positions
    float scale, scale2;                  // scale2 = scale log2(e)
    const void *q, *k, *v, *dy;
    void *y, *dq, *dk, *dv;
    const int32_t *len, *start, *map;
    const float* table;
    float2_* stats;                       // per row (n, h, i): maximum of the scores in units of log2, -log2 of the sum (-inf: no visible key)
    bf16_t* low;                          // what the rounding of y took away, [m][pq][H d] (bfloat16)
    float *part, *part_ml;                // splits: [split][row][d] and [split][row][2]
    float *delta, *diag;                  // backward: [row], [m H ceil(pq / 32)][2 reach + 1]
};

template <typename T, int DP> struct Ra {
    static constexpr int EPC = Mm<T>::EPC, CHUNKS = DP / EPC, KS = DP / (2 * EPC), ES = (int)sizeof(T);
    static constexpr int BN = ES == 2 ? 64 : 32;              // rows of a staged tile
    static constexpr int PITCH = DP * ES + 32;                // rows 8 dwords apart in the banks: row-wise and column-wise reads are free of conflicts
    static constexpr int TILE = BN * PITCH;
    static constexpr int PER = BN * CHUNKS / RA_THREADS;      // chunks of a tile a thread brings
    static constexpr int DT = DP / 32;                        // 32-channel pieces of a head
};

// A tile on its way from memory to LDS, in registers meanwhile; rows from `rows` on and channels from d on are zeros and not read
template <typename T, int DP> struct RaTile {
    typedef Ra<T, DP> R;
    uint4 v[R::PER];
    __device__ __forceinline__ void load(const T* base, int64_t ld, int row0, int rows, int d) {
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            const int at = i * RA_THREADS + (int)threadIdx.x, r = at / R::CHUNKS, c = (at - r * R::CHUNKS) * R::EPC;
            const bool there = row0 + r < rows && c < d;
            v[i] = ld16(there ? base + (int64_t)(row0 + r) * ld + c : base, there ? d - c : 0);
        }
    }
    __device__ __forceinline__ void store(unsigned char* lds) const {
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            const int at = i * RA_THREADS + (int)threadIdx.x, r = at / R::CHUNKS, c = at - r * R::CHUNKS;
            *reinterpret_cast<uint4*>(lds + r * R::PITCH + c * 16) = v[i];
        }
    }
};
// a wavefront's 32 rows as an operand: the lane's row, its half of every 2 * EPC channels
template <typename T, int DP> struct RaRows {
    typedef Ra<T, DP> R;
    uint4 v[R::KS];
    __device__ __forceinline__ void load(const T* row, bool there, int d, int g) {
#pragma unroll
        for (int s = 0; s < R::KS; ++s) {
            const int c = (2 * s + g) * R::EPC;
            v[s] = ld16(there && c < d ? row + c : row, there ? d - c : 0);
        }
    }
};
// rows row .. row + 31 of a tile times such rows: result[tile row][own row]
template <typename T, int DP>
__device__ __forceinline__ mm_f16 ra_products(const unsigned char* tile, int row, const RaRows<T, DP>& own, int lane) {
    typedef Ra<T, DP> R;
    mm_f16 acc = {};
    const unsigned char* p = tile + (row + (lane & 31)) * R::PITCH + (lane >> 5) * 16;
#pragma unroll
    for (int s = 0; s < R::KS; ++s) acc = Mm<T>::mul(*reinterpret_cast<const uint4*>(p + s * 32), own.v[s], acc);
    return acc;
}
// out[t][channel 32 t + .][own row] += sum over the tile's rows row .. row + 31 of tile[row][channel] w[row][own row], w as a result lies
template <typename T, int DP>
__device__ __forceinline__ void ra_mix(const unsigned char* tile, int row, const float (&w)[16], mm_f16 (&out)[DP / 32], int lane) {
    typedef Ra<T, DP> R;
#pragma unroll
    for (int u = 0; u < 16 / R::EPC; ++u) {
        const uint4 b = Mm<T>::pack(w + u * R::EPC);
#pragma unroll
        for (int t = 0; t < R::DT; ++t) out[t] = Mm<T>::mul(Mm<T>::columns(tile, R::PITCH, row + 2 * R::EPC * u, 32 * t, lane), b, out[t]);
    }
}
// four consecutive channels of a row
template <typename T>
__device__ __forceinline__ void ra_store4(T* p, int n, const float (&v)[4]) {
    T e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = to_store<T>(v[k]);
    if (n >= 4) { __builtin_memcpy(p, e, 4 * sizeof(T)); return; }
#pragma unroll
    for (int k = 0; k < 4; ++k) if (k < n) p[k] = e[k];
}

__device__ __forceinline__ int ra_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ int ra_keys(const AttnArgs& a, int n) { return a.len ? ra_clamp(a.len[n], 0, a.pk) : a.pk; }
__device__ __forceinline__ int ra_start(const AttnArgs& a, int n) { return a.start ? ra_clamp(a.start[n], -(1 << 29), 1 << 29) : 0; }

// The bias of head h by distance, lut[rel + reach + RA_PAD], in units of log2.  Finite values stay finite (a mask of the type's lowest value
// leaves a row of such values with equal probabilities, as the formula does).
__device__ __forceinline__ void ra_bias(const AttnArgs& a, int h, float* lut) {
    for (int t = threadIdx.x; t < 2 * a.reach + 1 + 2 * RA_PAD; t += RA_THREADS) {
        float b = 0.f;
        if (a.table) {
            b = a.table[(int64_t)h * a.nb + ra_clamp(a.map[ra_clamp(t - RA_PAD, 0, 2 * a.reach)], 0, a.nb - 1)];
            const float big = 3.402823466e38f;
            b = fabsf(b) <= big ? fminf(fmaxf(b * RA_LOG2E, -big), big) : b;
        }
        lut[t] = b;
    }
}

// The bias of a 32-row tile (keys or queries row0 ..) for this lane: 16 values at compile-time distances from one place, or one value
struct RaBias {
    const float* at;      // NULL: `far` everywhere
    float far;
};
// relmin, relmax: the least and largest distance of the wavefront's tile; rel: that of the lane's element 0
__device__ __forceinline__ RaBias ra_tile_bias(const float* lut, int reach, int relmin, int relmax, int rel) {
    if (relmax <= -reach) return {nullptr, lut[RA_PAD]};
    if (relmin >= reach) return {nullptr, lut[RA_PAD + 2 * reach]};
    return {lut + rel + reach + RA_PAD, 0.f};
}

struct RaBlock { int n, h, tile, split; };
__device__ __forceinline__ RaBlock ra_block(const AttnArgs& a, int heads, int tiles, int splits) {
    const int b = xcd_remap((int)blockIdx.x, (int)gridDim.x);
    RaBlock r;
    r.split = b % splits;
    const int x = b / splits, y = x / tiles;
    r.tile = x - y * tiles;
    r.h = y % heads;
    r.n = y / heads;
    return r;
}

// KEEP (a backward pass follows, bfloat16): p enters its product as two terms, and y is kept with what its rounding takes away.  In the gradient of
// the table most of ds cancels, and delta's error does not: with p of 8 bits the sum of a bucket is off by 3e-4, with 16 by 1e-6.
template <typename T, int DP, bool KEEP>
__global__ void __launch_bounds__(RA_THREADS, 2) relattn_fwd(AttnArgs a) {
    typedef Ra<T, DP> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char ra_lds[];
    unsigned char *kt = ra_lds, *vt = ra_lds + R::TILE;
    float* lut = reinterpret_cast<float*>(ra_lds + 2 * R::TILE);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 31, g = lane >> 5;
    const int tiles = (a.pq + RA_BM - 1) / RA_BM;
    RaBlock b = ra_block(a, a.H, tiles, a.splits);
    if (a.causal) b.tile = tiles - 1 - b.tile;             // (the blocks with the most keys first)
    const int n = b.n, h = b.h, hk = h / (a.H / a.G);
    const int i0 = b.tile * RA_BM + wave * 32, i = min(i0 + l, a.pq - 1);
    const bool work = i0 < a.pq;
    const int start = ra_start(a, n), keys = ra_keys(a, n), qmin = i0 + start, qmax = min(i0 + 31, a.pq - 1) + start, qpos = i + start;
    const T* kb = (const T*)a.k + (int64_t)n * a.pk * a.ldk + (int64_t)hk * a.d;
    const T* vb = (const T*)a.v + (int64_t)n * a.pk * a.ldv + (int64_t)hk * a.d;
    int end = keys;
    if (a.causal) end = ra_clamp(min(b.tile * RA_BM + RA_BM, a.pq) + start, 0, keys);
    const int all = (end + R::BN - 1) / R::BN, per = (all + a.splits - 1) / a.splits, t0 = b.split * per, t1 = min(all, t0 + per);
    RaTile<T, DP> kr, vr;
    if (t0 < t1) { kr.load(kb, a.ldk, t0 * R::BN, end, a.d); vr.load(vb, a.ldv, t0 * R::BN, end, a.d); }
    RaRows<T, DP> qr;
    qr.load((const T*)a.q + ((int64_t)n * a.pq + i) * a.ldq + (int64_t)h * a.d, work, a.d, g);
    ra_bias(a, h, lut);
    mm_f16 o[R::DT] = {};
    float top = -INFINITY, sum = 0.f;
    for (int t = t0; t < t1; ++t) {
        __syncthreads();
        kr.store(kt);
        vr.store(vt);
        __syncthreads();
        if (t + 1 < t1) { kr.load(kb, a.ldk, (t + 1) * R::BN, end, a.d); vr.load(vb, a.ldv, (t + 1) * R::BN, end, a.d); }
        const int j0 = t * R::BN;
        if (!work || (a.causal && j0 > qmax)) continue;
        const bool edge = j0 + R::BN > keys || (a.causal && j0 + R::BN - 1 > qmin);
        float s[R::BN / 32][16];
        const RaBias bias = ra_tile_bias(lut, a.reach, j0 - qmax, j0 + R::BN - 1 - qmin, j0 + 4 * g - qpos);
        float mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < R::BN / 32; ++u) {
            const mm_f16 acc = ra_products<T, DP>(kt, 32 * u, qr, lane);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float v = fmaf(acc[r], a.scale2, bias.at ? bias.at[32 * u + (r & 3) + 8 * (r >> 2)] : bias.far);
                if (edge) {
                    const int j = j0 + 32 * u + 4 * g + (r & 3) + 8 * (r >> 2);
                    if (j >= keys || (a.causal && j > qpos)) v = -INFINITY;
                }
                s[u][r] = v;
                mx = fmaxf(mx, v);
            }
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        mx = fmaxf(mx, top);
        const float base = mx == -INFINITY ? 0.f : mx, shrink = exp2_fast(top - base);
        top = mx;
        float part = 0.f;
#pragma unroll
        for (int u = 0; u < R::BN / 32; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) { s[u][r] = exp2_fast(s[u][r] - base); part += s[u][r]; }
        sum = fmaf(sum, shrink, part);
#pragma unroll
        for (int c = 0; c < R::DT; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[c][r] *= shrink;
        // (p enters the product in the element type: for bfloat16 an error of 2^-9 of each term, below the rounding of y)
#pragma unroll
        for (int u = 0; u < R::BN / 32; ++u) {
            ra_mix<T, DP>(vt, 32 * u, s[u], o, lane);
            if constexpr (KEEP && R::ES == 2) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[u][r] -= bf2f(f2bf(s[u][r]));
                ra_mix<T, DP>(vt, 32 * u, s[u], o, lane);
            }
        }
    }
    sum += __shfl_xor(sum, 32, 64);
    if (i0 + l >= a.pq) return;
    const int64_t row = ((int64_t)n * a.H + h) * a.pq + i;
    if (a.splits > 1) {
        const int64_t rows = (int64_t)a.m * a.H * a.pq, at = b.split * rows + row;
        if (g == 0) { a.part_ml[2 * at] = top; a.part_ml[2 * at + 1] = sum; }
#pragma unroll
        for (int c = 0; c < R::DT; ++c)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int ch = 32 * c + 4 * g + 2 * r;
                const float v[4] = {o[c][r], o[c][r + 1], o[c][r + 2], o[c][r + 3]};
                if (ch < a.d) ra_store4(a.part + at * a.d + ch, a.d - ch, v);
            }
        return;
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (KEEP && g == 0) a.stats[row] = {top, sum == 0.f ? -INFINITY : -log2f(sum)};
    T* yr = (T*)a.y + ((int64_t)n * a.pq + i) * a.ldy + (int64_t)h * a.d;
    bf16_t* low = a.low ? a.low + ((int64_t)n * a.pq + i) * a.H * a.d + (int64_t)h * a.d : nullptr;
#pragma unroll
    for (int c = 0; c < R::DT; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int ch = 32 * c + 4 * g + 2 * r;
            if (ch >= a.d) continue;
            float v[4] = {o[c][r] * inv, o[c][r + 1] * inv, o[c][r + 2] * inv, o[c][r + 3] * inv};
            ra_store4(yr + ch, a.d - ch, v);
            if (KEEP && R::ES == 2) {
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] -= bf2f(f2bf(v[k]));
                ra_store4(low + ch, a.d - ch, v);
            }
        }
}

// Joins the parts of a row: a wavefront per row, a lane per channel
template <typename T>
__global__ void __launch_bounds__(RA_THREADS) relattn_join(AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.m * a.H * a.pq, row = (int64_t)blockIdx.x * RA_WAVES + (threadIdx.x >> 6);
    if (row >= rows) return;
    float top = -INFINITY;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, a.part_ml[2 * (s * rows + row)]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int s = 0; s < a.splits; ++s) sum = fmaf(a.part_ml[2 * (s * rows + row) + 1], exp2_fast(a.part_ml[2 * (s * rows + row)] - base), sum);
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    if (a.stats && lane == 0) a.stats[row] = {top, sum == 0.f ? -INFINITY : -log2f(sum)};
    const int64_t nh = row / a.pq;
    const int i = (int)(row - nh * a.pq), h = (int)(nh % a.H), n = (int)(nh / a.H);
    T* yr = (T*)a.y + ((int64_t)n * a.pq + i) * a.ldy + (int64_t)h * a.d;
    for (int c = lane; c < a.d; c += 64) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s) v = fmaf(a.part[(s * rows + row) * a.d + c], exp2_fast(a.part_ml[2 * (s * rows + row)] - base), v);
        v *= inv;
        st(yr, c, v);
        if (sizeof(T) == 2 && a.low) st(a.low, ((int64_t)n * a.pq + i) * a.H * a.d + (int64_t)h * a.d + c, v - bf2f(f2bf(v)));
    }
}

// Sums of ds along the diagonals, carried over a wavefront's tiles of 32 keys (its 32 queries stay): `held` is this lane's sum for distance rel0 + lane
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
    // ds of keys j0 .. j0 + 31 (positions) by queries q0 .. q0 + 31: relmin = j0 - q0 - 31
    __device__ __forceinline__ void add(const float (&ds)[16], int relmin, float* area, int lane) {
        if (relmin + 62 <= -reach || relmin >= reach) {
            flush(lane);
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) s += ds[r];
            if (relmin >= reach) hi += s; else lo += s;
            return;
        }
        const int l = lane & 31, g = lane >> 5;
        if (!carrying) rel0 = relmin, carrying = true;
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

// dq of 128 queries, their delta, and the wavefronts' sums of ds by distance
template <typename T, int DP>
__global__ void __launch_bounds__(RA_THREADS, 1) relattn_bwd_q(AttnArgs a) {
    typedef Ra<T, DP> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char ra_lds[];
    unsigned char *kt = ra_lds, *vt = ra_lds + R::TILE;
    float* area = reinterpret_cast<float*>(ra_lds + 2 * R::TILE) + (threadIdx.x >> 6) * 63 * RA_DIAG_PITCH;
    float* lut = reinterpret_cast<float*>(ra_lds + 2 * R::TILE) + RA_WAVES * 63 * RA_DIAG_PITCH;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 31, g = lane >> 5;
    const int tiles = (a.pq + RA_BM - 1) / RA_BM;
    RaBlock b = ra_block(a, a.H, tiles, 1);
    if (a.causal) b.tile = tiles - 1 - b.tile;
    const int n = b.n, h = b.h, hk = h / (a.H / a.G);
    const int i0 = b.tile * RA_BM + wave * 32, i = min(i0 + l, a.pq - 1);
    const bool work = i0 < a.pq, mine = i0 + l < a.pq;
    const int start = ra_start(a, n), keys = ra_keys(a, n), qmin = i0 + start, qmax = min(i0 + 31, a.pq - 1) + start, qpos = i + start;
    const T* kb = (const T*)a.k + (int64_t)n * a.pk * a.ldk + (int64_t)hk * a.d;
    const T* vb = (const T*)a.v + (int64_t)n * a.pk * a.ldv + (int64_t)hk * a.d;
    int end = keys;
    if (a.causal) end = ra_clamp(min(b.tile * RA_BM + RA_BM, a.pq) + start, 0, keys);
    const int all = (end + R::BN - 1) / R::BN;
    RaTile<T, DP> kr, vr;
    if (all > 0) { kr.load(kb, a.ldk, 0, end, a.d); vr.load(vb, a.ldv, 0, end, a.d); }
    const int64_t row = ((int64_t)n * a.H + h) * a.pq + i, place = ((int64_t)n * a.pq + i) * a.ldy + (int64_t)h * a.d;
    RaRows<T, DP> qr, gr;
    qr.load((const T*)a.q + ((int64_t)n * a.pq + i) * a.ldq + (int64_t)h * a.d, mine, a.d, g);
    gr.load((const T*)a.dy + place, mine, a.d, g);
    // delta: y with what its rounding took away, or the sum over a bucket, in which most of ds cancels, would lose half of its digits
    float delta = 0.f;
    if (work) {
        const T* yr = (const T*)a.y + place;
        const bf16_t* low = a.low ? a.low + (((int64_t)n * a.pq + i) * a.H + h) * a.d : nullptr;
#pragma unroll
        for (int s = 0; s < R::KS; ++s) {
            const int c = (2 * s + g) * R::EPC;
            T e[R::EPC];
            __builtin_memcpy(e, &gr.v[s], 16);
#pragma unroll
            for (int k = 0; k < R::EPC; ++k)
                if (c + k < a.d) delta = fmaf(ld(e, k), ld(yr, c + k) + (low ? ld(low, c + k) : 0.f), delta);
        }
    }
    delta += __shfl_xor(delta, 32, 64);
    if (mine && g == 0) a.delta[row] = delta;
    const float2_ stat = mine ? a.stats[row] : float2_{0.f, -INFINITY};
    const float top = stat.y == -INFINITY ? 0.f : stat.x;
    ra_bias(a, h, lut);
    for (int t = lane; t < 63 * RA_DIAG_PITCH; t += 64) area[t] = 0.f;
    RaDiagonals dg;
    dg.reach = a.reach;
    dg.line = a.diag ? a.diag + (((int64_t)n * a.H + h) * ((a.pq + 31) / 32) + i0 / 32) * (2 * a.reach + 1) : nullptr;
    mm_f16 dq[R::DT] = {};
    for (int t = 0; t < all; ++t) {
        __syncthreads();
        kr.store(kt);
        vr.store(vt);
        __syncthreads();
        if (t + 1 < all) { kr.load(kb, a.ldk, (t + 1) * R::BN, end, a.d); vr.load(vb, a.ldv, (t + 1) * R::BN, end, a.d); }
#pragma unroll 1
        for (int u = 0; u < R::BN / 32; ++u) {
            const int j0 = t * R::BN + 32 * u;
            if (!work || j0 >= end || (a.causal && j0 > qmax)) continue;
            const bool edge = j0 + 32 > keys || i0 + 32 > a.pq || (a.causal && j0 + 31 > qmin);
            const RaBias bias = ra_tile_bias(lut, a.reach, j0 - qmax, j0 + 31 - qmin, j0 + 4 * g - qpos);
            const mm_f16 s = ra_products<T, DP>(kt, 32 * u, qr, lane), dp = ra_products<T, DP>(vt, 32 * u, gr, lane);
            float ds[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float v = fmaf(s[r], a.scale2, bias.at ? bias.at[(r & 3) + 8 * (r >> 2)] : bias.far);
                ds[r] = exp2_fast((v - top) + stat.y) * (dp[r] - delta);
                if (edge) {
                    const int j = j0 + 4 * g + (r & 3) + 8 * (r >> 2);
                    if (!mine || j >= keys || (a.causal && j > qpos)) ds[r] = 0.f;
                }
            }
            if (stat.y == -INFINITY) {
#pragma unroll
                for (int r = 0; r < 16; ++r) ds[r] = 0.f;
            }
            if (dg.line) dg.add(ds, j0 - i0 - start - 31, area, lane);
            ra_mix<T, DP>(kt, 32 * u, ds, dq, lane);
        }
    }
    if (!work) return;
    if (dg.line) dg.finish(lane);
    if (!mine) return;
    T* out = (T*)a.dq + ((int64_t)n * a.pq + i) * a.ldq + (int64_t)h * a.d;
#pragma unroll
    for (int c = 0; c < R::DT; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int ch = 32 * c + 4 * g + 2 * r;
            const float v[4] = {dq[c][r] * a.scale, dq[c][r + 1] * a.scale, dq[c][r + 2] * a.scale, dq[c][r + 3] * a.scale};
            if (ch < a.d) ra_store4(out + ch, a.d - ch, v);
        }
}

// dk and dv of 128 keys: the queries of every head that shares them, one head after the other
template <typename T, int DP>
__global__ void __launch_bounds__(RA_THREADS, 1) relattn_bwd_kv(AttnArgs a) {
    typedef Ra<T, DP> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char ra_lds[];
    unsigned char *qt = ra_lds, *gt = ra_lds + R::TILE;
    float* rowv = reinterpret_cast<float*>(ra_lds + 2 * R::TILE);          // [3][BN]: top, -log2 sum, delta
    float* lut = rowv + 3 * R::BN;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 31, g = lane >> 5;
    const int tiles = (a.pk + RA_BM - 1) / RA_BM;
    const RaBlock b = ra_block(a, a.G, tiles, 1);
    const int n = b.n, hk = b.h, share = a.H / a.G;
    const int j0 = b.tile * RA_BM + wave * 32, j = min(j0 + l, a.pk - 1);
    const int start = ra_start(a, n), keys = ra_keys(a, n);
    const bool work = j0 < keys, mine = j0 + l < keys;
    RaRows<T, DP> kr, vr;
    kr.load((const T*)a.k + ((int64_t)n * a.pk + j) * a.ldk + (int64_t)hk * a.d, mine, a.d, g);
    vr.load((const T*)a.v + ((int64_t)n * a.pk + j) * a.ldv + (int64_t)hk * a.d, mine, a.d, g);
    mm_f16 dk[R::DT] = {}, dv[R::DT] = {};
    const int first = a.causal ? ra_clamp(b.tile * RA_BM - start, 0, a.pq) : 0;       // no query before it sees one of the block's keys
    const int t0 = first / R::BN, t1 = b.tile * RA_BM < keys ? (a.pq + R::BN - 1) / R::BN : 0;
    for (int hh = 0; hh < share; ++hh) {
        const int h = hk * share + hh;
        const T* qb = (const T*)a.q + (int64_t)n * a.pq * a.ldq + (int64_t)h * a.d;
        const T* gb = (const T*)a.dy + (int64_t)n * a.pq * a.ldy + (int64_t)h * a.d;
        const int64_t row0 = ((int64_t)n * a.H + h) * a.pq;
        RaTile<T, DP> qs, gs;
        float2_ st = {0.f, -INFINITY};
        float dl = 0.f;
        auto load = [&](int t) __attribute__((always_inline)) {
            qs.load(qb, a.ldq, t * R::BN, a.pq, a.d);
            gs.load(gb, a.ldy, t * R::BN, a.pq, a.d);
            st = {0.f, -INFINITY};
            dl = 0.f;
            const int i = t * R::BN + (int)threadIdx.x;
            if ((int)threadIdx.x < R::BN && i < a.pq) { st = a.stats[row0 + i]; dl = a.delta[row0 + i]; }
        };
        if (t0 < t1) load(t0);
        __syncthreads();                                   // (the bias of the head before has been read)
        ra_bias(a, h, lut);
        for (int t = t0; t < t1; ++t) {
            __syncthreads();
            qs.store(qt);
            gs.store(gt);
            if ((int)threadIdx.x < R::BN) {
                rowv[threadIdx.x] = st.y == -INFINITY ? 0.f : st.x;
                rowv[R::BN + threadIdx.x] = st.y;
                rowv[2 * R::BN + threadIdx.x] = dl;
            }
            __syncthreads();
            if (t + 1 < t1) load(t + 1);
#pragma unroll 1
            for (int u = 0; u < R::BN / 32; ++u) {
                const int i0 = t * R::BN + 32 * u, qmin = i0 + start, qmax = min(i0 + 31, a.pq - 1) + start;
                if (!work || i0 >= a.pq || (a.causal && j0 > qmax)) continue;
                const bool edge = j0 + 32 > keys || i0 + 32 > a.pq || (a.causal && j0 + 31 > qmin);
                const RaBias bias = ra_tile_bias(lut, a.reach, j0 - i0 - start - 31, j0 + 31 - qmin, j0 + l - i0 - start - 4 * g);
                const mm_f16 s = ra_products<T, DP>(qt, 32 * u, kr, lane), dp = ra_products<T, DP>(gt, 32 * u, vr, lane);
                float p[16], ds[16];
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const float* rv = rowv + 32 * u + 8 * r4 + 4 * g;
                    const float4 tp = *reinterpret_cast<const float4*>(rv), ls = *reinterpret_cast<const float4*>(rv + R::BN), de = *reinterpret_cast<const float4*>(rv + 2 * R::BN);
                    const float tops[4] = {tp.x, tp.y, tp.z, tp.w}, logs[4] = {ls.x, ls.y, ls.z, ls.w}, deltas[4] = {de.x, de.y, de.z, de.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 4 * r4 + e;
                        const float v = fmaf(s[r], a.scale2, bias.at ? bias.at[-(e + 8 * r4)] : bias.far);
                        p[r] = exp2_fast((v - tops[e]) + logs[e]);
                        ds[r] = p[r] * (dp[r] - deltas[e]);
                        if (edge || logs[e] == -INFINITY) {
                            const int i = i0 + 4 * g + e + 8 * r4;
                            if (!mine || i >= a.pq || (a.causal && j > i + start) || logs[e] == -INFINITY) p[r] = ds[r] = 0.f;
                        }
                    }
                }
                ra_mix<T, DP>(gt, 32 * u, p, dv, lane);
                ra_mix<T, DP>(qt, 32 * u, ds, dk, lane);
            }
        }
    }
    if (j0 + l >= a.pk) return;                            // (keys behind the last one of the sample have gradients of zero)
    T* ok = (T*)a.dk + ((int64_t)n * a.pk + j) * a.ldk + (int64_t)hk * a.d;
    T* ov = (T*)a.dv + ((int64_t)n * a.pk + j) * a.ldv + (int64_t)hk * a.d;
#pragma unroll
    for (int c = 0; c < R::DT; ++c)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int ch = 32 * c + 4 * g + 2 * r;
            const float vk[4] = {dk[c][r] * a.scale, dk[c][r + 1] * a.scale, dk[c][r + 2] * a.scale, dk[c][r + 3] * a.scale};
            const float vv[4] = {dv[c][r], dv[c][r + 1], dv[c][r + 2], dv[c][r + 3]};
            if (ch < a.d) { ra_store4(ok + ch, a.d - ch, vk); ra_store4(ov + ch, a.d - ch, vv); }
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
    const int h = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int c = threadIdx.x; c < nd; c += RA_THREADS) {
        float s = 0.f;
        for (int k = 0; k < RA_SHARES; ++k) s += shares[((int64_t)k * H + h) * nd + c];
        ra_sums[c] = s;
    }
    __syncthreads();
    for (int b = wave; b < nb; b += RA_WAVES) {
        float s = 0.f;
        for (int c = lane; c < nd; c += 64) if (ra_clamp(map[c], 0, nb - 1) == b) s += ra_sums[c];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
        if (lane == 0) dtable[(int64_t)h * nb + b] = accumulate ? dtable[(int64_t)h * nb + b] + s : s;
    }
}

static size_t ra_up(size_t b) { return (b + 255) & ~(size_t)255; }
// Keys over several blocks where queries and heads do not fill the card twice: parts of at least 256 keys.
static int ra_splits(const lpm_attn_geom& g, int32_t dtype) {
    const int64_t blocks = (int64_t)g.m * g.heads * ((g.pq + RA_BM - 1) / RA_BM);
    const int most = std::max(1, g.pk / 256);
    if (blocks == 0 || blocks >= 512) return 1;
    return (int)std::min<int64_t>(most, (512 + blocks - 1) / blocks);
}
struct AttnLayout { size_t low, stats_all, part, part_ml, fwd_all, delta, diag, shares, bwd_all; };
static AttnLayout ra_layout(const lpm_attn_geom& g, int32_t dtype, int splits) {
    AttnLayout o;
    const size_t rows = (size_t)g.m * g.heads * g.pq, nd = 2 * (size_t)g.reach + 1;
    o.low = ra_up(rows * 8);
    o.stats_all = o.low + (dtype == LPM_BF16 ? ra_up(rows * g.d * 2) : 0);
    o.part = 0;
    o.part_ml = splits > 1 ? ra_up((size_t)splits * rows * g.d * 4) : 0;
    o.fwd_all = splits > 1 ? o.part_ml + ra_up((size_t)splits * rows * 8) : 0;
    o.delta = 0;
    o.diag = ra_up(rows * 4);
    o.shares = o.diag + (g.n_buckets ? ra_up((size_t)g.m * g.heads * ((g.pq + 31) / 32) * nd * 4) : 0);
    o.bwd_all = o.shares + (g.n_buckets ? ra_up((size_t)RA_SHARES * g.heads * nd * 4) : 0);
    return o;
}

template <typename T, int DP, bool KEEP> static hipError_t ra_forward(const AttnArgs& a, hipStream_t st) {
    typedef Ra<T, DP> R;
    static DeviceSet done;
    const size_t lds = 2 * R::TILE + (2 * (size_t)a.reach + 1 + 2 * RA_PAD) * 4;
    const hipError_t e = allow_lds(relattn_fwd<T, DP, KEEP>, 160 * 1024 - 256, done);
    if (e != hipSuccess) return e;
    const int tiles = (a.pq + RA_BM - 1) / RA_BM;
    hipLaunchKernelGGL((relattn_fwd<T, DP, KEEP>), dim3((unsigned)(a.m * a.H * tiles * a.splits)), dim3(RA_THREADS), lds, st, a);
    return hipGetLastError();
}
template <typename T, int DP> static hipError_t ra_backward(const AttnArgs& a, hipStream_t st) {
    typedef Ra<T, DP> R;
    static DeviceSet done_q, done_kv;
    const size_t lut = (2 * (size_t)a.reach + 1 + 2 * RA_PAD) * 4;
    hipError_t e = allow_lds(relattn_bwd_q<T, DP>, 160 * 1024 - 256, done_q);
    if (e == hipSuccess) e = allow_lds(relattn_bwd_kv<T, DP>, 160 * 1024 - 256, done_kv);
    if (e != hipSuccess) return e;
    const int qt = (a.pq + RA_BM - 1) / RA_BM, kt = (a.pk + RA_BM - 1) / RA_BM;
    if (qt) hipLaunchKernelGGL((relattn_bwd_q<T, DP>), dim3((unsigned)(a.m * a.H * qt)), dim3(RA_THREADS), 2 * R::TILE + RA_WAVES * 63 * RA_DIAG_PITCH * 4 + lut, st, a);
    if (kt) hipLaunchKernelGGL((relattn_bwd_kv<T, DP>), dim3((unsigned)(a.m * a.G * kt)), dim3(RA_THREADS), 2 * R::TILE + 3 * R::BN * 4 + lut, st, a);
    return hipGetLastError();
}
#define LPM_RA(dtype_, d_, call_)                                                          \
    ((dtype_) == LPM_BF16 ? ((d_) <= 32 ? call_(bf16_t, 32) : (d_) <= 64 ? call_(bf16_t, 64) : (d_) <= 96 ? call_(bf16_t, 96) : call_(bf16_t, 128)) \
                          : ((d_) <= 32 ? call_(float, 32) : (d_) <= 64 ? call_(float, 64) : (d_) <= 96 ? call_(float, 96) : call_(float, 128)))

}  // namespace lpm

static int32_t ra_check(const lpm_attn_geom* g, int32_t dtype, lpm_attn_geom& o) {
    if (!g) return fail(LPM_EINVAL, "geometry is NULL");
    if (dtype != LPM_F32 && dtype != LPM_BF16) return fail(LPM_EINVAL, "dtype must be LPM_F32 or LPM_BF16");
    o = *g;
    if (o.m < 0 || o.pq < 0 || o.pk < 0 || o.pq > (1 << 28) || o.pk > (1 << 28) || o.heads <= 0 || o.heads > 65535 || o.kv_heads <= 0 || o.heads % o.kv_heads)
        return fail(LPM_ESHAPE, "attention of %d samples, %d queries, %d keys, %d heads on %d", o.m, o.pq, o.pk, o.heads, o.kv_heads);
    if (o.d < 1 || o.d > 128) return fail(LPM_ESHAPE, "heads of %d channels (1 to 128)", o.d);
    if (o.n_buckets < 0 || o.n_buckets > 65536 || o.reach < 0 || o.reach > RA_MAX_REACH)
        return fail(LPM_ESHAPE, "%d buckets (0 to 65536) of distances up to %d (0 to %d)", o.n_buckets, o.reach, RA_MAX_REACH);
    if (!(o.scale >= 0.f) || o.scale > 1e30f) return fail(LPM_EINVAL, "scale must be a number of 0 (for 1 / sqrt(d)) or more");
    const int64_t wq = (int64_t)o.heads * o.d, wk = (int64_t)o.kv_heads * o.d;
    if (wq >= (1 << 28)) return fail(LPM_ESHAPE, "%d heads of %d channels", o.heads, o.d);
    if (!o.ldq) o.ldq = (int32_t)wq;
    if (!o.ldk) o.ldk = (int32_t)wk;
    if (!o.ldv) o.ldv = (int32_t)wk;
    if (!o.ldy) o.ldy = (int32_t)wq;
    if (o.ldq < wq || o.ldy < wq || o.ldk < wk || o.ldv < wk) return fail(LPM_ESHAPE, "positions closer than their heads are wide");
    if (o.scale == 0.f) o.scale = 1.f / sqrtf((float)o.d);
    if (!o.n_buckets) o.reach = 0;
    const int64_t most = std::max<int64_t>(o.pq, o.pk) / 32 + 1;
    if ((int64_t)o.m * o.heads > (int64_t)1 << 31 || (int64_t)o.m * o.heads * most >= (int64_t)1 << 31) return fail(LPM_ESHAPE, "more blocks than a launch takes");
    return LPM_OK;
}
static AttnArgs ra_args(const lpm_attn_geom& g, const void* q, const void* k, const void* v, const int32_t* len, const int32_t* start, const int32_t* map,
                        const float* table) {
    AttnArgs a{};
    a.m = g.m; a.H = g.heads; a.G = g.kv_heads; a.pq = g.pq; a.pk = g.pk; a.d = g.d; a.causal = g.causal != 0;
    a.nb = g.n_buckets; a.reach = g.reach; a.splits = 1;
    a.ldq = g.ldq; a.ldk = g.ldk; a.ldv = g.ldv; a.ldy = g.ldy;
    a.scale = g.scale; a.scale2 = g.scale * RA_LOG2E;
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
    const AttnLayout o = ra_layout(g, dtype, ra_splits(g, dtype));
    if (forward) *forward = o.fwd_all;
    if (backward) *backward = o.bwd_all;
    return LPM_OK;
}

extern "C" int32_t lpm_attn_stats_bytes(const lpm_attn_geom* geom, int32_t dtype, size_t* bytes) {
    if (!bytes) return fail(LPM_EINVAL, "bytes is NULL");
    lpm_attn_geom g;
    const int32_t rc = ra_check(geom, dtype, g);
    if (rc) return rc;
    *bytes = ra_layout(g, dtype, 1).stats_all;
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
    a.splits = ra_splits(g, dtype);
    if (a.splits > 1 && !ws) return fail(LPM_EINVAL, "scratch required");
    const AttnLayout o = ra_layout(g, dtype, a.splits);
    a.y = y;
    a.stats = (float2_*)stats;
    a.low = stats && dtype == LPM_BF16 ? (bf16_t*)((char*)stats + o.low) : nullptr;
    a.part = (float*)ws;
    a.part_ml = (float*)((char*)ws + o.part_ml);
    hipStream_t st = (hipStream_t)stream;
#define LPM_RA_CALL(T_, DP_) (stats ? ra_forward<T_, DP_, true>(a, st) : ra_forward<T_, DP_, false>(a, st))
    LPM_HIP(LPM_RA(dtype, g.d, LPM_RA_CALL));
#undef LPM_RA_CALL
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
    const AttnLayout o = ra_layout(g, dtype, 1);
    AttnArgs a = ra_args(g, q, k, v, key_len, q_start, map, table);
    a.y = const_cast<void*>(y);
    a.dy = dy;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.stats = (float2_*)const_cast<void*>(stats);
    a.low = dtype == LPM_BF16 && stats ? (bf16_t*)((char*)const_cast<void*>(stats) + o.low) : nullptr;
    a.delta = (float*)ws;
    a.diag = dtable ? (float*)((char*)ws + o.diag) : nullptr;
    hipStream_t st = (hipStream_t)stream;
    if (queries || keys) {
#define LPM_RA_CALL(T_, DP_) ra_backward<T_, DP_>(a, st)
        LPM_HIP(LPM_RA(dtype, g.d, LPM_RA_CALL));
#undef LPM_RA_CALL
    }
    if (dtable) {
        const int nd = 2 * g.reach + 1, lines = (g.pq + 31) / 32;
        float* shares = (float*)((char*)ws + o.shares);
        hipLaunchKernelGGL(relattn_diagonals, dim3((unsigned)((nd + 63) / 64), (unsigned)g.heads, RA_SHARES), dim3(RA_THREADS), 0, st, (const float*)a.diag, g.m,
                           g.heads, lines, nd, shares);
        hipLaunchKernelGGL(relattn_buckets, dim3((unsigned)g.heads), dim3(RA_THREADS), (size_t)nd * 4, st, (const float*)shares, map, g.heads, g.n_buckets, nd, dtable,
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
