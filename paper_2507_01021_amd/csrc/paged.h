// Kernels of a paged key/value cache: appending rows, copying pages, reading
// sequences out, and causal attention of new tokens over the pages.
//
// Memory: page g of layer l holds, for every key/value head, P positions of
// keys and P of values, D numbers each, both in the order in which a matrix
// instruction takes them (16-byte pieces of 64 lanes, 1 KiB blocks), so that
// an operand fragment is one contiguous load and needs no transposition:
//   pages [page][layer][K, V][kv head][P * D]
//   keys:   blocks of 16 positions x 16 bytes x 4 of dims (dec_off with row =
//           position), as the A operand of S^T = K Q^T;
//   values: blocks of 16 dims x 32 positions (bf16) or 16 (fp32), as the A
//           operand of O^T += V^T P^T, whose positions are ordered so that a
//           lane's scores are its own weights (val_off).
// A page is one contiguous block over all layers, so copying one is one long
// run.
#pragma once

#include <type_traits>

#include "common.h"

namespace wmi {

// Element offset of (position p, dim c) in a head's values of D dims.
template <class T>
__host__ __device__ inline int val_off(int p, int c, int D) {
    if constexpr (sizeof(T) == 2)
        return ((p >> 5) * (D >> 4) + (c >> 4)) * 512 + (((p >> 2) & 3) * 16 + (c & 15)) * 8 + ((p & 16) >> 2) + (p & 3);
    else
        return ((p >> 4) * (D >> 4) + (c >> 4)) * 256 + (((p >> 2) & 3) * 16 + (c & 15)) * 4 + (p & 3);
}

// An entry of a list that no running kernel writes, at an address that is the
// same in all lanes: a scalar load, which does not queue behind vector loads.
typedef const int __attribute__((address_space(4))) * ScalarList;
__device__ __forceinline__ int list_at(const int* list, int i) { return ((ScalarList)(uintptr_t)list)[i]; }

// The pages of a cache as a kernel sees them. table[seq * ld + i] is the
// i-th page of a sequence.
struct PagedView {
    unsigned char* pages;
    const int* table;
    int ld;
    int shift;             // log2 of the positions per page
    int n_layer, Hkv;
    long long head_elems;  // P * D
    // 1 once a value that is not finite was appended: attention then takes care
    // of 0 * inf at hidden positions. Null: it always does.
    int* odd;
    __device__ __forceinline__ bool may_be_odd() const { return !odd || list_at(odd, 0) != 0; }
    template <class T>
    __device__ T* head(int page, int layer, int kv, int h) const {
        return reinterpret_cast<T*>(pages) + (((long long)page * n_layer + layer) * 2 + kv) * Hkv * head_elems +
               (long long)h * head_elems;
    }
};

// Whether a 16-byte piece has a number that is not finite (all exponent bits set).
template <class T>
__device__ __forceinline__ bool not_finite(u32x4 x) {
    bool odd = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        odd = odd || (x[k] & 0x7f800000u) == 0x7f800000u;
        if (sizeof(T) == 2) odd = odd || (x[k] & 0x7f80u) == 0x7f80u;
    }
    return odd;
}

// A run of up to 32 positions of one sequence inside one block of 32, and the
// row of its first position in the caller's rows.
struct PageTile {
    int seq, pos, n;
    int row;
};

// Head of a device list: what it holds and where (in ints from its start).
// Kernels read it when they run and go through their part in strides of the
// grid, so a recorded launch serves whatever list is current at its replay.
struct ListHead {
    int items, merges, tiles, merges_at, tiles_at, bigs, bigs_at, pad;
};
constexpr int HEAD_INTS = sizeof(ListHead) / sizeof(int);

// ------------------------------------------------------------------ small lists
//
// Lists of up to PUT_INTS numbers reach the device as a kernel argument: no
// copy engine, nothing to wait for, and the host may go on at once.
constexpr int PUT_INTS = 960;
struct PutInts {
    int n;
    int v[PUT_INTS];
};
// The list's numbers upd .. upd + 2 n - 1 are changes of page lists as well
// (table[first] = second), made at once.
static __global__ __launch_bounds__(256) void put_ints_kernel(PutInts a, int* __restrict__ dst, int upd, int n,
                                                              int* __restrict__ table) {
    for (int i = threadIdx.x; i < a.n; i += 256) dst[i] = a.v[i];
    for (int i = threadIdx.x; i < n; i += 256) table[a.v[upd + 2 * i]] = a.v[upd + 2 * i + 1];
}
// table[at[2 i]] = at[2 i + 1]
static __global__ __launch_bounds__(256) void table_update_kernel(const int* __restrict__ at, int n, int* __restrict__ table) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) table[at[2 * i]] = at[2 * i + 1];
}

// ------------------------------------------------------------------ rows in and out
//
// Rows [layer][row][kv head][D] (layer stride layer_ld, row stride row_ld
// elements). One workgroup per (tile, kv head, layer) moves a tile's keys and
// values through LDS, so that memory is accessed in 16-byte pieces on both
// sides; a tile that does not cover a whole value piece writes single
// elements. VEC: rows are 16-byte aligned. Bound by HBM: 2514 tokens, 12 heads of
// 64, 12 layers in bf16 are written in 36 us (5.1 TB/s read and written); five
// sequences of 229, 20 heads, 32 layers read out in 57 us (6.6 TB/s, three pages
// of four being shared). A single appended token's values are 2-byte stores 16
// bytes apart: 32 tokens, 20 heads of 64 take 28 us for 32 layers at once, 5 for one.
template <class T, int D, bool VEC>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                           const T* __restrict__ k, const T* __restrict__ v,
                                                           long long k_ld, long long v_ld, long long k_layer,
                                                           long long v_layer) {
    constexpr int EL = 16 / sizeof(T);  // elements of a 16-byte piece
    constexpr int CH = D / EL;          // pieces of a row
    constexpr int LD = D + EL;          // LDS row
    __shared__ __align__(16) T sv[32 * LD];
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int h = blockIdx.y, layer = layer0 + blockIdx.z, tid = threadIdx.x;
    for (int it = blockIdx.x; it < head.tiles; it += gridDim.x) {
        const PageTile t = tiles[it];
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        const int p0 = t.pos & ((1 << c.shift) - 1);
        T* kd = c.head<T>(page, layer, 0, h);
        T* vd = c.head<T>(page, layer, 1, h);
        const T* ks = k + blockIdx.z * k_layer + (long long)t.row * k_ld + h * D;
        const T* vs = v + blockIdx.z * v_layer + (long long)t.row * v_ld + h * D;
        bool odd = false;
        for (int i = tid; i < t.n * CH; i += 256) {
            const int r = i / CH, ch = i - r * CH;
            if constexpr (VEC) {
                const u32x4 a = *reinterpret_cast<const u32x4*>(ks + r * k_ld + ch * EL);
                const u32x4 b = *reinterpret_cast<const u32x4*>(vs + r * v_ld + ch * EL);
                *reinterpret_cast<u32x4*>(kd + dec_off<T>(p0 + r, ch * EL, D)) = a;
                *reinterpret_cast<u32x4*>(sv + ((p0 + r) & 31) * LD + ch * EL) = b;
                odd = odd || not_finite<T>(b);
            } else {
                for (int e = 0; e < EL; ++e) {
                    odd = odd || !(fabsf(ldf(vs + r * v_ld + ch * EL + e)) < INFINITY);
                    kd[dec_off<T>(p0 + r, ch * EL + e, D)] = ks[r * k_ld + ch * EL + e];
                    sv[((p0 + r) & 31) * LD + ch * EL + e] = vs[r * v_ld + ch * EL + e];
                }
            }
        }
        if (c.odd && odd) *c.odd = 1;
        __syncthreads();
        // value pieces of the tile's block of 32 positions: EL positions of one dim each
        const int lo = p0 & 31, hi = lo + t.n;
        T* vb = vd + val_off<T>(p0 & ~31, 0, D);
        for (int i = tid; i < 32 * CH; i += 256) {
            // piece i: block i / 64 (16 dims; in fp32 the 16-position halves come first), lane i % 64
            const int blk = i >> 6, ln = i & 63;
            const int half = sizeof(T) == 2 ? 0 : blk / (D >> 4);
            const int dim = (blk - half * (D >> 4)) * 16 + (ln & 15), g = ln >> 4;
            struct Elems { T e[EL]; } e;
            bool all = true;
#pragma unroll
            for (int j = 0; j < EL; ++j) {
                const int pos = sizeof(T) == 2 ? g * 4 + (j & 3) + (j >> 2) * 16 : half * 16 + g * 4 + j;
                all = all && pos >= lo && pos < hi;
                e.e[j] = sv[pos * LD + dim];
            }
            T* dst = vb + blk * (1024 / sizeof(T)) + ln * EL;
            if (all) {
                *reinterpret_cast<u32x4*>(dst) = __builtin_bit_cast(u32x4, e);
            } else {
#pragma unroll
                for (int j = 0; j < EL; ++j) {
                    const int pos = sizeof(T) == 2 ? g * 4 + (j & 3) + (j >> 2) * 16 : half * 16 + g * 4 + j;
                    if (pos >= lo && pos < hi) dst[j] = e.e[j];
                }
            }
        }
        __syncthreads();  // the next tile's LDS
    }
}

template <class T, int D, bool VEC>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                         T* __restrict__ k, T* __restrict__ v, long long k_ld,
                                                         long long v_ld, long long k_layer, long long v_layer) {
    constexpr int EL = 16 / sizeof(T);
    constexpr int CH = D / EL;
    constexpr int LD = D + EL;
    __shared__ __align__(16) T sv[32 * LD];
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int h = blockIdx.y, layer = layer0 + blockIdx.z, tid = threadIdx.x;
    for (int it = blockIdx.x; it < head.tiles; it += gridDim.x) {
        const PageTile t = tiles[it];
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        const int p0 = t.pos & ((1 << c.shift) - 1);
        const T* kd = c.head<T>(page, layer, 0, h);
        const T* vb = c.head<T>(page, layer, 1, h) + val_off<T>(p0 & ~31, 0, D);
        T* ks = k + blockIdx.z * k_layer + (long long)t.row * k_ld + h * D;
        T* vs = v + blockIdx.z * v_layer + (long long)t.row * v_ld + h * D;
        for (int i = tid; i < 32 * CH; i += 256) {
            const int blk = i >> 6, ln = i & 63;
            const int half = sizeof(T) == 2 ? 0 : blk / (D >> 4);
            const int dim = (blk - half * (D >> 4)) * 16 + (ln & 15), g = ln >> 4;
            const u32x4 a = *reinterpret_cast<const u32x4*>(vb + blk * (1024 / sizeof(T)) + ln * EL);
            struct Elems { T e[EL]; };
            const Elems e = __builtin_bit_cast(Elems, a);
#pragma unroll
            for (int j = 0; j < EL; ++j) {
                const int pos = sizeof(T) == 2 ? g * 4 + (j & 3) + (j >> 2) * 16 : half * 16 + g * 4 + j;
                sv[pos * LD + dim] = e.e[j];
            }
        }
        __syncthreads();
        for (int i = tid; i < t.n * CH; i += 256) {
            const int r = i / CH, ch = i - r * CH;
            if constexpr (VEC) {
                *reinterpret_cast<u32x4*>(ks + r * k_ld + ch * EL) =
                    *reinterpret_cast<const u32x4*>(kd + dec_off<T>(p0 + r, ch * EL, D));
                *reinterpret_cast<u32x4*>(vs + r * v_ld + ch * EL) =
                    *reinterpret_cast<const u32x4*>(sv + ((p0 + r) & 31) * LD + ch * EL);
            } else {
                for (int e = 0; e < EL; ++e) {
                    ks[r * k_ld + ch * EL + e] = kd[dec_off<T>(p0 + r, ch * EL + e, D)];
                    vs[r * v_ld + ch * EL + e] = sv[((p0 + r) & 31) * LD + ch * EL + e];
                }
            }
        }
        __syncthreads();  // the next tile's LDS
    }
}

// Copies whole pages (all layers): pairs (source, destination), `bytes` each,
// a multiple of 4096; five pages of 10.5 MB in 12.8 us (from L2 and the cache behind it). Workgroups of a pair take 16 KiB each.
constexpr int PAGE_RUN = 16384;
static __global__ __launch_bounds__(256) void paged_copy_kernel(unsigned char* __restrict__ pages,
                                                         const int* __restrict__ pairs, long long bytes) {
    const long long at = (long long)blockIdx.x * PAGE_RUN + threadIdx.x * 16;
    const unsigned char* s = pages + pairs[2 * blockIdx.y] * bytes + at;
    unsigned char* d = pages + pairs[2 * blockIdx.y + 1] * bytes + at;
    u32x4 a[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (at + u * 4096 < bytes) a[u] = *reinterpret_cast<const u32x4*>(s + u * 4096);
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (at + u * 4096 < bytes) *reinterpret_cast<u32x4*>(d + u * 4096) = a[u];
}

// ------------------------------------------------------------------ attention of few rows
//
// Query rows of a sequence and kv head: row j = token * G + g of the chunk's
// `count` tokens and the G query heads that share the kv head. Token i of a
// sequence that held `past` positions sees positions 0 .. past + i.
// An item is 16 such rows and a range of positions [kv0, kv1); the ranges of
// rows that are cut over several items are joined by paged_merge_kernel.
struct AttnItem {
    int seq, past, count;
    int tok0;       // the sequence's first token row in q and out
    int j0;         // first of up to 16 rows
    int kv0, kv1;   // positions, kv0 a multiple of 32
    int part;       // result slot of a cut range, or -1: the result itself
};
// Rows j0 .. j0 + 15 of a sequence whose positions were cut into n parts, in
// slots part, part + step, ...
struct MergeItem {
    int count, tok0, j0, part, n, step;
};
struct AttnArgs {
    PagedView c;
    int layer, H, G;
    const void* q;
    void* out;
    long long q_ld, out_ld;  // elements per token row
    float scale;             // of the scores, times log2(e)
    const int* plan;         // ListHead, then the items; merges at its merges_at
    float* parts;            // [part][kv head][16][D + 2]: sums, maximum, weight
};

// Four consecutive outputs of a row, row-major or as the projections take
// their activations (dec_off).
template <class T, bool FRAG>
__device__ inline void attn_store(const AttnArgs& a, int row, int h, int D, int dim, float x, float y, float z, float w) {
    T* out = static_cast<T*>(a.out);
    if constexpr (FRAG)
        st4(out + dec_off<T>(row, h * D + dim, a.H * D), x, y, z, w);
    else
        st4(out + (long long)row * a.out_ld + h * D + dim, x, y, z, w);
}

// Fragments of 16 bytes and the products over them. bf16: one 16x16x32
// instruction per fragment pair; fp32: four 16x16x4 ones.
template <class T> struct Piece;
template <> struct Piece<bf16> {
    typedef mfma_bf16x8 V;
    __device__ static inline mfma_f32x4 mul(V a, V b, mfma_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Piece<float> {
    typedef mfma_f32x4 V;
    __device__ static inline mfma_f32x4 mul(V a, V b, mfma_f32x4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

// 16 rows per workgroup; its four waves take the item's blocks of 32 positions
// in turn and join their results in LDS. Per wave and block
//   S^T[position][row] = K Q^T, running maximum and sum per row (a lane holds
//   8 positions of one row), O^T[dim][row] += V^T P^T with the lane's own
//   weights as the B operand.
// Bound by the bytes of the cache where it is long (4 tokens over 60001
// positions at most, 32 / 8 heads of 128 in bf16, 733 MB: 128 us, 5.7 TB/s), else
// by the chain of loads plan - page - keys (32 tokens over 447 positions at most,
// 20 heads of 64: 8.7 us for 40 MB). Ranges of up to 512 positions are not cut:
// cut from 256 on, those 32 tokens took 14.5 us, the merge included; 2048
// workgroups instead of 1024 took 196 instead of 162 us for the long ones.
// Scores, maxima, sums and outputs are fp32; a weight enters the product with
// bf16 values as the sum of two bf16 numbers, which leaves 2^-16 of it at most
// (rounded to one it would lose 2^-8): 9.7 instead of 9.6 us for the 32 tokens,
// 133 for the long ones either way, 3 % on average for 4 to 96 rows a sequence.
// Positions at or beyond kv1 may hold what was there before, and a block may
// have positions that only some rows see: weights 0, and since 0 * inf is not
// 0, values behind kv1 are replaced by zeros and such a block is multiplied row
// by row if its values are not all finite (if any ever was not).
template <class T, int D, bool FRAG>
__global__ __launch_bounds__(256) void paged_attn_kernel(AttnArgs a) {
    typedef typename Piece<T>::V V;
    constexpr int EL = 16 / sizeof(T), NK = D / KSTEP<T>, ND = D / 16, BLK = 1024 / sizeof(T);
    constexpr int NV = sizeof(T) == 2 ? 1 : 2;  // value blocks per 32 positions and 16 dims
    constexpr bool TWO = sizeof(T) == 2;        // weights as two numbers of the values' type
    __shared__ float so[4][16][D + 4];
    __shared__ float sm[4][16], sl[4][16];
    const ListHead head = *reinterpret_cast<const ListHead*>(a.plan);
    const AttnItem* items = reinterpret_cast<const AttnItem*>(a.plan + HEAD_INTS);
    const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool check = a.c.may_be_odd();
    for (int w0 = blockIdx.x; w0 < head.items * a.c.Hkv; w0 += gridDim.x) {
        const int it = w0 / a.c.Hkv, h = w0 - it * a.c.Hkv;
        const AttnItem t = items[it];
        const int rows = t.count * a.G;
        const int j = min(t.j0 + fr, rows - 1), tok = j / a.G, g = j - tok * a.G;
        const int lim = t.past + tok + 1;            // positions this lane's row sees
        const int all = t.past + t.j0 / a.G + 1;     // positions every row sees
        const T* q = static_cast<const T*>(a.q) + (long long)(t.tok0 + tok) * a.q_ld + (h * a.G + g) * D + fc * EL;
        V qf[NK];
#pragma unroll
        for (int s = 0; s < NK; ++s) qf[s] = *reinterpret_cast<const V*>(q + s * KSTEP<T>);
        mfma_f32x4 o[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        const int* table = a.c.table + (long long)t.seq * a.c.ld;
        const int pmask = (1 << a.c.shift) - 1;
        int next = list_at(table, min(t.kv0 + wave * 32, t.kv1 - 1) >> a.c.shift);  // pages are looked up a block ahead
        for (int p = t.kv0 + wave * 32; p < t.kv1; p += 128) {
            const int page = next, p0 = p & pmask;
            next = list_at(table, min(p + 128, t.kv1 - 1) >> a.c.shift);
            const T* kb = a.c.template head<T>(page, a.layer, 0, h) + (p0 >> 4) * (NK * BLK) + lane * EL;
            const T* vb = a.c.template head<T>(page, a.layer, 1, h) + val_off<T>(p0, 0, D) + lane * EL;
            V kf[2][NK], vf[NV][ND];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int s = 0; s < NK; ++s) kf[b][s] = *reinterpret_cast<const V*>(kb + (b * NK + s) * BLK);
#pragma unroll
            for (int b = 0; b < NV; ++b)
#pragma unroll
                for (int d = 0; d < ND; ++d) vf[b][d] = *reinterpret_cast<const V*>(vb + (b * ND + d) * BLK);
            mfma_f32x4 sc[2];
            float mx = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                mfma_f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < NK; ++s) x = Piece<T>::mul(kf[b][s], qf[s], x);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] *= a.scale;
                    if (p + 32 > all && p + b * 16 + fc * 4 + r >= lim) x[r] = -INFINITY;
                    mx = fmaxf(mx, x[r]);
                }
                sc[b] = x;
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float mn = fmaxf(m, mx);
            const float mu = mn == -INFINITY ? 0.f : mn;  // a row that has seen nothing, or only -inf
            if (__any(mn > m)) {
                const float alpha = exp2_softmax(m - mu);
                l *= alpha;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[d][r] *= alpha;
                m = mn;
            }
            {
#pragma clang fp contract(off)  // mu is a rounded product, and so is what it is taken from
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        sc[b][r] = exp2_softmax(sc[b][r] - mu);
                        l += sc[b][r];
                    }
            }
            V pf[NV], pl;
            if constexpr (TWO) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const __bf16 w = (__bf16)sc[b][r];
                        pf[0][b * 4 + r] = w;
                        pl[b * 4 + r] = (__bf16)(sc[b][r] - (float)w);
                    }
            } else {
                pf[0] = sc[0];
                pf[1] = sc[1];
            }
            // adds what the weights' rounding left, times a fragment: with an infinite
            // value, which the weights make infinite already, that says nothing
            auto add_left = [&](const V& y, mfma_f32x4& x) __attribute__((always_inline)) {
                if constexpr (TWO) {
                    if (!check) {
                        x = Piece<T>::mul(y, pl, x);
                    } else {
                        const mfma_f32x4 z = Piece<T>::mul(y, pl, mfma_f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[r] += fabsf(z[r]) < INFINITY ? z[r] : 0.f;
                    }
                }
            };
            // position of element e of a value fragment
            auto vpos = [&](int b, int e) { return p + fc * 4 + (sizeof(T) == 2 ? (e & 3) + (e >> 2) * 16 : b * 16 + e); };
            bool by_row = false;
            if (check && p + 32 > all) {
                bool odd = false;
#pragma unroll
                for (int b = 0; b < NV; ++b)
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int e = 0; e < EL; ++e) {
                            if (vpos(b, e) >= t.kv1) vf[b][d][e] = 0.f;
                            odd = odd || !(fabsf((float)vf[b][d][e]) < INFINITY);
                        }
                by_row = __any(odd);
            }
            if (!by_row) {
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    add_left(vf[0][d], o[d]);
#pragma unroll
                    for (int b = 0; b < NV; ++b) o[d] = Piece<T>::mul(vf[b][d], pf[b], o[d]);
                }
            } else {
#pragma unroll 1
                for (int r = 0; r < 16; ++r) {
                    const int lr = __shfl(lim, r, 64);
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        mfma_f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int b = 0; b < NV; ++b) {
                            V y = vf[b][d];
#pragma unroll
                            for (int e = 0; e < EL; ++e)
                                if (vpos(b, e) >= lr) y[e] = 0.f;
                            add_left(y, x);
                            x = Piece<T>::mul(y, pf[b], x);
                        }
                        if (fr == r) o[d] += x;
                    }
                }
            }
        }
        // the lanes of a row hold different positions' weights
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (fc == 0) {
            sm[wave][fr] = m;
            sl[wave][fr] = l;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) so[wave][fr][d * 16 + fc * 4 + r] = o[d][r];
        __syncthreads();
        // thread: row tid / 16, dims 4 (tid % 16) .. + 3 (and 64 further on)
        const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * 4;
        if (t.j0 + row < rows) {
        const float mt = fmaxf(fmaxf(sm[0][row], sm[1][row]), fmaxf(sm[2][row], sm[3][row]));
        const float mu = mt == -INFINITY ? 0.f : mt;
        float w[4], lt = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = exp2_softmax(sm[i][row] - mu);
            lt += sl[i][row] * w[i];
        }
#pragma unroll
        for (int d = d0; d < D; d += 64) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = so[0][row][d + e] * w[0] + so[1][row][d + e] * w[1] + so[2][row][d + e] * w[2] + so[3][row][d + e] * w[3];
            if (t.part < 0) {
                const int jr = t.j0 + row, tk = jr / a.G, gg = jr - tk * a.G;
                const float inv = lt == 0.f ? 0.f : 1.0f / lt;
                attn_store<T, FRAG>(a, t.tok0 + tk, h * a.G + gg, D, d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
            } else {
                float* ps = a.parts + ((long long)t.part * a.c.Hkv + h) * (16 * (D + 2)) + row * D + d;
                st4(ps, x[0], x[1], x[2], x[3]);
            }
        }
        if (t.part >= 0 && (threadIdx.x & 15) == 0) {
            float* ps = a.parts + ((long long)t.part * a.c.Hkv + h) * (16 * (D + 2)) + 16 * D;
            ps[row] = mt;
            ps[16 + row] = lt;
        }
        }
        __syncthreads();  // the next item's LDS
    }
}

// Joins the parts of cut ranges: one workgroup per 16 rows and kv head. Four
// lanes take a row of a part; where there are fewer than 16 rows the other
// lanes take further parts, up to 64 at a time. Parts are weighted by the largest
// maximum of all of them; the lanes' sums are added in order. Bound by the
// latency of reading what other workgroups wrote: 47 parts of 4 rows 7 us (29
// with four parts at a time).
template <class T, int D, bool FRAG>
__global__ __launch_bounds__(256) void paged_merge_kernel(AttnArgs a) {
    constexpr int N = D / 16;  // 16-byte pieces of a lane
    __shared__ float so[64][D + 4];
    __shared__ float sl[64], sm[64];
    const ListHead head = *reinterpret_cast<const ListHead*>(a.plan);
    const MergeItem* merges = reinterpret_cast<const MergeItem*>(a.plan + head.merges_at);
    const int quad = threadIdx.x >> 2, q4 = threadIdx.x & 3;
    for (int w0 = blockIdx.x; w0 < head.merges * a.c.Hkv; w0 += gridDim.x) {
        const int it = w0 / a.c.Hkv, h = w0 - it * a.c.Hkv;
        const MergeItem t = merges[it];
        const int rows = min(16, t.count * a.G - t.j0);
        const int lg = rows > 8 ? 4 : rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0;  // rows, rounded up to a power of two
        const int row = quad & ((1 << lg) - 1), first = quad >> lg, stride = 64 >> lg;
        const bool live = row < rows;
        const long long step = (long long)t.step * a.c.Hkv * (16 * (D + 2));
        const float* ps = a.parts + ((long long)t.part * a.c.Hkv + h) * (16 * (D + 2));
        // the largest maximum: a quad's lanes take its parts in turn
        float m = -INFINITY;
        for (int i = first + q4 * stride; i < t.n; i += 4 * stride) m = fmaxf(m, live ? ps[i * step + 16 * D + row] : -INFINITY);
        m = fmaxf(m, __shfl_xor(m, 1, 64));
        m = fmaxf(m, __shfl_xor(m, 2, 64));
        if (q4 == 0) sm[quad] = m;
        __syncthreads();
        for (int i = row; i < 64; i += 1 << lg) m = fmaxf(m, sm[i]);
        const float mu = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        mfma_f32x4 x[N];
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        if (live) {
#pragma unroll 2
            for (int i = first; i < t.n; i += stride) {
                const float* p = ps + i * step;
                const float w = exp2_softmax(p[16 * D + row] - mu);
                l += w * p[16 * D + 16 + row];
#pragma unroll
                for (int c = 0; c < N; ++c) x[c] += w * *reinterpret_cast<const mfma_f32x4*>(p + row * D + (c * 4 + q4) * 4);
            }
        }
        if (q4 == 0) sl[quad] = l;
#pragma unroll
        for (int c = 0; c < N; ++c) *reinterpret_cast<mfma_f32x4*>(&so[quad][(c * 4 + q4) * 4]) = x[c];
        __syncthreads();
        for (int i = threadIdx.x; i < rows * (D / 4); i += 256) {
            const int r = i / (D / 4), d = (i - r * (D / 4)) * 4;
            mfma_f32x4 y{0.f, 0.f, 0.f, 0.f};
            float lt = 0.f;
            for (int k = r; k < 64; k += 1 << lg) {
                y += *reinterpret_cast<const mfma_f32x4*>(&so[k][d]);
                lt += sl[k];
            }
            const float inv = lt == 0.f ? 0.f : 1.0f / lt;
            const int j = t.j0 + r, tk = j / a.G, gg = j - tk * a.G;
            attn_store<T, FRAG>(a, t.tok0 + tk, h * a.G + gg, D, d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
        }
        __syncthreads();  // the next item's LDS
    }
}

// ------------------------------------------------------------------ attention of many rows (bf16)
//
// 128 rows per workgroup, 32 per wave in two tiles of 16, and blocks of 64
// positions that all waves read from LDS: two or three buffers, filled by direct global->LDS loads of whole 1 KiB fragments, so that every
// LDS access is a linear 16 bytes per lane. Two waves share a SIMD: the matrix
// products of one run beside the other's softmax. A row's reference moves only
// when a score is more than 2^8 above it, so the sums are rescaled rarely.
// Scores, maxima, sums and outputs are fp32; the weights enter the product with
// the values rounded to bf16 (2^-8 of each at most), their sum does not. As two
// bf16 numbers, as above, they would take half as many products again: 569 instead
// of 436 us for the 4096 tokens below, 39 instead of 30 for the nine prompts.
// Bound by the matrix cores, the issue of the softmax beside them and LDS reads
// (a fragment serves two products): 4096 tokens over 4097 positions, 32 / 8 heads
// of 128, 436 us (946 TFLOP/s; the 16-row kernel 967 us) at full clocks, up to 540
// in the first launches after a pause. Few prompts are bound by a workgroup's
// chain of blocks: 4.6 us and 1.15 per block, alone on its CU. 256 rows per workgroup take 448 instead of 466 us there, but 51
// instead of 34 for nine prompts of up to 513 tokens, which then give fewer
// workgroups than CUs; 64 rows per wave at head size 128 leave one wave a SIMD
// and took 1040.
// An item's rows may be fewer than 128 (its waves and tiles without rows do
// nothing but help loading) and its positions a part of a cut range; slot
// part + i then holds the i-th 16 rows.
__device__ __forceinline__ void load_to_lds(const bf16* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds(src, dst, 16, 0, 0);
}
constexpr int BIG_ROWS = 128;
constexpr int BIG_TILES = 2;  // tiles of 16 rows per wave
constexpr int BIG_THREADS = BIG_ROWS / 16 / BIG_TILES * 64;
template <int D>
__global__ __launch_bounds__(BIG_THREADS, 2) void paged_attn_big_kernel(AttnArgs a) {
    typedef mfma_bf16x8 V;
    constexpr int NK = D / 32, ND = D / 16, UT = BIG_TILES, NW = BIG_THREADS / 64;
    constexpr int HALF = 64 * D;           // bytes of the keys, or of the values, of 32 positions
    constexpr int TILE = 4 * HALF;         // a block: keys, keys, values, values
    constexpr int NB = D == 64 ? 3 : 2;    // buffers: two workgroups per CU at least
    __shared__ __align__(16) unsigned char lds[NB * TILE];
    const ListHead head = *reinterpret_cast<const ListHead*>(a.plan);
    const AttnItem* items = reinterpret_cast<const AttnItem*>(a.plan + head.bigs_at);
    const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pmask = (1 << a.c.shift) - 1;
    const bool check = a.c.may_be_odd();
    for (int w0 = blockIdx.x; w0 < head.bigs * a.c.Hkv; w0 += gridDim.x) {
        const int it = w0 / a.c.Hkv, h = w0 - it * a.c.Hkv;
        const AttnItem t = items[it];
        const int rows = t.count * a.G;
        const int r0 = t.j0 + wave * 16 * UT;
        const int nu = min(UT, max(0, (min(rows, t.j0 + BIG_ROWS) - r0 + 15) / 16));  // this wave's tiles
        int lim[UT];  // positions of the range that the lane's row of each tile sees
        V qf[UT][NK];
#pragma unroll
        for (int u = 0; u < UT; ++u) {
            const int j = min(r0 + u * 16 + fr, rows - 1), tok = j / a.G, g = j - tok * a.G;
            lim[u] = min(t.past + tok + 1, t.kv1);
            const bf16* q = static_cast<const bf16*>(a.q) + (long long)(t.tok0 + tok) * a.q_ld + (h * a.G + g) * D + fc * 8;
#pragma unroll
            for (int s = 0; s < NK; ++s) qf[u][s] = *reinterpret_cast<const V*>(q + s * 32);
        }
        // positions that every row of the wave sees, and the last one does (a wave without rows: none)
        const int all = nu ? t.past + r0 / a.G + 1 : 0;
        const int end = nu ? min(t.kv1, t.past + (min(r0 + 16 * UT, rows) - 1) / a.G + 1) : 0;
        mfma_f32x4 o[ND][UT];
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int u = 0; u < UT; ++u) o[d][u] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        float m[UT], l[UT];
#pragma unroll
        for (int u = 0; u < UT; ++u) {
            m[u] = -INFINITY;
            l[u] = 0.f;
        }
        // positions p .. p + 63 into buffer b: a quarter of the waves load each
        // of the halves' keys and values. A half behind the range's last block of
        // 32 loads that block again (its scores are masked).
        const int* table = a.c.table + (long long)t.seq * a.c.ld;
        const int last = (t.kv1 - 1) & ~31;
        constexpr int WP = NW / 4, N = HALF / 1024 / WP;  // waves per quarter, loads per wave
        const int part = wave / WP, sub = wave % WP;
        auto place = [&](int p) __attribute__((always_inline)) { return min(p + (part & 1) * 32, last); };
        auto issue = [&](int p, int page, int b) __attribute__((always_inline)) {
            const int pp = place(p);
            const bf16* src = a.c.template head<bf16>(page, a.layer, part >> 1, h) +
                              ((pp & pmask) >> 5) * (HALF / 2) + sub * N * 512 + lane * 8;
            unsigned char* dst = lds + b * TILE + part * HALF + sub * N * 1024;
#pragma unroll
            for (int i = 0; i < N; ++i) load_to_lds(src + i * 512, dst + i * 1024);
        };
        // One block of 64 positions from LDS. MASKED: not every row sees all of
        // them. ODD: values may be anything; behind the range they count as 0,
        // and so do those that are not finite: 0 * inf would reach rows that do
        // not see them (what they are to the others is added at the end).
        bool odd = false;
        auto block = [&](auto is_masked, auto is_odd, int p, const unsigned char* tk) __attribute__((always_inline)) {
            constexpr bool MASKED = decltype(is_masked)::value, ODD = decltype(is_odd)::value;
            const unsigned char* tv = tk + 2 * HALF;
            mfma_f32x4 sc[UT][4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                V kf[NK];
#pragma unroll
                for (int s = 0; s < NK; ++s) kf[s] = *reinterpret_cast<const V*>(tk + (b * NK + s) * 1024);
#pragma unroll
                for (int u = 0; u < UT; ++u) {
                    mfma_f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < NK; ++s) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[s], qf[u][s], x, 0, 0, 0);
                    if constexpr (MASKED) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (b * 16 + r >= lim[u] - p - fc * 4) x[r] = -INFINITY;
                    }
                    sc[u][b] = x;
                }
            }
            V pf[UT][2];
#pragma unroll
            for (int u = 0; u < UT; ++u) {
                mfma_f32x4 (&cur)[4] = sc[u];
                float mx = cur[0][0];
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, cur[b][r]);
                mx *= a.scale;
                if (__any(mx > m[u] + 8.f)) {  // (m starts at -inf)
                    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    const float mn = mx > m[u] + 8.f ? mx : m[u];
                    const float alpha = mn == m[u] ? 1.f : exp2_softmax(m[u] - mn);
                    m[u] = mn;
                    l[u] *= alpha;
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[d][u][r] *= alpha;
                }
                const float mu = m[u] == -INFINITY ? 0.f : m[u];  // a row that has seen nothing, or only -inf
                // m is a rounded product: the exact one exceeds it by up to 2^-24 |m|,
                // which is an exponent. Harmless below 2^30 (all of a row's weights
                // have it alike); above, products are rounded before m is taken off.
                float scale = a.scale;
                if (__any(fabsf(mu) >= 0x1p30f)) {
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r) cur[b][r] *= a.scale;
                    scale = 1.f;
                }
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        cur[b][r] = exp2_softmax(fmaf(cur[b][r], scale, -mu));
                        l[u] += cur[b][r];
                    }
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        pf[u][s][r] = (__bf16)cur[2 * s][r];
                        pf[u][s][4 + r] = (__bf16)cur[2 * s + 1][r];
                    }
            }
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    V vf = *reinterpret_cast<const V*>(tv + (s * ND + d) * 1024);
                    if constexpr (ODD) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const bool in = s * 32 + (e & 3) + (e >> 2) * 16 < t.kv1 - p - fc * 4;
                            const bool fin = fabsf((float)vf[e]) < INFINITY;
                            odd = odd || (in && !fin);
                            if (!in || !fin) vf[e] = 0.f;
                        }
                    }
#pragma unroll
                    for (int u = 0; u < UT; ++u)
                        o[d][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][s], o[d][u], 0, 0, 0);
                }
        };
        int buf = 0;
        auto page_of = [&](int p) __attribute__((always_inline)) { return list_at(table, place(p) >> a.c.shift); };
        constexpr int AHEAD = (NB - 1) * 64;
#pragma unroll
        for (int i = 0; i < NB - 1; ++i)
            if (t.kv0 + 64 * i < t.kv1) issue(t.kv0 + 64 * i, page_of(t.kv0 + 64 * i), i);
        int page = page_of(t.kv0 + AHEAD);  // of the block that is issued next
        for (int p = t.kv0; p < t.kv1; p += 64) {
            // this block is in LDS (the later ones' loads may be on their way), and
            // every wave is done with the one before; no read moves across
            __builtin_amdgcn_sched_barrier(0);
            if (NB == 3 && p + 64 < t.kv1) __builtin_amdgcn_s_waitcnt(WMI_VMCNT_LDS(N));
            else __builtin_amdgcn_s_waitcnt(WMI_VMCNT_LDS(0));
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            if (p + AHEAD < t.kv1) {
                issue(p + AHEAD, page, buf == 0 ? NB - 1 : buf - 1);
                page = page_of(p + 64 + AHEAD);
            }
            const unsigned char* tk = lds + buf * TILE + lane * 16;
            buf = buf + 1 == NB ? 0 : buf + 1;
            if (p + 64 <= all && p + 64 <= t.kv1) block(std::false_type{}, std::false_type{}, p, tk);
            else if (p < end && !check) block(std::true_type{}, std::false_type{}, p, tk);
            else if (p < end) block(std::true_type{}, std::true_type{}, p, tk);
        }
        // values of masked blocks that are not finite: what they add to the rows
        // that see them, inf, -inf or NaN, by products of indicators
        if (__any(odd)) {
#pragma unroll 1
            for (int p = max(t.kv0, (min(all, t.kv1) & ~63) - 64); p < end; p += 32) {
                // (a block is masked or not as a whole; its blocks begin at kv0)
                const int b0 = t.kv0 + ((p - t.kv0) & ~63);
                if (b0 + 64 <= all && b0 + 64 <= t.kv1) continue;
                const bf16* vb = a.c.template head<bf16>(table[p >> a.c.shift], a.layer, 1, h) + ((p & pmask) >> 5) * (HALF / 2) + lane * 8;
#pragma unroll 1
                for (int kind = 0; kind < 3; ++kind) {
                    const float what = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const V vf = *reinterpret_cast<const V*>(vb + d * 512);
                        V is;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float y = (float)vf[e];
                            is[e] = (__bf16)((kind == 2 ? y != y : y == what) ? 1.f : 0.f);
                        }
#pragma unroll
                        for (int u = 0; u < UT; ++u) {
                            V seen;
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                seen[e] = (__bf16)((e & 3) + (e >> 2) * 16 < lim[u] - p - fc * 4 ? 1.f : 0.f);
                            const mfma_f32x4 x =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(is, seen, mfma_f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 4; ++r) o[d][u][r] += x[r] > 0.f ? what : 0.f;
                        }
                    }
                }
            }
        }
        // lane: O^T[dim d * 16 + fc * 4 + r][row r0 + u * 16 + fr]
#pragma unroll
        for (int u = 0; u < UT; ++u) {
            float lt = l[u];
            lt += __shfl_xor(lt, 16, 64);
            lt += __shfl_xor(lt, 32, 64);
            const int j = r0 + u * 16 + fr;
            if (u >= nu || j >= rows) continue;
            if (t.part < 0) {
                const int tk = j / a.G, gg = j - tk * a.G;
                const float inv = lt == 0.f ? 0.f : 1.0f / lt;
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    attn_store<bf16, false>(a, t.tok0 + tk, h * a.G + gg, D, d * 16 + fc * 4, o[d][u][0] * inv, o[d][u][1] * inv,
                                            o[d][u][2] * inv, o[d][u][3] * inv);
            } else {
                float* ps = a.parts + ((long long)(t.part + wave * UT + u) * a.c.Hkv + h) * (16 * (D + 2));
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    st4(ps + fr * D + d * 16 + fc * 4, o[d][u][0], o[d][u][1], o[d][u][2], o[d][u][3]);
                if (fc == 0) {
                    ps[16 * D + fr] = m[u];
                    ps[16 * D + 16 + fr] = lt;
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(WMI_VMCNT_LDS(0));
        __syncthreads();  // the next item's LDS
    }
}

// A decode step's plan, made on the device: one item per row, of the slot
// list[r] at its position pos[list[r]].
static __global__ __launch_bounds__(128) void paged_rows_kernel(const int* __restrict__ list,
                                                                const int* __restrict__ pos, int n,
                                                                int* __restrict__ plan) {
    const int r = threadIdx.x;
    if (r == 0) *reinterpret_cast<ListHead*>(plan) = ListHead{n, 0, 0, 0, 0, 0, 0, 0};
    if (r < n) {
        const int s = list[r], p = pos[s];
        reinterpret_cast<AttnItem*>(plan + HEAD_INTS)[r] = AttnItem{s, p, 1, r, 0, 0, p + 1, -1};
    }
}

}  // namespace wmi
