// Kernels of a packed key/value cache: keys and values in 8 or 4 bits, in
// pages as paged.h has them. Appending quantises, reading gives back what the
// codes stand for, and attention works on the codes.
//
// 64 numbers of a position's head row form a group. With lo and hi their least
// and largest, 0 included,
//   step = the smallest number with 4 (8 bits: 1) significant bits that is at
//          least (hi - lo) / 15 (255), and at least 2^-100
//   zero = round(-lo / step),  code = round(x / step) + zero, in 0 .. 15 (255)
// (halves to even), and the value is (code - zero) * step: at most half a step
// off. Few bits in the step make that product exact: 4 bits times 4, or 8 times 1,
// fit a bf16 number, so all kernels see the same values and nothing is rounded
// after the quantiser. A group with a number that is not below 2^125 in
// magnitude holds NaN throughout. Step and zero take 2 bytes a group:
//   4 bits: the step as bf16, whose low 4 bits are free, with zero in them
//   8 bits: the step's exponent in the high byte, zero in the low one
// so a number takes 4.25 or 8.25 bits. A step of any 8 bits would be 3 % finer on
// average in 4 bits, but its values would need 12 bits and be rounded in bf16. (In 8
// bits a step of one bit is up to twice what the range needs, 1.44 times on average
// over ranges of all sizes: half a bit of the 8.)
//
// Memory: pages [page][layer][K, V][kv head], each head P * D codes and behind
// them the groups' words [D / 64][P]. The codes are in the order in which
// matrix instructions take the unpacked numbers (dec_off, val_off), 16 bytes per
// lane:
//   keys    a lane's 8 dims of one position are 4 (8) consecutive bytes; in 4
//           bits element e is nibble e / 2 + 4 (e % 2), so that the elements of a
//           pair are 16 bits apart;
//   values  a lane's 16 bytes are 8 positions of 4 (8 bits: 2) dims that are 16
//           apart; a position's dims are the nibbles (bytes) of one half word, so
//           that a single position is written without reading its neighbours.
#pragma once

#include "paged.h"

namespace wmi {

constexpr int GROUP = 64;
// Attention adds up weighted codes before it divides by the weights: numbers of up to
// 143 steps in 4 bits (128 + 15), 255 in 8, for each of up to 2^24 positions, in the
// kernel of many rows up to 2^8 times that. From steps of 2^80 on, fp32 might not hold
// such sums (a step is below 2^123). Once values with such a step have been appended
// to a cache, its attention multiplies all weights, or unpacked values, by SHRINK,
// 2^-36, so that a sum is below 2^122; the division takes it back. Products with
// steps below 2^-50 or so then lose bits, among values of 2^80 and more.
// (Other caches run the code they would run without it: a loop of its own in the
// kernel of 4 rows, where a branch in the loop took 7.38 instead of 7.19 us for 32 tokens
// over 447 positions at most; in that of 16 rows a branch, 13.8 us for 16 drafts of 5
// tokens either way, where a second loop takes 17 to 54 registers more.)
constexpr float LARGE_STEP = 0x1p80f;

// Bytes of a head's codes and of all it holds.
template <int BITS> constexpr int packed_codes(int P, int D) { return P * D * BITS / 8; }
inline long long packed_head(int P, int D, int bits) { return (long long)P * D * bits / 8 + P * (D / GROUP) * 2; }

// Byte offset of the piece of 8 dims from d on of a position's keys.
template <int BITS>
__device__ __forceinline__ int pkey_off(int p, int d, int D) {
    constexpr int PER = 32 / (BITS * 2);  // fragments of 16 positions x 32 dims per 1 KiB
    const int i = (p >> 4) * (D >> 5) + (d >> 5), lane = ((d >> 3) & 3) * 16 + (p & 15);
    return (i / PER) * 1024 + lane * 16 + (i % PER) * BITS;
}
// Byte offset of the half word that holds dim d of a position's values.
template <int BITS>
__device__ __forceinline__ int pval_off(int p, int d, int D) {
    constexpr int DIMS = 256 / BITS;  // of 1 KiB: 64 or 32, of 32 positions
    return ((p >> 5) * (D / DIMS) + d / DIMS) * 1024 + (((p >> 2) & 3) * 16 + (d & 15)) * 16 +
           ((p & 3) + ((p & 16) >> 2)) * 2;
}

// Step and zero from a group's word. A group of NaN has code and zero 0 throughout
// and NaN, or (8 bits) +inf, as its step: 0 times either is NaN.
template <int BITS>
__device__ __forceinline__ float group_step(unsigned w) {
    return __uint_as_float(BITS == 4 ? (w & 0x7ff0u) << 16 : (w & 0xff00u) << 15);
}
template <int BITS>
__device__ __forceinline__ float group_zero(unsigned w) {
    return (float)(w & (BITS == 4 ? 15u : 255u));
}

// The range of a group, 0 included, and the bits of its largest magnitude (NaN's
// among them).
struct Range {
    float lo = 0.f, hi = 0.f;
    unsigned big = 0;
    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            lo = fminf(lo, x[e]);
            hi = fmaxf(hi, x[e]);
            big = max(big, __float_as_uint(x[e]) & 0x7fffffffu);
        }
    }
    // with that of the lane `st` away
    __device__ __forceinline__ void join(int st) {
        lo = fminf(lo, __shfl_xor(lo, st, 64));
        hi = fmaxf(hi, __shfl_xor(hi, st, 64));
        big = max(big, (unsigned)__shfl_xor((int)big, st, 64));
    }
};

// A group's quantiser. Quotients are rounded to fp32 before they are rounded to
// integers: the step has so few bits that no quotient of a 24-bit number comes to
// lie on a half, or on a step, by that. Division by a step of one bit is a product.
// By one of four it is a product with the rounded reciprocal, and its remainder
// times that again, which gives the rounded quotient (Markstein's theorem on
// division by fused multiply-add).
template <int BITS>
struct Quantiser {
    static constexpr unsigned TOP = BITS == 4 ? 15 : 255, LOW = BITS == 4 ? 0xfffffu : 0x7fffffu;
    float step, inv;
    int shift;
    unsigned word;
    bool bad;
    __device__ __forceinline__ explicit Quantiser(const Range& r) {
        bad = r.big >= 0x7e000000u;  // 2^125
        step = fmaxf(__uint_as_float((__float_as_uint((r.hi - r.lo) / (float)TOP) + LOW) & ~LOW), 0x1p-100f);
        inv = 1.f / step;
        const float zero = rintf(quotient(-r.lo));
        shift = (int)zero - 0x4b400000;
        if constexpr (BITS == 4) word = bad ? 0x7ff0u : (__float_as_uint(step) >> 16) | (unsigned)zero;
        else word = bad ? 0xff00u : (__float_as_uint(step) >> 23) << 8 | (unsigned)zero;
    }
    __device__ __forceinline__ bool large() const { return step >= LARGE_STEP && !bad; }
    __device__ __forceinline__ float quotient(float x) const {
        const float t = x * inv;
        return BITS == 8 ? t : fmaf(fmaf(-t, step, x), inv, t);
    }
    __device__ __forceinline__ unsigned code(float x) const {
        const int n = __float_as_int(quotient(x) + 12582912.f) + shift;  // (the sum with 1.5 2^23 rounds to an integer)
        return bad ? 0 : min(max(n, 0), (int)TOP);
    }
};

// The codes of 8 numbers of a group whose other numbers are those of the
// lanes beside this one (8 lanes at a multiple of 8); returns the group's word.
template <int BITS>
__device__ __forceinline__ unsigned quantise(const float (&x)[8], unsigned (&code)[8], bool& odd, bool& large) {
    Range r;
    r.add(x);
#pragma unroll
    for (int st = 1; st < 8; st <<= 1) r.join(st);
    const Quantiser<BITS> q(r);
#pragma unroll
    for (int e = 0; e < 8; ++e) code[e] = q.code(x[e]);
    odd = odd || q.bad;
    large = large || q.large();
    return q.word;
}

// A group's values as the half words that hold a position's dims (lane j of 8
// lanes): in 4 bits those of dims 2 j and 2 j + 1 (and 16, 32 and 48 further on),
// in 8 those of dims 32 (j / 4) + 4 (j % 4) .. + 3 (and 16 further on).
template <int BITS>
__device__ __forceinline__ void value_halves(const unsigned (&code)[8], int lane, unsigned (&half)[BITS / 2]) {
    const int j = lane & 7, team = lane & ~7;
    if constexpr (BITS == 4) {
        unsigned w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= code[e] << (4 * e);
        half[0] = half[1] = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const unsigned v = (unsigned)__shfl((int)w, team + (j >> 2) + 2 * t, 64) >> (8 * (j & 3));
            half[0] |= (v & 15u) << (4 * t);
            half[1] |= (v >> 4 & 15u) << (4 * t);
        }
    } else {
        const unsigned w0 = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
        const unsigned w1 = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
        unsigned v[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int from = team + (j & 4) + ((j & 3) >> 1) + 2 * t;
            const unsigned a = __shfl((int)w0, from, 64), b = __shfl((int)w1, from, 64);
            v[t] = j & 1 ? b : a;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) half[i] = (v[0] >> (8 * i) & 255u) | (v[1] >> (8 * i) & 255u) << 8;
    }
}
// Dim, in its group, of half word i of lane j.
template <int BITS>
__device__ __forceinline__ int half_dim(int lane, int i) {
    const int j = lane & 7;
    return BITS == 4 ? 2 * j + i : (j >> 2) * 32 + (j & 3) * 4 + i;
}
// Keys' codes as they are held: 8 nibbles, or 4 bytes from e on.
__device__ __forceinline__ unsigned key_word(const unsigned (&q)[8]) {
    unsigned w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= q[e] << ((e >> 1) * 4 + (e & 1) * 16);
    return w;
}
__device__ __forceinline__ unsigned four(const unsigned (&q)[8], int e) {
    return q[e] | q[e + 1] << 8 | q[e + 2] << 16 | q[e + 3] << 24;
}
template <int BITS>
__device__ __forceinline__ void store_key(unsigned char* dst, const unsigned (&q)[8]) {
    if constexpr (BITS == 4) *reinterpret_cast<unsigned*>(dst) = key_word(q);
    else *reinterpret_cast<u32x2*>(dst) = u32x2{four(q, 0), four(q, 4)};
}

// Eight numbers of a row, or into one.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    if constexpr (VEC && sizeof(T) == 2) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? a[e >> 1] & 0xffff0000u : a[e >> 1] << 16);
    } else if constexpr (VEC) {
        const float4 a = ld4(p), b = ld4(p + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = ldf(p + e);
    }
}
template <class T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    if constexpr (VEC && sizeof(T) == 2) {
        *reinterpret_cast<u32x4*>(p) =
            u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    } else if constexpr (VEC) {
        st4(p, x[0], x[1], x[2], x[3]);
        st4(p + 4, x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) stf(p + e, x[e]);
    }
}

// What the lane 1, 2 or 4 away holds (within 8 lanes): lane permutations of the
// vector unit itself.
template <int ST>
__device__ __forceinline__ unsigned lane_xor(unsigned v) {
    if constexpr (ST == 1) return __builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true);
    else if constexpr (ST == 2) return __builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true);
    else return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);  // 7, then 3
}
// Eight lanes' eight half words, transposed: half word e of lane j becomes half
// word j of lane e. Three exchanges with the lanes 1, 2 and 4 away.
__device__ __forceinline__ void transpose8(u32x4& w, int lane) {
    const unsigned sel = lane & 1 ? 0x03020706u : 0x05040100u;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(lane_xor<1>(w[i]), w[i], sel);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const unsigned got = lane_xor<2>(lane & 2 ? w[i] : w[i + 1]);
        w[i] = lane & 2 ? got : w[i];
        w[i + 1] = lane & 2 ? w[i + 1] : got;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned got = lane_xor<4>(lane & 4 ? w[i] : w[i + 2]);
        w[i] = lane & 4 ? got : w[i];
        w[i + 2] = lane & 4 ? w[i + 2] : got;
    }
}

// ------------------------------------------------------------------ rows in and out
//
// A wave per (tile, keys or values, head) and layer goes through the tile's block of
// 32 positions in units of 64 dims (values) or two groups a lane (keys), entirely
// in registers: a lane holds 32 numbers.
//   keys    lane (position % 16, c): dims 8 c .. + 7 of each 32, its 16 bytes of
//           the page; a group's numbers are 16 of four lanes (16 apart);
//   values  lane (position, half): dims 8 half .. + 7 of each 16 of a group's 64,
//           which two lanes (8 apart) share; the half words that hold a
//           position's dims are transposed over 8 lanes, to or from the page's
//           pieces of 8 positions.
// Workgroups are dealt to the 8 XCDs in turn; place_of_group gives those of one
// XCD consecutive work, so that rows of neighbouring heads meet in its L2 and
// reach memory together (grids are multiples of 8).
// Bound by memory, in rows and pages of 64-byte segments: 40 sequences of 62 positions,
// 32 layers, 20 heads of 64 in 4 bits are read out in 111 us (406 MB written; 4.6 TB/s
// read and written; 121 to 160 with nontemporal stores, with keys and values in one
// wave, or persistent and reading ahead); up to 224 new tokens of 16 sequences, 12
// layers, 12 heads of 64 are appended in 28 us (41 through LDS, a workgroup per tile).
__device__ __forceinline__ unsigned place_of_group() { return (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3); }
// Position, in its block of 32, and dims of a lane of the values:
__device__ __forceinline__ int value_row(int lane) { return (lane >> 4) * 4 + (lane & 3) + (lane & 4) * 4; }
__device__ __forceinline__ int value_dim(int lane, int i) { return i * 16 + (lane & 8); }
// Words of a lane's key piece i (of 8 dims): its position in the block and its dim.
// Unit n of a head's 32 positions: in D = 64 the one, in 128 the n-th 16 positions.
template <int D>
__device__ __forceinline__ int key_row(int n, int i, int lane) { return (D == 64 ? i / 2 : n) * 16 + (lane & 15); }
template <int D>
__device__ __forceinline__ int key_dim(int i, int lane) { return (D == 64 ? i & 1 : i) * 32 + (lane >> 4) * 8; }

template <class T, int D, int BITS, bool VEC>
__global__ __launch_bounds__(256) void packed_append_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                            const T* __restrict__ k, const T* __restrict__ v,
                                                            long long k_ld, long long v_ld, long long k_layer,
                                                            long long v_layer, int n_layers) {
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int lane = threadIdx.x & 63, P = 1 << c.shift;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned all = 2u * head.tiles * c.Hkv;  // (tile, keys or values, head) of a layer; less than 2^30
    for (long long u0 = place_of_group() * 4LL + wave; u0 < (long long)all * n_layers; u0 += gridDim.x * 4LL) {
        const int z = u0 >> 32 ? (int)(u0 / all) : (int)((unsigned)u0 / all), layer = layer0 + z;
        const unsigned w = (unsigned)(u0 - (long long)z * all);
        const unsigned wt = w / c.Hkv;
        const int h = w - wt * c.Hkv, kv = wt & 1;
        const PageTile t = tiles[wt >> 1];
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        const int b0 = t.pos & (P - 1) & ~31, lo = t.pos & 31, hi = lo + t.n;  // the block, and its new positions
        const long long ld = kv ? v_ld : k_ld;
        const T* src = (kv ? v + z * v_layer : k + z * k_layer) + t.row * ld + h * D;
        unsigned char* dst = c.head<unsigned char>(page, layer, kv, h);
        unsigned short* words = reinterpret_cast<unsigned short*>(dst + packed_codes<BITS>(P, D)) + b0;
        // a position's row in the caller's; of positions that are not new, the first or last new one's
        auto row = [&](int p) __attribute__((always_inline)) { return src + (min(max(p, lo), hi - 1) - lo) * ld; };
        auto is_new = [&](int p) __attribute__((always_inline)) { return p >= lo && p < hi; };
        bool odd = false, large = false;
#pragma unroll 1
        for (int n = 0; n < D / 64; ++n) {
            float x[4][8];
            if (kv == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) load8<T, VEC>(row(key_row<D>(n, i, lane)) + key_dim<D>(i, lane), x[i]);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int p = key_row<D>(n, 2 * u, lane), d = key_dim<D>(2 * u, lane);
                    Range r;
                    r.add(x[2 * u]);
                    r.add(x[2 * u + 1]);
                    r.join(16);
                    r.join(32);
                    const Quantiser<BITS> q(r);
                    unsigned code[2][8];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 8; ++e) code[i][e] = q.code(x[2 * u + i][e]);
                    if (!is_new(p)) continue;
                    odd = odd || q.bad;
                    unsigned char* to = dst + pkey_off<BITS>(b0 + p, d, D);  // (the second piece is right behind)
                    if constexpr (BITS == 4) {
                        *reinterpret_cast<u32x2*>(to) = u32x2{key_word(code[0]), key_word(code[1])};
                    } else {
                        *reinterpret_cast<u32x4*>(to) = u32x4{four(code[0], 0), four(code[0], 4), four(code[1], 0), four(code[1], 4)};
                    }
                    if (lane < 16) words[(d / GROUP) * P + p] = (unsigned short)q.word;
                }
            } else {
                const int p = value_row(lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) load8<T, VEC>(row(p) + n * GROUP + value_dim(lane, i), x[i]);
                Range r;
#pragma unroll
                for (int i = 0; i < 4; ++i) r.add(x[i]);
                r.join(8);
                const Quantiser<BITS> q(r);
                odd = odd || (q.bad && is_new(p));
                large = large || (q.large() && is_new(p));
                if (!(lane & 8) && is_new(p)) words[n * P + p] = (unsigned short)q.word;
                // half words of dims 8 half + j: 16 dims on in the next nibble (byte), 32 on in the next block (8 bits)
                constexpr int BLOCKS = BITS / 4, TILES = 4 / BLOCKS;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    u32x4 y;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        y[j] = 0;
#pragma unroll
                        for (int i = 0; i < TILES; ++i)
                            y[j] |= (q.code(x[b * TILES + i][2 * j]) | q.code(x[b * TILES + i][2 * j + 1]) << 16) << (BITS * i);
                    }
                    transpose8(y, lane);
                    // now the 8 positions (lane / 16) * 4 .. + 3 and 16 on of dim lane % 16
                    const int g = (lane >> 4) * 4;
                    unsigned char* to = dst + pval_off<BITS>(b0, n * GROUP + b * 32, D) + lane * 16;
                    if (g >= lo && g + 20 <= hi) {
                        *reinterpret_cast<u32x4*>(to) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (is_new(g + (e & 3) + (e >> 2) * 16))
                                reinterpret_cast<unsigned short*>(to)[e] = (unsigned short)(y[e >> 1] >> (e & 1) * 16);
                    }
                }
            }
        }
        if (c.odd && odd) *c.odd = 1;
        if (c.odd && large) c.odd[1] = 1;
    }
}

// Tiles of few rows: a row of a head's keys, or values, per D / 8 lanes, and its
// half words written one by one. (A workgroup per tile would have 8 of its 256
// lanes at work on a decode step.) Bound by the latency of the list, the page and the
// row, and by the values' half words, stores of 2 bytes that lie 16 apart: 32 tokens, 32
// layers, 20 heads of 64 take 9.1 us in 8 bits and 6.3 in 4, which have half as many of
// them for the same rows (32 with a wave per tile).
template <class T, int D, int BITS, bool VEC>
__global__ __launch_bounds__(256) void packed_append_few_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                                const T* __restrict__ k, const T* __restrict__ v,
                                                                long long k_ld, long long v_ld, long long k_layer,
                                                                long long v_layer) {
    constexpr int CH = D / 8;
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int layer = layer0 + blockIdx.z, tid = threadIdx.x, d = tid % CH * 8, P = 1 << c.shift;
    const unsigned all = 2u * head.tiles * c.Hkv;  // (tile, keys or values, head); less than 2^30
    for (unsigned w = blockIdx.x * (256u / CH) + tid / CH; w < all; w += gridDim.x * (256u / CH)) {
        const unsigned wt = w / c.Hkv;
        const int h = w - wt * c.Hkv, kv = wt & 1;
        const PageTile t = tiles[wt >> 1];
        const long long ld = kv ? v_ld : k_ld;
        const T* src = (kv ? v + blockIdx.z * v_layer : k + blockIdx.z * k_layer) + t.row * ld + h * D + d;
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        unsigned char* dst = c.head<unsigned char>(page, layer, kv, h);
        bool odd = false, large = false;
        for (int r = 0; r < t.n; ++r) {
            const int p = (t.pos & (P - 1)) + r;
            float x[8];
            unsigned q[8], half[BITS / 2];
            load8<T, VEC>(src + r * ld, x);
            const unsigned word = quantise<BITS>(x, q, odd, large);
            value_halves<BITS>(q, tid, half);
            if (kv == 0) {
                store_key<BITS>(dst + pkey_off<BITS>(p, d, D), q);
            } else {
#pragma unroll
                for (int e = 0; e < BITS / 2; ++e) {
                    const int dim = (d & ~(GROUP - 1)) + half_dim<BITS>(tid, e);
                    *reinterpret_cast<unsigned short*>(dst + pval_off<BITS>(p, dim, D)) = (unsigned short)half[e];
                }
            }
            if ((d & (GROUP - 1)) == 0)
                *reinterpret_cast<unsigned short*>(dst + packed_codes<BITS>(P, D) + ((d / GROUP) * P + p) * 2) = (unsigned short)word;
        }
        if (c.odd && odd) *c.odd = 1;
        if (c.odd && large && kv) c.odd[1] = 1;
    }
}

template <class T, int D, int BITS, bool VEC>
__global__ __launch_bounds__(256) void packed_read_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                          T* __restrict__ k, T* __restrict__ v, long long k_ld,
                                                          long long v_ld, long long k_layer, long long v_layer,
                                                          int n_layers) {
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int lane = threadIdx.x & 63, P = 1 << c.shift;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned all = 2u * head.tiles * c.Hkv;
    for (long long u0 = place_of_group() * 4LL + wave; u0 < (long long)all * n_layers; u0 += gridDim.x * 4LL) {
        const int z = u0 >> 32 ? (int)(u0 / all) : (int)((unsigned)u0 / all), layer = layer0 + z;
        const unsigned w = (unsigned)(u0 - (long long)z * all);
        const unsigned wt = w / c.Hkv;
        const int h = w - wt * c.Hkv, kv = wt & 1;
        const PageTile t = tiles[wt >> 1];
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        const int b0 = t.pos & (P - 1) & ~31, lo = t.pos & 31, hi = lo + t.n;
        const long long ld = kv ? v_ld : k_ld;
        T* dst = (kv ? v + z * v_layer : k + z * k_layer) + t.row * ld + h * D;
        const unsigned char* src = c.head<unsigned char>(page, layer, kv, h);
        const unsigned short* words = reinterpret_cast<const unsigned short*>(src + packed_codes<BITS>(P, D)) + b0;
#pragma unroll 1
        for (int n = 0; n < D / 64; ++n) {
            float x[8];
            if (kv == 0) {
                u32x4 y[BITS / 4];
#pragma unroll
                for (int i = 0; i < BITS / 4; ++i)  // (in 8 bits the second half of the positions, or dims, is 1 KiB on)
                    y[i] = *reinterpret_cast<const u32x4*>(src + (b0 / 32 * (D / 64) + n) * (BITS * 256) + i * 1024 + lane * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int p = key_row<D>(n, i, lane), d = key_dim<D>(i, lane);
                    const unsigned word = words[(d / GROUP) * P + p];
                    const float step = group_step<BITS>(word), off = -group_zero<BITS>(word) * step;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const unsigned q = BITS == 4 ? y[0][i] >> ((e >> 1) * 4 + (e & 1) * 16) & 15u
                                                     : y[i >> 1 & (BITS == 8)][(i & 1) * 2 + (e >> 2)] >> ((e & 3) * 8) & 255u;
                        x[e] = fmaf((float)q, step, off);
                    }
                    if (p >= lo && p < hi) store8<T, VEC>(dst + (p - lo) * ld + d, x);
                }
            } else {
                constexpr int BLOCKS = BITS / 4, TILES = 4 / BLOCKS;
                const int p = value_row(lane);
                const unsigned word = words[n * P + p];
                const float step = group_step<BITS>(word), off = -group_zero<BITS>(word) * step;
                u32x4 y[BLOCKS], r[4];
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
                    y[b] = *reinterpret_cast<const u32x4*>(src + pval_off<BITS>(b0, n * GROUP + b * 32, D) + lane * 16);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    transpose8(y[b], lane);
#pragma unroll
                    for (int i = 0; i < TILES; ++i) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            x[e] = fmaf((float)(y[b][e >> 1] >> ((e & 1) * 16 + i * BITS) & (BITS == 4 ? 15u : 255u)), step, off);
                        if constexpr (VEC && sizeof(T) == 2)
                            r[b * TILES + i] = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                                     pack_bf16x2(x[6], x[7])};
                        else if (p >= lo && p < hi) store8<T, VEC>(dst + (p - lo) * ld + n * GROUP + value_dim(lane, b * TILES + i), x);
                    }
                }
                if constexpr (VEC && sizeof(T) == 2) {
                    // neighbouring lanes have neighbouring rows: they swap halves, so that a
                    // store's segments are 64 bytes long instead of 32
                    const bool second = lane & 1;
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const unsigned got = lane_xor<1>(second ? r[i][j] : r[i + 1][j]);
                            r[i][j] = second ? got : r[i][j];
                            r[i + 1][j] = second ? r[i + 1][j] : got;
                        }
                        const int d = n * GROUP + value_dim(lane, i + second);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int q = (p & ~1) + j;
                            if (q >= lo && q < hi) *reinterpret_cast<u32x4*>(dst + (q - lo) * ld + d) = r[i + j];
                        }
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------ unpacked fragments
//
// Codes as matrix operands. In bf16 a nibble c under the exponent of 128 is the
// number 128 + c, one instruction for two of them; the 128 leaves with the zero,
// in sums of fp32 that are 2^4 times what they would be without it. Bytes
// become bf16 numbers by way of fp32, exactly.
template <class T, int BITS> constexpr float CODE_OFF = sizeof(T) == 2 && BITS == 4 ? 128.f : 0.f;

typedef float f32x8 __attribute__((ext_vector_type(8)));
template <class T> struct Codes;
template <> struct Codes<bf16> {
    typedef mfma_bf16x8 V;
    __device__ static __forceinline__ V load(const bf16* p) { return *reinterpret_cast<const V*>(p); }
    unsigned mask = 0x000f000fu, exponent = 0x43004300u;
    // (in vector registers, an instruction takes both; of constants it takes one)
    __device__ __forceinline__ Codes() { asm volatile("" : "+v"(mask), "+v"(exponent)); }
    __device__ __forceinline__ unsigned pair4(unsigned w) const { return (w & mask) | exponent; }
    __device__ static __forceinline__ unsigned pair8(unsigned a, unsigned b) {  // two numbers up to 255
        return __builtin_amdgcn_perm(__float_as_uint((float)b), __float_as_uint((float)a), 0x07060302u);
    }
    __device__ static __forceinline__ V of(unsigned a, unsigned b, unsigned c, unsigned d) {
        return __builtin_bit_cast(V, (u32x4{a, b, c, d}));
    }
    template <int BITS>
    __device__ __forceinline__ V key(const unsigned* w) const {  // one word, or two
        if constexpr (BITS == 4) return of(pair4(w[0]), pair4(w[0] >> 4), pair4(w[0] >> 8), pair4(w[0] >> 12));
        else
            return of(pair8(w[0] & 255u, w[0] >> 8 & 255u), pair8(w[0] >> 16 & 255u, w[0] >> 24),
                      pair8(w[1] & 255u, w[1] >> 8 & 255u), pair8(w[1] >> 16 & 255u, w[1] >> 24));
    }
    template <int BITS>
    __device__ __forceinline__ V val(u32x4 w, int u) const {  // the u-th of the dims that are 16 apart
        if constexpr (BITS == 4) return of(pair4(w[0] >> 4 * u), pair4(w[1] >> 4 * u), pair4(w[2] >> 4 * u), pair4(w[3] >> 4 * u));
        else
            return of(pair8(w[0] >> 8 * u & 255u, w[0] >> (8 * u + 16) & 255u), pair8(w[1] >> 8 * u & 255u, w[1] >> (8 * u + 16) & 255u),
                      pair8(w[2] >> 8 * u & 255u, w[2] >> (8 * u + 16) & 255u), pair8(w[3] >> 8 * u & 255u, w[3] >> (8 * u + 16) & 255u));
    }
    template <int BITS>
    __device__ __forceinline__ V zeros(u32x4 w) const {  // of 8 positions' words, the codes' offset added
        if constexpr (BITS == 4) return of(pair4(w[0]), pair4(w[1]), pair4(w[2]), pair4(w[3]));
        else return val<8>(w, 0);
    }
    __device__ static __forceinline__ mfma_f32x4 mul(V a, V b, mfma_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Codes<float> {
    typedef f32x8 V;
    __device__ static __forceinline__ V load(const float* p) {  // (16-byte aligned, V is 32)
        const mfma_f32x4 a = *reinterpret_cast<const mfma_f32x4*>(p), b = *reinterpret_cast<const mfma_f32x4*>(p + 4);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    template <int BITS>
    __device__ __forceinline__ V key(const unsigned* w) const {
        V x;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = BITS == 4 ? (float)(w[0] >> ((e >> 1) * 4 + (e & 1) * 16) & 15u) : (float)(w[e >> 2 & (BITS == 8)] >> ((e & 3) * 8) & 255u);
        return x;
    }
    template <int BITS>
    __device__ __forceinline__ V val(u32x4 w, int u) const {
        V x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)(w[e >> 1] >> ((e & 1) * 16 + u * BITS) & (BITS == 4 ? 15u : 255u));
        return x;
    }
    template <int BITS>
    __device__ __forceinline__ V zeros(u32x4 w) const { return val<BITS>(w, 0); }
    __device__ static __forceinline__ mfma_f32x4 mul(V a, V b, mfma_f32x4 c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

// ------------------------------------------------------------------ attention of few rows
//
// As paged_attn_kernel, on codes. With k = (c - z) s a score is
//   q . k = s (q . c - z sum(q)), per group,
// and with v = (c - z) s the weighted sum of the values is
//   sum p v = sum (p s) c - sum (p s) z
// so the products take codes as they are: steps scale scores and weights, and the
// zeros are one rank-1 term of the scores and one more "dim" of the values (a
// fragment whose 16 rows are all z). In fp32 the operands are c - z itself: terms
// that leave again would cost bits of a result of 24 (one token over 37 positions, 6
// heads of 64, 4 bits: 1.1e-6 off instead of 3.3e-7, and no slower).
// Codes are finite whatever was there before; hidden positions' steps are taken as
// 0, so no value of theirs enters.
// Bound by the chain list - page - codes where contexts are short, else by unpacking:
// 5 tokens each of 16 sequences over 4001 positions at most, 16 / 4 heads of 64 in 8
// bits, 10.6 us. (With all of a block's reads before it 10.9, and 113 instead of 93
// for 32 tokens with 4 query heads each of 32 sequences over 1000 positions, 8 heads of
// 128 in 8 bits.)
template <class T, int D, int BITS>
__global__ __launch_bounds__(256) void packed_attn_kernel(AttnArgs a) {
    typedef Codes<T> C;
    typedef typename C::V V;
    constexpr int NK = D / 32, ND = D / 16, NG = D / GROUP;
    constexpr int NB = D * BITS / 256;  // 16-byte pieces per lane of 32 positions' codes
    constexpr int PER = 16 / BITS;      // dim tiles of a value piece
    constexpr bool TWO = sizeof(T) == 2;
    __shared__ float so[4][16][D + 4];
    __shared__ float sm[4][16], sl[4][16];
    const ListHead head = *reinterpret_cast<const ListHead*>(a.plan);
    const AttnItem* items = reinterpret_cast<const AttnItem*>(a.plan + HEAD_INTS);
    const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int P = 1 << a.c.shift;
    const bool large = a.c.large();
    const C codes{};
    for (int w0 = blockIdx.x; w0 < head.items * a.c.Hkv; w0 += gridDim.x) {
        const int it = w0 / a.c.Hkv, h = w0 - it * a.c.Hkv;
        const AttnItem t = items[it];
        const int rows = t.count * a.G;
        const int j = min(t.j0 + fr, rows - 1), tok = j / a.G, g = j - tok * a.G;
        const int lim = t.past + tok + 1;            // positions this lane's row sees
        const int all = t.past + t.j0 / a.G + 1;     // positions every row sees
        const T* q = static_cast<const T*>(a.q) + (long long)(t.tok0 + tok) * a.q_ld + (h * a.G + g) * D + fc * 8;
        V qf[NK];
#pragma unroll
        for (int s = 0; s < NK; ++s) qf[s] = C::load(q + s * 32);
        // bf16: the zeros' term of the scores as a product too, of -(zero + offset) and
        // the row's sums as three bf16 numbers each, which leave 2^-24 of them
        V qz[NG];
        if constexpr (TWO) {
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                float sum = 0.f;
#pragma unroll
                for (int s = 2 * i; s < 2 * i + 2; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += (float)qf[s][e];
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                float left = fc == 0 ? sum : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    qz[i][e] = (__bf16)(e < 3 ? left : 0.f);
                    left -= (float)qz[i][e];
                }
            }
        }
        mfma_f32x4 o[ND], oz[NG];
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NG; ++i) oz[i] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        const int* table = a.c.table + (long long)t.seq * a.c.ld;
        // pages are looked up a block ahead, a block's codes read when the former's have been used
        auto page_of = [&](int p) __attribute__((always_inline)) { return list_at(table, min(p, t.kv1 - 1) >> a.c.shift); };
        u32x4 kw[NB], vw[NB];
        u32x2 ks[NG][2], vs[NG][2];  // words of positions b * 16 + fc * 4 .. + 3
        unsigned kz[NG][2];          // and of position b * 16 + fr
        auto read_keys = [&](int page, int p) __attribute__((always_inline)) {
            const int p0 = p & (P - 1);
            const unsigned char* kb = a.c.head<unsigned char>(page, a.layer, 0, h);
            const unsigned char* words = kb + packed_codes<BITS>(P, D) + p0 * 2;
#pragma unroll
            for (int i = 0; i < NB; ++i) kw[i] = *reinterpret_cast<const u32x4*>(kb + (p0 >> 5) * (NB * 1024) + lane * 16 + i * 1024);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    ks[i][b] = *reinterpret_cast<const u32x2*>(words + (i * P + b * 16 + fc * 4) * 2);
                    kz[i][b] = *reinterpret_cast<const unsigned short*>(words + (i * P + b * 16 + fr) * 2);
                }
        };
        auto read_values = [&](int page, int p) __attribute__((always_inline)) {
            const int p0 = p & (P - 1);
            const unsigned char* vb = a.c.head<unsigned char>(page, a.layer, 1, h);
            const unsigned char* words = vb + packed_codes<BITS>(P, D) + p0 * 2;
#pragma unroll
            for (int i = 0; i < NB; ++i) vw[i] = *reinterpret_cast<const u32x4*>(vb + (p0 >> 5) * (NB * 1024) + lane * 16 + i * 1024);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) vs[i][b] = *reinterpret_cast<const u32x2*>(words + (i * P + b * 16 + fc * 4) * 2);
        };
        const int p1 = t.kv0 + wave * 32;
        int next = page_of(p1);
        if (p1 < t.kv1) {
            read_keys(next, p1);
            read_values(next, p1);
        }
        next = page_of(p1 + 128);
        for (int p = p1; p < t.kv1; p += 128) {
            const int page = next;
            const bool more = p + 128 < t.kv1;
            next = page_of(p + 256);
            const int end = p + 32 > all ? lim - p - fc * 4 : 32;  // positions of the block, from this lane's first, that it sees
            mfma_f32x4 sc[2];
            float mx = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                mfma_f32x4 x[NG];
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    x[i] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
                    if constexpr (TWO) {
                        unsigned z;  // -(zero + offset), twice
                        if constexpr (BITS == 4) z = (kz[i][b] & 15u) | 0xc300u;
                        else z = __float_as_uint(-(float)(kz[i][b] & 255u)) >> 16;
                        z |= z << 16;
                        x[i] = C::mul(C::of(z, z, z, z), qz[i], x[i]);
                    }
#pragma unroll
                    for (int s = 2 * i; s < 2 * i + 2; ++s) {
                        const int n = b * NK + s;
                        unsigned w[2];
                        if constexpr (BITS == 4) w[0] = w[1] = kw[n >> 2][n & 3];
                        else w[0] = kw[n >> 1][(n & 1) * 2], w[1] = kw[n >> 1][(n & 1) * 2 + 1];
                        V kf = codes.template key<BITS>(w);
                        if constexpr (!TWO) kf -= group_zero<BITS>(kz[i][b]);
                        x[i] = C::mul(kf, qf[s], x[i]);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float y = 0.f;
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        const unsigned w = ks[i][b][r >> 1] >> (r & 1) * 16;
                        y = fmaf(x[i][r], group_step<BITS>(w), y);
                    }
                    y *= a.scale;
                    y = b * 16 + r >= end ? -INFINITY : y;
                    sc[b][r] = y;
                    mx = fmaxf(mx, y);
                }
            }
            if (more) read_keys(page, p + 128);
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
#pragma unroll
                for (int i = 0; i < NG; ++i) oz[i][0] *= alpha;
                m = mn;
            }
            {
#pragma clang fp contract(off)  // mu is a rounded product, and so is what it is taken from
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[b][r] = exp2_softmax(sc[b][r] - mu);
                if (large) sc[0] *= SHRINK, sc[1] *= SHRINK;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) l += sc[b][r];
            }
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                V pf, pl;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float st = group_step<BITS>(vs[i][b][r >> 1] >> (r & 1) * 16);
                        const float y = sc[b][r] * (b * 16 + r >= end ? 0.f : st);
                        if constexpr (TWO) {
                            const __bf16 w = (__bf16)y;
                            pf[b * 4 + r] = w;
                            // (a weight that is not finite says so by itself)
                            const float left = y - (float)w;
                            pl[b * 4 + r] = (__bf16)left;
                        } else {
                            pf[b * 4 + r] = y;
                        }
                    }
                const V z = codes.template zeros<BITS>(u32x4{vs[i][0][0], vs[i][0][1], vs[i][1][0], vs[i][1][1]});
                if constexpr (TWO) {
                    oz[i] = C::mul(z, pl, oz[i]);
                    oz[i] = C::mul(z, pf, oz[i]);
                }
#pragma unroll
                for (int d = i * (GROUP / 16); d < (i + 1) * (GROUP / 16); ++d) {
                    V vf = codes.template val<BITS>(vw[d / PER], d % PER);
                    if constexpr (TWO) o[d] = C::mul(vf, pl, o[d]);
                    else vf -= z;
                    o[d] = C::mul(vf, pf, o[d]);
                }
            }
            if (more) read_values(page, p + 128);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[d][r] -= oz[d * 16 / GROUP][0];
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
                    attn_store<T, false>(a, t.tok0 + tk, h * a.G + gg, D, d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
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

// Up to 4 rows in bf16 (a decode step of up to 4 query heads per kv head): 16 columns of a
// product would hold them four times. Here 64 positions at once make use of the
// 16: column 4 b + g is row g over the b-th 16 positions, so the softmax of 64
// positions takes as many instructions as that of 16 rows over 16 positions. The
// four blocks' scores are products with the same queries in all columns, of which
// each column keeps its own block's; the weights enter the product with a value
// block of 32 positions in the columns of its two blocks, zeros in the others, and
// a row's four columns are added up at the end.
// Bound by reading and unpacking beside each other: one token of 4 sequences over 60001
// positions at most, 32 / 8 heads of 128 in 4 bits, 37.4 us (161 MB, 4.3 TB/s;
// unpacked in bf16 127), of 32 over 447 at most, 20 heads of 64, 7.4 us.
template <int D, int BITS>
__global__ __launch_bounds__(256) void packed_attn_four_kernel(AttnArgs a) {
    typedef bf16 T;
    typedef Codes<T> C;
    typedef C::V V;
    constexpr int NK = D / 32, ND = D / 16, NG = D / GROUP;
    constexpr int NB = D * BITS / 256;  // 16-byte pieces per lane of 32 positions' codes
    constexpr int PER = 16 / BITS;      // dim tiles of a value piece
    constexpr float OFF = CODE_OFF<T, BITS>;
    __shared__ float so[4][4][D + 4];
    __shared__ float sm[4][4], sl[4][4];
    const ListHead head = *reinterpret_cast<const ListHead*>(a.plan);
    const AttnItem* items = reinterpret_cast<const AttnItem*>(a.plan + head.fours_at);
    const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4, g = fr & 3, blk = fr >> 2;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int P = 1 << a.c.shift;
    const bool large = a.c.large();
    const C codes{};
    for (int w0 = blockIdx.x; w0 < head.fours * a.c.Hkv; w0 += gridDim.x) {
        const int it = w0 / a.c.Hkv, h = w0 - it * a.c.Hkv;
        const AttnItem t = items[it];
        const int rows = t.count * a.G;
        const int j = min(t.j0 + g, rows - 1), tok = j / a.G;
        const int lim = t.past + tok + 1;         // positions this lane's row sees
        const int all = t.past + t.j0 / a.G + 1;  // positions every row sees
        const T* q = static_cast<const T*>(a.q) + (long long)(t.tok0 + tok) * a.q_ld + (h * a.G + j - tok * a.G) * D + fc * 8;
        V qf[NK];
        float qs[NG];  // the row's sums
#pragma unroll
        for (int i = 0; i < NG; ++i) qs[i] = 0.f;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            qf[s] = C::load(q + s * 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) qs[s / 2] += (float)qf[s][e];
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            qs[i] += __shfl_xor(qs[i], 16, 64);
            qs[i] += __shfl_xor(qs[i], 32, 64);
        }
        mfma_f32x4 o[ND], oz[NG];
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NG; ++i) oz[i] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        const int* table = a.c.table + (long long)t.seq * a.c.ld;
        // 32 positions from p, or (where the range ends before) its last 32 again, hidden
        const int last = (t.kv1 - 1) & ~31;
        auto place = [&](int p) __attribute__((always_inline)) { return min(p, last); };
        auto page_of = [&](int p) __attribute__((always_inline)) { return list_at(table, place(p) >> a.c.shift); };
        int next[2];  // pages are looked up a block ahead
#pragma unroll
        for (int i = 0; i < 2; ++i) next[i] = page_of(t.kv0 + wave * 64 + i * 32);
        auto blocks = [&](auto is_large) __attribute__((always_inline)) {
            for (int p = t.kv0 + wave * 64; p < t.kv1; p += 256) {
                u32x4 kw[2][NB], vw[2][NB];
                u32x2 vs[NG][2][2];  // words of the halves' positions b * 16 + fc * 4 .. + 3
                u32x2 ks[NG], vo[NG];  // of positions blk * 16 + fc * 4 .. + 3, this column's
                const unsigned char *kb[2], *vb[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int p0 = place(p + 32 * i) & (P - 1);
                    kb[i] = a.c.head<unsigned char>(next[i], a.layer, 0, h);
                    vb[i] = a.c.head<unsigned char>(next[i], a.layer, 1, h);
                    next[i] = page_of(p + 256 + 32 * i);
                    const int at = (p0 >> 5) * (NB * 1024) + lane * 16;
#pragma unroll
                    for (int n = 0; n < NB; ++n) kw[i][n] = *reinterpret_cast<const u32x4*>(kb[i] + at + n * 1024);
#pragma unroll
                    for (int n = 0; n < NB; ++n) vw[i][n] = *reinterpret_cast<const u32x4*>(vb[i] + at + n * 1024);
                    kb[i] += packed_codes<BITS>(P, D) + (p0 + fc * 4) * 2;
                    vb[i] += packed_codes<BITS>(P, D) + (p0 + fc * 4) * 2;
                }
                const unsigned char *kc = (blk & 2 ? kb[1] : kb[0]) + (blk & 1) * 32, *vc = (blk & 2 ? vb[1] : vb[0]) + (blk & 1) * 32;
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    ks[i] = *reinterpret_cast<const u32x2*>(kc + i * P * 2);
                    vo[i] = *reinterpret_cast<const u32x2*>(vc + i * P * 2);
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int b = 0; b < 2; ++b) vs[i][n][b] = *reinterpret_cast<const u32x2*>(vb[n] + i * P * 2 + b * 32);
                }
                mfma_f32x4 x[NG];
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        mfma_f32x4 y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 2 * i; s < 2 * i + 2; ++s) {
                            const int n = (b & 1) * NK + s;
                            unsigned w[2];
                            if constexpr (BITS == 4) w[0] = w[1] = kw[b >> 1][n >> 2][n & 3];
                            else w[0] = kw[b >> 1][n >> 1][(n & 1) * 2], w[1] = kw[b >> 1][n >> 1][(n & 1) * 2 + 1];
                            y = C::mul(codes.key<BITS>(w), qf[s], y);
                        }
#pragma unroll
                        for (int r = 0; r < 4; ++r) x[i][r] = b == 0 || blk == b ? y[r] : x[i][r];
                    }
                // of this lane's 4 positions, those it sees
                const int end = p + 64 > min(all, t.kv1) ? min(lim, t.kv1) - (p + blk * 16 + fc * 4) : 4;
                float sc[4], mx = -INFINITY;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float y = 0.f;
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        const unsigned w = ks[i][r >> 1] >> (r & 1) * 16;
                        y = fmaf(fmaf(-(group_zero<BITS>(w) + OFF), qs[i], x[i][r]), group_step<BITS>(w), y);
                    }
                    y *= a.scale;
                    y = r >= end ? -INFINITY : y;
                    sc[r] = y;
                    mx = fmaxf(mx, y);
                }
                mx = fmaxf(mx, __uint_as_float(lane_xor<4>(__float_as_uint(mx))));
                mx = fmaxf(mx, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(mx), 0x128, 0xf, 0xf, true)));  // 8 lanes on
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
#pragma unroll
                    for (int i = 0; i < NG; ++i) oz[i][0] *= alpha;
                    m = mn;
                }
                {
#pragma clang fp contract(off)  // mu is a rounded product, and so is what it is taken from
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[r] = exp2_softmax(sc[r] - mu);
                    if constexpr (decltype(is_large)::value)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sc[r] *= SHRINK;
#pragma unroll
                    for (int r = 0; r < 4; ++r) l += sc[r];
                }
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    float y[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float st = group_step<BITS>(vo[i][r >> 1] >> (r & 1) * 16);
                        y[r] = sc[r] * (r >= end ? 0.f : st);
                    }
                    V pf[2], pl[2];
                    unsigned hi[2], lo[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        hi[u] = pack_bf16x2(y[2 * u], y[2 * u + 1]);
                        lo[u] = pack_bf16x2(y[2 * u] - __uint_as_float(hi[u] << 16), y[2 * u + 1] - __uint_as_float(hi[u] & 0xffff0000u));
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const bool one = blk == 2 * n, two = blk == 2 * n + 1;
                        pf[n] = C::of(one ? hi[0] : 0, one ? hi[1] : 0, two ? hi[0] : 0, two ? hi[1] : 0);
                        pl[n] = C::of(one ? lo[0] : 0, one ? lo[1] : 0, two ? lo[0] : 0, two ? lo[1] : 0);
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const V z = codes.zeros<BITS>(u32x4{vs[i][n][0][0], vs[i][n][0][1], vs[i][n][1][0], vs[i][n][1][1]});
                        oz[i] = C::mul(z, pl[n], oz[i]);
                        oz[i] = C::mul(z, pf[n], oz[i]);
#pragma unroll
                        for (int d = i * (GROUP / 16); d < (i + 1) * (GROUP / 16); ++d) {
                            const V vf = codes.val<BITS>(vw[n][d / PER], d % PER);
                            o[d] = C::mul(vf, pl[n], o[d]);
                            o[d] = C::mul(vf, pf[n], o[d]);
                        }
                    }
                }
            }
        };
        if (large) blocks(std::true_type{});
        else blocks(std::false_type{});
        // a row's columns 4 and 8 lanes away, the lanes' weights
        auto add_blocks = [&](float v) __attribute__((always_inline)) {
            v += __uint_as_float(lane_xor<4>(__float_as_uint(v)));
            return v + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x128, 0xf, 0xf, true));
        };
        l = add_blocks(l);
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (lane < 4) {
            sm[wave][g] = m;
            sl[wave][g] = l;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float y = add_blocks(o[d][r] - oz[d * 16 / GROUP][0]);
                if (blk == 0) so[wave][g][d * 16 + fc * 4 + r] = y;
            }
        __syncthreads();
        // thread: row tid / (D / 4), 4 dims
        const int row = threadIdx.x / (D / 4), d = (threadIdx.x % (D / 4)) * 4;
        if (row < 4 && t.j0 + row < rows) {
            const float mt = fmaxf(fmaxf(sm[0][row], sm[1][row]), fmaxf(sm[2][row], sm[3][row]));
            const float mu = mt == -INFINITY ? 0.f : mt;
            float w[4], lt = 0.f, y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = exp2_softmax(sm[i][row] - mu);
                lt += sl[i][row] * w[i];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                y[e] = so[0][row][d + e] * w[0] + so[1][row][d + e] * w[1] + so[2][row][d + e] * w[2] + so[3][row][d + e] * w[3];
            if (t.part < 0) {
                const int jr = t.j0 + row, tk = jr / a.G, gg = jr - tk * a.G;
                const float inv = lt == 0.f ? 0.f : 1.0f / lt;
                attn_store<T, false>(a, t.tok0 + tk, h * a.G + gg, D, d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
            } else {
                float* ps = a.parts + ((long long)t.part * a.c.Hkv + h) * (16 * (D + 2));
                st4(ps + row * D + d, y[0], y[1], y[2], y[3]);
                if (d == 0) {
                    ps[16 * D + row] = mt;
                    ps[16 * D + 16 + row] = lt;
                }
            }
        }
        __syncthreads();  // the next item's LDS
    }
}

// ------------------------------------------------------------------ attention of many rows
//
// The 128-row kernel goes through a sequence's positions once for every 128
// rows, so unpacking inside it would be done as many times. Pages of sequences
// with that many rows are unpacked once instead, one layer's keys and values as
// a cache of bf16 has them (page for page, so page lists hold for both), and
// paged_attn_big_kernel reads those. Bound by the latency of the list and by writing:
// 8193 positions, 8 heads of 128 in 4 bits 10 us (34 MB written), beside some 430 of the
// attention of 4096 tokens over them.
template <int D, int BITS>
__global__ __launch_bounds__(256) void packed_unpack_kernel(PagedView c, int layer, const int* __restrict__ list,
                                                            bf16* __restrict__ out) {
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const int* pages = list + head.pages_at;  // as places in the page lists, which may change while the list is current
    const int P = 1 << c.shift, lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    constexpr int NB = D * BITS / 256, NK = D / 32, PER = 16 / BITS;
    const float shrink = c.large() ? SHRINK : 1.f;  // (the attention's weights take it back)
    // a wave per 32 positions of a head's keys or values
    const int blocks = P / 32, n = head.pages * c.Hkv * 2 * blocks;
    for (int i = blockIdx.x * 4 + (threadIdx.x >> 6); i < n; i += gridDim.x * 4) {
        const int b32 = i % blocks, kv = i / blocks % 2, h = i / blocks / 2 % c.Hkv, page = c.table[pages[i / blocks / 2 / c.Hkv]];
        const unsigned char* src = c.head<unsigned char>(page, layer, kv, h);
        const unsigned short* words = reinterpret_cast<const unsigned short*>(src + packed_codes<BITS>(P, D)) + b32 * 32;
        bf16* dst = out + ((long long)(page * 2LL + kv) * c.Hkv + h) * (P * D) + b32 * (32 * D) + lane * 8;
        u32x4 w[NB];
#pragma unroll
        for (int k = 0; k < NB; ++k) w[k] = *reinterpret_cast<const u32x4*>(src + (b32 * NB + k) * 1024 + lane * 16);
        auto put = [&](int f, const f32x8& y) __attribute__((always_inline)) {
            u32x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = pack_bf16x2(y[2 * e], y[2 * e + 1]);
            *reinterpret_cast<u32x4*>(dst + f * 512) = r;
        };
        if (kv == 0) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int s = 0; s < NK; ++s) {
                    const int f = b * NK + s;
                    const unsigned m = words[s / 2 * P + b * 16 + fr];
                    unsigned x[2];
                    if constexpr (BITS == 4) x[0] = x[1] = w[f >> 2][f & 3];
                    else x[0] = w[f >> 1][(f & 1) * 2], x[1] = w[f >> 1][(f & 1) * 2 + 1];
                    put(f, (Codes<float>{}.key<BITS>(x) - group_zero<BITS>(m)) * group_step<BITS>(m));
                }
        } else {
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                f32x8 y = Codes<float>{}.val<BITS>(w[d / PER], d % PER);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned m = words[d / 4 * P + fc * 4 + (e & 3) + (e >> 2) * 16];
                    y[e] = (y[e] - group_zero<BITS>(m)) * (group_step<BITS>(m) * shrink);
                }
                put(d, y);
            }
        }
    }
}

}  // namespace wmi
