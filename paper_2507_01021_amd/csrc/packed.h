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
// average in 4 bits, but its values would need 12 bits and be rounded in bf16.
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

// Step and zero from a group's word. CHECK: 8-bit words may be NaN's.
template <int BITS, bool CHECK = true>
__device__ __forceinline__ float group_step(unsigned w) {
    if constexpr (BITS == 4) return __uint_as_float((w & 0x7ff0u) << 16);
    const float s = __uint_as_float((w & 0xff00u) << 15);
    return CHECK && (w & 0xff00u) == 0xff00u ? NAN : s;
}
template <int BITS>
__device__ __forceinline__ float group_zero(unsigned w) {
    return (float)(w & (BITS == 4 ? 15u : 255u));
}

// The codes of 8 numbers of a group whose other numbers are those of the
// lanes beside this one (8 lanes at a multiple of 8); returns the group's word.
// Quotients are rounded to fp32 before they are rounded to integers: the step
// has so few bits that no quotient of a 24-bit number comes to lie on a half, or
// on a step, by that.
template <int BITS>
__device__ __forceinline__ unsigned quantise(const float (&x)[8], unsigned (&code)[8], bool& odd) {
    constexpr unsigned TOP = BITS == 4 ? 15 : 255, LOW = BITS == 4 ? 0xfffffu : 0x7fffffu;
    float lo = 0.f, hi = 0.f;
    int bad = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        bad |= !(fabsf(x[e]) < 0x1p125f);
    }
#pragma unroll
    for (int st = 1; st < 8; st <<= 1) {
        lo = fminf(lo, __shfl_xor(lo, st, 64));
        hi = fmaxf(hi, __shfl_xor(hi, st, 64));
        bad |= __shfl_xor(bad, st, 64);
    }
    const float step = fmaxf(__uint_as_float((__float_as_uint((hi - lo) / (float)TOP) + LOW) & ~LOW), 0x1p-100f);
    const float zero = rintf(-lo / step);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        code[e] = bad ? 0 : (unsigned)fminf(fmaxf(rintf(x[e] / step) + zero, 0.f), (float)TOP);
    odd = odd || bad;
    if constexpr (BITS == 4) return bad ? 0x7ff0u : (__float_as_uint(step) >> 16) | (unsigned)zero;
    return bad ? 0xff00u : (__float_as_uint(step) >> 23) << 8 | (unsigned)zero;
}

// Eight numbers of a row, or into one.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    if constexpr (VEC) {
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
    if constexpr (VEC) {
        st4(p, x[0], x[1], x[2], x[3]);
        st4(p + 4, x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) stf(p + e, x[e]);
    }
}

// ------------------------------------------------------------------ rows in and out
//
// As paged_append_kernel and paged_read_kernel: a workgroup per (tile, kv head,
// layer), rows of up to 32 positions. Eight lanes have a group. Keys are written
// as they come; values go through LDS, so that a block's 16-byte pieces are
// written whole where all their positions are new.
template <class T, int D, int BITS, bool VEC>
__global__ __launch_bounds__(256) void packed_append_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                            const T* __restrict__ k, const T* __restrict__ v,
                                                            long long k_ld, long long v_ld, long long k_layer,
                                                            long long v_layer) {
    constexpr int CH = D / 8, LD = D + 4, TILES = 16 / BITS;
    __shared__ __align__(16) unsigned char sv[32 * LD];
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int h = blockIdx.y, layer = layer0 + blockIdx.z, tid = threadIdx.x, P = 1 << c.shift;
    for (int it = blockIdx.x; it < head.tiles; it += gridDim.x) {
        const PageTile t = tiles[it];
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        const int p0 = t.pos & (P - 1);
        unsigned char* kd = c.head<unsigned char>(page, layer, 0, h);
        unsigned char* vd = c.head<unsigned char>(page, layer, 1, h);
        const T* ks = k + blockIdx.z * k_layer + (long long)t.row * k_ld + h * D;
        const T* vs = v + blockIdx.z * v_layer + (long long)t.row * v_ld + h * D;
        bool odd = false;
        for (int i = tid; i < t.n * CH; i += 256) {
            const int r = i / CH, d = (i - r * CH) * 8, p = p0 + r;
            float x[8];
            unsigned q[8];
            load8<T, VEC>(ks + r * k_ld + d, x);
            const unsigned wk = quantise<BITS>(x, q, odd);
            unsigned char* dst = kd + pkey_off<BITS>(p, d, D);
            if constexpr (BITS == 4) {
                unsigned w = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) w |= q[e] << ((e >> 1) * 4 + (e & 1) * 16);
                *reinterpret_cast<unsigned*>(dst) = w;
            } else {
                *reinterpret_cast<u32x2*>(dst) = u32x2{q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24,
                                                       q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24};
            }
            load8<T, VEC>(vs + r * v_ld + d, x);
            const unsigned wv = quantise<BITS>(x, q, odd);
            unsigned* sd = reinterpret_cast<unsigned*>(sv + (p & 31) * LD + d);
            sd[0] = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
            sd[1] = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
            if ((d & (GROUP - 1)) == 0) {
                const int at = packed_codes<BITS>(P, D) + ((d / GROUP) * P + p) * 2;
                *reinterpret_cast<unsigned short*>(kd + at) = (unsigned short)wk;
                *reinterpret_cast<unsigned short*>(vd + at) = (unsigned short)wv;
            }
        }
        if (c.odd && odd) *c.odd = 1;
        __syncthreads();
        const int lo = p0 & 31, hi = lo + t.n;
        unsigned char* vb = vd + pval_off<BITS>(p0 & ~31, 0, D);
        for (int i = tid; i < D * BITS / 4; i += 256) {  // 16-byte pieces of the block of 32 positions
            const int ln = i & 63, dim = (i >> 6) * (256 / BITS) + (ln & 15), g = ln >> 4;
            unsigned half[8];
            bool all = true;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int pos = g * 4 + (e & 3) + (e >> 2) * 16;
                all = all && pos >= lo && pos < hi;
                half[e] = 0;
#pragma unroll
                for (int u = 0; u < TILES; ++u) half[e] |= (unsigned)sv[pos * LD + dim + u * 16] << (u * BITS);
            }
            unsigned char* dst = vb + i * 16;
            if (all) {
                *reinterpret_cast<u32x4*>(dst) =
                    u32x4{half[0] | half[1] << 16, half[2] | half[3] << 16, half[4] | half[5] << 16, half[6] | half[7] << 16};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int pos = g * 4 + (e & 3) + (e >> 2) * 16;
                    if (pos >= lo && pos < hi) reinterpret_cast<unsigned short*>(dst)[e] = (unsigned short)half[e];
                }
            }
        }
        __syncthreads();  // the next tile's LDS
    }
}

template <class T, int D, int BITS, bool VEC>
__global__ __launch_bounds__(256) void packed_read_kernel(PagedView c, const int* __restrict__ list, int layer0,
                                                          T* __restrict__ k, T* __restrict__ v, long long k_ld,
                                                          long long v_ld, long long k_layer, long long v_layer) {
    constexpr int CH = D / 8, LD = D + 4, TILES = 16 / BITS;
    __shared__ __align__(16) unsigned char sv[32 * LD];
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const PageTile* tiles = reinterpret_cast<const PageTile*>(list + head.tiles_at);
    const int h = blockIdx.y, layer = layer0 + blockIdx.z, tid = threadIdx.x, P = 1 << c.shift;
    for (int it = blockIdx.x; it < head.tiles; it += gridDim.x) {
        const PageTile t = tiles[it];
        const int page = c.table[(long long)t.seq * c.ld + (t.pos >> c.shift)];
        const int p0 = t.pos & (P - 1);
        const unsigned char* kd = c.head<unsigned char>(page, layer, 0, h);
        const unsigned char* vd = c.head<unsigned char>(page, layer, 1, h);
        const unsigned char* vb = vd + pval_off<BITS>(p0 & ~31, 0, D);
        T* ks = k + blockIdx.z * k_layer + (long long)t.row * k_ld + h * D;
        T* vs = v + blockIdx.z * v_layer + (long long)t.row * v_ld + h * D;
        for (int i = tid; i < D * BITS / 4; i += 256) {
            const int ln = i & 63, dim = (i >> 6) * (256 / BITS) + (ln & 15), g = ln >> 4;
            const u32x4 a = *reinterpret_cast<const u32x4*>(vb + i * 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int pos = g * 4 + (e & 3) + (e >> 2) * 16;
#pragma unroll
                for (int u = 0; u < TILES; ++u)
                    sv[pos * LD + dim + u * 16] = (unsigned char)(a[e >> 1] >> ((e & 1) * 16 + u * BITS) & (BITS == 4 ? 15u : 255u));
            }
        }
        __syncthreads();
        for (int i = tid; i < t.n * CH; i += 256) {
            const int r = i / CH, d = (i - r * CH) * 8, p = p0 + r;
            const int at = packed_codes<BITS>(P, D) + ((d / GROUP) * P + p) * 2;
            float x[8];
            unsigned q[8];
            const unsigned char* src = kd + pkey_off<BITS>(p, d, D);
            if constexpr (BITS == 4) {
                const unsigned w = *reinterpret_cast<const unsigned*>(src);
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = w >> ((e >> 1) * 4 + (e & 1) * 16) & 15u;
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2*>(src);
#pragma unroll
                for (int e = 0; e < 8; ++e) q[e] = w[e >> 2] >> ((e & 3) * 8) & 255u;
            }
            const unsigned wk = *reinterpret_cast<const unsigned short*>(kd + at);
            const unsigned wv = *reinterpret_cast<const unsigned short*>(vd + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = ((float)q[e] - group_zero<BITS>(wk)) * group_step<BITS>(wk);
            store8<T, VEC>(ks + r * k_ld + d, x);
            const unsigned* sd = reinterpret_cast<const unsigned*>(sv + (p & 31) * LD + d);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = ((float)(sd[e >> 2] >> ((e & 3) * 8) & 255u) - group_zero<BITS>(wv)) * group_step<BITS>(wv);
            store8<T, VEC>(vs + r * v_ld + d, x);
        }
        __syncthreads();  // the next tile's LDS
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
    __device__ static __forceinline__ unsigned pair4(unsigned w) { return (w & 0x000f000fu) | 0x43004300u; }
    __device__ static __forceinline__ unsigned pair8(unsigned a, unsigned b) {  // two numbers up to 255
        return __builtin_amdgcn_perm(__float_as_uint((float)b), __float_as_uint((float)a), 0x07060302u);
    }
    __device__ static __forceinline__ V of(unsigned a, unsigned b, unsigned c, unsigned d) {
        return __builtin_bit_cast(V, (u32x4{a, b, c, d}));
    }
    template <int BITS>
    __device__ static __forceinline__ V key(const unsigned* w) {  // one word, or two
        if constexpr (BITS == 4) return of(pair4(w[0]), pair4(w[0] >> 4), pair4(w[0] >> 8), pair4(w[0] >> 12));
        else
            return of(pair8(w[0] & 255u, w[0] >> 8 & 255u), pair8(w[0] >> 16 & 255u, w[0] >> 24),
                      pair8(w[1] & 255u, w[1] >> 8 & 255u), pair8(w[1] >> 16 & 255u, w[1] >> 24));
    }
    template <int BITS>
    __device__ static __forceinline__ V val(u32x4 w, int u) {  // the u-th of the dims that are 16 apart
        if constexpr (BITS == 4) return of(pair4(w[0] >> 4 * u), pair4(w[1] >> 4 * u), pair4(w[2] >> 4 * u), pair4(w[3] >> 4 * u));
        else
            return of(pair8(w[0] >> 8 * u & 255u, w[0] >> (8 * u + 16) & 255u), pair8(w[1] >> 8 * u & 255u, w[1] >> (8 * u + 16) & 255u),
                      pair8(w[2] >> 8 * u & 255u, w[2] >> (8 * u + 16) & 255u), pair8(w[3] >> 8 * u & 255u, w[3] >> (8 * u + 16) & 255u));
    }
    template <int BITS>
    __device__ static __forceinline__ V zeros(u32x4 w) {  // of 8 positions' words, the codes' offset added
        if constexpr (BITS == 4) return of(pair4(w[0]), pair4(w[1]), pair4(w[2]), pair4(w[3]));
        else return val<8>(w, 0);
    }
    __device__ static __forceinline__ mfma_f32x4 mul(V a, V b, mfma_f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Codes<float> {
    typedef f32x8 V;
    template <int BITS>
    __device__ static __forceinline__ V key(const unsigned* w) {
        V x;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = BITS == 4 ? (float)(w[0] >> ((e >> 1) * 4 + (e & 1) * 16) & 15u) : (float)(w[e >> 2 & (BITS == 8)] >> ((e & 3) * 8) & 255u);
        return x;
    }
    template <int BITS>
    __device__ static __forceinline__ V val(u32x4 w, int u) {
        V x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)(w[e >> 1] >> ((e & 1) * 16 + u * BITS) & (BITS == 4 ? 15u : 255u));
        return x;
    }
    template <int BITS>
    __device__ static __forceinline__ V zeros(u32x4 w) { return val<BITS>(w, 0); }
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
// fragment whose 16 rows are all z). Codes are finite whatever was there before;
// hidden positions' steps are taken as 0, so no value of theirs enters.
template <class T, int D, int BITS>
__global__ __launch_bounds__(256) void packed_attn_kernel(AttnArgs a) {
    typedef Codes<T> C;
    typedef typename C::V V;
    constexpr int NK = D / 32, ND = D / 16, NG = D / GROUP;
    constexpr int NB = D * BITS / 256;  // 16-byte pieces per lane of 32 positions' codes
    constexpr int PER = 16 / BITS;      // dim tiles of a value piece
    constexpr float OFF = CODE_OFF<T, BITS>;
    constexpr bool TWO = sizeof(T) == 2;
    __shared__ float so[4][16][D + 4];
    __shared__ float sm[4][16], sl[4][16];
    const ListHead head = *reinterpret_cast<const ListHead*>(a.plan);
    const AttnItem* items = reinterpret_cast<const AttnItem*>(a.plan + HEAD_INTS);
    const int lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int P = 1 << a.c.shift;
    for (int w0 = blockIdx.x; w0 < head.items * a.c.Hkv; w0 += gridDim.x) {
        const int it = w0 / a.c.Hkv, h = w0 - it * a.c.Hkv;
        const AttnItem t = items[it];
        const int rows = t.count * a.G;
        const int j = min(t.j0 + fr, rows - 1), tok = j / a.G, g = j - tok * a.G;
        const int lim = t.past + tok + 1;            // positions this lane's row sees
        const int all = t.past + t.j0 / a.G + 1;     // positions every row sees
        const T* q = static_cast<const T*>(a.q) + (long long)(t.tok0 + tok) * a.q_ld + (h * a.G + g) * D + fc * 8;
        V qf[NK];
        float qs[NG];  // the row's sums
#pragma unroll
        for (int i = 0; i < NG; ++i) qs[i] = 0.f;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            qf[s] = *reinterpret_cast<const V*>(q + s * 32);
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
        int next = list_at(table, min(t.kv0 + wave * 32, t.kv1 - 1) >> a.c.shift);  // pages are looked up a block ahead
        for (int p = t.kv0 + wave * 32; p < t.kv1; p += 128) {
            const int page = next, p0 = p & (P - 1);
            next = list_at(table, min(p + 128, t.kv1 - 1) >> a.c.shift);
            const unsigned char* kb = a.c.head<unsigned char>(page, a.layer, 0, h);
            const unsigned char* vb = a.c.head<unsigned char>(page, a.layer, 1, h);
            const int at = (p0 >> 5) * (NB * 1024) + lane * 16, ws = packed_codes<BITS>(P, D) + (p0 + fc * 4) * 2;
            u32x4 kw[NB], vw[NB];
            u32x2 ks[NG][2], vs[NG][2];  // words of positions b * 16 + fc * 4 .. + 3
#pragma unroll
            for (int i = 0; i < NB; ++i) kw[i] = *reinterpret_cast<const u32x4*>(kb + at + i * 1024);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) ks[i][b] = *reinterpret_cast<const u32x2*>(kb + ws + (i * P + b * 16) * 2);
#pragma unroll
            for (int i = 0; i < NB; ++i) vw[i] = *reinterpret_cast<const u32x4*>(vb + at + i * 1024);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) vs[i][b] = *reinterpret_cast<const u32x2*>(vb + ws + (i * P + b * 16) * 2);
            const bool edge = p + 32 > all;
            auto hidden = [&](int b, int r) { return edge && p + b * 16 + fc * 4 + r >= lim; };
            mfma_f32x4 sc[2];
            float mx = -INFINITY;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                mfma_f32x4 x[NG];
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    x[i] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 2 * i; s < 2 * i + 2; ++s) {
                        const int n = b * NK + s;
                        unsigned w[2];
                        if constexpr (BITS == 4) w[0] = w[1] = kw[n >> 2][n & 3];
                        else w[0] = kw[n >> 1][(n & 1) * 2], w[1] = kw[n >> 1][(n & 1) * 2 + 1];
                        x[i] = C::mul(C::template key<BITS>(w), qf[s], x[i]);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float y = 0.f;
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        const unsigned w = ks[i][b][r >> 1] >> (r & 1) * 16;
                        y += fmaf(-(group_zero<BITS>(w) + OFF), qs[i], x[i][r]) * group_step<BITS>(w);
                    }
                    y *= a.scale;
                    if (hidden(b, r)) y = -INFINITY;
                    sc[b][r] = y;
                    mx = fmaxf(mx, y);
                }
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
#pragma unroll
                for (int i = 0; i < NG; ++i) oz[i][0] *= alpha;
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
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                V pf, pl;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float st = group_step<BITS>(vs[i][b][r >> 1] >> (r & 1) * 16);
                        const float y = hidden(b, r) ? 0.f : sc[b][r] * st;
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
                const V z = C::template zeros<BITS>(u32x4{vs[i][0][0], vs[i][0][1], vs[i][1][0], vs[i][1][1]});
                if constexpr (TWO) oz[i] = C::mul(z, pl, oz[i]);
                oz[i] = C::mul(z, pf, oz[i]);
#pragma unroll
                for (int d = i * (GROUP / 16); d < (i + 1) * (GROUP / 16); ++d) {
                    const V vf = C::template val<BITS>(vw[d / PER], d % PER);
                    if constexpr (TWO) o[d] = C::mul(vf, pl, o[d]);
                    o[d] = C::mul(vf, pf, o[d]);
                }
            }
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

// ------------------------------------------------------------------ attention of many rows
//
// The 128-row kernel goes through a sequence's positions once for every 128
// rows, so unpacking inside it would be done as many times. Pages of sequences
// with that many rows are unpacked once instead, one layer's keys and values as
// a cache of bf16 has them (page for page, so page lists hold for both), and
// paged_attn_big_kernel reads those.
template <int D, int BITS>
__global__ __launch_bounds__(256) void packed_unpack_kernel(PagedView c, int layer, const int* __restrict__ list,
                                                            bf16* __restrict__ out) {
    const ListHead head = *reinterpret_cast<const ListHead*>(list);
    const int* pages = list + head.pages_at;  // as places in the page lists, which may change while the list is current
    const int P = 1 << c.shift, lane = threadIdx.x & 63, fr = lane & 15, fc = lane >> 4;
    constexpr int NB = D * BITS / 256, NK = D / 32, PER = 16 / BITS;
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
                    put(f, (Codes<float>::key<BITS>(x) - group_zero<BITS>(m)) * group_step<BITS>(m));
                }
        } else {
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                f32x8 y = Codes<float>::val<BITS>(w[d / PER], d % PER);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned m = words[d / 4 * P + fc * 4 + (e & 3) + (e >> 2) * 16];
                    y[e] = (y[e] - group_zero<BITS>(m)) * group_step<BITS>(m);
                }
                put(d, y);
            }
        }
    }
}

}  // namespace wmi
