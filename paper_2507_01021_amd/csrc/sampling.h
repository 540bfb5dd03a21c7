// Choice of a token per row of logits with temperature, top-k, top-p and
// min-p from one given uniform number.
//
// With l_max the row's largest admissible logit, id i has the weight
//   w_i = round(2^43 exp((l_i - l_max) / T)),
// an integer, so that sums of weights are exact: they depend neither on the
// order of the additions nor on how a row is cut over threads, and a row's
// token is the same in every batch. (A weight is off by half a unit of
// 2^-43 of the largest at most, less than the 2^-24 of fp32 sums by far; V is
// at most 2^20, so a sum fits 64 bits.) Ids are ordered by (logit descending, id
// ascending); each filter keeps a prefix of that order, so the filters
// together keep the shortest: a cut, found by counting digits of the order's
// 52-bit key (32 bits of the logit, 20 of the id), highest first, until one
// digit decides.
#pragma once

#include "common.h"

namespace wmi {

struct SampleRow {  // whisper_sampling
    float temperature;
    int top_k;
    float top_p, min_p;
};

typedef unsigned long long u64;

struct SampleArgs {
    const void* logits;
    long long ld;
    int V;
    const SampleRow* rows;
    const unsigned* never;   // [V / 32 + 1] ids never chosen, or null
    const float* u;
    int* tok;                // or null
    float* logp;             // or null
    // decode steps: ids not chosen as a slot's first generated token (or
    // null), the rows' slots and their positions and prompt lengths, and the
    // choice as a greedy-choice key (0: none) for the step's last kernel
    const unsigned* first;
    const int* list;
    const int* pos;
    const int* n_prompt;
    u64* keys;
};

namespace smp {
constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048;
constexpr double ONE = 8796093022208.0;  // 2^43, the weight of the largest logit

// round(2^43 e^x) for x <= 0: e^x = 2^n e^r with |r| <= ln 2 / 2, e^r by its
// Taylor series to r^11 (remainder below 1e-14), the integer from the low
// bits of a sum with 2^52.
__device__ inline u64 weight(double x) {
    if (!(x > -32.0)) return 0;  // below half a unit (e^-32 2^43 < 0.12)
    const double n = __builtin_rint(x * 1.4426950408889634074);
    const double r = fma(n, -0.69314718055994530942, x);
    double p = 1.0 / 39916800.0;
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const double w = __builtin_amdgcn_ldexp(p, (int)n + 43) + 4503599627370496.0;
    return __builtin_bit_cast(u64, w) & 0xfffffffffffffull;
}

// 52-bit key of the order: larger means earlier.
__device__ inline u64 order_key(float l, int id) {
    return ((u64)f2ord(l == 0.f ? 0.f : l) << 20) | (u64)(0xfffff - id);
}

__device__ inline u64 wave_sum64(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// An id's logit; -inf for an inadmissible one.
template <class T>
__device__ inline float load_logit(const SampleArgs& a, const T* row, int id) {
    const float l = ldf(row + id);
    if (a.never && ((a.never[id >> 5] >> (id & 31)) & 1u)) return -INFINITY;
    if (a.first && ((a.first[id >> 5] >> (id & 31)) & 1u)) return -INFINITY;
    return l == l ? l : -INFINITY;  // NaN is never chosen
}
}  // namespace smp

// One workgroup per row. Every pass goes over the row again (it stays in the
// L2 cache). Wave w owns the ids [w C, w C + C), so that sums in the order of
// ids are sums over waves first.
template <class T>
__global__ __launch_bounds__(smp::THREADS) void sample_kernel(SampleArgs a) {
    using namespace smp;
    __shared__ u64 hw[BINS];
    __shared__ unsigned hc[BINS];
    __shared__ u64 red[WAVES];
    __shared__ double redd[WAVES];
    __shared__ u64 sh_prefix, sh_need;
    __shared__ int sh_done;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* row = static_cast<const T*>(a.logits) + (long long)r * a.ld;
    const SampleRow o = a.rows[r];
    if (a.first) {  // only for a row at its slot's first generated token
        const int slot = a.list[r];
        if (a.pos[slot] != a.n_prompt[slot] - 1) a.first = nullptr;
    }
    const int V = a.V, C = ((V + WAVES - 1) / WAVES + 63) / 64 * 64;
    const int lo = min(V, wave * C), hi = min(V, lo + C);

    // the largest key: its logit is l_max, its id the greedy choice
    u64 best = 0;
    for (int i = lo + lane; i < hi; i += 64) {
        const float l = load_logit(a, row, i);
        if (l > -INFINITY) {
            const u64 k = order_key(l, i);
            best = k > best ? k : best;
        }
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const u64 c = __shfl_xor(best, s, 64);
        best = c > best ? c : best;
    }
    if (lane == 0) red[wave] = best;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) best = red[w] > best ? red[w] : best;
    __syncthreads();
    if (best == 0) {  // no admissible id
        if (tid == 0) {
            if (a.tok) a.tok[r] = -1;
            if (a.keys) a.keys[r] = 0;
            if (a.logp) a.logp[r] = -INFINITY;
        }
        return;
    }
    const float lmax = ord2f((uint32_t)(best >> 20));
    // log of the sum of exp(l - l_max) over the admissible ids
    double lse = 0.0;
    if (a.logp) {
        double s = 0.0;
        for (int i = lo + lane; i < hi; i += 64) {
            const float l = load_logit(a, row, i);
            s += l == lmax ? 1.f : expf(l - lmax);
        }
#pragma unroll
        for (int o2 = 32; o2 > 0; o2 >>= 1) s += __shfl_xor(s, o2, 64);
        if (lane == 0) redd[wave] = s;
        __syncthreads();
        s = 0.0;
        for (int w = 0; w < WAVES; ++w) s += redd[w];
        __syncthreads();
        lse = log(s);
    }
    int token = 0xfffff - (int)(best & 0xfffff);
    if (o.temperature > 0.f) {
        const double invT = 1.0 / (double)o.temperature;
        // weight of an admissible logit; +inf and ids equal to the largest: 2^43
        auto weigh = [&](float l) { return l == lmax ? (u64)ONE : weight(((double)l - (double)lmax) * invT); };
        // Kept so far: key >> shift >= prefix, for each filter (a later one's
        // digits may stop short of telling what an earlier one left out).
        struct Cut { u64 prefix; int shift; } cut[2] = {{0, 0}, {0, 0}};
        // Finds the shortest prefix of the ids kept by cut[0] with `need` ids
        // (by count), or with `share` of their weight, and puts it into `to`.
        auto find = [&](bool by_count, double share, u64 need, Cut& to) {
            int shift = 52, bits = 0;
            u64 prefix = 0;
            for (int pass = 0; pass < 5; ++pass) {
                bits = pass < 2 ? 11 : 10;
                shift -= bits;
                for (int i = tid; i < BINS; i += THREADS) {
                    hw[i] = 0;
                    hc[i] = 0;
                }
                __syncthreads();
                for (int i = lo + lane; i < hi; i += 64) {
                    const float l = load_logit(a, row, i);
                    if (!(l > -INFINITY)) continue;
                    const u64 k = order_key(l, i);
                    if ((k >> cut[0].shift) < cut[0].prefix || (k >> shift >> bits) != prefix) continue;
                    const int d = (int)(k >> shift) & ((1 << bits) - 1);
                    atomicAdd(&hc[d], 1u);
                    if (!by_count) atomicAdd(&hw[d], weigh(l));
                }
                __syncthreads();
                // thread t: digits BINS - 1 - 2 t and the next lower one
                const int d1 = BINS - 1 - 2 * tid, d0 = d1 - 1;
                const u64 m1 = by_count ? hc[d1] : hw[d1], m0 = by_count ? hc[d0] : hw[d0];
                u64 s = m1 + m0;
#pragma unroll
                for (int st = 1; st < 64; st <<= 1) {
                    const u64 c = __shfl_up(s, st, 64);
                    if (lane >= st) s += c;
                }
                if (lane == 63) red[wave] = s;
                if (tid == 0) sh_done = -1;
                __syncthreads();
                u64 before = 0, total = 0;
                for (int w = 0; w < WAVES; ++w) {
                    if (w < wave) before += red[w];
                    total += red[w];
                }
                if (pass == 0) {
                    if (by_count) {
                        if (total <= need) {  // all of them are kept
                            __syncthreads();
                            return;
                        }
                    } else {
                        need = (u64)ceil(share * (double)total);
                        need = need < 1 ? 1 : need > total ? total : need;
                    }
                }
                const u64 e1 = before + s - m0 - m1;  // measure of the digits above d1
                if (e1 < need && e1 + m1 >= need) {
                    sh_prefix = (prefix << bits) | d1;
                    sh_need = need - e1;
                    sh_done = hc[d1] == 1 || e1 + m1 == need ? 1 : 0;
                } else if (e1 + m1 < need && e1 + m1 + m0 >= need) {
                    sh_prefix = (prefix << bits) | d0;
                    sh_need = need - e1 - m1;
                    sh_done = hc[d0] == 1 || e1 + m1 + m0 == need ? 1 : 0;
                }
                __syncthreads();
                prefix = sh_prefix;
                need = sh_need;
                const int done = sh_done;
                __syncthreads();
                if (done != 0) break;
            }
            to = Cut{prefix, shift};
        };
        if (o.top_k > 0) find(true, 0.0, (u64)o.top_k, cut[0]);
        if (o.top_p < 1.f) find(false, (double)o.top_p, 0, cut[1]);
        const double minw = (double)o.min_p * ONE;
        // the kept weights, and the place of u times their sum among them
        auto kept = [&](int i) -> u64 {
            const float l = load_logit(a, row, i);
            const u64 k = order_key(l, i);
            if (!(l > -INFINITY) || (k >> cut[0].shift) < cut[0].prefix || (k >> cut[1].shift) < cut[1].prefix) return 0;
            const u64 w = weigh(l);
            return (double)w >= minw ? w : 0;
        };
        u64 s = 0;
        for (int i = lo + lane; i < hi; i += 64) s += kept(i);
        s = wave_sum64(s);
        if (lane == 0) red[wave] = s;
        __syncthreads();
        u64 total = 0;
        for (int w = 0; w < WAVES; ++w) total += red[w];
        // the first id whose running sum passes u * total, the last kept one at most
        const double u = a.u[r];
        double t = u * (double)total;
        u64 target = t > 0.0 ? (u64)t : 0;  // running sum > target  <=>  running sum > u * total
        if (target >= total) target = total - 1;
        u64 before = 0;
        for (int w = 0; w < wave; ++w) before += red[w];
        if (before > target || before + s <= target) return;  // another wave has it
        for (int i0 = lo; i0 < hi; i0 += 64) {
            const int i = i0 + lane;
            const u64 w = i < hi ? kept(i) : 0;
            u64 c = w;
#pragma unroll
            for (int st = 1; st < 64; st <<= 1) {
                const u64 x = __shfl_up(c, st, 64);
                if (lane >= st) c += x;
            }
            const unsigned long long hit = __ballot(before + c > target);
            if (hit) {
                token = i0 + __builtin_ctzll(hit);
                break;
            }
            before += __shfl(c, 63, 64);
        }
        if (lane != 0) return;
    } else if (tid != 0) {
        return;
    }
    if (a.tok) a.tok[r] = token;
    if (a.keys) a.keys[r] = amax_key(0.f, token);
    if (a.logp) {
        const float l = ldf(row + token);
        a.logp[r] = (float)((l == lmax ? 0.0 : (double)l - (double)lmax) - lse);
    }
}

}  // namespace wmi
