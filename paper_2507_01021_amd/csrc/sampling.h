// Choice of a token per row of logits with temperature, top-k, top-p and
// min-p from one given uniform number.
//
// With l_max the row's largest admissible logit, id i has the weight
//   w_i = round(2^43 exp((l_i - l_max) / T)),
// an integer, so that sums of weights are exact: they depend neither on the
// order of the additions nor on how a row is cut over workgroups, and a row's
// token is the same in every batch. (A weight is off by a unit or two of 2^-43
// of the largest, far less than fp32 sums would be; V is at most 2^20, so a sum
// fits 64 bits.) Ids are ordered by (logit descending, id ascending); each filter
// keeps a prefix of that order, so the filters together keep the shortest.
//
// Four kernels. Three of them cut every row over enough workgroups to fill the
// GPU: sample_max_kernel finds the largest logit; sample_sum_kernel the sum of
// the exponentials and, over 2047 bins of distance from the largest logit, the
// ids (top-k) or the weights (top-p) of every bin, or without both filters the
// weights' sums by position; sample_list_kernel the bin in which the first
// filter cuts. For top-k it lists the ids up to that bin, for top-p alone those
// in it, and adds up the weights of the ids before it by position.
// sample_pick_kernel, a workgroup per row, settles the rest with the list, or
// if that was too long, by further passes over the row.
//
// One row of 51865 fp32 logits: 16.5 us without filters, 27 with top-k 50, 32 with
// top-p 0.9 (launches of 4, 6, 7 and 12 us, each a chain of dependent loads; one
// workgroup that reads the row once per digit of a 52-bit key took 98 to 133).
// 384 rows of 151937 bf16 logits (117 MB): 140 us without filters or with top-k,
// 280 with top-p 0.9, of which the fp64 instructions of the weights (13 of about
// 35 per id) are most. Weights from fp32 exponentials would be off by 2^-22: sums
// of 50000 of them would then put one row in a hundred on the other side of a border.
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
    // workspace of SAMPLE_ROWS rows at most, and the workgroups a row is cut over
    unsigned char* ws;
    int chunks;
};
constexpr int SAMPLE_ROWS = 512;

namespace smp {
constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2048;
constexpr int CUT_WAVES = 4, MAX_CHUNKS = 64;  // waves of the first two kernels' workgroups, workgroups of a row
constexpr int BLOCKS = 512, BLOCK = 64;        // a row's list: blocks of ids, each of one wave's
// What the first three kernels leave of a row for the last.
struct RowWork {
    u64 bins[BINS];                       // by distance: ids, or weights
    u64 sums[MAX_CHUNKS * CUT_WAVES];     // a wave's weights: without filters, or top-p's before the cut's bin
    double exps[MAX_CHUNKS * CUT_WAVES];  // sums of exp(l - l_max)
    float max[MAX_CHUNKS];
    int id[MAX_CHUNKS];                   // lowest id with that maximum
    u64 need;                             // the first cut: what its bin has to give,
    int bin;                              // the bin, or -1 if the filter keeps all
    int n_blocks;                         // blocks of the list (more than BLOCKS: it is not whole)
    unsigned block[BLOCKS];               // wave << 24 | number in the wave << 8 | ids
    u32x2 list[BLOCKS * BLOCK];           // id, logit; a wave's blocks in the order of its ids
};
constexpr double ONE = 8796093022208.0;  // 2^43, the weight of the largest logit

// round(2^43 2^y) for y <= 0: y to the nearest 1/256 by the low bits of a
// sum with 1.5 2^44, its power of two from a table, the rest (2^-9 at most) by
// three terms of the exponential series (the fourth is below 2^-42), the
// integer from the low bits of a sum with 2^52.
__device__ __forceinline__ u64 weight(double y, const double* tab) {
    if (!(y > -44.5)) return 0;  // below half a unit
    const double t = y + 26388279066624.0;
    const int k = (int)__builtin_bit_cast(u64, t);
    const double f = y - (t - 26388279066624.0);
    double p = fma(f, 0.055504108664821580, 0.24022650695910072);
    p = fma(p, f, 0.69314718055994531);
    p = fma(p, f, 1.0);
    const double w = __builtin_amdgcn_ldexp(p * tab[k & 255], (k >> 8) + 43) + 4503599627370496.0;
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

// A row of logits in device memory as one workgroup reads it: 16-byte pieces
// at 16-byte addresses, wave w taking the pieces of one contiguous range of
// ids, so that sums in the order of ids are sums over waves first. The row
// may begin at any element: `shift` elements of its first piece are not its own.
template <class T>
struct LogitRow {
    static constexpr int EL = 16 / sizeof(T);
    const T* row;
    int V, shift, lo, hi;    // the wave's pieces lo .. hi - 1
    int whole_lo, whole_hi;  // pieces all of whose ids are the row's
    const unsigned *never, *first;

    // The pieces of wave `wave` of `waves` that share row r.
    __device__ __forceinline__ LogitRow(const SampleArgs& a, int r, int wave, int waves) {
        row = static_cast<const T*>(a.logits) + (long long)r * a.ld;
        V = a.V;
        shift = (int)(reinterpret_cast<uintptr_t>(row) & 15) / (int)sizeof(T);
        whole_lo = shift ? 1 : 0;
        whole_hi = (V + shift) / EL - 1;
        take(wave, waves);
        never = a.never;
        first = a.first;
        if (first) {  // only for a row at its slot's first generated token
            const int slot = a.list[r];
            if (a.pos[slot] != a.n_prompt[slot] - 1) first = nullptr;
        }
    }
    __device__ __forceinline__ int pieces() const { return (V + shift + EL - 1) / EL; }
    __device__ __forceinline__ int per_wave(int waves) const { return ((pieces() + waves - 1) / waves + 63) / 64 * 64; }
    __device__ __forceinline__ void take(int wave, int waves) {
        lo = min(pieces(), wave * per_wave(waves));
        hi = min(pieces(), lo + per_wave(waves));
    }
    __device__ __forceinline__ int wave_of(int id, int waves) const { return (id + shift) / EL / per_wave(waves); }
    // Piece v as loaded: its 16 bytes and the bits of ids that are left out.
    // Loads of pieces that are not wholly the row's go to a whole one instead,
    // so that a run of loads has no branches; unpack() then reads their ids one by one.
    struct Raw {
        u32x4 x;
        unsigned m;
    };
    __device__ __forceinline__ Raw fetch(int v) const {
        const int id0 = min(max(v, whole_lo), whole_hi) * EL - shift;
        Raw r;
        r.x = *reinterpret_cast<const u32x4*>(row + id0);
        r.m = 0;
        if (never) r.m |= bits(never, id0);
        if (first) r.m |= bits(first, id0);
        return r;
    }
    // Logits of piece v < end, inadmissible ids (filtered, NaN, outside the row) as -inf.
    __device__ __forceinline__ void unpack(int v, int end, const Raw& r, float (&l)[EL]) const {
#pragma unroll
        for (int e = 0; e < EL; ++e) {
            if constexpr (sizeof(T) == 4) l[e] = __uint_as_float(r.x[e]);
            else l[e] = __uint_as_float(e & 1 ? r.x[e >> 1] & 0xffff0000u : r.x[e >> 1] << 16);
            l[e] = ((r.m >> e) & 1u) || !(l[e] > -INFINITY) ? -INFINITY : l[e];
        }
        if (v < whole_lo || v > whole_hi || v >= end) {
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                const int i = v * EL - shift + e;
                l[e] = -INFINITY;
                if (v >= end || i < 0 || i >= V) continue;
                const float y = ldf(row + i);
                const bool out = (never && ((never[i >> 5] >> (i & 31)) & 1u)) || (first && ((first[i >> 5] >> (i & 31)) & 1u));
                l[e] = out || !(y > -INFINITY) ? -INFINITY : y;
            }
        }
    }
    // The mask's bits from id0 on (masks have a word to spare behind the last).
    __device__ __forceinline__ unsigned bits(const unsigned* m, int id0) const {
        const u64 w = (u64)m[id0 >> 5] | (u64)m[(id0 >> 5) + 1] << 32;
        return (unsigned)(w >> (id0 & 31));
    }
    // f(id of the first, logits) for every piece of the wave, lane by lane in
    // turn. The next D pieces are on their way while one is worked on; the body
    // is there once, so that it stays in the instruction cache.
    template <int D, class F>
    __device__ __forceinline__ void each(int lane, F&& f) const {
        const bool any = whole_lo <= whole_hi;
        Raw x[D];
#pragma unroll
        for (int u = 0; u < D; ++u) x[u] = any ? fetch(lo + lane + u * 64) : Raw{};
#pragma unroll 1
        for (int v0 = lo; v0 < hi; v0 += 64) {
            const Raw now = x[0];
#pragma unroll
            for (int u = 0; u + 1 < D; ++u) x[u] = x[u + 1];
            const int v = v0 + lane;
            x[D - 1] = any ? fetch(v + D * 64) : Raw{};
            float l[EL];
            unpack(v, hi, now, l);
            f(v * EL - shift, l);
        }
    }
};

// e^x for x <= 0 with an error of a few 2^-24: the rounding of x log2(e) is
// made up for by a factor. 0 below e^-150, which no sum of 2^20 terms up to 1 feels.
__device__ __forceinline__ float exp_neg(float x) {
    x = fmaxf(x, -150.f);
    const float t = x * 1.44269504f;
    const float lo = fmaf(x, 1.44269504f, -t) + x * 1.925963e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, lo * 0.69314718f, e);
}

// What the options and the largest logit make of a logit.
struct Scale {
    float lmax;
    float unit, per_bin;  // of a distance from lmax
    double top, per;      // the largest logit; log2 of a weight per logit
    u64 least;            // min_p
    const double* tab;
    __device__ __forceinline__ Scale(const SampleRow& o, float m, const double* t) : lmax(m), top(m), tab(t) {
        per = 1.4426950408889634074 / (double)o.temperature;
        // distances that have a weight may exceed fp32 at the highest temperatures, and
        // bins per logit at the lowest (where a logit that exceeds it then has no weight)
        unit = per < 0x1p-100 ? 0.5f : per > 0x1p100 ? 0x1p64f : 1.f;
        per_bin = 2047.f / 45.f * (float)(per / unit);
        least = (u64)ceil((double)o.min_p * ONE);
    }
    // weight of an admissible logit (0 for -inf); the largest, +inf too: 2^43
    __device__ __forceinline__ u64 weigh(float l) const {
        if (lmax == INFINITY) return l == lmax ? (u64)ONE : 0;
        return weight(((double)l - top) * per, tab);
    }
    // bin by distance, as wide as 45 T ln 2 / 2047; 2047: weight 0
    __device__ __forceinline__ int bin(float l) const {
        return l == lmax ? 0 : (int)fminf(fabsf(fmaf(-l, unit, lmax * unit)) * per_bin, 2047.f);
    }
};
__device__ __forceinline__ void fill_table(double* tab) {
    if (threadIdx.x < 256) tab[threadIdx.x] = exp2((double)threadIdx.x / 256.0);
}
// The row's largest logit from its chunks (MAX_CHUNKS lanes).
__device__ __forceinline__ float row_max(const RowWork& w, int chunks, int lane) {
    return wave_max(lane < chunks ? w.max[lane] : -INFINITY);
}
// Inclusive sums over the lanes, and over all lanes.
__device__ __forceinline__ u64 wave_scan64(u64 v, int lane) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) {
        const u64 x = __shfl_up(v, st, 64);
        if (lane >= st) v += x;
    }
    return v;
}
}  // namespace smp

template <class T>
__global__ __launch_bounds__(64 * smp::CUT_WAVES) void sample_max_kernel(SampleArgs a) {
    using namespace smp;
    __shared__ float redf[CUT_WAVES];
    __shared__ int redi[CUT_WAVES];
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const LogitRow<T> row(a, r, blockIdx.x * CUT_WAVES + wave, a.chunks * CUT_WAVES);
    RowWork& ws = reinterpret_cast<RowWork*>(a.ws)[r];
    constexpr int EL = LogitRow<T>::EL;
    for (int i = blockIdx.x * 64 * CUT_WAVES + tid; i < BINS; i += a.chunks * 64 * CUT_WAVES) ws.bins[i] = 0;
    if (blockIdx.x == 0 && tid == 0) ws.n_blocks = 0;
    float m = -INFINITY;
    int id = 0x7fffffff;
    row.template each<4>(lane, [&](int i0, const float (&l)[EL]) __attribute__((always_inline)) {
        float mx = l[0];
#pragma unroll
        for (int e = 1; e < EL; ++e) mx = fmaxf(mx, l[e]);
        if (mx > m) {
            m = mx;
#pragma unroll
            for (int e = EL - 1; e >= 0; --e)
                if (l[e] == mx) id = i0 + e;
        }
    });
    const float wm = wave_max(m);
    if (m != wm) id = 0x7fffffff;
#pragma unroll
    for (int st = 32; st > 0; st >>= 1) id = min(id, __shfl_xor(id, st, 64));
    if (lane == 0) {
        redf[wave] = wm;
        redi[wave] = id;
    }
    __syncthreads();
    if (tid != 0) return;
    for (int w = 1; w < CUT_WAVES; ++w)
        if (redf[w] > redf[0]) {  // ids rise from wave to wave: the first one's is the lowest
            redf[0] = redf[w];
            redi[0] = redi[w];
        }
    ws.max[blockIdx.x] = redf[0];
    ws.id[blockIdx.x] = redi[0];
}

template <class T>
__global__ __launch_bounds__(64 * smp::CUT_WAVES) void sample_sum_kernel(SampleArgs a) {
    using namespace smp;
    __shared__ u64 hw[BINS];
    __shared__ double tab[256];
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int gw = blockIdx.x * CUT_WAVES + wave;
    const LogitRow<T> row(a, r, gw, a.chunks * CUT_WAVES);
    RowWork& ws = reinterpret_cast<RowWork*>(a.ws)[r];
    constexpr int EL = LogitRow<T>::EL;
    const SampleRow o = a.rows[r];
    const float lmax = row_max(ws, a.chunks, lane);
    const bool draws = o.temperature > 0.f && lmax > -INFINITY;
    const bool log_sum = a.logp && lmax > -INFINITY;
    if (!draws && !log_sum) return;
    // top-k counts ids (1), top-p adds weights (2), neither: sums in the order of ids (0)
    const int mode = !draws ? -1 : o.top_k > 0 ? 1 : o.top_p < 1.f ? 2 : 0;
    fill_table(tab);
    for (int i = tid; i < BINS; i += 64 * CUT_WAVES) hw[i] = 0;
    __syncthreads();
    const Scale sc(o, lmax, tab);
    double se = 0.0;
    u64 sum = 0;
    row.template each<4>(lane, [&](int, const float (&l)[EL]) __attribute__((always_inline)) {
        if (log_sum) {
#pragma unroll
            for (int e = 0; e < EL; e += 4) {
                float x = 0.f;
#pragma unroll
                for (int k = e; k < e + 4; ++k) x += l[k] == lmax ? 1.f : exp_neg(l[k] - lmax);
                se += x;
            }
        }
        if (mode == 0) {
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                const u64 w = sc.weigh(l[e]);
                sum += !sc.least || w >= sc.least ? w : 0;
            }
        } else if (mode > 0) {
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                const int b = sc.bin(l[e]);
                if (b < 2047) atomicAdd(&hw[b], mode == 1 ? 1ull : sc.weigh(l[e]));
            }
        }
    });
    if (log_sum) {
#pragma unroll
        for (int st = 32; st > 0; st >>= 1) se += __shfl_xor(se, st, 64);
        if (lane == 0) ws.exps[gw] = se;
    }
    if (mode == 0) {
        sum = wave_sum64(sum);
        if (lane == 0) ws.sums[gw] = sum;
    } else if (mode > 0) {
        __syncthreads();
        // sums of integers: the order of the additions does not matter
        for (int i = tid; i < BINS; i += 64 * CUT_WAVES)
            if (hw[i]) atomicAdd(&ws.bins[i], hw[i]);
    }
}

// Bin of the first cut among the summed bins (every workgroup finds it by
// itself), and the ids up to it (top-k) or in it (top-p alone): each wave lists
// its own in their order, in blocks that it takes from the row's pool.
template <class T>
__global__ __launch_bounds__(64 * smp::CUT_WAVES) void sample_list_kernel(SampleArgs a) {
    using namespace smp;
    constexpr int PER = BINS / (64 * CUT_WAVES);
    __shared__ u64 red[CUT_WAVES];
    __shared__ u64 sh_need;
    __shared__ double tab[256];
    __shared__ int sh_bin;
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int gw = blockIdx.x * CUT_WAVES + wave;
    const SampleRow o = a.rows[r];
    RowWork& ws = reinterpret_cast<RowWork*>(a.ws)[r];
    if (!(o.temperature > 0.f) || (o.top_k <= 0 && !(o.top_p < 1.f))) return;
    const LogitRow<T> row(a, r, gw, a.chunks * CUT_WAVES);
    constexpr int EL = LogitRow<T>::EL;
    const float lmax = row_max(ws, a.chunks, lane);
    if (lmax == -INFINITY) return;
    u64 m[PER], run = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        m[k] = ws.bins[PER * tid + k];
        run += m[k];
    }
    u64 e = wave_scan64(run, lane);
    if (lane == 63) red[wave] = e;
    fill_table(tab);
    if (tid == 0) {
        sh_bin = -1;
        sh_need = 0;
    }
    __syncthreads();
    e -= run;
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < CUT_WAVES; ++w) {
        if (w < wave) e += red[w];
        total += red[w];
    }
    const u64 need = o.top_k > 0 ? (u64)o.top_k : max((u64)1, (u64)ceil((double)o.top_p * (double)total));
    if (total > need) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (e < need && e + m[k] >= need) {
                sh_bin = PER * tid + k;
                sh_need = need - e;
            }
            e += m[k];
        }
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        ws.bin = sh_bin;
        ws.need = sh_need;
    }
    const int bin = sh_bin < 0 ? 2047 : sh_bin;  // 2047: a filter that keeps all ids of some weight
    const bool by_weight = o.top_k <= 0;
    const Scale sc(o, lmax, tab);
    u64 sum = 0;
    int own = 0, last = 0;  // the wave's ids so far, the block it is filling
    row.template each<4>(lane, [&](int i0, const float (&l)[EL]) __attribute__((always_inline)) {
        unsigned in = 0;
#pragma unroll
        for (int x = 0; x < EL; ++x) {
            const int b = sc.bin(l[x]);
            if (b > bin || b == 2047) continue;
            if (!by_weight || b == bin) {
                in |= 1u << x;
            } else {
                const u64 w = sc.weigh(l[x]);
                sum += w >= sc.least ? w : 0;
            }
        }
        if (!__any(in)) return;
        const int c = __popc(in);
        int before = c;
#pragma unroll
        for (int st = 1; st < 64; st <<= 1) {
            const int x = __shfl_up(before, st, 64);
            if (lane >= st) before += x;
        }
        const int n = __shfl(before, 63, 64);
        before -= c;
        // blocks first .. first + more - 1 of the wave are new: numbers base on
        const int first = (own + BLOCK - 1) / BLOCK, more = (own + n + BLOCK - 1) / BLOCK - first;
        int base = 0;
        if (more) {
            if (lane == 0) base = atomicAdd(&ws.n_blocks, more);
            base = __shfl(base, 0, 64);
        }
#pragma unroll
        for (int x = 0; x < EL; ++x) {
            if (!((in >> x) & 1u)) continue;
            const int p = own + before++, q = p / BLOCK, at = q < first ? last : base + q - first;
            if (at < BLOCKS) ws.list[at * BLOCK + p % BLOCK] = u32x2{(unsigned)(i0 + x), __float_as_uint(l[x])};
        }
        own += n;
        // how full every block is that this run has touched
        const int q = max(first - 1, 0) + lane, at = q < first ? last : base + q - first;
        if (q * BLOCK < own && at < BLOCKS)
            ws.block[at] = (unsigned)gw << 24 | (unsigned)(q & 0xffff) << 8 | (unsigned)min(BLOCK, own - q * BLOCK);
        if (more) last = base + more - 1;
    });
    if (by_weight) {
        sum = wave_sum64(sum);
        if (lane == 0) ws.sums[gw] = sum;
    }
}

template <class T>
__global__ __launch_bounds__(smp::THREADS) void sample_pick_kernel(SampleArgs a) {
    using namespace smp;
    constexpr int BIN_IDS = THREADS;         // ids of a cut's bin that are ranked at once
    __shared__ u64 hw[BINS];
    __shared__ u64 lk[BIN_IDS], lw[BIN_IDS];
    __shared__ unsigned block[BLOCKS];
    __shared__ u64 sums[MAX_CHUNKS * CUT_WAVES];
    __shared__ int in_order[BLOCKS];  // the list's blocks in the order of ids: number << 8 | ids
    __shared__ u64 red[WAVES];
    __shared__ double tab[256];
    __shared__ u64 sh_cut, sh_need;
    __shared__ int sh_bin, n_ids;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    LogitRow<T> row(a, r, wave, WAVES);
    const RowWork& ws = reinterpret_cast<const RowWork*>(a.ws)[r];
    const SampleRow o = a.rows[r];
    const float u = a.u[r];
    constexpr int EL = LogitRow<T>::EL;
    constexpr int PER = MAX_CHUNKS * CUT_WAVES / 64;  // sums of the second kernel's waves per lane
    const int cut_waves = a.chunks * CUT_WAVES;

    const float lmax = row_max(ws, a.chunks, lane);
    if (lmax == -INFINITY) {  // no admissible id
        if (tid == 0) {
            if (a.tok) a.tok[r] = -1;
            if (a.keys) a.keys[r] = 0;
            if (a.logp) a.logp[r] = -INFINITY;
        }
        return;
    }
    double se = 0.0;
    if (a.logp) {
#pragma unroll
        for (int k = 0; k < PER; ++k) se += PER * lane + k < cut_waves ? ws.exps[PER * lane + k] : 0.0;
#pragma unroll
        for (int st = 32; st > 0; st >>= 1) se += __shfl_xor(se, st, 64);
    }
    // writes the row's results (one thread)
    auto finish = [&](int token, float l) __attribute__((always_inline)) {
        if (a.tok) a.tok[r] = token;
        if (a.keys) a.keys[r] = amax_key(0.f, token);
        if (a.logp) a.logp[r] = (float)((l == lmax ? 0.0 : (double)l - (double)lmax) - log(se));
    };
    if (!(o.temperature > 0.f)) {
        // ids rise from chunk to chunk: the first that has the maximum
        const unsigned long long has = __ballot(lane < a.chunks && ws.max[min(lane, a.chunks - 1)] == lmax);
        if (tid == 0) finish(ws.id[__builtin_ctzll(has)], lmax);
        return;
    }
    fill_table(tab);
    const Scale sc(o, lmax, tab);
    // where u falls: the first id whose running sum passes u * total, the last kept one at most
    auto target_of = [&](u64 total) __attribute__((always_inline)) {
        const double t = (double)u * (double)total;
        const u64 x = t > 0.0 ? (u64)t : 0;  // an integer passes t if it passes t's integer part
        return x < total ? x : total - 1;
    };
    float cut_l = -INFINITY;  // kept: larger logits, and equal ones up to id cut_id
    int cut_id = -1;
    auto kept = [&](int i, float l) __attribute__((always_inline)) { return l > cut_l || (l == cut_l && i <= cut_id); };

    // All ids of the row, or if there is a whole list, of the list, are gone
    // through once per stage: BIN adds up the bins, RANK lists the ids of the
    // cut's bin, DIGIT adds up digits of their keys if they are too many, SUM
    // adds the kept weights. Cut 0 is top-k's (every id measures 1), cut 1
    // top-p's (an id measures its weight); the first of them has its bin already.
    enum { BIN, RANK, DIGIT, SUM };
    int cut = o.top_k > 0 ? 0 : o.top_p < 1.f ? 1 : 2;
    const bool none = cut == 2, by_weight = cut == 1;  // no filter, top-p alone
    int stage = BIN, digit = 0, shift = 52, nb = 0, bin = -1;
    u64 prefix = 0, sum = 0;
    const int n_blocks = ws.n_blocks;
    const bool listed = !none && n_blocks <= BLOCKS;
    // the sums by position are there: all of them, or (top-p) but for the cut's bin
    const bool summed = none || (by_weight && listed);
    if (!none) {
        if (ws.bin >= 0) stage = RANK;
        else ++cut;  // it keeps all
        if (tid == 0) {
            sh_bin = ws.bin;
            sh_need = ws.need;
        }
    }
    if (listed) {
        // the list's blocks in the order of their waves and numbers
        for (int i = tid; i < n_blocks; i += THREADS) block[i] = ws.block[i];
        __syncthreads();
        for (int i = tid; i < n_blocks; i += THREADS) {
            const unsigned k = block[i];
            int before = 0;
#pragma unroll 8
            for (int j = 0; j < n_blocks; ++j) before += block[j] < k;
            in_order[before] = i << 8 | (int)(k & 0xff);
        }
    }
    // this wave's blocks
    const int b_lo = n_blocks * wave / WAVES, b_hi = n_blocks * (wave + 1) / WAVES;
    auto visit = [&](int i, float l) __attribute__((always_inline)) {
        const int b = sc.bin(l);
        if (!kept(i, l) || b == 2047 || ((stage == RANK || stage == DIGIT) && b != bin)) return;
        if (stage == RANK) {
            const int at = atomicAdd(&n_ids, 1);
            if (at < BIN_IDS) lk[at] = order_key(l, i);
            return;
        }
        const u64 w = cut == 0 ? 1 : sc.weigh(l);
        if (stage == SUM) {
            sum += w >= sc.least ? w : 0;
        } else if (stage == BIN) {
            atomicAdd(&hw[b], w);
        } else {
            const u64 k = order_key(l, i);
            if ((k >> shift >> nb) == prefix) atomicAdd(&hw[(k >> shift) & ((1 << nb) - 1)], w);
        }
    };
    // f(id, logit) for this wave's listed ids, 64 at a time (-inf: a lane
    // without one), until it returns true; the next blocks are on their way meanwhile
    auto each_listed = [&](auto&& f) __attribute__((always_inline)) {
        constexpr int D = 4;
        u32x2 x[D];
        int n[D];
        auto fetch = [&](int b, u32x2& y, int& m) __attribute__((always_inline)) {
            const int q = b < b_hi ? in_order[b] : 0;
            m = q & 0xff;
            y = ws.list[(q >> 8) * BLOCK + lane];
        };
#pragma unroll
        for (int u = 0; u < D; ++u) fetch(b_lo + u, x[u], n[u]);
#pragma unroll 1
        for (int b = b_lo; b < b_hi; ++b) {
            const u32x2 y = x[0];
            const int m = n[0];
#pragma unroll
            for (int u = 0; u + 1 < D; ++u) {
                x[u] = x[u + 1];
                n[u] = n[u + 1];
            }
            fetch(b + D, x[D - 1], n[D - 1]);
            if (f((int)y.x, lane < m ? __uint_as_float(y.y) : -INFINITY)) break;
        }
    };
    for (;;) {
        if (stage == BIN && cut == 0 && o.top_k <= 0) cut = 1;
        if (stage == BIN && cut == 1 && !(o.top_p < 1.f)) cut = 2;
        if (cut == 2) stage = SUM;
        if (cut == 2 && summed) break;
        nb = digit < 2 ? 11 : 10;
        if (stage == DIGIT) shift -= nb;
        if (stage == BIN || stage == DIGIT)
            for (int i = tid; i < BINS; i += THREADS) hw[i] = 0;
        if (tid == 0) n_ids = 0;
        __syncthreads();
        bin = sh_bin;
        if (listed) {
            each_listed([&](int i, float l) __attribute__((always_inline)) {
                if (l > -INFINITY) visit(i, l);
                return false;
            });
        } else {
            row.template each<4>(lane, [&](int i0, const float (&l)[EL]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < EL; ++e) visit(i0 + e, l[e]);
            });
        }
        if (stage == SUM) break;
        __syncthreads();
        if (stage == RANK) {
            const int n = n_ids;
            __syncthreads();
            if (n > BIN_IDS) {  // 11 11 10 bits of the logit, 10 10 of the id
                stage = DIGIT;
                digit = 0;
                shift = 52;
                prefix = 0;
                continue;
            }
            // thread t has the bin's id t, and adds up what comes before it
            const u64 k = tid < n ? lk[tid] : 0;
            const u64 w = cut == 0 ? 1 : sc.weigh(ord2f((uint32_t)(k >> 20)));
            lw[tid] = w;
            __syncthreads();
            if (tid < n) {
                u64 before = 0;
#pragma unroll 4
                for (int j = 0; j < n; ++j) before += lk[j] > k ? lw[j] : 0;
                if (before < sh_need && before + w >= sh_need) sh_cut = k;
            }
            __syncthreads();
            prefix = sh_cut;
        } else {
            // bins by distance, digits highest first: thread t takes the places 2 t and 2 t + 1
            const int p0 = stage == BIN ? 2 * tid : BINS - 1 - 2 * tid, p1 = stage == BIN ? p0 + 1 : p0 - 1;
            const u64 m0 = hw[p0], m1 = hw[p1];
            const u64 run = wave_scan64(m0 + m1, lane);
            if (lane == 63) red[wave] = run;
            if (tid == 0 && stage == BIN) sh_bin = -1;
            __syncthreads();
            u64 e = run - m0 - m1, total = 0;  // measure before place 2 t
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) e += red[w];
                total += red[w];
            }
            u64 need = sh_need;
            if (stage == BIN) need = cut == 0 ? (u64)o.top_k : max((u64)1, (u64)ceil((double)o.top_p * (double)total));
            __syncthreads();
            if (total > need || stage == DIGIT) {
                const bool first = e < need && e + m0 >= need;
                if (first || (e + m0 < need && e + m0 + m1 >= need)) {
                    sh_need = first ? need - e : need - e - m0;  // still wanted from this place
                    if (stage == BIN) sh_bin = first ? p0 : p1;
                    else sh_cut = prefix << nb | (u64)(first ? p0 : p1);
                }
            }
            __syncthreads();
            if (stage == BIN) {
                if (sh_bin < 0) ++cut;  // nothing is cut off
                else stage = RANK;
                continue;
            }
            prefix = sh_cut;
            if (++digit < 5) continue;
        }
        cut_l = ord2f((uint32_t)(prefix >> 20));
        cut_id = 0xfffff - (int)(prefix & 0xfffff);
        ++cut;
        stage = BIN;
        __syncthreads();
    }

    // The place of u times the sum of the kept weights. The waves' sums, in the
    // order of their ids, say which wave's ids it is among.
    const int waves = summed ? cut_waves : WAVES;
    if (summed) {
        for (int i = tid; i < cut_waves; i += THREADS) sums[i] = ws.sums[i];
        __syncthreads();
        if (by_weight)  // and the kept ids of the cut's bin
            each_listed([&](int i, float l) __attribute__((always_inline)) {
                if (!(l > -INFINITY) || !kept(i, l)) return false;
                const u64 w = sc.weigh(l);
                if (w >= sc.least) atomicAdd(&sums[row.wave_of(i, cut_waves)], w);
                return false;
            });
    } else {
        sum = wave_sum64(sum);
        if (lane == 0) sums[wave] = sum;
    }
    __syncthreads();
    u64 part[PER], mine = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int w = PER * lane + k;
        part[k] = w < waves ? sums[w] : 0;
        mine += part[k];
    }
    u64 run = wave_scan64(mine, lane);
    const u64 target = target_of(__shfl(run, 63, 64));
    const int at_lane = __builtin_ctzll(__ballot(run > target));
    run -= mine;
    int owner = PER * lane;
#pragma unroll
    for (int k = 0; k < PER - 1; ++k)
        if (owner == PER * lane + k && run + part[k] <= target) {
            run += part[k];
            ++owner;
        }
    owner = __shfl(owner, at_lane, 64);
    u64 before = __shfl(run, at_lane, 64);
    if (listed && !summed) {
        if (wave != owner) return;
        each_listed([&](int i, float l) __attribute__((always_inline)) {
            u64 w = l > -INFINITY && kept(i, l) ? sc.weigh(l) : 0;
            if (w < sc.least) w = 0;
            const u64 c = wave_scan64(w, lane);
            const unsigned long long hit = __ballot(before + c > target);
            if (hit && lane == __builtin_ctzll(hit)) finish(i, l);
            before += __shfl(c, 63, 64);
            return hit != 0;
        });
        return;
    }
    // the owner's pieces, 64 at a time, are added up by all of this workgroup's waves
    row.take(owner, waves);
    const int lo = row.lo, hi = row.hi;
    auto piece = [&](int v, float (&l)[EL], u64 (&w)[EL]) __attribute__((always_inline)) {
        typename LogitRow<T>::Raw x{};
        if (row.whole_lo <= row.whole_hi) x = row.fetch(v);
        row.unpack(v, hi, x, l);
        u64 c = 0;
#pragma unroll
        for (int e = 0; e < EL; ++e) {
            w[e] = kept(v * EL + e - row.shift, l[e]) ? sc.weigh(l[e]) : 0;
            if (w[e] < sc.least) w[e] = 0;
            c += w[e];
        }
        return c;
    };
    float l[EL];
    u64 w[EL];
    for (int g = wave; lo + g * 64 < hi; g += WAVES) {
        const u64 c = wave_sum64(piece(lo + g * 64 + lane, l, w));
        if (lane == 0) hw[g] = c;
    }
    __syncthreads();
    int g = 0;
    for (; lo + (g + 1) * 64 < hi && before + hw[g] <= target; ++g) before += hw[g];
    if (wave != g % WAVES) return;
    const int v = lo + g * 64 + lane;
    const u64 all = piece(v, l, w), c = wave_scan64(all, lane);
    if (lane != __builtin_ctzll(__ballot(before + c > target))) return;
    u64 at = before + c - all;
    int e = 0;
    float lt = l[0];
#pragma unroll
    for (int x = 0; x < EL; ++x) {
        if (at <= target) {
            e = x;
            lt = l[x];
        }
        at += w[x];
    }
    finish(v * EL + e - row.shift, lt);
}

// Workgroups that a row of V logits is cut over when n rows are drawn at a
// time: as many as fill 256 CUs four times, if every wave has 128 pieces of 16 bytes.
template <class T>
inline int sample_chunks(int n, int V) {
    const int pieces = V / (16 / (int)sizeof(T)) + 1;
    const int most = (pieces + 128 * smp::CUT_WAVES - 1) / (128 * smp::CUT_WAVES), want = (1024 + n - 1) / n;
    const int c = want < most ? want : most;
    return c < 1 ? 1 : c > smp::MAX_CHUNKS ? smp::MAX_CHUNKS : c;
}
inline size_t sample_ws_bytes(int rows) {
    return sizeof(smp::RowWork) * (size_t)(rows < SAMPLE_ROWS ? rows : SAMPLE_ROWS);
}
// The choice for n rows; a.ws has sample_ws_bytes(n). `filters`: some row may
// have top-k or top-p.
template <class T>
inline void sample_rows(SampleArgs a, int n, bool filters, hipStream_t st) {
    for (int r = 0; r < n; r += SAMPLE_ROWS) {
        const int m = n - r < SAMPLE_ROWS ? n - r : SAMPLE_ROWS;
        SampleArgs b = a;
        b.logits = static_cast<const T*>(a.logits) + (long long)r * a.ld;
        b.rows += r;
        b.u += r;
        if (b.tok) b.tok += r;
        if (b.logp) b.logp += r;
        b.chunks = sample_chunks<T>(m, a.V);
        hipLaunchKernelGGL(sample_max_kernel<T>, dim3(b.chunks, m), dim3(64 * smp::CUT_WAVES), 0, st, b);
        hipLaunchKernelGGL(sample_sum_kernel<T>, dim3(b.chunks, m), dim3(64 * smp::CUT_WAVES), 0, st, b);
        if (filters) hipLaunchKernelGGL(sample_list_kernel<T>, dim3(b.chunks, m), dim3(64 * smp::CUT_WAVES), 0, st, b);
        hipLaunchKernelGGL(sample_pick_kernel<T>, dim3(m), dim3(smp::THREADS), 0, st, b);
    }
}

}  // namespace wmi
