// The likeliest continuations of groups of beams.
//
// Beam b of a group has a score c_b, the log-probability of what it holds, and
// a row of logits; continuation (b, i) has
//   c_b + l_i - log(sum over j of exp(l_j)),
// the sum over the ids that are not suppressed. A group's n best are wanted, in
// descending order, equal ones by (b, i).
//
// Two kernels. beam_rows_kernel cuts every row over workgroups: in one pass it
// adds up exponentials and keeps the n largest logits of its piece. Within a row
// the order of the logits is that of the continuations, so a row's n largest
// are enough. beam_pick_kernel, a workgroup per group, joins the pieces' sums and
// picks from their lists.
// Scores of different beams may lie close together, so sums, logarithms and
// scores are fp64: exponentials of fp32 would be off by 2^-23 of a weight, and
// one choice in some thousands would be another. An fp64 exponential is 16 of some
// 24 instructions per id.
#pragma once

#include "beam.h"
#include "common.h"

namespace wmi {

typedef unsigned long long u64;

struct BeamArgs {
    const void* logits;
    long long ld;
    int V, width, best;
    const unsigned* never;  // [V / 32 + 1] ids never chosen, or null
    const float* scores;
    int* parents;
    int* tokens;
    float* out;
    // per (row, piece): the sum and what its exponents were taken from; the largest logits' keys
    unsigned char* ws;
    int chunks;
};
constexpr int BEAM_ROWS = 512, BEAM_WGS = 1024;  // rows a launch, workgroups that rows are cut into

namespace bm {
constexpr int WAVES = 4, THREADS = 64 * WAVES;
struct Piece {
    double sum;  // of exp(l - ref); ref = +inf: how many logits are
    float ref;   // -inf: no admissible id
    int n;       // keys
    u64 key[BEAM_BEST];
};

// e^x for x <= 700 with a relative error of 2 10^-12 (x log2(e) as an integer
// and a rest; 2^rest by Chebyshev interpolation of degree 8 on [-1/2, 1/2]).
// Anything below -700, and NaN, counts as -700: 10^-304.
__device__ __forceinline__ double exp_sum(double x) {
    const double y = fmax(x, -700.0) * 1.4426950408889634074;
    const double k = rint(y), f = y - k;
    double p = fma(f, 1.3255179556479267e-06, 1.5310080611926545e-05);
    p = fma(p, f, 0.00015403456082633648);
    p = fma(p, f, 0.0013333450563173552);
    p = fma(p, f, 0.009618129159053034);
    p = fma(p, f, 0.055504109412108156);
    p = fma(p, f, 0.24022650695814518);
    p = fma(p, f, 0.6931471805459332);
    p = fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)k);
}

// A row of logits as a wave reads it: pieces of 16 bytes' worth of ids, counted
// from the row's first id wherever that lies (16-byte loads need no alignment
// here), so that a row's sums are the same at every address: beams that are
// alike stay equal to the last bit.
template <class T>
struct Row {
    static constexpr int EL = 16 / sizeof(T);
    typedef unsigned Raw128 __attribute__((ext_vector_type(4), aligned(2)));
    const T* row;
    int V, whole, lo, hi;  // pieces all of whose ids there are; the wave's pieces lo .. hi - 1
    const unsigned* never;
    __device__ __forceinline__ Row(const BeamArgs& a, int r, int wave, int waves) {
        row = static_cast<const T*>(a.logits) + (long long)r * a.ld;
        V = a.V;
        never = a.never;
        whole = V / EL;
        const int pieces = (V + EL - 1) / EL, per = ((pieces + waves - 1) / waves + 63) / 64 * 64;
        lo = min(pieces, wave * per);
        hi = min(pieces, lo + per);
    }
    struct Raw {
        u32x4 x;
        unsigned m;
    };
    // Piece v, or the last whole one instead, and the bits of its suppressed ids.
    __device__ __forceinline__ Raw fetch(int v) const {
        const int id0 = min(v, whole - 1) * EL;
        Raw r;
        r.x = *reinterpret_cast<const Raw128*>(row + id0);
        r.m = never ? never[id0 >> 5] >> (id0 & 31) : 0;
        return r;
    }
    // Its logits; -inf for suppressed ids, NaN, and ids that there are not.
    __device__ __forceinline__ void unpack(int v, const Raw& r, float (&l)[EL]) const {
#pragma unroll
        for (int e = 0; e < EL; ++e) {
            if constexpr (sizeof(T) == 4) l[e] = __uint_as_float(r.x[e]);
            else l[e] = __uint_as_float(e & 1 ? r.x[e >> 1] & 0xffff0000u : r.x[e >> 1] << 16);
            l[e] = ((r.m >> e) & 1u) || !(l[e] > -INFINITY) ? -INFINITY : l[e];
        }
        if (v >= whole || v >= hi) {
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                const int i = v * EL + e;
                l[e] = -INFINITY;
                if (v >= hi || i >= V) continue;
                const float y = ldf(row + i);
                l[e] = (never && (never[i >> 5] >> (i & 31) & 1u)) || !(y > -INFINITY) ? -INFINITY : y;
            }
        }
    }
    // f(id of the first, logits) for the wave's pieces, 64 at a time; the next D
    // are on their way while one is worked on.
    template <int D, class F>
    __device__ __forceinline__ void each(int lane, F&& f) const {
        Raw x[D];
#pragma unroll
        for (int u = 0; u < D; ++u) x[u] = whole > 0 ? fetch(lo + lane + u * 64) : Raw{};
#pragma unroll 1
        for (int v0 = lo; v0 < hi; v0 += 64) {
            const Raw now = x[0];
#pragma unroll
            for (int u = 0; u + 1 < D; ++u) x[u] = x[u + 1];
            const int v = v0 + lane;
            x[D - 1] = whole > 0 ? fetch(v + D * 64) : Raw{};
            float l[EL];
            unpack(v, now, l);
            f(v * EL, l);
        }
    }
};

// Keys of a wave's or workgroup's largest logits, unordered: key[i] of n.
// Moves the `best` largest to the front, in descending order (all of the
// waves that share it call this; `lanes` threads of which this is number t).
// Keys are distinct, so an entry's place is the number of larger ones.
template <int CAP, int LANES, class Sync>
__device__ __forceinline__ int keep_best(u64* key, int n, int best, int t, Sync&& sync) {
    constexpr int PER = (CAP + LANES - 1) / LANES;
    u64 mine[PER];
    int place[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = t + u * LANES;
        mine[u] = i < n ? key[i] : 0;
        place[u] = 0;
    }
    const int turns = (n + LANES - 1) / LANES;
    for (int j = 0; j < n; ++j) {
        const u64 k = key[j];
#pragma unroll
        for (int u = 0; u < PER; ++u)
            if (u < turns) place[u] += k > mine[u];
    }
    sync();
#pragma unroll
    for (int u = 0; u < PER; ++u)
        if (t + u * LANES < n && place[u] < best) key[place[u]] = mine[u];
    sync();
    return n < best ? n : best;
}

// The k-th largest (k >= 1) of the lanes' numbers.
__device__ __forceinline__ float kth_largest(float x, int k, int lane) {
    int before = 0;  // lanes with a larger number, or an equal one and a lower lane
#pragma unroll
    for (int i = 0; i < 64; ++i) {
        const float y = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
        before += y > x || (y == x && i < lane);
    }
    const unsigned long long at = __ballot(before == k - 1);
    return __shfl(x, __builtin_ctzll(at), 64);
}
}  // namespace bm

// Whether a beam of that score is there.
__device__ __forceinline__ bool beam_lives(float score) { return fabsf(score) < INFINITY; }

template <class T>
__global__ __launch_bounds__(bm::THREADS) void beam_rows_kernel(BeamArgs a) {
    using namespace bm;
    constexpr int EL = Row<T>::EL;
    constexpr int FULL = 128, CAP = FULL + 64 * EL;  // a wave's keys: put in order when there are more than FULL
    __shared__ u64 key[WAVES][CAP];
    __shared__ double wsum[WAVES];
    __shared__ float wref[WAVES];
    __shared__ int wn[WAVES];
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (!beam_lives(a.scores[r])) return;
    const Row<T> row(a, r, blockIdx.x * WAVES + wave, a.chunks * WAVES);
    u64* mine = key[wave];
    auto sync = [] {  // a wave's LDS accesses are in order; the compiler keeps them so
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    float ref = -INFINITY, thr = -INFINITY;
    double sum = 0.0;
    int n = 0;
    row.template each<4>(lane, [&](int i0, const float (&l)[EL]) __attribute__((always_inline)) {
        float mx = l[0];
#pragma unroll
        for (int e = 1; e < EL; ++e) mx = fmaxf(mx, l[e]);
        if (mx > ref + 100.f) {  // exponents are small enough for fp64 till then
            sum = ref == -INFINITY ? 0.0 : sum * exp_sum((double)ref - (double)mx);
            if (mx == INFINITY) sum = 0.0;
            ref = mx;
        }
        if (ref == INFINITY) {
#pragma unroll
            for (int e = 0; e < EL; ++e) sum += l[e] == INFINITY ? 1.0 : 0.0;
        } else if (ref > -INFINITY) {
#pragma unroll
            for (int e = 0; e < EL; ++e) sum += exp_sum((double)l[e] - (double)ref);
        }
        // logits above the wave's n-th largest so far
        unsigned long long some = __ballot(mx > thr);
        if (!some) return;
        if (__popcll(some) > FULL / 4) {  // too many to list: at least n are no smaller than the n-th largest lane's
            const float x = kth_largest(mx, a.best, lane);
            if (x > thr) thr = x == 0.f ? -1e-45f : ord2f(f2ord(x) - 1);  // (equal ones count)
        }
#pragma unroll
        for (int e = 0; e < EL; ++e) {
            const unsigned long long in = __ballot(l[e] > thr);
            if (l[e] > thr)
                mine[n + __popcll(in & ((1ull << lane) - 1))] = amax_key(l[e] + 0.f, i0 + e);  // (-0 and 0 are equal)
            n += __popcll(in);
        }
        if (n > FULL) {
            sync();
            n = keep_best<CAP, 64>(mine, n, a.best, lane, sync);
            if (n == a.best) thr = fmaxf(thr, ord2f((uint32_t)(mine[n - 1] >> 32)));
        }
    });
    // the lanes' sums to one exponent: the largest of theirs
    const float top = wave_max(ref);
    if (top == INFINITY) sum = ref == INFINITY ? sum : 0.0;
    else sum = ref == -INFINITY ? 0.0 : sum * exp_sum((double)ref - (double)top);
#pragma unroll
    for (int st = 32; st > 0; st >>= 1) sum += __shfl_xor(sum, st, 64);
    sync();
    n = keep_best<CAP, 64>(mine, n, a.best, lane, sync);
    if (lane == 0) {
        wsum[wave] = sum;
        wref[wave] = top;
        wn[wave] = n;
    }
    __syncthreads();
    // the waves' lists as one
    const float t = fmaxf(fmaxf(wref[0], wref[1]), fmaxf(wref[2], wref[3]));
    Piece& out = reinterpret_cast<Piece*>(a.ws)[(long long)r * a.chunks + blockIdx.x];
    int total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += wn[w];
    // thread: one key of a wave (best <= 64)
    if (lane < wn[wave]) {
        const u64 k = mine[lane];
        int place = lane;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) continue;
            for (int j = 0; j < wn[w]; ++j) place += key[w][j] > k;
        }
        if (place < a.best) out.key[place] = k;
    }
    if (tid == 0) {
        double y = 0.0;
        for (int w = 0; w < WAVES; ++w) {
            if (wref[w] == -INFINITY) continue;
            if (t == INFINITY) y += wref[w] == INFINITY ? wsum[w] : 0.0;
            else y += wsum[w] * exp_sum((double)wref[w] - (double)t);
        }
        out.sum = y;
        out.ref = t;
        out.n = min(total, a.best);
    }
}

// A group's n best from its pieces' lists (each in descending order). Lists as
// long as j + 1 hold at least (lists) (j + 1) continuations no worse than their
// j-th, so one of those entries is a bound below which nothing can be among
// the n best; what is left is put in order by counting.
static __global__ __launch_bounds__(256) void beam_pick_kernel(BeamArgs a) {
    using namespace bm;
    constexpr int CAP = BEAM_WGS;  // lists at most
    __shared__ double off[BEAM_WIDTH];   // score - log(sum)
    __shared__ float refs[BEAM_WIDTH];
    __shared__ double val[CAP];
    __shared__ int idx[CAP];
    __shared__ double bound[4];
    __shared__ int count;
    __shared__ double sh_val;
    __shared__ int sh_idx;
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Piece* pieces = reinterpret_cast<const Piece*>(a.ws) + (long long)g * a.width * a.chunks;
    const int lists = a.width * a.chunks;
    // a wave per row
    for (int b = wave; b < a.width; b += 4) {
        const float c = a.scores[g * a.width + b];
        float t = -INFINITY;
        double y = 0.0;
        if (beam_lives(c)) {
            for (int k = lane; k < a.chunks; k += 64) t = fmaxf(t, pieces[b * a.chunks + k].ref);
            t = wave_max(t);
            for (int k = lane; k < a.chunks; k += 64) {
                const Piece& p = pieces[b * a.chunks + k];
                if (p.ref == -INFINITY) continue;
                if (t == INFINITY) y += p.ref == INFINITY ? p.sum : 0.0;
                else y += p.sum * exp_sum((double)p.ref - (double)t);
            }
#pragma unroll
            for (int st = 32; st > 0; st >>= 1) y += __shfl_xor(y, st, 64);
        }
        if (lane == 0) {
            refs[b] = t;  // -inf: no continuation
            off[b] = t == -INFINITY ? 0.0 : log(y);
        }
    }
    if (tid == 0) count = 0;
    __syncthreads();
    // entry e of list i (i = row * chunks + piece): its score, or -inf
    auto score = [&](int i, int e, int& at) __attribute__((always_inline)) {
        const int b = i / a.chunks;
        at = 0x7fffffff;
        if (refs[b] == -INFINITY || e >= pieces[i].n) return -(double)INFINITY;
        const u64 k = pieces[i].key[e];
        const float l = ord2f((uint32_t)(k >> 32));
        if (refs[b] == INFINITY && l != INFINITY) return -(double)INFINITY;
        const int id = (int)(0xffffffffu - (unsigned)k);
        at = b * a.V + id;
        return (double)a.scores[g * a.width + b] + ((refs[b] == INFINITY ? 0.0 : (double)l - (double)refs[b]) - off[b]);
    };
    // the bound: the k-th largest of the lists' j-th entries, k (j + 1) >= best
    const int j = (a.best + lists - 1) / lists - 1, k = (a.best + j) / (j + 1);
    for (int i = tid; i < lists; i += 256) {
        int at;
        val[i] = score(i, j, at);
    }
    __syncthreads();
    for (int i = tid; i < lists; i += 256) {
        const double x = val[i];
        int before = 0;
        for (int q = 0; q < lists; ++q) before += val[q] > x || (val[q] == x && q < i);
        if (before == k - 1) bound[0] = x;
    }
    __syncthreads();
    const double low = bound[0];
    __syncthreads();
    for (int i = tid; i < lists; i += 256) {
        for (int e = 0; e < a.best; ++e) {
            int at;
            const double x = score(i, e, at);
            if (!(x >= low) || x == -(double)INFINITY) break;  // lists descend
            const int p = atomicAdd(&count, 1);
            if (p < CAP) {
                val[p] = x;
                idx[p] = at;
            }
        }
    }
    __syncthreads();
    const int n = count;
    int* parents = a.parents + g * a.best;
    int* tokens = a.tokens + g * a.best;
    float* out = a.out + g * a.best;
    auto put = [&](int place, double x, int at) __attribute__((always_inline)) {
        parents[place] = at / a.V;
        tokens[place] = at - at / a.V * a.V;
        out[place] = (float)x;
    };
    if (n <= CAP) {
        for (int i = tid; i < n; i += 256) {
            const double x = val[i];
            const int at = idx[i];
            int place = 0;
            for (int q = 0; q < n; ++q) place += val[q] > x || (val[q] == x && idx[q] < at);
            if (place < a.best) put(place, x, at);
        }
        for (int i = n + tid; i < a.best; i += 256) {
            parents[i] = tokens[i] = -1;
            out[i] = -INFINITY;
        }
        return;
    }
    // many equal ones: the next best after the last, one by one
    double last = (double)INFINITY;
    int last_at = -1;
    for (int m = 0; m < a.best; ++m) {
        double bx = -(double)INFINITY;
        int bi = 0x7fffffff;
        for (int i = tid; i < lists; i += 256) {
            for (int e = 0; e < a.best; ++e) {
                int at;
                const double x = score(i, e, at);
                if (x == -(double)INFINITY) break;
                if (x > last || (x == last && at <= last_at)) continue;  // chosen already
                if (x > bx || (x == bx && at < bi)) {
                    bx = x;
                    bi = at;
                }
            }
        }
#pragma unroll
        for (int st = 32; st > 0; st >>= 1) {
            const double x = __shfl_xor(bx, st, 64);
            const int i = __shfl_xor(bi, st, 64);
            if (x > bx || (x == bx && i < bi)) {
                bx = x;
                bi = i;
            }
        }
        if (lane == 0) {
            bound[wave] = bx;
            idx[wave] = bi;
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < 4; ++w)
                if (bound[w] > bound[0] || (bound[w] == bound[0] && idx[w] < idx[0])) {
                    bound[0] = bound[w];
                    idx[0] = idx[w];
                }
            sh_val = bound[0];
            sh_idx = idx[0];
            if (bound[0] > -(double)INFINITY) {
                put(m, bound[0], idx[0]);
            } else {
                parents[m] = tokens[m] = -1;
                out[m] = -INFINITY;
            }
        }
        __syncthreads();
        last = sh_val;
        last_at = sh_idx;
    }
}

// Workgroups that a row of V logits is cut over when n rows are looked at: as
// many as fill 256 CUs four times, if every wave has 128 pieces of 16 bytes.
template <class T>
inline int beam_chunks(int n, int V) {
    const int pieces = V / (16 / (int)sizeof(T)) + 1;
    const int most = (pieces + 128 * bm::WAVES - 1) / (128 * bm::WAVES), want = BEAM_WGS / n;
    return most < want ? most : want;
}
// Workspace of a launch, of up to BEAM_ROWS rows cut into up to BEAM_WGS pieces.
inline size_t beam_ws_bytes() { return sizeof(bm::Piece) * (size_t)BEAM_WGS; }
static_assert(BEAM_ROWS <= BEAM_WGS, "a piece per row at least");
template <class T>
inline void beam_rows(BeamArgs a, int groups, hipStream_t st) {
    const int most = BEAM_ROWS / a.width;  // groups of a launch
    for (int g = 0; g < groups; g += most) {
        const int m = groups - g < most ? groups - g : most, n = m * a.width;
        BeamArgs b = a;
        b.logits = static_cast<const T*>(a.logits) + (long long)g * a.width * a.ld;
        b.scores += (long long)g * a.width;
        b.parents += (long long)g * a.best;
        b.tokens += (long long)g * a.best;
        b.out += (long long)g * a.best;
        b.chunks = beam_chunks<T>(n, a.V);
        hipLaunchKernelGGL(beam_rows_kernel<T>, dim3(b.chunks, n), dim3(bm::THREADS), 0, st, b);
        hipLaunchKernelGGL(beam_pick_kernel, dim3(m), dim3(256), 0, st, b);
    }
}

}  // namespace wmi
