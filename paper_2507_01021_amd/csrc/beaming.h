// The likeliest continuations of groups of beams.
//
// Beam b of a group has a score c_b, the log-probability of what it holds, and
// a row of logits; continuation (b, i) has
//   c_b + l_i - log(sum over j of exp(l_j)),
// the sum over the ids that are not suppressed. A group's n best are wanted, in
// descending order, equal ones by (b, i).
//
// Two kernels. beam_rows_kernel cuts every row into pieces, a workgroup's each,
// and finds their largest logit, the sum of their exponentials and their n largest
// logits. Within a row the order of the logits is that of the continuations, so a
// row's n largest are enough. beam_pick_kernel, a workgroup per group, joins the
// pieces' sums and picks from their lists. (As one kernel, whose last workgroup of
// a group goes on with the choice, the fences that make the others' lists visible
// cost more than the launch: 1, 64 and 16 groups of 5, 5 and 12 beams of 51865, 51866
// and 151937 ids took 20, 107 and 165 us, as two 12.5, 32 and 45.)
// The n largest of many numbers: the n-th largest of the lanes' maxima is a
// bound that at least n numbers reach, and few more than n; those are listed, and
// put in order by counting for each the larger ones.
// Scores of different beams may lie close together, so sums, logarithms and
// scores are fp64: exponentials of fp32 would be off by 2^-23 of a weight, and
// one choice in some thousands would be another. An fp64 exponential, with its
// conversion, difference and sum, is 16 of some 22 vector instructions per id of the
// pass over a row, half of all that a launch takes (see beam_rows_kernel).
#pragma once

#include <cfloat>

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
    // per (row, piece): its sum, and its largest logits' keys
    struct BeamPiece* pieces;
    u64* keys;
    int chunks, batches;  // pieces of a row, batches of a piece
};
// What a piece of a row left beside `best` keys in descending order (0: no more): the
// sum of exp(l - ref), ref one of its largest logits (-inf: no admissible id; +inf:
// how many such logits there are).
struct BeamPiece {
    double sum;
    float ref;
};
// Rows a launch takes at most, pieces that they are cut into, pieces of a group.
constexpr int BEAM_ROWS = 512, BEAM_PIECES = 1280, BEAM_LISTS = 1024;
constexpr int BEAM_BATCHES = 16;  // batches of a piece

namespace bm {
constexpr int WAVES = 4, THREADS = 64 * WAVES;
// e^x for -700 <= x <= 700 with a relative error of 2 10^-12: x log2(e) as an
// integer, by a sum with 1.5 2^52, and a rest; 2^rest by Chebyshev interpolation of
// degree 8 on [-1/2, 1/2]; the integer is added to the exponent.
__device__ __forceinline__ double exp_sum(double x) {
    const double y = fma(x, 1.4426950408889634074, 6755399441055744.0);
    const double f = fma(x, 1.4426950408889634074, -(y - 6755399441055744.0));
    double p = fma(f, 1.3255179556479267e-06, 1.5310080611926545e-05);
    p = fma(p, f, 0.00015403456082633648);
    p = fma(p, f, 0.0013333450563173552);
    p = fma(p, f, 0.009618129159053034);
    p = fma(p, f, 0.055504109412108156);
    p = fma(p, f, 0.24022650695814518);
    p = fma(p, f, 0.6931471805459332);
    p = fma(p, f, 1.0);
    const u64 bits = __builtin_bit_cast(u64, p);
    const int k = (int)__builtin_bit_cast(u64, y);
    return __builtin_bit_cast(double, bits + ((u64)(unsigned)k << 52));
}

// Bounds that at least k[i] (1 <= k[i] <= 64) of the lanes' numbers (no NaN) reach, and
// few more: the k[i]-th largest, bit by bit (without branches: two searches beside
// each other), its last 16 bits only if many share the first.
__device__ __forceinline__ void bounds_of(float x, const int (&k)[2], float (&bound)[2]) {
    const unsigned mine = f2ord(x);
    unsigned t[2] = {0, 0};
    int n[2] = {64, 64};
    auto bits = [&](int from) __attribute__((always_inline)) {
#pragma unroll
        for (int b = from; b > from - 16; --b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned c = t[i] | 1u << b;
                const int m = __popcll(__ballot(mine >= c));
                t[i] = m >= k[i] ? c : t[i];
                n[i] = m >= k[i] ? m : n[i];
            }
    };
    bits(31);
    if (n[0] > k[0] + 4 || n[1] > k[1] + 4) bits(15);
#pragma unroll
    for (int i = 0; i < 2; ++i) bound[i] = t[i] <= f2ord(-INFINITY) ? -INFINITY : ord2f(t[i]);
}

// Sum over the 64 lanes, the same in all.
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A sum of exponentials taken from `from`, as one that is taken from `to` >= `from`.
__device__ __forceinline__ double sum_from(double v, float from, float to) {
    if (from == to) return v;
    return from == -INFINITY || to == INFINITY ? 0.0 : v * exp_sum(fmax((double)from - (double)to, -700.0));
}

// A wave's LDS accesses are in order; this keeps the compiler's in order too.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
}  // namespace bm

// Whether a beam of that score is there.
__device__ __forceinline__ bool beam_lives(float score) { return fabsf(score) < INFINITY; }

// Places of n numbers in descending order, by counting the larger ones: calls
// f(i, place) for those whose place is below `best` (all 256 threads call this;
// larger(j, i): whether number j comes before number i). Where there are fewer than
// 256, several lanes share a number's count.
template <class L, class F>
__device__ __forceinline__ void in_order(int n, int best, L&& larger, F&& f) {
    const int lg = n > 128 ? 0 : n > 64 ? 1 : n > 32 ? 2 : 3, team = 1 << lg;
    const int sub = threadIdx.x & (team - 1);
    for (int i = threadIdx.x >> lg; i - (int)(threadIdx.x >> lg) < n; i += bm::THREADS >> lg) {
        int place = 0;
        if (i < n)
#pragma unroll 8
            for (int j = sub; j < n; j += team) place += larger(j, i);
        for (int st = 1; st < team; st <<= 1) place += __shfl_xor(place, st, 64);
        if (i < n && sub == 0 && place < best) f(i, place);
    }
}

// A workgroup goes through its piece once, every wave through its part in batches of
// U 16-byte loads a lane, the next one's under way: it adds up exponentials, from
// its first batch's largest logit on, and keeps a lane's largest logit of every
// batch in LDS. What passes the bound that these give is then read again: as a rule
// some 30 lanes' batches, a thread each; where many logits are equal, everything,
// a wave's list being cut to its n largest when it is full. NEVER: some ids are
// suppressed. Ids are counted from the row's first wherever that lies (16-byte
// loads need no alignment here), so that a row's sums are the same at every
// address: beams that are alike stay equal to the last bit.
// Bound by the issue of vector instructions (64 groups of 5 beams of 51866 ids in bf16:
// 26.2 us, 1.3 TB/s; 33 are counted per id of a lane, 55 % of the cycles, 16 of them the
// exponentials', 6 unpacking and maxima, the others bounds and lists) and by the waits
// around it: first loads, joined bounds, what is read again.
template <class T, int U, bool NEVER>
__global__ __launch_bounds__(bm::THREADS, 4) void beam_rows_kernel(BeamArgs a) {
    using namespace bm;
    constexpr int EL = 16 / sizeof(T), CAP = 192;  // keys of a wave
    static_assert(CAP >= BEAM_BEST + 64, "a list has room for one number of every lane");
    typedef unsigned Raw128 __attribute__((ext_vector_type(4), aligned(2)));
    __shared__ u64 key[WAVES * CAP], joined[WAVES * CAP];
    __shared__ float most[BEAM_BATCHES][THREADS];
    __shared__ int pair[THREADS];
    __shared__ double wsum[WAVES];
    __shared__ float wref[WAVES], wbound[2][WAVES];
    __shared__ int wn[WAVES], pairs, count;
    const int r = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (!beam_lives(a.scores[r])) return;
    const T* row = static_cast<const T*>(a.logits) + (long long)r * a.ld;
    const int whole = a.V / EL;
    // the ids behind the last whole 16 bytes: one a lane of the last piece's first wave (NaN counts as -inf)
    float lx = -INFINITY;
    const int ix = whole * EL + tid;
    if (blockIdx.x == gridDim.x - 1 && ix < a.V) {
        lx = fmaxf(ldf(row + ix), -INFINITY);
        if (NEVER && (a.never[ix >> 5] >> (ix & 31) & 1u)) lx = -INFINITY;
    }
    // (a row of less than 16 bytes is all behind: what is loaded is not looked at)
    const T* from = whole > 0 ? row : reinterpret_cast<const T*>(a.keys);
    // the first 16 bytes of a thread's batch, a batch's loads, and its logits
    auto start = [&](int t, int bt) __attribute__((always_inline)) {
        return ((blockIdx.x * WAVES + (t >> 6)) * a.batches + bt) * U * 64 + (t & 63);
    };
    auto fetch = [&](int v0, u32x4 (&x)[U], unsigned (&m)[U]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int id0 = max(0, min(v0 + u * 64, whole - 1)) * EL;
            x[u] = *reinterpret_cast<const Raw128*>(from + id0);
            if constexpr (NEVER) m[u] = a.never[id0 >> 5] >> (id0 & 31);
            else m[u] = 0;
        }
    };
    auto unpack = [&](int v0, const u32x4 (&x)[U], const unsigned (&m)[U], float (&l)[U][EL]) __attribute__((always_inline)) {
        float mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // suppressed ids, and those behind the row's, are few
            const unsigned out = v0 + u * 64 < whole ? m[u] & ((1u << EL) - 1) : ~0u;
#pragma unroll
            for (int e = 0; e < EL; ++e) {
                float y;
                if constexpr (sizeof(T) == 4) y = __uint_as_float(x[u][e]);
                else y = __uint_as_float(e & 1 ? x[u][e >> 1] & 0xffff0000u : x[u][e >> 1] << 16);
                l[u][e] = fmaxf(y, -INFINITY);
            }
            if (out)
#pragma unroll
                for (int e = 0; e < EL; ++e) l[u][e] = (out >> e) & 1u ? -INFINITY : l[u][e];
#pragma unroll
            for (int e = 0; e < EL; ++e) mx = fmaxf(mx, l[u][e]);
        }
        return mx;
    };
    // a wave's batches that are not all behind the row (and one for the ids behind the last 16 bytes)
    const int ids = whole - start(wave * 64, 0), tail = blockIdx.x == gridDim.x - 1 && wave == 0;
    const int batches = min(a.batches, max(tail, ids > 0 ? (ids + U * 64 - 1) / (U * 64) : 0));
    u32x4 x[U];
    unsigned m[U];
    float l[U][EL];
    fetch(start(tid, 0), x, m);
    float ref = -INFINITY, all_most = lx;
    double sum = 0.0;
#pragma unroll 1
    for (int bt = 0; bt < batches; ++bt) {
        const int v0 = start(tid, bt);
        const float last = bt == batches - 1 ? lx : -INFINITY;
        float mx = unpack(v0, x, m, l);
        most[bt][tid] = mx;
        mx = fmaxf(mx, last);
        all_most = fmaxf(all_most, mx);
        if (bt + 1 < batches) fetch(v0 + U * 64, x, m);
        // (fp64 has room for exponents up to there)
        if (__any(mx > ref + 500.f)) {
            const float t = wave_max(mx);
            sum = ref == -INFINITY || t == INFINITY ? 0.0 : sum * exp_sum(fmax((double)ref - (double)t, -700.0));
            ref = t;
        }
        if (ref < INFINITY && ref > -INFINITY) {
            const double base = ref;
            if (last > -INFINITY) sum += exp_sum(fmax((double)last - base, -700.0));
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < EL; e += 4) {
#pragma unroll
                    for (int i = e; i < e + 4; ++i) sum += exp_sum(fmax((double)l[u][i] - base, -700.0));
                    __builtin_amdgcn_sched_barrier(0);  // four at a time: more would take more registers than there are
                }
        } else if (ref == INFINITY) {
            sum += last == INFINITY ? 1.0 : 0.0;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < EL; ++e) sum += l[u][e] == INFINITY ? 1.0 : 0.0;
        }
    }
    {
        const int k[2] = {a.best, (a.best + WAVES - 1) / WAVES};
        float y[2];
        bounds_of(all_most, k, y);
        sum = wave_sum_f64(sum);
        if (lane == 0) {
            wbound[0][wave] = y[0];
            wbound[1][wave] = y[1];
            wsum[wave] = sum;
            wref[wave] = ref;
        }
        if (tid == 0) pairs = count = 0;
    }
    __syncthreads();
    // `best` logits of one wave, or a quarter of them of every wave's
    float bound = INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) bound = fminf(bound, wbound[1][w]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) bound = fmaxf(bound, wbound[0][w]);
    bound = fmaxf(bound, -FLT_MAX);
    for (int bt = 0; bt < batches; ++bt)
        if (most[bt][tid] >= bound) {
            const int p = atomicAdd(&pairs, 1);
            if (p < THREADS) pair[p] = bt << 8 | tid;
        }
    __syncthreads();
    int n = THREADS * CAP;  // keys that were listed: too many till then
    if (pairs <= THREADS) {
        auto put = [&](float y, int id) __attribute__((always_inline)) {
            if (!(y >= bound)) return;
            const int p = atomicAdd(&count, 1);
            if (p < WAVES * CAP) joined[p] = amax_key(y + 0.f, id);  // (-0 and 0 are equal)
        };
        if (tid < pairs) {
            const int v0 = start(pair[tid] & 255, pair[tid] >> 8);
            fetch(v0, x, m);
            unpack(v0, x, m, l);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < EL; ++e) put(l[u][e], (v0 + u * 64) * EL + e);
        }
        put(lx, ix);
        __syncthreads();
        n = count;
    }
    if (n > WAVES * CAP) {
        u64* mine = key + wave * CAP;
        int bound_id = 0x7fffffff;  // of those equal to the bound, lower ids pass
        n = 0;
        // lists the lanes' logits that pass; where the list is full, its `best` largest
        // are kept, and the last of them is the bound from then on
        auto list = [&](float y, int id) __attribute__((always_inline)) {
            auto passes = [&]() __attribute__((always_inline)) { return (y > bound) | ((y == bound) & (id < bound_id)); };
            unsigned long long in = __ballot(passes());
            if (!in) return;
            if (n + __popcll(in) > CAP) {
                u64 own[CAP / 64];
                int place[CAP / 64];
#pragma unroll
                for (int i = 0; i < CAP / 64; ++i) {
                    own[i] = lane + i * 64 < n ? mine[lane + i * 64] : 0;
                    place[i] = own[i] ? 0 : a.best;
                }
#pragma unroll 1
                for (int j = 0; j < n; ++j) {
                    const u64 k = mine[j];
#pragma unroll
                    for (int i = 0; i < CAP / 64; ++i) place[i] += k > own[i];
                }
                wave_lds_fence();
#pragma unroll
                for (int i = 0; i < CAP / 64; ++i)
                    if (place[i] < a.best) mine[place[i]] = own[i];
                wave_lds_fence();
                n = a.best;
                const u64 k = mine[n - 1];
                bound = ord2f((uint32_t)(k >> 32));
                bound_id = (int)(0xffffffffu - (unsigned)k);
                in = __ballot(passes());
            }
            if (passes()) mine[n + __popcll(in & ((1ull << lane) - 1))] = amax_key(y + 0.f, id);
            n += __popcll(in);
        };
#pragma unroll 1
        for (int bt = 0; bt < batches; ++bt) {
            if (!__any(most[bt][tid] >= bound)) continue;
            const int v0 = start(tid, bt);
            fetch(v0, x, m);
            unpack(v0, x, m, l);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < EL; ++e) list(l[u][e], (v0 + u * 64) * EL + e);
        }
        list(lx, ix);
        if (lane == 0) wn[wave] = n;
        __syncthreads();
        // the waves' lists as one
        int to = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            for (int i = tid; i < wn[w]; i += THREADS) joined[to + i] = key[w * CAP + i];
            to += wn[w];
        }
        n = to;
        __syncthreads();
    }
    const long long at = (long long)r * a.chunks + blockIdx.x;
    u64* out = a.keys + at * a.best;
    in_order(n, a.best, [&](int j, int i) { return joined[j] > joined[i]; }, [&](int i, int place) { out[place] = joined[i]; });
    for (int i = n + tid; i < a.best; i += THREADS) out[i] = 0;
    if (tid == 0) {
        const float t = fmaxf(fmaxf(wref[0], wref[1]), fmaxf(wref[2], wref[3]));
        double y = 0.0;
        for (int w = 0; w < WAVES; ++w) y += sum_from(wsum[w], wref[w], t);
        a.pieces[at] = BeamPiece{y, t};
    }
}

// A group's n best from its pieces' lists (each in descending order). A list whose
// j-th entry is some score has j + 1 continuations no worse, so the k-th largest of
// the lists' j-th entries, k (j + 1) >= n, is a bound that n continuations reach
// (rounded down to fp32, it still is). What reaches it is put in order by counting.
// Bound by the latency of two rounds of loads and of the counting: 5.5 us for one
// group of 5 beams, 7.6 for 64, 9.5 for 16 of 12.
static __global__ __launch_bounds__(bm::THREADS) void beam_pick_kernel(BeamArgs a) {
    using namespace bm;
    constexpr int CAP = 1024, PER = BEAM_LISTS / 256, FEW = BEAM_BEST;
    __shared__ double off[BEAM_WIDTH];  // log of the row's sum
    __shared__ float refs[BEAM_WIDTH], score[BEAM_WIDTH];
    __shared__ double val[CAP];
    __shared__ int idx[CAP], act[BEAM_LISTS];
    __shared__ float head[256];
    __shared__ double red[4];
    __shared__ int redi[4];
    __shared__ double sh_val;
    __shared__ int count, n_act, sh_idx;
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lists = a.width * a.chunks;
    const BeamPiece* pieces = a.pieces + (long long)g * lists;
    const u64* keys = a.keys + (long long)g * lists * a.best;
    u64 first[PER];  // of lists tid, tid + 256, ...
#pragma unroll
    for (int s = 0; s < PER; ++s) first[s] = tid + s * 256 < lists ? keys[(long long)(tid + s * 256) * a.best] : 0;
    {
        // eight lanes per row, four pieces each at a time
        const int b = tid >> 3, sub = tid & 7;
        const float c = b < a.width ? a.scores[g * a.width + b] : -INFINITY;
        float t = -INFINITY;
        double y = 0.0;
        if (b < a.width) {
            for (int k0 = sub; k0 < a.chunks; k0 += 32) {
                BeamPiece p[4];
#pragma unroll
                for (int s = 0; s < 4; ++s) p[s] = pieces[b * a.chunks + min(k0 + 8 * s, a.chunks - 1)];
                float to = t;
#pragma unroll
                for (int s = 0; s < 4; ++s) to = fmaxf(to, p[s].ref);
                y = sum_from(y, t, to);
                t = to;
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    if (k0 + 8 * s < a.chunks) y += sum_from(p[s].sum, p[s].ref, t);
            }
        }
        {
            float to = t;
#pragma unroll
            for (int st = 1; st < 8; st <<= 1) to = fmaxf(to, __shfl_xor(to, st, 64));
            y = sum_from(y, t, to);
            t = beam_lives(c) ? to : -INFINITY;  // (what pieces of a beam that is not there hold is left over)
#pragma unroll
            for (int st = 1; st < 8; st <<= 1) y += __shfl_xor(y, st, 64);
        }
        if (sub == 0 && b < a.width) {
            refs[b] = t;  // -inf: no continuation
            score[b] = c;
            off[b] = t == -INFINITY ? 0.0 : log(y);
        }
    }
    if (tid == 0) count = n_act = 0;
    __syncthreads();
    // the continuation of a key of row b: its score, or -inf for none (keys of beams
    // that are not there are not read as such)
    auto total = [&](int b, u64 k) __attribute__((always_inline)) {
        const float l = ord2f((uint32_t)(k >> 32));
        if (refs[b] == -INFINITY || k == 0 || (refs[b] == INFINITY && l != INFINITY)) return -(double)INFINITY;
        return (double)score[b] + ((refs[b] == INFINITY ? 0.0 : (double)l - (double)refs[b]) - off[b]);
    };
    auto place_of = [&](int b, u64 k) __attribute__((always_inline)) { return b * a.V + (int)(0xffffffffu - (unsigned)k); };
    auto below = [](double x) __attribute__((always_inline)) {  // rounded down
        const float f = (float)x;
        return (double)f > x ? ord2f(f2ord(f) - 1) : f;
    };
    // a bound that at least k of the threads' numbers reach: the k-th largest to 16
    // bits (every wave finds it by itself)
    auto kth = [&](float x, int k) __attribute__((always_inline)) {
        head[tid] = x;
        __syncthreads();
        unsigned v[4], t = 0;
#pragma unroll
        for (int s = 0; s < 4; ++s) v[s] = f2ord(head[lane + s * 64]);
#pragma unroll
        for (int b = 31; b > 15; --b) {
            const unsigned c = t | 1u << b;
            int m = 0;
#pragma unroll
            for (int s = 0; s < 4; ++s) m += __popcll(__ballot(v[s] >= c));
            t = m >= k ? c : t;
        }
        __syncthreads();
        return t <= f2ord(-INFINITY) ? -INFINITY : ord2f(t);
    };
    float heads[PER], most = -INFINITY;
#pragma unroll
    for (int s = 0; s < PER; ++s) {
        heads[s] = -INFINITY;
        if (first[s]) heads[s] = below(total((tid + s * 256) / a.chunks, first[s]));
        most = fmaxf(most, heads[s]);
    }
    const int live = __syncthreads_count(most > -INFINITY);
    if (live > 0) {
        int k = a.best;
        if (live < a.best) {  // further down the lists
            const int j = (a.best + live - 1) / live - 1;
            k = (a.best + j) / (j + 1);
            most = -INFINITY;
#pragma unroll
            for (int s = 0; s < PER; ++s) {
                const int i = tid + s * 256;
                if (heads[s] > -INFINITY) most = fmaxf(most, below(total(i / a.chunks, keys[(long long)i * a.best + j])));
            }
        }
        const float low = kth(most, k);
        // lists that reach the bound, and their entries that do
#pragma unroll
        for (int s = 0; s < PER; ++s)
            if (heads[s] >= low && heads[s] > -INFINITY) act[atomicAdd(&n_act, 1)] = tid + s * 256;
        __syncthreads();
        const int all = n_act * a.best;
        for (int q = tid; q < all; q += 256) {
            const int i = act[q / a.best], b = i / a.chunks;
            const u64 key = keys[(long long)i * a.best + q % a.best];
            const double x = total(b, key);
            if (x >= (double)low && x > -(double)INFINITY) {
                const int p = atomicAdd(&count, 1);
                if (p < CAP) {
                    val[p] = x;
                    idx[p] = place_of(b, key);
                }
            }
        }
        __syncthreads();
    }
    int n = count;
    if (n > FEW && n <= CAP) {
        // a bound from among them: each thread's largest
        double own[CAP / 256];
        int at[CAP / 256];
        float x = -INFINITY;
#pragma unroll
        for (int s = 0; s < CAP / 256; ++s) {
            const int i = tid + s * 256;
            own[s] = i < n ? val[i] : -(double)INFINITY;
            at[s] = i < n ? idx[i] : 0;
            x = fmaxf(x, below(own[s]));
        }
        const float low = kth(x, a.best);
        if (tid == 0) count = 0;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < CAP / 256; ++s)
            if (tid + s * 256 < n && own[s] >= (double)low) {
                const int p = atomicAdd(&count, 1);
                val[p] = own[s];
                idx[p] = at[s];
            }
        __syncthreads();
        n = count;
    }
    int* parents = a.parents + (long long)g * a.best;
    int* tokens = a.tokens + (long long)g * a.best;
    float* out = a.out + (long long)g * a.best;
    auto put = [&](int place, double x, int at) __attribute__((always_inline)) {
        parents[place] = at / a.V;
        tokens[place] = at - at / a.V * a.V;
        out[place] = (float)x;
    };
    if (n <= CAP) {
        in_order(n, a.best, [&](int j, int i) { return (int)(val[j] > val[i]) | ((int)(val[j] == val[i]) & (int)(idx[j] < idx[i])); },
                 [&](int i, int place) { put(place, val[i], idx[i]); });
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
            const int b = i / a.chunks;
            for (int e = 0; e < a.best; ++e) {
                const u64 key = keys[(long long)i * a.best + e];
                const double x = total(b, key);
                if (x == -(double)INFINITY || x < bx) break;
                const int at = place_of(b, key);
                if (x > last || (x == last && at <= last_at)) continue;  // chosen already
                if (x > bx || at < bi) {
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
            red[wave] = bx;
            redi[wave] = bi;
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < 4; ++w)
                if (red[w] > red[0] || (red[w] == red[0] && redi[w] < redi[0])) {
                    red[0] = red[w];
                    redi[0] = redi[w];
                }
            sh_val = red[0];
            sh_idx = redi[0];
            put(m, red[0], redi[0]);  // (there are more than CAP >= best)
        }
        __syncthreads();
        last = sh_val;
        last_at = sh_idx;
    }
}

// A launch's pieces: what 1280 workgroups (five per CU) take in batches of 16 ids a
// thread, or, where that gives fewer than one per CU, in batches of 8 ids. (16 groups
// of 12 beams of 151937 ids: 36.8 us, 40.3 with 1024 pieces; 64 of 5 beams of 51866
// in bf16: 26.2 both.)
template <class T, int U>
inline void beam_launch(BeamArgs a, int n, int groups, int loads, hipStream_t st) {
    const int most = (loads + U * bm::THREADS - 1) / (U * bm::THREADS);
    int c = BEAM_PIECES / n < BEAM_LISTS / a.width ? BEAM_PIECES / n : BEAM_LISTS / a.width;
    if (c > most) c = most;
    a.batches = (most + c - 1) / c;
    a.chunks = (most + a.batches - 1) / a.batches;
    if (a.never) hipLaunchKernelGGL((beam_rows_kernel<T, U, true>), dim3(a.chunks, n), dim3(bm::THREADS), 0, st, a);
    else hipLaunchKernelGGL((beam_rows_kernel<T, U, false>), dim3(a.chunks, n), dim3(bm::THREADS), 0, st, a);
    hipLaunchKernelGGL(beam_pick_kernel, dim3(groups), dim3(256), 0, st, a);
}
inline size_t beam_ws_bytes() { return (sizeof(BeamPiece) + sizeof(u64) * BEAM_BEST) * (size_t)BEAM_PIECES; }
template <class T>
inline void beam_rows(BeamArgs a, int groups, hipStream_t st) {
    constexpr int U = sizeof(T);
    const int loads = (int)((a.V * (long long)sizeof(T) + 15) / 16);
    // pieces of BEAM_BATCHES batches have to do for a launch's rows
    const int least = (loads + BEAM_BATCHES * U * bm::THREADS - 1) / (BEAM_BATCHES * U * bm::THREADS);
    const int rows = BEAM_PIECES / least < BEAM_ROWS ? BEAM_PIECES / least : BEAM_ROWS, most = rows / a.width;
    for (int g = 0; g < groups; g += most) {
        const int m = groups - g < most ? groups - g : most, n = m * a.width;
        BeamArgs b = a;
        b.logits = static_cast<const T*>(a.logits) + (long long)g * a.width * a.ld;
        b.scores += (long long)g * a.width;
        b.parents += (long long)g * a.best;
        b.tokens += (long long)g * a.best;
        b.out += (long long)g * a.best;
        if ((long long)n * loads >= 256LL * U * bm::THREADS) beam_launch<T, U>(b, n, m, loads, st);
        else beam_launch<T, U / 2>(b, n, m, loads, st);
    }
}
// the widest group over the widest vocabulary (2^20 ids of 4 bytes) fits a launch, and its pieces the lists of a group
constexpr int BEAM_LEAST = (1 << 18) / (BEAM_BATCHES * 4 * bm::THREADS);
static_assert(BEAM_PIECES / BEAM_LEAST >= BEAM_WIDTH && BEAM_LISTS / BEAM_WIDTH >= BEAM_LEAST, "");

}  // namespace wmi
