// Tokens from rows of logits: temperature, top-k, top-p and min-p, with given random numbers.
//
// Weights are whole multiples of 2^-S of the row's largest one, S as large as sums of the vocabulary leave room for in 62 bits (45 for 128000 tokens): sums are then exact, do
// not hang on their order or on how a row is split, and compare with top_p and the random number as they are.  exp in 64 bits: 2^(y / 512) = 2^(k / 512) 2^(r / 512) with k the
// nearest whole number, 512 values of the first in LDS, three terms of the second beside its 1 (2^-46 of it are left out), and the addition of 2^52 rounds to a whole number of
// units.  That is about 24 instructions, 8 of them in 64 bits: 5 us for 32000 weights on one CU.
//
// The filters keep the front part of the order (value falling, index rising), so that what is kept is a bound: a value, and an index among those equal to it.  It is looked for
// among few candidates, which are gathered in LDS:
//   top_k: counts in 2048 bins over the distance to the largest value show up to which bin the first k reach; for a small k the largest values of the threads do (the k-th of them
//          is not above the row's k-th);
//   top_p of all tokens: sums in these bins show in which one the bound lies; what is above it is kept.
// Where there are more candidates than room (flat rows, thousands of equal logits, k near 4096 in rows of less than six workgroups, or above) the bound is found in the row itself, by bins over the bits of the values where it lies.
//
// What bounds it: latencies in short rows (32000 logits in bf16: 6 us greedy, 9.6 with top_k, 13 with none of the filters, 29 with top_p alone); in many long ones the passes over memory, three of
// them in four launches (256 rows of 128003 in f32: 21 us a pass, 45 greedy, 55 with top_k = 50, 61 with no filter), and 64-bit arithmetic (112 with top_p alone, where each weight is formed twice).
#include "clear.h"

#define SAMPLE_THREADS 1024
#define SAMPLE_WAVES (SAMPLE_THREADS / 64)
#define SAMPLE_BINS 2048
#define SAMPLE_SEGMENTS 512  // of a row: one wave looks through one of them at the end
#define SAMPLE_LIST 4096     // candidates
#define SAMPLE_LONG 8192     // of a row that six workgroups or more share
#define SAMPLE_PAIRS 256     // candidates that are compared each with each (64 rows of 128000, top 50 and top_p as arrays: 29 us, in bins 35; one of 32000 9.3 and 13.3)
#define SAMPLE_FEW 512       // top_k up to which the threads' largest values choose the candidates (256 rows, top 50: 55 us, with counts of all values 78; 64 rows 26 and 32)
#define SAMPLE_PARTS 8       // workgroups to a row
#define LN2 0.69314718055994530942

template <int LIST>
struct SampleLds {
    double roots[512];     // 2^(k / 512)
    u64 sum[SAMPLE_BINS];  // of the bins, of the segments of a row, or the candidates' weights
    u32 count[SAMPLE_BINS];
    u64 list[LIST];  // bits of the value in their order, and inverted index: the order of the filters is the falling one of these
    u64 part[SAMPLE_WAVES];
    u32 low[SAMPLE_WAVES], high[SAMPLE_WAVES];
    int found, listed, few;
    u64 found_before;
    u64 order[64], load[64];  // of the elements of one bin, for a wave to put in order
};

// What the workgroups of a row leave for each other, in the workspace
struct SampleShared {
    u64 bins[SAMPLE_BINS], sum[SAMPLE_SEGMENTS], list[SAMPLE_LONG];
    float most[SAMPLE_PARTS], threads[SAMPLE_PARTS * SAMPLE_THREADS];  // the largest values of the parts, and of their threads
    int first[SAMPLE_PARTS];
    int listed, border;  // the bin of top_p's bound, and what is left there of its target
    u64 rest;
};

// Values of other lanes, within a row of 16 and from the rows before: a scan takes 6 of them, a twentieth of what it takes through LDS.  Lanes without a source get `none`.
template <int CONTROL, int ROWS>
__device__ __forceinline__ u32 from_lane(u32 none, u32 v) {
    return (u32)__builtin_amdgcn_update_dpp((int)none, (int)v, CONTROL, ROWS, 0xf, false);
}
template <int CONTROL, int ROWS>
__device__ __forceinline__ u64 from_lane(u64 none, u64 v) {
    return (u64)from_lane<CONTROL, ROWS>((u32)(none >> 32), (u32)(v >> 32)) << 32 | from_lane<CONTROL, ROWS>((u32)none, (u32)v);
}
// Inclusive, over a wave of which all lanes are here; `none` is what changes nothing
template <class V, class OP>
__device__ __forceinline__ V wave_scan(V v, V none, const OP &op) {
    v = op(v, from_lane<0x111, 0xf>(none, v));  // one lane up, then two, four and eight
    v = op(v, from_lane<0x112, 0xf>(none, v));
    v = op(v, from_lane<0x114, 0xf>(none, v));
    v = op(v, from_lane<0x118, 0xf>(none, v));
    v = op(v, from_lane<0x142, 0xa>(none, v));  // the last lane of rows 0 and 2 into rows 1 and 3
    v = op(v, from_lane<0x143, 0xc>(none, v));  // and that of row 1 into rows 2 and 3
    return v;
}
__device__ __forceinline__ u64 wave_scan(u64 v) {
    return wave_scan(v, (u64)0, [](u64 a, u64 b) { return a + b; });
}
__device__ __forceinline__ u64 wave_last(u64 v) { return (u64)(u32)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (u32)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ u64 wave_sum(u64 v) { return wave_last(wave_scan(v)); }

// Numbers in their order as unsigned ones; both zeros are one
__device__ __forceinline__ u32 key_of(float x) {
    const u32 b = __builtin_bit_cast(u32, x + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(u32 k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffff : ~k); }

// floor(w f), and the same rounded up, for 0 <= f < 1
__device__ __forceinline__ u64 part_of(u64 w, float f, bool up) {
    const u32 b = __builtin_bit_cast(u32, f);
    const int e = (int)(b >> 23);
    const u64 m = e ? (b & 0x7fffff) | 0x800000 : b & 0x7fffff;
    const int shift = 150 - max(e, 1);  // f = m 2^-shift, 24 to 149
    const u64 low = w * m, high = __umul64hi(w, m);
    u64 whole, rest;  // of (high, low) 2^-shift, and what is left
    if (shift < 64) {
        whole = high << (64 - shift) | low >> shift;
        rest = low << (64 - shift);
    } else {
        const int s = min(shift - 64, 63);  // (high is below 2^24)
        whole = high >> s;
        rest = low | (high & (((u64)1 << s) - 1));
    }
    return whole + (up && rest ? 1 : 0);
}
// The running sum at which top_p's part ends, and the one that the random number exceeds by less than a token
__device__ __forceinline__ u64 part_target(u64 sum, float p) { return p > 0 ? max(part_of(sum, p, true), (u64)1) : 1; }
__device__ __forceinline__ u64 draw_target(u64 sum, float u) { return !(u > 0) ? 0 : u >= 1 ? sum - 1 : part_of(sum, u, false); }

enum SampleMode { SAMPLE_NONE, SAMPLE_FIRST, SAMPLE_TOP, SAMPLE_PART, SAMPLE_ALL, SAMPLE_SLOW };

__device__ __forceinline__ u32 larger(u32 a, u32 b) { return __builtin_bit_cast(u32, __builtin_elementwise_maximum(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b))); }

// HELD: a row of up to 64 tiles stays in registers, four tiles to a wave
template <int TYPE, bool HELD, int LIST = SAMPLE_LIST>
struct SampleRow {
    typedef typename Elem<TYPE>::type T;
    static constexpr int E = TYPE == ENSI_T_F32 ? 4 : 8, TILE = 64 * E, AHEAD = 2;  // elements of a lane and of a wave; tiles under way (four: 1 to 3 % slower)
    typedef T vec __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    SampleLds<LIST> &lds;
    const T *x;
    int vocab, tiles, per;  // tiles of a row, tiles to a segment
    int lane, wave;
    float t, p, m, u;
    int k;
    // weights
    float top, half_top;   // the largest value, and half of it
    double rate;           // y = (x - top) rate, 512 to a power of two
    int shift;             // S
    float bins;            // to two units of distance
    // kept so far: values above `edge`, and of the equal ones those up to index `last`
    float edge, small;     // small: the smallest value that min_p leaves
    int last;
    vec held0, held1, held2, held3;

    __device__ __forceinline__ SampleRow(const ensi_clear_sample_args &a, int64_t row, SampleLds<LIST> &l) : lds(l) {
        x = (const T *)a.logits + row * a.stride;
        vocab = a.vocab;
        tiles = (vocab + TILE - 1) / TILE;
        per = (tiles + SAMPLE_SEGMENTS - 1) / SAMPLE_SEGMENTS;
        lane = threadIdx.x % 64;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        t = a.temperature ? a.temperature[row] : a.all_temperature;
        p = a.top_p ? a.top_p[row] : a.all_top_p;
        m = a.min_p ? a.min_p[row] : a.all_min_p;
        k = a.top_k ? a.top_k[row] : a.all_top_k;
        u = a.uniform[row];
        if constexpr (HELD) {
            held0 = fetch(wave);
            held1 = fetch(wave + SAMPLE_WAVES);
            held2 = fetch(wave + 2 * SAMPLE_WAVES);
            held3 = fetch(wave + 3 * SAMPLE_WAVES);
        }
    }
    // With the row's largest value (NaN where it has one): what is to be done, and the constants for it
    __device__ __forceinline__ SampleMode begin(float most) {
        // no distribution: NaN or +inf among the logits, nothing but -inf, numbers out of range
        if (!(fabsf(most) < __builtin_inff()) || !(t >= 0) || !(t < __builtin_inff()) || p != p || m != m || u != u) return SAMPLE_NONE;
        top = most;
        edge = small = -__builtin_inff();
        last = INT32_MAX;
        if (t == 0) return SAMPLE_FIRST;
        const int bits = 32 - __clz(vocab);
        shift = min(50, 62 - bits);
        rate = 512 / LN2 / (double)t;
        half_top = 0.5f * top;
        bins = fminf((float)rate * (SAMPLE_BINS / 256) / (float)(shift + 2), 3e38f);  // 2^-(S + 2) after the last
        if (m > 0) {
            // min_p keeps values from some place on: found by all lanes, a 64th of what is left at a time
            const double least = 512 * log2((double)fminf(m, 1.0f));
            u32 low = 0, high = key_of(top);  // not kept, kept
            while (high - low > 1) {
                const u32 step = (high - low - 1) / 64 + 1, probe = high - low > (u32)lane * step + step ? low + ((u32)lane + 1) * step : high;
                const u64 hit = __ballot(place(of_key(probe)) >= least);  // (values below -inf are NaN)
                const int l = __ffsll((unsigned long long)hit) - 1;
                high = __shfl(probe, l);
                low += (u32)l * step;
            }
            small = of_key(high);
        }
        if (k <= 0 || k >= vocab) k = 0;
        if (!k && p >= 1) edge = small;
        return k ? (k <= SAMPLE_LIST ? SAMPLE_TOP : SAMPLE_SLOW) : p < 1 ? SAMPLE_PART : SAMPLE_ALL;
    }
    __device__ __forceinline__ void set_roots() const {
        if (threadIdx.x < 512) lds.roots[threadIdx.x] = exp2(threadIdx.x / 512.0);
    }

    // A lane's part of a tile, -inf behind the row's end
    __device__ __forceinline__ vec fetch(int tile) const {
        const int at = tile * TILE + lane * E;
        if (at + E <= vocab) return *(const vec *)(x + at);
        vec v;
#pragma unroll
        for (int i = 0; i < E; i++) v[i] = at + i < vocab ? x[at + i] : (T)-__builtin_inff();
        return v;
    }
    static __device__ __forceinline__ void widen(float (&f)[E], const vec &v) {
#pragma unroll
        for (int i = 0; i < E; i++) f[i] = (float)v[i];
    }
    // todo(values, index of the first) for the tiles that `step` apart follow `first`, up to `end`: little work, AHEAD whole tiles at a time ...
    template <class TODO>
    __device__ __forceinline__ void walk(int first, int end, int step, const TODO &todo) const {
        const int whole = min(end, vocab / TILE);
        int tile = first;
        for (; tile + (AHEAD - 1) * step < whole; tile += AHEAD * step) {
            vec v[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; a++) v[a] = *(const vec *)(x + (tile + a * step) * TILE + lane * E);
#pragma unroll
            for (int a = 0; a < AHEAD; a++) {
                float f[E];
                widen(f, v[a]);
                todo(f, (tile + a * step) * TILE + lane * E);
            }
        }
        walk_slowly(tile, end, step, todo);
    }
    // ... or much: the next tile is under way while one is worked on
    template <class TODO>
    __device__ __forceinline__ void walk_slowly(int first, int end, int step, const TODO &todo) const {
        if (first >= end) return;
        vec now = fetch(first);
        for (int tile = first; tile < end; tile += step) {
            vec next = now;
            if (tile + step < end) next = fetch(tile + step);
            float f[E];
            widen(f, now);
            todo(f, tile * TILE + lane * E);
            now = next;
        }
    }
    // Of a part, all waves
    template <class TODO>
    __device__ __forceinline__ void walk_part(int first, int end, const TODO &todo) const {
        if constexpr (HELD) {
            const auto one = [&](const vec &v, int tile) {
                if (tile >= tiles) return;
                float f[E];
                widen(f, v);
                todo(f, tile * TILE + lane * E);
            };
            one(held0, wave);
            one(held1, wave + SAMPLE_WAVES);
            one(held2, wave + 2 * SAMPLE_WAVES);
            one(held3, wave + 3 * SAMPLE_WAVES);
        } else
            walk(first + wave, end, SAMPLE_WAVES, todo);
    }
    template <class TODO>
    __device__ __forceinline__ void walk_part_slowly(int first, int end, const TODO &todo) const {
        walk_slowly(first + wave, end, SAMPLE_WAVES, todo);
    }
    __device__ __forceinline__ bool kept(float f, int index) const { return (f > edge) | ((f == edge) & (index <= last)); }
    __device__ __forceinline__ double place(float f) const { return ((double)f - (double)top) * rate; }
    // The weights of N values, 0 where `in` is not set; each 2^52 more than it is in its bits.  All at once, so that they hide each other's latencies.
    template <int N>
    __device__ __forceinline__ void weights(u64 (&w)[N], const float (&f)[N], const bool (&in)[N]) const {
        double r[N], root[N];
        int e[N];
#pragma unroll
        for (int i = 0; i < N; i++) {
            const double y = fmax(place(f[i]), -32768.0), z = y + 0x1.8p52;
            const int k = (int)__builtin_bit_cast(u64, z);
            r[i] = y - (z - 0x1.8p52);
            root[i] = lds.roots[k & 511];
            e[i] = (in[i] ? shift : -512) + (k >> 9);
        }
        const double a = LN2 / 512;
#pragma unroll
        for (int i = 0; i < N; i++) {
            double p = fma(r[i], a * a * a / 6, a * a / 2);
            p = fma(r[i], p, a);
            p = fma(r[i], p, 1.0);
            const double high = __builtin_bit_cast(double, __builtin_bit_cast(u64, root[i]) + ((u64)(u32)e[i] << 52));
            w[i] = __builtin_bit_cast(u64, fma(high, p, 0x1p52));
        }
    }
    static constexpr u64 NO_WEIGHT = 0x4330000000000000;  // 2^52
    __device__ __forceinline__ u64 weight(float f) const {
        u64 w[1];
        const float v[1] = {f};
        const bool in[1] = {true};
        weights<1>(w, v, in);
        return w[0] - NO_WEIGHT;
    }
    // Bins over the distance to the largest value: what lies beyond the last has no weight.  Half of the distance stays in range where the logits are at both ends of 32 bits, and at high
    // temperatures what lies that far off has a weight.
    __device__ __forceinline__ float half_distance(float f) const { return __builtin_fmaf(-0.5f, f, half_top); }
    __device__ __forceinline__ int bin(float f) const { return (int)fminf(half_distance(f) * bins, (float)SAMPLE_BINS); }

    // ---- over the workgroup
    __device__ __forceinline__ u64 total(u64 v) const {
        v = wave_sum(v);
        __syncthreads();
        if (lane == 0) lds.part[wave] = v;
        __syncthreads();
        u64 sum = 0;
#pragma unroll
        for (int w = 0; w < SAMPLE_WAVES; w++) sum += lds.part[w];
        return sum;
    }
    template <class OP>
    __device__ __forceinline__ u32 reduce(u32 v, u32 none, u32 (&each)[SAMPLE_WAVES], const OP &op) const {  // (a barrier before `each` is written again is the caller's)
        v = (u32)__builtin_amdgcn_readlane((int)wave_scan(v, none, op), 63);
        if (lane == 0) each[wave] = v;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < SAMPLE_WAVES; w++) v = op(v, each[w]);
        return v;
    }
    // The first of lds.sum[0 .. n) (or of lds.count, by COUNTS) at which the running sum reaches target(the whole sum) >= 1: into lds.found, with the sum before it; n if none does.
    // Two to a thread; returns that target
    template <bool COUNTS, class TARGET>
    __device__ __forceinline__ u64 find(int n, const TARGET &target_of) const {
        __syncthreads();
        const int at = 2 * threadIdx.x;
        const u64 v0 = at < n ? (COUNTS ? (u64)lds.count[at] : lds.sum[at]) : 0, v1 = at + 1 < n ? (COUNTS ? (u64)lds.count[at + 1] : lds.sum[at + 1]) : 0;
        const u64 s = wave_scan(v0 + v1);
        if (lane == 63) lds.part[wave] = s;
        if (threadIdx.x == 0) lds.found = n;
        __syncthreads();
        u64 before = s - v0 - v1, sum = 0;
#pragma unroll
        for (int w = 0; w < SAMPLE_WAVES; w++) {
            const u64 one = lds.part[w];
            sum += one;
            before += w < wave ? one : 0;
        }
        const u64 target = target_of(sum);
        if (before < target && before + v0 + v1 >= target) {  // (of one thread)
            const bool second = before + v0 < target;
            lds.found = at + second;
            lds.found_before = before + (second ? v0 : 0);
        }
        __syncthreads();
        return target;
    }
    template <bool COUNTS>
    __device__ __forceinline__ void find_at(int n, u64 target) const {
        find<COUNTS>(n, [=](u64) { return target; });
    }
    __device__ __forceinline__ void clear_bins() const {
        __syncthreads();
        for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS) {
            lds.count[i] = 0;
            lds.sum[i] = 0;
        }
        __syncthreads();
    }
    // Of the elements that each(todo) hands over as todo(key, weight), with keys from low to high: the key at which the running sum of counts or weights, from the largest key on, reaches
    // `target` >= 1, which it does; `target` becomes what is left of it there, `ties` how many have that key.
    template <bool COUNTS, class EACH>
    __device__ __forceinline__ u32 select(u32 low, u32 high, u64 &target, int &ties, const EACH &each) const {
        for (;;) {
            const int bits = 32 - __clz((int)((high - low) | 1)), step = max(0, bits - 11);
            clear_bins();
            each([&](u32 k, const auto &weight) {
                if (k >= low && k <= high) {
                    const u32 b = (high - k) >> step;
                    atomicAdd(&lds.count[b], 1u);
                    if (!COUNTS) atomicAdd((unsigned long long *)&lds.sum[b], (unsigned long long)weight());
                }
            });
            find_at<COUNTS>(SAMPLE_BINS, target);
            const u32 b = lds.found, first = high - (b << step);
            target -= lds.found_before;
            ties = (int)lds.count[b];
            if (step == 0) return first;
            const u32 width = (1u << step) - 1;
            if (first - low > width) low = first - width;
            high = first;
        }
    }
    // ---- in the tiles from `first` to `end`
    __device__ __forceinline__ float largest(int first, int end) const {  // of a thread; NaN where it has one
        float most = -__builtin_inff();
        walk_part(first, end, [&](const float (&f)[E], int) {
#pragma unroll
            for (int i = 0; i < E; i++) most = __builtin_elementwise_maximum(most, f[i]);
        });
        return most;
    }
    __device__ __forceinline__ int first_largest(int first, int end) const {
        int index = INT32_MAX;
        walk_part(first, end, [&](const float (&f)[E], int at) {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (f[i] == top) index = min(index, at + i);
        });
        return (int)reduce((u32)index, ~0u, lds.high, [](u32 a, u32 b) { return min(a, b); });
    }
    __device__ __forceinline__ void count_bins(int first, int end) const {
        clear_bins();
        walk_part(first, end, [&](const float (&f)[E], int) {
#pragma unroll
            for (int i = 0; i < E; i++) {
                const int b = bin(f[i]);
                if (b < SAMPLE_BINS) atomicAdd(&lds.count[b], 1u);
            }
        });
        __syncthreads();
    }
    __device__ __forceinline__ void sum_bins(int first, int end) const {
        clear_bins();
        walk_part_slowly(first, end, [&](const float (&f)[E], int at) {
            u64 w[E];
            bool in[E];
#pragma unroll
            for (int i = 0; i < E; i++) in[i] = kept(f[i], at + i);
            weights<E>(w, f, in);
#pragma unroll
            for (int i = 0; i < E; i++) {
                const int b = bin(f[i]);
                if (b < SAMPLE_BINS) atomicAdd((unsigned long long *)&lds.sum[b], (unsigned long long)(w[i] - NO_WEIGHT));
            }
        });
        __syncthreads();
    }
    // Puts the values of the bins from `low` to `high` into the list
    __device__ __forceinline__ void enlist(const float (&f)[E], int at, int low, int high) const {
#pragma unroll
        for (int i = 0; i < E; i++) {
            const int b = bin(f[i]);
            if (b >= low && b <= high) {
                const int n = atomicAdd(&lds.listed, 1);
                if (n < LIST) lds.list[n] = (u64)key_of(f[i]) << 32 | ~(u32)(at + i);
            }
        }
    }
    __device__ __forceinline__ void gather(int first, int end, int high) const {
        walk_part(first, end, [&](const float (&f)[E], int at) {
            float most = f[0];
#pragma unroll
            for (int i = 1; i < E; i++) most = fmaxf(most, f[i]);
            if (bin(most) <= high) enlist(f, at, 0, high);
        });
        __syncthreads();
    }
    // Weights of what `in` holds for, summed over each segment; look(values, index of the first) sees all
    template <class IN, class LOOK>
    __device__ __forceinline__ void sums(int first_segment, int end_segment, u64 *into, const IN &in, const LOOK &look) const {
        u64 s = 0;
        const auto add = [&](const float (&f)[E], int at) {
            u64 w[E];
            bool is[E], any = false;
#pragma unroll
            for (int i = 0; i < E; i++) any |= is[i] = in(f[i], at + i);
            look(f, at);
            if (!__any(any)) return;
            weights<E>(w, f, is);
#pragma unroll
            for (int i = 0; i < E; i++) s += w[i];
            s -= E * NO_WEIGHT;
        };
        for (int segment = first_segment + wave; segment < end_segment; segment += SAMPLE_WAVES) {
            s = 0;
            walk_slowly(segment * per, min((segment + 1) * per, tiles), 1, add);
            s = wave_sum(s);
            if (lane == 0) into[segment] = s;
        }
    }
    __device__ __forceinline__ void kept_sums(int first_segment, int end_segment, u64 *into) const {
        sums(first_segment, end_segment, into, [&](float f, int at) { return kept(f, at); }, [](const float (&)[E], int) {});
    }
    // Those above a bin, which goes into the list
    __device__ __forceinline__ void sums_above(int first_segment, int end_segment, u64 *into, int border) const {
        sums(first_segment, end_segment, into, [&](float f, int) { return bin(f) < border && f >= small; }, [&](const float (&f)[E], int at) { enlist(f, at, border, border); });
        __syncthreads();
    }
    // The first index at which the running sum of of(weights, values, index of the first), whose sums over segments are in lds.sum, reaches target(the whole sum) >= 1
    template <class OF, class TARGET>
    __device__ __forceinline__ int pick(const OF &of, const TARGET &target_of) const {
        const u64 target = find<false>((tiles + per - 1) / per, target_of);
        const int segment = lds.found;
        u64 before = lds.found_before;
        __syncthreads();
        if (wave == 0) {
            for (int tile = segment * per; tile < min((segment + 1) * per, tiles); tile++) {
                float f[E];
                widen(f, fetch(tile));
                u64 w[E], mine = 0;
                of(w, f, tile * TILE + lane * E);
#pragma unroll
                for (int i = 0; i < E; i++) mine += w[i];
                const u64 s = wave_scan(mine), reached = __ballot(before + s >= target);
                if (reached) {
                    if (lane == __ffsll((unsigned long long)reached) - 1) {
                        u64 run = before + s - mine;
                        int at = 0;
#pragma unroll
                        for (int i = 0; i < E; i++) {
                            if (run < target) at = i;
                            run += w[i];
                        }
                        lds.found = tile * TILE + lane * E + at;
                    }
                    break;
                }
                before += wave_last(s);
            }
        }
        __syncthreads();
        return lds.found;
    }
    // The token, once the bound is known and the sums of the segments are in lds.sum
    __device__ __forceinline__ int draw() const {
        return pick(
            [&](u64(&w)[E], const float (&f)[E], int at) {
                bool is[E];
#pragma unroll
                for (int i = 0; i < E; i++) is[i] = kept(f[i], at + i);
                weights<E>(w, f, is);
#pragma unroll
                for (int i = 0; i < E; i++) w[i] -= NO_WEIGHT;
            },
            [&](u64 sum) { return draw_target(sum, u) + 1; });
    }
    // min_p leaves the front part of what is kept
    __device__ __forceinline__ void keep_small() {
        if (small > edge) {
            edge = small;
            last = INT32_MAX;
        }
    }
    // Moves the bound to where the running sum of counts or weights, in the order, reaches `target` >= 1; leaves it where the whole is less.  In the whole row.
    template <bool COUNTS>
    __device__ __forceinline__ void bound(u64 target) {
        const auto each = [&](const auto &todo) {
            walk(wave, tiles, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
#pragma unroll
                for (int i = 0; i < E; i++)
                    if (kept(f[i], at + i)) todo(key_of(f[i]), [&] { return weight(f[i]); });
            });
        };
        if (COUNTS) count_bins(0, tiles);  // (nothing is cut before)
        else sum_bins(0, tiles);
        find_at<COUNTS>(SAMPLE_BINS, target);
        const int border = lds.found;
        if (border == SAMPLE_BINS) return;
        target -= lds.found_before;
        // the values in that bin
        u32 low = ~0u, high = 0;
        walk(wave, tiles, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (bin(f[i]) == border && kept(f[i], at + i)) {
                    low = min(low, key_of(f[i]));
                    high = max(high, key_of(f[i]));
                }
        });
        low = reduce(low, ~0u, lds.low, [](u32 a, u32 b) { return min(a, b); });
        high = reduce(high, 0, lds.high, [](u32 a, u32 b) { return max(a, b); });
        int ties;
        const float at = of_key(select<COUNTS>(low, high, target, ties, each));
        if (edge != at) last = INT32_MAX;  // (equal ones may have been cut before)
        edge = at;
        u64 needed = target;
        if (!COUNTS) {
            const u64 w = weight(edge);
            needed = w ? (target + w - 1) / w : ties;
        }
        if (needed >= (u64)ties) return;
        // how many of the equal ones each segment has
        __syncthreads();
        for (int segment = wave; segment * per < tiles; segment += SAMPLE_WAVES) {
            u32 n = 0;
            walk(segment * per, min((segment + 1) * per, tiles), 1, [&](const float (&f)[E], int) {
#pragma unroll
                for (int i = 0; i < E; i++) n += f[i] == at;
            });
#pragma unroll
            for (int k = 1; k < 64; k *= 2) n += __shfl_xor(n, k);
            if (lane == 0) lds.sum[segment] = n;
        }
        last = pick(
            [&](u64(&w)[E], const float (&f)[E], int) {
#pragma unroll
                for (int i = 0; i < E; i++) w[i] = f[i] == at ? 1 : 0;
            },
            [=](u64) { return needed; });
    }
    __device__ __forceinline__ int slowly() {
        if (k) bound<true>(k);
        if (p < 1) {
            u64 sum = 0;
            if (k) {
                walk_slowly(wave, tiles, SAMPLE_WAVES, [&](const float (&f)[E], int at) {
                    u64 w[E];
                    bool is[E];
#pragma unroll
                    for (int i = 0; i < E; i++) is[i] = kept(f[i], at + i);
                    weights<E>(w, f, is);
#pragma unroll
                    for (int i = 0; i < E; i++) sum += w[i] - NO_WEIGHT;
                });
            } else {
                sum_bins(0, tiles);
                sum = lds.sum[threadIdx.x] + lds.sum[threadIdx.x + SAMPLE_THREADS];
            }
            bound<false>(part_target(total(sum), p));
        }
        keep_small();
        __syncthreads();
        kept_sums(0, (tiles + per - 1) / per, lds.sum);
        return draw();
    }
    // The same for few elements that are spread over the bins, each(todo) with todo(bin, order, weight).  First the bin where the running sum reaches `target`: into lds.found, how many
    // there are in lds.count; returns what is left of the target
    template <bool COUNTS, class EACH>
    __device__ __forceinline__ u64 find_spread(u64 target, const EACH &each) const {
        clear_bins();
        if (threadIdx.x == 0) lds.few = 0;
        each([&](int b, u64, const auto &weight) {
            atomicAdd(&lds.count[b], 1u);
            if (!COUNTS) atomicAdd((unsigned long long *)&lds.sum[b], (unsigned long long)weight());
        });
        find_at<COUNTS>(SAMPLE_BINS, target);
        return target - lds.found_before;
    }
    // then, for up to 64 of them, the order (a falling one, never 0) of the element: a wave compares each with each
    template <bool COUNTS, class EACH>
    __device__ __forceinline__ u64 order_spread(u64 target, const EACH &each) const {
        const int border = lds.found;
        each([&](int b, u64 order, const auto &weight) {
            if (b == border) {
                const int i = atomicAdd(&lds.few, 1);
                lds.order[i] = order;
                lds.load[i] = COUNTS ? 1 : weight();
            }
        });
        __syncthreads();
        if (wave == 0) {
            const int n = lds.few;
            const u64 mine = lane < n ? lds.order[lane] : 0, w = lane < n ? lds.load[lane] : 0;
            u64 before = 0;
            for (int i = 0; i < n; i++) before += lds.order[i] > mine ? lds.load[i] : 0;
            if (before < target && before + w >= target) lds.found_before = mine;  // (of one lane: the orders differ)
        }
        __syncthreads();
        return lds.found_before;  // (a barrier before it is written again is clear_bins')
    }
    // ---- in the list of candidates
    template <class TODO>
    __device__ __forceinline__ void each_listed(const TODO &todo) const {
        for (int i = threadIdx.x; i < lds.listed; i += SAMPLE_THREADS) {
            const u64 e = lds.list[i];
            if (kept(of_key((u32)(e >> 32)), (int)~(u32)e)) todo((u32)(e >> 32), ~(u32)e);
        }
    }
    __device__ __forceinline__ int index_bin(u32 i) const { return (int)(i >> max(0, 21 - __clz(vocab - 1))); }  // 2048 bins of indices
    // Moves the bound as above, to one among the candidates, which are in the bins from `from` to `to`.
    template <bool COUNTS>
    __device__ __forceinline__ void bound_listed(u64 target, int from, int to) {
        const float finer = (float)SAMPLE_BINS / (to + 1 - from);
        const auto bin_of = [&](u32 key) { return max(0, min((int)((half_distance(of_key(key)) * bins - from) * finer), SAMPLE_BINS - 1)); };
        const auto by_value = [&](const auto &todo) {
            each_listed([&](u32 key, u32 i) { todo(bin_of(key), (u64)key << 32 | ~i, [&] { return weight(of_key(key)); }); });
        };
        target = find_spread<COUNTS>(target, by_value);
        const int border = lds.found;
        int ties = (int)lds.count[border];
        if (ties <= 64) {
            const u64 order = order_spread<COUNTS>(target, by_value);
            edge = of_key((u32)(order >> 32));
            last = (int)~(u32)order;
            return;
        }
        // many: 16 bits leave few values to a bin
        u32 low = ~0u, high = 0;
        each_listed([&](u32 key, u32) {
            if (bin_of(key) != border) return;
            low = min(low, key);
            high = max(high, key);
        });
        low = reduce(low, ~0u, lds.low, [](u32 a, u32 b) { return min(a, b); });
        high = reduce(high, 0, lds.high, [](u32 a, u32 b) { return max(a, b); });
        if (low != high) high = select<COUNTS>(low, high, target, ties, [&](const auto &todo) { each_listed([&](u32 key, u32) { todo(key, [&] { return weight(of_key(key)); }); }); });
        const u32 key = high;
        const float value = of_key(key);
        u64 needed = target;
        if (!COUNTS) {
            const u64 w = weight(value);
            needed = w ? (target + w - 1) / w : ties;
        }
        int index = edge == value ? last : INT32_MAX;
        if (needed < (u64)ties) index = index_listed<true>(needed, [=](u32 k) { return k == key; });
        edge = value;
        last = index;
    }
    // The index at which the running sum of the candidates `in` holds for, by index, reaches `target`
    template <bool COUNTS, class IN>
    __device__ __forceinline__ int index_listed(u64 target, const IN &in) const {
        const auto by_index = [&](const auto &todo) {
            each_listed([&](u32 key, u32 i) {
                if (in(key)) todo(index_bin(i), ~(u64)i, [&] { return weight(of_key(key)); });
            });
        };
        u64 rest = find_spread<COUNTS>(target, by_index);
        if (lds.count[lds.found] <= 64) return (int)~(u32)order_spread<COUNTS>(rest, by_index);
        int ties;
        return (int)~select<COUNTS>(~(u32)(vocab - 1), ~0u, target, ties, [&](const auto &todo) {
            each_listed([&](u32 key, u32 i) {
                if (in(key)) todo(~i, [&] { return weight(of_key(key)); });
            });
        });
    }
    // The token of a row whose top k are among few candidates, four threads to each; waves without one are done.  -1 in threads that do not have it.
    __device__ __forceinline__ int finish_pairs(int n) const {
        if (16 * wave >= n) return -1;
        const int mine = threadIdx.x / 4, sub = threadIdx.x % 4;
        const bool there = mine < n;
        u64 *const w_of = lds.sum, *const run_of = lds.sum + SAMPLE_PAIRS, *const sorted_w = lds.sum + 2 * SAMPLE_PAIRS, *const sorted = lds.list + SAMPLE_PAIRS;
        const auto quad = [](auto v) {  // sum over the four
            v += from_lane<0xb1, 0xf>((decltype(v))0, v);
            v += from_lane<0x4e, 0xf>((decltype(v))0, v);
            return v;
        };
        const u64 e = there ? lds.list[mine] : 0;
        u64 w = weight(of_key((u32)(e >> 32)));
        if (sub == 0 && there) w_of[mine] = w;
        __syncthreads();
        // how many come before it, and what they weigh
        u32 rank = 0;
        u64 before = 0;
        for (int i = sub; i < n; i += 4) {
            const bool ahead = lds.list[i] > e;
            rank += ahead;
            before += ahead ? w_of[i] : 0;
        }
        rank = quad(rank);
        before = quad(before);
        if (sub == 0 && there) {
            sorted[rank] = e;
            sorted_w[rank] = w;
            run_of[rank] = before + w;
        }
        __syncthreads();
        // how many the filters leave: each leaves the front ones
        const int most = min(k, n);
        const u64 target = p < 1 ? part_target(run_of[most - 1], p) : ~(u64)0;
        int left = 0;
        for (int at = 0; at < most; at += 64) {
            const int i = at + lane;
            const bool in = i < most && (i == 0 || run_of[max(i, 1) - 1] < target) && of_key((u32)(sorted[min(i, most - 1)] >> 32)) >= small;
            left += __popcll(__ballot(in));
        }
        const u64 at = draw_target(run_of[left - 1], u);
        before = 0;
        for (int i = sub; i < left; i += 4) before += (u32)sorted[i] > (u32)e ? sorted_w[i] : 0;  // (indices are inverted)
        before = quad(before);
        return there && (int)rank < left && before <= at && at < before + w ? (int)~(u32)e : -1;
    }
    // The token of a row whose top k are among the candidates
    __device__ __forceinline__ int finish_listed(int limit) {
        const int n = lds.listed;
        if (n <= SAMPLE_PAIRS) return finish_pairs(n);
        const auto sum = [&] {
            u64 s = 0;
            each_listed([&](u32 key, u32) { s += weight(of_key(key)); });
            return total(s);
        };
        if (k < n) bound_listed<true>(k, 0, limit);
        if (p < 1) bound_listed<false>(part_target(sum(), p), 0, limit);
        keep_small();
        return index_listed<false>(draw_target(sum(), u) + 1, [](u32) { return true; });
    }
    // The token of a row whose bound by top_p is among the candidates, where it leaves `rest` of the sum; the segments' sums of what is above are in lds.sum
    __device__ __forceinline__ int finish_part(u64 rest, int border, u64 *sums) {
        bound_listed<false>(rest, border, border);  // (it works in lds.sum)
        keep_small();
        __syncthreads();
        for (int i = threadIdx.x; i * per < tiles; i += SAMPLE_THREADS) lds.sum[i] = sums[i];
        __syncthreads();
        each_listed([&](u32 key, u32 i) { atomicAdd((unsigned long long *)&lds.sum[i / TILE / per], (unsigned long long)weight(of_key(key))); });
        return draw();
    }
};

// A workgroup to a row
template <int TYPE, bool HELD>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample(ensi_clear_sample_args a) {
    __shared__ SampleLds<SAMPLE_LIST> lds;
    __shared__ u64 above[SAMPLE_SEGMENTS];
    SampleRow<TYPE, HELD> r(a, blockIdx.x, lds);
    r.set_roots();
    if (threadIdx.x == 0) lds.listed = 0;
    const float mine = r.largest(0, r.tiles);
    SampleMode mode = r.begin(__builtin_bit_cast(float, r.reduce(__builtin_bit_cast(u32, mine), __builtin_bit_cast(u32, -__builtin_inff()), lds.low, larger)));
    const int tiles = r.tiles, segments = (tiles + r.per - 1) / r.per;
    int token = -1;
    if (mode == SAMPLE_FIRST) token = r.first_largest(0, tiles);
    if (mode == SAMPLE_TOP) {
        int limit = SAMPLE_BINS - 1;  // candidates: the bins up to this one
        if (a.vocab > SAMPLE_LIST) {
            if (r.k <= SAMPLE_FEW) {
                r.clear_bins();
                const int b = r.bin(mine);
                if (b < SAMPLE_BINS) atomicAdd(&lds.count[b], 1u);
            } else
                r.count_bins(0, tiles);
            r.template find_at<true>(SAMPLE_BINS, r.k);
            limit = min(lds.found, limit);
        }
        r.gather(0, tiles, limit);
        if (lds.listed <= SAMPLE_PAIRS) {
            token = r.finish_pairs(lds.listed);
            if (token >= 0) a.out[blockIdx.x] = token;
            return;
        }
        if (lds.listed <= SAMPLE_LIST) token = r.finish_listed(limit);
        else mode = SAMPLE_SLOW;
    }
    if (mode == SAMPLE_PART) {
        r.sum_bins(0, tiles);
        const u64 target = r.template find<false>(SAMPLE_BINS, [&](u64 sum) { return part_target(sum, r.p); });
        const int border = lds.found;
        const u64 rest = target - lds.found_before;
        r.sums_above(0, segments, above, border);
        if (lds.listed <= SAMPLE_LIST) token = r.finish_part(rest, border, above);
        else mode = SAMPLE_SLOW;
    }
    if (mode == SAMPLE_ALL) {
        __syncthreads();
        r.kept_sums(0, segments, lds.sum);
        token = r.draw();
    }
    if (mode == SAMPLE_SLOW) token = r.slowly();
    if (threadIdx.x == 0) a.out[blockIdx.x] = token;
}

// ---- Several workgroups to a row, for rows that are fewer than the CUs: the same in four launches, which leave in the workspace what the next one needs.  All sums are exact, so
// the token is the same, and neither the order in which bins are added up nor that of the list matters.
struct SampleParts {
    ensi_clear_sample_args a;
    SampleShared *row;
    int parts;
};
// The segments and tiles of a part
template <class ROW>
struct SampleRange {
    int segment0, segment1, tile0, tile1;
    __device__ __forceinline__ SampleRange(const ROW &r, int parts, int i) {
        const int segments = (r.tiles + r.per - 1) / r.per, each = (segments + parts - 1) / parts;
        segment0 = min(i * each, segments);
        segment1 = min(segment0 + each, segments);
        tile0 = segment0 * r.per;
        tile1 = min(segment1 * r.per, r.tiles);
    }
};
template <class ROW>
__device__ __forceinline__ SampleMode begin_part(ROW &r, const SampleShared &row, int parts) {
    static_assert(SAMPLE_PARTS == 8, "one of them to a lane of each eight");
    const u32 most = __builtin_bit_cast(u32, row.most[min((int)threadIdx.x % 8, parts - 1)]);
    return r.begin(__builtin_bit_cast(float, __builtin_amdgcn_readlane((int)wave_scan(most, __builtin_bit_cast(u32, -__builtin_inff()), larger), 63)));
}
// The bin with the bound into lds.found; what is left there of the target
template <class ROW>
__device__ __forceinline__ u64 find_part(const ROW &r, const SampleShared &row, SampleMode mode) {
    const u64 b0 = row.bins[threadIdx.x], b1 = row.bins[threadIdx.x + SAMPLE_THREADS];
    r.lds.sum[threadIdx.x] = b0;
    r.lds.sum[threadIdx.x + SAMPLE_THREADS] = b1;
    const u64 target = r.template find<false>(SAMPLE_BINS, [&](u64 sum) { return mode == SAMPLE_TOP ? (u64)r.k : part_target(sum, r.p); });
    return target - r.lds.found_before;
}

template <int TYPE>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample_most(SampleParts s) {
    __shared__ SampleLds<SAMPLE_LIST> lds;
    SampleShared &row = s.row[blockIdx.y];
    const SampleRow<TYPE, false> r(s.a, blockIdx.y, lds);
    const SampleRange<SampleRow<TYPE, false>> g(r, s.parts, blockIdx.x);
    for (int i = blockIdx.x * SAMPLE_THREADS + threadIdx.x; i < SAMPLE_BINS; i += s.parts * SAMPLE_THREADS) row.bins[i] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) row.listed = 0;
    const float mine = r.largest(g.tile0, g.tile1);
    row.threads[blockIdx.x * SAMPLE_THREADS + threadIdx.x] = mine;
    const u32 most = r.reduce(__builtin_bit_cast(u32, mine), __builtin_bit_cast(u32, -__builtin_inff()), lds.low, larger);
    if (threadIdx.x == 0) row.most[blockIdx.x] = __builtin_bit_cast(float, most);
}
template <int TYPE>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample_bins(SampleParts s) {
    __shared__ SampleLds<SAMPLE_LIST> lds;
    SampleShared &row = s.row[blockIdx.y];
    SampleRow<TYPE, false> r(s.a, blockIdx.y, lds);
    const SampleRange<SampleRow<TYPE, false>> g(r, s.parts, blockIdx.x);
    const SampleMode mode = begin_part(r, row, s.parts);
    if (mode == SAMPLE_FIRST) {
        const int first = r.first_largest(g.tile0, g.tile1);
        if (threadIdx.x == 0) row.first[blockIdx.x] = first;
    } else if (mode == SAMPLE_TOP && r.k > SAMPLE_FEW * s.parts) {
        r.count_bins(g.tile0, g.tile1);
        for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS)
            if (lds.count[i]) atomicAdd((unsigned long long *)&row.bins[i], (unsigned long long)lds.count[i]);
    } else if (mode == SAMPLE_PART) {
        r.set_roots();
        r.sum_bins(g.tile0, g.tile1);
        for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_THREADS)
            if (lds.sum[i]) atomicAdd((unsigned long long *)&row.bins[i], (unsigned long long)lds.sum[i]);
    } else if (mode == SAMPLE_ALL) {
        r.set_roots();
        __syncthreads();
        r.kept_sums(g.segment0, g.segment1, row.sum);
    }
}
template <int TYPE>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample_gather(SampleParts s) {
    __shared__ SampleLds<SAMPLE_LIST> lds;
    __shared__ int at;
    SampleShared &row = s.row[blockIdx.y];
    SampleRow<TYPE, false> r(s.a, blockIdx.y, lds);
    const SampleRange<SampleRow<TYPE, false>> g(r, s.parts, blockIdx.x);
    const SampleMode mode = begin_part(r, row, s.parts);
    if (mode != SAMPLE_TOP && mode != SAMPLE_PART) return;
    if (threadIdx.x == 0) lds.listed = 0;
    if (mode == SAMPLE_TOP) {
        if (r.k <= SAMPLE_FEW * s.parts) {
            r.clear_bins();
            float most[SAMPLE_PARTS];
#pragma unroll
            for (int i = 0; i < SAMPLE_PARTS; i++) most[i] = i < s.parts ? row.threads[i * SAMPLE_THREADS + threadIdx.x] : -__builtin_inff();
#pragma unroll
            for (int i = 0; i < SAMPLE_PARTS; i++) {
                const int b = r.bin(most[i]);
                if (b < SAMPLE_BINS) atomicAdd(&lds.count[b], 1u);
            }
            r.template find_at<true>(SAMPLE_BINS, r.k);
        } else
            find_part(r, row, mode);
        r.gather(g.tile0, g.tile1, min(lds.found, SAMPLE_BINS - 1));
    } else {
        r.set_roots();
        const u64 rest = find_part(r, row, mode);
        const int border = lds.found;
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            row.border = border;
            row.rest = rest;
        }
        r.sums_above(g.segment0, g.segment1, row.sum, border);
    }
    const int listed = lds.listed;
    if (threadIdx.x == 0) at = atomicAdd(&row.listed, listed <= SAMPLE_LIST ? listed : SAMPLE_LONG + 1);  // (past the list's end where there are too many, of this part or of all)
    __syncthreads();
    for (int i = threadIdx.x; i < min(listed, SAMPLE_LIST) && at + i < SAMPLE_LONG; i += SAMPLE_THREADS) row.list[at + i] = lds.list[i];
}
template <int TYPE, int LIST>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_clear_sample_finish(SampleParts s) {
    __shared__ SampleLds<LIST> lds;
    SampleShared &row = s.row[blockIdx.x];
    SampleRow<TYPE, false, LIST> r(s.a, blockIdx.x, lds);
    SampleMode mode = begin_part(r, row, s.parts);
    int token = -1;
    r.set_roots();
    if (mode == SAMPLE_FIRST) {
        token = INT32_MAX;
        for (int i = 0; i < s.parts; i++) token = min(token, row.first[i]);
    }
    if (mode == SAMPLE_TOP || mode == SAMPLE_PART) {
        const int listed = row.listed;
        if (listed <= LIST) {
            for (int i = threadIdx.x; i < listed; i += SAMPLE_THREADS) lds.list[i] = row.list[i];
            if (threadIdx.x == 0) lds.listed = listed;
            if (mode == SAMPLE_TOP && listed <= SAMPLE_PAIRS) {
                __syncthreads();
                token = r.finish_pairs(listed);
                if (token >= 0) s.a.out[blockIdx.x] = token;
                return;
            }
            const int border = row.border;
            const u64 rest = row.rest;
            __syncthreads();
            token = mode == SAMPLE_TOP ? r.finish_listed(SAMPLE_BINS - 1) : r.finish_part(rest, border, row.sum);
        } else {
            mode = SAMPLE_SLOW;
            __syncthreads();
        }
    }
    if (mode == SAMPLE_ALL) {
        for (int i = threadIdx.x; i * r.per < r.tiles; i += SAMPLE_THREADS) lds.sum[i] = row.sum[i];
        token = r.draw();
    }
    if (mode == SAMPLE_SLOW) {
        __syncthreads();
        token = r.slowly();
    }
    if (threadIdx.x == 0) s.a.out[blockIdx.x] = token;
}

template <int TYPE>
static void sample_type(ensi_ctx *ctx, const ensi_clear_sample_args &a, hipStream_t st) {
    constexpr int E = SampleRow<TYPE, false>::E, TILE = SampleRow<TYPE, false>::TILE;
    const dim3 block(SAMPLE_THREADS);
    // As many workgroups to a row as give the CUs four each, while a thread has two turns of its part (of 128000 logits: 64 rows 54 us in eight parts, 90 whole; 256 rows in f32 95 in four, 112 in
    // two, 110 whole).  A row that the registers of one workgroup hold stays there between the passes (32000: 9.7 us, 10.2 without).
    int parts = (int)min((int64_t)SAMPLE_PARTS, 1024 / a.rows);
    parts = min(parts, a.vocab / (2 * SAMPLE_THREADS * E));
    static_assert(512 * sizeof(SampleShared) <= CLEAR_WS_FLOATS * 4, "rows that are split are 512 at most");
    ScopedTimer timer(ctx, "k_clear_sample", st);
    if (parts < 2 || !ctx->ws_clear) {
        if (a.vocab <= 64 * TILE) hipLaunchKernelGGL((k_clear_sample<TYPE, true>), dim3((u32)a.rows), block, 0, st, a);
        else hipLaunchKernelGGL((k_clear_sample<TYPE, false>), dim3((u32)a.rows), block, 0, st, a);
        return;
    }
    const SampleParts s = {a, (SampleShared *)ctx->ws_clear, parts};
    const dim3 grid(parts, (u32)a.rows);
    hipLaunchKernelGGL(k_clear_sample_most<TYPE>, grid, block, 0, st, s);
    // (nothing to do there with a few of every row's tokens: 64 rows of 128000, top 50 29 us with it, 26 without)
    const bool few = !a.temperature && a.all_temperature > 0 && !a.top_k && a.all_top_k > 0 && a.all_top_k <= SAMPLE_FEW * parts && a.all_top_k < a.vocab;
    if (!few) hipLaunchKernelGGL(k_clear_sample_bins<TYPE>, grid, block, 0, st, s);
    if (a.top_k || a.top_p || a.all_top_k > 0 || a.all_top_p < 1) hipLaunchKernelGGL(k_clear_sample_gather<TYPE>, grid, block, 0, st, s);
    // The k-th of T largest values of threads leaves T ln(T / (T - k)) candidates on the average, 1.4 k of them for the largest k that is looked for there: from six workgroups on more than
    // SAMPLE_LIST, which two rows to a CU have room for; rows that so many share are one to a CU.  (One row of 131072, top 3584: 37 us, 174 where the row itself is searched; 128 rows 70 and 209.)
    if (SAMPLE_FEW * parts * 1.5f > SAMPLE_LIST) hipLaunchKernelGGL((k_clear_sample_finish<TYPE, SAMPLE_LONG>), dim3((u32)a.rows), block, 0, st, s);
    else hipLaunchKernelGGL((k_clear_sample_finish<TYPE, SAMPLE_LIST>), dim3((u32)a.rows), block, 0, st, s);
}

void launch_clear_sample(ensi_ctx *ctx, const ensi_clear_sample_args &a, hipStream_t st) {
    if (a.type == ENSI_T_F32) sample_type<ENSI_T_F32>(ctx, a, st);
    else if (a.type == ENSI_T_BF16) sample_type<ENSI_T_BF16>(ctx, a, st);
    else sample_type<ENSI_T_F16>(ctx, a, st);
}
