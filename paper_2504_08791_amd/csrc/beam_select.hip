// The best continuations of a set of beams: score = the beam's + x - log sum exp x over beams and vocabulary, the n_best highest, of equal ones
// the lowest index.  The logits are read once:
//  * beam_scan_kernel: a wave takes 64 E consecutive logits of a row into registers and forms their maximum and sum of exponentials; a workgroup of four waves keeps its
//    `keep` largest logits (of equal ones the lowest token first).  A number that `keep` of its 256 lanes' maxima reach, found with a few ballots, is a threshold
//    that at least `keep` elements reach and few others; those are ranked by counting.  A row's score order is its logit order, so no sum is needed yet.
//  * beam_pick_kernel: a workgroup takes a sequence: the sums of each beam joined, the kept logits turned into scores, the same threshold over
//    its threads' maxima, ranks by counting.
// Where more elements than fit reach a threshold (many equal ones, or rows in order of their logits) the best are taken out one by one, or, of a whole workgroup, the threshold is
// raised by counting.
// Measured: 16 searches of 8 beams over 128256 fp32 logits (65.7 MB) 20.5 us, some 14.5 of them the first launch at 4.5 TB/s (vector units: an exponential, a maximum, a comparison
// and a ballot a logit; its last wave ranks alone), the rest latencies of one workgroup a search; one of 4 beams over 32000 8.2; 4 of 16 over 151936 19.1.  16-bit
// logits are no faster (20.7): what a logit costs the vector units does not halve with its bytes.
// Rounding: x - log sum exp x and the sum with the beam's score never reorder logits but may make two of them equal, and then the lower token comes
// first, though a workgroup may have kept the other.  That needs a list all of whose elements are chosen or tie with the last one chosen: it has one more than can be
// chosen, and where even that one ties, its logits are read again for tokens of exactly that score.
#include "common.h"

namespace prima {

typedef float v4f_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef _Float16 v8h_a2 __attribute__((ext_vector_type(8), aligned(2)));
typedef unsigned short v8s_a2 __attribute__((ext_vector_type(8), aligned(2)));

struct LogitF32 {
    typedef float type;
    static constexpr int N = 4; // elements of a load
    __device__ static float one(const float *p) { return *p; }
    __device__ static void load(const float *p, float *x)
    {
        const v4f_a4 v = *reinterpret_cast<const v4f_a4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
};
struct LogitF16 {
    typedef _Float16 type;
    static constexpr int N = 8;
    __device__ static float one(const _Float16 *p) { return static_cast<float>(*p); }
    __device__ static void load(const _Float16 *p, float *x)
    {
        const v8h_a2 v = *reinterpret_cast<const v8h_a2 *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(v[i]);
    }
};
struct LogitBF16 {
    typedef unsigned short type;
    static constexpr int N = 8;
    __device__ static float one(const unsigned short *p) { return __builtin_bit_cast(float, static_cast<unsigned>(*p) << 16); }
    __device__ static void load(const unsigned short *p, float *x)
    {
        const v8s_a2 v = *reinterpret_cast<const v8s_a2 *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(float, static_cast<unsigned>(v[i]) << 16);
    }
};

struct Kept { // an element a wave keeps
    float x;
    int token; // -1: the wave has no more
};
struct BeamArgs {
    const void *logits;
    int64_t ld;
    int B, W, V, n_best, keep, nc, eos; // nc: workgroups a row
    const float *scores;
    const uint8_t *done;
    float *out_scores;
    int32_t *out_beams, *out_tokens;
    float2 *part; // [B W][nc] (maximum, sum)
    Kept *kept;   // [B W][nc][keep]
};

// a float as an unsigned number of the same order
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// how many of the lanes' N keys reach t
template <int N>
__device__ __forceinline__ int reaching(const uint32_t (&key)[N], uint32_t t)
{
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __builtin_popcountll(__ballot(key[i] >= t));
    return n;
}
// A threshold that at least n of the 64 N keys reach (n <= 64 N) and few more: down from the largest in growing steps until n do, then halfway back until no more
// than one too many does or nothing lies between.  (The n-th largest itself, bit by bit, takes 20 to 32 counts; this 5 to 10.)
template <int N>
__device__ __forceinline__ uint32_t nth_largest(const uint32_t (&key)[N], uint32_t largest, int n)
{
    largest = __builtin_amdgcn_readfirstlane(largest); // (the same in all lanes)
    uint32_t over = largest, step = 1u << 20; // over: too few reach it (or it is the largest)
    uint32_t t = largest;
    int have = reaching(key, t);
    while (have < n) { // (all of them reach 0)
        over = t;
        t = t > step ? t - step : 0;
        step = step < 1u << 30 ? 2 * step : step;
        have = reaching(key, t);
    }
    while (have > n + 1 && over - t > 1) {
        const uint32_t mid = t + (over - t) / 2;
        const int h = reaching(key, mid);
        if (h >= n) { t = mid; have = h; }
        else over = mid;
    }
    return t;
}
// A threshold t that `have` numbers reach, too many, raised until between n and `most` of them do, or nothing lies between it and `over`, which fewer than n reach.
// count(float): how many of the wave's numbers reach it.  (t and over are those of numbers, never of NaN.)
template <class F>
__device__ __forceinline__ void raise_threshold(uint32_t &t, int &have, uint32_t over, int n, int most, F count)
{
    while (have > most && over - t > 1) {
        const uint32_t mid = t + (over - t) / 2;
        const int h = count(unordered(mid));
        if (h >= n) { t = mid; have = h; }
        else over = mid;
    }
}

constexpr float LOG2E = 1.44269504088896340736f;

// Sums of exponentials are kept as (m, s): 2^m s, m the largest logit times log2 e, rounded (the same number in every term, so its rounding is in none).
// Two of them together; a sum that is NaN stays NaN
__device__ __forceinline__ float2 add_sums(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x);
    if (m == -INFINITY) return make_float2(m, a.y + b.y);
    return make_float2(m, a.y * __builtin_amdgcn_exp2f(a.x - m) + b.y * __builtin_amdgcn_exp2f(b.x - m));
}

// how many of the lanes in `who` come before this one
__device__ __forceinline__ int lanes_below(uint64_t who)
{
    return __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(who >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(who), 0));
}

constexpr int SCAN_WAVES = 4;

constexpr int SCAN_FEW = 48; // to keep: of those that reach the threshold, a sixth more or so, one wave has hardly ever more than 64

// SCAN_LIST: what a wave hands on at most: 64, or 128 for many to keep
// (E == 32: 85 registers for 32 logits, and still 24 waves a compute unit with 8 KiB each on their way.)
template <class L, int E, int SCAN_LIST>
__global__ void __launch_bounds__(64 * SCAN_WAVES, E == 32 ? 6 : 8) beam_scan_kernel(BeamArgs a)
{
    typedef typename L::type T;
    constexpr int N = L::N, G = E / N;
    __shared__ Kept list[SCAN_WAVES][SCAN_LIST], top[SCAN_WAVES * SCAN_LIST];
    __shared__ float2 sums[SCAN_WAVES];
    __shared__ uint32_t maxima[SCAN_WAVES * 64];
    __shared__ int counts[SCAN_WAVES];
    const int row = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (a.done && a.done[row]) return; // (the whole workgroup)
    const T *p = static_cast<const T *>(a.logits) + row * a.ld;
    const int start = (blockIdx.x * SCAN_WAVES + wave) * 64 * E;
    const bool full = start + 64 * E <= a.V;
    auto token_of = [&](int e) { return start + (e / N) * 64 * N + lane * N + e % N; };
    float x[E];
    if (full) {
#pragma unroll
        for (int g = 0; g < G; ++g) L::load(p + token_of(g * N), x + g * N);
#pragma unroll
        for (int e = 0; e < E; ++e) asm("" : "+v"(x[e])); // (numbers: nothing needs to be made one, or widened, at every use)
    } else { // past the end: NaN, which no comparison takes
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = token_of(e) < a.V ? L::one(p + token_of(e)) : __builtin_nanf("");
    }
    float most = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) most = fmaxf(most, x[e]);
    const float m = wave_max(most), m2 = m == -INFINITY ? 0.f : m * LOG2E;
    float s = 0.f;
    if (full) {
#pragma unroll
        for (int e = 0; e < E; ++e) s += __builtin_amdgcn_exp2f(fmaf(x[e], LOG2E, -m2)); // (+infinity and NaN make it NaN)
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) s += token_of(e) < a.V ? __builtin_amdgcn_exp2f(fmaf(x[e], LOG2E, -m2)) : 0.f;
    }
    s = wave_sum(s);
    if (lane == 0) sums[wave] = make_float2(m == -INFINITY ? -INFINITY : m2, s);
    if (a.V - start < 64 * N) { // few: for the threshold, dealt to all lanes (N in a row to each of the first would leave the others without a maximum)
        most = -INFINITY;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (start + 64 * e + lane < a.V) most = fmaxf(most, L::one(p + start + 64 * e + lane));
    }
    if (!(s == s)) { // the beam's scores are all -infinity: the lowest tokens first
        most = -INFINITY;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = token_of(e) < a.V ? -INFINITY : __builtin_nanf("");
    }

    // what reaches the workgroup's threshold, in any order.  (Among the maxima of 256 lanes it is one that few more than are to be kept reach; each wave's own, among 64, three times as
    // many.  us of both launches, a wave's / the workgroup's: 4 searches of 16 beams over 151936 fp32 logits 20.7 / 19.1, 16 of eight over 128256 20.8 / 19.9, 2 of 32 25.0 / 22.7; 16-bit
    // logits with few to keep wait for the barrier: 16 of eight over 128256 19.9 / 20.7, bfloat16 20.5 / 21.7, 64 of four over 32000 12.5 / 13.0 and 13.0 / 13.8.)
    maxima[threadIdx.x] = ordered(most);
    __syncthreads();
    uint32_t keys[SCAN_WAVES], largest = 0;
#pragma unroll
    for (int w = 0; w < SCAN_WAVES; ++w) {
        keys[w] = maxima[w * 64 + lane];
        largest = max(largest, keys[w]);
    }
    largest = __builtin_amdgcn_readfirstlane(ordered(wave_max(unordered(largest))));
    const float least = unordered(max(nth_largest(keys, largest, a.keep), ordered(-INFINITY)));
    int count = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const bool in = x[e] >= least;
        const uint64_t who = __ballot(in);
        if (who == 0) continue;
        const int at = count + lanes_below(who);
        if (in && at < SCAN_LIST) list[wave][at] = Kept{x[e], token_of(e)};
        count += __builtin_popcountll(who);
    }
    if (count > SCAN_LIST) { // many equal ones: the best one by one
        uint32_t last_key = 0xffffffffu; // everything up to here, and of equal ones up to last_token, is taken
        int last_token = -1;
        for (int r = 0; r < a.keep; ++r) {
            uint32_t bk = 0;
            int bt = INT32_MAX;
            float bx = -INFINITY;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t k = ordered(x[e]);
                const int t = token_of(e);
                const bool left = (full || t < a.V) && (k < last_key || (k == last_key && t > last_token));
                if (left && (k > bk || (k == bk && t < bt))) { bk = k; bt = t; bx = x[e]; }
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const uint32_t ok = __shfl_xor(bk, d);
                const int ot = __shfl_xor(bt, d);
                const float ox = __shfl_xor(bx, d);
                if (ok > bk || (ok == bk && ot < bt)) { bk = ok; bt = ot; bx = ox; }
            }
            if (lane == 0) list[wave][r] = Kept{bx, bt};
            last_key = bk;
            last_token = bt;
        }
        count = a.keep;
    }
    if (lane == 0) counts[wave] = count;
    __syncthreads();
    if (wave) return;
    const int64_t at = static_cast<int64_t>(row) * a.nc + blockIdx.x;
    float2 sum = sums[0];
    float bar = least;
#pragma unroll
    for (int w = 1; w < SCAN_WAVES; ++w) sum = add_sums(sum, sums[w]);
    if (lane == 0) a.part[at] = sum;
    constexpr int EACH = SCAN_LIST / 64;
    Kept mine[SCAN_WAVES * EACH];
    float best = -INFINITY;
    int n = 0;
#pragma unroll
    for (int i = 0; i < SCAN_WAVES * EACH; ++i) {
        const int w = i / EACH, at = lane + i % EACH * 64;
        mine[i] = at < counts[w] ? list[w][at] : Kept{__builtin_nanf(""), -1}; // (NaN reaches nothing)
        best = fmaxf(best, mine[i].x);
        n += __builtin_popcountll(__ballot(mine[i].x >= bar));
    }
    if (n > 64) {
        uint32_t t = ordered(bar);
        raise_threshold(t, n, __builtin_amdgcn_readfirstlane(ordered(wave_max(best))) + 1, a.keep, 64, [&](float v) {
            int k = 0;
#pragma unroll
            for (int i = 0; i < SCAN_WAVES * EACH; ++i) k += __builtin_popcountll(__ballot(mine[i].x >= v));
            return k;
        });
        bar = unordered(t);
    }
    n = 0;
#pragma unroll
    for (int i = 0; i < SCAN_WAVES * EACH; ++i) {
        const bool in = mine[i].x >= bar;
        const uint64_t who = __ballot(in);
        if (in) top[n + lanes_below(who)] = mine[i];
        n += __builtin_popcountll(who);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    Kept *const kept = a.kept + at * a.keep;
    if (n <= 64) {
        const Kept own = lane < n ? top[lane] : Kept{-INFINITY, -1};
        const uint32_t key = ordered(own.x);
        int rank = 0;
        for (int j = 0; j < n; ++j) {
            const uint32_t k = __builtin_amdgcn_readlane(key, j);
            const int t = __builtin_amdgcn_readlane(own.token, j);
            rank += k > key || (k == key && t < own.token);
        }
        if (lane < n && rank < a.keep) kept[rank] = own;
    } else
        for (int i = lane; i < n; i += 64) {
            const Kept own = top[i];
            const uint32_t key = ordered(own.x);
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += ordered(top[j].x) > key || (ordered(top[j].x) == key && top[j].token < own.token);
            if (rank < a.keep) kept[rank] = own;
        }
    if (lane >= n && lane < a.keep) kept[lane] = Kept{-INFINITY, -1}; // (n >= keep unless there are fewer tokens)
}

constexpr int PICK_THREADS = 1024, PICK_LIST = 1024, PICK_HELD = 8; // PICK_HELD: candidates a thread keeps in registers at most, if that is all of them

template <class L, int E, int HELD>
__global__ void __launch_bounds__(PICK_THREADS) beam_pick_kernel(BeamArgs a)
{
    typedef typename L::type T;
    __shared__ float lse[PRIMA_BEAM_MAX], own[PRIMA_BEAM_MAX], win_score[PRIMA_BEAM_MAX];
    __shared__ uint8_t ended[PRIMA_BEAM_MAX];
    __shared__ int win_at[PRIMA_BEAM_MAX];
    __shared__ uint32_t wave_t[PICK_THREADS / 64], wave_key[PICK_THREADS / 64], all_keys[PICK_THREADS];
    __shared__ __align__(16) float l_score[PICK_LIST + 4];
    __shared__ __align__(16) int l_at[PICK_LIST + 4];
    __shared__ int wave_at[PICK_THREADS / 64];
    __shared__ int count, suspect, again;
    const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int WAVES = PICK_THREADS / 64;
    const int lists = a.W * a.nc, total = lists * a.keep;
    if (threadIdx.x == 0) { count = 0; suspect = 0; again = 0; }
    const Kept *const kept = a.kept + static_cast<int64_t>(b) * total;
    const bool held = total <= HELD * PICK_THREADS;
    Kept mine[HELD];
    if (held) { // on their way while the sums are joined
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int at = threadIdx.x + i * PICK_THREADS;
            if (at < total) mine[i] = kept[at]; // (of a beam that has ended: whatever is there)
        }
    }
    for (int w = wave; w < a.W; w += WAVES) {
        const int row = b * a.W + w;
        const bool end = a.done && a.done[row];
        float2 v = make_float2(-INFINITY, 0.f);
        if (!end)
            for (int c = lane; c < a.nc; c += 64) v = add_sums(v, a.part[static_cast<int64_t>(row) * a.nc + c]);
        const float m = wave_max(v.x), s = wave_sum(m == -INFINITY ? v.y : v.y * __builtin_amdgcn_exp2f(v.x - m));
        if (lane == 0) {
            // m ln 2 + ln s, rounded once; NaN: the beam has no scores
            lse[w] = m == -INFINITY ? __builtin_nanf("") : static_cast<float>(static_cast<double>(m) * 0.693147180559945309417 + static_cast<double>(logf(s)));
            own[w] = a.scores[row];
            ended[w] = end;
        }
    }
    __syncthreads();
    // the score of a logit, of an element `at` of the kept ones; NaN is -infinity, as is what a beam that has ended left behind
    auto score_of = [&](int w, float x) {
        const float v = own[w] + (x - lse[w]) + 0.f; // (+ 0: no negative zero)
        return v == v ? v : -INFINITY;
    };
    // candidate `at`, which is k of beam w: score and w * V + token (-1: none).  The first candidate of a beam that has ended is its eos.
    auto candidate_of = [&](int at, int w, Kept k, float &score) {
        score = -INFINITY;
        if (ended[w]) {
            if (at != w * a.nc * a.keep) return -1;
            score = own[w] == own[w] ? own[w] + 0.f : -INFINITY;
            return w * a.V + a.eos;
        }
        if (k.token < 0) return -1;
        score = score_of(w, k.x);
        return w * a.V + k.token;
    };
    auto candidate = [&](int at, float &score) { return candidate_of(at, at / (a.nc * a.keep), kept[at], score); };
    const unsigned inverse = 0xffffffffu / static_cast<unsigned>(a.nc * a.keep) + 1; // (at nc keep < 2^32: the high word of the product is the quotient)
    float most = -INFINITY, held_score[HELD];
    int held_flat[HELD];
    if (held) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int at = threadIdx.x + i * PICK_THREADS;
            held_flat[i] = -1;
            if (at < total) held_flat[i] = candidate_of(at, static_cast<int>(__umulhi(at, inverse)), mine[i], held_score[i]);
            if (held_flat[i] >= 0) most = fmaxf(most, held_score[i]);
        }
    } else
        for (int at = threadIdx.x; at < total; at += PICK_THREADS) {
            float s;
            if (candidate(at, s) >= 0) most = fmaxf(most, s);
        }
    // Of few candidates the best of the waves' thresholds will do; else the maxima of all threads are one set, whose threshold far fewer reach.  (us, waves / all: eight
    // beams' 4536 candidates, eight chosen, 14.4 / 12.1; 16 beams' 4080, 16 chosen, 21.4 / 15.4; 825 16.9 / 15.6; 288 13.6 / 14.3; 72 10.4 / 11.9)
    uint32_t tk = ordered(-INFINITY);
    if (total <= 512) {
        const uint32_t key[1] = {ordered(most)}, t = nth_largest(key, ordered(wave_max(most)), a.n_best);
        if (lane == 0) wave_t[wave] = t;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) tk = max(tk, wave_t[w]);
    } else {
        all_keys[threadIdx.x] = ordered(most);
        __syncthreads();
        if (wave == 0) {
            uint32_t key[WAVES], largest = 0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                key[i] = all_keys[i * 64 + lane];
                largest = max(largest, key[i]);
            }
            const uint32_t t = nth_largest(key, ordered(wave_max(unordered(largest))), a.n_best);
            if (lane == 0) wave_t[0] = t;
        }
        __syncthreads();
        tk = max(tk, wave_t[0]);
    }
    const float least = unordered(tk);
    auto collect = [&](int at, int flat, float s) {
        if (flat < 0 || !(s >= least)) return;
        const int n = atomicAdd(&count, 1);
        if (n < PICK_LIST) { l_score[n] = s; l_at[n] = flat; }
        if (at % a.keep == a.keep - 1) suspect = 1; // a list all of whose elements reach the threshold
    };
    if (held) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) collect(threadIdx.x + i * PICK_THREADS, held_flat[i], held_score[i]);
    } else
        for (int at = threadIdx.x; at < total; at += PICK_THREADS) {
            float s;
            const int flat = candidate(at, s);
            collect(at, flat, s);
        }
    __syncthreads();
    const int n = count;
    if (n <= PICK_LIST) {
        if (threadIdx.x < 4) { l_score[n + threadIdx.x] = -INFINITY; l_at[n + threadIdx.x] = INT32_MAX; } // (nothing ranks behind these: read four at a time)
        __syncthreads();
        // (the order in which the list was filled does not matter: every element finds its own rank)
        for (int i = threadIdx.x; i < n; i += PICK_THREADS) {
            const float s = l_score[i];
            const int at = l_at[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; j += 4) {
                const float4 sj = *reinterpret_cast<const float4 *>(l_score + j);
                const int4 aj = *reinterpret_cast<const int4 *>(l_at + j);
                rank += (sj.x > s || (sj.x == s && aj.x < at)) + (sj.y > s || (sj.y == s && aj.y < at)) + (sj.z > s || (sj.z == s && aj.z < at)) +
                        (sj.w > s || (sj.w == s && aj.w < at));
            }
            if (rank < a.n_best) { win_score[rank] = s; win_at[rank] = at; }
        }
        for (int r = n + threadIdx.x; r < a.n_best; r += PICK_THREADS) { win_score[r] = -INFINITY; win_at[r] = -1; }
    } else {
        uint32_t last_key = 0xffffffffu;
        int last_at = -1;
        for (int r = 0; r < a.n_best; ++r) {
            uint32_t bk = 0;
            int bt = INT32_MAX;
            for (int at = threadIdx.x; at < total; at += PICK_THREADS) {
                float s;
                const int flat = candidate(at, s);
                if (flat < 0) continue;
                const uint32_t k = ordered(s);
                if ((k < last_key || (k == last_key && flat > last_at)) && (k > bk || (k == bk && flat < bt))) { bk = k; bt = flat; }
            }
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const uint32_t ok = __shfl_xor(bk, d);
                const int ot = __shfl_xor(bt, d);
                if (ok > bk || (ok == bk && ot < bt)) { bk = ok; bt = ot; }
            }
            if (lane == 0) { wave_key[wave] = bk; wave_at[wave] = bt; }
            __syncthreads();
            for (int w = 0; w < WAVES; ++w)
                if (wave_key[w] > bk || (wave_key[w] == bk && wave_at[w] < bt)) { bk = wave_key[w]; bt = wave_at[w]; }
            __syncthreads();
            if (threadIdx.x == 0) {
                win_score[r] = bt == INT32_MAX ? -INFINITY : unordered(bk);
                win_at[r] = bt == INT32_MAX ? -1 : bt;
            }
            last_key = bk;
            last_at = bt;
        }
    }
    __syncthreads();
    if (suspect && win_at[a.n_best - 1] >= 0) {
        const float tie = win_score[a.n_best - 1];
        // (list c of beam w may have left out elements of this score)
        auto left_out = [&](int list) {
            if (ended[list / a.nc]) return false;
            const Kept k = kept[static_cast<int64_t>(list) * a.keep + a.keep - 1];
            return k.token >= 0 && score_of(list / a.nc, k.x) >= tie;
        };
        for (int list = threadIdx.x; list < lists; list += PICK_THREADS)
            if (left_out(list)) again = 1;
        __syncthreads();
        if (again) {
            int first = 0;
            while (win_score[first] > tie) ++first;
            int last = -1;
            for (int r = first; r < a.n_best; ++r) { // the lowest index of this score behind the last
                int best = INT32_MAX;
                for (int at = threadIdx.x; at < total; at += PICK_THREADS) {
                    float s;
                    const int flat = candidate(at, s);
                    if (flat > last && s == tie) best = min(best, flat);
                }
                for (int list = wave; list < lists; list += WAVES) {
                    if (!left_out(list)) continue;
                    const int w = list / a.nc, start = (list - w * a.nc) * 64 * SCAN_WAVES * E, end = min(start + 64 * SCAN_WAVES * E, a.V);
                    const T *p = static_cast<const T *>(a.logits) + (static_cast<int64_t>(b) * a.W + w) * a.ld;
                    for (int v = start + lane; v < end; v += 64)
                        if (w * a.V + v > last && score_of(w, L::one(p + v)) == tie) best = min(best, w * a.V + v);
                }
#pragma unroll
                for (int d = 32; d; d >>= 1) best = min(best, __shfl_xor(best, d));
                if (lane == 0) wave_at[wave] = best;
                __syncthreads();
                for (int w = 0; w < WAVES; ++w) best = min(best, wave_at[w]);
                __syncthreads();
                if (threadIdx.x == 0) win_at[r] = best;
                last = best;
            }
            __syncthreads();
        }
    }
    if (threadIdx.x < a.n_best) {
        const int at = win_at[threadIdx.x], w = at < 0 ? -1 : at / a.V;
        const int64_t o = static_cast<int64_t>(b) * a.n_best + threadIdx.x;
        a.out_scores[o] = win_score[threadIdx.x];
        a.out_beams[o] = w;
        a.out_tokens[o] = at < 0 ? -1 : at - w * a.V;
    }
}

static int beam_keep(int n_best) { return n_best < PRIMA_BEAM_MAX ? n_best + 1 : n_best; }
// Logits a lane takes.  32, or
//  8 where that leaves fewer than two workgroups a compute unit (one search of four beams over 32000 tokens: 16 or 64 workgroups), unless the lists, four times as many, are
//    then more than the second launch holds in registers;
//  16 of 16-bit logits, which come in half the time, so that loads of some waves run beside the exponentials of others, as long as the lists are few (us of both launches, 32 / 16: 16
//    searches of eight beams over 128256 binary16 logits 22.7 / 20.7, bfloat16 23.1 / 21.7, 64 of four over 32000 14.0 / 13.0 and 14.8 / 13.8, but 24 of four over 151936 15.8 / 16.8 and
//    16.2 / 16.9; before there was one threshold a workgroup: fp32 21.3 and 21.6; 4 searches of 16 beams over 151936, 10336 candidates each, 19.5 -> 26.7).
static int beam_lane_logits(int dtype, int n_seqs, int n_beams, int64_t vocab, int n_best)
{
    auto candidates = [&](int E) { return n_beams * ((vocab + 64 * SCAN_WAVES * E - 1) / (64 * SCAN_WAVES * E)) * beam_keep(n_best); };
    if (static_cast<int64_t>(n_seqs) * n_beams * ((vocab + 8191) / 8192) < 512 && candidates(8) <= PICK_HELD * PICK_THREADS) return 8;
    return dtype != PRIMA_DT_F32 && candidates(16) <= PICK_HELD / 2 * PICK_THREADS ? 16 : 32;
}
static int64_t beam_row_lists(int dtype, int n_seqs, int n_beams, int64_t vocab, int n_best) // workgroups a row
{
    const int64_t each = 64 * SCAN_WAVES * beam_lane_logits(dtype, n_seqs, n_beams, vocab, n_best);
    return (vocab + each - 1) / each;
}
static size_t beam_bytes(int64_t rows, int64_t lists, int n_best) // lists: of a row
{
    return round_up(rows * lists * sizeof(float2), 256) + round_up(rows * lists * beam_keep(n_best) * sizeof(Kept), 256);
}

static bool beam_shape_ok(int n_seqs, int n_beams, int64_t vocab, int n_best)
{
    return n_seqs >= 1 && n_beams >= 1 && n_beams <= PRIMA_BEAM_MAX && n_best >= 1 && n_best <= PRIMA_BEAM_MAX && vocab >= 1 && vocab < INT32_MAX - 65536 &&
           n_beams * vocab < INT32_MAX && n_best <= n_beams * vocab && static_cast<int64_t>(n_seqs) * n_beams <= 65535;
}

template <class L, int E>
static void launch_beam_select(const BeamArgs &a, hipStream_t st)
{
    const dim3 grid(a.nc, a.B * a.W);
    if (a.keep <= SCAN_FEW) hipLaunchKernelGGL((beam_scan_kernel<L, E, 64>), grid, dim3(64 * SCAN_WAVES), 0, st, a);
    else hipLaunchKernelGGL((beam_scan_kernel<L, E, 128>), grid, dim3(64 * SCAN_WAVES), 0, st, a);
    // (numbers held: four a thread are a little faster than eight where they do)
    if (static_cast<int64_t>(a.W) * a.nc * a.keep <= PICK_HELD / 2 * PICK_THREADS) hipLaunchKernelGGL((beam_pick_kernel<L, E, PICK_HELD / 2>), dim3(a.B), dim3(PICK_THREADS), 0, st, a);
    else hipLaunchKernelGGL((beam_pick_kernel<L, E, PICK_HELD>), dim3(a.B), dim3(PICK_THREADS), 0, st, a);
}
template <class L>
static void launch_beam_select(const BeamArgs &a, int E, hipStream_t st) // (16: of 16-bit logits)
{
    if (E == 32) launch_beam_select<L, 32>(a, st);
    else if (L::N == 8 && E == 16) launch_beam_select<L, L::N == 8 ? 16 : 8>(a, st);
    else launch_beam_select<L, 8>(a, st);
}

} // namespace prima

using namespace prima;

extern "C" {

size_t prima_beam_select_workspace_bytes(int32_t n_seqs, int32_t n_beams, int64_t vocab, int32_t n_best)
{
    if (!beam_shape_ok(n_seqs, n_beams, vocab, n_best)) return 0;
    const int64_t rows = static_cast<int64_t>(n_seqs) * n_beams;
    const size_t wide = beam_bytes(rows, beam_row_lists(PRIMA_DT_F32, n_seqs, n_beams, vocab, n_best), n_best);
    const size_t narrow = beam_bytes(rows, beam_row_lists(PRIMA_DT_F16, n_seqs, n_beams, vocab, n_best), n_best);
    return wide > narrow ? wide : narrow; // (whatever the logits' type)
}

prima_status prima_beam_select(int32_t dtype, const void *logits, int64_t ld, int32_t n_seqs, int32_t n_beams, int64_t vocab, const float *scores,
                               const uint8_t *done, int32_t eos, int32_t n_best, float *out_scores, int32_t *out_beams, int32_t *out_tokens,
                               void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!logits || !scores || !out_scores || !out_beams || !out_tokens || !workspace) return PRIMA_E_NULL;
    if (dtype != PRIMA_DT_F32 && dtype != PRIMA_DT_F16 && dtype != PRIMA_DT_BF16) return PRIMA_E_SHAPE;
    if (!beam_shape_ok(n_seqs, n_beams, vocab, n_best) || ld < vocab) return PRIMA_E_SHAPE;
    if (done && (eos < 0 || eos >= vocab)) return PRIMA_E_RANGE;
    if (!aligned(logits, dtype == PRIMA_DT_F32 ? 4 : 2) || !aligned(scores, 4) || !aligned(out_scores, 4) || !aligned(out_beams, 4) || !aligned(out_tokens, 4) ||
        !aligned(workspace, 256))
        return PRIMA_E_ALIGN;
    if (workspace_bytes < prima_beam_select_workspace_bytes(n_seqs, n_beams, vocab, n_best)) return PRIMA_E_WORKSPACE;
    const int64_t rows = static_cast<int64_t>(n_seqs) * n_beams;
    const int E = beam_lane_logits(dtype, n_seqs, n_beams, vocab, n_best);
    BeamArgs a{};
    a.logits = logits; a.ld = ld; a.B = n_seqs; a.W = n_beams; a.V = static_cast<int>(vocab);
    a.n_best = n_best; a.keep = beam_keep(n_best); a.nc = static_cast<int>(beam_row_lists(dtype, n_seqs, n_beams, vocab, n_best)); a.eos = eos;
    a.scores = scores; a.done = done; a.out_scores = out_scores; a.out_beams = out_beams; a.out_tokens = out_tokens;
    a.part = static_cast<float2 *>(workspace);
    a.kept = reinterpret_cast<Kept *>(static_cast<char *>(workspace) + round_up(rows * a.nc * sizeof(float2), 256));
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == PRIMA_DT_F32) launch_beam_select<LogitF32>(a, E, st);
    else if (dtype == PRIMA_DT_F16) launch_beam_select<LogitF16>(a, E, st);
    else launch_beam_select<LogitBF16>(a, E, st);
    return last_launch_status();
}

} // extern "C"
