// Selection of a beam search's next beams (nkv_beam_select): of every prompt's B * V candidates scores[b] + x - log sum exp x the n_out largest.
//
// Every logit is read once, for one exponential and one comparison: bound by memory.  A workgroup keeps a stretch of one beam's row in registers
// (beam_scan_kernel) and leaves its maximum, its sum of exponentials and its n_out largest logits; a workgroup for a prompt joins them
// (beam_join_kernel): the sums in 64 bits, the candidates by their value in 64 bits.
//
// us, scan and join (reading the logits alone): one prompt of 4 beams of 32768 fp32 logits 5.0 + 4.3 (0.1), 16 of 8 of 131072 bf16 13.0 + 6.3 (4.8), 5 of 5 of 50021 fp16 6.1 + 6.2 (0.4).
// The small ones are what a launch takes with a few trips to memory one after the other; in the large one a compute unit's eight workgroups load at once, then bound, gather and count at
// once, in some 8 us that no load hides.
//
// Within a beam the order of the candidates is that of the logits, so no sum is needed to drop nearly all of them.  The threads' largest logits are dealt out to the W
// wavefronts; the least of their n_out / W-th largest is a bound that n_out of the logits reach at least, and few more: those are gathered, and each counts those before
// it.  Where too many reach it (equal ones, or large ones side by side in a few threads) lists are sorted and joined instead.  Lists are 64 keys, one a lane, sorted and joined by
// bitonic steps between lanes (21 steps to sort, 7 to join two).  A key holds the logit and, of equal ones, the lower token as the larger key, so that
// no two are alike and the answer does not depend on the order of anything.
#include "nkv_device.h"

#include <algorithm>
#include <type_traits>

namespace nkv {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave, kJoin = 1024, kJoinWaves = kJoin / kWave;
constexpr int kGather = 512, kGatherJoin = 1024;   // candidates that are counted one against the other, of a stretch and of a prompt
constexpr float kLog2e = 1.4426950408889634f;

// Partial result of a stretch, in front of its n_out keys.
struct Head {
    float top, sum;                      // sum of exp(x - top), or of exp(x) where all of them are -inf
};

// the word of the lane whose number differs in the bits M, a power of two
template <int M> __device__ __forceinline__ uint32_t lane_xor(uint32_t v)
{
    if constexpr (M == 1) return dpp_word<0xB1>(v);                        // quad_perm [1,0,3,2]
    else if constexpr (M == 2) return dpp_word<0x4E>(v);                   // quad_perm [2,3,0,1]
    else if constexpr (M == 4) return dpp_word<0x1B>(dpp_word<0x141>(v));  // 7 by row_half_mirror, and 3 by quad_perm [3,2,1,0]
    else if constexpr (M == 8) return dpp_word<0x128>(v);                  // row_ror:8
    else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (threadIdx.x & 16) ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (threadIdx.x & 32) ? r[0] : r[1];
    }
}
// lane 63 - i's
__device__ __forceinline__ uint32_t lane_mirror(uint32_t v) { return lane_xor<32>(lane_xor<16>(dpp_word<0x140>(v))); }

// A logit of a beam: its order and, inverted, its token.  Zero: none.
struct Key {
    uint32_t value, token;
    __device__ __forceinline__ bool operator>(const Key &o) const { return ((uint64_t)value << 32 | token) > ((uint64_t)o.value << 32 | o.token); }
    template <typename F> __device__ __forceinline__ Key moved(F f) const { return {f(value), f(token)}; }
    __device__ static Key none() { return {0u, 0u}; }
};
// A candidate of a prompt: the order of its value in 64 bits and, inverted, beam * V + token.
struct Candidate {
    uint32_t hi, lo, at;
    __device__ __forceinline__ uint64_t value() const { return (uint64_t)hi << 32 | lo; }
    __device__ __forceinline__ bool operator>(const Candidate &o) const { return value() > o.value() || (value() == o.value() && at > o.at); }
    template <typename F> __device__ __forceinline__ Candidate moved(F f) const { return {f(hi), f(lo), f(at)}; }
    __device__ static Candidate none() { return {0u, 0u, 0u}; }
};

template <int J, typename K> __device__ __forceinline__ K step(const K &a, bool larger)
{
    const K b = a.moved([](uint32_t v) { return lane_xor<J>(v); });
    return (b > a) == larger ? b : a;                                      // (equal ones are the same)
}
// the 64 lanes' keys, largest first, where every stretch of 2 J is bitonic
template <int J, typename K> __device__ __forceinline__ K ordered(K a, bool descending)
{
    const int lane = threadIdx.x & (kWave - 1);
    a = step<J>(a, ((lane & J) == 0) == descending);
    if constexpr (J > 1) return ordered<J / 2>(a, descending);
    else return a;
}
template <typename K> __device__ __forceinline__ K sorted(K a)
{
    const int lane = threadIdx.x & (kWave - 1);
    a = ordered<1>(a, (lane & 2) == 0);
    a = ordered<2>(a, (lane & 4) == 0);
    a = ordered<4>(a, (lane & 8) == 0);
    a = ordered<8>(a, (lane & 16) == 0);
    a = ordered<16>(a, (lane & 32) == 0);
    return ordered<32>(a, true);
}
// the 64 largest of two lists that are largest first
template <typename K> __device__ __forceinline__ K joined(const K &a, const K &b)
{
    const K c = b.moved([](uint32_t v) { return lane_mirror(v); });
    return ordered<32>(c > a ? c : a, true);
}
template <typename K> __device__ __forceinline__ K of_lane(const K &a, int lane)
{
    return a.moved([lane](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); });
}

__device__ __forceinline__ int sum_of_8(int x)                            // over lanes 8 i .. 8 i + 7, all of them active
{
    x += dpp_partner<0xB1>(x);                                             // quad_perm [1,0,3,2]
    x += dpp_partner<0x4E>(x);                                             // quad_perm [2,3,0,1]
    return x + dpp_partner<0x141>(x);                                      // row_half_mirror: the other quad
}

// The largest number that n of the 64 lanes' reach, bit by bit from the first in which they differ.  (Where a few more than n reach it a bit earlier that will do.)
__device__ __forceinline__ uint32_t reached(uint32_t x, int n)
{
    const uint32_t top = wave_reduce(x, [](uint32_t a, uint32_t b) { return max(a, b); }), least = wave_reduce(x, [](uint32_t a, uint32_t b) { return min(a, b); });
    uint32_t bound = least;
    if (top != least) {
        int bit = 31 - __builtin_clz(top ^ least);
        bound = top & ~((2u << bit) - 1u);                                 // (2 << 31 is 0: nothing in common)
        for (; bit >= 0; --bit) {
            const uint32_t trial = bound | 1u << bit;
            const int reach = __popcll(__ballot(x >= trial));
            if (reach >= n) bound = trial;
            if (reach >= n && reach <= n + n / 4) break;
        }
    }
    return bound;
}

// A bound that n of a workgroup's numbers reach at least, and few more, with its barriers (what was written to LDS before it is there afterwards).  For few: the largest of the
// wavefronts' n-th largest.  For more: the numbers are dealt out anew, so that all wavefronts have their share of any stretch of large ones, and the least of the
// n / W-th largest is taken; tighter, and some 1 us more.
template <int W> __device__ __forceinline__ uint32_t bound_of(uint32_t x, int n, uint32_t *dealt, uint32_t *bounds)
{
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
    const bool few = n < 12;
    if (!few) {
        dealt[tid] = x;
        __syncthreads();
        x = dealt[lane * W + ((w + lane) & (W - 1))];
        n = (n + W - 1) / W;
    }
    const uint32_t mine = reached(x, n);
    if (lane == 0) bounds[w] = mine;
    __syncthreads();
    uint32_t bound = bounds[0];
#pragma unroll
    for (int i = 1; i < W; ++i) bound = few ? max(bound, bounds[i]) : min(bound, bounds[i]);
    return bound;
}

template <typename T> struct Logits;
template <> struct Logits<float> { static constexpr int kWords = 8; };
template <> struct Logits<f16_t> { static constexpr int kWords = 4; };
template <> struct Logits<uint16_t> { static constexpr int kWords = 4; };   // bf16

template <typename T> __device__ __forceinline__ float logit(const uint32_t *w, int i)
{
    if constexpr (std::is_same_v<T, float>) return __uint_as_float(w[i]);
    else if constexpr (std::is_same_v<T, f16_t>) return (float)__builtin_bit_cast(_Float16, (uint16_t)(i % 2 ? w[i / 2] >> 16 : w[i / 2]));
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}

// logit e of a lane's, chosen among its registers
template <typename T, int VECS> __device__ __forceinline__ float logit_at(const uint32_t (&w)[VECS][Logits<T>::kWords], int e)
{
    constexpr int N = VECS * Logits<T>::kWords;
    constexpr bool kHalf = !std::is_same_v<T, float>;
    uint32_t x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = w[i / Logits<T>::kWords][i % Logits<T>::kWords];
    int at = kHalf ? e / 2 : e;
#pragma unroll
    for (int n = N / 2; n > 0; n /= 2) {
        const uint32_t upper = 0u - (uint32_t)(at & 1);                    // (a choice by bits: one by condition becomes an address in memory)
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = (x[2 * i + 1] & upper) | (x[2 * i] & ~upper);
        at >>= 1;
    }
    if constexpr (kHalf) x[0] = e % 2 ? x[0] >> 16 : x[0] & 0xffffu;
    return logit<T>(x, 0);
}

struct ScanArgs {
    const void *logits;
    int64_t prompt, beam;                // strides
    int32_t B, V, n_out, stretches;
    Head *heads;                         // [row][stretch]
    Key *keys;                           // [row][stretch][n_out]
};

// grid: rows * stretches.  E logits a thread, eight side by side, or, where a stretch (the row's last one, or its only one) has no more than eight for every thread, a workgroup's
// width apart, so that as many threads have one as can.  Which thread has which does not depend on where a row begins, so that equal rows have equal sums.
template <typename T, int E> __global__ __launch_bounds__(kThreads) void beam_scan_kernel(const ScanArgs a)
{
    using L = Logits<T>;
    using Words = unsigned int __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    constexpr int kVecs = E / 8;
    __shared__ Key buffer[kWaves][2 * kWave];
    __shared__ uint64_t gathered[kGather];
    __shared__ Head heads[kWaves];
    __shared__ uint32_t best[kThreads], bounds[kWaves];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid / kWave), n_out = a.n_out;
    const int row = blockIdx.x / a.stretches, stretch = blockIdx.x - row * a.stretches;
    const int p = row / a.B, b = row - p * a.B;
    const T *x = (const T *)a.logits + p * a.prompt + b * a.beam;
    const int first = stretch * (kThreads * E);                         // (V is under 2^31 - kThreads * 32)
    const bool spread = a.V - first <= kThreads * 8;
    uint32_t raw[kVecs][L::kWords];
    // logits at, at + apart, ..: what is behind the row's end counts as -inf
    auto one_by_one = [&](uint32_t (&to)[L::kWords], int at, int apart) {
#pragma unroll
        for (int i = 0; i < L::kWords; ++i) {
            if constexpr (std::is_same_v<T, float>) to[i] = at + i * apart < a.V ? reinterpret_cast<const uint32_t *>(x)[at + i * apart] : 0xff800000u;
            else {
                constexpr uint32_t none = std::is_same_v<T, f16_t> ? 0xfc00u : 0xff80u;
                const uint16_t *h = reinterpret_cast<const uint16_t *>(x);
                const int lo_at = at + 2 * i * apart, hi_at = lo_at + apart;
                const uint32_t lo = lo_at < a.V ? h[lo_at] : none, hi = hi_at < a.V ? h[hi_at] : none;
                to[i] = lo | hi << 16;
            }
        }
    };
    if (spread) {
        one_by_one(raw[0], first + tid, kThreads);
#pragma unroll
        for (int j = 1; j < kVecs; ++j)
#pragma unroll
            for (int i = 0; i < L::kWords; ++i) raw[j][i] = std::is_same_v<T, float> ? 0xff800000u : std::is_same_v<T, f16_t> ? 0xfc00fc00u : 0xff80ff80u;
    } else {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int at = first + (j * kThreads + tid) * 8;
            if (at + 8 <= a.V) {
#pragma unroll
                for (int i = 0; i < L::kWords; i += 4) {
                    const Words v = __builtin_nontemporal_load(reinterpret_cast<const Words *>(x + at) + i / 4);
                    raw[j][i] = v.x, raw[j][i + 1] = v.y, raw[j][i + 2] = v.z, raw[j][i + 3] = v.w;
                }
            } else {
                one_by_one(raw[j], at, 1);
            }
        }
    }
    float mine = -INFINITY;
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) mine = fmaxf(mine, logit<T>(raw[j], i));
    const float top = wave_max(mine), base = top == -INFINITY ? 0.f : top;
    // 2^(x L - c) with c = base L as rounded is off by 2^(base L - c), whose exponent one more fma gives exactly: one operation a logit in front of the exponential.
    // Far from zero, where that is more than a fraction, the distance is taken first.
    float sum = 0.f;
    auto add = [&](auto exponent) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += __builtin_amdgcn_exp2f(exponent(logit<T>(raw[j], i)));
            sum += s;
        }
    };
    if (fabsf(base) < 0x1p20f) {
        const float c = base * kLog2e, rest = fmaf(base, kLog2e, -c);
        add([c](float x) { return fmaf(x, kLog2e, -c); });
        sum *= __builtin_amdgcn_exp2f(-rest);
    } else {
        add([base](float x) { return (x - base) * kLog2e; });
    }
    sum = wave_sum(sum);
    if (lane == 0) heads[w] = Head{top, sum};
    if (tid == 0) count = 0;
    const uint32_t bound = bound_of<kWaves>(ord_key(mine), n_out, best, bounds);
    const int64_t part = blockIdx.x;
    if (tid == 0) {
        float m = -INFINITY, s = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) m = fmaxf(m, heads[i].top);
#pragma unroll
        for (int i = 0; i < kWaves; ++i) s += heads[i].top == -INFINITY ? heads[i].sum : heads[i].sum * __builtin_amdgcn_exp2f((heads[i].top - m) * kLog2e);
        a.heads[part] = Head{m, s};
    }
    const float from = key_value(max(bound, ord_key(-3.402823466e38f)));   // -inf and NaN are no candidates
    uint32_t takes = 0u;                                                   // bit 8 j + i: the lane's logit i of vector j
    if (__any(mine >= from)) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) takes |= logit<T>(raw[j], i) >= from ? 1u << (8 * j + i) : 0u;
    }
    auto key_of = [&](int e) {
        return Key{ord_key(logit_at<T, kVecs>(raw, e)), ~(uint32_t)(first + (spread ? e * kThreads + tid : (e / 8 * kThreads + tid) * 8 + e % 8))};
    };
    for (uint32_t left = takes; left != 0u; left &= left - 1u) {
        const Key k = key_of(__builtin_ctz(left));
        const int at = atomicAdd(&count, 1);
        if (at < kGather) gathered[at] = (uint64_t)k.value << 32 | k.token;
    }
    __syncthreads();
    const int found = __builtin_amdgcn_readfirstlane(count);
    if (found <= kGather) {
        for (int i = tid / 8; i < found; i += kThreads / 8) {              // eight threads a candidate
            const uint64_t key = gathered[i];
            int before = 0;
#pragma unroll 8
            for (int k = tid % 8; k < found; k += 8) before += gathered[k] > key ? 1 : 0;
            before = sum_of_8(before);
            if (tid % 8 == 0 && before < n_out) a.keys[part * n_out + before] = Key{(uint32_t)(key >> 32), (uint32_t)key};
        }
        if (tid >= found && tid < n_out) a.keys[part * n_out + tid] = Key::none();
        return;
    }
    // Too many that are equal, or side by side in few lanes: the lanes' one after the other, 64 at a time.
    Key list = Key::none(), least = Key::none();
    int held = 0;
    Key *mine_b = buffer[w];
    auto flush = [&](int count) {                                          // the first `count` of the buffer
        __builtin_amdgcn_wave_barrier();
        const Key k = lane < count ? mine_b[lane] : Key::none();
        list = joined(list, sorted(k));
        least = of_lane(list, n_out - 1);
    };
    do {                                                                   // one of every lane's at a time; fewer than 64 are held
        const bool left = takes != 0u;
        const int e = left ? __builtin_ctz(takes) : 0;
        takes &= takes - 1u;
        const Key k = key_of(e);
        const bool counts = left && k > least;
        const unsigned long long mask = __ballot(counts);
        if (counts) mine_b[held + __popcll(mask & ((1ull << lane) - 1ull))] = k;
        held += __popcll(mask);
        if (held >= kWave) {
            flush(kWave);
            held -= kWave;
            const Key rest = mine_b[kWave + lane];
            __builtin_amdgcn_wave_barrier();
            mine_b[lane] = rest;
        }
        __builtin_amdgcn_wave_barrier();
    } while (__any(takes != 0u));
    if (held > 0) flush(held);
    __builtin_amdgcn_wave_barrier();
    mine_b[lane] = list;
    __syncthreads();
    if (w > 0) return;
    static_assert(kWaves == 4, "two steps");
    list = joined(joined(list, buffer[1][lane]), joined(buffer[2][lane], buffer[3][lane]));
    if (lane < n_out) a.keys[part * n_out + lane] = list;
}

__device__ __forceinline__ uint64_t ord64(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x == 0.0 ? 0.0 : x);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double value64(uint64_t k) { return __builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k); }

// grid: a workgroup a prompt.  Nearly all of its time is waiting, so it does little in a row: all candidates (of many lists: the first ones) at once to a bound, and those
// that reach it one against the other.  (Lists joined in the wavefronts and then in a tree: 8, 12 and 12 us for one prompt of 4 beams and 64 lists of 8, 16 of 8 and 128 lists of 16, 5 of 5 and 125
// lists of 10.)
constexpr int kHold = 8;
// MANY: more candidates than the threads hold, of which more are left after the first bound: 6 prompts of 32 beams and 11 lists of 64, 15.3 us.  (In one kernel for both 0.3 us more for few.)
template <bool MANY> __global__ __launch_bounds__(kJoin) void beam_join_kernel(const Head *__restrict__ heads, const Key *__restrict__ keys, const float *scores, int B,
                                                         int V, int n_out, int stretches, float *out_scores, int32_t *__restrict__ out_beams,
                                                         int32_t *__restrict__ out_tokens)
{
    __shared__ union {
        Candidate lists[kJoinWaves][kWave];
        struct {
            uint64_t value[kGatherJoin];
            uint32_t at[kGatherJoin];
        } gathered;
    } lds;
    __shared__ double lses[NKV_MAX_BEAMS];
    __shared__ float score_of[NKV_MAX_BEAMS];
    __shared__ uint32_t all_best[kJoin], bounds[kJoinWaves];
    __shared__ int count, again;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid / kWave), p = blockIdx.x;
    const int parts = B * stretches, in_beam = stretches * n_out;
    const int64_t total = (int64_t)parts * n_out;
    keys += p * total;
    Key held[kHold];
#pragma unroll
    for (int k = 0; k < kHold; ++k) held[k] = !MANY && tid + kJoin * k < total ? keys[tid + kJoin * k] : Key::none();
    // log sum exp of every beam, NaN for a beam without candidates: where it is not finite, or the beam's score is not.  The stretches' sums are of 32 bits and so are their
    // factors; 64 bits where they are added up and for the logarithm, a thread a beam.  (Factors in 64 bits, and a wavefront a logarithm: 2 us more with 32 beams, 0.2 with a few.)
    for (int b = w; b < B; b += kJoinWaves) {
        const Head *h = heads + ((int64_t)p * B + b) * stretches;
        const Head first = lane < stretches ? h[lane] : Head{-INFINITY, 0.f};
        float m = first.top;
        for (int i = lane + kWave; i < stretches; i += kWave) m = fmaxf(m, h[i].top);
        m = wave_max(m);
        auto share = [m](const Head &x) { return x.top == -INFINITY ? (double)x.sum : (double)(x.sum * __builtin_amdgcn_exp2f((x.top - m) * kLog2e)); };
        double s = share(first);
        for (int i = lane + kWave; i < stretches; i += kWave) s += share(h[i]);
        s = wave_sum(s);
        if (lane == 0) lses[b] = s, score_of[b] = m;
    }
    __syncthreads();
    for (int b = tid; b < B; b += kJoin) {
        const double lse = (double)score_of[b] + log(lses[b]);
        const float score = scores[(int64_t)p * B + b];
        lses[b] = isfinite(lse) && isfinite(score) ? lse : (double)NAN, score_of[b] = score;
    }
    if (tid == 0) count = 0, again = 0;
    __syncthreads();
    auto candidate = [&](const Key &k, int b) {
        const double lse = lses[b];
        if (k.value == 0u || lse != lse) return Candidate::none();
        const uint64_t v = ord64((double)score_of[b] + ((double)key_value(k.value) - lse));
        return Candidate{(uint32_t)(v >> 32), (uint32_t)v, ~((uint32_t)b * (uint32_t)V + ~k.token)};
    };
    Candidate some[kHold];
    uint32_t best = 0u;
#pragma unroll
    for (int k = 0; k < kHold; ++k) {
        some[k] = Candidate::none();
        if (MANY || kJoin * k >= total) continue;
        some[k] = candidate(held[k], (int)min((uint32_t)(tid + kJoin * k) / (uint32_t)in_beam, (uint32_t)(B - 1)));
        best = max(best, some[k].hi);
    }
    auto best_at = [&](int r) {                                            // of the thread's lists' r-th candidates
        uint32_t b = 0u;
        for (int i = tid; i < parts; i += kJoin) b = max(b, candidate(keys[(int64_t)i * n_out + r], i / stretches).hi);
        return b;
    };
    if constexpr (MANY) best = best_at(0);
    uint32_t bound = max(bound_of<kJoinWaves>(best, n_out, all_best, bounds), 1u);   // (0: no candidate)
    // Of many lists a few may hold nearly all: n_out / r lists whose r-th candidates reach a number have n_out that do.
    if constexpr (MANY) {
        constexpr int kRank = 8;
        if (n_out >= kRank) {
            __syncthreads();
            bound = max(bound, bound_of<kJoinWaves>(best_at(kRank - 1), (n_out + kRank - 1) / kRank, all_best, bounds));
        }
    }
    auto gather_by = [&](const Candidate &c, int *n) {
        if (c.hi < bound) return false;
        const int at = atomicAdd(n, 1);
        if (at < kGatherJoin) lds.gathered.value[at] = c.value(), lds.gathered.at[at] = c.at;
        return true;
    };
    auto gather = [&](const Candidate &c) { return gather_by(c, &count); };
    if constexpr (!MANY) {
#pragma unroll
        for (int k = 0; k < kHold; ++k) gather(some[k]);
    } else {
        // eight threads a list, eight of its candidates at a time for as long as the last one reaches the bound
        for (int i = tid / 8; i < parts; i += kJoin / 8) {
            bool more = true;
            for (int r = tid % 8; more && r - tid % 8 < n_out; r += 8) {
                const bool in = gather(r < n_out ? candidate(keys[(int64_t)i * n_out + r], i / stretches) : Candidate::none());
                more = __ballot(in) >> (lane & 56) >> 7 & 1;
            }
        }
    }
    __syncthreads();
    int found = count;
    if (MANY && found > 2 * n_out + kWave && found <= kGatherJoin) {               // a thread each: a tighter bound, and fewer to count (400 of them 9 us, 200 of them 3)
        const Candidate c = tid < found ? Candidate{(uint32_t)(lds.gathered.value[tid] >> 32), (uint32_t)lds.gathered.value[tid], lds.gathered.at[tid]} : Candidate::none();
        bound = max(bound, bound_of<kJoinWaves>(c.hi, n_out, all_best, bounds));
        gather_by(c, &again);
        __syncthreads();
        found = again;
    }
    auto put = [&](int at, const Candidate &c) {
        const bool none = c.value() == 0ull;
        const uint32_t number = ~c.at;
        out_scores[(int64_t)p * n_out + at] = none ? -INFINITY : (float)value64(c.value());
        out_beams[(int64_t)p * n_out + at] = none ? -1 : (int32_t)(number / (uint32_t)V);
        out_tokens[(int64_t)p * n_out + at] = none ? -1 : (int32_t)(number % (uint32_t)V);
    };
    if (found <= kGatherJoin) {
        for (int i = tid / 8; i < found; i += kJoin / 8) {                 // eight threads a candidate
            const uint64_t value = lds.gathered.value[i];
            const uint32_t at = lds.gathered.at[i];
            int before = 0;
#pragma unroll 8
            for (int k = tid % 8; k < found; k += 8) {
                const uint64_t other = lds.gathered.value[k];
                const uint32_t other_at = lds.gathered.at[k];
                before += (other > value) | ((other == value) & (other_at > at)) ? 1 : 0;
            }
            before = sum_of_8(before);
            if (tid % 8 == 0 && before < n_out) put(before, Candidate{(uint32_t)(value >> 32), (uint32_t)value, at});
        }
        if (tid >= found && tid < n_out) put(tid, Candidate::none());
        return;
    }
    __syncthreads();
    Candidate list = Candidate::none();
#pragma unroll 1
    for (int i = w; i < parts; i += kJoinWaves) {
        const Candidate c = lane < n_out ? candidate(keys[(int64_t)i * n_out + lane], i / stretches) : Candidate::none();
        if (of_lane(c, 0) > of_lane(list, n_out - 1)) list = joined(list, c);
    }
    lds.lists[w][lane] = list;
#pragma unroll 1
    for (int half = kJoinWaves / 2; half > 0; half /= 2) {
        __syncthreads();
        if (w < half) {
            list = joined(list, lds.lists[w + half][lane]);
            lds.lists[w][lane] = list;
        }
    }
    if (tid < n_out) put(tid, list);
}

// Long stretches where there are enough of them to fill the chip: fewer lists to join.  (4 x 8 rows of 141945 fp32 logits, 576 of them: 16.0 us, with short
// ones 24.8.)
int logits_of_thread(const nkv_beams &s)
{
    return s.vocab > kThreads * 8 && (int64_t)s.n_prompts * s.n_beams * ((s.vocab + kThreads * 32 - 1) / (kThreads * 32)) >= 512 ? 32 : 8;
}
int stretches_of(const nkv_beams &s)
{
    const int at_once = kThreads * logits_of_thread(s);
    return (int)(((int64_t)s.vocab + at_once - 1) / at_once);
}
size_t up(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

bool beam_one_launch(const nkv_beams &s)
{
    // fewer than 2^32 threads: 1024 a prompt where its lists are joined, 256 a stretch
    const int64_t rows = (int64_t)s.n_prompts * s.n_beams;
    return s.n_prompts < (1 << 22) && rows < (1 << 24) && rows * stretches_of(s) < (1 << 24);
}

size_t beam_ws_bytes(const nkv_beams &s)
{
    const size_t parts = (size_t)s.n_prompts * s.n_beams * stretches_of(s);
    return up(parts * sizeof(Head)) + parts * s.n_out * sizeof(Key);
}

hipError_t launch_beam_select(const nkv_beams &s, float *out_scores, int32_t *out_beams, int32_t *out_tokens, void *ws, hipStream_t st)
{
    const size_t rows = (size_t)s.n_prompts * s.n_beams;
    const int stretches = stretches_of(s);
    Head *heads = (Head *)ws;
    Key *keys = (Key *)((char *)heads + up(rows * stretches * sizeof(Head)));
    const ScanArgs a{s.logits, s.strides[0], s.strides[1], s.n_beams, s.vocab, s.n_out, stretches, heads, keys};
    const unsigned grid = (unsigned)(rows * stretches);
    auto go = [&](auto type) {
        using T = decltype(type);
        (logits_of_thread(s) == 32 ? beam_scan_kernel<T, 32> : beam_scan_kernel<T, 8>)<<<grid, kThreads, 0, st>>>(a);
    };
    if (s.dtype == NKV_DTYPE_F32) go(float{});
    else if (s.dtype == NKV_DTYPE_F16) go(f16_t{});
    else go(uint16_t{});
    const bool many = (int64_t)s.n_beams * stretches * s.n_out > kJoin * kHold;
    (many ? beam_join_kernel<true> : beam_join_kernel<false>)<<<(unsigned)s.n_prompts, kJoin, 0, st>>>(heads, keys, s.scores, s.n_beams, s.vocab, s.n_out, stretches, out_scores, out_beams, out_tokens);
    return hipGetLastError();
}

}  // namespace nkv
