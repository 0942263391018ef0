// The likeliest tokens of each row, with the log-prob of a given one and the entropy: ulorl_token_topk.
//
// For x = z / T: lse = ln sum e^x, logp = x[y] - lse, H = ln S - (sum e^(x-m) (x-m)) / S with S = sum e^(x-m), and the K
// largest x with their ids.  One read of the logits is the bound, so the search for the K largest has to ride on the
// stream of the statistics and leave the vector ALUs (82 % used by the statistics alone at the rate of memory) their room:
//
//   1. The stream keeps, besides the sums, the largest logit of each group of neighbouring vectors (64 elements at large
//      vocabularies): the maximum of a vector is formed for the running maximum anyway, a group takes three lane
//      permutations more.  The groups' maxima stay in LDS (at most kMaxGroups).
//   2. A lower bound t of the K-th largest element: each wave finds the ceil(K / waves)-th largest of its lanes' largest
//      group maxima by bisection over ballots; t is the smallest of the waves' values, so at least K groups reach t.
//   3. Only groups that reach t (about 1.5 K of 2374) are read again, and their elements that reach t are collected: about as
//      many.  Each one's rank among them is its place in the answer.
//
// Ties: the order is by logit and then by the lower id, as one 64-bit key per element, so every rank is taken once.
// Where more groups or elements reach t than the lists hold (rows of equal logits, a vocabulary masked down to less than K
// tokens is not one), t is replaced by the K-th largest key itself, found by bisection over its 64 bits, first of the
// groups (of equal maxima those with the lowest ids: they hold the elements with the lowest ids), then of the elements of
// these K groups.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "logits_stream.hpp"
#include "ulorl.h"
#include "ulorl_internal.hpp"

using namespace ulorl_detail;

#pragma clang fp contract(off)

namespace {

constexpr int kTopkThreads = 256;
constexpr int kTopkWaves = kTopkThreads / 64;
constexpr int kTopkUnroll = 8;
constexpr int kMaxK = 128;
constexpr int kMaxGroups = 2560;      // group maxima of a row: 10 KB of LDS
constexpr int kGroupList = 512;
constexpr int kElemList = 768;
// Logits at or below -9e29 are masked (the filler of short vectors is one of them).  A lane's running maximum starts a little
// above: by so much that the terms of masked logits are 0 against it (the rounding of m scale is 1e23 there).
constexpr float kFloor = -8.99e29f;

struct TopkArgs {
    const int32_t* token_ids;   // may be NULL
    int32_t* top_ids;           // [N, K]
    float* top_logp;            // [N, K]
    float* logp;                // may be NULL
    float* entropy;
    float* lse;
    int64_t N, row_stride;
    int32_t V, K;
    int32_t lg;                 // log2 of the vectors in a group
    float scale;                // log2(e) / T
    double inv_t;
};

// Per-lane statistics of the stream; x = z scale in log2 units, relative to the lane's maximum.
// S + Sc: sum 2^(x - mL), its rounding residuals carried in Sc; T: sum 2^(x - mL) (x - mL).
struct Lane {
    float m, mL, S, Sc, T;
};

// The larger, not-a-number if one is (a row that holds one is refused at its end): one instruction for three values, and none to
// quiet what came out of bit operations, which fmaxf needs.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }

template <int COUNT>
__device__ __forceinline__ void absorb_scaled(const float* f, float cm, float scale, Lane& a)
{
    const float mn = larger(a.m, cm);
    const float mLn = mn * scale;
    const float d = a.mL - mLn;
    const float sc = fast_exp2(d);
    float T = sc * fmaf(d, a.S, a.T);
    const float S = sc * a.S, Sc = sc * a.Sc;
    // the terms as a tree over neighbours: a sum of eight is done before the next eight terms are formed
    float e[COUNT / 8 > 0 ? COUNT / 8 : 1];
#pragma unroll
    for (int c = 0; c < COUNT; c += 8) {
        constexpr int W = COUNT < 8 ? COUNT : 8;
        float p[W];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const float x = fmaf(f[c + k], scale, -mLn);
            p[k] = fast_exp2(x);
            T = fmaf(p[k], x, T);
        }
#pragma unroll
        for (int w = W / 2; w >= 1; w >>= 1)
#pragma unroll
            for (int k = 0; k < w; ++k) p[k] += p[k + w];
        e[c / 8] = p[0];
    }
#pragma unroll
    for (int w = COUNT / 16; w >= 1; w >>= 1)
#pragma unroll
        for (int k = 0; k < w; ++k) e[k] += e[k + w];
    const float t = S + e[0];                   // TwoSum: the residual of a small term against a sum near 1 is kept
    const float bv = t - S;
    a.Sc = Sc + ((S - (t - bv)) + (e[0] - bv));
    a.S = t;
    a.T = T;
    a.m = mn;
    a.mL = mLn;
}

// Absorbs U vectors and gives each one's largest element.
template <class Tr, int U>
__device__ __forceinline__ void absorb_vectors(const u32x4 (&v)[U], float scale, Lane& a, float (&vm)[U])
{
    constexpr int E = Tr::kPerVec;
    float f[U * E];
    float cm = kFloor;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        Tr::unpack(v[k], f + k * E);
        float m = f[k * E];
#pragma unroll
        for (int e = 1; e < E; ++e) m = larger(m, f[k * E + e]);
        vm[k] = m;
        cm = larger(cm, m);
    }
    const Lane before = a;
    absorb_scaled<U * E>(f, cm, scale, a);
    // -infinity (and what the scale takes there) makes 0 * infinity of a term of T: once more, vector by vector, with such logits at
    // kEmpty, whose terms are 0.  NaN and +infinity stay what they are.
    if (__any(a.T != a.T)) {
        a = before;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            u32x4 again = v[k];
            asm volatile("" : "+v"(again));      // unpacked anew, instead of every logit being kept until here
            float g[E];
            Tr::unpack(again, g);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = g[e] < kEmpty ? kEmpty : g[e];
            absorb_scaled<E>(g, larger(vm[k], kFloor), scale, a);
        }
    }
}

template <int CTRL>
__device__ __forceinline__ float from_lane(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140, kRotate8 = 0x128;      // 7 - lane in each 8, 15 - lane in each 16
// Of two vectors' maxima a lane keeps the one that its bit says, with what its partner has of it.
template <int CTRL>
__device__ __forceinline__ float keep_one(float lo, float hi, bool bit)
{
    const float keep = bit ? hi : lo, send = bit ? lo : hi;
    return larger(keep, from_lane<CTRL>(send));
}
// Of four vectors' maxima per lane, over aligned runs of 2^LG lanes: the one that kept_vector says.  (Halving the values with each
// step takes 14 instructions where reducing each vector takes 24.)
template <int LG>
__device__ __forceinline__ float run_max4(const float (&vm)[4], int lane)
{
    static_assert(LG >= 2 && LG <= 4, "runs of 4, 8 or 16 lanes");
    if constexpr (LG == 2) {
        const bool b1 = (lane & 2) != 0, b0 = (lane & 1) != 0;
        return keep_one<kXor1>(keep_one<kXor2>(vm[0], vm[2], b1), keep_one<kXor2>(vm[1], vm[3], b1), b0);
    } else {
        const bool b2 = (lane & 4) != 0, b1 = (lane & 2) != 0;
        float x = keep_one<kXor2>(keep_one<kMirror8>(vm[0], vm[2], b2), keep_one<kMirror8>(vm[1], vm[3], b2), b1);
        x = larger(x, from_lane<kXor1>(x));
        if constexpr (LG == 4) x = larger(x, from_lane<kRotate8>(x));
        return x;
    }
}
template <int LG>
__device__ __forceinline__ int kept_vector(int lane)
{
    return LG == 2 ? (lane & 3) : ((lane >> 1) & 3);
}
__device__ __forceinline__ float wave_max(float x)
{
    x = larger(x, from_lane<kXor1>(x));
    x = larger(x, from_lane<kXor2>(x));
    x = larger(x, from_lane<kMirror8>(x));
    x = larger(x, from_lane<kMirror16>(x));
    const int i = __float_as_int(x);
    return larger(larger(__int_as_float(__builtin_amdgcn_readlane(i, 0)), __int_as_float(__builtin_amdgcn_readlane(i, 16))),
                  larger(__int_as_float(__builtin_amdgcn_readlane(i, 32)), __int_as_float(__builtin_amdgcn_readlane(i, 48))));
}

// Order-preserving bits of a logit, -0 as +0; 0: masked.
__device__ __forceinline__ uint32_t key_of(float f)
{
    if (!(f > kFloor)) return 0u;
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint32_t key_of_floor() { return ~__float_as_uint(kFloor); }
// Of equal logits the lower id is the larger key; 0: masked.
__device__ __forceinline__ uint64_t ranked(uint32_t key, uint32_t id) { return key == 0u ? 0ull : ((uint64_t)key << 32) | (0xffffffffu - id); }

struct Shared {
    float gmax[kMaxGroups];
    alignas(16) uint64_t elems[kElemList + 8];
    uint32_t groups[kGroupList];
    double S[kTopkWaves], T[kTopkWaves];
    float m[kTopkWaves];
    uint32_t bound[kTopkWaves];
    uint32_t counts[2][kTopkWaves];
    uint32_t n_groups, n_elems;
    double ln_s;                    // ln of the row's sum, by thread 0
};

// The statistics of a row, from the lanes': largest logit, sum and weighted sum (log2 units), in every thread.
struct Row {
    float m;
    double S, T;
};
__device__ __forceinline__ Row merge_lanes(const Lane& a, float scale, Shared& sh)
{
    const int wave = threadIdx.x >> 6;
    const float wm = wave_max(a.m);
    // The argument z scale - mL differs from (z - m) scale by the rounding of mL, the same for every term of the lane; taken out
    // here, so that the term of the maximum is exactly 1.
    const float delta = fmaf(a.m, scale, -a.mL);
    const float d = fmaf(a.m - wm, scale, -delta);
    const float s = a.S == 0.0f ? 0.0f : fast_exp2(d);       // nothing but masked logits: delta is anything there
    const double S = (double)s * ((double)a.S + (double)a.Sc);
    const double T = (double)s * ((double)a.T + (double)d * (double)a.S);
    const double wS = wave_sum_f64(S), wT = wave_sum_f64(T);
    if ((threadIdx.x & 63) == 0) {
        sh.m[wave] = wm;
        sh.S[wave] = wS;
        sh.T[wave] = wT;
    }
    __syncthreads();
    Row r = {sh.m[0], 0.0, 0.0};
#pragma unroll
    for (int w = 1; w < kTopkWaves; ++w) r.m = fmaxf(r.m, sh.m[w]);
#pragma unroll
    for (int w = 0; w < kTopkWaves; ++w) {
        const float dw = (sh.m[w] - r.m) * scale;
        const double sw = (double)fast_exp2(dw);
        r.S += sw * sh.S[w];
        r.T += sw * (sh.T[w] + (double)dw * sh.S[w]);
    }
    return r;
}

// A vector of a row; behind the row's end, and where V ends inside a vector, the filler.
template <class Tr>
__device__ __forceinline__ u32x4 load_vector(const typename Tr::elem* rowp, int32_t V, int i)
{
    constexpr int E = Tr::kPerVec;
    const int nvec = V / E;
    if (i < nvec) return load_stream(reinterpret_cast<const u32x4*>(rowp) + i);
    u32x4 v = Tr::filler();
    if (i == nvec) {
        for (int e = 0; e < V - nvec * E; ++e) {
            if constexpr (E == 8) {
                const uint32_t b = rowp[i * E + e];
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w == (e >> 1)) v[w] = (e & 1) ? (v[w] & 0xffffu) | (b << 16) : (v[w] & 0xffff0000u) | b;
            } else {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w == e) v[w] = __float_as_uint(rowp[i * E + e]);
            }
        }
    }
    return v;
}

// Number of threads' items that hold, over the workgroup (uniform).  turn alternates, so that one barrier a call is enough.
__device__ __forceinline__ uint32_t block_count(uint32_t mine, int turn, Shared& sh)
{
    double x = wave_sum_f64((double)mine);
    if ((threadIdx.x & 63) == 0) sh.counts[turn & 1][threadIdx.x >> 6] = (uint32_t)x;
    __syncthreads();
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < kTopkWaves; ++w) n += sh.counts[turn & 1][w];
    return n;
}

// The largest key that at least K of the ranked keys reach (0: there are fewer).  each(f) calls f(key) for every key of
// this thread.
template <class Each>
__device__ uint64_t kth_ranked(const Each& each, uint32_t K, Shared& sh)
{
    uint64_t t = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t c = t | (1ull << bit);
        uint32_t mine = 0;
        each([&](uint64_t key) { mine += key >= c ? 1u : 0u; });
        if (block_count(mine, bit, sh) >= K) t = c;
    }
    __syncthreads();
    return t;
}

// The K largest of a row whose groups' maxima are in sh.gmax, written in order.  All threads of the workgroup call it after a
// barrier; row is the same in all of them.
template <class Tr>
__device__ void select_and_write(const TopkArgs& a, const typename Tr::elem* rowp, int64_t row, int ngroups, const Row& st, Shared& sh)
{
    constexpr int E = Tr::kPerVec;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t K = (uint32_t)a.K;
    const uint32_t per_wave = (K + kTopkWaves - 1) / kTopkWaves;

    // lower bound of the K-th largest; neighbouring groups go to different waves, so that each wave has its share of a short row
    constexpr int kPerLane = kMaxGroups / kTopkThreads;
    float mine[kPerLane];
    float best = kFloor;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        const int g = (i * 64 + lane) * kTopkWaves + wave;
        mine[i] = g < ngroups ? sh.gmax[g] : kFloor;
        best = fmaxf(best, mine[i]);
    }
    const uint32_t best_key = key_of(best);
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = t | (1u << bit);
        const uint32_t n = (uint32_t)__popcll(__ballot(best_key >= c));
        if (n >= per_wave) t = c;
        if (n == per_wave) break;
    }
    if (lane == 0) sh.bound[wave] = t;
    if (tid == 0) sh.n_groups = sh.n_elems = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTopkWaves; ++w) t = min(t, sh.bound[w]);
    const float bound = value_of(max(t, key_of_floor() + 1u));

#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        if (mine[i] >= bound) {
            const uint32_t at = atomicAdd(&sh.n_groups, 1u);
            if (at < kGroupList) sh.groups[at] = (uint32_t)((i * 64 + lane) * kTopkWaves + wave);
        }
    }
    __syncthreads();
    uint32_t n_groups = sh.n_groups;
    // f(logit, id) of every element of the listed groups and of those behind the last whole vector, shared out over the threads;
    // four loads at a time, since each one is a round trip to memory
    const int nvec = a.V / E;
    auto each_element = [&](const auto& f) {
        const uint64_t units = (uint64_t)n_groups << a.lg;
        for (uint64_t u0 = 0; u0 < units; u0 += 4 * kTopkThreads) {
            u32x4 v[4];
            int at[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint64_t u = u0 + q * kTopkThreads + tid;
                v[q] = Tr::filler();
                at[q] = nvec;
                if (u < units) {
                    const int64_t i = ((int64_t)sh.groups[u >> a.lg] << a.lg) + (int64_t)(u & ((1u << a.lg) - 1u));
                    if (i < nvec) {
                        at[q] = (int)i;
                        v[q] = reinterpret_cast<const u32x4*>(rowp)[i];
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (at[q] == nvec) continue;
                float x[E];
                Tr::unpack(v[q], x);
#pragma unroll
                for (int e = 0; e < E; ++e) f(x[e], (uint32_t)(at[q] * E + e));
            }
        }
        if (tid < a.V - nvec * E) f(Tr::load1(rowp + nvec * E + tid), (uint32_t)(nvec * E + tid));
    };
    bool full = n_groups > kGroupList;
    if (!full) {
        each_element([&](float x, uint32_t id) {
            if (x >= bound) {
                const uint32_t at = atomicAdd(&sh.n_elems, 1u);
                if (at < kElemList) sh.elems[at] = ranked(key_of(x), id);
            }
        });
        __syncthreads();
        full = sh.n_elems > kElemList;
    }
    if (full) {     // uniform
        const uint64_t tg = kth_ranked([&](const auto& f) {
            for (int g = tid; g < ngroups; g += kTopkThreads) f(ranked(key_of(sh.gmax[g]), (uint32_t)g));
        }, K, sh);
        if (tid == 0) sh.n_groups = sh.n_elems = 0;
        __syncthreads();
        for (int g = tid; g < ngroups; g += kTopkThreads) {
            const uint64_t r = ranked(key_of(sh.gmax[g]), (uint32_t)g);
            if (r != 0ull && r >= tg) sh.groups[atomicAdd(&sh.n_groups, 1u)] = (uint32_t)g;      // K at most: the keys differ
        }
        __syncthreads();
        n_groups = sh.n_groups;
        const uint64_t te = kth_ranked([&](const auto& f) { each_element([&](float x, uint32_t id) { f(ranked(key_of(x), id)); }); }, K, sh);
        each_element([&](float x, uint32_t id) {
            const uint64_t r = ranked(key_of(x), id);
            if (r == 0ull || r < te) return;
            const uint32_t at = atomicAdd(&sh.n_elems, 1u);
            if (at < kElemList) sh.elems[at] = r;
        });
        __syncthreads();
    }
    const uint32_t n = min(sh.n_elems, (uint32_t)kElemList);
    if (tid < 8) sh.elems[n + tid] = 0ull;                 // the ranks are counted eight keys at a time
    __syncthreads();
    const double ln_s = sh.ln_s;
    int32_t* ids = a.top_ids + row * a.K;
    float* logp = a.top_logp + row * a.K;
    for (uint32_t j = tid; j < n; j += kTopkThreads) {
        const uint64_t mine = sh.elems[j];
        uint32_t rank = 0;
        for (uint32_t i = 0; i < n; i += 8) {
#pragma unroll
            for (int q = 0; q < 8; ++q) rank += sh.elems[i + q] > mine ? 1u : 0u;
        }
        if (rank < K) {
            ids[rank] = (int32_t)(0xffffffffu - (uint32_t)mine);
            logp[rank] = (float)(((double)value_of((uint32_t)(mine >> 32)) - (double)st.m) * a.inv_t - ln_s);
        }
    }
    for (uint32_t j = n + tid; j < K; j += kTopkThreads) {      // fewer unmasked tokens than were asked for
        ids[j] = -1;
        logp[j] = -INFINITY;
    }
}

// One workgroup per row.  LG: log2 of the vectors in a group, kManyVectors: a.lg, more than a run of 16 lanes.
constexpr int kManyVectors = 5;
template <class Tr, int LG>
__global__ __launch_bounds__(kTopkThreads) void topk_row_kernel(const typename Tr::elem* __restrict__ logits, TopkArgs a)
{
    constexpr int NT = kTopkThreads, U = kTopkUnroll, E = Tr::kPerVec;
    __shared__ Shared sh;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const typename Tr::elem* rowp = logits + row * a.row_stride;
    const int nvec = a.V / E, all = (a.V + E - 1) / E;
    const int ngroups = (all + (1 << a.lg) - 1) >> a.lg;
    if constexpr (LG == kManyVectors) {
        for (int g = tid; g < ngroups; g += NT) sh.gmax[g] = kEmpty;
        __syncthreads();
    }
    // the largest of each of this thread's four vectors, 256 apart from `first` on, into their groups'
    auto note = [&](const float (&vm)[4], int first, auto whole) {
        if constexpr (LG < 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float g = vm[k];
                if constexpr (LG == 1) g = larger(g, from_lane<kXor1>(g));
                if (whole || first + k * NT + tid < all) sh.gmax[(first >> LG) + k * (NT >> LG) + (tid >> LG)] = g;
            }
        } else {
            constexpr int RUN = LG < 4 ? LG : 4;
            const float g = run_max4<RUN>(vm, tid);
            const int k = kept_vector<RUN>(tid), at = k * NT + (tid & -(1 << RUN));      // from first on
            if (whole || first + at < all) {
                if constexpr (LG == kManyVectors) atomicMax(&sh.gmax[(first + at) >> a.lg], g);
                else sh.gmax[(first >> LG) + (at >> LG)] = g;
            }
        }
    };
    const int32_t y = a.token_ids ? a.token_ids[row] : -1;
    const bool has_y = y >= 0 && y < a.V;
    const float zy = has_y ? Tr::load1(rowp + y) : 0.0f;      // ahead of the stream, so that nothing waits for it at the end
    Lane acc = {kFloor, kFloor * a.scale, 0.0f, 0.0f, 0.0f};
    auto take = [&](const u32x4* v, int first, auto whole) {
        const u32x4 four[4] = {v[0], v[1], v[2], v[3]};
        float vm[4];
        absorb_vectors<Tr, 4>(four, a.scale, acc, vm);
        note(vm, first, whole);
    };
    int base = 0;
    for (; base + U * NT <= nvec; base += U * NT) {
        u32x4 v[U];
#pragma unroll
        for (int k = 0; k < U; ++k)      // uniform base, lane offset
            v[k] = load_stream(reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(rowp) + ((size_t)(base + k * NT) << 4) + ((uint32_t)tid << 4)));
        __builtin_amdgcn_sched_barrier(0);      // all of them on their way before the first is used
#pragma unroll
        for (int k = 0; k < U; k += 4) take(v + k, base + k * NT, std::true_type{});
    }
    if (base < all) {       // the rest, its loads together
        u32x4 v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) v[k] = load_vector<Tr>(rowp, a.V, base + k * NT + tid);
#pragma unroll
        for (int k = 0; k < U; k += 4)
            if (base + k * NT < all) take(v + k, base + k * NT, std::false_type{});
    }
    const Row st = merge_lanes(acc, a.scale, sh);       // its barrier also closes the groups' maxima
    const bool ok = st.m > kFloor && st.S >= 0.5 && st.S < 1.0e30;       // neither NaN, +infinity nor everything masked
    if (tid == 0) {
        const double ln_s = log(st.S);
        sh.ln_s = ln_s;
        const float nan = __builtin_nanf("");
        a.lse[row] = ok ? (float)((double)st.m * a.inv_t + ln_s) : nan;
        a.entropy[row] = ok ? (float)(ln_s - st.T * (double)kLn2 / st.S) : nan;
        if (a.logp) a.logp[row] = ok && has_y ? (float)(((double)zy - (double)st.m) * a.inv_t - ln_s) : nan;
    }
    if (!ok) {
        for (int j = tid; j < a.K; j += NT) {
            a.top_ids[row * a.K + j] = -1;
            a.top_logp[row * a.K + j] = __builtin_nanf("");
        }
        return;
    }
    select_and_write<Tr>(a, rowp, row, ngroups, st, sh);
}

template <class Tr>
void launch_topk_rows(const void* logits, const TopkArgs& a, hipStream_t st)
{
    auto go = [&](auto lg) {
        constexpr int LG = decltype(lg)::value;
        hipLaunchKernelGGL((topk_row_kernel<Tr, LG>), dim3((unsigned)a.N), dim3(kTopkThreads), 0, st, (const typename Tr::elem*)logits, a);
    };
    switch (a.lg) {
    case 0: return go(std::integral_constant<int, 0>{});
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 3: return go(std::integral_constant<int, 3>{});
    case 4: return go(std::integral_constant<int, 4>{});
    default: return go(std::integral_constant<int, kManyVectors>{});
    }
}

}  // namespace

extern "C" {

size_t ulorl_token_topk_workspace_bytes(int64_t N, int64_t V)
{
    if (!shape_ok(N, V, V) || N > 0x7fffffffLL) return 0;
    return 256;
}

int32_t ulorl_token_topk(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t row_stride, const int32_t* token_ids,
                         int32_t K, float temperature, int32_t* top_ids, float* top_logp, float* logp, float* entropy, float* lse,
                         void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (N == 1 && row_stride >= V) row_stride = (V + 7) / 8 * 8;       // a lone row has no stride
    int32_t rc = check_logits(logits, dt, N, V, row_stride);
    if (rc != ULORL_OK) return rc;
    if (N > 0x7fffffffLL || K < 1 || K > kMaxK) return ULORL_ERR_SHAPE;
    if (!top_ids || !top_logp || !entropy || !lse || (token_ids && !logp)) return ULORL_ERR_NULL;
    if (!(temperature >= 1.0e-3f && temperature <= 1.0e3f)) return ULORL_ERR_PARAM;
    if (workspace && (((uintptr_t)workspace & 255u) != 0 || workspace_bytes < ulorl_token_topk_workspace_bytes(N, V))) return ULORL_ERR_WORKSPACE;
    TopkArgs a;
    a.token_ids = token_ids;
    a.top_ids = top_ids; a.top_logp = top_logp; a.logp = token_ids ? logp : nullptr; a.entropy = entropy; a.lse = lse;
    a.N = N; a.row_stride = row_stride; a.V = (int32_t)V; a.K = K;
    a.inv_t = 1.0 / (double)temperature;
    a.scale = (float)(1.4426950408889634074 * a.inv_t);
    const int64_t all = (V + (dt == ULORL_F32 ? 3 : 7)) / (dt == ULORL_F32 ? 4 : 8);
    a.lg = 0;
    while (((all + ((int64_t)1 << a.lg) - 1) >> a.lg) > kMaxGroups) ++a.lg;
    hipStream_t st = (hipStream_t)hip_stream;
    if (dt == ULORL_BF16)
        launch_topk_rows<StoreBF16>(logits, a, st);
    else
        launch_topk_rows<StoreF32>(logits, a, st);
    return hipGetLastError() == hipSuccess ? ULORL_OK : ULORL_ERR_HIP;
}

}  // extern "C"
