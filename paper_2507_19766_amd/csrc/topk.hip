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
//      group maxima by bisection over ballots; t is the smallest of the waves' values, so at least K groups reach t.  (One bound
//      over all lanes' maxima would leave 1.05 K groups at four times the ballots: no faster up to K 64, 5 % at 128.)
//   3. Only groups that reach t (about 1.3 K of 2374 at K 64) are read again, and their elements that reach t are listed: about as
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

#include "kth_key.hpp"
#include "logits_stream.hpp"
#include "row_sums.hpp"
#include "ulorl.h"
#include "ulorl_internal.hpp"

using namespace ulorl_detail;

#pragma clang fp contract(off)

namespace {

constexpr int kTopkThreads = 256;     // of a workgroup; 64 where a row is a wave's
// Vectors a thread has in flight: eight (four workgroups a compute unit) on rows of 256 KB and more, four (seven workgroups) on
// shorter ones, where the search is a larger part and more rows hide it.  us, eight / four with six workgroups: 4096 x 151936 bf16
// 201 / 203, 8192 x 64000 181 / 173, 8000 x 32000 119 / 110; six / seven workgroups: 1777 x 32000 29.5 / 28.2, 20000 x 8192 112 / 106.
constexpr int kLongRow = 16384;       // vectors
constexpr int kMaxK = 128;
constexpr int groups_per_lane(int nt) { return nt <= 256 ? 10 : 2560 / nt; }
constexpr int max_groups(int nt) { return nt * groups_per_lane(nt); }     // group maxima of a row: 10 KB of LDS with 256 threads
constexpr int kMaxGroups = max_groups(kTopkThreads);                  // and of a split row's, with 512
constexpr uint32_t kOverflow = 0xffffffffu;
// Where rows are split: few of them, each long.  us, split / one workgroup a row, K 8: 1 row of 151936 bf16 11 / 16, fp32 11 / 25; 100 rows 15.2 / 20.8
// and 18.3 / 27.3; 200 rows 20.1 / 21.6 and 28.0 / 29.0; 256 rows 22.9 / 22.1 and 33.5 / 30.3; 1 row of 32000 bf16 11.5 / 9.1.
constexpr int kMaxPieces = 64;
constexpr int64_t kSplitRows = 200;
constexpr int64_t kSplitBatches = 8;          // of 16 KB
constexpr int64_t kFewWorkgroups = 1024;
// Of the workgroup that finishes a split row, whose chain of steps is what such a call waits for.  us with 256 / 512 / 1024, K 20 (K 128):
// 1 row of 151936 bf16 11.5 / 10.9 / 13.2 (17 / 14 / 16), 64 rows 15.1 / 15.1 / 17.0 (28 / 20.5 / 20.2).
constexpr int kMergeThreads = 512;

// Where one wave does a row: short rows, enough of them to fill the chip.  No barriers, and what a row costs besides its stream (joining
// the lanes, the search) is done once instead of by four waves.  us, wave / workgroup of four, K 10, 64 and 128: 20000 x 2048 fp32
// 38 / 93, 51 / 102 and 86 / 148, 20000 x 8192 bf16 64 / 102, 87 / 122 and 135 / 173, 20000 x 16384 bf16 112 / 136, 141 / 157 and 211 / 218,
// 4096 x 4096 fp32 14.8 / 22.5, 19 / 26 and 33 / 41; and where it is not taken, K 10, 256 x 4096 fp32 8.0 / 6.4, 1024 x 16384 bf16 14.6 / 12.4,
// 20000 x 32000 bf16 (K 33) 226 / 226.  Rows as many as vectors in one, and 1024, is where both are alike with K 64 (1024 x 4096 fp32 10.3 /
// 10.1, 2048 x 16384 bf16 23.6 / 22.9); there a wave is up to 16 % faster with K 10 (7.3 / 8.7, 17.9 / 20.5) and up to 10 % slower with K 128
// (19.4 / 17.7, 36.7 / 33.4), whose ranks are a larger part.
constexpr int kWaveRow = 2048;        // vectors
constexpr int64_t kManyRows = 1024;
static_assert(kWaveRow <= (max_groups(64) << 2), "a wave's row has groups of four vectors at most");

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
    int32_t piece_vectors;      // vectors of a piece, where a row is split
    float scale;                // log2(e) / T
    double inv_t;
};

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
            if (!__any(!(vm[k] <= kFloor))) continue;        // all masked, most of a row under a grammar: nothing to add
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

template <int NT>
struct Shared {
    static constexpr int kWaves = NT / 64;
    static constexpr int kGroupsPerWave = kWaves == 1 ? 256 : 128;     // of the lists that a wave makes
    static constexpr int kElemsPerWave = kWaves == 1 ? 288 : 192;
    static constexpr int kElemSlots = kElemsPerWave + 8;
    static_assert(kMaxK <= kElemsPerWave && kMaxK <= kGroupsPerWave, "where a list overflows, K groups and K elements take its place");
    float gmax[max_groups(NT)];
    alignas(16) uint64_t elems[kWaves * kElemSlots];
    uint32_t groups[kWaves * kGroupsPerWave];
    double S[kWaves], T[kWaves];
    float m[kWaves];
    uint32_t bound[kWaves];
    uint32_t counts[2][kWaves];
    uint32_t found[kWaves + 1];        // the second counter of a lone wave's exact search included
    double ln_s;                    // ln of the row's sum, by thread 0
};

// The statistics of a row, from the lanes': largest logit, sum and weighted sum (log2 units), in every thread.
struct Row {
    float m;
    double S, T;
};
template <int NT>
__device__ __forceinline__ Row merge_lanes(const Lane& a, float scale, Shared<NT>& sh)
{
    const int wave = threadIdx.x >> 6;
    const float wm = wave_max(a.m);
    // The argument z scale - mL differs from (z - m) scale by the rounding of mL, the same for every term of the lane; taken out
    // here, so that the term of the maximum is exactly 1.
    const float delta = fmaf(a.m, scale, -a.mL);
    const float d = fmaf(a.m - wm, scale, -delta);
    const float s = a.S == 0.0f ? 0.0f : fast_exp2(d);       // nothing but masked logits: delta is anything there
    const double S = (double)s * ((double)a.S + (double)a.Sc);
    const double T = (double)s * (((double)a.T + (double)a.Tc) + (double)d * ((double)a.S + (double)a.Sc));
    const double wS = wave_sum_f64(S), wT = wave_sum_f64(T);
    if ((threadIdx.x & 63) == 0) {
        sh.m[wave] = wm;
        sh.S[wave] = wS;
        sh.T[wave] = wT;
    }
    __syncthreads();
    Row r = {sh.m[0], 0.0, 0.0};
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r.m = fmaxf(r.m, sh.m[w]);
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const float dw = (sh.m[w] - r.m) * scale;
        const double sw = (double)fast_exp2(dw);
        r.S += sw * sh.S[w];
        r.T += sw * (sh.T[w] + (double)dw * sh.S[w]);
    }
    return r;
}

// Number of threads' items that hold, over the workgroup (uniform).  turn is one more with every call, so that one barrier a call is enough.
template <int NT>
__device__ __forceinline__ uint32_t block_count(uint32_t mine, int turn, Shared<NT>& sh)
{
    double x = wave_sum_f64((double)mine);
    if ((threadIdx.x & 63) == 0) sh.counts[turn & 1][threadIdx.x >> 6] = (uint32_t)x;
    __syncthreads();
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) n += sh.counts[turn & 1][w];
    return n;
}

// kth_key over the keys of all threads: each(f) calls f(key) for every key of this thread.
template <int NT, class Each>
__device__ uint64_t kth_ranked(const Each& each, uint32_t K, uint32_t n, Shared<NT>& sh)
{
    const uint64_t t = kth_key(K, n, [&](uint64_t c, int turn) {
        uint32_t mine = 0;
        each([&](uint64_t key) { mine += key >= c ? 1u : 0u; });
        return block_count(mine, turn, sh);
    });
    __syncthreads();            // the next search starts at turn 0 again
    return t;
}

// The lanes of this wave that hit, below this one.
__device__ __forceinline__ uint32_t hits_below(uint64_t hits)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)hits, 0u));
}

// f(logit, id) of every element of n listed groups, shared out over `lanes` threads of which this is number `lane`; all threads of
// a wave call f together, one that has no element with a masked logit.  Eight loads at a time: each is a round trip to memory.
template <class Tr, class F>
__device__ __forceinline__ void each_element(const TopkArgs& a, const typename Tr::elem* rowp, const uint32_t* list, uint32_t n, uint32_t lane,
                                             uint32_t lanes, const F& f)
{
    constexpr int E = Tr::kPerVec, B = 8;
    const int nvec = a.V / E;
    const uint64_t units = (uint64_t)n << a.lg;
    for (uint64_t u0 = 0; u0 < units; u0 += B * lanes) {
        u32x4 v[B];
        int at[B];
#pragma unroll
        for (int q = 0; q < B; ++q) {
            const uint64_t u = u0 + q * lanes + lane;
            v[q] = Tr::filler();
            at[q] = 0;
            if (u < units) {
                const int64_t i = ((int64_t)list[u >> a.lg] << a.lg) + (int64_t)(u & ((1u << a.lg) - 1u));
                if (i < nvec) {
                    at[q] = (int)i;
                    v[q] = reinterpret_cast<const u32x4*>(rowp)[i];
                }
            }
        }
#pragma unroll
        for (int q = 0; q < B; ++q) {
            if (u0 + q * lanes >= units) break;
            float x[E];
            Tr::unpack(v[q], x);
#pragma unroll
            for (int e = 0; e < E; ++e) f(x[e], (uint32_t)(at[q] * E + e));
        }
    }
}

// The K largest of a row whose groups' maxima are in sh.gmax, written in order.  All threads of the workgroup call it after a
// barrier; row is the same in all of them.  Each wave lists the groups and elements that are its own (neighbouring groups are
// different waves'), so that two barriers are enough.  Cycles of a row at 2048 x 151936 bf16, K 64 (K 128): stream and
// statistics 70000, bound 1900, list 1400, elements 7500 (13000), ranks and results 3100 (8300).
template <class Tr, int NT>
__device__ void select_and_write(const TopkArgs& a, const typename Tr::elem* rowp, int64_t row, int ngroups, const Row& st, Shared<NT>& sh)
{
    constexpr int E = Tr::kPerVec, W = NT / 64, kGroupsPerWave = Shared<NT>::kGroupsPerWave, kElemsPerWave = Shared<NT>::kElemsPerWave,
                  kElemSlots = Shared<NT>::kElemSlots, kGroupsPerLane = groups_per_lane(NT);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t K = (uint32_t)a.K;
    const uint32_t per_wave = (K + W - 1) / W;
    const int behind = (a.V / E) * E, tail = a.V - behind;       // elements behind the last whole vector

    // lower bound of the K-th largest
    auto group_of = [&](int i) { return (i * 64 + lane) * W + wave; };
    constexpr int P = W < 4 ? 4 / W : 1;            // of a lane's maxima this many take part: 256 over the workgroup at least, two times the largest K
    float mine[kGroupsPerLane], best[P];
    uint32_t best_key[P];
#pragma unroll
    for (int p = 0; p < P; ++p) best[p] = kFloor;
#pragma unroll
    for (int i = 0; i < kGroupsPerLane; ++i) {
        mine[i] = group_of(i) < ngroups ? sh.gmax[group_of(i)] : kFloor;
        best[i % P] = larger(best[i % P], mine[i]);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) best_key[p] = key_of(best[p]);
    auto reach = [&](uint32_t c) {
        uint32_t n = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) n += (uint32_t)__popcll(__ballot(best_key[p] >= c));
        return n;
    };
    uint32_t t = 0;
    for (int bit = 30; bit >= 0; bit -= 2) {        // two bits a step: the steps are a chain of scalar instructions
        const uint32_t c1 = t | (1u << bit), c2 = t | (2u << bit), c3 = t | (3u << bit);
        const uint32_t n1 = reach(c1), n2 = reach(c2), n3 = reach(c3);
        const uint32_t n = n3 >= per_wave ? n3 : n2 >= per_wave ? n2 : n1;
        t = n3 >= per_wave ? c3 : n2 >= per_wave ? c2 : n1 >= per_wave ? c1 : t;
        if (n == per_wave) break;
    }
    if (lane == 0) sh.bound[wave] = t;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) t = min(t, sh.bound[w]);
    const float bound = value_of(max(t, key_of_floor() + 1u));

    // this wave's groups that reach it, and their elements that do
    uint32_t* groups = sh.groups + wave * kGroupsPerWave;
    uint64_t* elems = sh.elems + wave * kElemSlots;
    uint32_t n_groups = 0, n_elems = 0;         // uniform
#pragma unroll
    for (int i = 0; i < kGroupsPerLane; ++i) {
        const uint64_t hits = __ballot(mine[i] >= bound);
        const uint32_t at = n_groups + hits_below(hits);
        if (mine[i] >= bound && at < kGroupsPerWave) groups[at] = (uint32_t)group_of(i);
        n_groups += (uint32_t)__popcll(hits);
    }
    auto collect = [&](float x, uint32_t id) {
        const uint64_t hits = __ballot(x >= bound);
        if (hits == 0ull) return;
        const uint32_t at = n_elems + hits_below(hits);
        if (x >= bound && at < kElemsPerWave) elems[at] = ranked(key_of(x), id);
        n_elems += (uint32_t)__popcll(hits);
    };
    if (n_groups <= kGroupsPerWave) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        each_element<Tr>(a, rowp, groups, n_groups, lane, 64, collect);
        if (wave == 0 && tail > 0) collect(lane < tail ? Tr::load1(rowp + behind + lane) : kEmpty, (uint32_t)behind + (uint32_t)lane);
    }
    const bool overflow = n_groups > kGroupsPerWave || n_elems > kElemsPerWave;
    if (lane == 0) sh.found[wave] = overflow ? kOverflow : n_elems;
    if (!overflow && lane < 8) elems[n_elems + lane] = 0ull;        // the ranks are counted eight keys at a time
    __syncthreads();
    uint32_t n[W];
    bool full = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        n[w] = sh.found[w];
        full = full || n[w] == kOverflow;
    }
    if (full) {     // uniform: the K-th largest key itself, of the groups and then of the elements of the K first groups
        const uint64_t tg = kth_ranked([&](const auto& f) {
            for (int g = tid; g < ngroups; g += NT) f(ranked(key_of(sh.gmax[g]), (uint32_t)g));
        }, K, (uint32_t)ngroups, sh);
        if (tid == 0) sh.found[0] = sh.found[1] = 0;
        __syncthreads();
        for (int g = tid; g < ngroups; g += NT) {
            const uint64_t r = ranked(key_of(sh.gmax[g]), (uint32_t)g);
            if (r != 0ull && r >= tg) sh.groups[atomicAdd(&sh.found[0], 1u)] = (uint32_t)g;      // K at most: the keys differ
        }
        __syncthreads();
        const uint32_t listed = sh.found[0];
        auto each_key = [&](const auto& f) {
            each_element<Tr>(a, rowp, sh.groups, listed, tid, NT, [&](float x, uint32_t id) { f(ranked(key_of(x), id)); });
            if (tid < tail) f(ranked(key_of(Tr::load1(rowp + behind + tid)), (uint32_t)(behind + tid)));
        };
        const uint64_t te = kth_ranked(each_key, K, (uint32_t)a.V, sh);
        each_key([&](uint64_t r) {
            if (r != 0ull && r >= te) sh.elems[atomicAdd(&sh.found[1], 1u)] = r;                    // K at most
        });
        __syncthreads();
        n[0] = sh.found[1];
#pragma unroll
        for (int w = 1; w < W; ++w) n[w] = 0;
        if (tid < 8) sh.elems[n[0] + tid] = 0ull;
        __syncthreads();
    }

    const double ln_s = sh.ln_s;
    int32_t* ids = a.top_ids + row * a.K;
    float* logp = a.top_logp + row * a.K;
    uint32_t total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) total += n[w];
    // a key's rank is its place; with few keys two or four lanes count for each
    const uint32_t lg_parts = total <= NT / 4 ? 2 : total <= NT / 2 ? 1 : 0;
    const uint32_t part = (uint32_t)tid & ((1u << lg_parts) - 1u);
    for (uint32_t j0 = 0; j0 < total; j0 += NT >> lg_parts) {
        const uint32_t j = j0 + ((uint32_t)tid >> lg_parts);
        uint64_t key = 0;
        uint32_t at = j;
        if (j < total) {
            uint32_t w = 0;
            while (at >= n[w]) at -= n[w++];
            key = sh.elems[w * kElemSlots + at];
        }
        uint32_t rank = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            for (uint32_t i = part * 8; i < n[w]; i += 8u << lg_parts) {
#pragma unroll
                for (int q = 0; q < 8; ++q) rank += sh.elems[w * kElemSlots + i + q] > key ? 1u : 0u;
            }
        }
        if (lg_parts >= 1) rank += (uint32_t)__builtin_amdgcn_mov_dpp((int)rank, kXor1, 0xF, 0xF, true);
        if (lg_parts >= 2) rank += (uint32_t)__builtin_amdgcn_mov_dpp((int)rank, kXor2, 0xF, 0xF, true);
        if (j < total && part == 0 && rank < K) {
            ids[rank] = (int32_t)(0xffffffffu - (uint32_t)key);
            logp[rank] = (float)(((double)value_of((uint32_t)(key >> 32)) - (double)st.m) * a.inv_t - ln_s);
        }
    }
    for (uint32_t j = total + tid; j < K; j += NT) {      // fewer unmasked tokens than were asked for
        ids[j] = -1;
        logp[j] = -INFINITY;
    }
}

// The stream over vectors [begin, end) of a row (begin and, unless it is the row's end, end whole groups): the lane's statistics,
// and the groups' maxima in sh.gmax, from begin's group on, valid after a barrier.
// LG: log2 of the vectors in a group, or kManyVectors: a.lg, more than a run of 16 lanes.
constexpr int kManyVectors = 5;
template <class Tr, int LG, int U, int NT>
__device__ __forceinline__ Lane stream_vectors(const TopkArgs& a, const typename Tr::elem* rowp, int begin, int end, Shared<NT>& sh)
{
    constexpr int E = Tr::kPerVec;
    const int tid = threadIdx.x;
    const int whole_end = min(a.V / E, end);        // where the whole vectors end
    const int g0 = begin >> a.lg;
    if constexpr (LG == kManyVectors) {
        for (int g = tid; g <= ((end - 1) >> a.lg) - g0; g += NT) sh.gmax[g] = kEmpty;
        __syncthreads();
    }
    // the largest of each of this thread's four vectors, NT apart from `first` on, into their groups'
    auto note = [&](const float (&vm)[4], int first, auto whole) {
        if constexpr (LG < 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float g = vm[k];
                if constexpr (LG == 1) g = larger(g, from_lane<kXor1>(g));
                if (whole || first + k * NT + tid < end) sh.gmax[((first >> LG) - g0) + k * (NT >> LG) + (tid >> LG)] = g;
            }
        } else {
            constexpr int RUN = LG < 4 ? LG : 4;
            const float g = run_max4<RUN>(vm, tid);
            const int k = kept_vector<RUN>(tid), at = k * NT + (tid & -(1 << RUN));      // from first on
            if (whole || first + at < end) {
                if constexpr (LG == kManyVectors) atomicMax(&sh.gmax[((first + at) >> a.lg) - g0], g);
                else sh.gmax[((first >> LG) - g0) + (at >> LG)] = g;
            }
        }
    };
    Lane acc = {kFloor, kFloor * a.scale, 0.0f, 0.0f, 0.0f, 0.0f};
    auto take = [&](const u32x4* v, int first, auto whole) {
        const u32x4 four[4] = {v[0], v[1], v[2], v[3]};
        float vm[4];
        absorb_vectors<Tr, 4>(four, a.scale, acc, vm);
        note(vm, first, whole);
    };
    int base = begin;
    for (; base + U * NT <= whole_end; base += U * NT) {
        u32x4 v[U];
#pragma unroll
        for (int k = 0; k < U; ++k)      // uniform base, lane offset
            v[k] = load_stream(reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(rowp) + ((size_t)(base + k * NT) << 4) + ((uint32_t)tid << 4)));
        __builtin_amdgcn_sched_barrier(0);      // all of them on their way before the first is used
#pragma unroll
        for (int k = 0; k < U; k += 4) take(v + k, base + k * NT, std::true_type{});
    }
    if (base < end) {       // the rest, its loads together
        u32x4 v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) v[k] = base + k * NT + tid < end ? load_vector<Tr>(rowp, a.V, base + k * NT + tid) : Tr::filler();
#pragma unroll
        for (int k = 0; k < U; k += 4)
            if (base + k * NT < end) take(v + k, base + k * NT, std::false_type{});
    }
    return acc;
}

// What a row's token has to do with its results, fetched ahead of what they are waited for with.
struct Token {
    bool has;
    float z;
};
template <class Tr>
__device__ __forceinline__ Token token_of(const TopkArgs& a, const typename Tr::elem* rowp, int64_t row)
{
    const int32_t y = a.token_ids ? a.token_ids[row] : -1;
    const bool has = y >= 0 && y < a.V;
    const float z = has ? Tr::load1(rowp + y) : 0.0f;
    return Token{has, z <= kFloor ? -INFINITY : z};         // masked: of probability 0
}

// A row's results from its statistics and its groups' maxima in sh.gmax.  All threads call it after a barrier.
template <class Tr, int NT>
__device__ __forceinline__ void finish_row(const TopkArgs& a, const typename Tr::elem* rowp, int64_t row, const Row& st, const Token& token, Shared<NT>& sh)
{
    const int all = vectors_of<Tr>(a.V), ngroups = (all + (1 << a.lg) - 1) >> a.lg;
    const bool ok = st.m > kFloor && st.S >= 0.5 && st.S < 1.0e30;       // neither NaN, +infinity nor everything masked
    if (threadIdx.x == 0) {
        const double ln_s = log64(st.S);
        sh.ln_s = ln_s;
        const float nan = __builtin_nanf("");
        a.lse[row] = ok ? (float)((double)st.m * a.inv_t + ln_s) : nan;
        a.entropy[row] = ok ? (float)(ln_s - st.T * (double)kLn2 / st.S) : nan;
        if (a.logp) a.logp[row] = ok && token.has ? (float)(((double)token.z - (double)st.m) * a.inv_t - ln_s) : nan;
    }
    if (!ok) {
        for (int j = threadIdx.x; j < a.K; j += NT) {
            a.top_ids[row * a.K + j] = -1;
            a.top_logp[row * a.K + j] = __builtin_nanf("");
        }
        return;
    }
    select_and_write<Tr, NT>(a, rowp, row, ngroups, st, sh);
}

// Rows over grid dimensions x and y: a launch holds at most 2^32 threads along one.
constexpr int64_t kRowsPerGridX = 1 << 20;
__device__ __forceinline__ int64_t row_of_grid() { return (int64_t)blockIdx.y * kRowsPerGridX + blockIdx.x; }

// One workgroup per row.  At 151936 bf16 logits and K 64 it reads 6.4 TB/s (the statistics alone: 7.0): its vector ALUs are
// 89 % busy, the search adds instructions (to those of ulorl_token_loss_fwd's statistics, K 1: 7 %, K 33: 11 %, K 128: 33 %) and 6 us in
// which a workgroup loads little; four workgroups share a
// compute unit (five, with registers in scratch memory for it, 20 % slower; 12 loads in flight instead of 8, three workgroups, 2 %).
// Short rows take 72 registers for seven (eight: scratch, 8000 x 32000 124 us instead of 104), in fp32 64 for eight (seven: 2000 x 64000
// 87 us instead of 83, a second round).
template <class Tr, int LG, int U, int NT>
__global__ __launch_bounds__(NT, U == 4 && NT == 256 ? (Tr::kPerVec == 4 ? 8 : 7) : 1) void topk_row_kernel(const typename Tr::elem* __restrict__ logits, TopkArgs a)
{
    __shared__ Shared<NT> sh;
    const int64_t row = row_of_grid();
    if (row >= a.N) return;
    const typename Tr::elem* rowp = logits + row * a.row_stride;
    const Token token = token_of<Tr>(a, rowp, row);
    const Lane acc = stream_vectors<Tr, LG, U, NT>(a, rowp, 0, vectors_of<Tr>(a.V), sh);
    const Row st = merge_lanes(acc, a.scale, sh);       // its barrier also closes the groups' maxima
    finish_row<Tr, NT>(a, rowp, row, st, token, sh);
}

// Few rows: several workgroups stream a row's pieces, one more finishes it.  What a row's pieces leave for it:
struct RowParts {
    float gmax[kMaxGroups];
    Row piece[kMaxPieces];
};
template <class Tr, int LG>
__global__ __launch_bounds__(kTopkThreads) void topk_piece_kernel(const typename Tr::elem* __restrict__ logits, TopkArgs a, RowParts* parts)
{
    __shared__ Shared<kTopkThreads> sh;
    const int64_t row = blockIdx.y;
    const int all = vectors_of<Tr>(a.V);
    const int begin = (int)blockIdx.x * a.piece_vectors, end = min(all, begin + a.piece_vectors);
    const Lane acc = stream_vectors<Tr, LG, 4, kTopkThreads>(a, logits + row * a.row_stride, begin, end, sh);
    const Row st = merge_lanes(acc, a.scale, sh);
    RowParts& to = parts[row];
    if (threadIdx.x == 0) to.piece[blockIdx.x] = st;
    const int g0 = begin >> a.lg, g1 = (end - 1) >> a.lg;
    for (int g = g0 + (int)threadIdx.x; g <= g1; g += kTopkThreads) to.gmax[g] = sh.gmax[g - g0];
}
template <class Tr>
__global__ __launch_bounds__(kMergeThreads) void topk_merge_kernel(const typename Tr::elem* __restrict__ logits, TopkArgs a, int32_t pieces, const RowParts* parts)
{
    __shared__ Shared<kMergeThreads> sh;
    __shared__ Row merged;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const typename Tr::elem* rowp = logits + row * a.row_stride;
    const RowParts& from = parts[row];
    const Token token = token_of<Tr>(a, rowp, row);
    const int all = vectors_of<Tr>(a.V), ngroups = (all + (1 << a.lg) - 1) >> a.lg;
#pragma unroll
    for (int i = 0; i < groups_per_lane(kMergeThreads); ++i)
        if (i * kMergeThreads + tid < ngroups) sh.gmax[i * kMergeThreads + tid] = from.gmax[i * kMergeThreads + tid];
    if (tid < 64) {         // a piece per lane
        static_assert(kMaxPieces == 64 && max_groups(kMergeThreads) == kMaxGroups, "one piece per lane; the pieces' groups");
        Row p = {kFloor, 0.0, 0.0};
        if (tid < pieces) p = from.piece[tid];
        const float m = wave_max(p.m);
        const float d = (p.m - m) * a.scale;
        const double s = (double)fast_exp2(d);
        const double S = wave_sum_f64(s * p.S), T = wave_sum_f64(s * (p.T + (double)d * p.S));
        if (tid == 0) merged = Row{m, S, T};
    }
    __syncthreads();
    const Row st = merged;
    finish_row<Tr, kMergeThreads>(a, rowp, row, st, token, sh);
}

// f(constant) for the log2 of a group's vectors.
template <class F>
void with_group(int lg, const F& f)
{
    switch (lg) {
    case 0: return f(std::integral_constant<int, 0>{});
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    default: return f(std::integral_constant<int, kManyVectors>{});
    }
}

template <class Tr>
void launch_topk(const void* logits, TopkArgs a, RowParts* parts, hipStream_t st)
{
    const typename Tr::elem* z = (const typename Tr::elem*)logits;
    const int64_t all = vectors_of<Tr>(a.V);
    a.lg = 0;
    while (((all + ((int64_t)1 << a.lg) - 1) >> a.lg) > kMaxGroups) ++a.lg;
    // Pieces of whole batches of 1024 vectors, as many as bring the launch to about kFewWorkgroups workgroups.
    const int64_t batch = 4 * kTopkThreads, batches = (all + batch - 1) / batch;
    int64_t per = (batches * a.N + kFewWorkgroups - 1) / kFewWorkgroups;
    if (per < (batches + kMaxPieces - 1) / kMaxPieces) per = (batches + kMaxPieces - 1) / kMaxPieces;
    const int64_t pieces = (batches + per - 1) / per;
    if (parts != nullptr && a.N <= kSplitRows && batches >= kSplitBatches && pieces > 1 && ((int64_t)1 << a.lg) <= batch) {
        a.piece_vectors = (int32_t)(per * batch);
        with_group(a.lg, [&](auto lg) {
            constexpr int LG = decltype(lg)::value;
            static_assert(kSplitBatches > 7 && 7 * 4 * kTopkThreads > (kMaxGroups << 1), "rows that are split have groups of four vectors or more");
            if constexpr (LG >= 2)
                hipLaunchKernelGGL((topk_piece_kernel<Tr, LG>), dim3((unsigned)pieces, (unsigned)a.N), dim3(kTopkThreads), 0, st, z, a, parts);
        });
        hipLaunchKernelGGL((topk_merge_kernel<Tr>), dim3((unsigned)a.N), dim3(kMergeThreads), 0, st, z, a, (int32_t)pieces, parts);
        return;
    }
    const dim3 grid((unsigned)(a.N < kRowsPerGridX ? a.N : kRowsPerGridX), (unsigned)((a.N + kRowsPerGridX - 1) / kRowsPerGridX));
    if (all <= kWaveRow && a.N >= kManyRows && a.N >= all) {
        a.lg = 0;
        while (((all + ((int64_t)1 << a.lg) - 1) >> a.lg) > max_groups(64)) ++a.lg;
        with_group(a.lg, [&](auto lg) {
            constexpr int LG = decltype(lg)::value;
            if constexpr (LG <= 2) hipLaunchKernelGGL((topk_row_kernel<Tr, LG, LG == 0 ? 4 : 8, 64>), grid, dim3(64), 0, st, z, a);
        });
        return;
    }
    with_group(a.lg, [&](auto lg) {
        constexpr int LG = decltype(lg)::value;
        static_assert((kMaxGroups << 2) < kLongRow && kLongRow < (kMaxGroups << 3), "long rows have groups of eight vectors or more");
        auto launch = [&](auto u) {
            hipLaunchKernelGGL((topk_row_kernel<Tr, LG, decltype(u)::value, kTopkThreads>), grid, dim3(kTopkThreads), 0, st, z, a);
        };
        if constexpr (LG >= 4) launch(std::integral_constant<int, 8>{});
        else if constexpr (LG < 3) launch(std::integral_constant<int, 4>{});
        else if (all >= kLongRow) launch(std::integral_constant<int, 8>{});
        else launch(std::integral_constant<int, 4>{});
    });
}

}  // namespace

extern "C" {

size_t ulorl_token_topk_workspace_bytes(int64_t N, int64_t V)
{
    if (!shape_ok(N, V, V) || N > 0x7fffffffLL) return 0;
    return (size_t)(N < kSplitRows ? N : kSplitRows) * sizeof(RowParts);
}

int32_t ulorl_token_topk(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t row_stride, const int32_t* token_ids,
                         int32_t K, float temperature, int32_t* top_ids, float* top_logp, float* logp, float* entropy, float* lse,
                         void* workspace, size_t workspace_bytes, void* hip_stream)
{
    row_stride = row_stride_of(N, V, row_stride);
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
    a.lg = 0; a.piece_vectors = 0;
    hipStream_t st = (hipStream_t)hip_stream;
    if (dt == ULORL_BF16)
        launch_topk<StoreBF16>(logits, a, (RowParts*)workspace, st);
    else
        launch_topk<StoreF32>(logits, a, (RowParts*)workspace, st);
    return hipGetLastError() == hipSuccess ? ULORL_OK : ULORL_ERR_HIP;
}

}  // extern "C"
