// Distillation from a teacher's recorded tokens: ulorl_distill_fwd / _bwd / _fwd_bwd.
//
// A row's target is a distribution over the listed tokens and one bucket for all others.  With x = z / T, p = softmax(x), q_k the
// teacher's probabilities, q_rest what it leaves to the others, Q = sum q_k + q_rest, and "rest" the unlisted tokens:
//     kl      = sum_k q_k (ln q_k - ln p_k) + q_rest (ln q_rest - ln p_rest)
//     d kl / d x_k (listed)   = p_k Q - q_k
//     d kl / d x_j (unlisted) = (Q p_rest - q_rest) softmax_rest(j),    softmax_rest(j) = e^(x_j) / sum_rest e^x
// So the vocabulary enters a row by two numbers, the largest unlisted logit and the sum S over the unlisted ones relative to it;
// the listed logits are K numbers that are gathered on the way.  S leaves the listed tokens out while it is formed: p_rest as 1 minus
// the listed probabilities would lose all its digits where the student is sure of them.  What a row is made of after that (K terms)
// is in 64 bits: a divergence is a small sum of larger terms.
//
//   distill_target_kernel   is the target a distribution; what the row's gradient needs of it (unless the stream's workgroups do it)
//   distill_piece_kernel    the stream over the logits: a row's pieces, each a workgroup's registers (a short row a wave's), to (max, S);
//                           listed logits
//   distill_row_kernel      one call: the same pieces, which tell each other their sums and write the gradient from the registers
//   distill_finish_kernel   kl, the listed tokens' gradients, the unlisted ones' coefficient; the loss
//   distill_dense_kernel    the gradient of all tokens as if unlisted, one 16-byte vector per thread
//   distill_top_kernel      the listed tokens' gradients over it
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "logits_stream.hpp"
#include "row_sums.hpp"
#include "ulorl.h"
#include "ulorl_internal.hpp"

using namespace ulorl_detail;

#pragma clang fp contract(off)

namespace {

constexpr int kMaxK = 128;              // two listed tokens per lane of a wave
constexpr int64_t kMaxDistillRows = 1 << 24;
constexpr int kThreads = 256;           // of a workgroup; 64 where a row is a wave's
// The finishing kernel takes no more workgroups than take their tickets quickly (2048 of them, 20 us; 256, 3):
// small ones, spread over the chip, while 256 of them are enough (256 rows 7.5 us, in large ones 11.7), else large ones, which fill it
// (8192 rows 27 us, in small ones 38).
constexpr int kFinishGroups = 256;
constexpr int kFinishSmall = 256, kFinishLarge = 1024;

// Where one wave does a row: short rows, enough of them to fill the chip.  No barriers, and what a row costs besides its logits (target,
// lists, joining the lanes) is done by one wave instead of four.  One call, K 8 (K 64), us, wave / workgroup of four: 16384 x 1000 bf16
// 44 / 86 (53 / 97), 16384 x 4096 68 / 91 (90 / 110), 4096 x 2048 fp32 22 / 28 (30 / 36), 2048 x 4096 bf16 19 / 22 (24 / 25); and where it is
// not taken, 1024 x 2048 fp32 15.4 / 15.4 (18.3 / 17.7), 16384 x 8192 bf16 113 / 107 (139 / 131).
constexpr int64_t kWaveRow = 512;       // vectors
constexpr int64_t kManyRows = 2048;

// Where pieces work their row's target out themselves: one to a row, or few enough of them to wait for it all at once; pieces that tell each other
// their sums need a kernel before them, which clears what they tell them through.  Forward, us, themselves / distill_target_kernel: 1 x 151936
// bf16 12.2 / 14.8, 256 x 32000 14.4 / 16.5, 256 x 151936 26.3 / 26.3, 1024 x 64000 34.3 / 32.5, 8192 x 32000 (K 128) 127 / 117.
constexpr int64_t kFewPieces = 1024;

// Listed probabilities may sum to more than 1 by their rounding (log-probs kept in bf16: 2 %); beyond this they are no log-probs.
constexpr double kMostMass = 1.25;

enum { ROW_ON = 0, ROW_WEIGHTLESS = 1, ROW_EMPTY = 2, ROW_BAD_TOKEN = 3, ROW_BAD_TARGET = 4 };

// What the stream has to know of a row's target: g Q and g q_rest, with g = weight / (D T).  twice: an id is listed twice, which the
// stream finds (and publishes as a sum that is no number; with own_target in the forward call, as a piece's second word).
struct RowTarget {
    float mass, rest;
    int32_t state;
    int32_t twice;
};

struct Partial {
    double loss;
    int64_t on, weightless, empty, status;
};

struct DistillArgs {
    const int32_t* ids;         // [N, K]
    const float* teacher;       // [N, K]
    const float* weights;       // may be NULL
    float* loss;
    float* kl;
    float* lse;
    float* rest_max;
    float* rest_coef;
    float* top_grad;            // [N, K]; the listed logits until the row is finished
    int64_t* counters;          // may be NULL
    RowTarget* target;          // [N]
    unsigned long long* slots;  // [N * C * 2]: {max, S} of a piece's unlisted logits, {max, S} of its listed ones (forward: an id twice)
    unsigned long long* pending;    // [N], one call: pieces whose gradient is not written, because a wait expired
    Partial* partial;           // [kFinishGroups]
    uint32_t* flags;            // ticket of the finishing kernel; one call: whether any wait expired
    int32_t spin_limit;         // one call: polls before a wait is given up; 0: two passes
    float grad_out;
    int64_t N, row_stride;
    int32_t V, K, C;
    int32_t tail;
    int32_t own_target;         // no distill_target_kernel
    float scale;                // log2(e) / T
    double inv_t, inv_D;
};

// A row's K terms are worked on by L lanes, two terms each: 16, 32 or 64 as K asks, so that a wave takes up to four rows (what is
// the same for all of a row's terms costs a wave the same however many rows it has).  Sums and maxima over the row's lanes, in
// each of them, in a fixed order.
template <int L>
struct Lanes {
    static_assert(L == 16 || L == 32 || L == 64, "whole rows of 16 lanes");
    template <int CTRL>
    static __device__ __forceinline__ double add(double x)
    {
        const int lo = __builtin_amdgcn_mov_dpp(__double2loint(x), CTRL, 0xF, 0xF, true), hi = __builtin_amdgcn_mov_dpp(__double2hiint(x), CTRL, 0xF, 0xF, true);
        return x + __hiloint2double(hi, lo);
    }
    static __device__ __forceinline__ double sum(double x)
    {
        if constexpr (L == 64) return wave_sum_f64(x);
        x = add<kMirror16>(add<kMirror8>(add<kXor2>(add<kXor1>(x))));
        if constexpr (L == 32) x += __shfl_xor(x, 16);
        return x;
    }
    static __device__ __forceinline__ float max(float x)
    {
        if constexpr (L == 64) return wave_max(x);
        x = larger(x, from_lane<kXor1>(x));
        x = larger(x, from_lane<kXor2>(x));
        x = larger(x, from_lane<kMirror8>(x));
        x = larger(x, from_lane<kMirror16>(x));
        if constexpr (L == 32) x = larger(x, __shfl_xor(x, 16));
        return x;
    }
    static __device__ __forceinline__ bool any(bool b)
    {
        const uint64_t row = L == 64 ? ~0ull : ((1ull << (L & 63)) - 1ull) << (threadIdx.x & 63 & ~(L - 1));
        return (__ballot(b) & row) != 0ull;
    }
};
inline int lanes_of(int K) { return K <= 32 ? 16 : K <= 64 ? 32 : 64; }

// ---------------------------------------------------------------------------------------------
// the targets
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.4028235e38f; }

// By L lanes, in each of them.
template <int L>
__device__ __forceinline__ RowTarget row_target(const DistillArgs& a, int64_t row, int lane)
{
    const float w = a.weights ? a.weights[row] : 1.0f;
    int32_t id[2];
    float l[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = lane + L * h;
        id[h] = j < a.K ? a.ids[row * a.K + j] : -1;
        l[h] = j < a.K ? a.teacher[row * a.K + j] : -INFINITY;
        l[h] = id[h] >= 0 ? l[h] : -INFINITY;
    }
    RowTarget t = {0.0f, 0.0f, ROW_ON, 0};
    if (w == 0.0f) {
        t.state = ROW_WEIGHTLESS;
        return t;
    }
    const bool beyond = id[0] >= a.V || id[1] >= a.V;
    const bool bad = !finite(w) || !(l[0] <= 3.4028235e38f) || !(l[1] <= 3.4028235e38f);
    if (Lanes<L>::any(beyond)) {
        t.state = ROW_BAD_TOKEN;
    } else if (Lanes<L>::any(bad)) {
        t.state = ROW_BAD_TARGET;
    } else if (!Lanes<L>::any(id[0] >= 0 || id[1] >= 0) || (a.tail == ULORL_TAIL_RENORM && !Lanes<L>::any(l[0] > -INFINITY || l[1] > -INFINITY))) {
        t.state = ROW_EMPTY;
    } else {
        const double g = (double)w * a.inv_D * a.inv_t;
        double mass = 1.0, rest = 0.0;
        if (a.tail != ULORL_TAIL_RENORM) {
            const double q = Lanes<L>::sum(exp64((double)l[0]) + (a.K > L ? exp64((double)l[1]) : 0.0));
            if (!(q <= kMostMass)) t.state = ROW_BAD_TARGET;
            rest = a.tail == ULORL_TAIL_BUCKET && q < 1.0 ? 1.0 - q : 0.0;
            mass = q + rest;
        }
        t.mass = (float)(g * mass);
        t.rest = (float)(g * rest);
    }
    return t;
}

// What all of a row's workgroups have to know.
template <int L>
__global__ __launch_bounds__(kThreads) void distill_target_kernel(DistillArgs a)
{
    const int lane = threadIdx.x & (L - 1);
    const int64_t row = (int64_t)blockIdx.x * (kThreads / L) + (int)threadIdx.x / L;
    if (blockIdx.x == 0 && threadIdx.x < 2) a.flags[threadIdx.x] = 0u;
    if (row >= a.N) return;
    if (a.spin_limit > 0) {         // the exchange of the one-call path starts from zeros
        if (lane == 0) a.pending[row] = 0ull;
        for (int k = lane; k < 2 * a.C; k += L) a.slots[row * a.C * 2 + k] = 0ull;
    }
    const RowTarget t = row_target<L>(a, row, lane);
    if (lane == 0) a.target[row] = t;
}

// ---------------------------------------------------------------------------------------------
// the stream
// ---------------------------------------------------------------------------------------------
// Takes element e out of a vector: a masked logit in its place.
template <class Tr>
__device__ __forceinline__ void take_out(u32x4& v, int e)
{
    if constexpr (Tr::kPerVec == 8) {
        const uint32_t keep = (e & 1) ? 0x0000ffffu : 0xffff0000u;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (w == (e >> 1)) v[w] = (v[w] & keep) | (Tr::filler()[0] & ~keep);
    } else {
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (w == e) v[w] = Tr::filler()[0];
    }
}

// Absorbs vectors v[K .. VPT) in groups of four, two and one.
template <class Tr, int VPT, int K>
__device__ __forceinline__ void absorb_rest(const u32x4 (&v)[VPT], float scale, Lane& acc)
{
    constexpr int REM = VPT - K;
    if constexpr (REM > 0) {
        constexpr int G = REM >= 4 ? 4 : REM >= 2 ? 2 : 1;
        constexpr int E = Tr::kPerVec;
        float f[G * E];
        float cm = kFloor;
#pragma unroll
        for (int q = 0; q < G; ++q) Tr::unpack(v[K + q], f + q * E);
#pragma unroll
        for (int k = 0; k < G * E; ++k) cm = larger(cm, f[k]);
        absorb_scaled<G * E, false>(f, cm, scale, acc);
        absorb_rest<Tr, VPT, K + G>(v, scale, acc);
    }
}

template <int NT>
struct PieceShared {
    static constexpr int kWaves = NT / 64;
    int32_t head[NT];           // of a thread's listed tokens, -1: none
    int32_t next[kMaxK];
    int32_t where[kMaxK];       // vector of the thread * 8 + element
    float m[kWaves], top_m[kWaves];
    double S[kWaves], top_S[kWaves];
    RowTarget target;           // where the workgroup works it out
    int32_t twice;
};

struct PieceSums {
    float m, top_m;
    double S, top_S;            // relative to them
};

// A row's piece c into registers.
template <class Tr, int VPT, int NT>
__device__ __forceinline__ void load_piece(const typename Tr::elem* rowp, int32_t V, int c, u32x4 (&v)[VPT])
{
    const int tid = threadIdx.x, first = c * NT * VPT;
    if (first + NT * VPT <= V / Tr::kPerVec) {
        const char* const piece = reinterpret_cast<const char*>(rowp) + ((size_t)first << 4);      // uniform base, lane offset
#pragma unroll
        for (int k = 0; k < VPT; ++k) v[k] = load_stream(reinterpret_cast<const u32x4*>(piece + (size_t)k * NT * 16 + ((uint32_t)tid << 4)));
    } else {
#pragma unroll
        for (int k = 0; k < VPT; ++k) v[k] = load_vector<Tr>(rowp, V, first + k * NT + tid);
    }
}

// A row's target, and its piece c on the way into registers; false: the row does not count (and is not read where its weight is 0).
// With own_target the workgroups work the target out themselves while the row is on its way, and no kernel runs before them.
template <class Tr, int VPT, int NT>
__device__ __forceinline__ bool start_piece(const DistillArgs& a, const typename Tr::elem* rowp, int64_t row, int c, u32x4 (&v)[VPT], RowTarget& target,
                                            PieceShared<NT>& sh)
{
    if (!a.own_target) {
        target = a.target[row];
        if (target.state != ROW_ON) return false;
        load_piece<Tr, VPT, NT>(rowp, a.V, c, v);
        return true;
    }
    const int tid = threadIdx.x;
    if (a.weights == nullptr || a.weights[row] != 0.0f) load_piece<Tr, VPT, NT>(rowp, a.V, c, v);
    if (row == 0 && c == 0 && tid < 2) a.flags[tid] = 0u;       // for the kernel that follows
    if (tid < 64) {
        const RowTarget t = row_target<64>(a, row, tid);
        if (tid == 0) sh.target = t;
    }
    __syncthreads();
    target = sh.target;
    if (target.state == ROW_ON) return true;
    if (tid == 0 && c == 0) a.target[row] = target;
    return false;
}

// A piece's registers (v) lose their listed tokens, whose logits go to a.top_grad; the piece's sums (thread 0).  TOP: the listed
// tokens' sum is wanted too.
template <class Tr, int VPT, bool TOP, int NT>
__device__ __forceinline__ PieceSums piece_sums(const DistillArgs& a, const typename Tr::elem* rowp, int64_t row, int c, u32x4 (&v)[VPT],
                                                const RowTarget& target, PieceShared<NT>& sh)
{
    constexpr int E = Tr::kPerVec, kWaves = NT / 64;
    constexpr int H = NT < kMaxK ? kMaxK / NT : 1;          // listed tokens a thread
    const int tid = threadIdx.x, wave = tid >> 6;
    const int first = c * NT * VPT;
    int32_t id[H];
#pragma unroll
    for (int h = 0; h < H; ++h) id[h] = tid + h * NT < a.K ? a.ids[row * a.K + tid + h * NT] : -1;

    // each thread's listed tokens as a chain in LDS
    sh.head[tid] = -1;
    if (tid == 0) sh.twice = 0;
    __syncthreads();
    float z[H];
    bool dead[H], in_piece[H];                  // dead: the row is no row, a token of the teacher's masked, or listed twice
    int at[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int j = tid + h * NT;
        z[h] = kFloor;
        dead[h] = false;
        at[h] = id[h] / E - first;              // id < V: the row's state says so
        in_piece[h] = id[h] >= 0 && at[h] >= 0 && at[h] < NT * VPT;
        if (in_piece[h]) {
            z[h] = Tr::load1(rowp + id[h]);
            a.top_grad[row * a.K + j] = z[h];
            sh.where[j] = (at[h] / NT) * 8 + (id[h] & (E - 1));
            sh.next[j] = atomicExch(&sh.head[at[h] & (NT - 1)], j);
            dead[h] = z[h] <= kFloor && a.teacher[row * a.K + j] > -INFINITY;
        }
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < H; ++h) {
        if (!in_piece[h]) continue;
        for (int j = sh.head[at[h] & (NT - 1)]; j >= 0; j = sh.next[j]) {
            if (j != tid + h * NT && sh.where[j] == sh.where[tid + h * NT]) {
                dead[h] = true;
                sh.twice = 1;
            }
        }
    }
    for (int j = sh.head[tid]; j >= 0; j = sh.next[j]) {
        const int k_j = sh.where[j] >> 3, e = sh.where[j] & 7;
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (k == k_j) take_out<Tr>(v[k], e);
    }

    Lane acc = {kFloor, kFloor * a.scale, 0.0f, 0.0f, 0.0f, 0.0f};
    absorb_rest<Tr, VPT, 0>(v, a.scale, acc);
    const float wm = wave_max(acc.m);
    // z scale - mL differs from (z - m) scale by the rounding of mL: taken out here (nothing to take out of an empty lane)
    const float d = fmaf(acc.m - wm, a.scale, -fmaf(acc.m, a.scale, -acc.mL));
    const double S = acc.S == 0.0f ? 0.0 : (double)fast_exp2(d) * ((double)acc.S + (double)acc.Sc);
    const double wS = wave_sum_f64(S);
    if ((tid & 63) == 0) {
        sh.m[wave] = wm;
        sh.S[wave] = wS;
    }
    if constexpr (TOP) {
        float mine = z[0];
        if constexpr (H > 1) mine = larger(mine, z[1]);
        const float wt = wave_max(mine);
        double top = 0.0;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            if (z[h] > kFloor) top += (double)fast_exp2((z[h] - wt) * a.scale);
            if (z[h] != z[h] || dead[h]) top = (double)__builtin_nanf("");
        }
        top = wave_sum_f64(top);
        if ((tid & 63) == 0) {
            sh.top_m[wave] = wt;
            sh.top_S[wave] = top;
        }
    }
    __syncthreads();
    PieceSums p = {kFloor, kFloor, 0.0, 0.0};
    if (tid == 0) {
        if (a.own_target) {
            if (c == 0) a.target[row] = RowTarget{target.mass, target.rest, target.state, TOP ? sh.twice : 0};
        } else if (sh.twice != 0) {
            a.target[row].twice = 1;
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) p.m = larger(p.m, sh.m[w]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) p.S += (double)fast_exp2((sh.m[w] - p.m) * a.scale) * sh.S[w];
        if constexpr (TOP) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) p.top_m = larger(p.top_m, sh.top_m[w]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) p.top_S += (double)fast_exp2((sh.top_m[w] - p.top_m) * a.scale) * sh.top_S[w];
        }
    }
    return p;
}

// Never 0: a maximum is kFloor where there is nothing, and a sum is 1 or more where the maximum is 0.
__device__ __forceinline__ unsigned long long slot_word(float m, double S)
{
    return ((unsigned long long)__float_as_uint((float)S) << 32) | __float_as_uint(m);
}

// Large bf16 pieces: four workgroups a compute unit at most, which keeps the chip's window of addresses narrow (8192 x 151936: 398 us with
// the six that would fit, 399 with five, 386 with four); small ones and fp32 take what fits (3001 x 32000: 53 us, with four 62).
template <class Tr, int VPT>
constexpr int kMostWaves = Tr::kPerVec == 8 && VPT >= 11 ? 4 : 8;

template <class Tr, int VPT, int NT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(1, kMostWaves<Tr, VPT>))) void distill_piece_kernel(const typename Tr::elem* logits, DistillArgs a)
{
    __shared__ PieceShared<NT> sh;
    const int64_t row = (int64_t)blockIdx.z * kRowsPerGridY + blockIdx.y;
    if (row >= a.N) return;
    const typename Tr::elem* rowp = logits + row * a.row_stride;
    u32x4 v[VPT];
    RowTarget target;
    if (!start_piece<Tr, VPT, NT>(a, rowp, row, (int)blockIdx.x, v, target, sh)) return;
    const PieceSums p = piece_sums<Tr, VPT, false, NT>(a, rowp, row, (int)blockIdx.x, v, target, sh);
    if (threadIdx.x == 0) {
        unsigned long long* slot = a.slots + (row * a.C + blockIdx.x) * 2;
        slot[0] = slot_word(p.m, p.S);
        if (a.own_target) slot[1] = (unsigned long long)sh.twice;
    }
}

// The gradient of a vector's tokens as if unlisted: c e^((z - m) / T).
// In bf16 c e^(x - m) = sign(c) 2^((z - m) scale + log2|c|), the sum a fused step; in fp32, where its rounding (|log2 c| is tens) would be
// ten units of the result, c 2^((z - m) scale).  z - m first: -m scale in the sum would be off by |m| scale 2^-24, 4 % of a value at logits of a million.
struct RestGradient {
    float c, m, shift, scale;
    bool none;                  // zeros: no coefficient
    __device__ __forceinline__ RestGradient(float coef, float max, float scale_) : c(coef), m(max), scale(scale_)
    {
        none = c == 0.0f;
        shift = none ? 0.0f : log2f(fabsf(c));
    }
    template <class Tr>
    __device__ __forceinline__ u32x4 of(const u32x4& v) const
    {
        constexpr int E = Tr::kPerVec;
        float f[E];
        Tr::unpack(v, f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = E == 4 ? c * fast_exp2((f[e] - m) * scale) : fast_exp2(fmaf(f[e] - m, scale, shift));
        u32x4 o = Tr::pack(f);
        if (E == 8 && c < 0.0f) o ^= Tr::sign_bits();
        return o;
    }
};

// Stores vector i of a row's gradient; where V ends inside it, the elements that there are.
template <class Tr>
__device__ __forceinline__ void store_vector(typename Tr::elem* outp, int32_t V, int i, const u32x4& o)
{
    constexpr int E = Tr::kPerVec;
    const int nvec = V / E;
    if (i < nvec) {
        store_stream(reinterpret_cast<u32x4*>(outp) + i, o);
    } else if (i == nvec) {
        float f[E];
        Tr::unpack(o, f);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < V - nvec * E) Tr::store1(outp + i * E + e, f[e]);
    }
}

// A row's gradient (a coefficient of it) under an upstream one: of rows that do not count 0, whatever the upstream is; of others what that
// makes of it, infinities and not-a-number included.
__device__ __forceinline__ float under(float g, float upstream) { return g == 0.0f ? 0.0f : g * upstream; }

// A listed token's gradient.
template <class Tr>
__device__ __forceinline__ void store_top(typename Tr::elem* outp, int32_t V, int32_t id, float g)
{
    if (id >= 0 && id < V) Tr::store1(outp + id, g);
}

// One call: the pieces of a row keep their logits in registers, tell each other their sums and write the gradient of their
// unlisted tokens; every logit is read once and every gradient written once (the listed tokens' over it, by
// distill_finish_kernel).  A piece's two words in a.slots, zero before, are relaxed agent-scope atomics that carry their own validity.
// A row's pieces are neighbours in dispatch order, so partners are resident or next in line; the wait is bounded all the same: a
// workgroup whose wait expires writes nothing (in place, its logits stay) and marks its piece, which distill_finish_kernel then
// writes.
template <class Tr, int VPT, int NT>
__global__ __launch_bounds__(NT) void distill_row_kernel(const typename Tr::elem* logits, typename Tr::elem* dlogits, DistillArgs a)
{
    __shared__ PieceShared<NT> sh;
    __shared__ float bc_coef, bc_max;
    __shared__ int bc_expired;
    const int64_t row = (int64_t)blockIdx.z * kRowsPerGridY + blockIdx.y;
    if (row >= a.N) return;
    const int tid = threadIdx.x, c = (int)blockIdx.x, first = c * NT * VPT;
    const int nvec = a.V / Tr::kPerVec;
    typename Tr::elem* outp = dlogits + row * a.row_stride;
    char* const piece_out = reinterpret_cast<char*>(outp) + ((size_t)first << 4);
    const bool full = first + NT * VPT <= nvec;
    RowTarget target;
    u32x4 v[VPT];
    auto store_all = [&](const auto& value) {
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            if (full) store_stream(reinterpret_cast<u32x4*>(piece_out + (size_t)k * NT * 16 + ((uint32_t)tid << 4)), value(k));
            else store_vector<Tr>(outp, a.V, first + k * NT + tid, value(k));
        }
    };
    const u32x4 zero = {0u, 0u, 0u, 0u};
    const typename Tr::elem* rowp = logits + row * a.row_stride;
    if (!start_piece<Tr, VPT, NT>(a, rowp, row, c, v, target, sh)) {
        store_all([&](int) { return zero; });
        return;
    }
    const PieceSums p = piece_sums<Tr, VPT, true, NT>(a, rowp, row, c, v, target, sh);
    if (tid < 64) {
        unsigned long long* slot = a.slots + row * a.C * 2;
        unsigned long long w0 = slot_word(p.m, p.S), w1 = slot_word(p.top_m, p.top_S);
        bool expired = false;
        if (tid == 0) {
            __hip_atomic_store(slot + 2 * c, w0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(slot + 2 * c + 1, w1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        if (a.C > 1) {
            w0 = w1 = 0;
            for (int spins = 0; tid < a.C;) {
                if (w0 == 0) w0 = __hip_atomic_load(slot + 2 * tid, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (w1 == 0) w1 = __hip_atomic_load(slot + 2 * tid + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                if (w0 != 0 && w1 != 0) break;
                if (++spins >= a.spin_limit) { expired = true; break; }
                __builtin_amdgcn_s_sleep(4);
            }
            expired = __any(expired);
        }
        const bool mine = tid < a.C;
        const float m = mine ? __uint_as_float((uint32_t)w0) : kFloor, tm = mine ? __uint_as_float((uint32_t)w1) : kFloor;
        const double S = mine ? (double)__uint_as_float((uint32_t)(w0 >> 32)) : 0.0, tS = mine ? (double)__uint_as_float((uint32_t)(w1 >> 32)) : 0.0;
        const float rest_max = wave_max(m), M = larger(rest_max, wave_max(tm));
        const double rest = wave_sum_f64((double)fast_exp2((m - rest_max) * a.scale) * S);      // relative to rest_max
        const double top = wave_sum_f64((double)fast_exp2((tm - M) * a.scale) * tS);            // relative to M
        const double R = (double)fast_exp2((rest_max - M) * a.scale) * rest;
        if (tid == 0) {
            const float coef = rest != 0.0 ? (float)(((double)target.mass * (R / (R + top)) - (double)target.rest) / rest) : 0.0f;
            bc_coef = finite(coef) ? under(coef, a.grad_out) : 0.0f;        // no number: a row that does not count
            bc_max = rest_max;
            bc_expired = expired;
            if (expired) {
                __hip_atomic_fetch_or(a.pending + row, 1ull << c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                a.flags[1] = 1u;
            }
        }
    }
    __syncthreads();
    if (bc_expired) return;
    const RestGradient grad(bc_coef, bc_max, a.scale);
    if (grad.none) store_all([&](int) { return zero; });
    else store_all([&](int k) { return grad.template of<Tr>(v[k]); });
}

// ---------------------------------------------------------------------------------------------
// the rows' results
// ---------------------------------------------------------------------------------------------
// Over a wave, in each lane: lanes in a fixed order, counts below 2^53 exactly.
__device__ __forceinline__ void wave_partial(Partial& p)
{
    p.loss = wave_sum_f64(p.loss);
    p.on = (int64_t)wave_sum_f64((double)p.on);
    p.weightless = (int64_t)wave_sum_f64((double)p.weightless);
    p.empty = (int64_t)wave_sum_f64((double)p.empty);
    int64_t status = 0;
#pragma unroll
    for (int bit = 1; bit <= ULORL_STATUS_BAD_TARGET; bit <<= 1) status |= __any((p.status & bit) != 0) ? bit : 0;
    p.status = status;
}
template <int NW>
__device__ __forceinline__ Partial all_partials(const Partial* part)
{
    Partial sum = part[0];
    for (int w = 1; w < NW; ++w) {
        sum.loss += part[w].loss;
        sum.on += part[w].on;
        sum.weightless += part[w].weightless;
        sum.empty += part[w].empty;
        sum.status |= part[w].status;
    }
    return sum;
}

template <class Tr, int NT, int L>
__global__ __launch_bounds__(NT) void distill_finish_kernel(const typename Tr::elem* logits, typename Tr::elem* dlogits, int32_t piece_vectors,
                                                                  DistillArgs a)
{
    constexpr int NW = NT / 64;
    __shared__ Partial part[NW];
    constexpr int ROWS = NT / L;                 // at a time
    const int lane = threadIdx.x & (L - 1);
    Partial mine = {0.0, 0, 0, 0, 0};
    for (int64_t row = (int64_t)blockIdx.x * ROWS + (int)threadIdx.x / L; row < a.N; row += (int64_t)gridDim.x * ROWS) {
        // everything a row needs is on its way before the first of it is looked at (of a row that does not count some of it is
        // anything)
        const RowTarget target = a.target[row];
        float* top = a.top_grad + row * a.K;
        const double w = a.weights ? (double)a.weights[row] : 1.0;
        int32_t id[2] = {-1, -1};
        float z[2] = {kFloor, kFloor}, listed[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (lane + L * h < a.K) {
                id[h] = a.ids[row * a.K + lane + L * h];
                z[h] = top[lane + L * h];
                listed[h] = a.teacher[row * a.K + lane + L * h];
            }
        }
        const unsigned long long slot = lane < a.C ? a.slots[(row * a.C + lane) * 2] : 0ull;
        bool twice = target.twice != 0;
        if (a.own_target && a.spin_limit == 0) {
            for (int c = lane; c < a.C; c += L) twice = twice || a.slots[(row * a.C + c) * 2 + 1] != 0ull;
            twice = Lanes<L>::any(twice);
        }
        const int32_t state = target.state == ROW_ON && twice ? ROW_BAD_TARGET : target.state;
        float grad[2] = {0.0f, 0.0f};
        float kl_out = 0.0f, lse_out = 0.0f, max_out = 0.0f, coef_out = 0.0f;
        if (state == ROW_ON) {
            // the listed tokens; the second of a lane's two only where there is one
            double l[2], e[2] = {0.0, 0.0}, q[2] = {0.0, 0.0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                z[h] = id[h] >= 0 ? z[h] : kFloor;
                l[h] = id[h] >= 0 ? (double)listed[h] : -INFINITY;
            }
            // the unlisted ones: the row's pieces
            float m = kFloor;
            double S = 0.0;
            if (lane < a.C) {
                m = __uint_as_float((uint32_t)slot);
                S = (double)__uint_as_float((uint32_t)(slot >> 32));
            }
            for (int c = lane + L; c < a.C; c += L) {
                const unsigned long long w0 = a.slots[(row * a.C + c) * 2];
                const float pm = __uint_as_float((uint32_t)w0), M = larger(m, pm);
                S = exp64(((double)m - (double)M) * a.inv_t) * S + exp64(((double)pm - (double)M) * a.inv_t) * (double)__uint_as_float((uint32_t)(w0 >> 32));
                m = M;
            }
            const float rest_max = Lanes<L>::max(m);
            if (a.C > 1) S *= exp64(((double)m - (double)rest_max) * a.inv_t);
            S = Lanes<L>::sum(S);
            const float M = larger(rest_max, Lanes<L>::max(larger(z[0], z[1])));
            const double R = exp64(((double)rest_max - (double)M) * a.inv_t) * S;         // relative to M, as the listed ones
            double norm = 0.0;
            if (a.tail == ULORL_TAIL_RENORM) {
                const double lm = (double)Lanes<L>::max(larger((float)l[0], (float)l[1]));
                norm = lm + log64(Lanes<L>::sum(exp64(l[0] - lm) + (a.K > L ? exp64(l[1] - lm) : 0.0)));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h == 1 && a.K <= L) break;
                if (!(z[h] <= kFloor)) e[h] = exp64(((double)z[h] - (double)M) * a.inv_t);
                l[h] -= norm;
                q[h] = exp64(l[h]);
            }
            const double total = R + Lanes<L>::sum(e[0] + e[1]), q_sum = Lanes<L>::sum(q[0] + q[1]);
            const double ln_total = log64(total), per_total = 1.0 / total, per_S = 1.0 / S;
            bool dead = false;
            double terms = 0.0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool masked = z[h] <= kFloor;
                dead = dead || (masked && l[h] > -INFINITY);
                if (q[h] > 0.0 && !masked) terms += q[h] * (l[h] - (((double)z[h] - (double)M) * a.inv_t - ln_total));
            }
            const bool has_rest = S > 0.0;
            const double q_rest = a.tail == ULORL_TAIL_BUCKET && has_rest && q_sum < 1.0 ? 1.0 - q_sum : 0.0;
            const double mass = q_sum + q_rest;
            double kl = Lanes<L>::sum(terms);
            if (q_rest > 0.0) kl += q_rest * (log64(q_rest * per_S) - (((double)rest_max - (double)M) * a.inv_t - ln_total));
            const bool ok = !Lanes<L>::any(dead) && total > 0.0 && total < 1.0e300 && fabs(kl) < 1.0e300;
            lse_out = total > 0.0 ? (float)((double)M * a.inv_t + ln_total) : __builtin_nanf("");
            if (ok) {
                const double g = w * a.inv_D * a.inv_t;
                kl_out = (float)kl;
                max_out = rest_max;
                if (has_rest) coef_out = (float)(g * (mass * (R * per_total) - q_rest) * per_S);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (id[h] >= 0) grad[h] = (float)(g * (e[h] * per_total * mass - q[h]));
                mine.loss += w * kl;
                mine.on += 1;
            } else {
                mine.status |= ULORL_STATUS_NONFINITE;
            }
        } else if (state == ROW_WEIGHTLESS) {
            mine.weightless += 1;
        } else if (state == ROW_EMPTY) {
            mine.empty += 1;
        } else {
            mine.status |= state == ROW_BAD_TOKEN ? ULORL_STATUS_BAD_TOKEN : ULORL_STATUS_BAD_TARGET;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (lane + L * h < a.K) top[lane + L * h] = grad[h];
            // one call: the unlisted tokens' gradients are there already
            if (a.spin_limit > 0 && state == ROW_ON) store_top<Tr>(dlogits + row * a.row_stride, a.V, id[h], under(grad[h], a.grad_out));
        }
        if (lane == 0) {
            a.kl[row] = kl_out;
            a.lse[row] = lse_out;
            a.rest_max[row] = max_out;
            a.rest_coef[row] = coef_out;
        }
    }
    if (a.spin_limit > 0 && a.flags[1] != 0u) {     // pieces whose workgroup waited in vain: their logits are whole, in place too
        __threadfence();                            // the rows' results are these lanes' own
        const int all = vectors_of<Tr>(a.V);
        for (int64_t row = (int64_t)blockIdx.x * ROWS + (int)threadIdx.x / L; row < a.N; row += (int64_t)gridDim.x * ROWS) {
            for (unsigned long long todo = a.pending[row]; todo != 0ull; todo &= todo - 1ull) {
                const RestGradient rest(under(a.rest_coef[row], a.grad_out), a.rest_max[row], a.scale);
                const int begin = (__ffsll((long long)todo) - 1) * piece_vectors;
                for (int i = begin + lane; i < min(all, begin + piece_vectors); i += L)
                    store_vector<Tr>(dlogits + row * a.row_stride, a.V, i,
                                     rest.none ? u32x4{0u, 0u, 0u, 0u} : rest.template of<Tr>(load_vector<Tr>(logits + row * a.row_stride, a.V, i)));
            }
            if (a.pending[row] == 0ull) continue;
            __threadfence();                        // the listed tokens' again, over them
            for (int j = lane; j < a.K; j += L)
                store_top<Tr>(dlogits + row * a.row_stride, a.V, a.ids[row * a.K + j], under(a.top_grad[row * a.K + j], a.grad_out));
        }
    }
    // a row's first lane has what it contributed
    const bool first = lane == 0;
    if (!first) mine = Partial{0.0, 0, 0, 0, 0};
    wave_partial(mine);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        const Partial sum = all_partials<NW>(part);
        Partial& to = a.partial[blockIdx.x];
        publish(&to.loss, sum.loss);
        publish(&to.on, sum.on);
        publish(&to.weightless, sum.weightless);
        publish(&to.empty, sum.empty);
        publish(&to.status, sum.status);
    }
    if (!last_workgroup(a.flags, gridDim.x)) return;
    // all sums in a fixed order: lanes over workgroups, then lanes, then waves
    Partial q = {0.0, 0, 0, 0, 0};
    for (unsigned b = threadIdx.x; b < gridDim.x; b += NT) {
        const Partial& from = a.partial[b];
        q.loss += published(&from.loss);
        q.on += published(&from.on);
        q.weightless += published(&from.weightless);
        q.empty += published(&from.empty);
        q.status |= published(&from.status);
    }
    wave_partial(q);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = q;
    __syncthreads();
    if (threadIdx.x == 0) {
        const Partial sum = all_partials<NW>(part);
        *a.loss = (float)(sum.loss * a.inv_D);
        if (a.counters) {
            a.counters[0] = sum.on;
            a.counters[1] = sum.weightless;
            a.counters[2] = sum.empty;
            a.counters[3] = sum.status;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// the gradient
// ---------------------------------------------------------------------------------------------
// rest_coef e^((z - rest_max) / T) of every token: 4 KB of one row per workgroup, the shape in which a read-and-write stream is
// fastest here.
template <class Tr>
__global__ __launch_bounds__(kThreads) void distill_dense_kernel(const typename Tr::elem* logits, int64_t N, int64_t row_stride, int32_t V, float scale,
                                                                 const float* rest_max, const float* rest_coef, float grad_out,
                                                                 const float* grad_scale, typename Tr::elem* dlogits)
{
    const int64_t row = (int64_t)blockIdx.z * kRowsPerGridY + blockIdx.y;
    if (row >= N) return;
    const RestGradient grad(under(rest_coef[row], grad_scale ? *grad_scale * grad_out : grad_out), rest_max[row], scale);
    const int i = (int)blockIdx.x * kThreads + (int)threadIdx.x;
    u32x4 o = {0u, 0u, 0u, 0u};
    if (!grad.none) o = grad.template of<Tr>(load_vector<Tr>(logits + row * row_stride, V, i));
    store_vector<Tr>(dlogits + row * row_stride, V, i, o);
}

template <class Tr>
__global__ __launch_bounds__(kThreads) void distill_top_kernel(const int32_t* ids, const float* top_grad, int64_t N, int64_t row_stride, int32_t V,
                                                               int32_t K, float grad_out, const float* grad_scale, typename Tr::elem* dlogits)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= N * K) return;
    store_top<Tr>(dlogits + (i / K) * row_stride, V, ids[i], under(top_grad[i], grad_scale ? *grad_scale * grad_out : grad_out));
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct Layout {
    size_t target, partial, flags, pending, slots, total;
    ClusterShape shape;         // vectors per thread, pieces per row
    int threads;                // of a piece's workgroup
    bool cooperative;           // a wave can poll a row's pieces
};

Layout layout_of(int64_t N, int64_t V, int32_t dt)
{
    Layout l;
    const int64_t E = dt == ULORL_F32 ? 4 : 8, all = (V + E - 1) / E;
    l.shape = cluster_shape(all * E, dt);
    l.threads = kThreads;
    if (all <= kWaveRow && N >= kManyRows) {
        l.threads = 64;
        l.shape = ClusterShape{all <= kWaveRow / 2 ? 4 : 8, 1};
    }
    l.cooperative = l.shape.pieces > 0;
    if (l.shape.pieces == 0) {                      // more than 64 pieces: no limit to the two-pass path
        l.shape.vpt = 15;
        l.shape.pieces = (int)((all + kThreads * 15 - 1) / (kThreads * 15));
    }
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    size_t off = 0;
    l.flags = off;   off += 256;
    l.partial = off; off = up(off + sizeof(Partial) * kFinishGroups);
    l.target = off;  off = up(off + sizeof(RowTarget) * (size_t)N);
    l.pending = off; off = up(off + sizeof(unsigned long long) * (size_t)N);
    l.slots = off;   off = up(off + 16 * (size_t)N * (size_t)l.shape.pieces);
    l.total = off;
    return l;
}

bool temperature_ok(float t) { return t >= 1.0e-3f && t <= 1.0e3f; }

int32_t check_distill(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t& row_stride, const int32_t* ids, int32_t K)
{
    row_stride = row_stride_of(N, V, row_stride);
    const int32_t rc = check_logits(logits, dt, N, V, row_stride);
    if (rc != ULORL_OK) return rc;
    if (N > kMaxDistillRows || K < 1 || K > kMaxK) return ULORL_ERR_SHAPE;
    return ids ? ULORL_OK : ULORL_ERR_NULL;
}

// The stream over the logits: with dlogits and a spin limit the one-call kernel, else the sums alone.
template <class Tr>
bool launch_stream(const Layout& l, const void* logits, void* dlogits, const DistillArgs& a, hipStream_t st)
{
    using elem = typename Tr::elem;
    // x: piece (fastest, so a row's pieces have consecutive linear ids), y/z: row
    const dim3 grid = rows_grid((unsigned)a.C, a.N);
    auto launch = [&](auto vpt, auto nt) {
        constexpr int VPT = decltype(vpt)::value, NT = decltype(nt)::value;
        if (a.spin_limit > 0)
            hipLaunchKernelGGL((distill_row_kernel<Tr, VPT, NT>), grid, dim3(NT), 0, st, (const elem*)logits, (elem*)dlogits, a);
        else
            hipLaunchKernelGGL((distill_piece_kernel<Tr, VPT, NT>), grid, dim3(NT), 0, st, (const elem*)logits, a);
        return true;
    };
#define ULORL_CASE(VPT_, NT_) \
    if (l.shape.vpt == VPT_ && l.threads == NT_) return launch(std::integral_constant<int, VPT_>{}, std::integral_constant<int, NT_>{});
    ULORL_CASE(4, 64) ULORL_CASE(8, 64)
    ULORL_CASE(4, kThreads) ULORL_CASE(8, kThreads) ULORL_CASE(13, kThreads) ULORL_CASE(15, kThreads)
    if constexpr (Tr::kPerVec == 8) {
        ULORL_CASE(6, kThreads) ULORL_CASE(7, kThreads) ULORL_CASE(11, kThreads)
    } else {
        ULORL_CASE(20, kThreads)
    }
#undef ULORL_CASE
    return false;
}

template <class Tr>
void launch_dense(const void* logits, int64_t N, int64_t V, int64_t row_stride, float scale, const float* rest_max, const float* rest_coef,
                  float grad_out, const float* grad_scale, void* dlogits, hipStream_t st)
{
    const int64_t all = (V + Tr::kPerVec - 1) / Tr::kPerVec;
    hipLaunchKernelGGL((distill_dense_kernel<Tr>), rows_grid((unsigned)((all + kThreads - 1) / kThreads), N), dim3(kThreads), 0, st,
                       (const typename Tr::elem*)logits, N, row_stride, (int32_t)V, scale, rest_max, rest_coef, grad_out, grad_scale,
                       (typename Tr::elem*)dlogits);
}

template <class Tr>
void launch_top(int64_t N, int64_t V, int64_t row_stride, const int32_t* ids, int32_t K, const float* top_grad, float grad_out,
                const float* grad_scale, void* dlogits, hipStream_t st)
{
    hipLaunchKernelGGL((distill_top_kernel<Tr>), dim3((unsigned)((N * K + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, ids, top_grad, N,
                       row_stride, (int32_t)V, K, grad_out, grad_scale, (typename Tr::elem*)dlogits);
}

// The forward call, and with dlogits the gradient too.
template <class Tr>
int32_t enqueue(const void* logits, void* dlogits, const Layout& l, DistillArgs a, hipStream_t st)
{
    using elem = typename Tr::elem;
    a.own_target = a.C == 1 || (a.spin_limit == 0 && a.N * a.C <= kFewPieces);
    const int L = lanes_of(a.K);
    auto with_lanes = [&](const auto& f) {
        if (L == 16) f(std::integral_constant<int, 16>{});
        else if (L == 32) f(std::integral_constant<int, 32>{});
        else f(std::integral_constant<int, 64>{});
    };
    auto groups = [&](int threads) { return (a.N * L + threads - 1) / threads; };
    if (!a.own_target) with_lanes([&](auto l_) {
        hipLaunchKernelGGL((distill_target_kernel<decltype(l_)::value>), dim3((unsigned)groups(kThreads)), dim3(kThreads), 0, st, a);
    });
    if (!launch_stream<Tr>(l, logits, dlogits, a, st)) return ULORL_ERR_HIP;
    with_lanes([&](auto l_) {
        auto finish = [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            const int64_t n = groups(NT);
            hipLaunchKernelGGL((distill_finish_kernel<Tr, NT, decltype(l_)::value>), dim3((unsigned)(n < kFinishGroups ? n : kFinishGroups)), dim3(NT), 0,
                               st, (const elem*)logits, (elem*)dlogits, (int32_t)(l.threads * l.shape.vpt), a);
        };
        if (groups(kFinishSmall) <= kFinishGroups) finish(std::integral_constant<int, kFinishSmall>{});
        else finish(std::integral_constant<int, kFinishLarge>{});
    });
    if (dlogits != nullptr && a.spin_limit == 0) {
        launch_dense<Tr>(logits, a.N, a.V, a.row_stride, a.scale, a.rest_max, a.rest_coef, a.grad_out, nullptr, dlogits, st);
        launch_top<Tr>(a.N, a.V, a.row_stride, a.ids, a.K, a.top_grad, a.grad_out, nullptr, dlogits, st);
    }
    return hipGetLastError() == hipSuccess ? ULORL_OK : ULORL_ERR_HIP;
}

int32_t distill_args(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t& row_stride, const int32_t* teacher_ids, const float* teacher_logp,
                     int32_t K, const float* weights, const ulorl_distill_params* p, float* loss, float* kl, float* lse, float* rest_max,
                     float* rest_coef, float* top_grad, int64_t* counters, void* workspace, size_t workspace_bytes, Layout& l, DistillArgs& a)
{
    const int32_t rc = check_distill(logits, dt, N, V, row_stride, teacher_ids, K);
    if (rc != ULORL_OK) return rc;
    if (!teacher_logp || !p || !loss || !kl || !lse || !rest_max || !rest_coef || !top_grad) return ULORL_ERR_NULL;
    if (!temperature_ok(p->temperature) || p->tail < ULORL_TAIL_BUCKET || p->tail > ULORL_TAIL_DROP || p->reserved[0] != 0 || p->reserved[1] != 0 ||
        !(p->denominator == p->denominator))
        return ULORL_ERR_PARAM;
    l = layout_of(N, V, dt);
    if (!workspace || ((uintptr_t)workspace & 255u) != 0 || workspace_bytes < l.total) return ULORL_ERR_WORKSPACE;
    char* ws = (char*)workspace;
    a.ids = teacher_ids; a.teacher = teacher_logp; a.weights = weights;
    a.loss = loss; a.kl = kl; a.lse = lse; a.rest_max = rest_max; a.rest_coef = rest_coef; a.top_grad = top_grad; a.counters = counters;
    a.target = (RowTarget*)(ws + l.target);
    a.slots = (unsigned long long*)(ws + l.slots);
    a.partial = (Partial*)(ws + l.partial);
    a.flags = (uint32_t*)(ws + l.flags);
    a.pending = (unsigned long long*)(ws + l.pending);
    a.spin_limit = 0;
    a.grad_out = 1.0f;
    a.N = N; a.row_stride = row_stride; a.V = (int32_t)V; a.K = K; a.C = l.shape.pieces; a.tail = p->tail;
    a.inv_t = 1.0 / (double)p->temperature;
    a.scale = (float)(1.4426950408889634074 * a.inv_t);
    a.inv_D = 1.0 / (p->denominator > 0.0 ? p->denominator : (double)N);
    return ULORL_OK;
}

}  // namespace

extern "C" {

size_t ulorl_distill_workspace_bytes(int64_t N, int64_t V, int32_t dt)
{
    if (!shape_ok(N, V, V) || N > kMaxDistillRows || (dt != ULORL_F32 && dt != ULORL_BF16)) return 0;
    return layout_of(N, V, dt).total;
}

int32_t ulorl_distill_fwd(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t row_stride, const int32_t* teacher_ids,
                          const float* teacher_logp, int32_t K, const float* weights, const ulorl_distill_params* p, float* loss, float* kl,
                          float* lse, float* rest_max, float* rest_coef, float* top_grad, int64_t* counters, void* workspace,
                          size_t workspace_bytes, void* hip_stream)
{
    Layout l;
    DistillArgs a;
    const int32_t rc = distill_args(logits, dt, N, V, row_stride, teacher_ids, teacher_logp, K, weights, p, loss, kl, lse, rest_max, rest_coef,
                                    top_grad, counters, workspace, workspace_bytes, l, a);
    if (rc != ULORL_OK) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    return dt == ULORL_BF16 ? enqueue<StoreBF16>(logits, nullptr, l, a, st) : enqueue<StoreF32>(logits, nullptr, l, a, st);
}

int32_t ulorl_distill_bwd(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t row_stride, const int32_t* teacher_ids, int32_t K,
                          float temperature, const float* rest_max, const float* rest_coef, const float* top_grad, float grad_out,
                          const float* grad_scale, void* dlogits, void* hip_stream)
{
    const int32_t rc = check_distill(logits, dt, N, V, row_stride, teacher_ids, K);
    if (rc != ULORL_OK) return rc;
    if (!rest_max || !rest_coef || !top_grad || !dlogits) return ULORL_ERR_NULL;
    if (((uintptr_t)dlogits & 15u) != 0) return ULORL_ERR_ALIGN;
    if (!temperature_ok(temperature)) return ULORL_ERR_PARAM;
    const float scale = (float)(1.4426950408889634074 / (double)temperature);
    hipStream_t st = (hipStream_t)hip_stream;
    auto go = [&](auto tr) {
        using Tr = decltype(tr);
        launch_dense<Tr>(logits, N, V, row_stride, scale, rest_max, rest_coef, grad_out, grad_scale, dlogits, st);
        launch_top<Tr>(N, V, row_stride, teacher_ids, K, top_grad, grad_out, grad_scale, dlogits, st);
    };
    if (dt == ULORL_BF16) go(StoreBF16{}); else go(StoreF32{});
    return hipGetLastError() == hipSuccess ? ULORL_OK : ULORL_ERR_HIP;
}

int32_t ulorl_distill_fwd_bwd(const void* logits, int32_t dt, int64_t N, int64_t V, int64_t row_stride, const int32_t* teacher_ids,
                              const float* teacher_logp, int32_t K, const float* weights, const ulorl_distill_params* p, float grad_out,
                              float* loss, float* kl, float* lse, float* rest_max, float* rest_coef, float* top_grad, int64_t* counters,
                              void* dlogits, void* workspace, size_t workspace_bytes, const ulorl_launch* launch, void* hip_stream)
{
    Layout l;
    DistillArgs a;
    int32_t rc = distill_args(logits, dt, N, V, row_stride, teacher_ids, teacher_logp, K, weights, p, loss, kl, lse, rest_max, rest_coef, top_grad,
                              counters, workspace, workspace_bytes, l, a);
    if (rc != ULORL_OK) return rc;
    if (!dlogits) return ULORL_ERR_NULL;
    if (((uintptr_t)dlogits & 15u) != 0) return ULORL_ERR_ALIGN;
    LaunchOpts opts;
    rc = resolve_launch(launch, &opts);
    if (rc != ULORL_OK) return rc;
    if (l.cooperative && !opts.per_row) a.spin_limit = opts.sync_spins;
    a.grad_out = grad_out;
    hipStream_t st = (hipStream_t)hip_stream;
    return dt == ULORL_BF16 ? enqueue<StoreBF16>(logits, dlogits, l, a, st) : enqueue<StoreF32>(logits, dlogits, l, a, st);
}

}  // extern "C"
