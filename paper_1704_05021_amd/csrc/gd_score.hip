// What is done with logits over a vocabulary: log probabilities of given
// tokens with entropy and the top alternatives, the distance to a teacher's top
// logits, and the gradients of both.
//
//   z = scale logits,  lse = log sum_v exp z_v,  p = exp(z - lse)
//   log probability of t: z_t - lse;  entropy H = -sum_v p_v log p_v
//     dz_v = dlogp (1[v = t] - p_v) - dentropy p_v (log p_v + H)
//   teacher: w = softmax(scale teacher) over the K ids that it names
//     loss = sum_j w_j (log w_j - (z_id_j - lse)),  dz_v = dloss (p_v sum_j w_j - sum over j with id_j = v of w_j)
//   dlogits = scale dz
//
// One pass over a row gives its largest logit, the sum of exp(d) and the sum of
// exp(d) d, where d = scale (logit - largest), each thread with a running
// maximum of its own, joined at the end; from these come log p = d - log s and
// H = log s - t / s.  The gradient takes a second pass.  Both are bound by
// memory.  Few long rows are cut into pieces, a block each, whose sums a second
// launch joins.
//
// The largest is taken off before the scale is put on: the difference of equal
// logits is 0 whatever their size and the scale's.  (z - largest z, with either
// product rounded, is 1e30 for the lowest value of binary32 at a scale of 0.7.)
//
// Top alternatives: a row's 64 groups of threads know their largest logits, the
// K-th largest of those is a bound that at least K elements reach, and few more:
// a second look at the row lists what reaches it, and each listed one counts
// those before it.  Where a mask makes very many equal to the bound, a third look
// lists what is above it.

#include <cfloat>
#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_rows.hpp"

namespace gd {

constexpr uint32_t kScoreMaxTop = 64, kScoreMaxTeacher = 256;
constexpr uint32_t kScoreBlocks = 512;       // pieces that few rows are cut into, about
constexpr uint32_t kScorePiece = 4096;       // elements of a piece, at least
constexpr uint32_t kScoreMaxPieces = 64;     // a lane each where they are joined
constexpr uint32_t kScoreTopRoom = 1024;     // alternatives that a row's pieces name, at most
constexpr uint32_t kListRoom = 1024;         // elements that a row's list holds; a row of more is looked through K times
constexpr int kScoreDeep = 2;                // vectors of a thread in a turn; the next turn's are on their way meanwhile

// A share of a row: the largest logit, and the sums of 2^d and of 2^d d, d = rate (logit - largest), rate = scale log2 e.
struct Soft {
    float m, s, t;
};
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }
// 2 to the power of this and of all below is 0 in binary32, and exp of it: farther terms are held there, as 0 times
// infinity is not 0.
constexpr float kFar = -200.0f;
constexpr float kLog2E = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
// The hardware's exponential in every type: scale and log2 e are put on with two roundings, whose share in exp(x) is up to
// |x| 2^-23, 4e-6 where exp(x) is 1e-15 (the library's errs by 1e-7 there).  What counts in sums is near x = 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float exp_fast(float x) { return exp2_fast(x * kLog2E); }

// The largest of three, NaN left out.  (Of fmaxf the compiler makes three instructions for a pair: it quiets both first.)
__device__ __forceinline__ float max_of(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

template <int CTRL, int MASK>
__device__ __forceinline__ float dpp_f32(float v, float none) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, MASK, 0xF, false));
}
// Over the 64 lanes, in every lane and in a fixed order.
template <typename Op>
__device__ __forceinline__ float wave_join(float v, float none, Op op) {
    v = op(v, dpp_f32<0x111, 0xF>(v, none));  // row_shr:1
    v = op(v, dpp_f32<0x112, 0xF>(v, none));  // row_shr:2
    v = op(v, dpp_f32<0x114, 0xF>(v, none));  // row_shr:4
    v = op(v, dpp_f32<0x118, 0xF>(v, none));  // row_shr:8
    v = op(v, dpp_f32<0x142, 0xA>(v, none));  // row_bcast:15, rows 1 and 3
    v = op(v, dpp_f32<0x143, 0xC>(v, none));  // row_bcast:31, rows 2 and 3
    return __uint_as_float(lane_value(__float_as_uint(v), kWave - 1));
}
__device__ __forceinline__ float wave_max_f32(float v) {
    return wave_join(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum_f32(float v) {
    return wave_join(v, -0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ Soft wave_soft(Soft a, float rate) {
    Soft r;
    r.m = wave_max_f32(a.m);
    const float gap = (a.m - reference(r.m)) * rate, f = exp2_fast(gap);
    r.t = wave_sum_f32(f * (a.t + a.s * fmaxf(gap, kFar)));
    r.s = wave_sum_f32(f * a.s);
    return r;
}
// Over the threads of a row; a barrier lies between this and the next use of lds.
template <int WAVES>
__device__ __forceinline__ Soft row_soft(Soft a, float rate, Soft* lds) {
    a = wave_soft(a, rate);
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) lds[wave_index()] = a;
        __syncthreads();
        a = Soft{-INFINITY, 0.0f, 0.0f};
        if (lane_id() < WAVES) a = lds[wave_index() / WAVES * WAVES + lane_id()];
        a = wave_soft(a, rate);
    }
    return a;
}

// Order of alternatives: larger logits first, of equal ones the lower id; zeros are equal whatever their sign, NaN is
// before all numbers.  Keys are unique, above 0 and below 2^64 - 1.
__device__ __forceinline__ uint32_t order_of(float x) {
    const int32_t b = __float_as_int(x + 0.0f);
    return x != x ? 0xFFFFFFFEu : (uint32_t)(b ^ (b >> 31 | (int32_t)0x80000000));
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint64_t key_of_element(uint32_t order, uint32_t id) { return (uint64_t)order << 32 | ~id; }

// What is named in a row or a piece of it, relative to a logit of it: of a token 0, 1 and its own logit; of a teacher the
// sum of w (log w - scale (logit - of)), that of w, and the largest logit that it names.  (Relative to 0, terms of the
// lowest value's size would leave nothing of the logs.)
struct Sight {
    double at, w;
    float of;
    // at, relative to the logit `to`.
    __device__ __forceinline__ double from(float to, float scale) const {
        return w == 0.0 ? at : at + w * (((double)to - (double)of) * (double)scale);
    }
};

// What a row's elements are measured from: log p = scale (logit - ref) - log_s.
struct Level {
    float ref, log_s;
};
// The two numbers that a gradient's call takes it from, of the largest logit and the log of the sum.  As long as they can
// be they are the largest z, rounded, and the log with what that rounding left, so that their sum is lse.  Where
// what it leaves is of any size, they are the logit itself and the log less than -1, which no log of the others is.
__device__ __forceinline__ void put_stats(float* to, float most, float log_s, float scale) {
    const float z = most * scale, rest = isinf(most) ? 0.0f : fmaf(most, scale, -z);
    const bool adds = fabsf(z) < 0x1p24f || rest == 0.0f;  // rest is at most 1/2, or none
    to[0] = adds ? z : most;
    to[1] = adds ? log_s + rest : -1.0f - log_s;
}
__device__ __forceinline__ Level get_stats(const float* from, float scale) {
    const float z = from[0], log_s = from[1];
    if (log_s <= -1.0f && log_s != -INFINITY) return {z, -1.0f - log_s};
    if (isinf(z)) return {z, log_s};
    // where z is past 2^24 it is exact, and so is this quotient
    const float ref = fminf(fmaxf(__fdiv_rn(z, scale), -FLT_MAX), FLT_MAX);
    return {ref, log_s - fmaf(ref, scale, -z)};
}

struct ScoreArgs {
    uint64_t rows;
    uint32_t vocab, pieces, piece;   // pieces of a row and the elements of one
    const void* logits;
    uint64_t stride;
    float scale, rate;               // rate: scale log2 e
    const void* ids;                 // [rows][count]
    uint64_t ids_stride;
    uint32_t count;
    int wide;                        // ids of 64 bits
    const void* teacher;             // [rows][count], or null: the ids are tokens
    uint64_t teacher_stride;
    int teacher_type;
    const float* g;                  // [rows] gradient of the log probability or the loss
    const float* h;                  // [rows] gradient of the entropy, or null
    const float* given;              // [rows][2] stats of a forward call, or null
    const float* given_entropy;      // [rows]
    void* dlogits;
    uint64_t dstride;
    float* out;                      // [rows] log probability or loss, or null
    float* entropy;                  // [rows], or null
    float* stats;                    // [rows][2], or null
    float* top_logp;                 // [rows][top]
    int64_t* top_id;
    uint32_t top;
    Soft* part;                      // [rows][pieces]
    Sight* part_sight;               // [rows][pieces]
    uint64_t* part_key;              // [rows][pieces][top]
};

// A row or a piece of it as vectors of eight; `mine` has a bit for each element that is this vector's: the last one of a
// ragged piece ends with it, and what it shares with the one before is left out.
struct Vec {
    uint32_t at, mine;
    __device__ __forceinline__ Vec(uint32_t v, uint32_t vecs, uint32_t n) {
        const uint32_t e = min(v, vecs - 1) * 8;
        at = n >= 8 ? min(e, n - 8) : 0;
        mine = v >= vecs ? 0 : n >= 8 ? 0xFFu << (e - at) & 0xFF : (1u << n) - 1;
    }
    template <typename T>
    __device__ __forceinline__ Pack<T, 8> load(const T* p, uint32_t n) const {
        if (n >= 8) return load_pack<8>(p + at);  // the same for every thread
        Pack<T, 8> r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = p[min((uint32_t)j, n - 1)];
        return r;
    }
};

// A row or a piece in turns of kScoreDeep vectors a thread: `whole` of them, in which every vector is, and what is left.
template <typename T, int ROW>
struct Turns {
    typedef Pack<T, 8> Turn[kScoreDeep];
    static constexpr uint32_t kVectors = ROW * kScoreDeep;
    const T* x;
    uint32_t t, n, vecs, whole;
    __device__ __forceinline__ Turns(const T* x, uint32_t t, uint32_t n) : x(x), t(t), n(n), vecs((n + 7) / 8), whole(n / (kVectors * 8)) {}
    __device__ __forceinline__ uint32_t vector(uint32_t turn, int k) const { return turn * kVectors + k * ROW + t; }
    __device__ __forceinline__ void load(Turn& raw, uint32_t turn) const {
#pragma unroll
        for (int k = 0; k < kScoreDeep; ++k) raw[k] = load_pack<8>(x + vector(turn, k) * 8);
    }
    __device__ __forceinline__ bool left() const { return whole * kVectors * 8 < n; }
    __device__ __forceinline__ Vec left_vec(int k) const { return Vec(vector(whole, k), vecs, n); }
    __device__ __forceinline__ void load_left(Turn& raw) const {
#pragma unroll
        for (int k = 0; k < kScoreDeep; ++k) raw[k] = left_vec(k).load(x, n);
    }
    // each(raw, turn) for the whole turns from `first` on, the next one's loads on their way meanwhile
    template <typename Each>
    __device__ __forceinline__ void walk(uint32_t first, Each each) const {
        if (first >= whole) return;
        Turn raw, next;
        load(next, first);
#pragma unroll 1
        for (uint32_t i = first; i < whole; ++i) {
#pragma unroll
            for (int k = 0; k < kScoreDeep; ++k) raw[k] = next[k];
            if (i + 1 < whole) load(next, i + 1);
            each(raw, i);
        }
    }
};

// What the gradient at an element takes: dz = p (c + e (log p + H)), both with the scale in them.
struct Slope {
    Level level;
    float c, e, entropy, c_s;  // c_s: c over the sum
    __device__ __forceinline__ float plain(float x, float rate) const { return exp2_fast((x - level.ref) * rate) * c_s; }
    __device__ __forceinline__ float at(float x, float scale) const {
        const float lp = fmaf(x - level.ref, scale, -level.log_s);  // log p
        return exp_fast(lp) * fmaf(e, fmaxf(lp, kFar) + entropy, c);
    }
};

__device__ __forceinline__ int64_t id_at(const ScoreArgs& a, uint64_t row, uint32_t j) {
    const uint64_t k = row * a.ids_stride + j;
    const int64_t v = a.wide ? ((const int64_t*)a.ids)[k] : (int64_t)((const int32_t*)a.ids)[k];
    return v >= 0 && v < (int64_t)a.vocab ? v : -1;
}
__device__ __forceinline__ float teacher_at(const ScoreArgs& a, uint64_t row, uint32_t j) {
    const uint64_t k = row * a.teacher_stride + j;
    return a.teacher_type == GD_F32    ? ((const float*)a.teacher)[k]
           : a.teacher_type == GD_BF16 ? (float)((const bf16*)a.teacher)[k]
                                       : (float)((const f16*)a.teacher)[k];
}

// A teacher's row, by one wave: the ids that lie in this piece, the logits there and the weights; `held` is the sum of
// all weights, 1, or 0 where the teacher names nothing.  What is seen of them is formed where it is asked for: not where the
// row's sums are given.
struct Named {
    float w[kScoreMaxTeacher], x[kScoreMaxTeacher];
    uint32_t id[kScoreMaxTeacher];  // within the piece, or kNotHere
    Sight sight;
    float held;
};
constexpr uint32_t kNotHere = 0xFFFFFFFFu;
template <typename T>
__device__ __forceinline__ void name_teacher(const ScoreArgs& a, uint64_t row, uint32_t begin, uint32_t n, const T* x, bool seen, Named& to) {
    constexpr int kEach = kScoreMaxTeacher / kWave;
    const uint32_t lane = lane_id();
    float w[kEach], most = -INFINITY, sum = 0.0f;
    uint32_t here[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t j = i * kWave + lane;
        w[i] = -INFINITY;
        here[i] = kNotHere;
        if (i * kWave >= (int)a.count) continue;
        const int64_t v = j < a.count ? id_at(a, row, j) : -1;
        if (v >= 0) {
            w[i] = teacher_at(a, row, j);
            if ((uint64_t)v - begin < n) here[i] = (uint32_t)v - begin;
        }
        most = fmaxf(most, w[i]);
    }
    most = reference(wave_max_f32(most));
#pragma unroll
    for (int i = 0; i < kEach; ++i) w[i] = (w[i] - most) * a.scale, sum += expf(w[i]);
    sum = wave_sum_f32(sum);
    const float log_sum = logf(sum);
    float weight[kEach], v[kEach], of = -INFINITY;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        weight[i] = sum == 0.0f ? 0.0f : expf(w[i]) / sum;
        v[i] = here[i] != kNotHere ? (float)x[here[i]] : 0.0f;
        if (here[i] != kNotHere && weight[i] != 0.0f) of = fmaxf(of, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t j = i * kWave + lane;
        if (j < a.count) to.w[j] = weight[i], to.x[j] = v[i], to.id[j] = here[i];
    }
    if (lane == 0) to.held = sum > 0.0f ? 1.0f : sum;
    if (!seen) return;
    of = reference(wave_max_f32(of));
    Sight sight{0.0, 0.0, of};
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (here[i] != kNotHere && weight[i] != 0.0f) {
            sight.at += (double)weight[i] * ((double)(w[i] - log_sum) - ((double)v[i] - (double)of) * (double)a.scale);
            sight.w += (double)weight[i];
        }
    sight.at = wave_sum(sight.at);
    sight.w = wave_sum(sight.w);
    if (lane == 0) to.sight = sight;
}

// What a row comes to: the token's log probability or the teacher's loss, its entropy and its sums.  at and w: of what is
// named, relative to the largest logit; weights as rounded, whose sum is not quite 1.
template <bool TEACHER>
__device__ __forceinline__ void put_row(const ScoreArgs& a, uint64_t row, const Soft& soft, double at, double w, bool held) {
    const float log_s = logf(soft.s);
    const bool none = soft.m == -INFINITY && soft.s == 0.0f;  // every logit is minus infinity
    if (a.out) {
        const double v = TEACHER ? at + w * (double)log_s : -at - (double)log_s;
        a.out[row] = !held ? 0.0f : none ? (TEACHER ? INFINITY : -INFINITY) : (float)v;
    }
    if (a.entropy) a.entropy[row] = none ? 0.0f : log_s - soft.t / soft.s * kLn2;
    if (a.stats) put_stats(a.stats + row * 2, soft.m, log_s, a.scale);
}

// The alternatives of a row or a piece, from the largest element of every thread.
template <typename T, int WAVES>
struct Alternatives {
    using S = NormShape<WAVES>;
    uint32_t group[S::kThreads / kWave][kWave], bound[S::kRows], n[S::kRows];
    uint64_t list[S::kRows][kListRoom], best[S::kThreads / kWave];

    // largest: this thread's, NaN left out.  odd: the row holds a NaN or plus infinity.
    template <typename Put>
    __device__ __forceinline__ void find(const T* x, uint32_t begin, uint32_t len, uint32_t K, float largest, bool on, bool odd,
                                         Put put) {
        const uint32_t t = threadIdx.x % S::kRow, r = threadIdx.x / S::kRow;
        const uint32_t wave = wave_index(), wave0 = wave / WAVES * WAVES;
        const auto row_sync = [] {  // a row's threads, whose paths may part from other rows' of the block
            if constexpr (WAVES > 1)
                __syncthreads();
            else
                wave_lds_sync();
        };
        // the bound: the K-th largest of 64 groups of threads
        group[wave][lane_id()] = order_of(largest);
        row_sync();
        if (t < (uint32_t)kWave) {
            uint32_t mine = 0, before = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mine = max(mine, group[wave0 + w][lane_id()]);
#pragma unroll
            for (int l = 0; l < kWave; ++l) {
                const uint32_t other = lane_value(mine, l);
                before += other > mine || (other == mine && l < lane_id());
            }
            if (before == K - 1) bound[r] = mine;
        }
        row_sync();
        const float least = value_of(bound[r]);
        const Turns<T, S::kRow> turns(x, t, len);
        // Lists what is above the bound, and with `equal` what equals it; how many there are.
        const auto look = [&](bool equal) {
            if (t == 0) n[r] = 0;
            row_sync();
            // one look a vector: hardly any holds an element to list
            const auto at_vector = [&](const Pack<T, 8>& raw, uint32_t at, uint32_t mine) {
                float v[8], top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = (float)raw.v[j];
#pragma unroll
                for (int j = 0; j < 8; j += 2) top = max_of(top, v[j], v[j + 1]);
                if (!(equal ? top >= least : top > least)) return;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if ((equal ? v[j] >= least : v[j] > least) && mine >> j & 1) {
                        const uint32_t place = atomicAdd(&n[r], 1u);
                        if (place < kListRoom) list[r][place] = key_of_element(order_of(v[j]), begin + at + j);
                    }
            };
            turns.walk(0, [&](const typename Turns<T, S::kRow>::Turn& raw, uint32_t turn) {
#pragma unroll
                for (int k = 0; k < kScoreDeep; ++k) at_vector(raw[k], turns.vector(turn, k) * 8, 0xFF);
            });
            if (turns.left()) {
                typename Turns<T, S::kRow>::Turn raw;
                turns.load_left(raw);
#pragma unroll
                for (int k = 0; k < kScoreDeep; ++k) at_vector(raw[k], turns.left_vec(k).at, turns.left_vec(k).mine);
            }
            row_sync();
            const uint32_t listed = n[r];
            row_sync();
            return listed;
        };
        if (!on) return;
        if (!odd) {
            uint32_t listed = look(true);
            // very many equal the bound (what a mask puts in its places): those above it, and behind them its first ones
            const bool many = listed > kListRoom;
            if (many) listed = look(false);
            if (listed <= kListRoom) {
                for (uint32_t i = t; i < listed; i += S::kRow) {
                    const uint64_t key = list[r][i];
                    uint32_t rank = 0;
                    for (uint32_t k = 0; k < listed; ++k) rank += list[r][k] > key;
                    if (rank < K) put(rank, key);
                }
                if (many && t < (uint32_t)kWave)  // in order of their ids, 64 elements at a time
                    for (uint32_t e = 0, found = listed; e < len && found < K; e += kWave) {
                        const bool here = e + t < len && (float)x[min(e + t, len - 1)] == least;
                        const uint64_t m = ballot(here);
                        const uint32_t rank = found + lanes_below(m);
                        if (here && rank < K) put(rank, key_of_element(order_of(least), begin + e + t));
                        found += popc64(m);
                    }
                if (!many)
                    for (uint32_t k = len + t; k < K; k += S::kRow) put(k, 0);  // a piece of fewer elements than K
                return;
            }
        }
        // Very many are above the bound (all of a few groups'), or not all are in order: the next largest, K times.
        uint64_t last = ~0ull;
        for (uint32_t k = 0; k < K; ++k) {
            uint64_t most = 0;
            for (uint32_t e = t; e < len; e += S::kRow) {
                const uint64_t key = key_of_element(order_of((float)x[e]), begin + e);
                most = key < last ? max(most, key) : most;
            }
            for (int d = kWave / 2; d; d /= 2) most = max(most, (uint64_t)__shfl_xor((unsigned long long)most, d));
            if constexpr (WAVES > 1) {
                if (lane_id() == 0) best[wave] = most;
                __syncthreads();
                most = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) most = max(most, best[w]);
                __syncthreads();
            }
            if (t == 0) put(k, most);
            last = most;
        }
    }
};
struct Nothing {};

enum ScoreKind { kSums = 0, kTop = 1, kGrad = 2, kGradEntropy = 3 };  // kGrad: no entropy is asked for, nor its gradient given
template <typename T, int WAVES, int KIND, bool TEACHER, int HELD = 0>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_score(ScoreArgs a, uint32_t first_unit) {
    using S = NormShape<WAVES>;
    __shared__ Soft lds_soft[S::kThreads / kWave];
    __shared__ std::conditional_t<TEACHER, Named, Nothing> named[S::kRows];
    __shared__ std::conditional_t<KIND == kTop, Alternatives<T, WAVES>, Nothing> top;
    static_assert(WAVES == 1 || S::kRows == 1);  // barriers are a row's own
    const uint32_t t = threadIdx.x % S::kRow, r = threadIdx.x / S::kRow, units = (uint32_t)a.rows * a.pieces;
    const bool on = blockIdx.x * S::kRows + r < units - first_unit;
    const uint32_t unit = on ? first_unit + blockIdx.x * S::kRows + r : units - 1;
    const uint32_t piece = unit % a.pieces, begin = piece * a.piece, n = min(a.vocab - begin, a.piece), vecs = (n + 7) / 8;
    const uint64_t row = unit / a.pieces;
    const T* x = (const T*)a.logits + row * a.stride + begin;
    const float scale = a.scale, rate = a.rate;
    constexpr bool GRAD = KIND >= kGrad;
    const bool stats = !GRAD || !a.given;  // the row's sums are formed here

    // the token and its logit, read before anything is written over it; a teacher's by the row's first wave
    int64_t token = -1;
    float token_x = 0.0f;
    if constexpr (TEACHER) {
        if (t < (uint32_t)kWave) name_teacher(a, row, begin, n, x, stats, named[r]);
    } else {
        token = id_at(a, row, 0);
        if (token >= 0) token_x = (float)((const T*)a.logits + row * a.stride)[token];
    }
    const float g = GRAD ? a.g[row] : 0.0f, e = KIND == kGradEntropy && a.h ? -a.h[row] * scale : 0.0f;
    const bool entropy = KIND == kGradEntropy || (!GRAD && a.entropy);
    // padding with nothing to say of it: its logits are not read
    const bool skip = GRAD && !TEACHER && token < 0 && e == 0.0f && !a.entropy;

    // The gradient's launch holds the row's first turns (HELD over the bytes of an element) and its last in registers
    // between its two passes, and reads the others twice.
    const Turns<T, S::kRow> turns(x, t, n);
    typedef typename Turns<T, S::kRow>::Turn Turn;
    constexpr int kHeld = GRAD ? HELD / (int)sizeof(T) : 0;
    Turn kept[kHeld > 0 ? kHeld : 1], last;
    const uint32_t held_turns = min((uint32_t)kHeld, turns.whole);
    if (!skip) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (i < (int)held_turns) turns.load(kept[i], i);
        if (turns.left()) turns.load_left(last);
    }

    Soft soft{-INFINITY, 0.0f, 0.0f};
    float most = -INFINITY;  // the thread's largest logit
    if (stats && !skip) {
        const auto add = [&](const float (&z)[kScoreDeep][8]) {
#pragma unroll
            for (int k = 0; k < kScoreDeep; ++k)
#pragma unroll
                for (int j = 0; j < 8; j += 2) most = max_of(most, z[k][j], z[k][j + 1]);
            const float to = reference(most), gap = (soft.m - to) * rate, f = exp2_fast(gap);
            float p[kScoreDeep] = {}, tt[kScoreDeep] = {};  // sums of a few, side by side
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < kScoreDeep; ++k) {
                    const float d = (z[k][j] - to) * rate, e = exp2_fast(d);
                    p[k] += e;
                    if (entropy) tt[k] = fmaf(e, fmaxf(d, kFar), tt[k]);
                }
            float ps = 0.0f, ts = 0.0f;
#pragma unroll
            for (int k = 0; k < kScoreDeep; ++k) ps += p[k], ts += tt[k];
            if (entropy) soft.t = f * (soft.t + soft.s * fmaxf(gap, kFar)) + ts;
            soft.s = fmaf(f, soft.s, ps);
            soft.m = most;
        };
        const auto add_whole = [&](const Turn& raw, uint32_t) {
            float z[kScoreDeep][8];
#pragma unroll
            for (int k = 0; k < kScoreDeep; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) z[k][j] = (float)raw[k].v[j];
            add(z);
        };
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (i < (int)held_turns) add_whole(kept[i], i);
        turns.walk(held_turns, add_whole);
        if (turns.left()) {
            float z[kScoreDeep][8];
#pragma unroll
            for (int k = 0; k < kScoreDeep; ++k) {
                const uint32_t mine = turns.left_vec(k).mine;
#pragma unroll
                for (int j = 0; j < 8; ++j) z[k][j] = mine >> j & 1 ? (float)last[k].v[j] : -INFINITY;
            }
            add(z);
        }
    }
    if (stats) soft = row_soft<WAVES>(soft, rate, lds_soft);
    if (TEACHER || GRAD) __syncthreads();

    Sight sight{0.0, 0.0, 0.0f};
    float held = 0.0f;
    if constexpr (TEACHER) {
        held = named[r].held;
        if (stats) sight = named[r].sight;
    } else if (token >= 0) {
        held = 1.0f;
        if ((uint64_t)token - begin < n) sight = {0.0, 1.0, token_x};
    }
    if (stats && t == 0 && on) {
        if (a.pieces > 1)
            a.part[unit] = soft, a.part_sight[unit] = sight;
        else
            put_row<TEACHER>(a, row, soft, sight.from(soft.m, scale), sight.w, held != 0.0f);
    }

    if constexpr (KIND == kTop) {
        const uint32_t K = a.top;
        const float log_s = logf(soft.s);
        top.find(x, begin, n, K, most, on, soft.s != soft.s, [&](uint32_t rank, uint64_t key) {
            if (!on) return;
            if (a.pieces > 1) {
                a.part_key[(uint64_t)unit * K + rank] = key;
            } else {
                const float lp = fmaf(value_of((uint32_t)(key >> 32)) - soft.m, scale, -log_s);
                a.top_logp[row * K + rank] = soft.m == -INFINITY && log_s == -INFINITY ? -INFINITY : lp;
                a.top_id[row * K + rank] = (int64_t)(uint32_t)~(uint32_t)key;
            }
        });
    }
    if constexpr (GRAD) {
        Slope sl;
        sl.level = stats ? Level{soft.m, logf(soft.s)} : get_stats(a.given + row * 2, scale);
        sl.entropy = stats ? sl.level.log_s - soft.t / soft.s * kLn2 : a.given_entropy ? a.given_entropy[row] : 0.0f;
        sl.c = held == 0.0f ? 0.0f : (TEACHER ? g : -g) * held * scale;
        sl.e = e;
        sl.c_s = sl.c / (stats ? soft.s : expf(sl.level.log_s));
        T* d = (T*)a.dlogits + row * a.dstride + begin;
        // a row that no gradient comes down to has none, whatever it holds, nor has one of which every logit is minus infinity
        const bool zeros = (sl.c == 0.0f && sl.e == 0.0f) || (sl.level.ref == -INFINITY && sl.level.log_s == -INFINITY);
        const auto write = [&](auto value) {  // of an element
            const auto of = [&](const Pack<T, 8>& raw) {
                Pack<T, 8> y;
#pragma unroll
                for (int j = 0; j < 8; ++j) y.v[j] = (T)value((float)raw.v[j]);
                return y;
            };
            const auto write_whole = [&](const Turn& raw, uint32_t turn) {
#pragma unroll
                for (int k = 0; k < kScoreDeep; ++k) store_stream<8>(d + turns.vector(turn, k) * 8, of(raw[k]), 8);
            };
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (i < (int)held_turns) write_whole(kept[i], i);
            turns.walk(held_turns, write_whole);
            if (!turns.left()) return;
#pragma unroll
            for (int k = 0; k < kScoreDeep; ++k) {
                const Vec p = turns.left_vec(k);
                const Pack<T, 8> y = of(last[k]);
                if (p.mine == 0xFF)
                    store_stream<8>(d + p.at, y, 8);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (p.mine >> j & 1) d[p.at + j] = y.v[j];
            }
        };
        if (on && zeros) {
            for (uint32_t v = t; v < vecs; v += S::kRow) store_stream<8>(d + v * 8, Pack<T, 8>{}, (int)(n - v * 8));
        } else if (on) {
            if constexpr (KIND == kGradEntropy)
                write([&](float v) { return sl.at(v, scale); });
            else
                write([&](float v) { return sl.plain(v, rate); });
        }
        // the elements that are named are written anew, with their weights in them and rounded once, behind the others
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (zeros || !on) return;
        if constexpr (TEACHER) {
            const Named& q = named[r];
            for (uint32_t j = t; j < a.count; j += S::kRow) {
                const uint32_t id = q.id[j];
                if (id == kNotHere) continue;
                float w = 0.0f;
                bool first = true;
                for (uint32_t k = 0; k < a.count; ++k)
                    if (q.id[k] == id) {
                        first = first && k >= j;
                        w += q.w[k];
                    }
                if (first) d[id] = (T)(sl.plain(q.x[j], rate) - g * w * scale);
            }
        } else if (t == 0 && token >= 0 && (uint64_t)token - begin < n) {
            d[(uint64_t)token - begin] = (T)((KIND == kGradEntropy ? sl.at(token_x, scale) : sl.plain(token_x, rate)) + g * scale);
        }
    }
}

// Joins the pieces of a row, a lane each; with alternatives their lists, each sorted.
constexpr int kScoreJoinThreads = 256;
template <bool TEACHER>
__global__ __launch_bounds__(kScoreJoinThreads) void k_score_join(ScoreArgs a) {
    __shared__ uint64_t keys[kScoreTopRoom];
    const uint64_t row = blockIdx.x;
    const uint32_t lane = lane_id();
    Soft soft{-INFINITY, 0.0f, 0.0f};
    Sight sight{0.0, 0.0, 0.0f};
    if (lane < a.pieces) soft = a.part[row * a.pieces + lane], sight = a.part_sight[row * a.pieces + lane];
    bool held = false;  // whether a token is there, or a teacher's logit above minus infinity (NaN is one)
    for (uint32_t j = lane; j < a.count; j += kWave)
        held = held || (id_at(a, row, j) >= 0 && (!TEACHER || !(teacher_at(a, row, j) == -INFINITY)));
    held = ballot(held) != 0;
    soft = wave_soft(soft, a.rate);
    const double at = wave_sum(sight.from(soft.m, a.scale)), w = wave_sum(sight.w);
    if (threadIdx.x == 0) put_row<TEACHER>(a, row, soft, at, w, held);
    if (!a.top) return;
    const float log_s = logf(soft.s);
    const uint32_t all = a.pieces * a.top;
    for (uint32_t i = threadIdx.x; i < all; i += kScoreJoinThreads) keys[i] = a.part_key[row * all + i];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < all; i += kScoreJoinThreads) {
        const uint64_t key = keys[i];
        uint32_t rank = 0;
        for (uint32_t k = 0; k < all; ++k) rank += keys[k] > key;
        if (rank >= a.top || key == 0) continue;
        const float lp = fmaf(value_of((uint32_t)(key >> 32)) - soft.m, a.scale, -log_s);
        a.top_logp[row * a.top + rank] = soft.m == -INFINITY && log_s == -INFINITY ? -INFINITY : lp;
        a.top_id[row * a.top + rank] = (int64_t)(uint32_t)~(uint32_t)key;
    }
}

// Calls f(grid, first unit) until all units are covered: a dispatch holds less than 2^32 threads.
template <int WAVES, typename F>
hipError_t over_units(const ScoreArgs& a, F f) {
    using S = NormShape<WAVES>;
    const uint32_t units = (uint32_t)a.rows * a.pieces;
    constexpr uint32_t kMost = 1u << 22;
    for (uint32_t first = 0; first < units; first += std::min(units - first, kMost)) {
        f(dim3((std::min(units - first, kMost) + S::kRows - 1) / S::kRows), dim3(S::kThreads), first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T, int WAVES>
hipError_t launch_sums(const ScoreArgs& a, hipStream_t st) {
    return over_units<WAVES>(a, [&](dim3 grid, dim3 block, uint32_t first) {
        if (a.teacher)
            k_score<T, WAVES, kSums, true><<<grid, block, 0, st>>>(a, first);
        else if (a.top)
            k_score<T, WAVES, kTop, false><<<grid, block, 0, st>>>(a, first);
        else
            k_score<T, WAVES, kSums, false><<<grid, block, 0, st>>>(a, first);
    });
}
template <typename T, int WAVES, int HELD>
hipError_t launch_gradient(const ScoreArgs& a, hipStream_t st) {
    return over_units<WAVES>(a, [&](dim3 grid, dim3 block, uint32_t first) {
        if (a.teacher)
            k_score<T, WAVES, kGrad, true, HELD><<<grid, block, 0, st>>>(a, first);
        else if (a.h || a.entropy)
            k_score<T, WAVES, kGradEntropy, false, HELD><<<grid, block, 0, st>>>(a, first);
        else
            k_score<T, WAVES, kGrad, false, HELD><<<grid, block, 0, st>>>(a, first);
    });
}
// Waves of a row, and turns that the gradient's launch holds.  Up to 8,192 elements one wave a row does best, as no
// barrier stands between its passes (gradient of 20,000 x 4,000 in bfloat16: 79 us, with four waves 186; of 9,000 x
// 8,000 63 and 75; of 5,000 x 16,000 80 and 69), where there are rows enough to fill the chip so.  Turns held spare a
// second reading but leave room for fewer waves: 3,000 x 85,000 take 220 us with six turns of four waves, 241 with two;
// 2,400 x 42,000 73 and 83, but 2,400 x 30,000 52 and 58 and 2,400 x 38,000 64 and 75: of bfloat16 the border could lie
// lower, between those and 5,000 x 16,000 (83 and 69).  Of 2,400 rows in binary32, 15,000 take 56 and 59, 25,000 101 and
// 109.  Four waves in place of eight take 248 and 262.
// The sums alone by four waves and by eight: 600 x 70,000 in bfloat16 20 and 22 us, 600 x 90,000 25 and 27, 600 x 110,000 29
// and 31, 600 x 200,000 47 and 48; in binary32 600 x 45,000 21 and 21, 600 x 60,000 26 and 26.
template <typename T>
hipError_t launch_score_type(const ScoreArgs& a, bool grad, hipStream_t st) {
    const uint32_t n = std::min(a.vocab, a.piece);
    if (grad) {
        if (n <= 2048 || (n <= 8192 && a.rows * a.pieces >= 1024)) return launch_gradient<T, 1, 4>(a, st);
        if (n <= 80'000 / sizeof(T)) return launch_gradient<T, 4, 4>(a, st);
        return launch_gradient<T, 4, 12>(a, st);
    }
    if (n <= 2048 || (n <= 8192 && a.rows * a.pieces >= 1024)) return launch_sums<T, 1>(a, st);
    if (n <= 200'000 / sizeof(T)) return launch_sums<T, 4>(a, st);
    return launch_sums<T, 8>(a, st);
}
hipError_t launch_score(const ScoreArgs& a, int type, bool grad, hipStream_t st) {
    return with_type(type, [&](auto zero) { return launch_score_type<decltype(zero)>(a, grad, st); });
}

// Cuts few long rows into pieces.
void cut(ScoreArgs& a) {
    uint32_t pieces = 1;
    if (a.rows && a.rows < kScoreBlocks / 2 && a.vocab >= 2 * kScorePiece)
        pieces = std::min({(uint32_t)(kScoreBlocks / a.rows), a.vocab / kScorePiece, kScoreMaxPieces,
                           a.top ? kScoreTopRoom / a.top : kScoreMaxPieces});
    a.piece = ((a.vocab + pieces - 1) / pieces + 7) / 8 * 8;
    a.pieces = (a.vocab + a.piece - 1) / a.piece;
}

// The scratch of a plan, shared by both operators: what pieces of few rows are joined from.
struct ScorePlan {
    int device = 0;
    uint32_t vocab = 0;
    int type = GD_F32;
    uint64_t max_rows = 0;
    Soft* part = nullptr;
    Sight* part_sight = nullptr;
    uint64_t* part_key = nullptr;
    float* stats = nullptr;    // of a call whose gradient takes a launch of its own
    float* entropy = nullptr;
    DeviceMemory mem;

    gd_status create(uint32_t words, int ty, uint64_t rows, bool top) {
        vocab = words, type = ty, max_rows = rows;
        if (hipGetDevice(&device) != hipSuccess) return GD_ERR_HIP;
        const bool ok = mem.alloc(&part, kScoreBlocks) && mem.alloc(&part_sight, kScoreBlocks) &&
                        (!top || mem.alloc(&part_key, (size_t)kScoreBlocks * kScoreMaxTop)) &&
                        mem.alloc(&stats, kScoreBlocks) && mem.alloc(&entropy, kScoreBlocks / 2);
        return ok ? GD_OK : GD_ERR_OOM;
    }
    ScoreArgs args(float scale) const {
        ScoreArgs a{};
        a.vocab = vocab;
        a.scale = scale;
        a.rate = std::min(scale * kLog2E, FLT_MAX);  // not infinity: 0 times that is not 0
        a.part = part, a.part_sight = part_sight, a.part_key = part_key;
        return a;
    }
    gd_status forward(ScoreArgs a, hipStream_t st) const {
        cut(a);
        if (launch_score(a, type, false, st) != hipSuccess) return GD_ERR_HIP;
        if (a.pieces == 1) return GD_OK;
        if (a.teacher)
            k_score_join<true><<<dim3((uint32_t)a.rows), dim3(kScoreJoinThreads), 0, st>>>(a);
        else
            k_score_join<false><<<dim3((uint32_t)a.rows), dim3(kScoreJoinThreads), 0, st>>>(a);
        return hipGetLastError() == hipSuccess ? GD_OK : GD_ERR_HIP;
    }
    // with a.given null the row's sums are formed here: in the launch that writes the gradient, or for rows in pieces before it
    gd_status backward(ScoreArgs a, hipStream_t st) const {
        cut(a);
        if (a.pieces > 1 && !a.given) {
            ScoreArgs f = a;
            f.stats = stats;
            float* const wanted = a.entropy;
            if (a.h && !wanted) f.entropy = entropy;
            const gd_status s = forward(f, st);
            if (s != GD_OK) return s;
            a.given = stats;
            a.given_entropy = f.entropy;
        }
        return launch_score(a, type, true, st) == hipSuccess ? GD_OK : GD_ERR_HIP;
    }
};

inline bool bad_scale(float s) { return !(s > 0.0f) || std::isinf(s); }

}  // namespace gd

struct gd_logprob {
    gd::ScorePlan plan;
};
struct gd_distill {
    gd::ScorePlan plan;
};

namespace {

template <typename H>
gd_status create_score(H** out, uint32_t vocab, gd_dtype type, uint64_t max_rows, bool top) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int ty = gd::enum_int(&type);
    if (vocab == 0 || vocab > 0x7FFFFFFFu || max_rows > 0x7FFFFFFFull || ty < GD_F32 || ty > GD_F16) return GD_ERR_ARG;
    H* h = new (std::nothrow) H();
    if (!h) return GD_ERR_OOM;
    gd_status st;
    try {
        st = h->plan.create(vocab, ty, max_rows, top);
    } catch (const std::bad_alloc&) {
        st = GD_ERR_OOM;
    }
    if (st != GD_OK) {
        delete h;
        return st;
    }
    *out = h;
    return GD_OK;
}
template <typename H>
void destroy_score(H* h) {
    if (!h) return;
    gd::DeviceGuard guard(h->plan.device);
    delete h;
}

// The arguments that both calls of a teacher have.
template <typename IO>
gd_status distill_args(const gd_distill* l, const IO* io, gd::ScoreArgs& a) {
    if (!l || !io || io->rows > l->plan.max_rows || gd::bad_scale(io->scale) || io->top == 0 ||
        io->top > gd::kScoreMaxTeacher)
        return GD_ERR_ARG;
    const int wide = gd::enum_int(&io->index), ty = gd::enum_int(&io->teacher_type);
    if (wide < GD_I32 || wide > GD_I64 || ty < GD_F32 || ty > GD_F16) return GD_ERR_ARG;
    if (io->rows && (!io->logits || !io->ids || !io->teacher || io->stride < l->plan.vocab || io->ids_stride < io->top ||
                     io->teacher_stride < io->top))
        return GD_ERR_ARG;
    a = l->plan.args(io->scale);
    a.rows = io->rows;
    a.logits = io->logits;
    a.stride = io->stride;
    a.ids = io->ids;
    a.ids_stride = io->ids_stride;
    a.count = io->top;
    a.wide = wide == GD_I64;
    a.teacher = io->teacher;
    a.teacher_stride = io->teacher_stride;
    a.teacher_type = ty;
    return GD_OK;
}

}  // namespace

extern "C" {

gd_status gd_logprob_create(gd_logprob** out, uint32_t vocab, gd_dtype type, uint64_t max_rows) {
    return create_score(out, vocab, type, max_rows, true);
}
void gd_logprob_destroy(gd_logprob* l) { destroy_score(l); }

gd_status gd_logprob_forward(gd_logprob* l, const gd_logprob_io* io, void* stream) {
    if (!l || !io || io->rows > l->plan.max_rows || gd::bad_scale(io->scale) || io->top > gd::kScoreMaxTop ||
        io->top > l->plan.vocab)
        return GD_ERR_ARG;
    const int wide = gd::enum_int(&io->index);
    if (wide < GD_I32 || wide > GD_I64) return GD_ERR_ARG;
    if (io->rows == 0) return GD_OK;
    if (!io->logits || !io->tokens || io->stride < l->plan.vocab || (io->top && (!io->top_logp || !io->top_id)))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(l->plan.device);
    if (!guard.ok) return GD_ERR_HIP;
    gd::ScoreArgs a = l->plan.args(io->scale);
    a.rows = io->rows;
    a.logits = io->logits;
    a.stride = io->stride;
    a.ids = io->tokens;
    a.ids_stride = a.count = 1;
    a.wide = wide == GD_I64;
    a.out = io->logp;
    a.entropy = io->entropy;
    a.stats = io->stats;
    a.top = io->top;
    a.top_logp = io->top_logp;
    a.top_id = io->top_id;
    return l->plan.forward(a, (hipStream_t)stream);
}

gd_status gd_logprob_backward(gd_logprob* l, const gd_logprob_grad* io, void* stream) {
    if (!l || !io || io->rows > l->plan.max_rows || gd::bad_scale(io->scale)) return GD_ERR_ARG;
    const int wide = gd::enum_int(&io->index);
    if (wide < GD_I32 || wide > GD_I64) return GD_ERR_ARG;
    if (io->rows == 0) return GD_OK;
    if (!io->logits || !io->tokens || !io->dlogits || !io->dlogp || io->stride < l->plan.vocab ||
        io->dlogits_stride < l->plan.vocab || (io->stats && (io->logp_out || io->entropy_out)) ||
        (io->stats && io->dentropy && !io->entropy))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(l->plan.device);
    if (!guard.ok) return GD_ERR_HIP;
    gd::ScoreArgs a = l->plan.args(io->scale);
    a.rows = io->rows;
    a.logits = io->logits;
    a.stride = io->stride;
    a.ids = io->tokens;
    a.ids_stride = a.count = 1;
    a.wide = wide == GD_I64;
    a.g = io->dlogp;
    a.h = io->dentropy;
    a.given = io->stats;
    a.given_entropy = io->entropy;
    a.dlogits = io->dlogits;
    a.dstride = io->dlogits_stride;
    a.out = io->logp_out;
    a.entropy = io->entropy_out;
    return l->plan.backward(a, (hipStream_t)stream);
}

gd_status gd_distill_create(gd_distill** out, uint32_t vocab, gd_dtype type, uint64_t max_rows) {
    return create_score(out, vocab, type, max_rows, false);
}
void gd_distill_destroy(gd_distill* l) { destroy_score(l); }

gd_status gd_distill_forward(gd_distill* l, const gd_distill_io* io, void* stream) {
    gd::ScoreArgs a;
    const gd_status st = distill_args(l, io, a);
    if (st != GD_OK || io->rows == 0) return st;
    gd::DeviceGuard guard(l->plan.device);
    if (!guard.ok) return GD_ERR_HIP;
    a.out = io->loss;
    a.stats = io->stats;
    return l->plan.forward(a, (hipStream_t)stream);
}

gd_status gd_distill_backward(gd_distill* l, const gd_distill_grad* io, void* stream) {
    gd::ScoreArgs a;
    const gd_status st = distill_args(l, io, a);
    if (st != GD_OK || io->rows == 0) return st;
    if (!io->dloss || !io->dlogits || io->dlogits_stride < l->plan.vocab || (io->stats && io->loss_out)) return GD_ERR_ARG;
    gd::DeviceGuard guard(l->plan.device);
    if (!guard.ok) return GD_ERR_HIP;
    a.g = io->dloss;
    a.dlogits = io->dlogits;
    a.dstride = io->dlogits_stride;
    a.given = io->stats;
    a.out = io->loss_out;
    return l->plan.backward(a, (hipStream_t)stream);
}

}  // extern "C"
