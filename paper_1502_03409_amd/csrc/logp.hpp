// What a softmax over a vocabulary answers: log probabilities of given words, the entropy, the likeliest words; and the gradients of the first two.
//
// The scores l = x w^T are never stored.  Each tile of the product leaves, per row, its largest score, the sum of the other words' exponentials
// relative to it, and the sum of those times the distance; and per row and group of 32 words the largest score, its place, and the second
// largest.  A small kernel joins the tiles: with m the largest score, r the sum of exp(l - m) over all words but one that has it, and
// U = sum exp(l - m) (m - l),
//   log sum exp(l) = m + log(1 + r),  H = log(1 + r) + U / (1 + r),
// neither of which cancels where one word has nearly all.
//
// The likeliest words are looked for among the groups: with t at most the K-th largest score, only groups whose largest reaches t hold any, and
// only where the second reaches it too is more than one of 32 a candidate.  Candidates' scores are formed again in 64 bits, and so are those of the
// given words; the order is that of these, equal ones in the vocabulary's order, so it does not hang on how a tile added up.
//
// Gradients: with a, b those of the log probabilities and the entropy, and A = sum of a row's a,
//   d[v] = sum of a over t with word[t] = v - p[v] (A + b (log p[v] + H)),  dx = d w,  dw = d^T x;
// the scores are formed once more, d leaves the product's tiles, given words get theirs in a kernel of its own, where with S the sum of a over a
// word, S - p A = (S - A) - A (p - 1) does not cancel where p is near one.  d meets bf16 operands as in xent.hpp.
//
// 8192 rows of 4096 over 128000 words in bf16, a tenth masked, one word given and ten asked for: scores 6.7 ms, joining 0.03, answers 0.31 (keys of
// 0.24 GB and candidates' weights of 0.9 GB, by workgroups that wait in 83 % of their cycles), d 6.8, dx and dw 6.7 each: four products of 7.7
// TFLOP each, bound as large products are.  One row: scores 201 us, the 1.05 GB of weights at 5.2 TB/s, answers 23.
#pragma once
#include "head_few.hpp"
#include "head_planes.hpp"

namespace lc {
namespace head {

constexpr long long kKeyBytes = 512LL << 20;      // groups' scores kept at a time
constexpr long long kGradBytes = 2LL << 30;       // of d
constexpr int kGroupWords = 32;

// Masked rows of large batches are left out: the others are gathered (count, place and index as in xent.hpp).  Up to kNarrow rows that would cost more
// than it saves, and each row stays where it is: where x is laid out, a masked row of it becomes zeros, so
// that what it holds makes no tile of fp32 planes form its sums again, and backward its d too, and its index -1.
struct LogpRows {
    int *count, *place, *index;   // null: all rows count, where they are
    float4 *sums;                 // by position: largest score, log(1 + r), entropy; 1 where masked
    float *a, *b;                 // by position: A and b
};
__device__ __forceinline__ bool any_given(const int64_t *words, int T) {
    bool any = false;
    for (int t = 0; t < T; ++t) any |= words[t] >= 0;
    return any;
}

// What a row without a word is answered, by a workgroup.
__device__ __forceinline__ void answer_masked(const LogpOut &out, long long n) {
    if (threadIdx.x == 0) {
        if (out.entropy) out.entropy[n] = 0.f;
        if (out.state) out.state[3 * n] = out.state[3 * n + 1] = out.state[3 * n + 2] = 0.f;
    }
    for (int t = threadIdx.x; t < out.T; t += blockDim.x) out.logp[n * out.T + t] = 0.f;
    for (int k = threadIdx.x; k < out.K; k += blockDim.x) out.top[n * out.K + k] = -1, out.top_logp[n * out.K + k] = 0.f;
}

// Positions of the rows that have a word; behind them in the index, from its end, those that have none.  One workgroup, 8192 rows at a time, eight a
// thread.
static __global__ __launch_bounds__(1024) void logp_rows_kernel(const int64_t *tags, int N, int T, LogpRows o) {
    constexpr int EACH = 8;
    __shared__ int part[EACH * 16 + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int total = 0;
    for (int n0 = 0; n0 < N; n0 += 1024 * EACH) {
        unsigned long long mask[EACH];
        bool in[EACH] = {};
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
                const int n = n0 + k * 1024 + (int)threadIdx.x;
                in[k] |= n < N && tags[(long long)min(n, N - 1) * T + t] >= 0;
            }
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            mask[k] = __ballot(in[k]);
            if (lane == 0) part[k * 16 + wave] = __popcll(mask[k]);
        }
        __syncthreads();
        if (wave == 0) {   // sums of all before, 128 of them
            const int a = part[2 * lane], b = part[2 * lane + 1];
            int s = a + b;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(s, d);
                if (lane >= d) s += other;
            }
            part[2 * lane] = s - a - b, part[2 * lane + 1] = s - b;
            if (lane == 63) part[EACH * 16] = s;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int n = n0 + k * 1024 + threadIdx.x, at = total + part[k * 16 + wave] + __popcll(mask[k] & ((1ull << lane) - 1));
            if (n >= N) continue;
            o.place[n] = in[k] ? at : -1;
            o.index[in[k] ? at : N - 1 - (n - at)] = n;
        }
        total += part[EACH * 16];
        __syncthreads();
    }
    if (threadIdx.x == 0) *o.count = total;
}

// The rows that count as planes, zeros in the other rows of dx (nullable); with gradients a row's A and b and what the forward pass left.
struct LogpGiven {
    const int64_t *tags;
    const float *state, *dlogp, *dentropy;
    int T, V;
};
template <typename T, bool GRADS>
__global__ __launch_bounds__(256) void logp_gather_kernel(const T *x, bf16_t *dst, T *dx, LogpRows o, LogpGiven given, int N, int D, int pieces,
                                                         long long from) {
    constexpr int PL = Planes<T>::N;
    const long long at = from + blockIdx.x * 256LL + threadIdx.x;
    const int n = (int)(at / pieces), piece = (int)(at - (long long)n * pieces), c = piece * 8;
    if (n >= N) return;
    const bool masked = o.place ? o.place[n] < 0 : given.T && !any_given(given.tags + (long long)n * given.T, given.T);
    const int to = o.place ? o.place[n] : n;
    if (to >= 0) {
        float v[8] = {};
        if (!masked) load8(x + (long long)n * D, c, D, v);
        put_planes<PL>(dst + (long long)to * pieces * 8 + c, (long long)N * pieces * 8, v);
        if (GRADS && piece == 0) {
            float a = 0.f;
            for (int t = 0; t < given.T; ++t) {
                const long long word = given.tags[(long long)n * given.T + t];
                if (word >= 0) a += word < given.V ? given.dlogp[(long long)n * given.T + t] : __builtin_nanf("");
            }
            o.a[to] = a;
            o.b[to] = given.dentropy && !masked ? given.dentropy[n] : 0.f;
            o.sums[to] = make_float4(given.state[3LL * n], given.state[3LL * n + 1], given.state[3LL * n + 2], masked ? 1.f : 0.f);
            if (o.index && !o.place) o.index[n] = masked ? -1 : n;
        }
    }
    if (masked && dx) {
        T *row = dx + (long long)n * D + c;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < D) row[e] = 0;
    }
}

// A group's scores: the largest, and the second largest with the place of the largest in its last five bits.
struct __attribute__((aligned(8))) Group {
    float first;
    unsigned second;
};

// Per wave and row: (largest score m, sum of exp(l - m) without one of the largest, sum of exp(l - m) (m - l)), and the groups.  A distance m - l is
// not negative, so distances compare as whole numbers, infinite and NaN ones as the largest; its last five bits make room for the word's place
// in the group.  WORDS: the scores themselves in the place of the groups, -inf behind the last word.
template <typename T, bool WORDS>
struct LogpEpi {
    float4 *stats;       // [wave's columns][stats_ld]
    long long stats_ld;
    void *groups;        // [M][groups_ld] Group or float, rows of whole 16 bytes
    int groups_ld;
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int V, int, char *lds) const {
        static_assert(NT == 1 || NT == 2 || NT == 4, "half the groups of a row for each of its two lanes, or one");
        const int h = lane >> 5;
        for_blocks<MT>([&](auto block) __attribute__((always_inline)) {
            constexpr int i = decltype(block)::value;
            const int m = m0 + 32 * i + (lane & 31);
            int end = V - n0 - 4 * h;   // columns of this wave that exist, as this lane counts: 0 .. 3, 8 .. 11, ..
            asm volatile("" : "+v"(end));
            if (__any(end < NT * 32)) {
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * j + 8 * (e >> 2) + (e & 3) >= end) acc[i][j][e] = -__builtin_inff();
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, acc[i][j][e]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -__builtin_inff() ? 0.f : top;   // all scores -inf: exponentials of 0, not of NaN
            float sum = 0.f, part = 0.f, apart = 0.f;   // of exponentials, of those below one, of those times the distance
            Group g[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                unsigned near = 0xffffffffu, next = 0xffffffffu;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float d = base - acc[i][j][e];
                    const float p = sizeof(T) == 4 ? expf(-d) : __builtin_amdgcn_exp2f(d * -1.44269504f);
                    sum += p;
                    part += __builtin_amdgcn_fractf(p);
                    apart += p * fminf(d, 256.f);   // beyond, and where l = -inf, p is zero
                    if constexpr (WORDS) continue;
                    const unsigned key = (__builtin_bit_cast(unsigned, d) & ~31u) | (8 * (e >> 2) + (e & 3) + 4 * h);
                    next = max(min(near, next), min(max(near, next), key));
                    near = min(near, key);
                }
                if constexpr (WORDS) continue;
                const unsigned near2 = __shfl_xor((int)near, 32), next2 = __shfl_xor((int)next, 32);
                next = min(min(next, next2), max(near, near2));
                near = min(near, near2);
                g[j].first = base - __builtin_bit_cast(float, near & ~31u);
                const float second = fmaxf(base - __builtin_bit_cast(float, next & ~31u), -3.4028234664e38f);   // 0xffffffff, NaN and infinity: none
                g[j].second = (__builtin_bit_cast(unsigned, second) & ~31u) | (near & 31u);
            }
            sum += __shfl_xor(sum, 32);
            part += __shfl_xor(part, 32);
            apart += __shfl_xor(apart, 32);
            if constexpr (WORDS) {
                const RowStage<float, NT * 32> stage = {lds, lane};
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                        stage.put(32 * j + 8 * q + 4 * h, v);
                    }
                stage.take([&](int r, int c, const u32x4 &w) {
                    const int to = m0 + 32 * i + r;
                    if (to < M && n0 + c < groups_ld) *(u32x4 *)((float *)groups + (long long)to * groups_ld + n0 + c) = w;
                });
            }
            if (m >= M) return;
            // what reaches one are the largest scores; one of them is left out
            const float rest = top == -__builtin_inff() ? sum * 0.f : part + (rintf(sum - part) - 1.f);
            if (h == 0) stats[(n0 / (NT * 32)) * stats_ld + m] = make_float4(top, rest, apart, 0.f);
            if constexpr (WORDS) return;
            Group *const to = (Group *)groups + (long long)m * groups_ld + n0 / kGroupWords + h * (NT / 2);
            if (n0 + 32 * (h * (NT / 2)) < V) {
                if constexpr (NT == 4) {   // the pair's second may be behind the last word, where the row still has room
                    const Group a = h ? g[2] : g[0], b = h ? g[3] : g[1];
                    *(u32x4 *)to = (u32x4){__builtin_bit_cast(unsigned, a.first), a.second, __builtin_bit_cast(unsigned, b.first), b.second};
                } else if constexpr (NT == 2) {
                    *to = h ? g[1] : g[0];
                } else if (h == 0) {
                    *to = g[0];
                }
            }
        });
    }
};

struct Joined {
    float top, rest, apart;
    __device__ __forceinline__ void join(float t, float r, float u) {
        if (t > top) {
            float s = t;
            t = top, top = s;
            s = r, r = rest, rest = s;
            s = u, u = apart, apart = s;
        }
        if (t != -__builtin_inff()) {
            const float d = top - t, f = expf(-d);
            apart += f * (u + fminf(d, 256.f) * (1.f + r));
            rest += f * (1.f + r);
        } else {
            rest += r * 0.f;   // nothing, unless it is NaN
        }
    }
};

// What joined tiles say of a row: its largest score, the logarithm of the sum relative to it, the entropy.
__device__ __forceinline__ float4 sums_of(const Joined &s) {
    const float log_sum = __builtin_isfinite(s.top) ? log1pf(s.rest) : __builtin_nanf("");   // no softmax without a finite largest score
    return make_float4(s.top, log_sum, log_sum + s.apart / (1.f + s.rest), 0.f);
}

// One thread's share of a row's tiles, four loads in flight.
__device__ __forceinline__ Joined join_some(const float4 *stats, long long stats_ld, int tiles, int m, int from, int step) {
    Joined s = {-__builtin_inff(), 0.f, 0.f};
    for (int t = from; t < tiles; t += 4 * step) {
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = stats[min(t + k * step, tiles - 1) * stats_ld + m];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (t + k * step < tiles) s.join(v[k].x, v[k].y, v[k].z);
    }
    return s;
}

// Many rows: 16 a workgroup, which reads whole lines of the statistics, 16 threads each, in a fixed order.
static __global__ __launch_bounds__(256) void logp_join_kernel(const float4 *stats, long long stats_ld, int tiles, LogpRows o, int first, int most) {
    __shared__ Joined all[16][17];
    const int row = threadIdx.x % 16, part = threadIdx.x / 16, m = blockIdx.x * 16 + row;
    const bool in = m < live(most, o.count, first);
    Joined s = join_some(stats, stats_ld, in ? tiles : 0, m, part, 16);
    all[part][row] = s;
    for (int w = 8; w; w >>= 1) {
        __syncthreads();
        if (part < w) {
            const Joined b = all[part + w][row];
            s.join(b.top, b.rest, b.apart);
            all[part][row] = s;
        }
    }
    if (part == 0 && in) o.sums[first + m] = sums_of(s);
}

// sum_k x[k] w_i[k] in 64 bits for W rows w_i by one wave; the same bits for a row whatever W is and whoever asks.
template <int W, typename T>
__device__ __forceinline__ void wave_dots(const T *x, const T *const (&w)[W], int D, int lane, double (&s)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) s[i] = 0.0;
    const auto step = [&](int c, int end) __attribute__((always_inline)) {
        float a[8], b[W][8];
#pragma unroll
        for (int i = 0; i < W; ++i) load8(w[i], c, end, b[i]);
        load8(x, c, end, a);
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < W; ++i) s[i] = __builtin_fma((double)a[e], (double)b[i][e], s[i]);
    };
    const int whole = D / 512 * 512;
#pragma unroll 4
    for (int c = lane * 8; c < whole; c += 512) step(c, c + 8);
    if (whole + lane * 8 < D) step(whole + lane * 8, D);
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int d = 32; d; d >>= 1) s[i] += __shfl_xor(s[i], d);
}

// Scores in a workgroup's list: candidates, and behind them the given words.
constexpr int most_candidates(int K) { return K * kGroupWords > 256 ? K * kGroupWords : 256; }

// One row a workgroup: its likeliest words, the log probabilities of its given words, and what the joined sums say.  JOIN: joins them too, where
// rows are few enough for their tiles not to be read by whole lines.  Bound by latency for few rows, so what one wait can bring is asked for at once;
// for many by the groups' scores and the candidates' weights.
// A workgroup looks at groups, or at words where their scores have been kept: PER of them in 16 bytes.
template <typename T, int THREADS, bool JOIN, bool WORDS>
__global__ __launch_bounds__(THREADS) void logp_answer_kernel(const T *x, const T *w, const int64_t *tags, const float4 *stats, long long stats_ld, int tiles,
                                                             const void *groups, int groups_ld, LogpRows o, LogpOut out, int first, int most, int D,
                                                             int V) {
    constexpr int WAVES = THREADS / 64, HELD = 8, PER = WORDS ? 4 : 2, SIZE = WORDS ? 1 : kGroupWords;   // words of a group
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ __attribute__((aligned(16))) float tops[THREADS];
    __shared__ float4 joined;
    __shared__ Joined shares[WAVES];
    __shared__ float limit, best;
    __shared__ double base64;
    __shared__ int found;
    __shared__ unsigned long long picked[WAVES];
    const int m = blockIdx.x, K = max(out.K, 1), room = most_candidates(K);
    double *const score = (double *)smem;
    int *const word = (int *)(score + room + out.T);
    const long long n = o.index ? o.index[first + m] : first + m;
    if (m >= live(most, o.count, first)) {
        answer_masked(out, n);
        return;
    }
    const int G = (V + SIZE - 1) / SIZE, pieces = (G + PER - 1) / PER;
    const u32x4 *const row = (const u32x4 *)((const char *)groups + (long long)m * groups_ld * (16 / PER));   // behind the last group: not looked at
    u32x4 held[HELD];   // this thread's first pieces
#pragma unroll
    for (int k = 0; k < HELD; ++k) held[k] = row[min(tid + k * THREADS, pieces - 1)];
    Joined share;
    if constexpr (JOIN) {
        share = join_some(stats, stats_ld, tiles, m, tid, THREADS);
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const Joined b = {__shfl_xor(share.top, d), __shfl_xor(share.rest, d), __shfl_xor(share.apart, d)};
            share.join(b.top, b.rest, b.apart);
        }
        if (lane == 0) shares[wave] = share;
    }
    // fn(group, its largest score, its second largest with the largest's place) for this thread's groups
    const auto for_groups = [&](const auto &fn) __attribute__((always_inline)) {
        const auto each = [&](int p, const u32x4 &v) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const unsigned f = v[WORDS ? k : 2 * k], second = v[WORDS ? k : 2 * k + 1];
                if (k == 0 || PER * p + k < G) fn(PER * p + k, __builtin_bit_cast(float, f), second);
            }
        };
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (tid + k * THREADS < pieces) each(tid + k * THREADS, held[k]);
        for (int p = tid + HELD * THREADS; p < pieces; p += THREADS) each(p, row[p]);
    };
    float own = -__builtin_inff();
    for_groups([&](int, float f, unsigned) __attribute__((always_inline)) { own = fmaxf(own, f); });
    // maxima of 256 parts of the groups: few groups are parts of their own
    const bool single = pieces <= 256 / PER;
    if (!single) {
        tops[tid] = own;
    } else if (tid < 256 / PER) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const unsigned f = held[0][WORDS ? k : 2 * k];
            tops[PER * tid + k] = PER * tid + k < G ? __builtin_bit_cast(float, f) : -__builtin_inff();
        }
    }
    if (tid == 0) found = 0, limit = -__builtin_inff();
    bool given = false;
    for (int t = tid; t < out.T; t += THREADS) {
        const long long v = tags[n * out.T + t];
        given |= v >= 0;
        word[room + t] = v < 0 ? -1 : v < V ? (int)v : -2;
    }
    if (out.T && !o.place) {
        if (!__syncthreads_or(given)) {
            answer_masked(out, n);
            return;
        }
    } else {
        __syncthreads();
    }
    if (JOIN && wave == 1) {
        share = lane < WAVES ? shares[lane] : Joined{-__builtin_inff(), 0.f, 0.f};
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            const Joined b = {__shfl_xor(share.top, d), __shfl_xor(share.rest, d), __shfl_xor(share.apart, d)};
            share.join(b.top, b.rest, b.apart);
        }
        if (lane == 0) joined = sums_of(share);
    }
    const auto part_top = [&](int i) {
        float v = tops[i];
        if (!single)
#pragma unroll
            for (int k = 256; k < THREADS; k += 256) v = fmaxf(v, tops[i + k]);
        return v;
    };
    // K of any number of parts' maxima are at least as large as the K-th: as many words' scores are.  64 parts are found faster, and of up to 16 the
    // K-th lets hardly more than K words through.
    if (K <= 16) {
        if (wave == 0) {
            float v = part_top(lane);
#pragma unroll
            for (int k = 1; k < 4; ++k) v = fmaxf(v, part_top(lane + 64 * k));
            int above = 0;
#pragma unroll
            for (int t = 0; t < 64; ++t) {
                const float b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), t));
                above += b > v || (b == v && t < lane);
            }
            if (above == 0) best = v;
            if (above == K - 1) limit = v;
        }
    } else {
        if constexpr (THREADS > 256) {
            const float v = tid < 256 ? part_top(tid) : 0.f;
            __syncthreads();
            if (tid < 256) tops[tid] = v;
            __syncthreads();
        }
        if (tid < 256) {
            const float v = tops[tid];
            int above = 0;
#pragma unroll 4
            for (int t = 0; t < 256; t += 4) {
                const f32x4 b = *(const f32x4 *)(tops + t);
#pragma unroll
                for (int k = 0; k < 4; ++k) above += b[k] > v || (b[k] == v && t + k < tid);
            }
            if (above == 0) best = v;
            if (above == K - 1) limit = v;
        }
    }
    __syncthreads();
    const float4 sums = JOIN ? joined : o.sums[first + m];
    if (tid == 0) {
        if (out.entropy) out.entropy[n] = sums.z;
        if (out.state) out.state[3 * n] = sums.x, out.state[3 * n + 1] = sums.y, out.state[3 * n + 2] = sums.z;
    }
    if (!(sums.y == sums.y)) {   // no distribution
        for (int k = tid; k < out.K; k += THREADS) out.top[n * out.K + k] = -1, out.top_logp[n * out.K + k] = __builtin_nanf("");
        for (int t = tid; t < out.T; t += THREADS) out.logp[n * out.T + t] = word[room + t] != -1 ? __builtin_nanf("") : 0.f;
        return;
    }
    // less what a product of tiles, and the places in a group, may be off by
    const float cut = limit == -__builtin_inff() ? limit : limit - 0x1p-16f * fmaxf(fabsf(limit), fabsf(best));
    if (own >= cut)   // few threads
        for_groups([&](int g, float f, unsigned second) __attribute__((always_inline)) {
            if (!(f >= cut)) return;
            if (!WORDS && __builtin_bit_cast(float, second) >= cut) {
                const int words = min(kGroupWords, V - g * kGroupWords), at = atomicAdd(&found, words);
                for (int i = 0; i < words; ++i)
                    if (at + i < room) word[at + i] = g * kGroupWords + i;
            } else {
                const int at = atomicAdd(&found, 1);
                if (at < room) word[at] = WORDS ? g : g * kGroupWords + (int)(second & 31u);
            }
        });
    __syncthreads();
    int candidates = found;
    if (candidates > room) {
        // Many words share nearly the same score.  The K groups whose largest scores come first hold the K first words, as far as
        // the product's scores tell; all of their words are candidates.
        unsigned long long last = ~0ull;   // a score as a whole number that orders alike, then the groups from the last to the first
        candidates = 0;
        for (int k = 0; k < min(K, G); ++k) {
            unsigned long long mine = 0;
            for_groups([&](int g, float f, unsigned) __attribute__((always_inline)) {
                const unsigned b = __builtin_bit_cast(unsigned, f + 0.f);   // one zero
                const unsigned long long key = (unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (unsigned)(0x7fffffff - g);
                if (key < last && key > mine) mine = key;
            });
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const unsigned long long other = __shfl_xor(mine, d);
                mine = other > mine ? other : mine;
            }
            __syncthreads();
            if (lane == 0) picked[wave] = mine;
            __syncthreads();
            for (int v = 0; v < WAVES; ++v) mine = picked[v] > mine ? picked[v] : mine;
            last = mine;
            const int g = 0x7fffffff - (int)(unsigned)mine, words = min(SIZE, V - g * SIZE);
            if (tid < words) word[candidates + tid] = g * SIZE + tid;
            candidates += words;
        }
        __syncthreads();
    }
    // scores of the candidates and, behind them, of the given words
    const int all = candidates + out.T;
    const auto place = [&](int c) { return c < candidates ? c : room + c - candidates; };
    const auto dots = [&](auto many) __attribute__((always_inline)) {
        constexpr int W = decltype(many)::value;
        for (int c = wave * W; c < all; c += WAVES * W) {
            const T *rows[W];
            double s[W];
#pragma unroll
            for (int i = 0; i < W; ++i) rows[i] = w + (long long)max(word[place(min(c + i, all - 1))], 0) * D;
            wave_dots<W>(x + n * D, rows, D, lane, s);
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (lane == 0 && c + i < all) score[place(c + i)] = s[i];
        }
    };
    if (all <= WAVES) dots(std::integral_constant<int, 1>());
    else if (all <= 2 * WAVES) dots(std::integral_constant<int, 2>());
    else dots(std::integral_constant<int, 4>());
    __syncthreads();
    const auto rank_of = [&](int c) {
        const double s = score[c];
        const int v = word[c];
        int rank = 0;
        for (int k = 0; k < candidates; ++k) rank += score[k] > s || (score[k] == s && word[k] < v);
        return rank;
    };
    int rank = tid < candidates ? rank_of(tid) : -1;
    if (rank == 0) base64 = score[tid];
    for (int c = tid + THREADS; c < candidates; c += THREADS)
        if (rank_of(c) == 0) base64 = score[c];
    __syncthreads();
    // The largest score has 64 bits here and 32 in the sum, where it stands for exp of itself: what the others' sum is relative to it moves by the
    // difference, times their share.
    const double top = base64, moved = (top - (double)sums.x) * (double)-expm1f(-sums.y);
    const auto log_p = [&](double s) { return (float)((s - top) + moved - (double)sums.y); };
    for (int c = tid; out.K && c < candidates; c += THREADS) {
        if (c != tid) rank = rank_of(c);
        if (rank >= out.K) continue;
        out.top[n * out.K + rank] = word[c];
        out.top_logp[n * out.K + rank] = log_p(score[c]);
    }
    for (int t = tid; t < out.T; t += THREADS) {
        const int v = word[room + t];
        out.logp[n * out.T + t] = v == -2 ? __builtin_nanf("") : v < 0 ? 0.f : log_p(fmin(score[room + t], top));
    }
}

// d of a row and word that is not given.  l - base first: the sum of both would be rounded at the scores' size
template <typename T>
__device__ __forceinline__ float logp_grad(float l, const float4 &sums, float a, float b) {
    const float lp = (l - sums.x) - sums.y;
    const float p = sizeof(T) == 4 ? expf(lp) : __builtin_amdgcn_exp2f(lp * 1.44269504f);
    return -p * (a + b * (fmaxf(lp, -256.f) + sums.z));
}

// V: bf16_t or float, what d is stored as; [M][ld], zeros behind the last word.
template <typename T, typename V>
struct LogpGradEpi {
    V *d;
    long long ld;
    const float4 *sums;
    const float *a, *b;
    template <int MT, int NT>
    __device__ __forceinline__ void run(f32x16 (&acc)[MT][NT], int m0, int n0, int lane, int M, int words, int, char *lds) const {
        const RowStage<V, NT * 32> stage = {lds, lane};
        const int h = lane >> 5;
        float4 s[MT];
        float ra[MT], rb[MT];   // all before the first store: a load behind a store waits until that has reached memory
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = min(m0 + 32 * i + (lane & 31), M - 1);
            s[i] = sums[m], ra[i] = a[m], rb[i] = b[m];
        }
        for_blocks<MT>([&](auto block) __attribute__((always_inline)) {
            constexpr int i = decltype(block)::value;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = 32 * j + 8 * q + 4 * h;
                    V v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float g = logp_grad<T>(acc[i][j][4 * q + r], s[i], ra[i], rb[i]);
                        v[r] = narrow<V>(n0 + c + r < words && s[i].w == 0.f ? g : 0.f);
                    }
                    stage.put(c, v);
                }
            stage.take([&](int r, int c, const u32x4 &w) {
                const int to = m0 + 32 * i + r;
                if (to < M && n0 + c < ld) *(u32x4 *)(d + to * ld + n0 + c) = w;
            });
        });
    }
};

// d where words are given, once for each word of a row.
template <typename V>
__global__ __launch_bounds__(256) void logp_given_kernel(V *d, long long ld, LogpRows o, LogpGiven g, const float *logp, int first, int most) {
    const long long at = blockIdx.x * 256LL + threadIdx.x;
    const int m = (int)(at / g.T), t = (int)(at - (long long)m * g.T);
    if (m >= live(most, o.count, first)) return;
    const long long n = o.index ? o.index[first + m] : first + m;
    if (n < 0) return;
    const int64_t *const words = g.tags + n * g.T;
    const float *const da = g.dlogp + n * g.T;
    const long long v = words[t];
    if (v < 0 || v >= g.V) return;
    float s = 0.f;
    for (int k = 0; k < g.T; ++k)
        if (words[k] == v) {
            if (k < t) return;
            s += da[k];
        }
    const float4 sums = o.sums[first + m];
    const float a = o.a[first + m], b = o.b[first + m], lp = logp[n * g.T + t];
    const float p = expf(lp), own = p > 0.5f ? (s - a) - a * expm1f(lp) : s - a * p;
    d[m * ld + v] = narrow<V>(own - b * p * (fmaxf(lp, -256.f) + sums.z));
}

// d as it is kept in fp32
struct KeptGrad {
    const float *d;
    long long ld;
    const int *count;
    int first, most;
    __device__ void beside() const {}
    __device__ bool skip(int m) const { return m >= live(most, count, first); }
    __device__ long long rows() const { return live(most, count, first); }
    __device__ void operator()(int m, int c, float (&v)[1][8]) const {
        const f32x4 *k = (const f32x4 *)(d + m * ld + c);
        const f32x4 a = k[0], b = k[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[0][e] = a[e], v[0][4 + e] = b[e];
    }
};

template <typename T>
__global__ __launch_bounds__(256) void logp_zero_kernel(T *p, long long n) {
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) p[i] = 0;
}

// Few rows' scores are formed by single blocks of 32 words: workgroups of half the size fill the compute units more evenly, and x is small (7 x
// 1021 times 20011 in fp32 57.7 us with two blocks, 47.3 with one; 1 x 4096 in bf16 51.5 and 46.5, times 50000 103 and 96, times 128000 214
// and 214).
constexpr int kFewCols = 32;
// Whether scores are kept as they are: for small vocabularies of which many words are asked for, about 16 K^2 / V groups hold two of them or more,
// and all their words' scores would be formed again (4046 x 256 over 2760 words, 30 likeliest: 391 us with groups).
inline bool keeps_words(int V, int K) { return V <= 8192 && 8LL * K * K > V; }

template <typename T>
struct LogpScratch {
    static constexpr int PL = Planes<T>::N;
    int Dp, Vp, block, blocks, wave_cols, tiles, groups_ld;
    bool direct, gathers, narrow;   // w is used where it is; rows are picked; tiles of 64 rows
    LogpRows rows = {};
    bf16_t *x = nullptr, *w = nullptr, *d = nullptr;
    float4 *stats = nullptr;
    void *groups = nullptr;
    float *kept = nullptr, *sum = nullptr;
    Parts part = {};
    bool words;   // scores are kept, and not those of groups
    LogpScratch(Scratch &sc, int N, int D, int V, int K, bool given, bool grads) {
        Dp = (int)round_up(D, 8), Vp = (int)round_up(V, 64);
        direct = PL == 1 && D == Dp, gathers = given && N > kNarrow;
        words = keeps_words(V, K);
        groups_ld = words ? (int)round_up(V, 4) : (int)round_up((V + kGroupWords - 1) / kGroupWords, 2);
        const long long row_bytes = grads ? (long long)Vp * (long long)sizeof(T) : groups_ld * (words ? 4LL : (long long)sizeof(Group));
        block = (int)std::min<long long>({round_up(N, 8), kMostGroups, std::max<long long>(kStep, (grads ? kGradBytes : kKeyBytes) / row_bytes / 256 * 256)});
        blocks = N ? (N + block - 1) / block : 0;
        const bool few = N <= kFewRows;
        narrow = !few && N <= kNarrow;
        wave_cols = few ? kFewCols : narrow ? 64 : product_wave_cols(block, V, D, Planes<T>::PAIRS);
        tiles = (V + wave_cols - 1) / wave_cols;
        rows.count = sc.take<int>(1);
        rows.place = sc.take<int>(N);
        rows.index = sc.take<int>(N);
        rows.sums = sc.take<float4>(N);
        rows.a = sc.take<float>(N);
        rows.b = sc.take<float>(N);
        if (!gathers) rows.count = rows.place = nullptr;
        if (!gathers && !(given && grads)) rows.index = nullptr;
        if (grads || (!few && (gathers || !direct))) x = sc.take<bf16_t>((long long)PL * N * Dp);
        if ((grads || !few) && !direct) w = sc.take<bf16_t>((long long)PL * V * Dp);
        if (!grads) {
            stats = sc.take<float4>(std::max((V + 63) / 64 * (long long)block, (V + kFewCols - 1) / kFewCols * std::min(round_up(N, 8), (long long)kFewRows)));
            groups = sc.take<char>(block * row_bytes);
            return;
        }
        const int twice = PL == 1 ? 2 * std::min(N, kFewRows) : 0;
        d = sc.take<bf16_t>((long long)Vp * std::max(PL * block, twice));
        kept = sc.take<float>((long long)Vp * (PL == 3 ? block : std::min(N, kFewRows)));
        part.floats = std::max({part_floats(std::max(block, twice), D, V), part_floats(V, D, block), twice * round_up(D, 4)});
        part.at = sc.take<float>(part.floats);
        sum = blocks > 1 ? sc.take<float>((long long)V * D) : nullptr;
    }
    int lay_out(const T *xs, const T *ws, T *dx, const LogpGiven &given, bool grads, int N, int D, int V, hipStream_t s) const {
        if (gathers) {
            const LaunchPlan p = make_plan("logp_rows", {}, {N, given.T}, dim3(1), 1024, 0);
            LC_LAUNCH(p, "logp (rows)", logp_rows_kernel, s, given.tags, N, given.T, rows);
        }
        if (x) {
            const auto gather = [&](auto kernel) -> int {
                return in_launches((long long)N * (Dp / 8), [&](long long from, unsigned n) -> int {
                    const LaunchPlan p = make_plan("logp_gather", {PL, grads}, {N, D}, dim3(n), 256, 0);
                    LC_LAUNCH(p, "logp (x)", kernel, s, xs, x, dx, rows, given, N, D, Dp / 8, from);
                    return LC_OK;
                });
            };
            if (int rc = grads ? gather(logp_gather_kernel<T, true>) : gather(logp_gather_kernel<T, false>)) return rc;
        }
        if (w) return launch_planes<PL, 1>("logp (w)", Stored<T>{ws, V, D}, w, Dp, (long long)V * Dp, V, Dp, 0, s);
        return LC_OK;
    }
};

template <typename T>
int logp_forward(const T *x, const T *w, const int64_t *tags, const LogpOut &out, int N, int D, int V, void *ws, hipStream_t s) {
    constexpr int PL = Planes<T>::N;
    if (N == 0) return LC_OK;
    Scratch sc(ws);
    const LogpScratch<T> g(sc, N, D, V, out.K, out.T > 0, false);
    if (int rc = g.lay_out(x, w, nullptr, LogpGiven{tags, nullptr, nullptr, nullptr, out.T, V}, false, N, D, V, s)) return rc;
    const bool few = N <= kFewRows;
    const Operand W = g.w ? Operand{g.w, g.w, g.Dp, (long long)V * g.Dp, V, 0, 0} : Operand{(const bf16_t *)w, (const bf16_t *)w, D, 0, V, 0, 0};
    for (int b = 0; b < g.blocks; ++b) {
        const int first = b * g.block, most = std::min(g.block, N - first);
        const auto scores = [&](const auto &epi) -> int {
            if (few)
                return launch_blocks<T, ROW, 1>("logp (few rows)", FewOperand<T>{x, x, D, N, nullptr}, FewOperand<T>{w, w, D, V, nullptr}, N, nullptr, V, D,
                                                epi, s);
            const bf16_t *const xs = g.x ? g.x : (const bf16_t *)x;   // as it lies, where rows are neither picked nor laid out
            const Operand X = {xs + (long long)first * g.Dp, xs, g.Dp, (long long)N * g.Dp, most, 0, 0};
            const Shape sh = {most, V, D, g.rows.count, first, nullptr, 0};
            return g.narrow ? launch_narrow<PL, ROW, 128>("logp", X, W, sh, epi, s)
                            : launch_cut<PL, ROW, ROW, 8>("logp", X, W, sh, choose_cut(g.block, V, D, Planes<T>::PAIRS, false), epi, s);
        };
        if (int rc = g.words ? scores(LogpEpi<T, true>{g.stats, g.block, g.groups, g.groups_ld}) : scores(LogpEpi<T, false>{g.stats, g.block, g.groups, g.groups_ld}))
            return rc;
        const bool apart = most >= 2048;
        if (apart) {
            const LaunchPlan p = make_plan("logp_join", {}, {most}, dim3((most + 15) / 16), 256, 0);
            LC_LAUNCH(p, "logp (join)", logp_join_kernel, s, g.stats, (long long)g.block, g.tiles, g.rows, first, most);
        }
        const int threads = most <= kComputeUnits ? 1024 : 256;
        const LaunchPlan p = make_plan("logp_answer", {(int)sizeof(T), apart}, {most, D, V, out.T, out.K}, dim3(most), threads,
                                       12 * (size_t)(most_candidates(std::max(out.K, 1)) + out.T));
        const auto answer = [&](auto kernel) -> int {
            LC_LAUNCH(p, "logp (answer)", kernel, s, x, w, tags, g.stats, (long long)g.block, g.tiles, g.groups, g.groups_ld, g.rows, out, first, most, D, V);
            return LC_OK;
        };
        if (int rc = g.words ? apart            ? answer(logp_answer_kernel<T, 256, false, true>)
                               : threads == 256 ? answer(logp_answer_kernel<T, 256, true, true>)
                                                : answer(logp_answer_kernel<T, 1024, true, true>)
                     : apart          ? answer(logp_answer_kernel<T, 256, false, false>)
                     : threads == 256 ? answer(logp_answer_kernel<T, 256, true, false>)
                                      : answer(logp_answer_kernel<T, 1024, true, false>))
            return rc;
    }
    return LC_OK;
}

template <typename T>
int logp_backward(const T *x, const T *w, const int64_t *tags, const float *logp, const float *state, const float *dlogp, const float *dentropy, T *dx,
                  T *dw, int N, int D, int V, int given_words, void *ws, hipStream_t s) {
    constexpr int PL = Planes<T>::N;
    if (N == 0) {
        const long long n = (long long)V * D;
        const LaunchPlan p = make_plan("logp_zero", {}, {}, dim3((unsigned)std::min<long long>((n + 255) / 256, 4096)), 256, 0);
        LC_LAUNCH(p, "logp_bwd (no rows)", (logp_zero_kernel<T>), s, dw, n);
        return LC_OK;
    }
    Scratch sc(ws);
    const LogpScratch<T> g(sc, N, D, V, 0, given_words > 0, true);
    const LogpGiven given = {tags, state, dlogp, dentropy, given_words, V};
    if (int rc = g.lay_out(x, w, dx, given, true, N, D, V, s)) return rc;
    const bool few = N <= kFewRows, fine = few && PL == 1;   // fine: d in two parts
    Operand W = g.w ? Operand{g.w, g.w, g.Dp, (long long)V * g.Dp, V, 0, 0} : Operand{(const bf16_t *)w, (const bf16_t *)w, D, 0, V, 0, 0};
    for (int b = 0; b < g.blocks; ++b) {
        const int first = b * g.block, most = std::min(g.block, N - first);
        Operand X = {g.x + (long long)first * g.Dp, g.x, g.Dp, (long long)N * g.Dp, most, 0, 0}, Wr = W;
        const Shape sh = {most, V, D, g.rows.count, first, nullptr, 0};
        const auto scores = [&](const auto &epi) -> int {
            if (few)
                return launch_blocks<T, ROW, 1>("logp_bwd (few rows)", FewOperand<T>{x, x, D, N, nullptr}, FewOperand<T>{w, w, D, V, nullptr}, N, nullptr,
                                          V, D, epi, s);
            if (g.narrow) return launch_narrow<PL, ROW, 128>("logp_bwd", X, Wr, sh, epi, s);
            return launch_cut<PL, ROW, ROW, 8>("logp_bwd", X, Wr, sh, choose_cut(g.block, V, D, Planes<T>::PAIRS, false), epi, s);
        };
        const auto words = [&](auto *d) -> int {
            typedef std::remove_reference_t<decltype(*d)> Stored_t;
            if (int rc = scores(LogpGradEpi<T, Stored_t>{d, g.Vp, g.rows.sums + first, g.rows.a + first, g.rows.b + first})) return rc;
            if (!given_words) return LC_OK;
            const long long n = ((long long)most * given_words + 255) / 256;
            const LaunchPlan p = make_plan("logp_given", {}, {most, given_words}, dim3((unsigned)n), 256, 0);
            LC_PLAN_REQUIRE(p, n <= 0x7fffffffLL);
            LC_LAUNCH(p, "logp_bwd (given)", (logp_given_kernel<Stored_t>), s, d, (long long)g.Vp, g.rows, given, logp, first, most);
            return LC_OK;
        };
        int rc;
        const bool kept = PL == 3 || fine;
        if ((rc = kept ? words(g.kept) : words(g.d))) return rc;
        const int *const index = g.rows.index ? g.rows.index + first : nullptr;
        const KeptGrad from = {g.kept, g.Vp, g.rows.count, first, most};
        T *const to = dx && !index ? dx + (long long)first * D : dx;
        if constexpr (PL == 1)
            if (fine) {   // one block
                const int two = 2 * N;
                if ((rc = launch_planes<2, 1>("logp_bwd (d)", from, g.d, g.Vp, 0, N, g.Vp, 0, s))) return rc;
                Operand d = {g.d, g.d, g.Vp, 0, two, 0, 0};
                Wr.rows = X.rows = g.Dp;
                if (dx) {
                    const Shape shx = {two, D, V, g.rows.count, 0, nullptr, 0, 2};
                    if ((rc = launch_product<PL, ROW, COL, true, 8>("logp_bwd (dx)", d, Wr, shx, StoreEpi<T>{dx, nullptr, 0x7fffffff, N, 0, D, index, nullptr, nullptr},
                                                                 g.part, s)))
                        return rc;
                }
                const Shape shw = {V, D, two, nullptr, 0, g.rows.count, 0, 2};
                d.rows = g.Vp;
                return launch_gemm<2, COL, COL, 8>("logp_bwd (dw)", d, X, shw, StoreEpi<T>{dw, nullptr, 0x7fffffff, V, 0, D, nullptr, nullptr, nullptr}, s);
            }
        const long long pd = (long long)g.block * g.Vp;
        if (kept && (rc = launch_planes<PL, 1>("logp_bwd (d)", from, g.d, g.Vp, pd, most, g.Vp, 0, s))) return rc;
        Operand d = {g.d, g.d, g.Vp, pd, most, 0, 0};
        Wr.rows = X.rows = g.Dp;
        if (dx) {
            const Shape shx = {most, D, V, g.rows.count, first, nullptr, 0};
            if ((rc = launch_product<PL, ROW, COL, false, 8>("logp_bwd (dx)", d, Wr, shx, StoreEpi<T>{to, nullptr, 0x7fffffff, most, 0, D, index, nullptr, nullptr}, g.part, s)))
                return rc;
        }
        const Shape shw = {V, D, most, nullptr, 0, g.rows.count, first};
        d.rows = g.Vp;
        const float *add = b ? g.sum : nullptr;
        if (b + 1 < g.blocks)
            rc = launch_product<PL, COL, COL, false, 8>("logp_bwd (dw)", d, X, shw, StoreEpi<float>{g.sum, nullptr, 0x7fffffff, V, 0, D, nullptr, add, nullptr}, g.part, s);
        else
            rc = launch_product<PL, COL, COL, false, 8>("logp_bwd (dw)", d, X, shw, StoreEpi<T>{dw, nullptr, 0x7fffffff, V, 0, D, nullptr, add, nullptr}, g.part, s);
        if (rc) return rc;
    }
    return LC_OK;
}

template <typename T>
size_t logp_scratch(int N, int D, int V, int K, bool given, bool grads) {
    Scratch sc(nullptr);
    (void)LogpScratch<T>(sc, N, D, V, K, given, grads);
    return sc.used;
}

}  // namespace head
}  // namespace lc
