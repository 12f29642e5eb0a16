// Distillation from a teacher's top logits: loss of each row (this file) and its gradient (distill_back.cu).
//
// Of a row of C logits s the teacher kept K classes i_k with logits t_k and, if given, the log-sum-exp over T of its
// other logits, `rest`.  With p the softmax of (t_k / T, rest) and q the student's probabilities at T of the same
// classes -- q_k = exp((s_{i_k} - m) / T) / Z_T, and of the others together q_0 = the sum over them --
//     loss = (1 - alpha) (log Z_1 + m - s_label) + alpha T^2 sum p (log p - log q),
// m the largest logit, Z_1 and Z_T the sums of exp(s - m) and exp((s - m) / T).
//
// q_0 is summed over the classes that are not kept, as 1 - sum q_k would lose it where the kept classes have nearly
// all: a bit for each 16-byte vector of logits in shared memory says whether a kept class is in it, and such a vector is left
// to the thread that has that class of the teacher's.  A thread keeps a running maximum and the sums below it, so that the
// row is read once; the kept logits themselves join at the end.
//
// The divergence is summed as sum of p f(delta), f(delta) = e^delta - 1 - delta and delta = log q - log p, whose terms are all positive and
// exact where student and teacher agree; its logarithms by themselves would cancel there.  Without `rest` that also takes
// 1 - sum q_k, the mass of the classes that are not kept: rows whose divergence is small beside its logarithms are read a
// second time for it, the others' logarithms are summed as they stand (8192 x 32768 bf16 89.8 us, 88.1 without the choice, 213
// where every row is read again; 8192 x 1000 fp32 with 16 kept 12.6, 12.3 and 21.2).
//
// What bounds it is memory, a row is read and next to nothing written, and issued instructions (69 % of the slots).  8192 x 32768 bf16 with 64 kept, labels and T = 2 takes 107
// us, 5.0 TB/s, of 80 at a copy's rate (GPU time, calls one after another in one graph); what is left is the rows' fixed work, the teacher's entries and the join.  The kept logits
// gathered before the row took 118 us; without the exponential's square, the prefetch and the batches a thread has under way 153.
#include <cooperative_groups.h>

#include <algorithm>

#include "rows.cuh"

namespace patconv {
namespace {

namespace cg = cooperative_groups;

constexpr int kWide = 128;            // threads of a CTA that has a row, or a part of one
constexpr int kRowsOfCta = 4;         // rows of a CTA whose warps have one each
constexpr int kStep = 1024;           // vectors that a CTA asks for ahead of its reading where it does not ask for its whole row
constexpr int kMostOfWarp = 1024;     // 16-byte vectors of a warp's row at most

constexpr int kBitsOfWarp = kMostOfWarp / 32;        // words of a warp's row: a bit a vector

// what a thread sums of the classes it sees: the largest x, and the sums of 2^((x - m) c) relative to it
// HARD: how the sum at T = 1 is had beside the one at T.  kNone: there are no labels, or T is 1; kApart: by an exponential of its
// own; kSquare, kFourth: T is 2 or 4, and exp(d) is exp(d / T) to that power -- the special function unit, with two
// exponentials a value, would bound the kernel before memory does.
enum { kNoHard = 0, kApart = 1, kSquare = 2, kFourth = 4 };
template <int HARD>
struct Running {
    float m = kNone, ref = 0;         // and m, or 0 before there is one
    float2 z1 = {0, 0}, zt = {0, 0};
    __device__ __forceinline__ void below(float top, float c1, float ct) {
        if (!(top > m)) return;
        if (m != kNone) {
            zt = mul(zt, both(power(m, top, ct)));
            if (HARD) z1 = mul(z1, both(power(m, top, c1)));
        }
        m = ref = top;
    }
    __device__ __forceinline__ void add_pair(float2 x, float2 c1, float2 ct) {
        const float2 d = add(x, both(-ref)), l = mul(d, ct), e = make_float2(approx_exp2(l.x), approx_exp2(l.y));
        zt = add(zt, e);
        if (HARD == kApart) {
            const float2 f = mul(d, c1);
            z1 = add(z1, make_float2(approx_exp2(f.x), approx_exp2(f.y)));
        } else if (HARD == kSquare) {
            z1 = fma(e, e, z1);
        } else if (HARD == kFourth) {
            const float2 q = mul(e, e);
            z1 = fma(q, q, z1);
        }
    }
};

// The threads of a row read it together; then their sums and the teacher's entries are joined by one warp, the others being
// done.  A row's fixed work is a good part of a row of 64 KB: 128 threads to a CTA and one warp at the end have it overlap
// the reading of the seven other rows on the SM, and cost four warps and not eight.
template <typename T, bool REST, int HARD, int N>
__global__ void __launch_bounds__(N == 32 ? 32 * kRowsOfCta : N, N == 32 ? 6 : 8) distill_rows(DistillArgs a) {
    constexpr int W = 16 / sizeof(T), U = N == 32 ? 4 : 2, kWarps = N / 32, kEntries = N == 32 ? 32 : kMostKept;
    extern __shared__ uint4 dynamic[];
    __shared__ float parts[16][3];                    // of a cluster's CTAs, in the first one
    __shared__ float sums[kRowsOfCta][kWarps][3];
    __shared__ __align__(16) int places[N == 32 ? kRowsOfCta : 1][kEntries];
    __shared__ float teacher[N == 32 ? kRowsOfCta : 1][kEntries], student[N == 32 ? kRowsOfCta : 1][kEntries];
    __shared__ bool before[N == 32 ? kRowsOfCta : 1][kEntries];
    __shared__ unsigned long long whole_of[kWarps];   // the warps' shares of a second reading
    __shared__ float again_from, again_least;         // what it is relative to, NaN: there is none; the least logit of the teacher's entries
    const int slot = N == 32 ? threadIdx.x / 32 : 0;
    const int part = N == 32 ? 0 : blockIdx.x % a.parts;
    const int row = N == 32 ? blockIdx.x * kRowsOfCta + slot : blockIdx.x / a.parts;
    if (row >= a.rows) return;
    Group<N> g(nullptr);
    const T* s = static_cast<const T*>(a.s) + row * a.stride;
    const Row<T, W> r(s, a.classes);
    // this group's vectors
    const int each = (r.vectors() + a.parts - 1) / a.parts, first = part * each, last = min(r.vectors(), first + each);
    unsigned* bits = reinterpret_cast<unsigned*>(dynamic) + (N == 32 ? slot * kBitsOfWarp : 0);
    int* kept = places[slot];                         // the entries' places in the row, -1: empty
    bool* came = before[slot];                        // whether an entry's class is that of an earlier one
    float *us = teacher[slot], *xs = student[slot];
    // the ends of a row that are no whole vectors are taken by themselves
    const int from = first < last && !r.whole(first) ? first + 1 : first;
    const int to = last > from && !r.whole(last - 1) ? last - 1 : last;
    // the logits are asked for at once, whatever the teacher's entries then say: on their way to L2, the first ones here
    if (N > 32 && threadIdx.x == 0) r.prefetch(first, a.stepwise ? min(last, first + kStep) : last);
    int v = from + g.lane;
    Vec<T, W> batch[U];
    const bool early = v + (U - 1) * N < to;
    if (early)
#pragma unroll
        for (int k = 0; k < U; ++k) batch[k] = r.at(v + k * N);

    // the teacher's entries
    bool any = false;
    for (int k = g.lane; k < (a.kept + 3) / 4 * 4; k += N) {
        const int64_t j = (int64_t)row * a.kept + k;
        int at = k < a.kept ? a.indices[j] : -1;
        float u = kNone;
        if (at >= 0 && at < a.classes)
            u = value_at(a.values, a.value_type, j) * a.inv_t;
        else
            at = -1;
        kept[k] = at < 0 ? -1 : at + r.pad;
        us[k] = u;
        any = any || u != kNone;
    }
    const float rest = REST ? a.rest[row] : kNone;
    int64_t label = a.labels ? a.labels[row] : -1;
    if (label >= a.classes) label = -1;
    if (REST)
        for (int w = g.lane; w < (max(0, last - first) + 31) / 32; w += N) bits[w] = 0;
    const bool taught = g.any(any || (REST && rest != kNone));
    if (!taught && label < 0) {                       // uniform over the row's CTAs: nothing to learn from this row
        if (part == 0 && g.lane < 5) {
            a.stats[(int64_t)row * 5 + g.lane] = 0;
            if (g.lane == 0) a.loss[row] = 0;
        }
        return;
    }
    if (REST) {
        if constexpr (N == 32) g.sync();
        for (int k = g.lane; k < a.kept; k += N) {
            const int home = kept[k] / W;
            if (kept[k] >= 0 && home >= first && home < last) atomicOr(&bits[(home - first) / 32], 1u << ((home - first) % 32));
        }
        g.sync();
    }
    if constexpr (N > 32)                             // the first CTA's memory is written by the others, once it has begun
        if (a.parts > 1) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");

    Running<HARD> sum;
    const float2 c1 = both(a.c1), ct = both(a.ct);
    // whether vector v is left out: its bit is the same one of a word for all of a thread's vectors
    const unsigned bit = 1u << ((v - first) % 32);
    const auto left_out = [&](int v) { return REST && bits[(v - first) / 32] & bit; };
    const auto take = [&](const auto& b) {
        constexpr int K = std::extent<std::remove_reference_t<decltype(b)>>::value;
        float2 f[K * W / 2];
        Largest<T> top;
#pragma unroll
        for (int k = 0; k < K; ++k) top.take(b[k]);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < W / 2; ++i) f[k * W / 2 + i] = pair(b[k], i);
        sum.below(top.get(), a.c1, a.ct);
#pragma unroll
        for (int i = 0; i < K * W / 2; ++i) sum.add_pair(f[i], c1, ct);
    };
    const auto clear = [&](Vec<T, W>& b, bool all) {  // nothing is there: -inf
        uint4 w;
        memcpy(&w, &b, 16);
        const unsigned none = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u;
        w.x = all ? none : w.x, w.y = all ? none : w.y, w.z = all ? none : w.z, w.w = all ? none : w.w;
        memcpy(&b, &w, 16);
    };
    const auto values_of = [&](const Vec<T, W>& b, unsigned but) {     // a vector's values but for some
        float y[W], top = kNone;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            y[i] = but >> i & 1 ? kNone : widen(b.v[i]);
            top = larger(top, y[i]);
        }
        sum.below(top, a.c1, a.ct);
#pragma unroll
        for (int i = 0; i < W; i += 2) sum.add_pair(make_float2(y[i], y[i + 1]), c1, ct);
    };
    const auto ready = [&](Vec<T, W> (&b)[U], int v) {
        if (REST)
#pragma unroll
            for (int k = 0; k < U; ++k) clear(b[k], left_out(v + k * N));
    };
    // the next ones are asked for before these are taken
    const int batches = v < to ? ((to - v + N - 1) / N) / U : 0;
    for (int i = 0; i < batches; i += 2, v += 2 * U * N) {
        if (N > 32 && threadIdx.x == 0 && a.stepwise && i * U * N % kStep == 0 && v + kStep < last) r.prefetch(v + kStep, min(last, v + 2 * kStep));
        Vec<T, W> next[U];
        if (i + 1 < batches)
#pragma unroll
            for (int k = 0; k < U; ++k) next[k] = r.at(v + (U + k) * N);
        ready(batch, v);
        take(batch);
        if (i + 1 == batches) {
            v += U * N;
            break;
        }
        if (i + 2 < batches)
#pragma unroll
            for (int k = 0; k < U; ++k) batch[k] = r.at(v + (2 * U + k) * N);
        ready(next, v + U * N);
        take(next);
    }
    for (; v < to; v += N) {
        Vec<T, W> b[1] = {r.at(v)};
        if (REST) clear(b[0], left_out(v));
        take(b);
    }
    const auto marked = [&](int v) { return REST && bits[(v - first) / 32] >> ((v - first) % 32) & 1; };
    if (from > first && g.lane == 0 && !marked(first)) values_of(r.some(first), 0);
    if (to < last && g.lane == N - 1 && !marked(to)) values_of(r.some(to), 0);
    // the kept classes' logits, and the others in the vectors that were left out for them: of those with several kept classes
    // the first entry has it
    for (int k = g.lane; k < a.kept; k += N) {
        const int place = kept[k], home = place / W;
        float x = kNone;
        bool again = false;
        if (place >= 0) {
            x = widen(r.base[place]);
            if (REST) {
                unsigned inside = 0;
                bool keeper = home >= first && home < last;
                for (int j = 0; j < a.kept; j += 32) {
                    unsigned same = 0;                // which of 32 entries are of this vector (an empty place is far from every one)
#pragma unroll 4
                    for (int i = 0; i < min(32, a.kept - j); i += 4) {
                        const int4 four = *reinterpret_cast<const int4*>(kept + j + i);
                        same |= ((unsigned)((unsigned)(four.x ^ place) < (unsigned)W) | (unsigned)((unsigned)(four.y ^ place) < (unsigned)W) << 1 |
                                 (unsigned)((unsigned)(four.z ^ place) < (unsigned)W) << 2 | (unsigned)((unsigned)(four.w ^ place) < (unsigned)W) << 3) << i;
                    }
                    for (; same; same &= same - 1) {
                        const int i = j + __ffs(same) - 1, other = kept[i];
                        inside |= 1u << (other % W);
                        keeper = keeper && i >= k;
                        again = again || (other == place && i < k);
                    }
                }
                if (keeper) values_of(r.some(home), inside);
            }
        }
        xs[k] = x;
        came[k] = again;
    }

    // A second reading of the whole row by this CTA's threads: a warp's sum of exp((s - m) / T) in units of 2^-52.  Of integers the kept
    // classes' can be subtracted, and nothing is lost; those below the least of them, as nearly all are, are no kept ones and summed
    // as they are (all of them as integers: 457 us for 8192 x 32768 bf16, 213 so).  What an integer loses by rounding is 2^-53.
    const auto unit = [&](float x, float m) { return __float2ull_rn(power(x, m, a.ct) * 0x1p52f); };
    const auto read_again = [&](float m, float least) {
        constexpr int A = 4;
        unsigned long long n = 0;
        float2 below = make_float2(0.0f, 0.0f);
        const auto add_vector = [&](const Vec<T, W>& b, int v) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                const float2 x = pair(b, i), l = mul(add(x, both(-m)), ct), e = make_float2(approx_exp2(l.x), approx_exp2(l.y));
                below = add(below, make_float2(x.x < least ? e.x : 0.0f, x.y < least ? e.y : 0.0f));
            }
            if (largest(b) < least) return;
            unsigned those = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) those |= (unsigned)(widen(b.v[i]) >= least) << i;
            for (; those; those &= those - 1) n += unit(widen(r.base[v * W + __ffs(those) - 1]), m);
        };
        const int last = r.vectors(), begin = r.whole(0) ? 0 : 1, end = last > begin && !r.whole(last - 1) ? last - 1 : last;
        for (int v = begin; v < end; v += A * N) {
            Vec<T, W> b[A];
#pragma unroll
            for (int k = 0; k < A; ++k) b[k] = r.at(min(v + k * N + g.lane, end - 1));
#pragma unroll
            for (int k = 0; k < A; ++k) {
                clear(b[k], v + k * N + g.lane >= end);
                add_vector(b[k], v + k * N + g.lane);
            }
        }
        if (begin > 0 && g.lane == 0) add_vector(r.some(0), 0);
        if (end < last && g.lane == N - 1) add_vector(r.some(last - 1), last - 1);
        n += __float2ull_rn((below.x + below.y) * 0x1p52f);
#pragma unroll
        for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        return n;
    };
    // the first warp and the others come to it from different places
    const auto meet = [] { asm volatile("barrier.sync 1, %0;" ::"n"(N) : "memory"); };
    const auto help = [&] {
        if constexpr (!REST && N > 32) {
            meet();
            const float from = again_from;
            if (from != from) return;
            const unsigned long long n = read_again(from, again_least);
            if (threadIdx.x % 32 == 0) whole_of[threadIdx.x / 32] = n;
            meet();
        }
    };

    // the warps' sums, and from here on one warp
    const int lane = threadIdx.x % 32, warp = N == 32 ? 0 : threadIdx.x / 32;
    Group<32> one(nullptr);
    float m, sum_t, sum_1;
    {
        float top[1] = {sum.m};
        one.max(top);
        const float zt = sum.zt.x + sum.zt.y, z1 = sum.z1.x + sum.z1.y;
        float z[2] = {zt == 0.0f ? 0.0f : zt * factor(sum.m, top[0], a.ct), !HARD || z1 == 0.0f ? 0.0f : z1 * factor(sum.m, top[0], a.c1)};
        one.sum(z);
        m = top[0], sum_t = z[0], sum_1 = z[1];
    }
    const auto joined = [&](const float (*of)[3], int n) {
        m = kNone;
        for (int i = 0; i < n; ++i) m = fmaxf(m, of[i][0]);
        sum_t = sum_1 = 0;
        for (int i = 0; i < n; ++i) {
            sum_t += of[i][1] == 0.0f ? 0.0f : of[i][1] * factor(of[i][0], m, a.ct);
            sum_1 += of[i][2] == 0.0f ? 0.0f : of[i][2] * factor(of[i][0], m, a.c1);
        }
    };
    if constexpr (N == 32) {
        g.sync();
    } else {
        if (lane == 0) sums[0][warp][0] = m, sums[0][warp][1] = sum_t, sums[0][warp][2] = sum_1;
        __syncthreads();
        if (a.parts == 1 && warp) return help();
        joined(sums[0], kWarps);
        if (a.parts > 1) {                            // the parts' sums, in the first CTA of the cluster
            cg::cluster_group cluster = cg::this_cluster();
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
            if (threadIdx.x == 0) {
                float* to0 = cluster.map_shared_rank(&parts[part][0], 0);
                to0[0] = m, to0[1] = sum_t, to0[2] = sum_1;
            }
            cluster.sync();
            if (part) return;
            if (warp) return help();
            joined(parts, a.parts);
        }
    }
    float top[2] = {rest, kNone};                     // the largest of the teacher's, and of the kept classes' logits
    for (int k = lane; k < a.kept; k += 32) top[0] = fmaxf(top[0], us[k]), top[1] = fmaxf(top[1], xs[k]);
    one.max(top);
    const float mu = reference(top[0]), mx = reference(top[1]);
    float total[4] = {0, 0, 0, 0};                    // of the teacher's masses; of the kept classes' at T and at 1, or of the logarithms' sizes; of p (log p - log q)
    for (int k = lane; k < a.kept; k += 32) {
        if (kept[k] < 0) continue;
        const float u = us[k], x = xs[k], e = power(u, mu, a.c1);
        total[0] += e;
        if (REST && !came[k]) {
            total[1] += power(x, mx, a.ct);
            if (HARD) total[2] += power(x, mx, a.c1);
        }
        if (!REST && e != 0.0f) {
            const float log_p = u - mu, log_q = (x - mx) * a.inv_t;
            total[1] -= e * (log_p + log_q);
            total[3] += e * (log_p - log_q);
        }
    }
    one.sum(total);
    const float other = m, other_t = sum_t;           // without `rest` the classes seen are all there are
    float kept_t = 0;
    if (REST) {
        m = fmaxf(m, top[1]);
        kept_t = total[1] == 0.0f ? 0.0f : total[1] * factor(top[1], m, a.ct);
        sum_t = (other_t == 0.0f ? 0.0f : other_t * factor(other, m, a.ct)) + kept_t;
        sum_1 = (sum_1 == 0.0f ? 0.0f : sum_1 * factor(other, m, a.c1)) + (total[2] == 0.0f ? 0.0f : total[2] * factor(top[1], m, a.c1));
    }
    if (!HARD) sum_1 = sum_t;
    float loss = 0;
    const bool weighed = taught && a.soft_loss != 0.0f;     // (no weight takes no part, an infinite one neither)
    const auto term = [](float p, float q, float delta, bool with_q) {     // p f(delta) = q - p - p delta
        if (p == 0.0f) return with_q ? q : 0.0f;
        if (with_q && fabsf(delta) < 0.25f)           // (e^delta - 1 - delta) / (delta^2 / 2) by its series, to delta^7 / 181440
            return p * delta * delta * fmaf(delta, fmaf(delta, fmaf(delta, fmaf(delta, fmaf(delta, fmaf(delta, 1.0f / 40320, 1.0f / 5040), 1.0f / 720),
                                                                               1.0f / 120), 1.0f / 24), 1.0f / 6), 0.5f);
        return (with_q ? q : 0.0f) - fmaf(p, delta, p);
    };
    if (REST && weighed) {
        // both sides are whole distributions over the kept classes and the others
        const float e0 = factor(rest, mu, a.c1), whole = total[0] + e0, per_t = 1.0f / sum_t, level = logf(sum_t / whole);
        float kl[1] = {0};
        for (int k = lane; k < a.kept; k += 32)
            if (kept[k] >= 0) {
                const float u = us[k], x = xs[k];
                kl[0] += term(power(u, mu, a.c1) / whole, power(x, reference(m), a.ct) * per_t, (x - m) * a.inv_t - (u - mu) - level, !came[k]);
            }
        if (lane == 0) {
            const float others = other_t * factor(other, m, a.ct);      // (of nothing: 0 times 0)
            // log p_0 and log q_0 as those of one minus what the kept classes have, and by their exponents where hardly
            // anything is left, or less than fp32 holds
            const float log_p = e0 > 1e-30f ? -log1pf(total[0] / e0) : (rest - mu) - logf(whole);
            const float log_q = others > 1e-30f ? -log1pf(kept_t / others) : (other - m) * a.inv_t + logf(other_t) - logf(sum_t);
            kl[0] += term(e0 / whole, others * per_t, log_q - log_p, true);
        }
        one.sum(kl);
        loss = a.soft_loss * kl[0];
    }
    if constexpr (!REST) {
        // As its logarithms stand the divergence is off by two or three roundings of 1 and their size as a rule; where it is below 2^-8 of
        // that it is summed by its positive terms, sum p f(delta) + 1 - sum q over the teacher's entries.
        // (Where Z_T is above 1024 the kept classes have a quarter at most, and the divergence is no less than log 4: the integers'
        // sums stay below 2^63.)
        bool again = false;
        if (weighed) {
            const float whole = total[0], kl = fmaf(whole, (m - mx) * a.inv_t, total[3]) / whole - logf(whole) + logf(sum_t);
            again = sum_t <= 1024.0f && kl < 0x1p-8f * (1.0f + total[1] / whole);
            loss = a.soft_loss * kl;
        }
        float least = INFINITY;
        if (again) {                                  // (the same in all lanes)
            for (int k = lane; k < a.kept; k += 32)
                if (kept[k] >= 0 && power(us[k], mu, a.c1) != 0.0f) least = fminf(least, xs[k]);
#pragma unroll
            for (int o = 16; o; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
        }
        if constexpr (N > 32) {
            if (lane == 0) again_from = again ? m : NAN, again_least = least;
            meet();
        }
        if (again) {
            unsigned long long left = read_again(m, least);
            if constexpr (N > 32) {
                meet();
                for (int w = 1; w < kWarps; ++w) left += whole_of[w];
            }
            const float whole = total[0], per_t = 1.0f / sum_t, level = logf(sum_t / whole);
            float kl[1] = {0};
            unsigned long long own = 0;
            for (int k = lane; k < a.kept; k += 32) {
                const float u = us[k], x = xs[k], mass = kept[k] < 0 ? 0.0f : power(u, mu, a.c1);
                if (mass == 0.0f) continue;
                kl[0] += term(mass / whole, power(x, m, a.ct) * per_t, (x - m) * a.inv_t - (u - mu) - level, true);
                own += unit(x, m);
            }
            one.sum(kl);
#pragma unroll
            for (int o = 16; o; o >>= 1) own += __shfl_xor_sync(0xffffffffu, own, o);
            loss = a.soft_loss * fmaf((float)(long long)(left - own) * 0x1p-52f, per_t, kl[0]);
        }
    }
    if (lane) return;
    if (label >= 0 && a.hard != 0.0f) loss += a.hard * (logf(sum_1) - (widen(s[label]) - m));
    a.loss[row] = loss;
    float* out = a.stats + (int64_t)row * 5;
    out[0] = m;
    out[1] = a.labels ? sum_1 : 0.0f;
    out[2] = sum_t;
    out[3] = other;
    out[4] = other_t;
}

template <typename T, bool REST, int HARD>
cudaError_t launch(DistillArgs a, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    const int vectors = (a.classes + 2 * W - 2) / W;  // of a row, wherever it begins
    a.parts = 1;
    // a warp where there are rows enough, or hardly any classes (8192 x 1000 fp32: 18.5 us, by a CTA 33; 8192 x 4000 39 and 47; 1216 x
    // 4000 8.5 and 8.2; 512 x 1000 6.4 and 6.0)
    if (vectors <= kMostOfWarp && a.kept <= 32 && (a.rows >= 8 * kSMs || a.classes <= 256)) {
        const size_t smem = REST ? kRowsOfCta * kBitsOfWarp * 4 : 0;
        distill_rows<T, REST, HARD, 32><<<(a.rows + kRowsOfCta - 1) / kRowsOfCta, 32 * kRowsOfCta, smem, st>>>(a);
        return cudaGetLastError();
    }
    // few long rows: a cluster of CTAs has one (6 x 200001 fp32: 42 us by one CTA, 12.9 by eight; 160 x 100000 26 by one, 20 by two,
    // 16 by four; but 400 x 65536 bf16 15.9 by one, 16.9 by two, 20.8 by four)
    while (a.parts < 8 && (int64_t)a.rows * a.parts < 3 * kSMs && a.classes / a.parts >= 4096 * 2) a.parts *= 2;
    const int each = (vectors + a.parts - 1) / a.parts;
    // Whole rows on their way to L2 are good as long as L2 holds those of all CTAs under way (8192 x 10000 fp32: 73 us, step by step 75; 6 x
    // 200001 18.2 and 19.5), and crowd one another out beyond that (2000 x 131072 bf16: 130 and 93; 4096 x 32768 65 and 61).
    a.stepwise = std::min((int64_t)a.rows, 8 * (int64_t)kSMs / a.parts) * vectors * 16 > (64 << 20);
    const size_t smem = REST ? ((size_t)each + 31) / 32 * 4 : 0;    // at most 32 KB
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.rows * (unsigned)a.parts);
    cfg.blockDim = dim3(kWide);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.parts > 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, distill_rows<T, REST, HARD, kWide>, a), l = cudaGetLastError();
    return e != cudaSuccess ? e : l;
}

template <typename T, bool REST>
cudaError_t forward(const DistillArgs& a, cudaStream_t st) {
    const float t = a.c1 / a.ct;
    if (!a.labels || t == 1.0f) return launch<T, REST, kNoHard>(a, st);
    if (t == 2.0f) return launch<T, REST, kSquare>(a, st);
    if (t == 4.0f) return launch<T, REST, kFourth>(a, st);
    return launch<T, REST, kApart>(a, st);
}
template <typename T>
cudaError_t forward(const DistillArgs& a, cudaStream_t st) {
    return a.rest ? forward<T, true>(a, st) : forward<T, false>(a, st);
}

int check(const void* s, int64_t stride, int dtype, int64_t rows, int64_t classes, int kept, const void* values, int value_type,
          const int* indices, const float* rest, const int64_t* labels, double temperature, double alpha) {
    if (!known(dtype) || !known(value_type)) return PP_ERR_DTYPE;
    if (rows < 0 || rows > (1 << 27) || classes < 1 || classes > kMostClasses || kept < 1 || kept > kMostKept || kept > classes ||
        !apart(rows, stride, classes))
        return PP_ERR_SHAPE;
    if (!(temperature >= 1e-3 && temperature <= 1e3) || !(alpha >= 0 && alpha <= 1)) return PP_ERR_ARG;
    if (!rows) return PP_OK;
    if (!s || !values || !indices) return PP_ERR_NULL;
    if (off(s, size_of(dtype)) || off(values, size_of(value_type)) || off(indices, 4) || off(rest, 4) || off(labels, 8))
        return PP_ERR_ALIGN;
    return PP_OK;
}

DistillArgs args_of(const void* s, int64_t stride, int64_t rows, int64_t classes, int kept, const void* values, int value_type,
                    const int* indices, const float* rest, const int64_t* labels, double temperature, double alpha) {
    DistillArgs a{};
    a.s = s;
    a.stride = rows > 1 ? stride : classes;
    a.rows = (int)rows;
    a.classes = (int)classes;
    a.kept = kept;
    a.value_type = value_type;
    a.values = values;
    a.indices = indices;
    a.rest = rest;
    a.labels = labels;
    const double log2e = 1.4426950408889634;
    a.c1 = (float)log2e;
    a.ct = (float)(log2e / temperature);
    a.inv_t = (float)(1 / temperature);
    a.hard = labels ? (float)(1 - alpha) : 0.0f;
    a.soft_loss = (float)(alpha * temperature * temperature);
    a.soft_slope = (float)(alpha * temperature);
    return a;
}

}  // namespace

cudaError_t distill_forward(const DistillArgs& a, int dtype, cudaStream_t st) {
    return dtype == PP_F32 ? forward<float>(a, st) : dtype == PP_F16 ? forward<__half>(a, st) : forward<__nv_bfloat16>(a, st);
}

}  // namespace patconv

using namespace patconv;

extern "C" {

int pp_distill(const void* logits, int64_t stride, int dtype, int64_t rows, int64_t classes, const void* values, int value_type,
               const int* indices, int kept, const float* rest, const int64_t* labels, double temperature, double alpha,
               float* loss, float* stats, void* stream) {
    if (const int e = check(logits, stride, dtype, rows, classes, kept, values, value_type, indices, rest, labels, temperature, alpha))
        return e;
    if (!rows) return PP_OK;
    if (!loss || !stats) return PP_ERR_NULL;
    if (off(loss, 4) || off(stats, 4)) return PP_ERR_ALIGN;
    const size_t sb = (size_t)row_extent(rows, stride, classes) * size_of(dtype), lb = (size_t)rows * 4;
    const struct { const void* p; size_t n; } in[] = {{logits, sb}, {values, lb / 4 * kept * size_of(value_type)}, {indices, lb * kept},
                                                      {rest, rest ? lb : 0}, {labels, labels ? 2 * lb : 0}};
    for (const auto& i : in)
        if (overlap(i.p, i.n, loss, lb) || overlap(i.p, i.n, stats, 5 * lb)) return PP_ERR_BUFFER;
    if (overlap(loss, lb, stats, 5 * lb)) return PP_ERR_BUFFER;
    DistillArgs a = args_of(logits, stride, rows, classes, kept, values, value_type, indices, rest, labels, temperature, alpha);
    a.loss = loss;
    a.stats = stats;
    return distill_forward(a, dtype, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

int pp_distill_backward(const float* dloss, int64_t dloss_stride, const void* logits, int64_t stride, int dtype, int64_t rows,
                        int64_t classes, const float* stats, const void* values, int value_type, const int* indices, int kept,
                        const float* rest, const int64_t* labels, double temperature, double alpha, void* dlogits, void* stream) {
    if (const int e = check(logits, stride, dtype, rows, classes, kept, values, value_type, indices, rest, labels, temperature, alpha))
        return e;
    if (!apart(rows, dloss_stride, 0)) return PP_ERR_SHAPE;
    if (!rows) return PP_OK;
    if (!dloss || !stats || !dlogits) return PP_ERR_NULL;
    if (off(dloss, 4) || off(stats, 4) || off(dlogits, size_of(dtype))) return PP_ERR_ALIGN;
    const size_t es = size_of(dtype), lb = (size_t)rows * 4, ob = (size_t)rows * classes * es;
    const bool over = dlogits == logits && (rows == 1 || stride == classes);      // every logit is read before it is written
    const struct { const void* p; size_t n; } in[] = {{logits, over ? 0 : (size_t)row_extent(rows, stride, classes) * es},
                                                      {values, lb / 4 * kept * size_of(value_type)}, {indices, lb * kept},
                                                      {rest, rest ? lb : 0}, {labels, labels ? 2 * lb : 0}, {stats, 5 * lb},
                                                      {dloss, (size_t)row_extent(rows, dloss_stride, 1) * 4}};
    for (const auto& i : in)
        if (overlap(i.p, i.n, dlogits, ob)) return PP_ERR_BUFFER;
    DistillArgs a = args_of(logits, stride, rows, classes, kept, values, value_type, indices, rest, labels, temperature, alpha);
    a.dloss = dloss;
    a.dloss_stride = dloss_stride;
    a.stats = const_cast<float*>(stats);
    a.ds = dlogits;
    return distill_backward(a, dtype, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}

}  // extern "C"
