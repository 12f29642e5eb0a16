// A teacher's top logits: of each row the k largest, in order, ties to the lowest index, their places, and the
// log-sum-exp of the others at a temperature, which with them is all that a distillation loss needs of the row.
//
// Values are compared as keys, integers in the same order: -0 and 0 are one, a NaN is above everything.
// A row is taken by a warp, a CTA or a cluster of CTAs, each its slice.  It is read twice: the second time from shared memory
// where its slice is of 16 KB at most, else from L2, which holds the rows that are under way.
//   1. A thread takes the largest of its values.  A bound that at least k + 1 of these reach, and not many more, is found
//      by halving their range and counting: at least k + 1 values of the row reach it, and few more on rows in no special order.
//   2. The values that reach it are listed, the exponentials of all others summed relative to it.
//   3. The listed values' ranks are counted: that orders the first k, and those after them join the others' sum, in order.
// Where more values reach the bound than the list holds (many equal ones, or the large ones all in a few threads'
// places), the (k + 1)-th in order is found by halving the keys' range, and the places' among its equals: 32 and at
// most 20 countings, which any row ends after.
//
// What bounds it: of many rows the two readings and the exponentials, about five instructions a value, beside memory; of few the
// chain of barriers.  4096 x 32768 bf16 with 64 kept takes 79 us, 3.4 TB/s of the 268 MB that have to be read (40 us at a copy's
// rate), 256 x 1000 fp32 with 16 kept 5.7 us, 6 x 200001 fp32 with 200 kept 12.4 (GPU time, calls one after another in one graph).  Rows of 64 KB held in shared memory, one reading but fewer rows under way, took
// 114 us where this took 94.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>

#include "rows.cuh"

namespace patconv {
namespace {

namespace cg = cooperative_groups;

constexpr int kClusterMost = 8;
constexpr size_t kHeld = 16 * 1024;   // bytes of a CTA's slice in shared memory at most: eight CTAs on an SM

struct TopArgs {
    const void* s;
    int64_t stride;
    int rows, classes, k;
    float c, inv_t;                   // log2(e) / T, 1 / T
    void* values;                     // [rows][k] of the logits' type
    int* indices;                     // [rows][k]
    float* rest;                      // [rows]
    int parts;                        // CTAs of a row, a cluster
    int held;                         // bytes of a slice that is kept in shared memory, 0: it is not
    int list;                         // values that reach the bound at most: 512, of a warp's row 256, of 512 threads' 1024
};

// an integer in the values' order
__device__ __forceinline__ int key_of(float x) {
    const int b = __float_as_int(x + 0.0f);          // -0 becomes 0
    return x == x ? b ^ ((b >> 31) & 0x7FFFFFFF) : INT_MAX;
}
__device__ __forceinline__ float of_key(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }
constexpr int kLeast = INT_MIN;       // below every key

// what the CTAs of a row tell one another
struct Shared {
    int found;                        // how many values are listed (the first CTA's)
    int flagged;                      // how many vectors of this CTA are noted
    unsigned long long beside;        // the sum of their other values' exponentials, in units of 2^-46
    int bounds[kClusterMost];
    int counted[2][kClusterMost];
    float sums[kClusterMost];         // of the values that are not listed (the first CTA's)
};

template <typename T, int N>
__global__ void __launch_bounds__(N, N == 32 ? 24 : N == 128 ? 8 : N == 256 ? 4 : 2) top_rows(TopArgs a) {
    constexpr int W = 16 / sizeof(T), kWarps = N / 32, U = N == 128 ? 8 : 4;
    extern __shared__ uint4 dynamic[];
    __shared__ Shared sh;
    __shared__ float scratch[2 * kWarps * 8];
    __shared__ int warp_counts[2][kWarps], warp_ends[2][kWarps];
    cg::cluster_group cluster = cg::this_cluster();
    const int part = blockIdx.x % a.parts, row = blockIdx.x / a.parts, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const T* s = static_cast<const T*>(a.s) + row * a.stride;
    const Row<T, W> r(s, a.classes);
    const int each = (r.vectors() + a.parts - 1) / a.parts, first = min(r.vectors(), part * each), last = min(r.vectors(), first + each);
    const int wanted = min(a.k + 1, a.classes);       // values to put in order: the kept ones and the one after them
    Vec<T, W>* held = reinterpret_cast<Vec<T, W>*>(dynamic);
    const auto everyone = [&] {
        if (a.parts > 1)
            cluster.sync();
        else
            __syncthreads();
    };
    // (key, ~place) of the values that reach the bound, the first CTA's those of all; the vectors that hold some; at the end, of
    // the values those after the k-th, in order, in the vectors' place
    unsigned long long* list = reinterpret_cast<unsigned long long*>(reinterpret_cast<char*>(dynamic) + a.held);
    int* noted = reinterpret_cast<int*>(list + a.list);
    float* after = reinterpret_cast<float*>(noted);
    const auto of = [&](int p) { return a.parts > 1 ? cluster.map_shared_rank(&sh, p) : &sh; };

    // 1. the largest of each thread's values; all of the slice goes to shared memory
    if (threadIdx.x == 0) sh.found = sh.flagged = 0, sh.beside = 0;
    Largest<T> seen;
    if (threadIdx.x == 0) r.prefetch(first, last);    // all on their way to L2
    // the ends of a row that are no whole vectors are taken by themselves
    const int from = first < last && !r.whole(first) ? first + 1 : first;
    const int to = last > from && !r.whole(last - 1) ? last - 1 : last;
    const auto first_seen = [&](int v, const Vec<T, W>& b) {
        seen.take(b);
        if (a.held) memcpy(held + (v - first), &b, 16);
    };
    int v = from + threadIdx.x;
    for (; v + (U - 1) * N < to; v += U * N) {
        Vec<T, W> b[U];
#pragma unroll
        for (int k = 0; k < U; ++k) b[k] = r.at(v + k * N);
#pragma unroll
        for (int k = 0; k < U; ++k) first_seen(v + k * N, b[k]);
    }
    for (; v < to; v += N) first_seen(v, r.at(v));
    if (from > first && threadIdx.x == 0) first_seen(first, r.some(first));
    if (to < last && threadIdx.x == N - 1) first_seen(to, r.some(to));

    // the bound: this CTA's share of the values wanted reach it here, so that all of them do where the least of the CTAs' does
    const int share = (wanted + a.parts - 1) / a.parts, own = min(N, to - from);
    const int key = (int)threadIdx.x < own ? key_of(seen.get()) : kLeast;
    int bound = kLeast;
    {
        const int high_lane = __reduce_max_sync(0xffffffffu, key), low_lane = __reduce_min_sync(0xffffffffu, (int)threadIdx.x < own ? key : INT_MAX);
        if (lane == 0) warp_ends[0][warp] = low_lane, warp_ends[1][warp] = high_lane;
        __syncthreads();
        long long low = INT_MAX, high = INT_MIN;
        for (int w = 0; w < kWarps; ++w) low = min(low, (long long)warp_ends[0][w]), high = max(high, (long long)warp_ends[1][w]);
        ++high;
        // the range's halves until `counted` says that `share` or few more reach it
        const auto halve = [&](int slack, const auto& counted) {       // `share` reach low, and not high
            for (int k = 0; k < 20 && high - low > 1; ++k) {
                const int middle = (int)((low + high) >> 1), n = counted(middle);
                if (n >= share)
                    low = middle;
                else
                    high = middle;
                if (n >= share && n <= share + slack) break;
            }
            bound = (int)low;
        };
        // a short row has as many vectors as values are wanted, or fewer: its values themselves are counted
        if (4 * own >= 5 * share) {
            // (where nearly all of the threads' reach it, of their other values many do)
            halve(max(2, min(share / 4, (own - share) / 8)), [&](int middle) { return __syncthreads_count(key >= middle); });
        } else if (a.parts == 1 && a.held && a.classes > 2 * share) {
            int turn = 0;
            low = kLeast;
            halve(max(2, share / 4), [&](int middle) {
                int n = 0;
                for (int v = first + threadIdx.x; v < last; v += N) {
                    const Vec<T, W> b = held[v - first];
#pragma unroll
                    for (int i = 0; i < W; ++i) n += key_of(widen(b.v[i])) >= middle && v * W + i >= r.pad && v * W + i < r.end;
                }
                n = __reduce_add_sync(0xffffffffu, n);
                turn ^= 1;
                if (lane == 0) warp_counts[turn][warp] = n;
                __syncthreads();
                n = 0;
                for (int w = 0; w < kWarps; ++w) n += warp_counts[turn][w];
                return n;
            });
        }
    }
    if (a.parts > 1) {
        cluster.sync();                               // every CTA has begun: its memory can be written
        if (threadIdx.x < a.parts) of(threadIdx.x)->bounds[part] = bound;
        cluster.sync();
        for (int p = 0; p < a.parts; ++p) bound = min(bound, sh.bounds[p]);
    }

    // 2. what is listed: the values that reach `bound`; the sum of the others.  A vector below the bound, as nearly all are, is
    // summed as it is read; the others are noted, and all threads go through their values afterwards.
    Shared* leader = of(0);
    unsigned long long* leader_list = a.parts > 1 ? cluster.map_shared_rank(list, 0) : list;
    Group<N> g(scratch);
    const float2 ct = both(a.c);
    const auto middle_at = [&](int v) {               // a whole one
        const uint4 w = a.held ? *reinterpret_cast<const uint4*>(held + (v - first)) : *reinterpret_cast<const uint4*>(r.base + (int64_t)v * W);
        Vec<T, W> b;
        memcpy(&b, &w, 16);
        return b;
    };
    const auto vector_at = [&](int v) { return r.whole(v) ? middle_at(v) : r.some(v); };
    const auto add_vector = [&](float2& sum, const Vec<T, W>& b, float2 far) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            const float2 e = mul(add(pair(b, i), far), ct);
            sum = add(sum, make_float2(approx_exp2(e.x), approx_exp2(e.y)));
        }
    };
    const auto entry = [](int key, int place) { return (unsigned long long)((unsigned)key ^ 0x80000000u) << 32 | (unsigned)~place; };
    const auto tell = [&](float2 sum) {               // every thread's sum, to the first CTA; how many values are listed
        float total[1] = {sum.x + sum.y};
        g.sum(total);
        if (threadIdx.x == 0) leader->sums[part] = total[0] + (float)sh.beside * 0x1p-46f;
        everyone();
        return leader->found;
    };
    const auto collect = [&](int bound) {
        const float limit = of_key(bound), below = reference(limit);
        const float2 far = both(-below);
        float2 sum = make_float2(0.0f, 0.0f);
        // a thread remembers which of its vectors reach the bound, 32 at a time, and notes them then
        unsigned reached = 0;
        const auto take = [&](const Vec<T, W>& b, int turn) {
            if (bound != kLeast && largest(b) < limit)                 // (places beside the row hold -inf, which adds nothing)
                add_vector(sum, b, far);
            else
                reached |= 1u << turn;
        };
        const auto noted_from = [&](int v) {          // vectors v, v + N and so on
            const int mine = __popc(reached);
            if (!__any_sync(0xffffffffu, mine)) return;
            int before = mine;                        // of the lanes up to this one
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int y = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += y;
            }
            int n = lane == 31 ? atomicAdd(&sh.flagged, before) : 0;
            n = __shfl_sync(0xffffffffu, n, 31) + before - mine;
            for (; reached; reached &= reached - 1, ++n)
                if (n < a.list) noted[n] = v + (__ffs(reached) - 1) * N;
        };
        for (int base = from; base < to; base += 32 * N) {             // (the same for all threads)
            const int v = base + threadIdx.x;
            int turn = 0;
#pragma unroll 1
            for (; turn < 33 - U && v + (turn + U - 1) * N < to; turn += U) {
                Vec<T, W> b[U];
#pragma unroll
                for (int k = 0; k < U; ++k) b[k] = middle_at(v + (turn + k) * N);
#pragma unroll
                for (int k = 0; k < U; ++k) take(b[k], turn + k);
            }
#pragma unroll 1
            for (; turn < 32 && v + turn * N < to; ++turn) take(middle_at(v + turn * N), turn);
            noted_from(v);
        }
        if (from > first) {                           // the ends
            if (threadIdx.x == 0) take(r.some(first), 0);
            noted_from(first);
        }
        if (to < last) {
            if (threadIdx.x == N - 1) take(r.some(to), 0);
            noted_from(to);
        }
        __syncthreads();
        const int flagged = sh.flagged, vectors = min(flagged, a.list);
        if (flagged > a.list && threadIdx.x == 0) atomicAdd(&leader->found, flagged);     // each has one at least
        // the noted vectors' values, M of them a thread
        const auto examine = [&](auto m) {
            constexpr int M = decltype(m)::value;
            for (int i = threadIdx.x; i - lane < vectors * (W / M); i += N) {      // (whole warps)
                const bool here = i < vectors * (W / M);
                const int v = here ? noted[i / (W / M)] : first, k0 = M == 1 ? i % W : 0;
                Vec<T, M> b;
                if constexpr (M == W) {
                    b = vector_at(v);
                } else {
                    const int place = v * W + k0;
                    b.v[0] = a.held ? held[v - first].v[k0] : place >= r.pad && place < r.end ? r.base[place] : T(kNone);
                }
                // integers: the vectors are noted in no order.  22 bits and 24 more: 256 values are below 2^32, 8192 of both below 2^60
                unsigned high = 0, low = 0, those = 0;
#pragma unroll
                for (int k = 0; k < M; ++k) {
                    const int place = v * W + k0 + k;
                    const float x = widen(b.v[k]);
                    if (!here || place < r.pad || place >= r.end) continue;
                    if (key_of(x) >= bound) {
                        those |= 1u << k;
                    } else {
                        const float e = power(x, below, a.c) * 4194304.0f, whole = truncf(e);
                        high += (unsigned)whole;
                        low += (unsigned)((e - whole) * 16777216.0f);
                    }
                }
                int up_to = __popc(those);            // of the lanes up to this one
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int y = __shfl_up_sync(0xffffffffu, up_to, o);
                    if (lane >= o) up_to += y;
                }
                int n = lane == 31 && up_to ? atomicAdd(&leader->found, up_to) : 0;
                n = __shfl_sync(0xffffffffu, n, 31) + up_to - __popc(those);
                for (; those; those &= those - 1, ++n) {
                    const int k = __ffs(those) - 1;
                    if (n < a.list) leader_list[n] = entry(key_of(widen(b.v[k])), v * W + k0 + k - r.pad);
                }
                high = __reduce_add_sync(0xffffffffu, high);
                low = __reduce_add_sync(0xffffffffu, low);
                if (lane == 0 && (high | low)) atomicAdd(&sh.beside, ((unsigned long long)high << 24) + low);
            }
        };
        // a thread has one where that takes two turns at most, else a vector (4096 x 32768 bf16 with 10 kept: 65 us, by vectors 71;
        // with 64 92 and 80, with 250 273 and 218)
        if (vectors * W <= 2 * N)
            examine(std::integral_constant<int, 1>());
        else
            examine(std::integral_constant<int, W>());
        __syncthreads();
        return tell(sum);
    };
    // the same, where ever so many equal one another: the values above key `bound`, and of those with this key the ones up to
    // place `until`
    const auto collect_exactly = [&](int bound, int until) {
        const float below = reference(of_key(bound));
        float2 sum = make_float2(0.0f, 0.0f);
        for (int v = first + threadIdx.x; v < last; v += N) {
            const Vec<T, W> b = vector_at(v);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int place = v * W + i - r.pad;
                if (place < 0 || place >= a.classes) continue;
                const float x = widen(b.v[i]);
                const int key = key_of(x);
                if (key > bound || (key == bound && place <= until)) {
                    const int n = atomicAdd(&leader->found, 1);
                    if (n < a.list) leader_list[n] = entry(key, place);
                } else {
                    sum.x += power(x, below, a.c);
                }
            }
        }
        return tell(sum);
    };
    int all = collect(bound);
    if (all > a.list) {                                // the same in every CTA of the row
        int turn = 0;
        const auto counted = [&](auto&& pred) {       // how many of the row's values are so, to every thread
            int n = 0;
            for (int v = first + threadIdx.x; v < last; v += N) {
                const Vec<T, W> b = vector_at(v);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const int place = v * W + i - r.pad;
                    n += place >= 0 && place < a.classes && pred(key_of(widen(b.v[i])), place);
                }
            }
            n = __reduce_add_sync(0xffffffffu, n);
            turn ^= 1;
            if (lane == 0) warp_counts[turn][warp] = n;
            __syncthreads();
            n = 0;
            for (int w = 0; w < kWarps; ++w) n += warp_counts[turn][w];
            if (a.parts > 1) {
                if (threadIdx.x < a.parts) of(threadIdx.x)->counted[turn][part] = n;
                cluster.sync();
                n = 0;
                for (int p = 0; p < a.parts; ++p) n += sh.counted[turn][p];
            }
            return n;
        };
        // the largest key that `wanted` values reach
        int low = kLeast, high = INT_MAX;
        while (low < high) {
            const int middle = (int)(((long long)low + high + 1) >> 1);
            if (counted([&](int key, int) { return key >= middle; }) >= wanted)
                low = middle;
            else
                high = middle - 1;
        }
        const int above = low == INT_MAX ? 0 : counted([&](int key, int) { return key > low; });
        // the least place up to which there are enough of the values of that key
        int left = 0, right = a.classes - 1;
        while (left < right) {
            const int middle = (left + right) / 2;
            if (above + counted([&](int key, int place) { return key == low && place <= middle; }) >= wanted)
                right = middle;
            else
                left = middle + 1;
        }
        if (threadIdx.x == 0) sh.found = 0, sh.beside = 0;
        everyone();
        bound = low;
        all = collect_exactly(low, left);
    }

    // 3. the listed values in order
    if (part == 0) {
        T* values = static_cast<T*>(a.values) + (int64_t)row * a.k;
        int* indices = a.indices + (int64_t)row * a.k;
        if (threadIdx.x == 0 && all % 2) list[all] = 0;                // (the list's room is even) above no value
        __syncthreads();
        for (int i = threadIdx.x; i < all; i += N) {
            const unsigned long long mine = list[i];
            int rank = 0;
#pragma unroll 4
            for (int n = 0; n < all; n += 2) {
                const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(list + n);
                rank += (two.x > mine) + (two.y > mine);
            }
            if (rank < a.k) {
                const int place = (int)~(unsigned)mine;
                values[rank] = s[place];
                indices[rank] = place;
            } else {
                after[rank - a.k] = of_key((int)((unsigned)(mine >> 32) ^ 0x80000000u));
            }
        }
        __syncthreads();
        if (a.k == a.classes) {
            if (threadIdx.x == 0) a.rest[row] = kNone;
        } else {
            const float m = after[0], below = reference(m);
            float sum[1] = {0};
            for (int i = threadIdx.x; i < all - a.k; i += N) sum[0] += power(after[i], below, a.c);
            g.sum(sum);
            if (threadIdx.x == 0) {
                float others = 0;
                for (int p = 0; p < a.parts; ++p) others += sh.sums[p];
                if (others != 0.0f) others *= factor(of_key(bound), m, a.c);
                a.rest[row] = fabsf(m) == INFINITY ? m : m * a.inv_t + logf(sum[0] + others);
            }
        }
    }
    if (a.parts > 1) cluster.sync();                  // the first CTA's memory has been read by the others
}

template <typename T>
int vectors_of(const TopArgs& a) {                    // of a row, wherever it begins
    constexpr int W = 16 / sizeof(T);
    return (a.classes + 2 * W - 2) / W;
}
template <typename T, int N>
cudaError_t launch(TopArgs a, cudaStream_t st) {
    const size_t slice = (size_t)((vectors_of<T>(a) + a.parts - 1) / a.parts) * 16;
    a.held = slice <= kHeld ? (int)slice : 0;
    a.list = N == 32 ? 256 : N < 512 ? 512 : 1024;
    constexpr int kLists = 1024 * 12;
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    if (const cudaError_t e = cudaGetDevice(&dev)) return e;
    if (dev >= 64 || !(allowed.load() >> dev & 1)) {
        if (const cudaError_t e = cudaFuncSetAttribute(top_rows<T, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kHeld + kLists)) {
            cudaGetLastError();
            return e;
        }
        if (dev < 64) allowed.fetch_or(uint64_t(1) << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.rows * (unsigned)a.parts);
    cfg.blockDim = dim3(N);
    cfg.dynamicSmemBytes = a.held + a.list * 12;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.parts > 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, top_rows<T, N>, a), l = cudaGetLastError();
    return e != cudaSuccess ? e : l;
}
template <typename T>
cudaError_t top(TopArgs a, cudaStream_t st) {
    constexpr int kThreads = 1024, kMost = 512;       // threads of an SM, and of a CTA at most
    a.parts = 1;
    // A warp where there are rows enough: 5424 x 746 takes 17 us, by 128 threads 29; 8192 x 2000 fp32 26 and 38, of bf16 22 and 37.
    // But 8192 x 4000 fp32 takes 59 and 56, and 256 x 1000 takes 10.5 and 8.4.
    if ((int64_t)vectors_of<T>(a) <= 512 && a.k < 24 && a.rows >= 8 * kSMs) return launch<T, 32>(a, st);
    // The bound is found among the threads' largest values, so there are half as many threads again as values are wanted: 256 x
    // 1000 with 95 kept takes 19 us by 128 threads and 7.7 by 256.  No more than that, as a row has its fixed work: 4096 x
    // 32768 bf16 with 60 kept takes 80 us by 128 threads and 89 by 256, with 10 65, 74 and by 512 107; but
    int n = a.k < 80 ? 128 : a.k < 160 ? 256 : kMost;
    const int64_t row = (int64_t)vectors_of<T>(a) * 16;
    // where the threads of all rows fit on the GPU, a row has more of them, eight vectors each: 64 x 32768 bf16 takes 9.6 us with 128
    // threads, 7.4 with 512,
    while (n < kMost && 2 * n * (int64_t)a.rows <= kSMs * kThreads && row >= 2 * n * 128) n *= 2;
    // and then a cluster of CTAs: 6 x 200001 takes 21.9 us by one CTA and 10.4 by eight (its barriers cost 2 us: 150 x 32768 fp32 takes
    // 8.2 us by one, 10.8 by two);
    while (a.parts < kClusterMost && n == kMost &&
           ((2 * a.parts * (int64_t)a.rows <= kSMs && row >= a.parts * (128 << 10)) ||
            (2 * a.parts * (int64_t)a.rows * n <= kSMs * kThreads && row >= a.parts * (512 << 10))))
        a.parts *= 2;
    // and the rows that are under way together stay in L2 for the second reading: 2000 x 65536 bf16 takes 94 us by 128 threads,
    // 75 by 256; 1000 x 100000 fp32 136 by 128, 130 by 512 and 120 by two CTAs of 512
    while ((n < kMost || a.parts < kClusterMost) &&
           std::min((int64_t)a.rows, kSMs * (int64_t)kThreads / n / a.parts) * row > (80 << 20)) {
        if (n < kMost)
            n *= 2;
        else
            a.parts *= 2;
    }
    return n == 128 ? launch<T, 128>(a, st) : n == 256 ? launch<T, 256>(a, st) : launch<T, kMost>(a, st);
}

}  // namespace
}  // namespace patconv

using namespace patconv;

extern "C" int pp_top_logits(const void* logits, int64_t stride, int dtype, int64_t rows, int64_t classes, int k, double temperature,
                             void* values, int* indices, float* rest, void* stream) {
    if (!known(dtype)) return PP_ERR_DTYPE;
    if (rows < 0 || rows > (1 << 27) || classes < 1 || classes > kMostClasses || k < 1 || k > kMostKept || k > classes ||
        !apart(rows, stride, classes))
        return PP_ERR_SHAPE;
    if (!(temperature >= 1e-3 && temperature <= 1e3)) return PP_ERR_ARG;
    if (!rows) return PP_OK;
    if (!logits || !values || !indices || !rest) return PP_ERR_NULL;
    const size_t es = size_of(dtype), sb = (size_t)row_extent(rows, stride, classes) * es, n = (size_t)rows;
    if (off(logits, es) || off(values, es) || off(indices, 4) || off(rest, 4)) return PP_ERR_ALIGN;
    if (overlap(logits, sb, values, n * k * es) || overlap(logits, sb, indices, n * k * 4) || overlap(logits, sb, rest, n * 4) ||
        overlap(values, n * k * es, indices, n * k * 4) || overlap(values, n * k * es, rest, n * 4) || overlap(indices, n * k * 4, rest, n * 4))
        return PP_ERR_BUFFER;
    TopArgs a{};
    a.s = logits;
    a.stride = rows > 1 ? stride : classes;
    a.rows = (int)rows;
    a.classes = (int)classes;
    a.k = k;
    a.c = (float)(1.4426950408889634 / temperature);
    a.inv_t = (float)(1 / temperature);
    a.values = values;
    a.indices = indices;
    a.rest = rest;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == PP_F32 ? top<float>(a, st) : dtype == PP_F16 ? top<__half>(a, st) : top<__nv_bfloat16>(a, st);
    return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}
