// A teacher's top logits: of each row the k largest, in order, ties to the lowest index, their places, and the
// log-sum-exp of the others at a temperature, which with them is all that a distillation loss needs of the row.
//
// Values are compared as keys, integers in the same order: -0 and 0 are one, a NaN is above everything.
// A row is read once and kept in shared memory where it fits (a cluster of CTAs has a long row, each its slice).
//   1. A thread takes the largest of its values.  With j = ceil((k + 1) / warps), the least of the warps' j-th largest
//      thread maxima is a bound that at least k + 1 values reach, and few more on rows in no special order.
//   2. The values that reach it are listed, and each one's rank among them is counted.  That orders the first k, and
//      the one after them is the largest of the others.
//   3. The others' exponentials, relative to that one, are summed.
// Where more values reach the bound than the list holds (many equal ones, or the large ones all in a few threads'
// places), the (k + 1)-th in order is found by halving the keys' range, and the places' among its equals: 32 and at
// most 20 countings, which any row ends after.
//
// What bounds it is memory, then the three readings of shared memory.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>

#include "rows.cuh"

namespace patconv {
namespace {

namespace cg = cooperative_groups;

constexpr int kList = 1024;           // values that reach the bound at most
constexpr int kClusterMost = 8;
constexpr size_t kHeld = 96 * 1024;   // bytes of a CTA's slice in shared memory at most: two CTAs on an SM

struct TopArgs {
    const void* s;
    int64_t stride;
    int rows, classes, k;
    float c, inv_t;                   // log2(e) / T, 1 / T
    void* values;                     // [rows][k] of the logits' type
    int* indices;                     // [rows][k]
    float* rest;                      // [rows]
    int parts;                        // CTAs of a row, a cluster
    int held;                         // whether a slice is kept in shared memory
};

// an integer in the values' order
__device__ __forceinline__ int key_of(float x) {
    const int b = __float_as_int(x + 0.0f);          // -0 becomes 0
    return x == x ? b ^ ((b >> 31) & 0x7FFFFFFF) : INT_MAX;
}
__device__ __forceinline__ float of_key(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }
constexpr int kLeast = INT_MIN;       // below every key

// the j-th largest (from 1) of the lanes' keys: a sorting network over the warp, the largest in lane 0
__device__ __forceinline__ int sorted(int x) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int step = size / 2; step; step /= 2) {
            const int y = __shfl_xor_sync(0xffffffffu, x, step);
            const bool larger_first = (lane & size) == 0, lower = (lane & step) == 0;
            x = larger_first == lower ? max(x, y) : min(x, y);
        }
    return x;
}

// what the CTAs of a row tell one another
struct Shared {
    unsigned long long list[kList];   // (key, ~place) of the values that reach the bound; the first CTA's: of all CTAs
    int bound[kClusterMost * 16];     // each warp's, from all CTAs
    int warps[kClusterMost];          // warps that gave a bound, of each CTA
    int counts[kClusterMost];
    int counted[2][kClusterMost];
    float sums[kClusterMost];
    int found, count;
    unsigned long long after, bottom; // the (k + 1)-th, and the last that is kept
};

template <typename T, int N>
__global__ void __launch_bounds__(N) top_rows(TopArgs a) {
    constexpr int W = 16 / sizeof(T), kWarps = N / 32, U = 4;
    extern __shared__ uint4 dynamic[];
    __shared__ Shared sh;
    __shared__ float scratch[2 * kWarps * 8];
    __shared__ int warp_counts[2][kWarps];
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
    const auto of = [&](int p) { return a.parts > 1 ? cluster.map_shared_rank(&sh, p) : &sh; };

    // 1. the largest of each thread's values; all of the slice goes to shared memory
    if (threadIdx.x == 0) sh.found = 0;
    int most = kLeast;
    const auto edge = [&](int v) {                    // a vector of which the row has a part: the rest lies outside
        Vec<T, W> b;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int place = v * W + i;
            b.v[i] = place >= r.pad && place < r.end ? r.base[place] : T(0.0f);
        }
        return b;
    };
    const auto see = [&](const Vec<T, W>& b, int v, bool whole) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int key = key_of(widen(b.v[i]));
            if (whole || (v * W + i >= r.pad && v * W + i < r.end)) most = max(most, key);
        }
        if (a.held) held[v - first] = b;
    };
    int v = first + threadIdx.x;
    for (; v + (U - 1) * N < last; v += U * N) {
        Vec<T, W> b[U];
        bool whole[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            whole[k] = r.whole(v + k * N);
            b[k] = whole[k] ? r.at(v + k * N) : edge(v + k * N);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) see(b[k], v + k * N, whole[k]);
    }
    for (; v < last; v += N) {
        const bool whole = r.whole(v);
        see(whole ? r.at(v) : edge(v), v, whole);
    }

    // the bound
    const auto full_warps = [&](int p) {              // warps of part p whose lanes all have a whole vector
        const int n = min(r.vectors(), (p + 1) * each) - min(r.vectors(), p * each) - 2;
        return n < 0 ? 0 : min(kWarps, n / 32);
    };
    int warps = 0;
    for (int p = 0; p < a.parts; ++p) warps += full_warps(p);
    const int j = warps ? (wanted + warps - 1) / warps : 33;
    const int order = sorted(most);
    if (a.parts > 1) cluster.sync();                  // every CTA has begun: its memory can be written
    if (lane == min(j, 32) - 1)
        for (int p = 0; p < a.parts; ++p) of(p)->bound[part * kWarps + warp] = j <= 32 && warp < full_warps(part) ? order : INT_MAX;
    everyone();
    int bound = INT_MAX;
    for (int w = lane; w < a.parts * kWarps; w += 32) bound = min(bound, sh.bound[w]);
    bound = __reduce_min_sync(0xffffffffu, bound);
    if (bound == INT_MAX) bound = kLeast;             // too few values for one

    // f(key, place) for each of the slice's values; from place on the row's own count
    const auto each_value = [&](auto&& f) {
        for (int v = first + threadIdx.x; v < last; v += N) {
            const bool whole = r.whole(v);
            const Vec<T, W> b = a.held ? held[v - first] : whole ? r.at(v) : edge(v);
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (whole || (v * W + i >= r.pad && v * W + i < r.end)) f(widen(b.v[i]), v * W + i - r.pad);
        }
    };
    const auto entry = [](int key, int place) {
        return (unsigned long long)((unsigned)key ^ 0x80000000u) << 32 | (unsigned)~place;
    };
    const auto list = [&](float x, int place) {
        const int n = atomicAdd(&sh.found, 1);
        if (n < kList) sh.list[n] = entry(key_of(x), place);
    };

    // 2. the values that reach the bound
    const float limit = of_key(bound);
    if (bound == kLeast)
        each_value(list);
    else
        each_value([&](float x, int place) {
            if (!(x < limit)) list(x, place);
        });
    __syncthreads();
    const auto gather = [&] {                         // all CTAs' numbers of listed values, then the lists, in the first CTA
        if (a.parts == 1) return sh.found;
        if (threadIdx.x < a.parts) of(threadIdx.x)->counts[part] = sh.found;
        cluster.sync();
        int all = 0, before = 0;
        for (int p = 0; p < a.parts; ++p) {
            if (p < part) before += sh.counts[p];
            all += sh.counts[p];
        }
        if (all <= kList) {
            if (part)
                for (int i = threadIdx.x; i < sh.found; i += N) of(0)->list[before + i] = sh.list[i];
            cluster.sync();
        }
        return all;
    };
    int all = gather();
    if (all > kList) {                                // the same in every CTA of the row
        int turn = 0;
        const auto counted = [&](auto&& pred) {       // how many of the row's values are so, to every thread
            int n = 0;
            each_value([&](float x, int place) { n += pred(key_of(x), place); });
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
        if (threadIdx.x == 0) sh.found = 0;
        everyone();
        each_value([&](float x, int place) {
            const int key = key_of(x);
            if (key > low || (key == low && place <= left)) list(x, place);
        });
        __syncthreads();
        all = gather();
    }
    if (part == 0) {
        T* values = static_cast<T*>(a.values) + (int64_t)row * a.k;
        int* indices = a.indices + (int64_t)row * a.k;
        for (int i = threadIdx.x; i < all; i += N) {
            const unsigned long long mine = sh.list[i];
            int rank = 0;
#pragma unroll 8
            for (int n = 0; n < all; ++n) rank += sh.list[n] > mine;
            if (rank < a.k) {
                const int place = (int)~(unsigned)mine;
                values[rank] = s[place];
                indices[rank] = place;
                if (rank == a.k - 1) sh.bottom = mine;
            } else if (rank == a.k) {
                sh.after = mine;
            }
        }
    }
    everyone();
    // 3. the others
    if (a.k == a.classes) {
        if (part == 0 && threadIdx.x == 0) a.rest[row] = kNone;
        return;
    }
    const Shared* leader = of(0);
    const unsigned long long bottom = leader->bottom, after = leader->after;
    const float last_kept = of_key((int)((unsigned)(bottom >> 32) ^ 0x80000000u)), m = of_key((int)((unsigned)(after >> 32) ^ 0x80000000u));
    const int last_place = (int)~(unsigned)bottom;
    const float below = reference(m);
    float sum[1] = {0};
    each_value([&](float x, int place) {
        if (x < last_kept || (!(x > last_kept) && place > last_place && key_of(x) == key_of(last_kept)) ||
            (x == x && last_kept != last_kept))
            sum[0] += power(x, below, a.c);
    });
    Group<N> g(scratch);
    g.sum(sum);
    if (a.parts > 1) {
        if (threadIdx.x == 0) of(0)->sums[part] = sum[0];
        cluster.sync();
        sum[0] = 0;
        for (int p = 0; p < a.parts; ++p) sum[0] += sh.sums[p];
    }
    if (part == 0 && threadIdx.x == 0) a.rest[row] = fabsf(m) == INFINITY ? m : m * a.inv_t + logf(sum[0]);
}

template <typename T, int N>
cudaError_t launch(TopArgs a, cudaStream_t st) {
    constexpr int W = 16 / sizeof(T);
    const int vectors = (a.classes + 2 * W - 2) / W;
    const auto slice = [&] { return (size_t)((vectors + a.parts - 1) / a.parts) * 16; };
    a.parts = 1;
    // a cluster where a slice does not fit, or where the rows are too few for the SMs
    while (N > 128 && a.parts < kClusterMost && (slice() > kHeld || ((int64_t)a.rows * a.parts < kSMs && slice() >= 16384))) a.parts *= 2;
    a.held = slice() <= kHeld;
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    if (const cudaError_t e = cudaGetDevice(&dev)) return e;
    if (dev >= 64 || !(allowed.load() >> dev & 1)) {
        if (const cudaError_t e = cudaFuncSetAttribute(top_rows<T, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kHeld)) {
            cudaGetLastError();
            return e;
        }
        if (dev < 64) allowed.fetch_or(uint64_t(1) << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.rows * (unsigned)a.parts);
    cfg.blockDim = dim3(N);
    cfg.dynamicSmemBytes = a.held ? slice() : 0;
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
cudaError_t top(const TopArgs& a, cudaStream_t st) {
    return a.classes <= 4096 ? launch<T, 128>(a, st) : launch<T, 512>(a, st);
}

}  // namespace
}  // namespace patconv

using namespace patconv;

extern "C" int pp_top_logits(const void* logits, int64_t stride, int dtype, int64_t rows, int64_t classes, int k, double temperature,
                             void* values, int* indices, float* rest, void* stream) {
    if (!known(dtype)) return PP_ERR_DTYPE;
    if (rows < 0 || rows > (1 << 27) || classes < 1 || classes > kMostClasses || k < 1 || k > kMostKept || k > classes ||
        (rows > 1 && stride < classes))
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
