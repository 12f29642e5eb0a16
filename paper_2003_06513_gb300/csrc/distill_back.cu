// The gradient of the distillation loss (distill.cu) by the logits.  With the row's gradient g, and of the forward
// pass m, Z_1, Z_T and, of the classes that are not kept, the largest logit m_o and the sum Z_o,
//     ds_v = g ((1 - alpha) (exp(s_v - m) / Z_1 - [v is the label]) + alpha T (q_v - p_v)),
// where for a class that is not kept q_v - p_v is, with the teacher's others as one class of mass p_0,
//     (q_0 - p_0) exp((s_v - m_o) / T) / Z_o,     q_0 = exp((m_o - m) / T) Z_o / Z_T,
// and without them q_v.  So every value is two exponentials times two numbers of the row; the kept classes and the
// label, which have a term of their own, are written again after their CTA's others, at a barrier.
//
// What bounds it is memory: a row is read and one of the same size written.  8192 x 65536 bf16 with 64 kept takes 334 us, 6.4 TB/s,
// 0.95 of a copy's rate; 512 x 1000 fp32 with 16 kept 4.5 us (GPU time, calls one after another in one graph).
#include <algorithm>

#include "rows.cuh"

namespace patconv {
namespace {

constexpr int kWide = 256;
constexpr int kRowsOfCta = 4;
constexpr int kMostOfWarp = 16384;    // bytes of a warp's row at most

// The 16 bytes at a place `off` bytes beyond a 16-byte boundary, from the two vectors that hold them.
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int off) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = off & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = off & 4 ? w[i + 1] : w[i];
    const int bits = off % 4 * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                      __funnelshift_r(w[3], w[4], bits));
}

// Both are read and written in 16-byte vectors, which begin at the gradient's boundaries.  SHIFT: the logits' boundaries are, or may be,
// at other places, and a vector is put together from two (1000 x 21841 fp16, rows 21844 apart: 17 us, value by value 31).  TWO: both exponentials, else the one at T alone, its factor standing for both.
template <typename T, bool REST, bool TWO, bool SHIFT, int N>
__global__ void __launch_bounds__(N == 32 ? 32 * kRowsOfCta : N) distill_slopes(DistillArgs a) {
    constexpr int W = 16 / sizeof(T), U = 2, P = kPairs<W>;
    __shared__ float scratch[N == 32 ? 1 : 2 * (N / 32) * 8];
    __shared__ int kept_of[N == 32 ? kRowsOfCta : 1][N == 32 ? 32 : kMostKept];
    __shared__ float p_of[N == 32 ? kRowsOfCta : 1][N == 32 ? 32 : kMostKept];
    const int slot = N == 32 ? threadIdx.x / 32 : 0;
    const int part = N == 32 ? 0 : blockIdx.x % a.parts;
    const int row = N == 32 ? blockIdx.x * kRowsOfCta + slot : blockIdx.x / a.parts;
    if (row >= a.rows) return;
    Group<N> g(scratch);
    const T* s = static_cast<const T*>(a.s) + row * a.stride;
    T* ds = static_cast<T*>(a.ds) + (int64_t)row * a.classes;
    const Row<T, W> r(ds, a.classes);                 // (its places; it is not read)
    T* out = ds - r.pad;                              // place 0 of the gradient
    const T* in = s - r.pad;                          // and of the logits
    const int off = SHIFT ? (int)(reinterpret_cast<uintptr_t>(in) % 16) : 0, before = off / (int)sizeof(T);
    const int each = (r.vectors() + a.parts - 1) / a.parts, first = part * each, last = min(r.vectors(), first + each);
    const int from = max(r.pad, first * W), to = min(r.end, last * W);    // this group's places
    int *kept = kept_of[slot];
    float* p_at = p_of[slot];

    const float slope = a.dloss[row * a.dloss_stride];
    int64_t label = a.labels ? a.labels[row] : -1;
    if (label >= a.classes) label = -1;
    int at = -1;
    float u = kNone, x = 0;
    bool owned = false;                               // whether this thread's class is among the group's places
    if (g.lane < a.kept) {
        const int64_t j = (int64_t)row * a.kept + g.lane;
        at = a.indices[j];
        if (at >= 0 && at < a.classes) {
            u = value_at(a.values, a.value_type, j) * a.inv_t;
            owned = at + r.pad >= from && at + r.pad < to;
            if (owned) x = widen(s[at]);
        } else {
            at = -1;
        }
        kept[g.lane] = at;
    }
    const float rest = REST ? a.rest[row] : kNone;
    const bool labelled = label >= 0 && label + r.pad >= from && label + r.pad < to;
    const float x_label = labelled ? widen(s[label]) : 0.0f;
    const float* stats = a.stats + (int64_t)row * 5;
    const float m = stats[0], z1 = stats[1], zt = stats[2], mo = stats[3], zo = stats[4];

    const bool taught = g.any((at >= 0 && u != kNone) || (REST && rest != kNone));
    // a part of weight 0 takes no part, whatever it holds, as in the loss
    const bool soft = taught && a.soft_slope != 0.0f, hard = label >= 0 && a.hard != 0.0f;
    if (slope == 0.0f || (!soft && !hard)) {
        for (int i = from + g.lane; i < to; i += N) narrow(0.0f, out[i]);
        return;
    }
    // the teacher's masses
    float top[1] = {fmaxf(u, rest)};
    g.max(top);
    const float mu = reference(top[0]);
    const float e = at >= 0 ? power(u, mu, a.c1) : 0.0f;
    float whole[1] = {e};
    g.sum(whole);
    const float e0 = REST ? factor(rest, mu, a.c1) : 0.0f;
    const float per = soft ? 1.0f / (whole[0] + e0) : 0.0f;
    if (g.lane < a.kept) p_at[g.lane] = e * per;
    g.sync();
    bool once = owned;
    float p = 0;
    if (owned)
        for (int j = 0; j < a.kept; ++j)
            if (kept[j] == at) {                      // a class that is given twice has both masses, at its first place
                once = once && j >= g.lane;
                p += p_at[j];
            }

    // ds = A 2^((x - m) c1) + B 2^((x - r) ct)
    const float weight = soft ? slope * a.soft_slope : 0.0f;
    const float A = hard ? slope * a.hard / z1 : 0.0f;
    float B = 0.0f;
    if (soft) {
        if (REST)
            B = zo == 0.0f ? 0.0f : weight * (factor(mo, m, a.ct) * (zo / zt) - e0 * per) / zo;
        else
            B = weight / zt;
    }
    const float one = TWO ? B : A + B;                // (without TWO both are relative to the same)
    const float2 c1 = both(a.c1), ct = both(a.ct), r1 = both(-m), rt = both(-(REST ? reference(mo) : m));
    const auto value = [&](float2 v) {
        const float2 d = add(v, rt), k = mul(d, ct);
        float2 y = mul(make_float2(approx_exp2(k.x), approx_exp2(k.y)), both(one));
        if (TWO) {
            const float2 l = mul(REST ? add(v, r1) : d, c1);
            y = fma(make_float2(approx_exp2(l.x), approx_exp2(l.y)), both(A), y);
        }
        return y;
    };
    const auto single = [&](float v) { return value(make_float2(v, v)).x; };
    const auto turn = [&](const Vec<T, W>& v) {
        Vec<T, W> y;
#pragma unroll
        for (int i = 0; i < P; ++i) set_pair(y, i, value(pair(v, i)));
        return y;
    };
    // the ends of a row that are no whole vectors, or whose logits are not in two of them, value by value
    const auto in_vectors = [&](int v) { return SHIFT ? v * W - before >= r.pad && v * W - before + 2 * W <= r.end : r.whole(v); };
    const auto vector_at = [&](int v) {
        if constexpr (SHIFT) {
            const uint4* p = reinterpret_cast<const uint4*>(in + (int64_t)v * W - before);
            const uint4 w = shifted(p[0], p[1], off);
            Vec<T, W> b;
            memcpy(&b, &w, 16);
            return b;
        } else {
            return load<T, W>(in + (int64_t)v * W);
        }
    };
    int begin = min(first, last), end = last;
    while (begin < end && !in_vectors(begin)) ++begin;
    while (end > begin && !in_vectors(end - 1)) --end;
    for (int place = max(r.pad, first * W) + g.lane; place < min(r.end, begin * W); place += N) narrow(single(widen(in[place])), out[place]);
    for (int place = max(r.pad, end * W) + g.lane; place < min(r.end, last * W); place += N) narrow(single(widen(in[place])), out[place]);
    int v = begin + g.lane;
    for (; v + (U - 1) * N < end; v += U * N) {
        Vec<T, W> b[U];
#pragma unroll
        for (int k = 0; k < U; ++k) b[k] = vector_at(v + k * N);
#pragma unroll
        for (int k = 0; k < U; ++k) store<T, W>(out + (int64_t)(v + k * N) * W, turn(b[k]));
    }
    for (; v < end; v += N) store<T, W>(out + (int64_t)v * W, turn(vector_at(v)));

    // the classes with a term of their own
    const bool among = g.any(once && at == label);
    g.sync();
    if (once) {
        float y;
        if (REST) {
            y = soft ? weight * (power(x, m, a.ct) / zt - p) : 0.0f;
            if (hard) y += A * power(x, m, a.c1);
        } else {
            y = single(x) - (soft ? weight * p : 0.0f);
        }
        if (at == label) y -= slope * a.hard;
        narrow(y, ds[at]);
    }
    if (labelled && !among && g.lane == 0) narrow(single(x_label) - slope * a.hard, ds[label]);
}

template <typename T, bool REST, bool TWO, bool SHIFT>
cudaError_t launch(DistillArgs a, cudaStream_t st) {
    a.parts = 1;
    // a warp where there are rows enough, or hardly any classes (8192 x 1000 fp32: 10.6 us, by a CTA 29; 8192 x 4000 52 and 54, of bf16 28
    // and 51; 1216 x 4000 fp32 8.5 and 7.8; 512 x 1000 4.6 and 4.7)
    if (a.classes <= kMostOfWarp / (int)sizeof(T) && a.kept <= 32 && (a.rows >= 8 * kSMs || a.classes <= 256)) {
        distill_slopes<T, REST, TWO, SHIFT, 32><<<(a.rows + kRowsOfCta - 1) / kRowsOfCta, 32 * kRowsOfCta, 0, st>>>(a);
    } else {
        // few long rows: several CTAs have one, each its stretch, with nothing to join (6 x 200001 fp32: 32 us by one, 4.9 by 32;
        // 400 x 65536 bf16 16.4 by one, 14.9 by two, 16.2 by four); of very long ones more, as the last CTAs end alone (300 x 1048576
        // bf16: 218 us by four, 196 by eight; 1000 x 21841 14.1 by one, 16.6 by two)
        while (a.parts < 64 && (((int64_t)a.rows * a.parts < 4 * kSMs && a.classes / a.parts >= 4096) ||
                                ((int64_t)a.rows * a.parts < 16 * kSMs && a.classes / a.parts >= 65536)))
            a.parts *= 2;
        distill_slopes<T, REST, TWO, SHIFT, kWide><<<(unsigned)a.rows * (unsigned)a.parts, kWide, 0, st>>>(a);
    }
    return cudaGetLastError();
}

template <typename T, bool SHIFT>
cudaError_t backward(const DistillArgs& a, cudaStream_t st) {
    if (a.rest) return a.labels ? launch<T, true, true, SHIFT>(a, st) : launch<T, true, false, SHIFT>(a, st);
    const bool two = a.labels && a.ct != a.c1;
    return two ? launch<T, false, true, SHIFT>(a, st) : launch<T, false, false, SHIFT>(a, st);
}
template <typename T>
cudaError_t backward(const DistillArgs& a, cudaStream_t st) {
    // rows of both lie alike where the first ones and, with more rows, the strides do
    const uintptr_t apart = reinterpret_cast<uintptr_t>(a.s) - reinterpret_cast<uintptr_t>(a.ds);
    const bool alike = apart % 16 == 0 && (a.rows == 1 || (a.stride - a.classes) * (int64_t)sizeof(T) % 16 == 0);
    return alike ? backward<T, false>(a, st) : backward<T, true>(a, st);
}

}  // namespace

cudaError_t distill_backward(const DistillArgs& a, int dtype, cudaStream_t st) {
    return dtype == PP_F32 ? backward<float>(a, st) : dtype == PP_F16 ? backward<__half>(a, st) : backward<__nv_bfloat16>(a, st);
}

}  // namespace patconv
