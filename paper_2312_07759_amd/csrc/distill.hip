// Kullback-Leibler loss of a student's logits z [n, V] against the teacher's largest logits (index, value; -1: no entry):
//   p = softmax(teacher / tau) over the row's entries,  q = softmax(z / tau) over all V,
//   loss = sum p (log p - log q),  lse = log sum exp(z / tau),  dz = weight / tau (q - p)   (zeros where a row has no entry)
// Entries of one index stay apart in the loss and add up in the gradient, which does not know how p is divided among them.
// Bound by memory: the row is read once and its gradient written once.  A row stays in the registers of its workgroup between
// the two (TH threads, NV pieces of 16 bytes each: rows up to 128 KB); with few rows several workgroups share one, a first launch
// leaving each part's maximum and sum (5 rows of 50001 float32 logits: 3.9 and 7.2 us).  Sums are float32: a lane adds up pieces' sums, and one piece in
// V / (logits of a piece) / TH of them is its own (32 for 128000 logits of 16 bits, 512 threads; 2^18 for the longest float32 rows), each addition off by at most
// 2^-24 of the lane's sum.  Exponents are taken of differences to the maximum, so that rows of the type's lowest value come out even and -inf as nothing.
#include <type_traits>

#include "layers.h"

namespace idkm {

namespace {

template <typename T>
__device__ __forceinline__ float element(u32x4 v, int e) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(floatx4, v)[e];
    } else if constexpr (__is_same(T, bf16)) {
        return __builtin_bit_cast(float, (e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
    } else {
        return (float)__builtin_bit_cast(f16x8, v)[e];
    }
}

typedef u32x4 u32x4_el __attribute__((aligned(2)));

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
constexpr float LOWEST = -3.4028234663852886e38f;

struct Two { float a, b; };

// Largest of three; of a NaN and a number the number.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

// exp((z - m) / tau) of a row: its exponent to the base 2 is one multiply-add of the logit, z c - k with k = m c rounded.  The
// rounding, up to |k| 2^-24, is an exponent that all of the row's exponentials and their sum get: a common factor of at most sqrt(2) while
// |k| <= 2^23, but infinities or nothing from 2^31 on (a row of -1e10, or small temperatures).  Beyond 2^23 the difference z - m
// comes first, which costs one instruction more for a logit.
struct Exponent {
    float c, m, k;
    bool difference;
    __device__ __forceinline__ Exponent(float tau, float m_) : c(LOG2E / tau), m(m_), difference(!(fabsf(m_) * c <= 8388608.f)) { k = difference ? 0.f : m * c; }
    template <bool DIFFERENCE>
    __device__ __forceinline__ float of(float z) const {
        return __builtin_amdgcn_exp2f(fmaf(DIFFERENCE ? z - m : z, c, -k));
    }
    __device__ __forceinline__ float of(float z) const { return difference ? of<true>(z) : of<false>(z); }
    // log of the same
    __device__ __forceinline__ float log(float z) const { return fmaf(difference ? z - m : z, c, -k) * LN2; }
    // log sum exp(z / tau) for sum exp = e^ln
    __device__ __forceinline__ float lse(float tau, float ln) const { return (difference ? m / tau : k * LN2) + ln; }
};

// max, or sum, of two values over a workgroup of TH threads; `scratch`: 2 x 16 floats
template <int TH, bool MAX>
__device__ __forceinline__ Two all_of(Two v, float* scratch) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float x = __shfl_xor(v.a, o), y = __shfl_xor(v.b, o);
        v.a = MAX ? fmaxf(v.a, x) : v.a + x;
        v.b = MAX ? fmaxf(v.b, y) : v.b + y;
    }
    if constexpr (TH > 64) {
        __syncthreads();  // the scratch of the last use has been read
        if ((threadIdx.x & 63) == 0) {
            scratch[threadIdx.x >> 6] = v.a;
            scratch[16 + (threadIdx.x >> 6)] = v.b;
        }
        __syncthreads();
        v.a = scratch[0];
        v.b = scratch[16];
#pragma unroll
        for (int w = 1; w < TH / 64; ++w) {
            v.a = MAX ? fmaxf(v.a, scratch[w]) : v.a + scratch[w];
            v.b = MAX ? fmaxf(v.b, scratch[16 + w]) : v.b + scratch[16 + w];
        }
    }
    return v;
}

// The teacher's list of one row in LDS: index, p, the student's logit there.
struct List {
    int* index;
    float* p;
    float* z;
};

struct RowTail {
    float loss, factor;  // factor: weight / tau, NaN for a list that is no list (see read_list)
    bool none;           // no entry: loss 0, gradient 0 whatever the logits hold
};

// Largest teacher value of the row, the list copied to LDS.  bad: an index that is no place of the row, or a NaN.
template <int TH>
__device__ __forceinline__ float read_list(const DistillArgs& a, int64_t row, List l, bool& bad) {
    float top = -INFINITY;
    for (int i = threadIdx.x; i < a.top; i += TH) {
        const int at = a.index[row * a.top + i];
        const float t = a.teacher[row * a.top + i];
        l.index[i] = at;
        l.p[i] = t;
        if (at >= a.V || (at >= 0 && t != t)) bad = true;
        if (at >= 0) top = fmaxf(top, t);
    }
    return top;
}

// From the logarithm of the row's sum of exponentials and the teacher's maximum and sum: p in LDS, the row's loss and the factor.
// listed: the student's logits at the list's places; null: they are taken from the row.
template <typename T, int TH>
__device__ __forceinline__ RowTail finish_row(const DistillArgs& a, int64_t row, List l, const Exponent& x, float ln_sum, Two teacher, bool bad,
                                              const float* listed, bool want_loss, float* scratch) {
    const float t_top = teacher.a, t_sum = teacher.b;
    const bool some = t_top > -INFINITY;  // entries, and not all of them -inf
    const float inv_tau = 1.f / a.tau, ln_t = logf(t_sum);
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz;
    float loss = 0.f;
    for (int i = threadIdx.x; i < a.top; i += TH) {
        const int at = l.index[i];
        float p = 0.f, zi = 0.f;
        if (at >= 0 && at < a.V && some) {
            const float logp = (l.p[i] - t_top) * inv_tau - ln_t;
            p = expf(logp);
            zi = listed ? listed[i] : Elem<T>::up(z[at]);
            if (p != 0.f) loss += p * (logp - (x.log(zi) - ln_sum));
        }
        l.p[i] = p;
        l.z[i] = zi;
    }
    RowTail t{0.f, a.weight ? a.weight[row] * inv_tau : 0.f, !some && !bad};
    if (want_loss) t.loss = all_of<TH, false>(Two{loss, 0.f}, scratch).a;
    if (bad) t.loss = t.factor = __builtin_nanf("");
    return t;
}

// Places of the list inside [from, to): q - p there, once for an index that is listed more than once.  over: factor / sum.
template <typename T, int TH>
__device__ __forceinline__ void correct(const DistillArgs& a, int64_t row, List l, const Exponent& x, float factor, float over, int64_t from, int64_t to) {
    T* out = static_cast<T*>(a.dlogits) + row * a.ldd;
    for (int i = threadIdx.x; i < a.top; i += TH) {
        const int at = l.index[i];
        if (at < from || at >= to) continue;
        float p = l.p[i];
        bool again = false;
        for (int j = 0; j < a.top; ++j) {
            if (l.index[j] != at) continue;
            if (j < i) again = true;
            if (j > i) p += l.p[j];
        }
        if (!again) out[at] = Elem<T>::down(over * x.of(l.z[i]) - factor * p);
    }
}

}  // namespace

// One workgroup to a row (TH > 64) or one wavefront, the row in registers.  Longer rows (up to any length) keep their first NV TH pieces
// there; the rest is read a second time for the gradient, from the last-level cache.  So two workgroups fit a compute unit, and one's
// memory traffic covers the other's exponentials: 2048 rows of 128000 bfloat16 logits, all of a row in the registers of the one workgroup
// that then fits, took 278 us; it is 250 now, where the logits read once and the gradient written once take 201 at the rate of a copy.
template <typename T, int TH, int NV, bool LONG>
__global__ __launch_bounds__(TH, TH == 512 ? 4 : 1) void k_distill_row(const DistillArgs a) {
    constexpr int PER = Elem<T>::PER16;
    extern __shared__ float lds[];
    List l{reinterpret_cast<int*>(lds), lds + a.top, lds + 2 * a.top};
    float* scratch = lds + 3 * a.top;
    const int pieces = (int)(a.V / PER), rest = (int)(a.V - (int64_t)pieces * PER);
    const bool tail = (int)threadIdx.x < rest;
    // 32-bit offsets from the row's uniform address; pieces behind the last are read as it and do not count
    auto load = [&](const T* z, int h) {
        const unsigned at = (unsigned)min(h * TH + (int)threadIdx.x, pieces - 1) * 16u;
        return *reinterpret_cast<const u32x4_el*>(reinterpret_cast<const unsigned char*>(z) + at);
    };
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz;
    u32x4 held[NV];
    // between two uses of the row: or the compiler keeps its elements as floats, in registers that are not there
    auto keep_packed = [&] {
#pragma unroll
        for (int h = 0; h < NV; ++h) asm volatile("" : "+v"(held[h]));
    };
#pragma unroll
    for (int h = 0; h < NV; ++h) held[h] = h * TH < pieces ? load(z, h) : u32x4{0, 0, 0, 0};
    float zt = tail ? Elem<T>::up(z[(int64_t)pieces * PER + threadIdx.x]) : LOWEST;
    bool bad = false;
    const float t_own = read_list<TH>(a, row, l, bad);
    float m = fmaxf(LOWEST, zt);
#pragma unroll
    for (int h = 0; h < NV; ++h)
        if (h * TH < pieces) {
#pragma unroll
            for (int e = 0; e < PER; e += 2) m = max3(m, element<T>(held[h], e), element<T>(held[h], e + 1));
        }
    // the rest: a running maximum and sum
    float m_rest = LOWEST, s_rest = 0.f;
    if constexpr (LONG) {
        const float c = LOG2E / a.tau;
        for (int i = NV * TH + (int)threadIdx.x; i < pieces; i += 4 * TH) {
            u32x4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                v[u] = *reinterpret_cast<const u32x4_el*>(reinterpret_cast<const unsigned char*>(z) + (unsigned)min(i + u * TH, pieces - 1) * 16u);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float top = m_rest, part = 0.f;
#pragma unroll
                for (int e = 0; e < PER; e += 2) top = max3(top, element<T>(v[u], e), element<T>(v[u], e + 1));
#pragma unroll
                for (int e = 0; e < PER; ++e) part += __builtin_amdgcn_exp2f((element<T>(v[u], e) - top) * c);
                if (i + u * TH < pieces) {
                    s_rest = fmaf(s_rest, __builtin_amdgcn_exp2f((m_rest - top) * c), part);
                    m_rest = top;
                }
            }
        }
        m = fmaxf(m, m_rest);
    }
    const Two tops = all_of<TH, true>(Two{m, t_own}, scratch);
    const Exponent x(a.tau, tops.a);
    keep_packed();
    float s = tail ? x.of(zt) : 0.f, ts = 0.f;
    if constexpr (LONG) s += s_rest != 0.f ? s_rest * x.of(m_rest) : 0.f;
    auto add = [&](auto difference) {
#pragma unroll
        for (int h = 0; h < NV; ++h)
            if (h * TH < pieces) {
                float part = 0.f;
#pragma unroll
                for (int e = 0; e < PER; ++e) part += x.template of<decltype(difference)::value>(element<T>(held[h], e));
                s += h * TH + (int)threadIdx.x < pieces ? part : 0.f;
            }
    };
    if (x.difference) add(std::true_type());
    else add(std::false_type());
    for (int i = threadIdx.x; i < a.top; i += TH)
        if (l.index[i] >= 0 && tops.b > -INFINITY) ts += expf((l.p[i] - tops.b) / a.tau);
    const Two sums = all_of<TH, false>(Two{s, ts}, scratch);
    const Two any_bad = all_of<TH, true>(Two{bad ? 1.f : 0.f, 0.f}, scratch);
    const float ln_sum = logf(sums.a);
    const RowTail t = finish_row<T, TH>(a, row, l, x, ln_sum, Two{tops.b, sums.b}, any_bad.a > 0.f, nullptr, true, scratch);
    if (threadIdx.x == 0) {
        a.loss[row] = t.loss;
        a.lse[row] = x.lse(a.tau, ln_sum);
    }
    keep_packed();
    if (!a.dlogits) return;
    T* out = static_cast<T*>(a.dlogits) + row * a.ldd;
    const float over = t.factor / sums.a;
    auto write = [&](auto difference) {
#pragma unroll
        for (int h = 0; h < NV; ++h)
            if (h * TH < pieces) {
                struct alignas(16) Piece { T v[PER]; } o;
#pragma unroll
                for (int e = 0; e < PER; ++e)
                    o.v[e] = Elem<T>::down(over * x.template of<decltype(difference)::value>(element<T>(held[h], e)));
                u32x4 v;
                __builtin_memcpy(&v, &o, 16);
                if (t.none) v = u32x4{0, 0, 0, 0};
                const int at = h * TH + (int)threadIdx.x;
                if (at < pieces) *reinterpret_cast<u32x4_el*>(reinterpret_cast<unsigned char*>(out) + (unsigned)at * 16u) = v;
            }
        if constexpr (LONG) {
            for (int i = NV * TH + (int)threadIdx.x; i < pieces; i += 4 * TH) {
                u32x4 r[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    r[u] = *reinterpret_cast<const u32x4_el*>(reinterpret_cast<const unsigned char*>(z) + (unsigned)min(i + u * TH, pieces - 1) * 16u);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    struct alignas(16) Piece { T v[PER]; } o;
#pragma unroll
                    for (int e = 0; e < PER; ++e) o.v[e] = Elem<T>::down(over * x.template of<decltype(difference)::value>(element<T>(r[u], e)));
                    u32x4 v;
                    __builtin_memcpy(&v, &o, 16);
                    if (t.none) v = u32x4{0, 0, 0, 0};
                    if (i + u * TH < pieces) *reinterpret_cast<u32x4_el*>(reinterpret_cast<unsigned char*>(out) + (unsigned)(i + u * TH) * 16u) = v;
                }
            }
        }
    };
    if (x.difference) write(std::true_type());
    else write(std::false_type());
    if (tail) out[(int64_t)pieces * PER + threadIdx.x] = t.none ? (T)0.f : Elem<T>::down(over * x.of(zt));
    __syncthreads();
    if (!t.none) correct<T, TH>(a, row, l, x, t.factor, over, 0, a.V);
}

// Part blockIdx.y of a row: [from, to).
__device__ __forceinline__ void part_of(const DistillArgs& a, int64_t& from, int64_t& to) {
    from = min(a.V, (int64_t)blockIdx.y * a.part);
    to = min(a.V, from + a.part);
}

template <typename T>
__global__ __launch_bounds__(256) void k_distill_stats(const DistillArgs a) {
    constexpr int PER = Elem<T>::PER16;
    __shared__ float scratch[32];
    const int64_t row = blockIdx.x;
    int64_t from, to;
    part_of(a, from, to);
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz + from;
    const int64_t pieces = (to - from) / PER;
    const int rest = (int)(to - from - pieces * PER);
    float m = LOWEST, s = 0.f;
    const float c = LOG2E / a.tau;
    for (int64_t i = threadIdx.x; i < pieces; i += 256) {
        const u32x4 v = reinterpret_cast<const u32x4_el*>(z)[i];
        float top = m;
#pragma unroll
        for (int e = 0; e < PER; ++e) top = fmaxf(top, element<T>(v, e));
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < PER; ++e) part += __builtin_amdgcn_exp2f((element<T>(v, e) - top) * c);
        s = s * __builtin_amdgcn_exp2f((m - top) * c) + part;
        m = top;
    }
    if ((int)threadIdx.x < rest) {
        const float x = Elem<T>::up(z[pieces * PER + threadIdx.x]), top = fmaxf(m, x);
        s = s * __builtin_amdgcn_exp2f((m - top) * c) + __builtin_amdgcn_exp2f((x - top) * c);
        m = top;
    }
    const float top = all_of<256, true>(Two{m, 0.f}, scratch).a;
    s = all_of<256, false>(Two{s * __builtin_amdgcn_exp2f((m - top) * c), 0.f}, scratch).a;
    // the logits at the list's places of this part, before the second launch may write their gradient over them
    for (int i = threadIdx.x; i < a.top; i += 256) {
        const int at = a.index[row * a.top + i];
        if (at >= from && at < to) a.listed[row * a.top + i] = Elem<T>::up(z[at - from]);
    }
    if (threadIdx.x == 0) {
        a.stats[(row * gridDim.y + blockIdx.y) * 2] = top;
        a.stats[(row * gridDim.y + blockIdx.y) * 2 + 1] = s;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_distill_parts(const DistillArgs a) {
    constexpr int PER = Elem<T>::PER16;
    extern __shared__ float lds[];
    List l{reinterpret_cast<int*>(lds), lds + a.top, lds + 2 * a.top};
    float* scratch = lds + 3 * a.top;
    const int64_t row = blockIdx.x;
    bool bad = false;
    const float t_own = read_list<256>(a, row, l, bad);
    const float* st = a.stats + row * a.parts * 2;
    float m = LOWEST;
    for (int i = threadIdx.x; i < a.parts; i += 256) m = fmaxf(m, st[2 * i]);
    const Two tops = all_of<256, true>(Two{m, t_own}, scratch);
    m = tops.a;
    const Exponent x(a.tau, m);
    float s = 0.f, ts = 0.f;
    for (int i = threadIdx.x; i < a.parts; i += 256) s += st[2 * i + 1] * x.of(st[2 * i]);
    for (int i = threadIdx.x; i < a.top; i += 256)
        if (l.index[i] >= 0 && tops.b > -INFINITY) ts += expf((l.p[i] - tops.b) / a.tau);
    const Two sums = all_of<256, false>(Two{s, ts}, scratch);
    const Two any_bad = all_of<256, true>(Two{bad ? 1.f : 0.f, 0.f}, scratch);
    const float ln_sum = logf(sums.a);
    const RowTail t = finish_row<T, 256>(a, row, l, x, ln_sum, Two{tops.b, sums.b}, any_bad.a > 0.f, a.listed + row * a.top,
                                         blockIdx.y == 0, scratch);
    if (threadIdx.x == 0 && blockIdx.y == 0) {
        a.loss[row] = t.loss;
        a.lse[row] = x.lse(a.tau, ln_sum);
    }
    if (!a.dlogits) return;
    __syncthreads();
    int64_t from, to;
    part_of(a, from, to);
    const T* z = static_cast<const T*>(a.logits) + row * a.ldz + from;
    T* out = static_cast<T*>(a.dlogits) + row * a.ldd + from;
    const int64_t pieces = (to - from) / PER;
    const int rest = (int)(to - from - pieces * PER);
    const float over = t.factor / sums.a;
    for (int64_t i = threadIdx.x; i < pieces; i += 256) {
        const u32x4 v = reinterpret_cast<const u32x4_el*>(z)[i];
        struct alignas(16) Piece { T v[PER]; } o;
#pragma unroll
        for (int e = 0; e < PER; ++e) o.v[e] = t.none ? (T)0.f : Elem<T>::down(over * x.of(element<T>(v, e)));
        u32x4 w;
        __builtin_memcpy(&w, &o, 16);
        reinterpret_cast<u32x4_el*>(out)[i] = w;
    }
    if ((int)threadIdx.x < rest) {
        out[pieces * PER + threadIdx.x] = t.none ? (T)0.f : Elem<T>::down(over * x.of(Elem<T>::up(z[pieces * PER + threadIdx.x])));
    }
    __syncthreads();
    if (!t.none) correct<T, 256>(a, row, l, x, t.factor, over, from, to);
}

template <typename T>
static void launch_for(const DistillArgs& a, hipStream_t s) {
    const size_t lds = (3 * (size_t)a.top + 32) * sizeof(float);
    if (a.parts > 0) {
        const dim3 grid((unsigned)a.n, (unsigned)a.parts);
        hipLaunchKernelGGL(k_distill_stats<T>, grid, dim3(256), 0, s, a);
        const dim3 second((unsigned)a.n, a.dlogits ? (unsigned)a.parts : 1u);
        hipLaunchKernelGGL(k_distill_parts<T>, second, dim3(256), lds, s, a);
        return;
    }
    const int64_t pieces = a.V / Elem<T>::PER16;
    // a launch has less than 2^32 threads
    constexpr int64_t ROWS = (int64_t)1 << 22;
    for (int64_t r = 0; r < a.n; r += ROWS) {
        DistillArgs b = a;
        b.n = a.n - r < ROWS ? a.n - r : ROWS;
        b.logits = static_cast<const T*>(a.logits) + r * a.ldz;
        b.index = a.index + r * a.top;
        b.teacher = a.teacher + r * a.top;
        if (a.weight) b.weight = a.weight + r;
        b.loss = a.loss + r;
        b.lse = a.lse + r;
        if (a.dlogits) b.dlogits = static_cast<T*>(a.dlogits) + r * a.ldd;
        const dim3 grid((unsigned)b.n);
        if (pieces <= 4 * 64) hipLaunchKernelGGL((k_distill_row<T, 64, 4, false>), grid, dim3(64), lds, s, b);
        else if (pieces <= 4 * 256) hipLaunchKernelGGL((k_distill_row<T, 256, 4, false>), grid, dim3(256), lds, s, b);
        else if (pieces <= 16 * 256) hipLaunchKernelGGL((k_distill_row<T, 256, 16, false>), grid, dim3(256), lds, s, b);
        else if (pieces <= 16 * 512) hipLaunchKernelGGL((k_distill_row<T, 512, 16, false>), grid, dim3(512), lds, s, b);
        else hipLaunchKernelGGL((k_distill_row<T, 512, 16, true>), grid, dim3(512), lds, s, b);
    }
}

void distill_plan(int64_t n, int64_t V, int esize, int64_t* part, int* parts) {
    const int64_t per = 16 / esize, row_bytes = V * esize;
    *part = 0;
    *parts = 0;
    const int64_t want = (1024 + n - 1) / n;  // four workgroups to a compute unit
    // One launch and one workgroup a row against two launches and several: rows of 32000 take 9.6 to 11.5 us against 9.8 to 13.4 (1 to 100
    // rows, float32 and bfloat16), of 50001 11.4 to 15 against 10 to 16, of 128000 20 to 24 against 11 to 21 (bfloat16); with 250 rows one
    // workgroup a row is always ahead (128000 bfloat16: 34 against 38).
    if (n >= 128 || V <= 32768) return;
    int64_t p = want;
    const int64_t most = (row_bytes + 16 * 1024 - 1) / (16 * 1024);
    if (p > most) p = most;
    *part = ((V + p - 1) / p + per - 1) / per * per;
    *parts = (int)((V + *part - 1) / *part);
}

void launch_distill(int dtype, const DistillArgs& a, hipStream_t s) {
    if (dtype == 0) launch_for<float>(a, s);
    else if (dtype == 1) launch_for<f16>(a, s);
    else launch_for<bf16>(a, s);
}

}  // namespace idkm
